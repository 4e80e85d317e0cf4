"""The buffers that ``experts.ExpertMLP`` keeps: bounded in number and size whatever token counts
come, apart for calls on different streams, and with addresses that a captured graph may hold."""
import pytest
import torch

from paper_2608_26574_gb300.experts import ExpertMLP

pytestmark = pytest.mark.gpu


def _layers(shared, n=6, k=2, d=64, f=96, count=2):
    g = torch.Generator().manual_seed(7)
    out = []
    for _ in range(count):
        w = [(torch.randn(*s, generator=g) / s[-1] ** 0.5).cuda().to(torch.bfloat16)
             for s in ((n, f, d), (n, f, d), (n, d, f))]
        router = (torch.randn(d, n, generator=g) / d ** 0.5).cuda().to(torch.bfloat16)
        out.append(ExpertMLP(*w, router, k, workspaces=shared))
    return out


def _rows(tokens, seed, d=64):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(tokens, d, generator=g, device="cuda").to(torch.bfloat16)


def test_many_token_counts_keep_little_memory():
    """Every count from 1 to 400 through two layers that share their buffers: together at most
    twice what the largest count alone makes them keep (sets for powers of two), and a megabyte
    for what the allocator rounds up."""
    _layers({})[0](_rows(1, 0))  # (libraries' own workspaces)
    torch.cuda.synchronize()

    def kept(counts):
        layers = _layers({})
        before = torch.cuda.memory_allocated()
        for t in counts:
            h = _rows(t, t)
            for m in layers:
                m(h)
        del h
        torch.cuda.synchronize()
        return torch.cuda.memory_allocated() - before

    largest = kept([400])
    assert kept(range(1, 401)) <= 2 * largest + (1 << 20)


def test_counts_up_and_down_through_one_set():
    """The counts between two powers of two share a set, whose workspaces serve each: the same bits
    as from a layer that sees no other count."""
    shared: dict = {}
    m = _layers(shared, count=1)[0]
    for t in (64, 33, 50, 63, 34, 64):
        assert torch.equal(m(_rows(t, t)), _layers({}, count=1)[0](_rows(t, t)))
    assert len(shared) == 1
    assert m(_rows(0, 0)).shape == (0, 64)


def test_two_streams_do_not_share_buffers():
    """One layer called on two streams in turn, without a wait between them, each with a count of
    its own and then with the same: every output as from that call alone."""
    m = _layers({}, n=8, k=4, d=512, f=768, count=1)[0]
    for counts in ((900, 1000), (700, 700)):
        hs = [[_rows(t, 10 * i + s, 512) for i in range(12)] for s, t in enumerate(counts)]
        want = [[m(h).clone() for h in row] for row in hs]
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        got: list = [[], []]
        for i in range(12):
            for s, stream in enumerate(streams):
                with torch.cuda.stream(stream):
                    got[s].append(m(hs[s][i]))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_graphs_of_several_counts_stay_valid():
    """Graphs captured for rising counts, replayed after calls with many other counts."""
    m = _layers({}, count=1)[0]
    graphs = {}
    for t in (3, 40, 200):
        h, out = _rows(t, t), torch.empty(t, 64, dtype=torch.bfloat16, device="cuda")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            m(h, out=out)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            m(h, out=out)
        graphs[t] = graph, h, out
    for t in range(1, 300):
        m(_rows(t, 7))
    for t, (graph, h, out) in graphs.items():
        for seed in (11, 12):
            h.copy_(_rows(t, seed))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, m(h))
