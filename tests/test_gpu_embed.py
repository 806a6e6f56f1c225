"""Embedding lookup and its gradient against 64 bits: types of activations and
tokens, odd widths and offsets, token counts on both sides of a chunk, a wave,
a sorted run and of one and two merges of runs, tokens that all are the same, padded or out of range, and the parts of a
row that are not the table's."""
import pytest

import layer_refs as ref

pytestmark = pytest.mark.gpu

# M, tokens, vocabulary, width, offset
SHAPES = [(1, 1, 1, 1, 0), (3, 1, 5, 7, 1), (2, 31, 2, 8, 4), (1, 32, 3, 9, 2), (2, 33, 40, 512, 0), (1, 64, 511, 513, 3),
          (3, 65, 512, 64, 7), (1, 300, 513, 1, 0), (2, 1000, 37, 100, 5), (3, 511, 700, 40, 1), (1, 512, 5, 1300, 0),
          (2, 513, 30, 16, 6), (1, 200, 9000, 3, 0), (1, 40, 20, 40000, 1), (2, 63, 4000, 50, 3), (3, 64, 9, 1301, 0), (1, 1025, 70000, 17, 0), (2, 2500, 300, 1030, 9),
          (1, 5000, 4, 520, 0), (5, 0, 10, 12, 2), (1, 4096, 300, 3, 0), (2, 4097, 60, 9, 3), (1, 9000, 300001, 1, 2),
          (1, 66000, 5, 3, 0), (2, 140001, 3000, 2, 1)]


def _tokens(kind, M, N, V, dtype, gen):
    import torch
    t = torch.randint(0, V, (M, N), generator=gen)
    if kind == "zipf":
        t = (torch.rand((M, N), generator=gen) ** 4 * V).long().clamp(max=V - 1)
        t[torch.rand((M, N), generator=gen) < 0.1] = -1
        t[torch.rand((M, N), generator=gen) < 0.05] = V
    elif kind == "same":
        t[:] = V - 1
    elif kind == "padded":
        t[:] = torch.tensor([-1, V, torch.iinfo(dtype).min, torch.iinfo(dtype).max])[
            torch.randint(0, 4, (M, N), generator=gen)]
    return t.to(dtype).cuda()


def _setup(shape, kind, index, seed=0):
    import torch
    M, N, V, D, off = shape
    gen = torch.Generator().manual_seed(seed)
    pl = ref.plan(off + V * D + 3, M)
    P = torch.randn((M, pl.ld), generator=gen).cuda()
    return pl, P, _tokens(kind, M, N, V, getattr(torch, index), gen), gen


@pytest.mark.parametrize("dt", sorted(ref.TYPES))
@pytest.mark.parametrize("index", ["int32", "int64"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(shape, index, dt):
    import torch
    from paper_2010_13359_amd import layers
    M, N, V, D, off = shape
    pl, P, t, _ = _setup(shape, "zipf", index)
    out = torch.full((M, N, D), float("nan"), dtype=ref.TYPES[dt], device="cuda")
    layers.embed_forward(pl, t, P, out, V, offset=off, scale=1.7)
    for m in range(M):
        want, err = ref.embed_forward(t[m], P[m, off:off + V * D].view(V, D), 1.7)
        ref.check("out", out[m], want, err)
    # one vector for all workers
    layers.embed_forward(pl, t, P[0].clone(), out, V, offset=off, scale=-0.5)
    for m in range(M):
        want, err = ref.embed_forward(t[m], P[0, off:off + V * D].view(V, D), -0.5)
        ref.check("out of one vector", out[m], want, err)
    pl.close()


@pytest.mark.parametrize("kind", ["zipf", "same", "padded", "uniform"])
@pytest.mark.parametrize("dt", sorted(ref.TYPES))
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(shape, dt, kind):
    import torch
    from paper_2010_13359_amd import layers
    M, N, V, D, off = shape
    pl, _, t, gen = _setup(shape, kind, "int64" if N % 2 else "int32", seed=N)
    dout = torch.randn((M, N, D), generator=gen).to(ref.TYPES[dt]).cuda()
    G = torch.randn((M, pl.ld), generator=gen).cuda()
    before = G.clone()
    ws = layers.embed_workspace(pl, N, V, D, dout.dtype, t.dtype, offset=off)
    if ws is not None:
        ws.fill_(0xFF)     # nothing in it is read before it is written
    layers.embed_backward(pl, t, dout, G, V, ws, offset=off, scale=0.3)
    first = G.clone()
    layers.embed_backward(pl, t, dout, G, V, ws, offset=off, scale=2.0, add=True)
    for m in range(M):
        want, err = ref.embed_backward(t[m], dout[m], V, 0.3)
        ref.check("G", first[m, off:off + V * D].view(V, D), want, err)
        want, err = ref.embed_backward(t[m], dout[m], V, 2.0, first[m, off:off + V * D].view(V, D))
        ref.check("G added to", G[m, off:off + V * D].view(V, D), want, err)
    for x in (first, G):
        assert torch.equal(x[:, :off], before[:, :off]) and torch.equal(x[:, off + V * D:], before[:, off + V * D:])
    # equal calls, equal bits
    again = before.clone()
    layers.embed_backward(pl, t, dout, again, V, ws, offset=off, scale=0.3)
    assert torch.equal(again.view(torch.int32), first.view(torch.int32))
    pl.close()


def test_gradient_is_the_lookups():
    """The lookup is linear in the table: <dout, out(P + h E) - out(P)> is h times
    <gradient, E> for every E, up to the roundings of three sums."""
    import torch
    from paper_2010_13359_amd import layers
    shape = (2, 77, 19, 24, 5)
    M, N, V, D, off = shape
    pl, P, t, gen = _setup(shape, "zipf", "int64", seed=3)
    E, dout = torch.randn(P.shape, generator=gen).cuda(), torch.randn((M, N, D), generator=gen).cuda()
    G = torch.zeros_like(P)
    layers.embed_backward(pl, t, dout, G, V, layers.embed_workspace(pl, N, V, D, dout.dtype, offset=off), offset=off,
                          scale=1.5)
    a, b = torch.empty_like(dout), torch.empty_like(dout)
    h = 0.25
    layers.embed_forward(pl, t, P, a, V, offset=off, scale=1.5)
    layers.embed_forward(pl, t, P + h * E, b, V, offset=off, scale=1.5)
    left = ((b.double() - a.double()) * dout.double()).sum() / h
    right = (G.double() * E.double()).sum()
    # each out is off by 1.5 (|P| + h|E|) times two roundings, the gradient by N + 2 roundings of its terms
    size = float(((a.abs() + b.abs()) * dout.abs()).double().sum()) / h + float((G.abs() * E.abs()).double().sum()) * N
    assert abs(float(left - right)) <= 4 * ref.U * size
    pl.close()


def test_nonfinite_gradients_stay_in_their_rows():
    import torch
    from paper_2010_13359_amd import layers
    M, N, V, D = 1, 100, 9, 20
    pl = ref.plan(V * D, M)
    t = (torch.arange(N) % V)[None].cuda()
    t[0, 50] = -1
    dout = torch.ones((M, N, D), dtype=torch.bfloat16, device="cuda")
    dout[0, 50] = float("nan")      # of a padded place: nowhere
    dout[0, 3, 4] = float("inf")
    dout[0, 7, 5] = float("nan")
    G = torch.zeros((M, pl.ld), device="cuda")
    layers.embed_backward(pl, t, dout, G, V, layers.embed_workspace(pl, N, V, D, dout.dtype))
    bad = (~torch.isfinite(G)).nonzero().tolist()
    assert bad == [[0, 3 * D + 4], [0, 7 * D + 5]]
    pl.close()


def test_tables_beyond_32_bits():
    """A table of more than 2^31 elements: its last rows."""
    import torch
    from paper_2010_13359_amd import layers
    V, D, off = 2_100_003, 1031, 3
    print("table of", V * D, "elements", flush=True)
    pl = ref.plan(off + V * D, 1)
    P = torch.zeros((1, pl.ld), device="cuda")
    t = torch.tensor([[V - 1, 0, V - 2, V, V - 1, 2_090_000]], device="cuda")
    rows = torch.randn((t.shape[1], D), device="cuda")
    for i, v in enumerate(t[0].tolist()):
        if v < V:
            P[0, off + v * D:off + (v + 1) * D] = rows[i]
    out = torch.empty((1, t.shape[1], D), device="cuda")
    layers.embed_forward(pl, t, P, out, V, offset=off)
    rows[0], rows[3] = rows[4], 0.0
    assert torch.equal(out[0], rows)
    G = P.fill_(7.0)
    dout = torch.randn_like(out)
    layers.embed_backward(pl, t, dout, G, V, layers.embed_workspace(pl, t.shape[1], V, D, dout.dtype, offset=off),
                          offset=off)
    table = G[0, off:off + V * D].view(V, D)
    assert torch.equal(table[V - 1], dout[0, 0] + dout[0, 4])
    for i in (1, 2, 5):
        assert torch.equal(table[int(t[0, i])], dout[0, i])
    assert int(torch.count_nonzero(table.any(1))) == 4
    assert bool((G[0, :off] == 7.0).all()) and bool((G[0, off + V * D:] == 7.0).all())
    pl.close()


def test_more_rows_than_a_launch_has_workgroups():
    """A table of 600 million rows of one channel: few tokens, at its ends."""
    import torch
    from paper_2010_13359_amd import layers
    V = 600_000_000
    print("rows", V, flush=True)
    plan = ref.plan(V, 1)
    G = torch.full((1, plan.ld), 7.0, device="cuda")
    tok = torch.tensor([[0, V - 1, V - 1, 5, V // 2, -1, V]], device="cuda")
    dout = torch.arange(1.0, 8.0, device="cuda").view(1, 7, 1)
    layers.embed_backward(plan, tok, dout, G, V, None)
    assert G[0, [0, V - 1, 5, V // 2, 1]].tolist() == [1.0, 5.0, 4.0, 5.0, 0.0]
    assert float(G[0, :V].sum(dtype=torch.float64)) == 15.0 and bool((G[0, V:] == 7.0).all())
    plan.close()


@pytest.mark.parametrize("dt", sorted(ref.TYPES))
@pytest.mark.parametrize("D", [1, 20, 64, 100, 128, 130, 600])
def test_tokens_of_very_many_places(D, dt):
    """One token that is all of a worker's places, or all but some at either end,
    over 64 and 4096 chunks.  Whole numbers, whose sums are exact in 32 bits."""
    import torch
    from paper_2010_13359_amd import layers
    V, N = 9, 140_000 if D < 100 else 40_000
    gen = torch.Generator().manual_seed(D)
    tok = torch.full((4, N), 4)
    tok[1, :70] = 2
    tok[2, N - 3:] = torch.tensor([8, 5, -1])
    tok[3] = torch.randint(3, 5, (N,), generator=gen)
    dout = torch.randint(-8, 9, (4, N, D), generator=gen).to(ref.TYPES[dt])
    plan = ref.plan(V * D, 4)
    G = torch.full((4, plan.ld), 3.0, device="cuda")
    ws = layers.embed_workspace(plan, N, V, D, dout.dtype)
    layers.embed_backward(plan, tok.cuda(), dout.cuda(), G, V, ws, scale=0.5)
    for m in range(4):
        keep = tok[m] >= 0
        want = torch.zeros((V, D)).index_add_(0, tok[m][keep], dout[m][keep].float()) * 0.5
        assert torch.equal(G[m, :V * D].view(V, D).cpu(), want), m
    plan.close()


def test_most_tokens():
    """2^30 tokens of one worker, all but some of whose gradients are 0, which add
    nothing to a sum."""
    import torch
    from paper_2010_13359_amd import layers
    N, V = 2 ** 30, 5
    pl = ref.plan(V, 1)
    g = torch.Generator(device="cuda").manual_seed(1)
    P = torch.randn((1, pl.ld), generator=g, device="cuda")
    tok = torch.randint(-1, V, (1, N), generator=g, device="cuda", dtype=torch.int32)
    x = torch.empty((1, N, 1), dtype=torch.float16, device="cuda")
    print("lookup", flush=True)
    layers.embed_forward(pl, tok, P, x, V, scale=2.0)
    part = 2 ** 27
    for a in range(0, N, part):
        t = tok[0, a:a + part].long()
        want = torch.where(t >= 0, 2.0 * P[0, t.clamp(min=0)], 0.0).half()
        assert torch.equal(x[0, a:a + part, 0], want), a
    del t, want
    at = torch.randint(0, N, (5000,), generator=g, device="cuda").unique()
    at = torch.cat([at, torch.tensor([0, N - 1], device="cuda")]).unique()
    x.zero_()
    x[0, at, 0] = torch.randn(at.numel(), generator=g, device="cuda").half()
    G = torch.full((1, pl.ld), 7.0, device="cuda")
    ws = layers.embed_workspace(pl, N, V, 1, x.dtype, tok.dtype)
    print("gradient", flush=True)
    layers.embed_backward(pl, tok, x, G, V, ws, scale=0.5)
    w = ref.embed_backward(tok[0, at], x[0, at], V, 0.5)
    ref.check("G", G[0, :V].view(V, 1), w[0], w[1])
    assert bool((G[0, V:] == 7.0).all())
    pl.close()
