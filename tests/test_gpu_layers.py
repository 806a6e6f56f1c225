"""The layer operators together, as a student's gradients for Algorithm 2, and
what they share: calls captured in a graph, on several streams at a time, with
arguments that are refused, and on more than 2^31 elements."""
import numpy as np
import pytest

import layer_refs as ref

pytestmark = pytest.mark.gpu


def _bits(t):
    import torch
    return t.contiguous().view({4: torch.int32, 2: torch.int16}[t.element_size()])


# ---------------------------------------------------------------------------
# together


@pytest.mark.parametrize("M,vocab,width,tokens,k,T", [(2, 60, 24, 40, 7, 1.0), (3, 301, 65, 200, 16, 2.0)])
def test_students_gradients(M, vocab, width, tokens, k, T):
    """Every stage of Student.gradients in 64 bits from the stage before it as the
    GPU left it.  A product of n terms is off by n u of its absolute values, and a
    logit that is off by e changes its token's softmax by at most a factor of
    exp(2 e / T)."""
    import torch
    from paper_2010_13359_amd import closed_loop, dqgan
    d, offsets = closed_loop.Student.parameters(vocab, width)
    plan = dqgan.Plan(d, M, "identity")
    gen = torch.Generator().manual_seed(M)
    P = (0.3 * torch.randn((M, plan.ld), generator=gen)).cuda()
    P[:, offsets[1]:offsets[2]] += 1.0
    tok = torch.randint(-1, vocab, (M, tokens), generator=gen).cuda()
    val = torch.randn((M, tokens, k), generator=gen).cuda()
    idx = torch.randint(0, vocab, (M, tokens, k), generator=gen).int().cuda()
    weight = torch.rand((M, tokens), generator=gen).cuda()
    G = torch.full((M, plan.ld), 5.0, device="cuda")
    st = closed_loop.Student(plan, vocab, width, tokens, k, T)
    loss = st.gradients(P, tok, val, idx, weight, G)
    assert bool((G[:, d:] == 5.0).all())
    for m in range(M):
        E = P[m, :offsets[1]].double().cpu().view(vocab, width)
        gamma, beta = P[m, offsets[1]:offsets[2]], P[m, offsets[2]:d]
        w = ref.embed_forward(tok[m], E, st.scale)
        ref.check("x", st.x[m], w[0], w[1])
        w = ref.norm_forward(st.x[m], gamma, beta, 1e-5)
        ref.check("y", st.y[m], w[0], w[1])
        y = st.y[m].double().cpu()
        z, off = y @ E.T, (width + 1) * ref.U * (y.abs() @ E.abs().T)
        w = ref.distill(z, val[m], idx[m], weight[m], vocab, T)
        e = torch.expm1(2 * off.max(1).values / T)
        a = weight[m].double().cpu()
        s = torch.softmax(z / T, 1)
        ref.check("loss", loss[m], w["loss"], w["loss_err"] + a * T * 2 * off.max(1).values)
        ref.check("dz", st.z[m], w["dz"], w["dz_err"] + a[:, None] * T * s * e[:, None])
        dz = st.z[m].double().cpu()
        dy, off = dz @ E, (vocab + 1) * ref.U * (dz.abs() @ E.abs())
        g, stats = gamma.double().cpu(), st.stats[m].double().cpu()
        xh = (st.x[m].double().cpu() - stats[:, :1]) * stats[:, 1:]
        w = ref.norm_backward(st.x[m], dy, gamma, st.stats[m])
        o = off * g.abs()
        dx_off = stats[:, 1:] * (o + o.mean(1, keepdim=True) + xh.abs() * (o * xh.abs()).mean(1, keepdim=True))
        ref.check("dx", st.dx[m], w[0], w[1] + dx_off * 1.001)
        ref.check("dgamma", G[m, offsets[1]:offsets[2]], w[2], w[3] + (off * xh.abs()).sum(0) * 1.001)
        ref.check("dbeta", G[m, offsets[2]:d], w[4], w[5] + off.sum(0) * 1.001)
        head, head_off = dz.T @ y, (tokens + 1) * ref.U * (dz.T.abs() @ y.abs())
        w = ref.embed_backward(tok[m], st.dx[m], vocab, st.scale, head)
        ref.check("dE", G[m, :offsets[1]].view(vocab, width), w[0], w[1] + head_off + ref.U * w[0].abs())
    plan.close()


@pytest.mark.parametrize("kind,extra", [("identity", {}), ("sign", {}), ("qsgd", {"levels": 15}), ("topk", {"keep": 300}),
                                        ("mbit", {"levels": 8, "norm": "linf"})])
def test_student_runs_with_every_compressor(kind, extra):
    from paper_2010_13359_amd import closed_loop
    hist = closed_loop.run_student(kind, T=6, **extra)
    assert len(hist) == 6 and np.isfinite(hist).all() and min(hist) > 0


def test_student_in_16_bits():
    import torch
    from paper_2010_13359_amd import closed_loop
    hist = closed_loop.run_student("sign", vocab=1000, width=96, tokens=300, T=4, temperature=2.0, dtype=torch.bfloat16)
    assert len(hist) == 4 and np.isfinite(hist).all() and min(hist) > 0


# ---------------------------------------------------------------------------
# graphs and streams


def _calls(seed, M, N, V, D, k, dt):
    """One set of buffers, and every operator on it."""
    import torch
    from paper_2010_13359_amd import layers
    gen = torch.Generator().manual_seed(seed)
    plan = ref.plan(V * D + 2 * D + 5, M)
    dtype = ref.TYPES[dt]
    where = dict(gamma=V * D, beta=V * D + D + 3)
    P = torch.randn((M, plan.ld), generator=gen).cuda()
    tok = torch.randint(-1, V, (M, N), generator=gen).cuda()
    dy = torch.randn((M, N, D), generator=gen).to(dtype).cuda()
    z = torch.randn((M, N, V), generator=gen).to(dtype).cuda()
    val = torch.randn((M, N, k), generator=gen).cuda()
    idx = torch.randint(0, V, (M, N, k), generator=gen).int().cuda()
    weight = torch.rand((M, N), generator=gen).cuda()
    out = {n: torch.empty((M, N, D), dtype=dtype, device="cuda") for n in ("x", "y", "dx")}
    out.update(stats=torch.empty((M, N, 2), device="cuda"), zstats=torch.empty((M, N, 2), device="cuda"),
               loss=torch.empty((M, N), device="cuda"), loss2=torch.empty((M, N), device="cuda"),
               dz=torch.empty_like(z), dz2=torch.empty_like(z), G=torch.empty((M, plan.ld), device="cuda"))
    ws = (layers.embed_workspace(plan, N, V, D, dtype), layers.norm_workspace(plan, N, D, dtype, **where),
          layers.distill_workspace(plan, N, V, k, dtype))

    def run(stream=None):
        layers.embed_forward(plan, tok, P, out["x"], V, scale=2.0, stream=stream)
        layers.norm_forward(plan, out["x"], P, out["y"], out["stats"], stream=stream, **where)
        layers.norm_backward(plan, out["x"], dy, P, out["stats"], out["dx"], out["G"], ws[1], stream=stream, **where)
        layers.embed_backward(plan, tok, out["dx"], out["G"], V, ws[0], scale=2.0, stream=stream)
        layers.embed_backward(plan, tok, dy, out["G"], V, ws[0], add=True, stream=stream)
        layers.distill_forward(plan, z, val, idx, weight, out["loss"], out["zstats"], V, ws[2], stream=stream)
        layers.distill_backward(plan, z, val, idx, weight, out["zstats"], out["dz"], V, stream=stream)
        layers.distill_fused(plan, z, val, idx, weight, out["loss2"], out["dz2"], V, ws[2], stream=stream)

    def scramble():
        for t in out.values():
            t.fill_(float("nan"))
        for t in ws:
            if t is not None:
                t.fill_(0xFF)

    def result():  # the padding of G is nobody's
        return {n: _bits(t[:, :V * D + D] if n == "G" else t).clone() for n, t in out.items()}
    return plan, run, scramble, result, (z, out)


# small and large: every operator's one-launch and several-launch forms
SIZES = [(2, 50, 300, 40, 5, "bf16"), (1, 300, 70001, 33, 9, "f32"), (2, 5000, 60, 600, 12, "f16"),
         (1, 3, 140001, 16, 20, "bf16")]


@pytest.mark.parametrize("size", SIZES)
def test_graph_replays(size):
    import torch
    plan, run, scramble, result, (z, out) = _calls(1, *size)
    scramble()
    run()
    torch.cuda.synchronize()
    want = result()
    assert torch.equal(want["dz"], want["dz2"]) and torch.equal(want["loss"], want["loss2"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run()
    for replay in range(3):
        scramble()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = result()
        for n in want:
            assert torch.equal(got[n], want[n]), (replay, n)
        run()      # eager work between the replays
        torch.cuda.synchronize()
        got = result()
        for n in want:
            assert torch.equal(got[n], want[n]), (replay, n)
    plan.close()


def test_calls_on_several_streams():
    """Two sets of calls on one stream each, interleaved call by call by the
    hardware: distinct workspaces, the same results as alone."""
    import torch
    sets = [_calls(5 + i, *SIZES[i]) for i in (0, 1, 2)]
    want = []
    for plan, run, scramble, result, _ in sets:
        scramble()
        run()
        torch.cuda.synchronize()
        want.append(result())
        scramble()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(3):
        for (plan, run, scramble, result, _), s in zip(sets, streams):
            run(stream=s)
    torch.cuda.synchronize()
    for (plan, run, scramble, result, _), w in zip(sets, want):
        got = result()
        for n in w:
            assert torch.equal(got[n], w[n]), n
        plan.close()


def test_one_plan_on_two_streams():
    """Calls use none of the plan's own scratch."""
    import torch
    from paper_2010_13359_amd import layers
    plan = ref.plan(3000 * 40, 2, kind="sign")
    gen = torch.Generator().manual_seed(2)
    tok = [torch.randint(0, 3000, (2, 700), generator=gen).cuda() for _ in range(2)]
    dout = [torch.randn((2, 700, 40), generator=gen).cuda() for _ in range(2)]
    G = [torch.zeros((2, plan.ld), device="cuda") for _ in range(4)]
    ws = [layers.embed_workspace(plan, 700, 3000, 40, torch.float32) for _ in range(2)]
    for i in range(2):
        layers.embed_backward(plan, tok[i], dout[i], G[2 + i], 3000, ws[i])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for i, s in enumerate(streams):
            layers.embed_backward(plan, tok[i], dout[i], G[i], 3000, ws[i], stream=s)
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(_bits(G[i]), _bits(G[2 + i]))
    plan.close()


# ---------------------------------------------------------------------------
# refusals


def test_refusals():
    """Wrong types, shapes, places and sizes are refused before anything runs."""
    import torch
    from paper_2010_13359_amd import dqgan, layers
    M, N, V, D, k = 2, 300, 30, 24, 4
    plan = ref.plan(V * D + 2 * D, M)
    new = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device="cuda")
    P, G = new(M, plan.ld), new(M, plan.ld)
    tok, x, y, dx = new(M, N, dtype=torch.int64), new(M, N, D), new(M, N, D), new(M, N, D)
    stats, z, dz = new(M, N, 2), new(M, N, V), new(M, N, V)
    val, idx, weight, loss = new(M, N, k), new(M, N, k, dtype=torch.int32), new(M, N), new(M, N)
    ews, nws = layers.embed_workspace(plan, N, V, D, torch.float32), layers.norm_workspace(plan, N, D, torch.float32, V * D)
    off = torch.zeros(M * N * D + 1, device="cuda")[1:].view(M, N, D)      # 4 bytes off
    wrong = (TypeError, ValueError)
    bad = [
        lambda: layers.embed_forward(plan, tok.float(), P, x, V),
        lambda: layers.embed_forward(plan, tok[:, :-1], P, x, V),
        lambda: layers.embed_forward(plan, tok.cpu(), P, x, V),
        lambda: layers.embed_forward(plan, tok, P[:, :-8], x, V),
        lambda: layers.embed_forward(plan, tok, P.double(), x, V),
        lambda: layers.embed_forward(plan, tok, P, x.double(), V),
        lambda: layers.embed_forward(plan, tok, P, x[0], V),
        lambda: layers.embed_forward(plan, tok, P, x.transpose(1, 2).contiguous().transpose(1, 2), V),
        lambda: layers.embed_backward(plan, tok, x, G, V, None),
        lambda: layers.embed_backward(plan, tok, x, G, V, ews[:-1]),
        lambda: layers.embed_backward(plan, tok, x, G[:, :100], V, ews),
        lambda: layers.norm_forward(plan, x, P, y.half(), stats),
        lambda: layers.norm_forward(plan, x, P, y[:, 1:], stats),
        lambda: layers.norm_forward(plan, x, P, y, stats[..., 0]),
        lambda: layers.norm_forward(plan, x[:1], P, y, stats),
        lambda: layers.norm_backward(plan, x, y, P, stats, dx, G, None, gamma=V * D),
        lambda: layers.norm_backward(plan, x, y.bfloat16(), P, stats, dx, G, nws, gamma=V * D),
        lambda: layers.norm_backward(plan, x, y, P, stats.double(), dx, G, nws, gamma=V * D),
        lambda: layers.distill_forward(plan, z, val[..., :-1], idx, weight, loss, stats),
        lambda: layers.distill_forward(plan, z, val, idx.long(), weight, loss, stats),
        lambda: layers.distill_forward(plan, z, val.half(), idx, weight, loss, stats),
        lambda: layers.distill_forward(plan, z, val, idx, weight[:, :-1], loss, stats),
        lambda: layers.distill_backward(plan, z, val, idx, weight, stats, dz.half()),
        lambda: layers.distill_fused(plan, z, val, idx, weight, loss.cpu(), dz),
        lambda: layers.distill_fused(plan, z.int(), val, idx, weight, loss, dz),
    ]
    status = [
        (dqgan.EALIGN, lambda: layers.embed_forward(plan, tok, P, off, V)),
        (dqgan.EALIGN, lambda: layers.norm_forward(plan, off, P, y, stats)),
        (dqgan.EINVAL, lambda: layers.embed_forward(plan, tok, P, x, V + 3)),          # beyond d
        (dqgan.EINVAL, lambda: layers.embed_forward(plan, tok, P, x, V, offset=-1)),
        (dqgan.EINVAL, lambda: layers.embed_forward(plan, tok, P, x, 0)),
        (dqgan.EINVAL, lambda: layers.embed_forward(plan, tok, P, x, V, scale=float("nan"))),
        (dqgan.EINVAL, lambda: layers.norm_forward(plan, x, P, y, stats, gamma=0, beta=D - 1)),   # overlap
        (dqgan.EINVAL, lambda: layers.norm_forward(plan, x, P, y, stats, gamma=V * D + D + 1)),
        (dqgan.EINVAL, lambda: layers.norm_forward(plan, x, P, y, stats, eps=-1.0)),
        (dqgan.EINVAL, lambda: layers.distill_forward(plan, z, val, idx, weight, loss, stats, vocab=V + 1)),
        (dqgan.EINVAL, lambda: layers.distill_forward(plan, z, val, idx, weight, loss, stats, temperature=0.0)),
        (dqgan.EINVAL, lambda: layers.distill_fused(plan, z, new(M, N, 0), new(M, N, 0, dtype=torch.int32), weight, loss, dz)),
        (dqgan.EINVAL, lambda: layers.norm_forward(plan, x, None, y, stats)),           # a weight, no parameters
        (dqgan.EINVAL, lambda: layers.distill_forward(plan, z, val, idx, weight, loss, None)),
    ]
    for t in (x, y, dx, stats, z, dz, loss, G):
        t.fill_(3.0)
    for i, f in enumerate(bad):
        with pytest.raises(wrong):
            f()
            print("not refused:", i)
    for i, (s, f) in enumerate(status):
        with pytest.raises(dqgan.DqganError) as e:
            f()
            print("not refused:", i)
        assert e.value.status == s, i
    torch.cuda.synchronize()
    for t in (x, y, dx, stats, z, dz, loss, G):
        assert bool((t == 3.0).all())
    plan.close()


# ---------------------------------------------------------------------------
# more than 2^31 elements


def test_many_elements():
    import torch
    from paper_2010_13359_amd import layers
    gen = torch.Generator().manual_seed(4)
    N, V, k = 16901, 127101, 8     # 2.148e9 logits
    print("logits", N * V, flush=True)
    plan = ref.plan(1024, 1)
    z = torch.zeros((1, N, V), dtype=torch.float16, device="cuda")
    last = (2 * torch.randn((2, V), generator=gen)).half()
    z[0, -2:] = last.cuda()
    val, idx = torch.randn((1, N, k), generator=gen).cuda(), torch.randint(0, V, (1, N, k), generator=gen).int().cuda()
    loss = torch.empty((1, N), device="cuda")
    layers.distill_fused(plan, z, val, idx, None, loss, z)
    w = ref.distill(last, val[0, -2:], idx[0, -2:], None, V, 1.0)
    ref.check("loss", loss[0, -2:], w["loss"], w["loss_err"])
    ref.check("dz", z[0, -2:], w["dz"], w["dz_err"])
    w = ref.distill(torch.zeros((1, V)), val[0, 5:6], idx[0, 5:6], None, V, 1.0)
    ref.check("dz", z[0, 5:6], w["dz"], w["dz_err"])
    plan.close()
    del z
    N, D = 150001, 14320           # 2.148e9 activations
    print("activations", N * D, flush=True)
    plan = ref.plan(2 * D, 1)
    x = torch.zeros((1, N, D), dtype=torch.bfloat16, device="cuda")
    rows = torch.randn((2, D), generator=gen).bfloat16()
    x[0, -2:] = rows.cuda()
    P = torch.randn((1, plan.ld), generator=gen).cuda()
    stats = torch.empty((1, N, 2), device="cuda")
    G = torch.zeros_like(P)
    ws = layers.norm_workspace(plan, N, D, x.dtype, 0, D)
    dy = x.clone()
    layers.norm_backward(plan, x, dy, P, torch.stack([torch.zeros(N), torch.ones(N)], -1)[None].cuda(), dy, G, ws, 0, D)
    w = ref.norm_backward(rows, rows, P[0, :D], torch.tensor([[0.0, 1.0]] * 2))
    ref.check("dx", dy[0, -2:], w[0], w[1])
    ref.check("dgamma", G[0, :D], w[2], w[3])
    layers.norm_forward(plan, x, P, x, stats, gamma=0, beta=D)
    w = ref.norm_forward(rows, P[0, :D], P[0, D:2 * D], 1e-5)
    ref.check("y", x[0, -2:], w[0], w[1])
    plan.close()


# ---------------------------------------------------------------------------
# most workers, widest rows


@pytest.mark.parametrize("N", [2, 230])
def test_most_workers(N):
    import torch
    from paper_2010_13359_amd import layers
    M, V, D, k = 1024, 21, 13, 5
    where = dict(gamma=V * D, beta=V * D + D)
    plan = ref.plan(V * D + 2 * D, M)
    gen = torch.Generator().manual_seed(N)
    P = torch.randn((M, plan.ld), generator=gen).cuda()
    tok = torch.randint(-1, V + 1, (M, N), generator=gen).int().cuda()
    dy = torch.randn((M, N, D), generator=gen).cuda()
    z, val = torch.randn((M, N, V), generator=gen).cuda(), torch.randn((M, N, k), generator=gen).cuda()
    idx = torch.randint(0, V + 2, (M, N, k), generator=gen).int().cuda()
    x, y, dx, dz = torch.empty_like(dy), torch.empty_like(dy), torch.empty_like(dy), torch.empty_like(z)
    stats, loss = torch.empty((M, N, 2), device="cuda"), torch.empty((M, N), device="cuda")
    G = torch.full((M, plan.ld), 7.0, device="cuda")
    layers.embed_forward(plan, tok, P, x, V)
    layers.norm_forward(plan, x, P, y, stats, **where)
    layers.norm_backward(plan, x, dy, P, stats, dx, G, layers.norm_workspace(plan, N, D, x.dtype, **where), **where)
    layers.embed_backward(plan, tok, dx, G, V, layers.embed_workspace(plan, N, V, D, x.dtype))
    layers.distill_fused(plan, z, val, idx, None, loss, dz)
    for m in (0, 1, 500, 1022, 1023):
        gamma, beta = P[m, V * D:V * D + D], P[m, V * D + D:V * D + 2 * D]
        w = ref.embed_forward(tok[m], P[m, :V * D].view(V, D), 1.0)
        ref.check("x", x[m], w[0], w[1])
        w = ref.norm_forward(x[m], gamma, beta, 1e-5)
        ref.check("y", y[m], w[0], w[1])
        w = ref.norm_backward(x[m], dy[m], gamma, stats[m])
        ref.check("dx", dx[m], w[0], w[1])
        ref.check("dgamma", G[m, V * D:V * D + D], w[2], w[3])
        ref.check("dbeta", G[m, V * D + D:V * D + 2 * D], w[4], w[5])
        w = ref.embed_backward(tok[m], dx[m], V, 1.0)
        ref.check("dE", G[m, :V * D].view(V, D), w[0], w[1])
        w = ref.distill(z[m], val[m], idx[m], None, V, 1.0)
        ref.check("loss", loss[m], w["loss"], w["loss_err"])
        ref.check("dz", dz[m], w["dz"], w["dz_err"])
    assert bool((G[:, V * D + 2 * D:] == 7.0).all())
    plan.close()


def test_widest_rows():
    """Rows of 2^24 elements; a width beyond is refused."""
    import torch
    from paper_2010_13359_amd import dqgan, layers
    D = 1 << 24
    gen = torch.Generator().manual_seed(6)
    plan = ref.plan(2 * D + 1, 1)
    P = torch.randn((1, plan.ld), generator=gen).cuda()
    G = torch.full((1, plan.ld), 7.0, device="cuda")
    tok = torch.tensor([[1, 0, 1]], device="cuda")
    x, dy = torch.empty((1, 3, D), dtype=torch.bfloat16, device="cuda"), torch.randn((1, 3, D), generator=gen).bfloat16().cuda()
    print("embedding", flush=True)
    layers.embed_forward(plan, tok, P, x, 2)
    w = ref.embed_forward(tok[0], P[0, :2 * D].view(2, D), 1.0)
    ref.check("x", x[0], w[0], w[1])
    layers.embed_backward(plan, tok, dy, G, 2, layers.embed_workspace(plan, 3, 2, D, x.dtype))
    w = ref.embed_backward(tok[0], dy[0], 2, 1.0)
    ref.check("dE", G[0, :2 * D].view(2, D), w[0], w[1])
    assert bool((G[:, 2 * D:] == 7.0).all())
    print("layer norm", flush=True)
    y, dx, stats = torch.empty_like(x), torch.empty_like(x), torch.empty((1, 3, 2), device="cuda")
    layers.norm_forward(plan, x, P, y, stats, gamma=1, beta=D + 1)
    w = ref.norm_forward(x[0], P[0, 1:D + 1], P[0, D + 1:2 * D + 1], 1e-5)
    ref.check("y", y[0], w[0], w[1])
    layers.norm_backward(plan, x, dy, P, stats, dx, G, layers.norm_workspace(plan, 3, D, x.dtype, 1, D + 1), 1, D + 1)
    w = ref.norm_backward(x[0], dy[0], P[0, 1:D + 1], stats[0])
    ref.check("dx", dx[0], w[0], w[1])
    ref.check("dgamma", G[0, 1:D + 1], w[2], w[3])
    with pytest.raises(dqgan.DqganError) as e:
        layers.embed_forward(plan, tok[:, :1], P, torch.empty((1, 1, D + 1), device="cuda"), 1)
    assert e.value.status == dqgan.EINVAL
    plan.close()


# ---------------------------------------------------------------------------
# beyond the type


@pytest.mark.parametrize("dt,big", [("f16", 1e4)])
@pytest.mark.parametrize("D", [5, 64, 131, 700])
def test_beyond_the_type(dt, big, D):
    """Results above the type's largest value are infinities of their sign, whole vectors
    and single elements alike, and their neighbours stay as they are.  (bf16 ends where
    binary32 does: what is beyond it is beyond the sums that it is made of.)"""
    import torch
    from paper_2010_13359_amd import layers
    M, N, V, k = 1, 12, 40, 3
    gen = torch.Generator().manual_seed(D)
    pl = ref.plan(V * D, M)
    dtype = ref.TYPES[dt]
    P = (big * torch.randn((M, pl.ld), generator=gen) ** 3).cuda()
    tok = torch.randint(0, V, (M, N), generator=gen).cuda()
    x = torch.empty((M, N, D), dtype=dtype, device="cuda")
    layers.embed_forward(pl, tok, P, x, V, scale=2.0)
    w = ref.embed_forward(tok[0], P[0, :V * D].view(V, D), 2.0)
    assert ref.check_range("lookup", x[0], w[0], w[1]) > 0
    x.copy_(torch.randn((M, N, D), generator=gen))
    y, stats, dx = torch.empty_like(x), torch.empty((M, N, 2), device="cuda"), torch.empty_like(x)
    layers.norm_forward(pl, x, P, y, stats, gamma=0, beta=2 * D, eps=1e-3)
    w = ref.norm_forward(x[0], P[0, :D], P[0, 2 * D:3 * D], 1e-3)
    assert ref.check_range("y", y[0], w[0], w[1]) > 0
    dy = (3 * torch.randn((M, N, D), generator=gen)).to(dtype).cuda()
    layers.norm_backward(pl, x, dy, P, stats, dx, P.clone(), layers.norm_workspace(pl, N, D, dtype, 0, 2 * D), 0, 2 * D)
    w = ref.norm_backward(x[0], dy[0], P[0, :D], stats[0])
    assert ref.check_range("dx", dx[0], w[0], w[1]) > 0
    z = (20 * torch.randn((M, N, D), generator=gen)).to(dtype).cuda()
    val, idx = torch.randn((M, N, k), generator=gen).cuda(), torch.randint(0, D, (M, N, k), generator=gen).int().cuda()
    weight, loss, dz = torch.full((M, N), 50 * big, device="cuda"), torch.empty((M, N), device="cuda"), torch.empty_like(z)
    layers.distill_fused(pl, z, val, idx, weight, loss, dz, D)
    w = ref.distill_close(z[0], val[0], idx[0], weight[0], D, 1.0)
    assert ref.check_range("dz", dz[0], w["dz"], w["dz_err"]) > 0
    pl.close()


@pytest.mark.parametrize("kind,extra", [("identity", {}), ("sign", {}), ("qsgd", {"levels": 15}), ("topk", {"keep": 300}),
                                        ("mbit", {"levels": 8, "norm": "linf"})])
def test_every_iteration_of_the_student(kind, extra, monkeypatch):
    """What the compressor takes in every iteration is written whole (G is NaN before), at
    evaluation points that the last iteration moved, and the losses are those of 64 bits
    there.  (The gradients themselves: test_students_gradients.)"""
    import torch
    from paper_2010_13359_amd import closed_loop
    real, points = closed_loop.Student.gradients, []

    def gradients(self, P, tokens, val, idx, weight, G):
        d = self.parameters(self.vocab, self.width)[0]
        G[:, :d] = float("nan")
        loss = real(self, P, tokens, val, idx, weight, G)
        assert bool(torch.isfinite(G[:, :d]).all()) and bool(G[:, :d].any(1).all())
        assert not points or not torch.equal(points[-1], P)
        points.append(P.clone())
        V, D = self.vocab, self.width
        for m in range(P.shape[0]):
            E, beta = P[m, :V * D].double().view(V, D), P[m, V * D + D:d].double()
            x = E[tokens[m]] * self.scale
            xc = x - x.mean(-1, keepdim=True)
            y = xc / ((xc * xc).mean(-1, keepdim=True) + 1e-5).sqrt() * P[m, V * D:V * D + D].double() + beta
            s = torch.log_softmax(y @ E.T / self.temperature, -1)
            t = torch.log_softmax(val[m].double() / self.temperature, -1)
            T2 = self.temperature ** 2
            want = weight[m].double() * T2 * (t.exp() * (t - s.gather(-1, idx[m].long()))).sum(-1)
            # a logit of D terms is off by D u of their sizes and by y's own error, up to 2 depth(D) u of
            # it; it comes twice into the loss, as itself and in the sum, and t (log t - log s), below 10
            # here, is off by some 20 u of itself
            off = (D + 2 * ref.depth(D)) * ref.U * (y.abs() @ E.abs().T).amax(-1)
            assert bool(((loss[m].double() - want).abs() <= weight[m] * T2 * (4 * off + 200 * ref.U)).all())
        return loss
    monkeypatch.setattr(closed_loop.Student, "gradients", gradients)
    hist = closed_loop.run_student(kind, T=4, **extra)
    assert len(hist) == 4 == len(points)
