"""The layer operators' forms of large batches, whose rows pass by the caches: on
both sides of every rule that chooses them, in place and not.  What a row becomes
does not go by how many rows a call has, so that the same rows in smaller calls,
which go through the caches, have to give the same bits; some rows, and every sum
over rows, are compared with 64 bits."""
import math

import pytest

import layer_refs as ref

pytestmark = pytest.mark.gpu


def _bits(t):
    import torch
    return t.contiguous().view({4: torch.int32, 2: torch.int16}[t.element_size()])


def _close(name, got, want, err):
    """ref.check for large tensors, without infinities, where they are."""
    import torch
    half = torch.finfo(got.dtype).eps / 2
    bound = err + half * (want.abs() + err) + torch.finfo(got.dtype).smallest_normal * half
    assert bool(((got.double() - want).abs() <= bound).all()), name


# ---------------------------------------------------------------------------
# distillation: type, workers, tokens, vocabulary, padding, entries.  Streamed from 64 MB
# read and written on, up to 1.4 GB or with rows that begin at lines of 128 bytes, and
# if there are fewer entries than such lines.

DISTILL = [
    ("bf16", 1, 1000, 17000, 3, 40), ("f16", 2, 300, 32001, 5, 9), ("f32", 1, 1200, 8193, 0, 64),    # 4 waves
    ("bf16", 4, 100, 50001, 0, 200), ("f16", 1, 300, 65536, 0, 33), ("f32", 2, 140, 32768, 1, 20),   # 8
    ("bf16", 1, 320, 65537, 2, 100), ("f32", 5, 50, 40001, 0, 7), ("f16", 1, 200, 98304, 0, 64),     # 16, in registers
    ("f16", 2, 100, 98305, 0, 50), ("bf16", 1, 150, 130560, 0, 31), ("f32", 1, 180, 65280, 0, 128),  # 16, in LDS too
    ("bf16", 1, 6000, 64000, 0, 16),      # above 1.4 GB, at lines
    ("bf16", 1, 6000, 64001, 0, 16),      # above 1.4 GB, not at lines: through the caches
    ("bf16", 1, 1000, 17000, 0, 300),     # more entries than lines: through the caches
    ("bf16", 1, 900, 17000, 3, 40),       # below 64 MB: through the caches
]


@pytest.mark.parametrize("case", DISTILL)
def test_distill(case):
    import torch
    from paper_2010_13359_amd import layers
    dt, M, N, V, pad, k = case
    T, dtype, ld = 2.0, ref.TYPES[dt], V + pad
    g = torch.Generator(device="cuda").manual_seed(V + N)
    pl, one = ref.plan(1024, M), ref.plan(1024, 1)
    z = torch.empty((M, N, ld), dtype=dtype, device="cuda")
    for row in z.view(M * N, ld).split(500):
        row.copy_(torch.randn(row.shape, generator=g, device="cuda") * 4.0)
    z[..., V:] = float("nan")
    val = 3.0 * torch.randn((M, N, k), generator=g, device="cuda")
    idx = torch.randint(0, V, (M, N, k), generator=g, device="cuda").int()      # in no order
    idx[torch.rand(idx.shape, generator=g, device="cuda") < 0.1] = -1
    weight = torch.rand((M, N), generator=g, device="cuda") + 0.5
    idx[0, 3] = idx[0, 3].sort().values
    idx[0, 5, k // 2:] = idx[0, 5, 0]            # an index named often
    idx[0, 7] = -1                               # no entry
    idx[0, 8] = torch.arange(V - k, V, device="cuda").int()
    weight[0, 9] = 0.0
    z[0, 9] = float("nan")
    z[0, 11, 1:V] = -math.inf
    idx[0, 11, :] = 0
    idx[0, 0, 0], idx[0, 0, k - 1] = V - 1, 0

    nan = lambda *s, dtype=torch.float32: torch.full(s, float("nan"), dtype=dtype, device="cuda")
    ws = layers.distill_workspace(pl, N, V, k, dtype, ld=ld)
    assert ws is None                            # a workgroup for each row
    loss, dz = nan(M, N), nan(M, N, ld, dtype=dtype)
    layers.distill_fused(pl, z, val, idx, weight, loss, dz, V, ws, temperature=T)
    stats, loss2, other = nan(M, N, 2), nan(M, N), nan(M, N, ld, dtype=dtype)
    layers.distill_forward(pl, z, val, idx, weight, loss2, stats, V, ws, temperature=T)
    layers.distill_backward(pl, z, val, idx, weight, stats, other, V, temperature=T)
    assert torch.equal(_bits(loss), _bits(loss2)) and torch.equal(_bits(dz), _bits(other))
    for call in (lambda: layers.distill_fused(pl, other, val, idx, weight, loss2, other, V, ws, temperature=T),
                 lambda: layers.distill_backward(pl, other, val, idx, weight, stats, other, V, temperature=T)):
        other.copy_(z)
        call()
        assert torch.equal(_bits(loss), _bits(loss2)) and torch.equal(_bits(dz), _bits(other))
    del other

    # fewer rows a call
    flat = [t.view((1, M * N) + t.shape[2:]) for t in (z, val, idx, weight, loss, dz)]
    row = V * z.element_size()
    some = min(int(63e6 / (2 * row)), 1000, M * N)
    if row <= 131072 or some > 128:              # (128 such rows and fewer would be shared out in slices)
        for a in range(0, M * N, some):
            a = max(0, min(a, M * N - some))
            x, v, i, w, l, d = (t[:, a:a + some].clone() for t in flat)      # aligned
            l1, d1 = nan(1, some), nan(1, some, ld, dtype=dtype)
            layers.distill_fused(one, x, v, i, w, l1, d1, V, None, temperature=T)
            assert torch.equal(_bits(l1), _bits(l)) and torch.equal(_bits(d1), _bits(d))

    # and in 64 bits
    at = [0, 3, 5, 7, 8, 9, 11, M * N // 2, M * N - 1]
    x, v, i, w, l, d = (t[0, at] for t in flat)
    want = ref.distill(x, v, i, w, V, T)
    ref.check("loss", l, want["loss"], want["loss_err"])
    ref.check("dz", d, want["dz"], want["dz_err"])
    assert not l[[3, 5]].any() and not d[[3, 5]].any() and bool(d[[0, 1, 2, 4]].any(-1).all())
    pl.close()
    one.close()


# ---------------------------------------------------------------------------
# layer norm: a width of every row shape.  Bytes read and written: forward, results
# pass by the caches above 100 MB; backward, above 80 MB the results, above 200 MB all.

WIDTHS = {2: [100, 201, 500, 1000, 1503, 2000, 4001, 6000, 8001, 12000, 20000],
          4: [61, 100, 300, 501, 800, 1003, 2000, 3001, 4000, 9000, 16001]}


@pytest.mark.parametrize("shape", range(11))
@pytest.mark.parametrize("dt", sorted(ref.TYPES))
def test_norm(dt, shape):
    import torch
    from paper_2010_13359_amd import layers
    dtype, size, M = ref.TYPES[dt], 4 if dt == "f32" else 2, 2
    D = WIDTHS[size][shape]
    pl = ref.plan(2 * D + 20, M)
    g = torch.Generator(device="cuda").manual_seed(D)
    P = torch.randn((M, pl.ld), generator=g, device="cuda")
    gamma, beta = 3, D + 5
    for bytes_ in (75e6, 120e6, 230e6):          # backward; forward two thirds of it, 153 MB the last
        N = int(bytes_ / (3 * size * M * D))
        x = (torch.randn((M, N, D), generator=g, device="cuda") + 0.3).to(dtype)
        y, stats = torch.full_like(x, float("nan")), torch.empty((M, N, 2), device="cuda")
        layers.norm_forward(pl, x, P, y, stats, gamma=gamma, beta=beta)
        dy = torch.randn((M, N, D), generator=g, device="cuda").to(dtype)
        dx, G = torch.full_like(x, float("nan")), torch.full((M, pl.ld), 7.0, device="cuda")
        ws = layers.norm_workspace(pl, N, D, dtype, gamma=gamma, beta=beta)
        if ws is not None:
            ws.fill_(0xFF)
        layers.norm_backward(pl, x, dy, P, stats, dx, G, ws, gamma=gamma, beta=beta)
        # in place
        inplace, G2 = x.clone(), torch.full((M, pl.ld), 7.0, device="cuda")
        layers.norm_forward(pl, inplace, P, inplace, gamma=gamma, beta=beta)
        assert torch.equal(_bits(inplace), _bits(y))
        inplace.copy_(dy)
        layers.norm_backward(pl, x, inplace, P, stats, inplace, G2, ws, gamma=gamma, beta=beta)
        assert torch.equal(_bits(inplace), _bits(dx)) and torch.equal(_bits(G2), _bits(G))
        del inplace
        # fewer rows a call
        some = max(1, int(70e6 / (3 * size * M * D)))
        ws = layers.norm_workspace(pl, some, D, dtype, gamma=gamma, beta=beta)
        for a in range(0, N, some):
            a = max(0, min(a, N - some))
            xs, dys, ss = (t[:, a:a + some].contiguous() for t in (x, dy, stats))
            ys, ss2, dxs = torch.empty_like(xs), torch.empty_like(ss), torch.empty_like(xs)
            layers.norm_forward(pl, xs, P, ys, ss2, gamma=gamma, beta=beta)
            layers.norm_backward(pl, xs, dys, P, ss, dxs, G2, ws, gamma=gamma, beta=beta)
            for small, large in ((ys, y), (ss2, stats), (dxs, dx)):
                assert torch.equal(_bits(small), _bits(large[:, a:a + some]))
        # and in 64 bits
        own = torch.zeros(pl.ld, dtype=torch.bool, device="cuda")
        own[gamma:gamma + D] = own[beta:beta + D] = True
        assert bool((G[:, ~own] == 7.0).all())
        for m in range(M):
            at = torch.tensor([0, N // 3, N - 1], device="cuda")
            gm, bm = P[m, gamma:gamma + D], P[m, beta:beta + D]
            w = ref.norm_forward(x[m, at], gm, bm, 1e-5)
            ref.check("y", y[m, at], w[0], w[1])
            w = ref.norm_backward(x[m, at], dy[m, at], gm, stats[m, at])
            ref.check("dx", dx[m, at], w[0], w[1])
            xh, d = (x[m].double() - stats[m, :, :1]) * stats[m, :, 1:].double(), dy[m].double()
            _close("dbeta", G[m, beta:beta + D], d.sum(0), (N + 1) * ref.U * d.abs().sum(0))
            d *= xh
            _close("dgamma", G[m, gamma:gamma + D], d.sum(0), (N + 4) * ref.U * d.abs().sum(0))
            del xh, d
    pl.close()


# ---------------------------------------------------------------------------
# embedding: the lookup's results pass by the caches above 30 MB, rows with single
# channels above 60 MB if they have 256 bytes, between 65 and 160 MB if they have 140;
# the gradient's rows above 100 MB.


@pytest.mark.parametrize("D", [31, 64, 99, 130, 1027])
@pytest.mark.parametrize("dt", sorted(ref.TYPES))
def test_lookup(dt, D):
    import torch
    from paper_2010_13359_amd import layers
    dtype, size, M, V = ref.TYPES[dt], 4 if dt == "f32" else 2, 2, 3001
    pl = ref.plan(V * D + 7, M)
    g = torch.Generator(device="cuda").manual_seed(D)
    P = torch.randn((M, pl.ld), generator=g, device="cuda")
    for bytes_ in (28e6, 34e6, 65e6, 90e6, 170e6):
        N = int(bytes_ / (M * D * size))
        tok = torch.randint(-1, V + 1, (M, N), generator=g, device="cuda")
        out = torch.full((M, N, D), float("nan"), dtype=dtype, device="cuda")
        layers.embed_forward(pl, tok, P, out, V, offset=7, scale=1.7)
        # a product that is rounded to 32 bits and then to the type, a single channel behind the last
        # vector of f16 at once (v_fma_mixlo_f16): off by 2^-24 of it before the last rounding, or nothing
        for m in range(M):
            there = (tok[m] >= 0) & (tok[m] < V)
            rows = P[m, 7:7 + V * D].view(V, D)[torch.where(there, tok[m], 0)].double() * float(torch.tensor(1.7))
            _close("out", out[m], rows * there[:, None], ref.U * rows.abs() * there[:, None])
    pl.close()


# widths of 8, 16 and 64 lanes a row, and of two slabs
@pytest.mark.parametrize("D", [21, 50, 100, 515, 1041])
@pytest.mark.parametrize("dt", sorted(ref.TYPES))
def test_embedding_gradient(dt, D):
    import torch
    from paper_2010_13359_amd import layers
    dtype, size, M, V = ref.TYPES[dt], 4 if dt == "f32" else 2, 2, 5003
    pl = ref.plan(V * D + 7, M)
    g = torch.Generator(device="cuda").manual_seed(D)
    for bytes_ in (95e6, 106e6):
        N = int(bytes_ / (M * D * size))
        u = torch.rand((M, N), generator=g, device="cuda") ** 4
        tok = (u * (V + 100)).long() - 40        # frequent ones first, some out of range on either side
        dout = torch.randn((M, N, D), generator=g, device="cuda").to(dtype)
        G = torch.full((M, pl.ld), 7.0, device="cuda")
        ws = layers.embed_workspace(pl, N, V, D, dtype, offset=7)
        ws.fill_(0xFF)
        for add in (False, True):
            before = G[:, 7:7 + V * D].view(M, V, D).double() if add else None
            layers.embed_backward(pl, tok, dout, G, V, ws, offset=7, scale=0.3, add=add)
            assert bool((G[:, :7] == 7.0).all() and (G[:, 7 + V * D:] == 7.0).all())
            for m in range(M):
                keep = (tok[m] >= 0) & (tok[m] < V)
                t, d = tok[m][keep], dout[m][keep].double()
                total, terms = (torch.zeros((V, D), dtype=torch.float64, device="cuda") for _ in range(2))
                total.index_add_(0, t, d)
                terms.index_add_(0, t, d.abs())
                count = torch.bincount(t, minlength=V)[:, None].double()
                s = float(torch.tensor(0.3))
                want, err = total * s, ref.U * (count + 1) * terms * s
                if add:
                    want = want + before[m]
                    err = torch.where(count > 0, err + ref.U * (want.abs() + err), 0.0)
                _close("G", G[m, 7:7 + V * D].view(V, D), want, err)
    pl.close()
