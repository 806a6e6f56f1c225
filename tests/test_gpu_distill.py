"""Distillation from a teacher's top logits against 64 bits: vocabularies on
both sides of a vector and a pass, padded rows, messages in any order, with
skipped and repeated entries, tokens that take no part, masked logits, and the
fused call against the two it stands for."""
import math

import pytest

import layer_refs as ref

pytestmark = pytest.mark.gpu

# M, tokens, vocabulary, padding, k
SHAPES = [(1, 1, 1, 0, 1), (2, 3, 2, 1, 4), (1, 5, 7, 0, 3), (1, 4, 8, 5, 8), (3, 2, 9, 0, 20), (2, 7, 1000, 24, 64),
          (1, 6, 4095, 0, 63), (1, 3, 4096, 1, 65), (2, 2, 4097, 7, 128), (1, 2, 32000, 0, 512), (1, 3, 33001, 3, 1024),
          (1, 2, 65536, 0, 7), (1, 2, 65537, 2, 100), (1, 1, 131072, 0, 32), (2, 1, 131073, 0, 33), (1, 1, 300007, 0, 5),
          (4, 300, 50, 14, 10), (1, 0, 100, 0, 4)]


def _setup(shape, dt, seed=0, spread=3.0):
    import torch
    M, N, V, pad, k = shape
    gen = torch.Generator().manual_seed(seed)
    pl = ref.plan(1024, M)
    z = (spread * torch.randn((M, N, V + pad), generator=gen)).to(ref.TYPES[dt])
    z[..., V:] = float("nan")                      # padding is not read
    val = spread * torch.randn((M, N, k), generator=gen) + 5.0
    idx = torch.randint(0, V, (M, N, k), generator=gen)
    skip = torch.rand((M, N, k), generator=gen) < 0.1
    idx = torch.where(skip, torch.where(torch.rand((M, N, k), generator=gen) < 0.5, V, 0xFFFFFFFF), idx)
    weight = torch.rand((M, N), generator=gen) + 0.5
    # the uint32 words in int32
    idx = torch.where(idx >= 2 ** 31, idx - 2 ** 32, idx).int()
    return pl, z.cuda(), val.cuda(), idx.cuda(), weight.cuda()


def _run(pl, z, val, idx, weight, V, T):
    """loss, stats, dz of the three calls, and that the fused one has the same bits."""
    import torch
    from paper_2010_13359_amd import layers
    M, N, ld = z.shape
    nan = lambda *s, dtype=torch.float32: torch.full(s, float("nan"), dtype=dtype, device="cuda")
    loss, stats, dz = nan(M, N), nan(M, N, 2), nan(M, N, ld, dtype=z.dtype)
    ws = layers.distill_workspace(pl, N, V, val.shape[2], z.dtype, ld=ld)
    if ws is not None:
        ws.fill_(0xFF)
    layers.distill_forward(pl, z, val, idx, weight, loss, stats, V, ws, temperature=T)
    layers.distill_backward(pl, z, val, idx, weight, stats, dz, V, temperature=T)
    loss2, dz2 = nan(M, N), nan(M, N, ld, dtype=z.dtype)
    layers.distill_fused(pl, z, val, idx, weight, loss2, dz2, V, ws, temperature=T)
    bits = lambda t: t.view(torch.int32 if t.element_size() == 4 else torch.int16)
    assert torch.equal(bits(loss), bits(loss2)) and torch.equal(bits(dz), bits(dz2))
    z2 = z.clone()                                 # in place
    layers.distill_fused(pl, z2, val, idx, weight, loss2, z2, V, ws, temperature=T)
    assert torch.equal(bits(z2), bits(dz)) and torch.equal(bits(loss), bits(loss2))
    z2.copy_(z)
    layers.distill_backward(pl, z2, val, idx, weight, stats, z2, V, temperature=T)
    assert torch.equal(bits(z2), bits(dz))
    return loss, stats, dz


def _compare(z, val, idx, weight, V, T, got):
    loss, stats, dz = got
    for m in range(z.shape[0]):
        w = ref.distill(z[m], val[m], idx[m], None if weight is None else weight[m], V, T)
        ref.check("largest", stats[m, :, 0], w["largest"], 0.0)
        ref.check("total", stats[m, :, 1], w["total"], w["total_err"])
        ref.check("loss", loss[m], w["loss"], w["loss_err"])
        ref.check("dz", dz[m], w["dz"], w["dz_err"])


@pytest.mark.parametrize("dt", sorted(ref.TYPES))
@pytest.mark.parametrize("shape", SHAPES)
def test_loss_and_gradient(shape, dt):
    V = shape[2]
    for T, spread in ((1.0, 3.0), (2.5, 8.0)):
        pl, z, val, idx, weight = _setup(shape, dt, seed=V, spread=spread)
        w = None if T == 2.5 else weight
        _compare(z, val, idx, w, V, T, _run(pl, z, val, idx, w, V, T))
        pl.close()


@pytest.mark.parametrize("dt,V", [("bf16", 65537), ("bf16", 98304), ("f16", 98305), ("bf16", 131072), ("f32", 40001),
                                  ("f32", 49152), ("f32", 49153), ("f32", 65533)])
def test_long_rows_of_many_tokens(dt, V):
    """Rows of half a CU's registers and more, enough of them for a workgroup each."""
    pl, z, val, idx, weight = _setup((1, 131, V, 1, 9), dt, seed=V)
    _compare(z, val, idx, weight, V, 1.0, _run(pl, z, val, idx, weight, V, 1.0))
    pl.close()


@pytest.mark.parametrize("dt", sorted(ref.TYPES))
@pytest.mark.parametrize("V", [40, 5000, 70001, 140000])
def test_tokens_that_take_no_part(V, dt):
    """Weight 0 (with NaN everywhere), no teacher entry, entries of -inf, no
    student logit; ordinary tokens between them."""
    import torch
    pl, z, val, idx, weight = _setup((2, 7, V, 3, 12), dt, seed=1)
    weight[:, 0] = 0.0
    z[:, 0] = float("nan")
    val[:, 0] = float("nan")
    idx[:, 2] = -1
    val[:, 3] = -math.inf
    z[:, 5, :V] = -math.inf
    loss, stats, dz = got = _run(pl, z, val, idx, weight, V, 2.0)
    for n in (0, 2, 3, 5):
        assert not loss[:, n].any() and not stats[:, n].any() and not dz[:, n].any()
    _compare(z, val, idx, weight, V, 2.0, got)
    assert bool((dz[..., V:] == 0).all())
    assert bool(dz[:, [1, 4, 6]].any(-1).all())
    pl.close()


@pytest.mark.parametrize("dt", sorted(ref.TYPES))
@pytest.mark.parametrize("V", [33, 4100, 66000, 132000])
def test_masked_logits(V, dt):
    """Logits of -inf and of the type's lowest value, alone or almost alone,
    where the teacher has mass and where it has none."""
    import torch
    lowest = torch.finfo(ref.TYPES[dt]).min
    pl, z, val, idx, weight = _setup((1, 6, V, 0, 5), dt, seed=2)
    idx[:] = torch.tensor([1, 4, 9, 20, 30], dtype=torch.int32)
    z[0, 0, 40 if V > 40 else 31:] = -math.inf      # a mask behind the teacher's entries
    z[0, 1] = -math.inf
    z[0, 1, 4] = 1.0                               # one logit left: the others' loss is infinite
    z[0, 2] = lowest                               # equal logits
    z[0, 3] = lowest
    z[0, 3, 9] = 0.5
    z[0, 4, ::2] = lowest
    z[0, 5] = -math.inf
    z[0, 5, V - 1] = -2.0
    loss, stats, dz = got = _run(pl, z, val, idx, weight, V, 1.0)
    assert math.isinf(float(loss[0, 1])) and math.isinf(float(loss[0, 5]))
    assert bool(torch.isfinite(dz).all())
    # the loss of tokens 3 and 4 goes with the lowest value itself; its bound with it
    _compare(z, val, idx, weight, V, 1.0, got)
    pl.close()


def test_repeated_entries():
    import torch
    V = 900
    pl, z, val, idx, weight = _setup((1, 3, V, 0, 200), "f32", seed=3)
    idx[0, 0] = 7                                  # one index for all
    idx[0, 1] = (torch.arange(200) // 2).int()     # in pairs
    idx[0, 2] = (torch.arange(200) % 50).int()     # apart
    _compare(z, val, idx, weight, V, 1.0, _run(pl, z, val, idx, weight, V, 1.0))
    pl.close()


@pytest.mark.parametrize("k", [2, 32, 33, 200, 1024])
@pytest.mark.parametrize("V", [3000, 140000])
def test_messages_in_any_order(V, k):
    """Distinct indices in no order, one pair of equal ones among them, skipped
    entries between, and indices close together or at steps of a Fibonacci number."""
    import torch
    pl, z, val, idx, weight = _setup((1, 5, V, 0, k), "bf16", seed=k)
    gen = torch.Generator().manual_seed(V + k)
    idx[0, 0] = torch.randperm(V, generator=gen)[:k].int()
    idx[0, 1] = idx[0, 0]
    idx[0, 1, 0] = idx[0, 1, k - 1]
    idx[0, 2] = idx[0, 0]
    idx[0, 2, ::3] = -1
    idx[0, 3] = (V - 1 - torch.arange(k)).int()
    idx[0, 4] = (torch.arange(k) * 2584 % V).flip(0).int()
    _compare(z, val, idx, weight, V, 1.0, _run(pl, z, val, idx, weight, V, 1.0))
    pl.close()


def test_nan_and_infinity_spread_over_their_token_only():
    import torch
    for V in (500, 70000, 140000):
        pl, z, val, idx, weight = _setup((1, 5, V, 0, 6), "bf16", seed=4)
        idx[:] = torch.arange(6, dtype=torch.int32)
        clean = [0, 2]
        z[0, 1, V // 2] = float("nan")
        z[0, 3, V - 1] = float("inf")
        val[0, 4, 2] = float("nan")
        loss, stats, dz = _run(pl, z, val, idx, weight, V, 1.0)
        assert bool(torch.isnan(loss[0, [1, 3, 4]]).all()) and bool(torch.isfinite(loss[0, clean]).all())
        assert bool(torch.isnan(dz[0, [1, 3]]).any(-1).all()) and bool(torch.isfinite(dz[0, clean]).all())
        assert bool(torch.isnan(dz[0, 4, :6]).all()) and bool(torch.isfinite(dz[0, 4, 6:]).all())
        w = ref.distill(z[0, clean], val[0, clean], idx[0, clean], weight[0, clean], V, 1.0)
        ref.check("dz", dz[0, clean], w["dz"], w["dz_err"])
        pl.close()


def test_a_student_that_is_its_teacher():
    """All logits sent, and the student's own: a loss of 0 up to its bound."""
    import torch
    V = 300
    pl, z, val, idx, weight = _setup((1, 4, V, 0, V), "f32", seed=5)
    idx[:] = torch.randperm(V, generator=torch.Generator().manual_seed(1)).int()
    val.copy_(z.gather(-1, idx.long()))
    got = _run(pl, z, val, idx, weight, V, 1.5)
    _compare(z, val, idx, weight, V, 1.5, got)
    pl.close()


def test_gradient_against_differences():
    """Central differences of the loss in 64 bits along one direction."""
    import torch
    V, T = 700, 1.3
    pl, z, val, idx, weight = _setup((1, 3, V, 0, 40), "f32", seed=6)
    _, _, dz = _run(pl, z, val, idx, weight, V, T)
    E = torch.randn(z.shape, generator=torch.Generator().manual_seed(9)).double()
    h = 2.0 ** -10
    lo, hi = (ref.distill(z[0].double().cpu() + s * E[0], val[0], idx[0], weight[0], V, T)["loss"].sum() for s in (-h, h))
    mine, size = (dz.double().cpu() * E).sum(), (dz.double().cpu() * E).abs().sum()
    # the softmax's third derivative along E is below 8 max|E|^3 / T^2 of weight and T
    third = 8 * float(E.abs().max()) ** 3 * float(weight.sum()) / T
    assert abs(float((hi - lo) / (2 * h) - mine)) <= h * h * third / 6 + 2e-5 * float(size)
    pl.close()


def _compare_closely(z, val, idx, weight, V, T, got):
    loss, stats, dz = got
    for m in range(z.shape[0]):
        w = ref.distill_close(z[m], val[m], idx[m], None if weight is None else weight[m], V, T)
        ref.check("largest", stats[m, :, 0], w["largest"], 0.0)
        ref.check("total", stats[m, :, 1], w["total"], w["total_err"])
        ref.check("loss", loss[m], w["loss"], w["loss_err"])
        ref.check_range("dz", dz[m], w["dz"], w["dz_err"])


@pytest.mark.parametrize("dt", sorted(ref.TYPES))
@pytest.mark.parametrize("shape", SHAPES)
def test_no_further_off_than_the_kernels_steps(shape, dt):
    V = shape[2]
    for T, spread in ((1.0, 3.0), (2.0, 12.0), (2.5, 8.0)):
        pl, z, val, idx, weight = _setup(shape, dt, seed=V + 1, spread=spread)
        _compare_closely(z, val, idx, weight, V, T, _run(pl, z, val, idx, weight, V, T))
        pl.close()


@pytest.mark.parametrize("V", [3, 200, 1001])
def test_small_probabilities_keep_their_digits(V):
    """Logits on a grid, so that their differences are exact: an exponential of 2^-100
    is off by 3 u in 32 bits, and would be by 40 u without the correction of its
    exponent's product."""
    import torch
    pl, z, val, idx, weight = _setup((1, 8, V, 0, 2), "f32", seed=7)
    gen = torch.Generator().manual_seed(V)
    z[..., :V] = -torch.randint(0, 80 * 256, (1, 8, V), generator=gen).cuda() / 256.0
    z[..., 0] = 0.0
    idx[..., 0], idx[..., 1] = 0, 1
    for T in (1.0, 0.5):
        _compare_closely(z * T, val, idx, weight, V, T, _run(pl, z * T, val, idx, weight, V, T))
    pl.close()
