"""The layer operators in 64 bits, and how far 32-bit arithmetic may be from
them: bounds built from the roundings on the way, u = 2^-24 each, and half a
step of the output's type at the end."""
import math

import torch

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def plan(d, M, **kw):
    from paper_2010_13359_amd import dqgan
    return dqgan.Plan(d, M, kw.pop("kind", "identity"), **kw)


def check(name, got, want, err):
    """|got - want| <= err (an absolute bound before the last rounding) and half
    a step of got's type; NaN and infinities where `want` has them."""
    t = got.dtype
    got, want = got.detach().double().cpu(), want.double().cpu()
    err = err.double().cpu() if isinstance(err, torch.Tensor) else err
    info = torch.finfo(t)
    half = info.eps / 2
    tiny = info.smallest_normal * half      # half a step of the subnormal range
    # a value that rounds beyond the largest one is an infinity of its sign
    over = torch.isfinite(want) & (want.abs() + err >= info.max * (1 + half))
    odd = ~torch.isfinite(want)
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    assert bool((same | ~odd | over).all()), "%s: infinities or NaN differ at %s" % (
        name, (odd & ~same).nonzero()[:3].tolist())
    bound = err + half * (want.abs() + err) + tiny
    off = (got - want).abs()
    bad = ~odd & ~over & ~(off <= bound)
    if bool(bad.any()):
        at = bad.nonzero()[0]
        i = tuple(at.tolist())
        b = bound[i] if isinstance(bound, torch.Tensor) else bound
        raise AssertionError("%s: %d of %d beyond the bound; first at %s: got %r, want %r, bound %r" % (
            name, int(bad.sum()), bad.numel(), i, float(got[i]), float(want[i]), float(b)))


def check_range(name, got, want, err):
    """check, with what lies beyond the type's range: a value is an infinity of its sign
    from half a step above the largest one on (a tie, whose even neighbour is the one that
    is not there); where `err` reaches across that edge, it is that infinity or finite.
    Returns how many have to be infinities."""
    info = torch.finfo(got.dtype)
    edge = info.max + 2.0 ** math.floor(math.log2(info.max)) * info.eps / 2
    got, want = got.detach().double().cpu(), want.double().cpu()
    err = err.double().cpu() if isinstance(err, torch.Tensor) else torch.full_like(want, err)
    infinite = torch.copysign(torch.full_like(want, math.inf), want)
    over = (want.abs() - err >= edge) | torch.isinf(want)
    near = (want.abs() + err >= edge) & ~over
    assert bool((got == infinite)[over].all()), "%s: not infinite" % name
    assert bool(torch.isnan(got[torch.isnan(want)]).all()), "%s: not NaN" % name
    half = info.eps / 2
    bound = err + half * (want.abs() + err) + info.smallest_normal * half
    good = ((got - want).abs() <= bound) | (near & (got == infinite)) | over | torch.isnan(want)
    assert bool(good.all()), "%s: beyond the bound at %s" % (name, (~good).nonzero()[:3].tolist())
    return int(over.sum())


def depth(D):
    """Additions on the way of one term into a row's sum: at most 8 per vector
    and lane, 6 across lanes, 16 across waves."""
    return 8 * max(4, math.ceil(D / 8192)) + 22


# ---------------------------------------------------------------------------


def embed_forward(tokens, table, scale):
    """[N] tokens, [V][D] table: (out, error)."""
    t, w = tokens.long().cpu(), table.double().cpu()
    there = (t >= 0) & (t < w.shape[0])
    s = float(torch.tensor(scale, dtype=torch.float32))
    out = w[torch.where(there, t, 0)] * s * there[:, None]
    return out, U * out.abs()


def embed_backward(tokens, dout, V, scale, before=None):
    t, g = tokens.long().cpu(), dout.double().cpu()
    s = float(torch.tensor(scale, dtype=torch.float32))
    keep = (t >= 0) & (t < V)
    total = torch.zeros((V, g.shape[1]), dtype=torch.float64)
    size, count = torch.zeros_like(total), torch.zeros(V, dtype=torch.float64)
    total.index_add_(0, t[keep], g[keep])
    size.index_add_(0, t[keep], g[keep].abs())
    count.index_add_(0, t[keep], torch.ones(int(keep.sum()), dtype=torch.float64))
    out, err = total * s, U * (count + 1)[:, None] * size * abs(s)
    if before is not None:
        out = out + before.double().cpu()
        err = torch.where(count[:, None] > 0, err + U * (out.abs() + err), 0.0)
    return out, err


def norm_forward(x, gamma, beta, eps):
    """[N][D]: (y, its error, mean, its error, rstd, its error)."""
    x = x.double().cpu()
    D = x.shape[1]
    k = depth(D)
    g = torch.ones(D, dtype=torch.float64) if gamma is None else gamma.double().cpu()
    b = torch.zeros(D, dtype=torch.float64) if beta is None else beta.double().cpu()
    e = float(torch.tensor(eps, dtype=torch.float32))
    mean = x.mean(1, keepdim=True)
    xc = x - mean
    var = (xc * xc).mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(var + e)
    mean_err = (k + 2) * U * x.abs().mean(1, keepdim=True)
    # the mean square about a mean that is off by mean_err; subtraction 2u, product and sums
    var_err = (k + 6) * U * (var + mean_err ** 2) + mean_err ** 2 + 2 * U * mean_err * var.sqrt()
    rstd_rel = var_err / (2 * (var + e - var_err).clamp(min=1e-300)) + 4 * U
    xh = xc * rstd
    y = xh * g + b
    y_err = g.abs() * ((xh.abs() + mean_err * rstd) * (rstd_rel + 3 * U) + mean_err * rstd) + U * y.abs()
    return y, y_err, mean[:, 0], mean_err[:, 0], rstd[:, 0], (rstd * rstd_rel)[:, 0]


def norm_forward_centred(x, gamma, beta, eps):
    """As norm_forward, with the bounds of a row whose mean m in binary32 (off by at
    most `off`) is corrected by the mean r of the f = x - m: f has one rounding, r
    those of its sum and two more, the variance mean(f^2) - r^2 those of both and one
    more, and y is taken from f and r in 32 bits."""
    x = x.double().cpu()
    D = x.shape[1]
    k = depth(D)
    g = torch.ones(D, dtype=torch.float64) if gamma is None else gamma.double().cpu()
    b = torch.zeros(D, dtype=torch.float64) if beta is None else beta.double().cpu()
    e = float(torch.tensor(eps, dtype=torch.float32))
    mean = x.mean(1, keepdim=True)
    xc = x - mean
    var = (xc * xc).mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(var + e)
    off = (k + 2) * U * x.abs().mean(1, keepdim=True)
    size = xc.abs() + off                               # of f
    r_err = (k + 4) * U * size.mean(1, keepdim=True)
    var_err = (k + 7) * U * (size * size).mean(1, keepdim=True) + 2 * off * r_err + r_err ** 2 + U * off ** 2
    rstd_rel = var_err / (2 * (var + e - var_err).clamp(min=1e-300)) + 4 * U
    xh = xc * rstd
    # f's rounding, r's error, the roundings of r * rstd and of the result; rstd's own
    xh_err = (rstd * (U * size + r_err + U * (off + r_err)) + 2 * U * xh.abs()) * (1 + rstd_rel) + xh.abs() * rstd_rel
    y = xh * g + b
    y_err = g.abs() * xh_err + U * (y.abs() + g.abs() * xh_err)
    return y, y_err, mean[:, 0], (r_err + U * (mean.abs() + r_err))[:, 0], rstd[:, 0], (rstd * rstd_rel)[:, 0]


def norm_backward(x, dy, gamma, stats):
    """[N][D], stats [N][2] as given: (dx, error, dgamma, error, dbeta, error)."""
    x, dy = x.double().cpu(), dy.double().cpu()
    N, D = x.shape
    mean, rstd = stats.double().cpu().split(1, 1)
    g = torch.ones(D, dtype=torch.float64) if gamma is None else gamma.double().cpu()
    xh, u = (x - mean) * rstd, dy * g
    c1, c2 = u.mean(1, keepdim=True), (u * xh).mean(1, keepdim=True)
    dx = rstd * (u - c1 - xh * c2)
    a1, a2 = u.abs().mean(1, keepdim=True), (u * xh).abs().mean(1, keepdim=True)
    err = rstd.abs() * (depth(D) + 8) * U * (u.abs() + a1 + xh.abs() * a2)
    dg, db = (dy * xh).sum(0), dy.sum(0)
    return dx, err, dg, (N + 4) * U * (dy * xh).abs().sum(0), db, (N + 1) * U * dy.abs().sum(0)


def distill(z, val, idx, weight, V, T):
    """[N][ld] logits, [N][k] message: dict of loss, stats, dz and their errors.

    An exponent x = (z - largest) / T is computed with three roundings of its
    own and one of its product with log2(e), whose constant is as exact: off by
    at most 5 u |x|; the exponential itself by 2 u.  So e is off by (5 |x| + 3)
    u, a sum of them by the mean of that and one u per addition; a sum that is
    rescaled when a larger logit appears is off by that of the rescaling
    factors too, whose exponents add up to the row's range."""
    z, val = z.double().cpu(), val.double().cpu()
    N, ld, k = z.shape[0], z.shape[1], val.shape[1]
    idx = idx.cpu().long() & 0xFFFFFFFF
    w = torch.ones(N, dtype=torch.float64) if weight is None else weight.double().cpu()
    out = {n: torch.zeros(N, dtype=torch.float64) for n in ("loss", "loss_err", "largest", "total", "total_err")}
    out["dz"] = torch.zeros((N, ld), dtype=torch.float64)
    out["dz_err"] = torch.zeros_like(out["dz"])
    for n in range(N):
        x = z[n, :V]
        use = (idx[n] < V) & ~(val[n] == -math.inf)
        nothing = bool((x == -math.inf).all())
        if w[n] == 0 or not bool(use.any()) or nothing:
            continue
        v, i = val[n][use], idx[n][use]
        # as maxima of numbers skip NaN here; it comes back through the sum
        most = torch.where(torch.isnan(x), -math.inf, x).max()
        top = torch.where(torch.isnan(v), -math.inf, v).max()
        ax = (x - most) / T
        e = ax.exp()
        total = e.sum()
        size = torch.where(e > 0, ax.abs(), 0.0)
        low = x[torch.isfinite(x)]
        reach = float((low.max() - low[low >= low.max() - 200 * T].min()) / T) if low.numel() else 0.0
        chunks = math.ceil(V / 1024)
        total_rel = U * (5 * float((e * size).sum() / total) + 3 + depth(V) + 5 * 2 * reach + 4 * chunks + 16)
        s = e / total
        s_err = s * (U * (5 * size + 6) + total_rel)
        av = (v - top) / T
        ev = av.exp()
        t = ev / ev.sum()
        ev_rel = U * (5 * torch.where(ev > 0, av.abs(), 0.0) + 3)
        sum_rel = float((ev_rel * ev).sum() / ev.sum()) + U * (k + 8)
        t_err = t * (ev_rel + sum_rel + 2 * U)
        logt = av - ev.sum().log()
        logs = (x[i] - most) / T - total.log()
        pos = t > 0
        term = torch.where(pos, t * (logt - logs), 0.0)
        logt_err = 4 * U * av.abs() + sum_rel + 3 * U * (ev.sum().log().abs() + logt.abs())
        logs_err = 4 * U * ((x[i] - most) / T).abs() + total_rel + 3 * U * (total.log().abs() + logs.abs())
        term_err = torch.where(pos, t_err * (logt - logs).abs() + t * (logt_err + logs_err)
                               + (k + 8) * U * term.abs() + U * t * (logt.abs() + logs.abs()), 0.0)
        out["loss"][n] = w[n] * T * T * term.sum()
        out["loss_err"][n] = w[n].abs() * T * T * (term_err.sum() + 4 * U * term.abs().sum())
        out["largest"][n], out["total"][n], out["total_err"][n] = most, total, total * total_rel
        g, g_err = s.clone(), s_err.clone()
        g.index_add_(0, i, -t)
        g_err.index_add_(0, i, t_err + k * U * t)
        out["dz"][n, :V] = w[n] * T * g
        out["dz_err"][n, :V] = w[n].abs() * T * (g_err + 4 * U * (s + (s - g).abs()))
    return out


def _additions(V, size):
    """Additions on the way of one exponential into its row's sum: a lane's vectors in
    registers and LDS, one single element, 6 across a wave and up to 4 across waves;
    and of a row in slices, those of a slice, then the slices of a lane and 8 more."""
    per, bytes_ = 16 // size, V * size
    for most, vectors in ((4096, 1), (8192, 2), (16384, 4), (32768, 8), (65536, 16), (131072, 16), (196608, 12), (261120, 16)):
        if bytes_ <= most:
            row = per * vectors + 1 + 6 + 4
            break
    else:
        row = 0
    slices = per * 4 + 1 + 6 + 2 + math.ceil(math.ceil(bytes_ / 16384) / 256) + 8
    return max(row, slices)


def distill_close(z, val, idx, weight, V, T):
    """As distill, with what the kernels' own steps may be off by and no more.

    x = (z - largest) / T: the difference's own rounding, taken as it is, and, if T is
    no power of two, two more.  exp(x) of 32-bit logits: 2 u of the exponential and one
    rounding (the product with log2(e) is corrected); of 16-bit ones u |x| each for
    log2(e) / T and the product, and 2 u.  A row in slices has one more exponential and a
    product for each slice."""
    dtype, size = z.dtype, z.element_size()
    fine = dtype == torch.float32
    z, val = z.detach().cpu(), val.detach().cpu()
    N, ld, k = z.shape[0], z.shape[1], val.shape[1]
    idx = idx.cpu().long() & 0xFFFFFFFF
    w = torch.ones(N, dtype=torch.float64) if weight is None else weight.double().cpu()
    inv = 0.0 if math.frexp(T)[0] == 0.5 else 2 * U
    adds, adds_k = _additions(V, size), math.ceil(k / 256) + 10
    out = {n: torch.zeros(N, dtype=torch.float64) for n in ("loss", "loss_err", "largest", "total", "total_err")}
    out["dz"], out["dz_err"] = (torch.zeros((N, ld), dtype=torch.float64) for _ in range(2))

    def exponent(a, top):
        """(a - top) / T and its error."""
        d32 = (a.float() - top.float()).double()
        d = a.double() - top.double()
        return d / T, (d32 - d).abs() / T + inv * d.abs() / T
    for n in range(N):
        use = (idx[n] < V) & ~(val[n] == -math.inf)
        if w[n] == 0 or not bool(use.any()):
            continue
        v, i = val[n][use], idx[n][use]
        top = z[n, :V].max()
        x, x_err = exponent(z[n, :V], top)
        e = x.exp()
        total = e.sum()
        e_rel = x_err + (3 * U if fine else 2 * U * (1 + x.abs()))
        slice_rel = (U * 3 if fine else U * (2 + 2 * float(x.abs().max()))) + U if V * size > 131072 else 0.0
        total_rel = float((e_rel * e).sum() / total) + slice_rel + adds * U
        s = e / total
        s_err = s * (e_rel + total_rel + 2 * U)
        av, av_err = exponent(v, v.max())
        ev = av.exp()
        sum_v = ev.sum()
        t = ev / sum_v
        sum_rel = float(((av_err + 2 * U) * t).sum()) + adds_k * U
        t_err = t * (av_err + 3 * U + sum_rel)
        logt = av - sum_v.log()
        logs = x[i] - total.log()
        gap = (logt - logs).abs()
        logt_err = av_err + sum_rel + 2 * U * sum_v.log().abs() + U * logt.abs()
        logs_err = x_err[i] + total_rel + 2 * U * total.log().abs() + U * logs.abs()
        term = t * (logt - logs)
        term_err = t_err * gap + t * (logt_err + logs_err + U * gap)
        out["loss"][n] = w[n] * T * T * term.sum()
        out["loss_err"][n] = w[n].abs() * T * T * (term_err.sum() + (adds_k + 3) * U * term.abs().sum()) * 1.001
        out["largest"][n], out["total"][n], out["total_err"][n] = top, total, total * total_rel * 1.001
        times = torch.bincount(i, minlength=V).double()
        g, g_err = s.clone(), s_err.clone()
        g.index_add_(0, i, -t)
        g_err.index_add_(0, i, t_err + U * t * times[i])
        g_err += torch.where(times > 0, U * g.abs(), 0.0)
        out["dz"][n, :V] = w[n] * T * g
        out["dz_err"][n, :V] = w[n].abs() * T * (g_err + 2 * U * g.abs()) * 1.001
    return out
