"""The layer operators: what the M workers of a language-model run call between
an evaluation point and the gradient that the compressor takes, over the range
of sizes, types and directions they serve.

A case names an operator (`op`):
  embed_fwd   rows of every worker's own embedding table (in its row of the
              evaluation points) looked up by its tokens and scaled;
  embed_bwd   the table's gradient, summed over sorted tokens into the worker's
              row of the gradients.  `sides` = 2: a source and a target side
              share one table, so a second call adds to the first one's result;
  norm_fwd    layer norm with the worker's own weight and bias;
  norm_bwd    its gradients: of the input, and of weight and bias into the
              worker's row of the gradients;
  distill_loss  the loss of student logits against a teacher's top logits,
              which come as a top-k message (values and indices per token);
  distill_bwd   its gradient from the statistics that the loss left;
  distill_both  loss and gradient in one call.
Sizes: M workers of N tokens each, V vocabulary entries, D channels, K logits
of the teacher per token; `off` is the place of the parameters in a worker's
row, `pad` what a row of logits has beyond V; activations and logits are of
type `dt`, parameters and their gradients in 32 bits.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5
SKIP = -1        # token of a padded place; as an index of the teacher: no entry


def listed():
    return [
        # one token for each of eight workers: a launch
        dict(name="embed_fwd_token", op="embed_fwd", dt="bf16", M=8, N=1, V=32000, D=512, off=0, sides=1),
        # a long batch: gathers of 4 KB rows from tables of 200 MB
        dict(name="embed_fwd_batch", op="embed_fwd", dt="bf16", M=8, N=8192, V=50304, D=1024, off=1024, sides=1),
        # an ordinary batch: the dense row of the gradients has to be written whole, mostly zeros
        dict(name="embed_bwd_batch", op="embed_bwd", dt="bf16", M=8, N=4096, V=32000, D=1024, off=0, sides=1),
        # one worker process, a long batch with much repetition, odd sizes, two sides that share the table
        dict(name="embed_bwd_shared", op="embed_bwd", dt="f16", M=1, N=65536, V=20011, D=1025, off=513, sides=2),
        # one token for each of four workers
        dict(name="norm_fwd_token", op="norm_fwd", dt="f32", M=4, N=1, D=512, off=0),
        # a long batch
        dict(name="norm_fwd_batch", op="norm_fwd", dt="bf16", M=8, N=8192, D=2048, off=1024),
        # an ordinary batch, backward
        dict(name="norm_bwd_batch", op="norm_bwd", dt="bf16", M=8, N=2048, D=1024, off=0),
        # odd sizes and wide rows, backward
        dict(name="norm_bwd_odd", op="norm_bwd", dt="f16", M=3, N=1111, D=4801, off=77),
        # one token scored against the teacher, in 32 bits
        dict(name="distill_loss_token", op="distill_loss", dt="f32", M=1, N=1, V=32000, K=32, pad=0, temp=1.0),
        # a gradient taken later than its loss, odd vocabulary with a padded row
        dict(name="distill_bwd_odd", op="distill_bwd", dt="f16", M=4, N=777, V=30011, K=20, pad=53, temp=2.0),
        # an ordinary training batch
        dict(name="distill_both_batch", op="distill_both", dt="bf16", M=8, N=512, V=32000, K=64, pad=0, temp=2.0),
        # the largest vocabulary
        dict(name="distill_both_large", op="distill_both", dt="bf16", M=4, N=2048, V=128000, K=128, pad=0, temp=1.0),
    ]


def _log(rng, a, b):
    return max(a, min(b, int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))))


def draw(rng):
    op = rng.choice(["embed_fwd", "embed_bwd", "norm_fwd", "norm_bwd", "distill_loss", "distill_bwd", "distill_both"])
    dt, M = rng.choice(list(TYPES)), _log(rng, 1, 32)
    size = 4 if dt == "f32" else 2
    if op.startswith("embed"):
        V, D = _log(rng, 64, 150000), _log(rng, 32, 4096) | rng.choice([0, 0, 1])
        M = max(1, min(M, int(2.5e9 / (4 * V * D))))
        N = min(_log(rng, 1, 65536), int(1e9 / (M * D * size)))
        return dict(op=op, dt=dt, M=M, N=N, V=V, D=D, off=rng.choice([0, 1024, 513]),
                    sides=rng.choice([1, 1, 2]) if op == "embed_bwd" else 1)
    if op.startswith("norm"):
        D = _log(rng, 32, 16384) | rng.choice([0, 0, 1])
        N = min(_log(rng, 1, 16384), int(1.2e9 / (M * D * size)))
        return dict(op=op, dt=dt, M=M, N=N, D=D, off=rng.choice([0, 1024, 77]))
    V = _log(rng, 1000, 160000)
    N = max(1, min(_log(rng, 1, 4096), int(1.5e9 / (M * V * size))))
    return dict(op=op, dt=dt, M=M, N=N, V=V, K=_log(rng, 4, 256), pad=rng.choice([0, 0, 1, 64]),
                temp=rng.choice([1.0, 2.0, 4.0]))


# ---------------------------------------------------------------------------
# inputs


def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * seed + salt)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _d(case):
    """Parameters of a worker that the case needs."""
    if "off" not in case:
        return 1024
    return case["off"] + (case["V"] * case["D"] if case["op"].startswith("embed") else 2 * case["D"])


def _rows(case):
    """[M][ld] parameters, as the step leaves its evaluation points."""
    return torch.empty((case["M"], (_d(case) + 1023) // 1024 * 1024), dtype=torch.float32, device="cuda")


def _tokens(case, seed, side):
    """Tokens by falling frequency (the v-th about 1 / v as often as the first),
    one place in twenty a padded one."""
    g, shape = _gen(seed, 10 + side), (case["M"], case["N"])
    u = torch.rand(shape, generator=g, device="cuda", dtype=torch.float64)
    t = torch.exp(u * math.log(case["V"] + 1)).long() - 1
    t.clamp_(0, case["V"] - 1)
    t[torch.rand(shape, generator=g, device="cuda") < 0.05] = SKIP
    return t


def _logits(case, seed):
    """Student logits, the teacher's message (its K largest logits, near the
    student's own, some tokens with fewer) and the weight of each token."""
    M, N, V, K, ld = case["M"], case["N"], case["V"], case["K"], case["V"] + case["pad"]
    g = _gen(seed, 20)
    z = torch.empty((M, N, ld), dtype=TYPES[case["dt"]], device="cuda")
    val = torch.empty((M, N, K), dtype=torch.float32, device="cuda")
    idx = torch.empty((M, N, K), dtype=torch.int32, device="cuda")
    part = max(1, int(1e8 / ld))
    zf, vf, xf = z.view(M * N, ld), val.view(M * N, K), idx.view(M * N, K)
    for a in range(0, M * N, part):
        x = _randn(g, min(part, M * N - a), ld).mul_(2.5)
        zf[a:a + part] = x
        top = torch.topk(x[:, :V].add_(_randn(g, x.shape[0], V)), K)
        order = top.indices.sort(dim=1)
        xf[a:a + part] = order.values.int()
        vf[a:a + part] = top.values.gather(1, order.indices).add_(3.0)
    fewer = torch.rand((M, N, 1), generator=g, device="cuda") < 0.1
    cut = torch.rand((M, N, 1), generator=g, device="cuda") * K
    idx[fewer & (torch.arange(K, device="cuda") > cut)] = SKIP
    # the mean over a worker's tokens, or, where the gradient's type has a short range, a loss scale
    weight = torch.rand((M, N), generator=g, device="cuda").add_(0.5).mul_(1024.0 if case["dt"] == "f16" else 1.0 / N)
    if N > 1:  # tokens that take no part: prompts, padded places
        weight[torch.rand((M, N), generator=g, device="cuda") < 0.05] = 0.0
    return z, val, idx, weight


def _inputs(case, seed):
    op, dt, s = case["op"], TYPES[case["dt"]], {}
    if op.startswith("embed"):
        s["tokens"] = [_tokens(case, seed, i) for i in range(case["sides"])]
        if op == "embed_fwd":
            s["P"] = _rows(case).normal_(0.0, 0.02, generator=_gen(seed, 1))
        else:
            s["dout"] = [_randn(_gen(seed, 2 + i), case["M"], case["N"], case["D"]).mul_(1e-3).to(dt)
                         for i in range(case["sides"])]
    elif op.startswith("norm"):
        g = _gen(seed, 4)
        s["P"] = _rows(case).normal_(0.0, 0.1, generator=g)
        s["P"][:, case["off"]:case["off"] + case["D"]] += 1.0
        x = _randn(g, case["M"], case["N"], case["D"])
        s["x"] = x.mul_(_randn(g, case["M"], case["N"], 1).exp_()).add_(_randn(g, case["M"], case["N"], 1)).to(dt)
        if op == "norm_bwd":
            s["dy"] = _randn(g, case["M"], case["N"], case["D"]).mul_(1e-3).to(dt)
            # what the forward pass left
            x = s["x"].float()
            mean = x.mean(-1)
            var = (x - mean[..., None]).square_().mean(-1)
            s["stats"] = torch.stack([mean, torch.rsqrt(var + EPS)], -1)
    else:
        s["z"], s["val"], s["idx"], s["weight"] = _logits(case, seed)
        if op == "distill_bwd":  # what the loss left: the row's maximum and its sum of exponentials
            zf = s["z"][..., :case["V"]]
            most = zf.amax(-1).float()
            total = torch.stack([((r.float() - m[:, None]) * (1.0 / case["temp"])).exp_().sum(-1)
                                 for r, m in zip(zf, most)])
            s["stats"] = torch.stack([most, total], -1)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s.update(case=case, scale=math.sqrt(case["D"]) if case["op"].startswith("embed") else 1.0)
    if own:
        from paper_2010_13359_amd import dqgan, layers
        op, M, N, dt = case["op"], case["M"], case["N"], TYPES[case["dt"]]
        new = lambda *shape, dtype=dt: torch.empty(shape, dtype=dtype, device="cuda")
        s["plan"] = plan = dqgan.Plan(_d(case), M, "identity")
        if op == "embed_fwd":
            s["out"] = new(M, N, case["D"])
        elif op == "embed_bwd":
            s["G"] = _rows(case).zero_()
            s["ws"] = layers.embed_workspace(plan, N, case["V"], case["D"], dt, torch.int64, offset=case["off"])
        elif op == "norm_fwd":
            s["y"], s["stats"] = new(M, N, case["D"]), new(M, N, 2, dtype=torch.float32)
        elif op == "norm_bwd":
            s["dx"], s["G"] = new(M, N, case["D"]), _rows(case).zero_()
            s["ws"] = layers.norm_workspace(plan, N, case["D"], dt, gamma=case["off"], beta=case["off"] + case["D"])
        else:
            s["ws"] = layers.distill_workspace(plan, N, case["V"], case["K"], dt, ld=case["V"] + case["pad"])
            s["loss"] = new(M, N, dtype=torch.float32)
            s["dz"] = new(M, N, case["V"] + case["pad"]) if op != "distill_loss" else None
            if op != "distill_bwd":
                s["stats"] = new(M, N, 2, dtype=torch.float32)
    return s


# ---------------------------------------------------------------------------
# one pass


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2010_13359_amd import layers
    c = s["case"]
    op, plan = c["op"], s["plan"]
    if op == "embed_fwd":
        layers.embed_forward(plan, s["tokens"][0], s["P"], s["out"], c["V"], offset=c["off"], scale=s["scale"])
        return {"out": s["out"]}
    if op == "embed_bwd":
        for i, (t, g) in enumerate(zip(s["tokens"], s["dout"])):
            layers.embed_backward(plan, t, g, s["G"], c["V"], s["ws"], offset=c["off"], scale=s["scale"], add=i > 0)
        return {"G": s["G"][:, c["off"]:_d(c)]}
    if op.startswith("norm"):
        where = dict(gamma=c["off"], beta=c["off"] + c["D"])
        if op == "norm_fwd":
            layers.norm_forward(plan, s["x"], s["P"], s["y"], s["stats"], eps=EPS, **where)
            return {"y": s["y"], "stats": s["stats"]}
        layers.norm_backward(plan, s["x"], s["dy"], s["P"], s["stats"], s["dx"], s["G"], s["ws"], **where)
        return {"dx": s["dx"], "G": s["G"][:, c["off"]:_d(c)]}
    teacher = (s["val"], s["idx"], s["weight"])
    if op == "distill_loss":
        layers.distill_forward(plan, s["z"], *teacher, s["loss"], s["stats"], c["V"], s["ws"], temperature=c["temp"])
        return {"loss": s["loss"], "stats": s["stats"]}
    if op == "distill_bwd":
        layers.distill_backward(plan, s["z"], *teacher, s["stats"], s["dz"], c["V"], temperature=c["temp"])
        return {"dz": s["dz"]}
    layers.distill_fused(plan, s["z"], *teacher, s["loss"], s["dz"], c["V"], s["ws"], temperature=c["temp"])
    return {"loss": s["loss"], "dz": s["dz"]}


def _run_plain(s):
    c = s["case"]
    op, M, dt = c["op"], c["M"], TYPES[c["dt"]]
    if op == "embed_fwd":
        t = s["tokens"][0]
        table = s["P"][:, c["off"]:_d(c)].unflatten(1, (c["V"], c["D"]))
        rows = table[torch.arange(M, device="cuda")[:, None], t.clamp(min=0)] * s["scale"]
        return {"out": (rows * (t >= 0)[..., None]).to(dt)}
    if op == "embed_bwd":
        t, g = torch.cat(s["tokens"], 1), torch.cat(s["dout"], 1).float() * s["scale"]
        at = torch.arange(M, device="cuda")[:, None] * c["V"] + t
        at = torch.where(t >= 0, at, M * c["V"])     # padded places add to a row of no use
        G = torch.zeros((M * c["V"] + 1, c["D"]), dtype=torch.float32, device="cuda")
        G.index_add_(0, at.view(-1), g.view(-1, c["D"]))
        return {"G": G[:-1].view(M, -1)}
    if op.startswith("norm"):
        gamma = s["P"][:, None, c["off"]:c["off"] + c["D"]]
        beta = s["P"][:, None, c["off"] + c["D"]:_d(c)]
        x = s["x"].float()
        if op == "norm_fwd":
            mean = x.mean(-1, keepdim=True)
            xc = x - mean
            rstd = torch.rsqrt((xc * xc).mean(-1, keepdim=True) + EPS)
            return {"y": (xc * rstd * gamma + beta).to(dt), "stats": torch.cat([mean, rstd], -1)}
        mean, rstd = s["stats"][..., :1], s["stats"][..., 1:]
        dy, xh = s["dy"].float(), (x - mean) * rstd
        w = dy * gamma
        dx = rstd * (w - w.mean(-1, keepdim=True) - xh * (w * xh).mean(-1, keepdim=True))
        return {"dx": dx.to(dt), "G": torch.cat([(dy * xh).sum(1), dy.sum(1)], -1)}
    # the teacher's distribution over the entries it sent
    T, V, have = c["temp"], c["V"], s["idx"] >= 0
    v = torch.where(have, s["val"], -math.inf) / T
    v = v - v.amax(-1, keepdim=True)
    t = v.exp()
    t = t / t.sum(-1, keepdim=True)
    logt = torch.where(have, v - v.exp().sum(-1, keepdim=True).log(), 0.0)
    at = torch.where(have, s["idx"], 0).long()
    z, weight = s["z"][..., :V].float(), s["weight"][..., None]
    if op == "distill_bwd":
        most, total = s["stats"][..., :1], s["stats"][..., 1:]
        e = ((z - most) / T).exp()
    else:
        most = z.amax(-1, keepdim=True)
        e = ((z - most) / T).exp()
        total = e.sum(-1, keepdim=True)
    out = {}
    if op != "distill_bwd":
        logs = (z.gather(-1, at) - most) / T - total.log()
        out["loss"] = T * T * s["weight"] * (t * (logt - logs)).sum(-1)
        if op == "distill_loss":
            # zeros of a token that takes no part
            out["stats"] = torch.where(weight == 0, 0.0, torch.cat([most, total], -1))
            return out
    dz = torch.zeros(s["z"].shape, dtype=torch.float32, device="cuda")
    dz[..., :V] = e / total
    dz.scatter_add_(-1, at, -t)
    out["dz"] = (dz * (T * weight)).to(dt)
    return out


# ---------------------------------------------------------------------------
# what a pass cannot do without


def _distinct(case):
    """Tokens of a worker's batch that differ, on the average."""
    v = np.arange(case["V"], dtype=np.float64)
    p = 0.95 * np.log((v + 2) / (v + 1)) / math.log(case["V"] + 1)
    return float(-np.expm1(case["N"] * np.log1p(-p)).sum())


def work(case):
    op, M, N = case["op"], case["M"], case["N"]
    size = 4 if case["dt"] == "f32" else 2
    if op.startswith("embed"):
        V, D, n = case["V"], case["D"], M * N * case["sides"]
        if op == "embed_fwd":
            return {"bytes": 8.0 * n + n * D * size + 4.0 * M * _distinct(case) * D, "flops": 1.0 * n * D}
        return {"bytes": 8.0 * n + n * D * size + 4.0 * M * V * D, "flops": 2.0 * n * D}
    if op.startswith("norm"):
        n, D = M * N, case["D"]
        if op == "norm_fwd":
            return {"bytes": 2.0 * n * D * size + 8.0 * M * D + 8.0 * n, "flops": 8.0 * n * D}
        return {"bytes": 3.0 * n * D * size + 12.0 * M * D + 8.0 * n, "flops": 14.0 * n * D}
    n, V, K = M * N, case["V"], case["K"]
    small = 8.0 * n * K + 16.0 * n
    if op == "distill_loss":
        return {"bytes": n * V * size + small, "flops": 4.0 * n * V}
    return {"bytes": n * V * size + n * (V + case["pad"]) * size + small,
            "flops": (4.0 if op == "distill_bwd" else 7.0) * n * V}


# ---------------------------------------------------------------------------
# the definitions in 64 bits


def _exact_embed(case, s):
    scale, V, D = math.sqrt(case["D"]), case["V"], case["D"]
    out = []
    for m in range(case["M"]):
        if case["op"] == "embed_fwd":
            t = s["tokens"][0][m]
            rows = s["P"][m, case["off"]:_d(case)].view(V, D)[t.clamp(min=0)].double() * scale
            rows[t < 0] = 0.0
            out.append(rows)
            continue
        total = torch.zeros((V, D), dtype=torch.float64, device="cuda")
        for t, g in zip(s["tokens"], s["dout"]):
            keep = t[m] >= 0
            total.index_put_((t[m][keep],), g[m][keep].double() * scale, accumulate=True)
        out.append(total.view(-1))
    return {"out" if case["op"] == "embed_fwd" else "G": torch.stack(out)}


def _exact_norm(case, s):
    D, ys, stats, dxs, Gs = case["D"], [], [], [], []
    for m in range(case["M"]):
        gamma, beta = s["P"][m, case["off"]:_d(case)].double().view(2, D)
        x = s["x"][m].double()
        if case["op"] == "norm_fwd":
            var, mean = torch.var_mean(x, -1, correction=0)
            rstd = 1.0 / torch.sqrt(var + EPS)
            ys.append((x - mean[:, None]) * rstd[:, None] * gamma + beta)
            stats.append(torch.stack([mean, rstd], -1))
            continue
        mean, rstd = s["stats"][m].double().unsqueeze(-1).unbind(1)
        xh, dy = (x - mean) * rstd, s["dy"][m].double()
        w = dy * gamma
        dxs.append((w - w.sum(-1, keepdim=True) / D - xh * ((w * xh).sum(-1, keepdim=True) / D)) * rstd)
        Gs.append(torch.cat([(dy * xh).sum(0), dy.sum(0)]))
    if case["op"] == "norm_fwd":
        return {"y": torch.stack(ys), "stats": torch.stack(stats)}
    return {"dx": torch.stack(dxs), "G": torch.stack(Gs)}


def _exact_distill(case, s):
    M, N, V, T, op = case["M"], case["N"], case["V"], case["temp"], case["op"]
    loss = torch.zeros((M, N), dtype=torch.float64, device="cuda")
    stats = torch.zeros((M, N, 2), dtype=torch.float64, device="cuda")
    dz = torch.zeros(s["z"].shape, dtype=torch.float64, device="cuda") if op != "distill_loss" else None
    part = max(1, int(2e8 / V))
    for m in range(M):
        for a in range(0, N, part):
            b = min(N, a + part)
            z = s["z"][m, a:b, :V].double()
            w = s["weight"][m, a:b].double()[:, None]
            idx = s["idx"][m, a:b].long()
            v = (s["val"][m, a:b].double() / T).masked_fill(idx < 0, -math.inf)
            logt = torch.log_softmax(v, -1)
            t = logt.exp()
            if op == "distill_bwd":
                most, total = s["stats"][m, a:b].double().unsqueeze(-1).unbind(1)
            else:
                most = z.max(-1, keepdim=True).values
                total = ((z - most) / T).exp().sum(-1, keepdim=True)
            stats[m, a:b] = torch.where(w == 0, 0.0, torch.cat([most, total], -1))
            logs = (z - most) / T - total.log()
            terms = t * (logt - logs.gather(1, idx.clamp(min=0)))
            loss[m, a:b] = T * T * (w * terms.masked_fill(idx < 0, 0.0)).sum(-1)
            if dz is not None:
                s_t = logs.exp_()
                row = torch.arange(b - a, device="cuda")[:, None].expand_as(idx)
                s_t.index_put_((row[idx >= 0], idx[idx >= 0]), -t[idx >= 0], accumulate=True)
                dz[m, a:b, :V] = T * w * s_t
    return {"distill_loss": {"loss": loss, "stats": stats}, "distill_bwd": {"dz": dz},
            "distill_both": {"loss": loss, "dz": dz}}[op]


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"].startswith("embed"):
        return _exact_embed(case, s)
    if case["op"].startswith("norm"):
        return _exact_norm(case, s)
    return _exact_distill(case, s)
