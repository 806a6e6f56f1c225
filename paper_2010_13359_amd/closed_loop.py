"""Closed-loop drivers on one GPU: Algorithm 2 (arXiv:2010.13359) with the
gradients of every worker taken at its own evaluation point.

The first is the bilinear game min_x max_y x^T A y, the textbook min-max
problem on which plain gradient steps cycle outward (Section 2.2) while the
optimistic method converges.

Each worker m evaluates a noisy gradient F(w^{(m)}_{t-1/2}) + xi at its own
evaluation point -- the WX row the previous iteration produced -- with
F(x, y) = (A y, -A^T x) (the game's operator, the role of the GAN's
gradients); the library then runs the iteration (EF accumulate, compress,
aggregate, OMD update, next evaluation points).  The gradient oracle is a
torch matmul: it is the input of the compression path, not part of it.

The second is a language-model student with tied embeddings that M workers
distil from a teacher's top logits, each from its own tokens: its layers are the
library's (``layers``), their parameter gradients go straight into the rows of
G, and the two matrix products are torch's.
"""
import torch

from . import dqgan, layers


class BilinearGame:
    def __init__(self, n, seed=0, device="cuda"):
        self.n, self.d = n, 2 * n
        gen = torch.Generator(device="cpu").manual_seed(seed)
        self.A = (torch.randn(n, n, generator=gen) / n ** 0.5).to(device)

    def operator(self, Z):
        """F applied to every row of Z ([rows][>= 2n]); returns [rows][2n]."""
        x, y = Z[:, :self.n], Z[:, self.n:self.d]
        return torch.cat([y @ self.A.T, -(x @ self.A)], dim=1)


def run_bilinear(kind, n=512, M=4, T=800, eta=0.2, noise=0.05, seed=0, record_every=100, on_step=None,
                 **plan_kwargs):
    """Run T iterations; returns the list of ||w_t|| / ||w_0|| every
    `record_every` iterations.  `on_step(t, state)` (optional) is called
    before iteration t with the device state (G, E, W) of that iteration."""
    dev = torch.device("cuda")
    game = BilinearGame(n, seed, dev)
    plan = dqgan.Plan(game.d, M, kind, seed=seed + 1, **plan_kwargs)
    ld = plan.ld
    gen = torch.Generator(device=dev).manual_seed(seed + 2)
    W = torch.zeros(ld, device=dev)
    W[:game.d] = torch.randn(game.d, device=dev, generator=gen)
    E = torch.zeros(M, ld, device=dev)
    WX = torch.zeros(M, ld, device=dev)
    G = torch.zeros(M, ld, device=dev)
    wire = plan.new_wire(dev)
    n0 = float(torch.linalg.vector_norm(W[:game.d]))
    # w_{-1/2} = w_0 and e_0 = 0: the first evaluation points are
    # w_0 - (eta g_0 + e_0), the library's OMD step with q-hat = 0 (w stays w_0)
    G[:, :game.d] = game.operator(W[:game.d].expand(M, -1)) + noise * torch.randn(M, game.d, device=dev,
                                                                                   generator=gen)
    Q0 = torch.zeros(ld, device=dev)
    dqgan.omd_step(plan, eta, Q0, W, G, E, WX)
    del Q0
    hist = []
    for t in range(1, T + 1):
        G[:, :game.d] = game.operator(WX) + noise * torch.randn(M, game.d, device=dev, generator=gen)
        if on_step is not None:
            on_step(t, {"G": G, "E": E, "W": W, "plan": plan, "wire": wire, "WX": WX})
        dqgan.step_fused(plan, eta, t, G, E, W, WX, wire)
        if t % record_every == 0:
            hist.append(float(torch.linalg.vector_norm(W[:game.d])) / n0)
    plan.close()
    return hist


def run_gradient_descent(n=512, T=800, eta=0.2, seed=0):
    """Plain simultaneous gradient steps on the same game (no extrapolation,
    no compression): ||z_T|| / ||z_0||."""
    dev = torch.device("cuda")
    game = BilinearGame(n, seed, dev)
    gen = torch.Generator(device=dev).manual_seed(seed + 2)
    z = torch.randn(1, game.d, device=dev, generator=gen)
    n0 = float(torch.linalg.vector_norm(z))
    for _ in range(T):
        z = z - eta * game.operator(z)
    return float(torch.linalg.vector_norm(z)) / n0


class Student:
    """Logits y E^T of y = norm(scale * E[token]) for the M workers of `plan`,
    each with its own table E ([vocab][width]), weight and bias, which lie in
    this order in a row of parameters, and the gradients of its distillation
    loss.  Holds the activations and workspaces of calls with `tokens` tokens
    per worker."""

    def __init__(self, plan, vocab, width, tokens, k, temperature=1.0, dtype=torch.float32):
        self.plan, self.vocab, self.width, self.temperature = plan, vocab, width, temperature
        self.scale = width ** 0.5
        self.where = dict(gamma=vocab * width, beta=vocab * width + width)
        dev = torch.device("cuda", plan.device)
        new = lambda *shape, dtype=dtype: torch.empty((plan.M, tokens) + shape, dtype=dtype, device=dev)
        self.x, self.y, self.dx = new(width), new(width), new(width)
        self.z = new(vocab)                       # the logits, then their gradient
        self.stats, self.loss = new(2, dtype=torch.float32), new(dtype=torch.float32)
        self.embed_ws = layers.embed_workspace(plan, tokens, vocab, width, dtype)
        self.norm_ws = layers.norm_workspace(plan, tokens, width, dtype, **self.where)
        self.distill_ws = layers.distill_workspace(plan, tokens, vocab, k, dtype)

    @staticmethod
    def parameters(vocab, width):
        """Parameters of a worker, and the offsets of its layers."""
        return vocab * width + 2 * width, [0, vocab * width, vocab * width + width, vocab * width + 2 * width]

    def table(self, P, m):
        return P[m, :self.vocab * self.width].view(self.vocab, self.width)

    def forward(self, P, tokens):
        """The logits [M][tokens][vocab] at the rows of P."""
        layers.embed_forward(self.plan, tokens, P, self.x, self.vocab, scale=self.scale)
        layers.norm_forward(self.plan, self.x, P, self.y, self.stats, **self.where)
        for m in range(self.plan.M):
            torch.mm(self.y[m], self.table(P, m).t().to(self.y.dtype), out=self.z[m])
        return self.z

    def gradients(self, P, tokens, val, idx, weight, G):
        """The gradients at the rows of P into the rows of G; returns the loss
        of every token."""
        plan, M = self.plan, self.plan.M
        self.forward(P, tokens)
        layers.distill_fused(plan, self.z, val, idx, weight, self.loss, self.z, self.vocab, self.distill_ws,
                             temperature=self.temperature)
        for m in range(M):  # the table as output layer, then (below, added) as embedding
            self.table(G, m).copy_(self.z[m].t().float() @ self.y[m].float())
            torch.mm(self.z[m], self.table(P, m).to(self.z.dtype), out=self.dx[m])
        layers.norm_backward(plan, self.x, self.dx, P, self.stats, self.dx, G, self.norm_ws, **self.where)
        layers.embed_backward(plan, tokens, self.dx, G, self.vocab, self.embed_ws, scale=self.scale, add=True)
        return self.loss


def run_student(kind, M=4, vocab=256, width=64, tokens=96, k=16, T=50, eta=0.05, temperature=1.0, seed=0,
                dtype=torch.float32, keep=0, **plan_kwargs):
    """T iterations of Algorithm 2 on the student, whose teacher sends k logits a
    token (`keep`: the top-k compressor's entries); returns the mean loss of each."""
    dev = torch.device("cuda")
    d, offsets = Student.parameters(vocab, width)
    if kind in ("sign", "qsgd", "mbit"):
        plan_kwargs.setdefault("seg_offsets", offsets)
    plan = dqgan.Plan(d, M, kind, k=keep, seed=seed + 1, **plan_kwargs)
    gen = torch.Generator(device=dev).manual_seed(seed)

    def draw(v):
        v[:offsets[1]].normal_(0.0, width ** -0.5, generator=gen)
        v[offsets[1]:offsets[2]] = 1.0
        return v

    teacher = draw(torch.zeros(plan.ld, device=dev)).expand(M, -1).contiguous()    # one for all workers
    W = draw(torch.zeros(plan.ld, device=dev))
    E, G = torch.zeros((M, plan.ld), device=dev), torch.zeros((M, plan.ld), device=dev)
    WX = W.expand(M, -1).clone()
    wire = plan.new_wire(dev)
    student = Student(plan, vocab, width, tokens, k, temperature, dtype)
    weight = torch.full((M, tokens), 1.0 / tokens, device=dev)
    hist = []
    for t in range(1, T + 1):
        tok = torch.randint(0, vocab, (M, tokens), generator=gen, device=dev)
        top = torch.topk(student.forward(teacher, tok).float(), k)
        loss = student.gradients(WX, tok, top.values.contiguous(), top.indices.int(), weight, G)
        hist.append(float(loss.sum()) / M)
        dqgan.step_fused(plan, eta, t, G, E, W, WX, wire)
    plan.close()
    return hist
