"""The operators of a vocabulary's network together: layers with activations and residuals under a loss over their logits, one
training step against automatic differentiation in 64 bits, captured and replayed, and the same network serving."""
import pytest

from tests.test_gpu_expert import _dt, _gen

pytestmark = pytest.mark.gpu


class Net:
    """x -> x + W2 act(W1 x + b1) + b2 (twice) -> logits = W x + b, logits in fp32."""

    def __init__(self, imbd, dev, B, d, hidden, V, dtype, act, seed=0):
        import torch
        g = _gen(seed, dev)
        self.m, self.dev, self.B, self.d, self.hidden, self.V, self.act, self.dt = imbd, dev, B, d, hidden, V, act, _dt(dtype)
        shapes = {"w1": (hidden, d), "b1": (hidden,), "w2": (d, hidden), "b2": (d,), "w3": (hidden, d), "b3": (hidden,),
                  "w4": (d, hidden), "b4": (d,), "w": (V, d), "b": (V,)}
        self.p = {k: torch.randn(*s, generator=g, device=dev) * (s[-1] ** -0.5 if len(s) == 2 else 0.1) for k, s in shapes.items()}
        self.lp = {k: v.to(self.dt) if v.dim() == 2 else v for k, v in self.p.items()}
        if dtype == "f32":
            self.lp = self.p
        self.grad = {k: torch.zeros_like(v) for k, v in self.p.items()}
        self.x = torch.randn(B, d, generator=g, device=dev).to(self.dt)
        e = lambda *s: torch.zeros(*s, dtype=self.dt, device=dev)  # noqa: E731
        self.z1, self.h1, self.y1, self.z3, self.h3, self.y3 = e(B, hidden), e(B, hidden), e(B, d), e(B, hidden), e(B, hidden), e(B, d)
        self.dz, self.dy3, self.dy1, self.dx = e(B, hidden), e(B, d), e(B, d), e(B, d)
        self.logits = torch.zeros(B, V, device=dev)
        self.dlogits = e(B, V)
        code = imbd.dtype_code(self.dt)
        n = max([imbd.linear_workspace_bytes(w, code, *s, B) for w in (0, 1) for s in shapes.values() if len(s) == 2] + [8])
        self.ws = torch.full((n,), 255, dtype=torch.uint8, device=dev)

    def forward(self):
        f, p, ws = self.m.linear_fwd, self.lp, self.ws
        f(p["w1"], self.x, self.h1, bias=p["b1"], act=self.act, z=self.z1, ws=ws)
        f(p["w2"], self.h1, self.y1, bias=p["b2"], residual=self.x, ws=ws)
        f(p["w3"], self.y1, self.h3, bias=p["b3"], act=self.act, z=self.z3, ws=ws)
        f(p["w4"], self.h3, self.y3, bias=p["b4"], residual=self.y1, ws=ws)
        f(p["w"], self.y3, self.logits, bias=p["b"], ws=ws)

    def backward(self):
        f, p, g, ws = self.m.linear_bwd, self.lp, self.grad, self.ws
        f(p["w"], self.dlogits, self.y3, dw=g["w"], db=g["b"], dx=self.dy3, ws=ws)
        f(p["w4"], self.dy3, self.h3, dw=g["w4"], db=g["b4"], dx=self.dz, act=self.act, z=self.z3, ws=ws)
        f(p["w3"], self.dz, self.y1, dw=g["w3"], db=g["b3"], dx=self.dy1, residual=self.dy3, ws=ws)
        f(p["w2"], self.dy1, self.h1, dw=g["w2"], db=g["b2"], dx=self.dz, act=self.act, z=self.z1, ws=ws)
        f(p["w1"], self.dz, self.x, dw=g["w1"], db=g["b1"], dx=self.dx, residual=self.dy1, ws=ws)

    def exact(self, p, x):
        import torch
        act = {"gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu, "relu": torch.relu,
               "gelu_tanh": lambda t: torch.nn.functional.gelu(t, approximate="tanh")}[self.act]
        for i in ("1", "3"):
            j = str(int(i) + 1)
            x = x + act(x @ p["w" + i].t() + p["b" + i]) @ p["w" + j].t() + p["b" + j]
        return x @ p["w"].t() + p["b"]


def _norm_close(got, ref, tol, what):
    err = (got.double() - ref).norm() / ref.norm()
    assert err <= tol, (what, err.item())


@pytest.mark.parametrize("dtype,B,d,hidden,V,act", [("f32", 37, 50, 122, 301, "gelu"), ("bf16", 64, 128, 512, 1000, "gelu_tanh"),
                                                    ("bf16", 300, 256, 640, 5003, "silu"), ("bf16", 16, 264, 1000, 777, "gelu")])
def test_training_step(imbd, dev, dtype, B, d, hidden, V, act):
    """Distillation through two residual blocks: every gradient, then AdamW. Each stored bf16 tensor of the eleven on the way
    is off by half a step, 2^-9 of its norm as these errors are spread, of which a gradient sees some at most twice: under 11 * 2 *
    2^-9 of the norm even if they all added up; fp32 has 2^-24 and sums of at most 1000 terms: 1e-4."""
    import torch
    net = Net(imbd, dev, B, d, hidden, V, dtype, act)
    K = 8
    g = _gen(7, dev)
    ids = torch.stack([torch.randperm(V, generator=g, device=dev)[:K] for _ in range(B)]).to(torch.int32)
    t = torch.randn(B, K, generator=g, device=dev) * 2
    weight = torch.ones(B, device=dev)
    weight[B // 3] = 0.0
    loss, row = torch.zeros(1, device=dev), torch.zeros(B, device=dev)
    dws = torch.zeros(max(8, imbd.distill_workspace_bytes(B, V, K)), dtype=torch.uint8, device=dev)
    state = {k: (torch.zeros_like(v), torch.zeros_like(v)) for k, v in net.p.items()}
    plan = imbd.AdamW([{"w": net.p[k], "grad": net.grad[k], "m": state[k][0], "v": state[k][1],
                        **({"w_lp": net.lp[k]} if net.lp[k].dtype == torch.bfloat16 else {})} for k in net.p])

    def gradients():
        net.forward()
        imbd.distill_xent(net.logits, ids, t, 1.0 / B, loss, row, dlogits=net.dlogits, temperature=2.0, weight=weight, ws=dws)
        net.backward()

    gradients()
    torch.cuda.synchronize()
    tol = 11 * 2 * 2.0 ** -9 if dtype == "bf16" else 1e-4
    p = {k: v.double().requires_grad_() for k, v in net.lp.items()}
    x = net.x.double().requires_grad_()
    logq = torch.log_softmax(net.exact(p, x) / 2.0, 1)
    q = torch.softmax(t.double() / 2.0, 1)
    kl = 4.0 * weight.double() * (q * (q.log() - logq.gather(1, ids.long()))).sum(1)
    (kl.sum() / B).backward()
    assert abs(loss.item() - kl.sum().item() / B) <= tol * kl.sum().item() / B
    _norm_close(row, kl.detach(), tol, "row_loss")
    for k in p:
        _norm_close(net.grad[k], p[k].grad, tol, k)
    _norm_close(net.dx, x.grad, tol, "dx")

    # the whole step in a graph: the same bits as eager steps from the same state
    before = {k: v.clone() for k, v in net.p.items()}

    def restore():
        for k in net.p:
            net.p[k].copy_(before[k])
            if net.lp[k] is not net.p[k]:
                net.lp[k].copy_(before[k])
            for s in state[k]:
                s.zero_()

    step = torch.zeros(1, dtype=torch.int32, device=dev)

    def train():
        step.add_(1)
        gradients()
        imbd.adamw_step(plan, lr=1e-2, step=step)

    def run(f):
        restore()
        step.zero_()
        losses = []
        for _ in range(3):
            f()
            losses.append(loss.clone())
        torch.cuda.synchronize()
        return torch.cat(losses), {k: v.clone() for k, v in net.p.items()}

    eager = run(train)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        train()
    replayed = run(graph.replay)
    assert torch.equal(eager[0], replayed[0]) and all(torch.equal(eager[1][k], replayed[1][k]) for k in eager[1])
    assert not torch.equal(eager[0][0], eager[0][1])


@pytest.mark.parametrize("B", [1, 8, 40])
def test_serving_step(imbd, dev, B):
    """Logits of single tokens, the chosen token's log probability and the alternatives."""
    import torch
    V = 2003
    net = Net(imbd, dev, B, 256, 1024, V, "bf16", "silu")
    net.forward()
    tokens = net.logits.argmax(1).to(torch.int32)
    logp, ids, top = torch.zeros(B, device=dev), torch.zeros(B, 5, dtype=torch.int32, device=dev), torch.zeros(B, 5, device=dev)
    ws = torch.zeros(max(8, imbd.token_logprobs_workspace_bytes(B, V, 5)), dtype=torch.uint8, device=dev)
    imbd.token_logprobs(net.logits, tokens, logp, top_ids=ids, top_logp=top, ws=ws)
    torch.cuda.synchronize()
    _norm_close(net.logits, net.exact({k: v.double() for k, v in net.lp.items()}, net.x.double()), 6 * 2.0 ** -9, "logits")
    assert torch.equal(ids[:, 0], tokens) and torch.equal(top[:, 0], logp)
    ref = torch.log_softmax(net.logits.double(), 1)
    order = torch.argsort(net.logits, dim=1, descending=True, stable=True)[:, :5]
    assert torch.equal(ids.long(), order) and (top.double() - ref.gather(1, order)).abs().max() <= 1e-5


def test_policy_gradient_step(imbd, dev):
    """Log probabilities and entropies of given tokens through the logits back to the weights."""
    import torch
    B, V = 50, 403
    net = Net(imbd, dev, B, 64, 96, V, "f32", "gelu")
    net.forward()
    tokens = torch.randint(0, V, (B,), generator=_gen(3, dev), device=dev, dtype=torch.int32)
    logp, ent, lse = (torch.zeros(B, device=dev) for _ in range(3))
    imbd.token_logprobs(net.logits, tokens, logp, entropy=ent, lse=lse)
    adv = torch.randn(B, generator=_gen(4, dev), device=dev)
    imbd.token_logprobs_bwd(net.logits, tokens, lse, net.dlogits, dlogp=adv / B, entropy=ent, dentropy=torch.full((B,), -0.01 / B, device=dev))
    net.backward()
    torch.cuda.synchronize()
    p = {k: v.double().requires_grad_() for k, v in net.p.items()}
    logq = torch.log_softmax(net.exact(p, net.x.double()), 1)
    picked = logq.gather(1, tokens.long()[:, None]).squeeze(1)
    ((adv.double() * picked).sum() / B + 0.01 * (logq.exp() * logq).sum() / B).backward()
    _norm_close(logp, picked.detach(), 1e-4, "logp")
    for k in p:
        _norm_close(net.grad[k], p[k].grad, 1e-4, k)
