"""The operators together, as a pre-norm residual sub-layer: two of them in a row, a training step
(forward, backward, orthogonalised update) and serving with the updated weights, against the
formulas in 64 bits with autograd."""
import pytest
import torch

from paper_2002_04013_amd import DMoESublayer, abi
from parity_util import say

NAMES = ("gamma", "beta", "Wg", "bg", "W1", "b1", "W2", "b2")


def _params(D, H, d, M, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    r = lambda *s, sc=1.0, at=0.0: (torch.randn(*s, generator=g) * sc + at).to(dt)
    N = M ** d
    return dict(gamma=r(D, sc=0.2, at=1.0), beta=r(D, sc=0.2), Wg=r(d * M, D, sc=D ** -0.5), bg=r(d * M, sc=0.1),
                W1=r(N, H, D, sc=D ** -0.5), b1=r(N, H, sc=0.2), W2=r(N, D, H, sc=H ** -0.5), b2=r(N, D, sc=0.2))


def _reference(x, res, p, alive, idx, d, M, act):
    """(s, y) in 64 bits with the given choice of experts."""
    s = x if res is None else x + res
    mean = s.mean(1, keepdim=True)
    n = p["gamma"] * (s - mean) / torch.sqrt(((s - mean) ** 2).mean(1, keepdim=True) + 1e-5) + p["beta"]
    S = n @ p["Wg"].t() + p["bg"]
    g = sum(S.gather(1, (idx // M ** (d - 1 - i)) % M + i * M) for i in range(d))
    live = alive[idx] != 0
    w = torch.softmax(torch.where(live, g, torch.full_like(g, -1e30)), 1) * live
    y = torch.zeros_like(s)
    for e in idx.unique().tolist():
        t, j = ((idx == e) & live).nonzero(as_tuple=True)
        h = n[t] @ p["W1"][e].t() + p["b1"][e]
        a = torch.relu(h) if act == "relu" else 0.5 * h * (1 + torch.erf(h * 0.5 ** 0.5))
        y = y.index_add(0, t, w[t, j][:, None] * (a @ p["W2"][e].t() + p["b2"][e]))
    return s, y


def _near(got, want, tol, name):
    got = got.double().cpu()
    rms = want.square().mean().sqrt()
    worst = ((got - want).abs() / (tol * (want.abs() + rms) + 1e-30)).max().item() if want.numel() else 0.0
    assert worst <= 1, f"{name}: {worst:.3g} of the tolerance"


@pytest.mark.gpu
@pytest.mark.parametrize("recompute", [False, True])
def test_training_step_of_two_sublayers(recompute):
    """fp32.  Tolerance 2e-4 of a value and the rms: sums of at most 256 products ((256 + 2) 2^-24 = 1.6e-5 of their
    absolute values' sum) in a chain of at most ten of them, forward and backward through both."""
    T, D, H, d, M, k, act = 96, 64, 192, 2, 3, 2, "gelu"
    tol = 2e-4
    p = [_params(D, H, d, M, "f32", s) for s in (1, 2)]
    dev = [{n: v.cuda() for n, v in q.items()} for q in p]
    g = torch.Generator().manual_seed(5)
    x, c = torch.randn(T, D, generator=g), torch.randn(T, D, generator=g)
    alive = torch.ones(M ** d, dtype=torch.uint8)
    alive[4] = 0
    sub = [DMoESublayer(T, D, H, d, M, k, "f32", act, recompute=recompute) for _ in range(2)]
    P = lambda i: [dev[i][n] for n in ("gamma", "beta", "Wg", "bg")] + [alive.cuda()] + [dev[i][n] for n in ("W1", "b1", "W2", "b2")]
    s0, y0 = sub[0].forward(x.cuda(), None, *P(0))
    s1, y1 = sub[1].forward(y0, s0, *P(1))
    grads = [{n: torch.full_like(v, 7.0) for n, v in q.items()} for q in dev]
    dout = c.cuda()                                       # of out = s1 + y1, L = <c, out>

    def back(i, dy, ds, s):
        q = dev[i]
        return sub[i].backward(dy, ds, s, q["gamma"], q["Wg"], alive.cuda(), q["W1"], q["W2"], grads[i], b1=q["b1"])

    dx1 = back(1, dout, dout, s1)                         # of y0 and of s0
    dx0 = back(0, dx1, dx1, s0)
    torch.cuda.synchronize()
    # 64 bits
    r = [{n: v.double().requires_grad_() for n, v in q.items()} for q in p]
    xr = x.double().requires_grad_()
    idx = [q.layer.idx.long().cpu() for q in sub]
    a0, b0 = _reference(xr, None, r[0], alive, idx[0], d, M, act)
    a1, b1 = _reference(b0, a0, r[1], alive, idx[1], d, M, act)
    ((a1 + b1) * c.double()).sum().backward()
    for got, want, name in ((y0, b0, "y0"), (s1, a1, "s1"), (y1, b1, "y1"), (dx0, xr.grad, "dx")):
        _near(got, want.detach(), tol, name)
    for i in range(2):
        rows = sub[i].layer.counts.cpu() > 0
        assert not rows[4]
        for n in NAMES:
            got, want = grads[i][n].cpu(), r[i][n].grad
            if n in ("W1", "b1", "W2", "b2"):
                assert (got[~rows] == 7).all()             # experts without rows keep the caller's
                got, want = got[rows], want[rows]
            _near(got, want, tol, f"d{n} of {i}")
    # the update: experts without rows keep their matrices; the others' steps are near-orthogonal
    mom = [{n: torch.zeros_like(q[n]) for n in ("W1", "W2", "Wg")} for q in dev]
    before = [{n: v.clone() for n, v in q.items()} for q in dev]
    for i in range(2):
        sub[i].update(dev[i], grads[i], mom[i], lr=0.125, mu=0.5)
    torch.cuda.synchronize()
    for i in range(2):
        rows = (sub[i].layer.counts > 0)
        for n in ("W1", "W2"):
            assert torch.equal(dev[i][n][~rows], before[i][n][~rows])
            step = (before[i][n] - dev[i][n])[rows].double() / 0.125
            top = torch.linalg.svdvals(step)[:, 0]
            # singular values end below 1.21; W's rounding adds 2^-24 |W| / lr
            assert (top < 1.211).all() and (top > 0.6).all(), n
        step = (before[i]["Wg"] - dev[i]["Wg"]).view(d, M, D).double() / 0.125
        assert (torch.linalg.svdvals(step)[:, 0] < 1.211).all()
        for n in ("gamma", "beta", "bg", "b1", "b2"):
            assert torch.equal(dev[i][n], before[i][n])
    # serving with the updated weights, a few of the tokens: as the regular pass gives them
    few = 5
    serve = [DMoESublayer(few, D, H, d, M, k, "f32", act) for _ in range(2)]
    o0 = serve[0].serve(x[:few].cuda(), None, *P(0))
    o1 = serve[1].serve(o0, None, *P(1))
    s0, y0 = sub[0].forward(x.cuda(), None, *P(0))
    s1, y1 = sub[1].forward(y0, s0, *P(1))
    assert torch.equal(serve[1].layer.few.idx, sub[1].layer.idx[:few])
    _near(o1, (s1 + y1)[:few].double().cpu(), tol, "served")


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 8, 40])
def test_serving_bf16(T):
    """bf16: the normalised row, the activations and the result are rounded once each on the way (2^-8 of a value,
    the first two carried on by matrices of gain about one, gelu' below 1.13; the gate's weights by a gain of
    their own): 6 x 2^-8 of a value and the rms."""
    D, H, d, M, k = 256, 512, 2, 4, 3
    p = _params(D, H, d, M, "bf16", 7)
    dev = {n: v.cuda() for n, v in p.items()}
    g = torch.Generator().manual_seed(T)
    x, res = (torch.randn(T, D, generator=g).bfloat16() for _ in range(2))
    alive = (torch.rand(M ** d, generator=g) < 0.8).to(torch.uint8)
    sub = DMoESublayer(T, D, H, d, M, k, "bf16")
    out = sub.serve(x.cuda(), res.cuda(), dev["gamma"], dev["beta"], dev["Wg"], dev["bg"], alive.cuda(), dev["W1"], dev["b1"],
                    dev["W2"], dev["b2"])
    r = {n: v.double() for n, v in p.items()}
    s = (x.double() + res.double()).bfloat16().double()
    _, y = _reference(s, None, r, alive, sub.layer.few.idx.long().cpu(), d, M, "gelu")
    say(f"[sublayer] {T}")
    _near(out, s + y, 6 * 2.0 ** -8, "out")


@pytest.mark.gpu
def test_graph_of_a_whole_step():
    """Forward, backward and update captured at once and replayed: bit for bit the eager steps."""
    T, D, H, d, M, k = 128, 128, 128, 2, 3, 2
    dev = {n: v.cuda() for n, v in _params(D, H, d, M, "bf16", 3).items()}
    x, r, dout = (torch.randn(T, D, device="cuda").bfloat16() for _ in range(3))
    sub = DMoESublayer(T, D, H, d, M, k, "bf16", "relu")
    grads = {n: torch.zeros_like(v) for n, v in dev.items()}
    mom = {n: torch.zeros(dev[n].shape, device="cuda") for n in ("W1", "W2", "Wg")}

    def step():
        s, _ = sub.forward(x, r, dev["gamma"], dev["beta"], dev["Wg"], dev["bg"], None, dev["W1"], dev["b1"], dev["W2"], dev["b2"])
        sub.backward(dout, dout, s, dev["gamma"], dev["Wg"], None, dev["W1"], dev["W2"], grads)
        sub.update(dev, grads, mom, lr=0.02)

    start = {n: v.clone() for n, v in dev.items()}
    for _ in range(3):
        step()
    torch.cuda.synchronize()
    want = [{n: v.clone() for n, v in q.items()} for q in (dev, grads, mom)]
    for n in dev:
        dev[n].copy_(start[n])
    for n in mom:
        mom[n].zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for w in (sub.norm_ws, sub.muon_ws, sub.layer.ws):
            w.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
    for q, ref in zip((dev, grads, mom), want):
        assert all(torch.equal(q[n], ref[n]) for n in q)


@pytest.mark.gpu
def test_serve_takes_few_tokens_only():
    sub = DMoESublayer(65, 64, 64, 1, 4, 2, "f32")
    dev = {n: v.cuda() for n, v in _params(64, 64, 1, 4, "f32", 1).items()}
    x = torch.zeros(65, 64, device="cuda")
    with pytest.raises(abi.DmoeError):
        sub.serve(x, None, dev["gamma"], dev["beta"], dev["Wg"], dev["bg"], None, dev["W1"], dev["b1"], dev["W2"], dev["b2"])


@pytest.mark.gpu
@pytest.mark.parametrize("recompute", [False, True])
def test_serving_between_forward_and_backward(recompute):
    """A served batch between a forward and its backward changes nothing of the step: bit for bit."""
    T, D, H, d, M, k = 24, 128, 192, 2, 3, 2
    dev = {n: v.cuda() for n, v in _params(D, H, d, M, "bf16", 5).items()}
    x, r, dout, x2, r2 = (torch.randn(T, D, device="cuda").bfloat16() for _ in range(5))
    P = [dev[n] for n in ("gamma", "beta", "Wg", "bg")] + [None] + [dev[n] for n in ("W1", "b1", "W2", "b2")]
    want = None
    for between in (False, True):
        sub = DMoESublayer(T, D, H, d, M, k, "bf16", recompute=recompute)
        grads = {n: torch.zeros_like(v) for n, v in dev.items()}
        s, y = sub.forward(x, r, *P)
        served = sub.serve(x2, r2, *P).clone() if between else None
        dx = sub.backward(dout, dout, s, dev["gamma"], dev["Wg"], None, dev["W1"], dev["W2"], grads, b1=dev["b1"])
        got = [s, y, dx] + [grads[n] for n in dev]
        if between:
            assert all(torch.equal(p, q) for p, q in zip(got, want))
            fresh = DMoESublayer(T, D, H, d, M, k, "bf16")
            assert torch.equal(served, fresh.serve(x2, r2, *P))
        want = [q.clone() for q in got]
