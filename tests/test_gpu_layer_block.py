"""GPU: the calls around a linear layer together, as one half of a block uses them: norm, product with bias and activation, product onto the residual stream, and the whole way back; eager, recorded
and replayed, on two streams at once, and into a Muon step.

Every call is held against the fp64 oracle on the inputs it really had (what the calls before it left), with the bounds of its own test, so that errors do not add up."""
import numpy as np
import pytest

from oracle import layer as L
from tests.layer_harness import BF16, F32, HALF, MX8, held, stream
from tests.test_gpu_act import bounds

pytestmark = pytest.mark.gpu

T, D, H = 150, 264, 520        # tokens, width, hidden: none a multiple of 128
EPS = 1e-5
KIND = L.GELU


class Block:
    """h = x + r; y = norm(h) in 8 bits; z = y W1^T + b1 kept in 8 bits, a = gelu(z); out = a W2^T + h.  Backward from dout to every gradient."""

    def __init__(self, canz, seed):
        import torch
        rng = np.random.default_rng(seed)
        bf, f = torch.bfloat16, torch.float32
        dev = lambda x, t: torch.from_numpy(np.ascontiguousarray(x)).float().to(t).cuda()  # noqa: E731
        self.canz = canz
        self.x, self.r = dev(rng.standard_normal((T, D)), bf), dev(rng.standard_normal((T, D)) * 2, bf)
        self.w = dev(1 + 0.2 * rng.standard_normal(D), f)
        self.w1, self.b1, self.w2 = dev(rng.standard_normal((H, D)) * D ** -0.5, bf), dev(rng.standard_normal(H) * 0.3, f), dev(rng.standard_normal((D, H)) * H ** -0.5, bf)
        self.dout = dev(rng.standard_normal((T, D)), bf)
        e = lambda *s, t=bf: torch.full(s, float("nan"), dtype=t, device="cuda")  # noqa: E731
        image = lambda r, c: torch.zeros(canz.canz_mx_eight_bytes(r, c), dtype=torch.uint8, device="cuda")  # noqa: E731
        self.h, self.rstd, self.y8, self.z8, self.a, self.out = e(T, D), e(T, t=f), image(T, D), image(T, H), e(T, H), e(T, D)
        self.da, self.again, self.dz, self.dy, self.dx = e(T, H), e(T, H), e(T, H), e(T, D), e(T, D)
        self.dw1, self.dw2, self.db1, self.dw = e(H, D, t=f), e(D, H, t=f), e(H, t=f), e(D, t=f)
        P = canz.Linear
        self.norm = [canz.Norm(rows=T, cols=D, x=self.x, residual=self.r, weight=self.w, sum=self.h, y8=self.y8, rstd=self.rstd, eps=EPS)]
        self.up = [P(m=T, n=H, k=D, a=[self.y8], b=[self.w1], c=[self.a], bias=[self.b1], pre8=[self.z8], a_dtype=MX8, act=KIND)]
        self.down = [P(m=T, n=D, k=H, a=[self.a], b=[self.w2], c=[self.out], residual=[self.h], beta=1.0)]
        self.back = [P(m=T, n=H, k=D, a=[self.dout], b=[self.w2], c=[self.da], b_trans=True)]
        self.act = [canz.ActGrad(rows=T, cols=H, dout=self.da, gate=self.z8, dgate=self.dz, out=self.again, act=KIND)]
        self.grads = [P(m=D, n=H, k=T, a=[self.dout], b=[self.again], c=[self.dw2], a_trans=True, b_trans=True, out_dtype=F32),
                      P(m=H, n=D, k=T, a=[self.dz], b=[self.y8], c=[self.dw1], a_sums=[self.db1], a_trans=True, b_trans=True, b_dtype=MX8, out_dtype=F32),
                      P(m=T, n=D, k=H, a=[self.dz], b=[self.w1], c=[self.dy], b_trans=True)]
        self.norm_grad = [canz.NormGrad(rows=T, cols=D, dy=self.dy, h=self.h, rstd=self.rstd, weight=self.w, dsum=self.dout, dx=self.dx, dweight=self.dw)]
        need = max([canz.canz_linear_workspace_bytes(g) for g in (self.up, self.down, self.back, self.grads)] + [canz.canz_norm_backward_workspace_bytes(self.norm_grad)])
        self.ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")

    def run(self, st):
        c, ws = self.canz, (self.ws, self.ws.numel(), st)
        c.canz_norm_forward(self.norm, st)
        c.canz_linear(self.up, *ws)
        c.canz_linear(self.down, *ws)
        c.canz_linear(self.back, *ws)
        c.canz_act_backward(self.act, st)
        c.canz_linear(self.grads, *ws)
        c.canz_norm_backward(self.norm_grad, *ws)

    RESULTS = ("h", "rstd", "y8", "z8", "a", "out", "da", "again", "dz", "dy", "dx", "dw1", "dw2", "db1", "dw")

    def results(self):
        return {k: getattr(self, k).clone() for k in self.RESULTS}

    def host(self, name):
        return getattr(self, name).double().cpu().numpy()

    def image(self, name, rows, cols):
        pitch = -(-cols // 128) * 128
        b = getattr(self, name).cpu().numpy()
        codes, scales = b[:rows * pitch].reshape(rows, pitch)[:, :cols], b[rows * pitch:][:rows * pitch // 32].reshape(rows, pitch // 32)
        return L.values(codes, scales[:, :-(-cols // 32)])


def near(got, want, mag, k, dtype, extra=0.0):
    """A sum of k products: (k + 4) 2^-23 of the sum of magnitudes, one rounding, and what an activation adds."""
    b = 1.13 * (k + 4) * 2.0 ** -23 * mag + extra
    assert (np.abs(got - want) <= b + HALF[dtype] * (np.abs(want) + b)).all()


def check(b):
    g = b.host
    x, r, w, w1, b1, w2, dout = (g(n) for n in ("x", "r", "w", "w1", "b1", "w2", "dout"))
    h = g("h")
    assert np.array_equal(h, held(x + r, BF16))
    y, rstd = L.norm(h, w, float(np.float32(EPS)))
    assert (np.abs(g("rstd") - rstd) <= rstd * 50 * 2.0 ** -24).all()
    y8 = b.image("y8", T, D)
    block = np.repeat(np.abs(np.pad(y, ((0, 0), (0, -D % 32)))).reshape(T, -1, 32).max(2), 32, axis=1)[:, :D]
    step = np.maximum(np.abs(y) * 2.0 ** -4, block * 2.0 ** -17)     # half a step: 2^-4 of the element, or 2^-10 X with X < amax / 224 and twice that at a border
    assert (np.abs(y8 - y) <= step * 1.01).all()
    a, z = L.linear(y8, w1, 1.0, b1, KIND)
    mag = np.abs(y8) @ np.abs(w1).T + np.abs(b1)
    near(g("a"), a, mag, D, BF16, bounds(KIND, z)[0])
    z8 = b.image("z8", T, H)
    block = np.repeat(np.abs(np.pad(z, ((0, 0), (0, -H % 32)))).reshape(T, -1, 32).max(2), 32, axis=1)[:, :H]
    assert (np.abs(z8 - z) <= np.maximum(np.abs(z) * 2.0 ** -4, block * 2.0 ** -17) * 1.01 + (D + 4) * 2.0 ** -23 * mag).all()
    av = g("a")
    near(g("out"), av @ w2.T + h, np.abs(av) @ np.abs(w2).T + np.abs(h), H, BF16)
    near(g("da"), dout @ w2, np.abs(dout) @ np.abs(w2), D, BF16)
    da = g("da")
    dz, _ = L.gated_grad(KIND, da, z8, None)
    near(g("dz"), dz, np.abs(dz), 0, BF16, np.abs(da) * bounds(KIND, z8)[1])
    near(g("again"), L.act(KIND, z8), 0 * z8, 0, BF16, bounds(KIND, z8)[0])
    dz, again = g("dz"), g("again")
    near(g("dw2"), dout.T @ again, np.abs(dout).T @ np.abs(again), T, F32)
    near(g("dw1"), dz.T @ y8, np.abs(dz).T @ np.abs(y8), T, F32)
    near(g("db1"), dz.sum(0), np.abs(dz).sum(0), T, F32)
    near(g("dy"), dz @ w1, np.abs(dz) @ np.abs(w1), H, BF16)
    dy, rstd = g("dy"), g("rstd")
    dx, dw = L.norm_grad(dy, h, rstd, w, dout)
    n, u = h * rstd[:, None], w * dy
    near(g("dx"), dx, rstd[:, None] * (np.abs(u) + np.abs(n) * np.abs(u * n).mean(1, keepdims=True)) + np.abs(dx), 40, BF16)
    near(g("dw"), dw, np.abs(dy * n).sum(0), 80, F32)


def test_block(canz):
    import torch
    b = Block(canz, 1)
    b.run(stream())
    torch.cuda.synchronize()
    check(b)


def test_gradients_against_differences(canz):
    """Along each gradient's own direction d = g / |g| the loss sum dout out, in 64 bits and without a rounding, has the slope |g| if g is right.  Two elements in a row are off by 2^-4 at
    most from their 8-bit images (y, z), a dozen by 2^-8 from bf16: below 0.18 of |g| if all of them conspired."""
    import torch
    b = Block(canz, 2)
    b.run(stream())
    torch.cuda.synchronize()
    v = {n: b.host(n) for n in ("x", "r", "w", "w1", "b1", "w2", "dout")}

    def loss(**moved):
        q = {**v, **moved}
        h = q["x"] + q["r"]
        a = L.act(KIND, L.norm(h, q["w"], EPS)[0] @ q["w1"].T + q["b1"])
        return (q["dout"] * (a @ q["w2"].T + h)).sum()

    for name, grad in (("x", "dx"), ("r", "dx"), ("w", "dw"), ("w1", "dw1"), ("b1", "db1"), ("w2", "dw2")):
        g = b.host(grad)
        d = g / np.linalg.norm(g)
        t = 1e-4
        slope = (loss(**{name: v[name] + t * d}) - loss(**{name: v[name] - t * d})) / (2 * t)
        assert abs(slope / np.linalg.norm(g) - 1) < 0.18, name


def test_recorded_and_replayed(canz):
    """Two graphs with workspaces of their own, replayed in turn on changing inputs with eager runs in between: the bits of an eager run every time."""
    import torch
    blocks = [Block(canz, 3), Block(canz, 4)]
    for b in blocks:
        b.run(stream())
    torch.cuda.synchronize()
    graphs = []
    for b in blocks:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            b.run(torch.cuda.current_stream().cuda_stream)
        graphs.append(g)
    other = Block(canz, 5)
    for turn in range(3):
        for b, g in zip(blocks, graphs):
            b.x.copy_(torch.randn(T, D, device="cuda"))
            b.dout.mul_(0.5)
            g.replay()
            other.run(stream())
        torch.cuda.synchronize()
        for b in blocks:
            got = b.results()
            b.run(stream())
            torch.cuda.synchronize()
            assert all(torch.equal(got[k], getattr(b, k)) for k in got)
    check(blocks[0])


def test_two_streams_at_once(canz):
    import torch
    blocks = [Block(canz, 6), Block(canz, 7)]
    want = []
    for b in blocks:
        b.run(stream())
        torch.cuda.synchronize()
        want.append(b.results())
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for b, s in zip(blocks, streams):
            b.run(s.cuda_stream)
    torch.cuda.synchronize()
    for b, w in zip(blocks, want):
        assert all(torch.equal(w[k], getattr(b, k)) for k in w)


@pytest.mark.parametrize("handle", [0, 1, 2])
def test_default_streams(canz, handle):
    """The null stream, the legacy and the per-thread default stream by their handles."""
    import torch
    b = Block(canz, 8)
    b.run(stream())
    torch.cuda.synchronize()
    want = b.results()
    for k in want:
        getattr(b, k).zero_()
    torch.cuda.synchronize()
    b.run(handle)
    torch.cuda.synchronize()
    assert all(torch.equal(want[k], getattr(b, k)) for k in want)


def test_gradient_enters_a_step(canz):
    """dW1 in bf16 straight into canz_muon_step, whose parameters are the next product's operand."""
    import torch
    from oracle import muon as OM
    b = Block(canz, 9)
    dw = torch.empty(H, D, dtype=torch.bfloat16, device="cuda")
    b.grads[1].c, b.grads[1].out_dtype = [dw], BF16
    mom, p = torch.zeros(H, D, device="cuda"), b.w1.clone()
    hp = canz.Hparams()
    group = canz.Group(rows=H, cols=D, grad=[dw], mom=[mom], out=[p], grad_dtype=canz.DT_BF16, out_dtype=canz.DT_BF16)
    ws = torch.empty(canz.canz_muon_workspace_bytes([group], hp), dtype=torch.uint8, device="cuda")
    b.run(stream())
    canz.canz_muon_step([group], hp, ws, ws.numel(), stream())
    c = torch.empty(T, H, device="cuda")
    canz.canz_linear([canz.Linear(m=T, n=H, k=D, a=[b.x], b=[p], c=[c], out_dtype=F32)], b.ws, b.ws.numel(), stream())
    torch.cuda.synchronize()
    f = lambda v: float(np.float32(v))  # noqa: E731
    ohp = OM.Hparams(beta=f(hp.beta), lr=f(hp.lr), weight_decay=f(hp.weight_decay), eps=f(hp.eps), ns_steps=5, a=f(hp.a), b=f(hp.b), c=f(hp.c), scale_mode=hp.scale_mode)
    delta = OM.muon_step(dw.double().cpu().numpy(), np.zeros((H, D)), ohp)["delta"]
    got = p.double().cpu().numpy() - b.host("w1")
    round_off = np.linalg.norm(b.host("w1")) * 2.0 ** -8
    assert np.linalg.norm(got - delta) <= 3e-2 * np.linalg.norm(delta) + round_off
    x, pv = b.host("x"), p.double().cpu().numpy()
    near(c.double().cpu().numpy(), x @ pv.T, np.abs(x) @ np.abs(pv).T, D, F32)
