"""Performance cases: microscaled 4-bit images of matrices and the products of such images.

An image holds a matrix as MXFP4: blocks of 32 consecutive elements along the contracted index share a power of two X, and each
element is one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times X with a sign.  With amax the largest magnitude of a block

  scale "floor"   X = 2^(floor(log2 amax) - 2)                   (magnitudes above 6 X become 6 X)
  scale "ceil"    X = the smallest power of two with amax <= 6 X  (nothing saturates)
  nearest         the nearest value, ties to the even code
  noise           with s the distance of the values around a = |v| / X: s floor((rint(256 a / s) + u) / 256), u a byte from
                  the caller; the mean over u is the value itself to within s / 512

Three kinds of case:

  op "round"      matrices -> images along rows and along columns (one call) -> the values these stand for (another)
                  rows, cols, count; dtype "f32" | "bf16"; noise 0 | 1; scale; side "both" | "row"
  op "product"    y = x W^T for activations as they come (bf16 or fp32, rounded within the call) and weights kept as images
                  m "1" or "<rows>+<rows>+...": one product for each part of x, with a W of its own (experts; a part may be empty)
                  n, k; x and out "f32" | "bf16"
  op "linear"     the three products of a linear layer's training pass: y = x W^T and dx = dy W in bf16, dW = dy^T x in fp32, from
                  x and dy in bf16; dy rounded with noise.  tokens, n, k

Shapes are those of this repository's workloads (paper_2602_06079_amd/workloads.py) and generic odd ones.
"""
import math

import torch

own = False

DEV = "cuda"
BLOCK = 32
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # the tiny workload's masters, 8 x 256 x 512: launches and latency
        dict(name="round_tiny", op="round", rows=256, cols=512, count=8, dtype="f32", noise=0, scale="floor", side="both"),
        # 0.6B-shaped set over 8 ranks: the masters of rank 0 after its step, both images (forward and input gradient)
        dict(name="round_0p6b_share", op="round", rows=2048, cols=1024, count=26, dtype="f32", noise=0, scale="floor", side="both"),
        # two masters of the 32B-shaped share
        dict(name="round_32b", op="round", rows=25600, cols=5120, count=2, dtype="f32", noise=0, scale="floor", side="both"),
        # gradients of odd extents, rounded with noise
        dict(name="round_ragged_noise", op="round", rows=4097, cols=1531, count=3, dtype="bf16", noise=1, scale="ceil", side="both"),
        # one token through a square projection of the 0.6B-shaped set: latency
        dict(name="product_token_small", op="product", m="1", n=1024, k=1024, x="bf16", out="bf16"),
        # one token through the 32B-shaped down projection: the weights are read once
        dict(name="product_token", op="product", m="1", n=5120, k=25600, x="bf16", out="bf16"),
        # a small batch of sequences, one token each
        dict(name="product_few", op="product", m="17", n=25600, k=5120, x="bf16", out="bf16"),
        # a prompt through the 32B-shaped gate
        dict(name="product_prompt", op="product", m="4096", n=25600, k=5120, x="bf16", out="bf16"),
        # odd extents, fp32 on both sides
        dict(name="product_odd", op="product", m="777", n=1531, k=1000, x="f32", out="f32"),
        # experts with the tokens a router gave them, two of them none
        dict(name="product_experts", op="product", m="0+1+37+400+5+128+0+1000", n=1536, k=4096, x="bf16", out="bf16"),
        # training pass of a 0.6B-shaped projection
        dict(name="linear_0p6b", op="linear", tokens=4096, n=2048, k=1024),
        # training pass of an 8B-shaped gate
        dict(name="linear_8b", op="linear", tokens=8192, n=12288, k=4096),
    ]


def draw(rng):
    """One more case of the same ranges: sizes spread over their logarithm, odd ones among them."""
    def extent(lo, hi):
        x = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        kind = rng.random()
        if kind < 0.3:
            x = max(1, round(x / 256)) * 256
        elif kind < 0.6:
            x = max(1, round(x / 32)) * 32
        return max(lo, min(hi, x))

    op = rng.choice(["round", "product", "product", "product", "linear"])
    if op == "round":
        rows, cols = extent(33, 25600), extent(33, 25600)
        most = max(1, min(26, (1 << 27) // (rows * cols)))
        if rows * cols > 1 << 28:
            rows = (1 << 28) // cols
        return dict(op=op, rows=rows, cols=cols, count=rng.randint(1, most), dtype=rng.choice(["f32", "bf16"]), noise=rng.randint(0, 1),
                    scale=rng.choice(["floor", "ceil"]), side=rng.choice(["both", "both", "row"]))
    if op == "linear":
        tokens, n, k = extent(33, 8192), extent(64, 12288), extent(64, 12288)
        while tokens * n * k > 8192 * 12288 * 4096:
            tokens, n, k = (max(33, e // 2) for e in (tokens, n, k))
        return dict(op=op, tokens=tokens, n=n, k=k)
    n, k = extent(33, 25600), extent(33, 25600)
    kind = rng.choice(["one", "few", "many", "experts"])
    if kind == "experts":
        n, k = min(n, 4096), min(k, 4096)
        m = "+".join(str(rng.choice([0, 1, rng.randint(2, 64), extent(33, 1000)])) for _ in range(rng.randint(2, 12)))
        m += "+%d" % rng.randint(1, 64)
    else:
        m = 1 if kind == "one" else rng.randint(2, 64) if kind == "few" else extent(65, 4096)
        m = str(max(1, min(m, 4096 * 25600 * 5120 // (n * k))))
    return dict(op=op, m=m, n=n, k=k, x=rng.choice(["bf16", "bf16", "f32"]), out=rng.choice(["bf16", "bf16", "f32"]))


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _weights(g, n, k):
    """W (n x k) with values an image holds exactly, as they are after an earlier rounding: bf16 holds them too."""
    kb = -(-k // BLOCK)
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=DEV)
    code = (torch.randn(n, kb * BLOCK, device=DEV, generator=g).abs() * 2.2).round().clamp(max=7).long()
    sign = torch.randint(0, 2, code.shape, device=DEV, generator=g, dtype=torch.int8) * 2 - 1
    x = torch.exp2(torch.randint(-8, -4, (n, kb, 1), device=DEV, generator=g).float())
    w = ((grid[code] * sign).view(n, kb, BLOCK) * x).view(n, kb * BLOCK)[:, :k]
    return w.to(torch.bfloat16).contiguous()


def _activations(g, m, k, dtype):
    """Gaussian rows with a few strong channels, one row in 16 all zero (padding)."""
    x = torch.randn(m, k, device=DEV, generator=g)
    x *= torch.where(torch.rand(k, device=DEV, generator=g) < 0.01, 20.0, 1.0)
    if m > 1:
        x *= (torch.rand(m, 1, device=DEV, generator=g) > 1.0 / 16).float()
    return x.to(dtype)


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case=case)
    if case["op"] == "round":
        r, c, count, dt = case["rows"], case["cols"], case["count"], DTYPES[case["dtype"]]
        s["x"] = [(torch.randn(r, c, device=DEV, generator=g) * 0.02).to(dt) for _ in range(count)]
        s["noise"] = [torch.randint(0, 256, (r, c), device=DEV, generator=g, dtype=torch.uint8) for _ in range(count)] if case["noise"] else []
    elif case["op"] == "product":
        ms = [int(m) for m in case["m"].split("+")]
        s["x"] = [_activations(g, m, case["k"], DTYPES[case["x"]]) for m in ms]
        s["w"] = [_weights(g, case["n"], case["k"]) for _ in ms]
    else:
        t, n, k = case["tokens"], case["n"], case["k"]
        s["x"] = _activations(g, t, k, torch.bfloat16)
        s["dy"] = (torch.randn(t, n, device=DEV, generator=g) * 1e-3).to(torch.bfloat16)
        s["noise"] = torch.randint(0, 256, (t, n), device=DEV, generator=g, dtype=torch.uint8)
        s["w"] = _weights(g, n, k)
    if own:
        _keep(s)
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ---------------------------------------------------------------- plain form

def _rounded(x, axis, scale, noise=None):
    """The values the images of the matrices x (... x rows x cols) with blocks along rows (axis 0) or columns (axis 1) stand for (fp32)."""
    v = x.float() if axis == 1 else x.float().mT
    k = v.shape[-1]
    blocks = v.shape[:-1] + (-(-k // BLOCK), BLOCK)
    v = torch.nn.functional.pad(v, (0, -k % BLOCK)).reshape(blocks)
    mant, exp = torch.frexp(v.abs().amax(-1, keepdim=True))      # amax = mant 2^exp, mant in [0.5, 1)
    e = exp - 3
    if scale == "ceil":
        e = e + (mant > 0.75).int()
    e = e.clamp(min=-127)
    a = torch.ldexp(v.abs(), -e)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    if noise is None:
        q = torch.round(a / step)
    else:
        u = noise if axis == 1 else noise.mT
        u = torch.nn.functional.pad(u, (0, -k % BLOCK)).reshape(blocks)
        q = torch.floor((torch.round(a / step * 256) + u) / 256)
    q = torch.ldexp((q * step).clamp(max=6.0) * torch.sign(v), e).flatten(-2)[..., :k]
    return q if axis == 1 else q.mT


def _run_plain(s):
    c = s["case"]
    if c["op"] == "round":
        x, u = torch.stack(s["x"]), torch.stack(s["noise"]) if s["noise"] else None
        sides = (1, 0) if c["side"] == "both" else (1,)
        return [list(_rounded(x, a, c["scale"], u).to(torch.bfloat16).contiguous()) for a in sides]
    if c["op"] == "product":
        x = _rounded(torch.cat(s["x"]), 1, "floor").split([x.shape[0] for x in s["x"]])
        return [torch.matmul(xi, w.float().t()).to(DTYPES[c["out"]]) for xi, w in zip(x, s["w"])]
    y = torch.matmul(_rounded(s["x"], 1, "floor"), s["w"].float().t())
    dx = torch.matmul(_rounded(s["dy"], 1, "ceil", s["noise"]), _rounded(s["w"], 0, "floor"))
    dw = torch.matmul(_rounded(s["dy"], 0, "ceil", s["noise"]).t(), _rounded(s["x"], 0, "floor"))
    return dict(y=y.to(torch.bfloat16), dx=dx.to(torch.bfloat16), dw=dw)


# ------------------------------------------------------- the framework's operators

def _keep(s):
    """What a program keeps from call to call: images of the weights, output buffers, groups, workspace."""
    from paper_2602_06079_amd import binding as canz
    c = s["case"]
    dt = dict(f32=canz.DT_F32, bf16=canz.DT_BF16)
    scale = dict(floor=canz.MX_SCALE_FLOOR, ceil=canz.MX_SCALE_CEIL)
    stream = torch.cuda.current_stream().cuda_stream

    def image(rows, cols):
        return torch.empty(canz.canz_mx_image_bytes(rows, cols), dtype=torch.uint8, device=DEV)

    s["canz"] = canz
    if c["op"] == "round":
        r, cc, count, both = c["rows"], c["cols"], c["count"], c["side"] == "both"
        by_row = [image(r, cc) for _ in range(count)]
        by_col = [image(cc, r) for _ in range(count)] if both else []
        s["scale"] = scale[c["scale"]]
        s["out"] = [[torch.empty(r, cc, dtype=torch.bfloat16, device=DEV) for _ in range(count)] for _ in range(2 if both else 1)]
        s["groups"] = [canz.MxGroup(rows=r, cols=cc, mat=s["x"], by_row=by_row, by_col=by_col, noise=s["noise"], dtype=dt[c["dtype"]])]
        s["back"] = [canz.MxGroup(rows=r, cols=cc, mat=s["out"][0], by_row=by_row, dtype=canz.DT_BF16)]
        if both:
            s["back"].append(canz.MxGroup(rows=r, cols=cc, mat=s["out"][1], by_col=by_col, dtype=canz.DT_BF16))
    elif c["op"] == "product":
        n, k = c["n"], c["k"]
        w = [image(n, k) for _ in s["w"]]
        canz.canz_mx_quantize([canz.MxGroup(rows=n, cols=k, mat=s["w"], by_row=w, dtype=canz.DT_BF16)], canz.MX_SCALE_FLOOR, stream)
        s["out"] = [torch.empty(x.shape[0], n, dtype=DTYPES[c["out"]], device=DEV) for x in s["x"]]
        s["groups"] = [canz.MxProduct(m=x.shape[0], n=n, k=k, a=[x], b=[wi], c=[y], a_dtype=dt[c["x"]], out_dtype=dt[c["out"]])
                       for x, wi, y in zip(s["x"], w, s["out"])]
    else:
        t, n, k = c["tokens"], c["n"], c["k"]
        w, wt, x, xt, dy, dyt = image(n, k), image(k, n), image(t, k), image(k, t), image(t, n), image(n, t)
        canz.canz_mx_quantize([canz.MxGroup(rows=n, cols=k, mat=[s["w"]], by_row=[w], by_col=[wt], dtype=canz.DT_BF16)],
                              canz.MX_SCALE_FLOOR, stream)
        s["rx"] = [canz.MxGroup(rows=t, cols=k, mat=[s["x"]], by_row=[x], by_col=[xt], dtype=canz.DT_BF16)]
        s["rdy"] = [canz.MxGroup(rows=t, cols=n, mat=[s["dy"]], by_row=[dy], by_col=[dyt], noise=[s["noise"]], dtype=canz.DT_BF16)]
        s["out"] = dict(y=torch.empty(t, n, dtype=torch.bfloat16, device=DEV), dx=torch.empty(t, k, dtype=torch.bfloat16, device=DEV),
                        dw=torch.empty(n, k, device=DEV))
        s["groups"] = [canz.MxProduct(m=t, n=n, k=k, a=[x], b=[w], c=[s["out"]["y"]], out_dtype=canz.DT_BF16),
                       canz.MxProduct(m=t, n=k, k=n, a=[dy], b=[wt], c=[s["out"]["dx"]], out_dtype=canz.DT_BF16),
                       canz.MxProduct(m=n, n=k, k=t, a=[dyt], b=[xt], c=[s["out"]["dw"]], out_dtype=canz.DT_F32)]
    if c["op"] != "round":
        s["ws"] = torch.empty(canz.canz_mx_product_workspace_bytes(s["groups"]), dtype=torch.uint8, device=DEV)


def _run_own(s):
    canz, c = s["canz"], s["case"]
    stream = torch.cuda.current_stream().cuda_stream
    if c["op"] == "round":
        canz.canz_mx_quantize(s["groups"], s["scale"], stream)
        canz.canz_mx_dequantize(s["back"], stream)
        return s["out"]
    if c["op"] == "linear":
        # forward, then backward
        canz.canz_mx_quantize(s["rx"], canz.MX_SCALE_FLOOR, stream)
        canz.canz_mx_product(s["groups"][:1], s["ws"], s["ws"].numel(), stream)
        canz.canz_mx_quantize(s["rdy"], canz.MX_SCALE_CEIL, stream)
        canz.canz_mx_product(s["groups"][1:], s["ws"], s["ws"].numel(), stream)
    else:
        canz.canz_mx_product(s["groups"], s["ws"], s["ws"].numel(), stream)
    return s["out"]


# ---------------------------------------------------------------- accounting and oracle

def work(case):
    size = dict(f32=4, bf16=2)
    image = 17.0 / 32          # bytes an element: a code of 4 bits and its share of a scale byte
    if case["op"] == "round":
        el = case["rows"] * case["cols"] * case["count"]
        sides = 2 if case["side"] == "both" else 1
        return {"bytes": el * (size[case["dtype"]] + case["noise"] + sides * (image + 2)), "flops": 0}
    if case["op"] == "product":
        ms, n, k = [int(m) for m in case["m"].split("+")], case["n"], case["k"]
        used = sum(m > 0 for m in ms)
        return {"bytes": sum(ms) * (k * size[case["x"]] + n * size[case["out"]]) + used * n * k * image, "flops": 2 * sum(ms) * n * k}
    t, n, k = case["tokens"], case["n"], case["k"]
    return {"bytes": t * k * 2 + t * n * 3 + 2 * n * k * image + t * n * 2 + t * k * 2 + n * k * 4, "flops": 6 * t * n * k}


def _rounded64(x, axis, scale, noise=None):
    """As the definition says, in 64 bits, by comparison with the values and the borders between them."""
    v = x.double() if axis == 1 else x.double().t().contiguous()
    u = None if noise is None else (noise if axis == 1 else noise.t().contiguous()).double()
    rows, k = v.shape
    pad = -k % BLOCK
    if pad:
        v = torch.cat([v, v.new_zeros(rows, pad)], 1)
        u = None if u is None else torch.cat([u, u.new_zeros(rows, pad)], 1)
    v = v.reshape(rows, (k + pad) // BLOCK, BLOCK)
    amax = v.abs().amax(2, keepdim=True)
    tiny = 2.0 ** -149
    e = torch.floor(torch.log2(amax.clamp(min=tiny))) - 2
    if scale == "ceil":
        e = torch.where(amax > 6 * torch.exp2(e), e + 1, e)
    unit = torch.exp2(e.clamp(min=-127))
    a = v.abs() / unit
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=x.device)
    if noise is None:
        border = (grid[1:] + grid[:-1]) / 2
        code = torch.bucketize(a, border)                                  # a tie stays below
        at = code.clamp(max=6)
        code = code + ((a == border[at]) & (at % 2 == 1)).long()           # ... unless that code is odd
    else:
        low = torch.bucketize(a, grid, right=True) - 1
        above = grid[(low + 1).clamp(max=7)]
        part = torch.where(low < 7, (a - grid[low]) / (above - grid[low]).clamp(min=0.5), torch.zeros_like(a))
        code = torch.where(torch.round(part * 256) + u.reshape(v.shape) >= 256, low + 1, low).clamp(max=7)
    q = (grid[code] * torch.sign(v) * unit).reshape(rows, k + pad)[:, :k]
    return q if axis == 1 else q.t()


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "round":
        sides = (1, 0) if case["side"] == "both" else (1,)
        u = s["noise"] or [None] * len(s["x"])
        return [[_rounded64(x, a, case["scale"], n).float() for x, n in zip(s["x"], u)] for a in sides]
    if case["op"] == "product":
        return [_rounded64(x, 1, "floor") @ w.double().t() for x, w in zip(s["x"], s["w"])]
    x, w, dy, u = s["x"], s["w"].double(), s["dy"], s["noise"]
    return dict(y=_rounded64(x, 1, "floor") @ w.t(), dx=_rounded64(dy, 1, "ceil", u) @ _rounded64(s["w"], 0, "floor"),
                dw=_rounded64(dy, 0, "ceil", u).t().contiguous() @ _rounded64(x, 0, "floor"))
