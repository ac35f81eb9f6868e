"""Performance cases of the operators of a transformer's feed-forward sublayer in 8 bits.

"norm": the residual's addition, the root-mean-square norm and 8-bit rows with one scale each (``irms_quant``; with ``norm`` 0 the
8-bit rows alone).  "product": int8 rows times int8 weights with scales, bias, activation and residual (``imat_forward``).  "gated":
both projections of a gated feed-forward block, the activation and the product (``imat_forward`` of a plan with two filters).
"ff": the sublayer that they make together.

Whatever is held in 8 bits is returned as the bfloat16 values that it stands for.
"""
import math

import torch

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-5

own = False                                      # True: run() makes the library's calls instead of computing the plain forms


def _norm(name, rows, width, dtype, residual, norm=1):
    return {"name": name, "kind": "norm", "rows": rows, "width": width, "dtype": dtype, "residual": residual, "norm": norm}


def _mat(name, kind, rows, k, n, dtype, act, bias, residual):
    return {"name": name, "kind": kind, "rows": rows, "k": k, "n": n, "dtype": dtype, "act": act, "bias": bias, "residual": residual}


def listed():
    return [
        # one token on its way into a layer
        _norm("norm_1x4096", 1, 4096, "bf16", True),
        # a long prompt, or a batch of them
        _norm("norm_8192x4096", 8192, 4096, "bf16", True),
        # odd rows of an odd width in 32 bits, the first layer (nothing to add yet)
        _norm("norm_777x2501_f32", 777, 2501, "f32", False),
        # the inner activations of a feed-forward block on their way to the second product
        _norm("rows_4096x16384", 4096, 16384, "bf16", False, norm=0),
        # one token through an output projection
        _mat("product_1x4096x4096", "product", 1, 4096, 4096, "bf16", "none", False, True),
        # a batch of sequences, one token each, through a wide layer; 32-bit results
        _mat("product_64x8192x8192_f32", "product", 64, 8192, 8192, "f32", "none", True, False),
        # an ungated block's first projection at sizes that divide by nothing
        _mat("product_333x1000x2049_gelu", "product", 333, 1000, 2049, "f16", "gelu", True, False),
        # a long prompt through a feed-forward block's second projection
        _mat("product_8192x16384x4096", "product", 8192, 16384, 4096, "bf16", "none", False, True),
        # one token through the gated projections
        _mat("gated_1x4096x16384", "gated", 1, 4096, 16384, "bf16", "silu", False, False),
        # a few sequences' tokens, odd sizes, biases, the tanh form
        _mat("gated_77x1500x2731_gelu", "gated", 77, 1500, 2731, "f16", "gelu_tanh", True, False),
        # a long prompt through the gated projections
        _mat("gated_4096x4096x16384", "gated", 4096, 4096, 16384, "bf16", "silu", False, False),
        # the sublayer as a service runs it for sixteen sequences at a time
        {"name": "ff_16x4096x16384", "kind": "ff", "rows": 16, "k": 4096, "n": 16384, "dtype": "bf16", "act": "silu"},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(["norm", "product", "product", "gated", "gated", "ff"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind == "norm":
        width = _log(rng, 64, 16384)
        return {"kind": kind, "rows": _log(rng, 1, min(8192, (1 << 25) // width)), "width": width, "dtype": dtype, "residual": rng.random() < 0.6,
                "norm": int(rng.random() < 0.7)}
    k, n = _log(rng, 128, 16384), _log(rng, 128, 16384)
    if rng.random() < 0.5:                       # as often sizes that tiles divide
        k, n = -(-k // 128) * 128, -(-n // 128) * 128
    rows = _log(rng, 1, min(8192, max(2, (1 << 37) // (k * n))))
    if kind == "ff":
        return {"kind": kind, "rows": rows, "k": min(k, 8192), "n": n, "dtype": rng.choice(["bf16", "f16"]), "act": rng.choice(["silu", "gelu_tanh"])}
    return {"kind": kind, "rows": rows, "k": k, "n": n, "dtype": dtype, "act": rng.choice(["none", "relu", "silu", "gelu", "gelu_tanh"]),
            "bias": rng.random() < 0.5, "residual": kind == "product" and rng.random() < 0.6}


def work(case):
    if case["kind"] == "norm":
        e = case["rows"] * case["width"]
        t = TYPES[case["dtype"]].itemsize
        return {"bytes": e * (t + (2 * t if case["residual"] else 0) + 1) + 4 * case["rows"] + (t * case["width"] if case["norm"] else 0), "flops": 6 * e}
    m, k, n, t = case["rows"], case["k"], case["n"], TYPES[case["dtype"]].itemsize
    if case["kind"] == "ff":                     # x, residual, sum, out; three filters with their scales
        return {"bytes": 4 * t * m * k + 3 * n * k + 4 * (2 * n + k) + t * k, "flops": 6 * m * n * k}
    mats = 2 if case["kind"] == "gated" else 1
    return {"bytes": m * k + 4 * m + mats * (n * k + 4 * n + (4 * n if case["bias"] else 0)) + m * n * t * (2 if case["residual"] else 1),
            "flops": 2 * mats * m * n * k}


def _weights(gen, n, k):
    """int8 rows as a quantiser leaves them, and their scales (of weights of variance 1 / k)."""
    q = torch.randn(n, k, generator=gen, device=DEVICE).mul_(30.0).round_().clamp_(-127, 127).to(torch.int8)
    return q, (torch.rand(n, generator=gen, device=DEVICE) * 0.5 + 0.75) / (30.0 * math.sqrt(k))


def _rows(gen, m, k):
    """8-bit activations with their scales, in rows that start on 16 bytes."""
    q = torch.zeros(m, -(-k // 16) * 16, dtype=torch.int8, device=DEVICE)
    q[:, :k] = torch.randn(m, k, generator=gen, device=DEVICE).mul_(33.0).round_().clamp_(-127, 127).to(torch.int8)
    return q, (torch.rand(m, generator=gen, device=DEVICE) + 0.5) / 33.0


def _stream():
    return torch.cuda.current_stream().cuda_stream


class _Plan:
    """A planned product (its weights laid out once), released with the state that holds it."""

    def __init__(self, dtype, act, w, up=None, bias=None, up_bias=None):
        from paper_2006_11735_b200 import binding as B
        self.B, self.handle = B, None
        n, k = w[0].shape
        ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        self.handle = B.imat_plan(n=n, k=k, out_dtype=B.DTYPE_CODE[dtype], act=B.ACT_CODE[act], weights=ptr(w[0]), scales=ptr(w[1]), bias=ptr(bias),
                                  up_weights=ptr(up[0]) if up else None, up_scales=ptr(up[1]) if up else None, up_bias=ptr(up_bias), stream=_stream())

    def __del__(self):
        if self.handle is not None:
            self.B.imat_plan_destroy(self.handle)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    dt = TYPES[case["dtype"]]
    s = dict(case)
    randn = lambda *shape: torch.randn(*shape, generator=gen, device=DEVICE)  # noqa: E731
    if case["kind"] == "norm":
        m, d = case["rows"], case["width"]
        s["x"] = randn(m, d).to(dt)
        s["r"] = (2 * randn(m, d)).to(dt) if case["residual"] else None
        s["g"] = (1 + 0.2 * randn(d)).to(dt) if case["norm"] else None
        s["sum"] = torch.empty(m, d, dtype=dt, device=DEVICE) if case["residual"] else None
        s["q"] = torch.empty(m, -(-d // 16) * 16, dtype=torch.int8, device=DEVICE)
        s["scale"] = torch.empty(m, dtype=torch.float32, device=DEVICE)
        s["value"] = torch.empty(m, d, dtype=torch.bfloat16, device=DEVICE)
        return s
    m, k, n = case["rows"], case["k"], case["n"]
    if case["kind"] == "ff":
        s["x"], s["r"], s["g"] = randn(m, k).to(dt), (2 * randn(m, k)).to(dt), (1 + 0.2 * randn(k)).to(dt)
        s["w"], s["up"], s["down"] = _weights(gen, n, k), _weights(gen, n, k), _weights(gen, k, n)
        if own:
            s["plan"] = _Plan(case["dtype"], case["act"], s["w"], s["up"])
            s["plan2"] = _Plan(case["dtype"], "none", s["down"])
            s["sum"], s["out"], s["h"] = torch.empty_like(s["x"]), torch.empty_like(s["x"]), torch.empty(m, n, dtype=dt, device=DEVICE)
            s["q"], s["q2"] = (torch.empty(m, -(-d // 16) * 16, dtype=torch.int8, device=DEVICE) for d in (k, n))
            s["scale"], s["scale2"] = (torch.empty(m, dtype=torch.float32, device=DEVICE) for _ in range(2))
        return s
    s["q"], s["scale"] = _rows(gen, m, k)
    s["w"] = _weights(gen, n, k)
    s["up"] = _weights(gen, n, k) if case["kind"] == "gated" else None
    s["b"] = 0.3 * randn(n) if case["bias"] else None
    s["up_b"] = 0.3 * randn(n) if case["bias"] and s["up"] else None
    s["r"] = randn(m, n).to(dt) if case["residual"] else None
    s["out"] = torch.empty(m, n, dtype=dt, device=DEVICE)
    if own:
        s["plan"] = _Plan(case["dtype"], case["act"], s["w"], s["up"], s["b"], s["up_b"])
    return s


# ---- the plain forms, in 32 bits


def _act(name, y):
    if name == "relu":
        return torch.where(y > 0, y, torch.zeros_like(y))
    if name == "silu":
        return y / (1 + torch.exp(-y))
    if name == "gelu":
        return 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)))
    return y


def _plain_quant(x, r, g, norm):
    """(x + r in x's type, the rows as whole numbers in 32 bits, their scales)"""
    s = x.float() if r is None else x.float() + r.float()
    v = s * g.float() if norm else s
    top = v.abs().amax(1, keepdim=True)
    # floor(t + 1/2) with the sum in 64 bits: in 32 it would take a value next to the border across it
    q = torch.floor((v * torch.where(top > 0, 127 / top, torch.zeros_like(top))).double() + 0.5).float()
    scale = top / 127
    if norm:
        scale = scale * torch.rsqrt((s * s).mean(1, keepdim=True) + EPS)
    return s.to(x.dtype), q, scale


def _plain_product(q, scale, w, b):
    y = (q @ w[0].float().t()) * scale * w[1]
    return y if b is None else y + b


def _plain(s):
    dt = TYPES[s["dtype"]]
    if s["kind"] == "norm":
        total, q, scale = _plain_quant(s["x"], s["r"], s["g"], s["norm"])
        out = {"value": (q * scale).to(torch.bfloat16), "scale": scale[:, 0]}
        return out if s["r"] is None else dict(out, sum=total)
    if s["kind"] == "ff":
        total, q, scale = _plain_quant(s["x"], s["r"], s["g"], 1)
        h = (_act(s["act"], _plain_product(q, scale, s["w"], None)) * _plain_product(q, scale, s["up"], None)).to(dt)
        _, q, scale = _plain_quant(h, None, None, 0)
        return {"sum": total, "out": (_plain_product(q, scale, s["down"], None) + total.float()).to(dt)}
    x, scale = s["q"][:, :s["k"]].float(), s["scale"][:, None]
    y = _act(s["act"], _plain_product(x, scale, s["w"], s["b"]))
    if s["up"]:
        y = y * _plain_product(x, scale, s["up"], s["up_b"])
    return (y if s["r"] is None else y + s["r"].float()).to(dt)


# ---- the library's calls


def _own(s):
    from paper_2006_11735_b200 import binding as B
    stream = _stream()
    code = B.DTYPE_CODE[s["dtype"]]
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    if s["kind"] == "norm":
        B.irms_quant(ptr(s["x"]), ptr(s["r"]), ptr(s["g"]), ptr(s["sum"]), ptr(s["q"]), ptr(s["scale"]), stream, rows=s["rows"], width=s["width"], dtype=code,
                     weight_dtype=code, eps=EPS, norm=s["norm"], q_stride=s["q"].stride(0))
        torch.mul(s["q"][:, :s["width"]], s["scale"][:, None], out=s["value"])
        out = {"value": s["value"], "scale": s["scale"]}
        return out if s["r"] is None else dict(out, sum=s["sum"])
    if s["kind"] == "ff":
        m, k, n = s["rows"], s["k"], s["n"]
        B.irms_quant(ptr(s["x"]), ptr(s["r"]), ptr(s["g"]), ptr(s["sum"]), ptr(s["q"]), ptr(s["scale"]), stream, rows=m, width=k, dtype=code,
                     weight_dtype=code, eps=EPS, q_stride=s["q"].stride(0))
        B.imat_forward(s["plan"].handle, m, ptr(s["q"]), s["q"].stride(0), ptr(s["scale"]), None, 0, ptr(s["h"]), n, stream)
        B.irms_quant(ptr(s["h"]), None, None, None, ptr(s["q2"]), ptr(s["scale2"]), stream, rows=m, width=n, dtype=code, norm=0, q_stride=s["q2"].stride(0))
        B.imat_forward(s["plan2"].handle, m, ptr(s["q2"]), s["q2"].stride(0), ptr(s["scale2"]), ptr(s["sum"]), k, ptr(s["out"]), k, stream)
        return {"sum": s["sum"], "out": s["out"]}
    B.imat_forward(s["plan"].handle, s["rows"], ptr(s["q"]), s["q"].stride(0), ptr(s["scale"]), ptr(s["r"]), s["n"] if s["residual"] else 0, ptr(s["out"]),
                   s["n"], stream)
    return s["out"]


def run(state):
    return _own(state) if own else _plain(state)


# ---- the definitions, in 64 bits


def _exact_act(name, y):
    if name == "none":
        return y
    if name == "relu":
        return y.clamp_min(0)
    if name == "silu":
        return y * torch.sigmoid(y)
    if name == "gelu":
        return y * 0.5 * torch.special.erfc(-y / math.sqrt(2))
    return y * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3))


def _exact_rows(s, g, norm):
    """What the 8-bit rows of the 64-bit sums `s` stand for, and their scales."""
    y = s if not norm else s / (s.pow(2).mean(dim=1, keepdim=True) + EPS).sqrt() * g.double()
    scale = y.abs().max(dim=1, keepdim=True).values / 127
    return torch.nan_to_num(torch.floor(y / scale + 0.5)) * scale, scale


def _exact_product(x, w, b):
    y = torch.einsum("mk,nk->mn", x, w[0].double() * w[1].double()[:, None])
    return y if b is None else y + b.double()


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm":
        total = s["x"].double() + (s["r"].double() if case["residual"] else 0)
        value, scale = _exact_rows(total, s["g"], case["norm"])
        out = {"value": value, "scale": scale.flatten()}
        return dict(out, sum=total) if case["residual"] else out
    if case["kind"] == "ff":
        total = s["x"].double() + s["r"].double()
        x, _ = _exact_rows(total, s["g"], 1)
        h, _ = _exact_rows(_exact_act(case["act"], _exact_product(x, s["w"], None)) * _exact_product(x, s["up"], None), None, 0)
        return {"sum": total, "out": _exact_product(h, s["down"], None) + total}
    x = s["q"][:, :case["k"]].double() * s["scale"].double()[:, None]
    y = _exact_act(case["act"], _exact_product(x, s["w"], s["b"]))
    if case["kind"] == "gated":
        y = y * _exact_product(x, s["up"], s["up_b"])
    return y + s["r"].double() if case["residual"] else y
