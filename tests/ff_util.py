"""Plain forms, in 64 bits, of the feed-forward sublayer's operators (``irms_quant``, ``imat_forward``) and the bounds their results are
held to."""
import math

import torch

from paper_2006_11735_b200 import binding as B

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = 2.0 ** -24                               # half a step of float, relative


def stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def ptr(t):
    return None if t is None else t.data_ptr()


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def half_step(dtype, value):
    """What rounding `value` (64 bits) to dtype may add."""
    info = torch.finfo(dtype)
    return (value.abs() * (info.eps / 2)).clamp_min(info.tiny * info.eps / 2)


# ---- irms_quant


def rms_call(x, r=None, g=None, *, norm=1, eps=1e-5, with_sum=True, q=None, total=None, scales=None):
    m, d = x.shape
    q = torch.full((m, d), 77, dtype=torch.int8, device="cuda") if q is None else q
    scales = torch.full((m,), -1.0, dtype=torch.float32, device="cuda") if scales is None else scales
    if total is None and with_sum:
        total = torch.full_like(x, 9, memory_format=torch.contiguous_format)
    code = {v: B.DTYPE_CODE[k] for k, v in TYPES.items()}
    B.irms_quant(ptr(x), ptr(r), ptr(g), ptr(total), ptr(q), ptr(scales), stream(), rows=m, width=d, dtype=code[x.dtype],
                 weight_dtype=code[g.dtype] if g is not None else code[x.dtype], eps=eps, norm=norm, x_stride=x.stride(0),
                 residual_stride=r.stride(0) if r is not None else 0, sum_stride=total.stride(0) if total is not None else 0, q_stride=q.stride(0))
    return q, scales, total


def rms_check(x, r, g, q, scales, total, *, norm=1, eps=1e-5):
    """Rows of finite values.  127 * v / max|v| in float: the sum and the product with the weight (2 roundings, and 2 in the maximum), the
    quotient and the product: 6 U of at most 127.  The scale: those 2 of the maximum, 1 / 127 and two products, and half of the mean's error:
    two roundings of s, one of the weight 1 / width, and at most one per addition (a thread's share, 5 shuffles, 31 warps)."""
    s = x.double() if r is None else x.double() + r.double()
    v = s if g is None else s * g.double()
    top = v.abs().amax(1, keepdim=True)
    some = top[:, 0] >= 2.0 ** -119
    t = torch.where(top > 0, 127 * v / top, torch.zeros_like(v))
    off = (q.double() - t).abs()
    assert (off[some] <= 0.5 + 127 * 6.5 * U).all(), float(off[some].max())
    assert (q[~some] == 0).all() and (scales[~some] == 0).all()
    want = top[:, 0] / 127
    if norm:
        want = want / (s.pow(2).mean(1) + eps).sqrt()
    adds = x.shape[1] / 1024 + 32 + 36
    bound = want * (2 + 1 + 2 + 4 + (adds + 4) / 2) * U
    assert ((scales.double() - want).abs()[some] <= bound[some]).all(), float(((scales.double() - want).abs() / want)[some].max() / U)
    if total is not None:
        assert ((total.double() - s).abs() <= half_step(x.dtype, s) + s.abs() * U).all()


# ---- imat_forward


def act64(name, y):
    if name == "relu":
        return torch.where(y < 0, torch.zeros_like(y), y)
    if name == "silu":
        return y * torch.sigmoid(y)
    if name == "gelu":
        return y * 0.5 * torch.special.erfc(-y / math.sqrt(2))
    if name == "gelu_tanh":
        return y * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3))
    return y


def act_bound(name, y, before):
    """Error of the activation in float at `y` whose argument is off by `before`: the slope (at most 1.13), then the function's own.
    y / (1 + exp(-z)): exp.approx is off by 2 + 1.173 |z| steps (2 U each) of a term that is (1 - sigmoid) of the sum, the division by 2 steps, the
    addition, z and the coefficients by 4 U times |z| slopes; erff by 2 steps of at most 1, the sums and products by 3 U."""
    if name in ("none", "relu"):
        return before
    if name == "gelu":
        return 1.13 * before + y.abs() * 8 * U
    z = y if name == "silu" else 2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)
    return 1.13 * before + act64(name, y).abs() * ((2 + 1.173 * z.abs()) * 2 + 5 * z.abs() + 8) * U * torch.sigmoid(-z) + act64(name, y).abs() * 6 * U + 2.0 ** -126


class Filter:
    """int8 weights with scales and, perhaps, a bias."""

    def __init__(self, gen, n, k, bias=True, w_stride=None, w=None):
        self.store = torch.full((n, w_stride or k), 99, dtype=torch.int8, device="cuda")
        self.w = self.store[:, :k]
        self.w.copy_(torch.randint(-128, 128, (n, k), generator=gen, device="cuda", dtype=torch.int16) if w is None else w)
        self.scales = (torch.rand(n, generator=gen, device="cuda") + 0.5) / (75.0 * math.sqrt(k))
        self.bias = 0.5 * torch.randn(n, generator=gen, device="cuda") if bias else None

    def sums(self, x):
        return x.double() @ self.w.double().t()

    def value(self, x, sx):
        """(value in 64 bits, bound of its error in float): the sum, its scale and the whole product are rounded, the last with the bias."""
        y = self.sums(x) * sx.double()[:, None] * self.scales.double()
        if self.bias is None:
            return y, y.abs() * 3 * U
        return y + self.bias.double(), y.abs() * 2 * U + (y + self.bias.double()).abs() * U


class Plan:
    def __init__(self, dtype, f, up=None, act="none"):
        n, k = f.w.shape
        self.n, self.k, self.dtype, self.act, self.f, self.up = n, k, TYPES[dtype], act, f, up
        self.handle = B.imat_plan(n=n, k=k, out_dtype=B.DTYPE_CODE[dtype], act=B.ACT_CODE[act], weights=ptr(f.w), w_stride=f.store.stride(0),
                                  scales=ptr(f.scales), bias=ptr(f.bias), up_weights=ptr(up.w) if up else None, up_scales=ptr(up.scales) if up else None,
                                  up_bias=ptr(up.bias) if up else None, stream=stream())

    def __call__(self, x, sx, r=None, out=None):
        m = x.shape[0]
        out = torch.full((m, self.n), 3.0, dtype=self.dtype, device="cuda") if out is None else out
        B.imat_forward(self.handle, m, ptr(x), x.stride(0), ptr(sx), ptr(r), r.stride(0) if r is not None else 0, ptr(out), out.stride(0), stream())
        return out

    def want(self, x, sx, r=None):
        """(value, bound) of every output."""
        y, e = self.f.value(x, sx)
        e, y = act_bound(self.act, y, e), act64(self.act, y)
        if self.up:
            u, eu = self.up.value(x, sx)
            y, e = y * u, e * (u.abs() + eu) + y.abs() * eu + (y * u).abs() * U
        if r is not None:
            y = y + r.double()
            e = e + y.abs() * U
        return y, e + half_step(self.dtype, y) + e * torch.finfo(self.dtype).eps

    def check(self, x, sx, out, r=None):
        y, e = self.want(x, sx, r)
        off = (out.double() - y).abs()
        assert (off <= e).all(), "off by %.3g bounds at %s" % (float((off / e).max()), divmod(int((off / e).argmax()), self.n))

    def describe(self, rows):
        return B.imat_plan_describe(self.handle, rows)

    def __del__(self):
        if getattr(self, "handle", None):
            B.imat_plan_destroy(self.handle)


def rows8(gen, m, k, stride=None):
    """8-bit rows, the whole range, in rows that start on 16 bytes."""
    store = torch.full((m, stride or -(-k // 16) * 16), 55, dtype=torch.int8, device="cuda")
    store[:, :k] = torch.randint(-128, 128, (m, k), generator=gen, device="cuda", dtype=torch.int16).to(torch.int8)
    return store[:, :k], torch.rand(m, generator=gen, device="cuda") / 60.0
