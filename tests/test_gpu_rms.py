"""``irms_quant`` against its definition in 64 bits."""
import pytest
import torch

from ff_util import TYPES, generator, ptr, rms_call, rms_check, stream
from paper_2006_11735_b200 import binding as B

pytestmark = pytest.mark.gpu


def _data(seed, m, d, dtype, residual=True, weight="same", pad=0):
    gen = generator(seed)
    rnd = lambda: torch.randn(m, d + pad, generator=gen, device="cuda").to(TYPES[dtype])[:, :d]
    x, r = rnd(), 2 * rnd() if residual else None
    g = None if weight is None else (1 + 0.3 * torch.randn(d, generator=gen, device="cuda")).to(TYPES[dtype] if weight == "same" else torch.float32)
    return x, r, g


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("d", [1, 7, 8, 64, 255, 256, 257, 513, 1000, 1024, 2048, 2056, 4096, 4100, 8192, 16384, 16392, 32768, 32776, 40001])
def test_widths(dtype, d):
    """Every instance of the kernel: rows in a warp, in a block, in registers and read twice; whole vectors and single elements."""
    for m in (1, 5):
        x, r, g = _data(d + m, m, d, dtype)
        q, scales, total = rms_call(x, r, g)
        rms_check(x, r, g, q, scales, total)
    B.iconv_check(stream())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("weight", [None, "same", "f32"])
@pytest.mark.parametrize("norm", [0, 1])
def test_forms(dtype, residual, weight, norm):
    for d in (520, 521):
        x, r, g = _data(3, 33, d, dtype, residual, weight)
        for with_sum in (True, False):
            q, scales, total = rms_call(x, r, g, norm=norm, with_sum=with_sum)
            rms_check(x, r, g, q, scales, total, norm=norm)


@pytest.mark.parametrize("pad", [1, 8])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_strides_leave_what_is_between_rows(pad, dtype):
    m, d = 19, 1024
    x, r, g = _data(5, m, d, dtype, pad=pad)
    q_store = torch.full((m + 1, d + 16), 77, dtype=torch.int8, device="cuda")
    sum_store = torch.full((m + 1, d + pad), 9, dtype=TYPES[dtype], device="cuda")
    scales = torch.full((m + 3,), 5.0, device="cuda")
    q, total = q_store[:m, :d], sum_store[:m, :d]
    rms_call(x, r, g, q=q, total=total, scales=scales)
    rms_check(x, r, g, q, scales[:m], total)
    assert (q_store[:, d:] == 77).all() and (q_store[m] == 77).all() and (sum_store[:, d:] == 9).all() and (sum_store[m] == 9).all()
    assert (scales[m:] == 5).all()


@pytest.mark.parametrize("d", [512, 513, 40000])
@pytest.mark.parametrize("into", ["x", "r"])
def test_sum_in_place(d, into):
    x, r, g = _data(7, 6, d, "bf16")
    want = rms_call(x, r, g)
    x2, r2 = x.clone(), r.clone()
    q, scales, total = rms_call(x2, r2, g, total=x2 if into == "x" else r2)
    assert torch.equal(q, want[0]) and torch.equal(scales, want[1]) and torch.equal(total, want[2])


@pytest.mark.parametrize("dtype", list(TYPES))
def test_rows_of_zeros_and_tiny_rows(dtype):
    x = torch.zeros(6, 300, dtype=TYPES[dtype], device="cuda")
    x[1, 5] = torch.finfo(TYPES[dtype]).tiny
    x[3] = 1.0
    if dtype != "f16":
        x[4, 7] = 2.0 ** -119
        x[5, 7] = 2.0 ** -120
    q, scales, total = rms_call(x)
    rms_check(x, None, None, q, scales, total)
    assert scales[0] == 0 and (q[0] == 0).all() and (q[3] == 127).all() and torch.equal(total, x)
    if dtype != "f16":
        assert q[4, 7] == 127 and q[5, 7] == 0
    q, scales, _ = rms_call(x[:1], eps=0.0)                 # nothing to divide by: still nothing
    assert scales[0] == 0 and (q == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 700, 40000])
def test_squares_that_do_not_fit(dtype, d):
    x = torch.randn(4, d, generator=generator(1), device="cuda") * torch.tensor([1e19, 1e25, 1e30, 3e37], device="cuda")[:, None]
    x = x.clamp(-3e38, 3e38).to(TYPES[dtype])
    q, scales, total = rms_call(x)
    rms_check(x, None, None, q, scales, total)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("d", [96, 1024, 1025, 40000])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_bad_value_spoils_its_row_alone(dtype, d, bad):
    x, r, g = _data(9, 5, d, dtype)
    clean = rms_call(x, r, g)
    x[2, d - 1] = bad
    for norm in (0, 1):
        q, scales, total = rms_call(x, r, g, norm=norm)
        assert torch.isnan(scales[2]) and (q[2] == 0).all()
        keep = [0, 1, 3, 4]
        assert torch.equal(q[keep], clean[0][keep]) and torch.isfinite(scales[keep]).all()
        assert torch.equal(total[keep], clean[2][keep])


def test_infinite_weight_and_infinities_that_cancel():
    x, r, g = _data(2, 3, 64, "f32")
    x[1, 3], r[1, 3] = float("inf"), float("-inf")          # NaN
    q, scales, _ = rms_call(x, r, g)
    assert torch.isnan(scales[1]) and not torch.isnan(scales[[0, 2]]).any()
    g[5] = float("inf")
    q, scales, _ = rms_call(x, r, g)
    assert torch.isnan(scales).all() and (q == 0).all()


def test_many_rows_and_offsets_past_32_bits():
    m, d = 70001, 96
    x, r, g = _data(4, m, d, "bf16")
    rms_check(x, r, g, *rms_call(x, r, g))
    far = torch.zeros(3, 1 << 30, dtype=torch.bfloat16, device="cuda")          # the last row starts 4 GB behind the first
    x = far[:, :d]
    x.copy_(torch.randn(3, d, generator=generator(6), device="cuda"))
    rms_check(x, None, None, *rms_call(x, with_sum=False), eps=1e-5)


def test_same_rows_in_another_call():
    x, r, g = _data(8, 40, 4096, "bf16")
    q, scales, total = rms_call(x, r, g)
    for i in (0, 17, 39):
        a, b, c = rms_call(x[i:i + 1], r[i:i + 1], g)
        assert torch.equal(a, q[i:i + 1]) and torch.equal(b, scales[i:i + 1]) and torch.equal(c, total[i:i + 1])


def test_captured_and_replayed_on_another_stream():
    x, r, g = _data(10, 12, 2048, "f16")
    q, scales, total = (torch.empty(12, 2048, dtype=torch.int8, device="cuda"), torch.empty(12, device="cuda"), torch.empty_like(x))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        rms_call(x, r, g, q=q, total=total, scales=scales)
        with torch.cuda.graph(graph, stream=side):
            rms_call(x, r, g, q=q, total=total, scales=scales)
    x.copy_(torch.randn(12, 2048, generator=generator(11), device="cuda"))
    graph.replay()
    torch.cuda.synchronize()
    rms_check(x, r, g, q, scales, total)


def test_no_rows():
    x = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    B.irms_quant(None, None, None, None, None, None, stream(), rows=0, width=64, dtype=B.BF16)
    assert rms_call(x)[0].shape == (0, 64) and ptr(x) is not None


@pytest.mark.parametrize("dtype,d", [("bf16", 4096), ("bf16", 4608), ("bf16", 9000), ("f16", 8192), ("bf16", 16384), ("f32", 2048), ("f32", 4100), ("f32", 8192), ("f16", 12008), ("f32", 16384),
                                     ("f32", 16380)])
@pytest.mark.parametrize("residual,weight,norm", [(True, "same", 1), (False, "f32", 1), (False, None, 0), (True, None, 1)])
def test_many_wide_rows(dtype, d, residual, weight, norm):
    """Rows that stream through shared memory, several for every block and not the same number for all; the same rows a block each."""
    m = 148 * 5 + 37
    x, r, g = _data(d, m, d, dtype, residual, weight)
    x[700, d - 1] = float("nan")
    q, scales, total = rms_call(x, r, g, norm=norm)
    keep = torch.arange(m, device="cuda") != 700
    assert torch.isnan(scales[700]) and (q[700] == 0).all()
    rms_check(x[keep], r[keep] if residual else None, g, q[keep], scales[keep], total[keep], norm=norm)
    for at in (0, 300, m - 20):
        a, b, c = rms_call(x[at:at + 20], r[at:at + 20] if residual else None, g, norm=norm)
        same = keep[at:at + 20]
        assert torch.equal(a, q[at:at + 20]) and torch.equal(c[same], total[at:at + 20][same])
        assert ((b - scales[at:at + 20]).abs()[same] <= 40 * 2.0 ** -24 * b[same]).all()       # (the squares are added in another order)
    B.iconv_check(stream())


def test_many_wide_rows_in_place_and_with_strides():
    m, d = 148 * 6 + 1, 5000
    x, r, g = _data(3, m, d, "bf16", pad=24)
    r = (2 * torch.randn(m, d + 8, generator=generator(4), device="cuda")).bfloat16()[:, :d]
    want = rms_call(x, r, g)
    rms_check(x, r, g, *want)
    for into in (x.clone(memory_format=torch.preserve_format), r.clone(memory_format=torch.preserve_format)):
        q_store = torch.full((m, d + 40), 77, dtype=torch.int8, device="cuda")
        first = into.shape == x.shape and torch.equal(into, x)
        q, scales, total = rms_call(into if first else x, r if first else into, g, q=q_store[:, :d], total=into)
        assert torch.equal(q, want[0]) and torch.equal(scales, want[1]) and torch.equal(total, want[2]) and (q_store[:, d:] == 77).all()
    B.iconv_check(stream())


def _anywhere(gen, m, d, stride, first, dtype):
    """A matrix whose first element is `first` elements into its memory, and the memory."""
    store = torch.randn(first + m * stride + 8, generator=gen, device="cuda").to(TYPES[dtype])
    return store.as_strided((m, d), (stride, 1), first), store


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("d", [9, 31, 33, 63, 100, 255, 257, 500, 511, 513, 1001, 2047, 2049, 4001, 4100, 8191, 16383, 16385])
def test_rows_that_start_anywhere(dtype, d):
    """Vectors cut out of aligned words: every phase of x, the residual, the sum and the weights, q in aligned rows, first and last rows of
    their memory; what lies around the rows stays."""
    gen = generator(d)
    for case, (px, pr, ps, fx, fr, fs, fg) in enumerate([(0, 0, 0, 0, 0, 0, 0), (1, 0, 3, 1, 2, 3, 5), (7, 2, 1, 5, 0, 7, 1), (0, 5, 8, 3, 3, 0, 2)]):
        for m in (1, 3, 10):
            x, _ = _anywhere(gen, m, d, d + px, fx, dtype)
            r, _ = _anywhere(gen, m, d, d + pr, fr, dtype)
            g = torch.randn(d + 8, generator=gen, device="cuda").to(TYPES[dtype])[fg:fg + d] if case != 2 else 1 + torch.rand(d, generator=gen, device="cuda")
            total, store = _anywhere(gen, m, d, d + ps, fs, dtype)
            before = store.clone()
            q_store = torch.full((m + 1, -(-d // 16) * 16 + 16), 77, dtype=torch.int8, device="cuda")
            q, scales, _ = rms_call(x, r, g, q=q_store[:m, :d], total=total)
            rms_check(x, r, g, q, scales, total)
            assert (q_store[:, d:] == 77).all() and (q_store[m] == 77).all()
            inside = torch.zeros_like(store, dtype=torch.bool)
            inside.as_strided((m, d), (d + ps, 1), fs).fill_(True)
            assert torch.equal(store[~inside], before[~inside])
            q, scales, _ = rms_call(x, norm=0, with_sum=False, q=q_store[:m, :d])
            rms_check(x, None, None, q, scales, None, norm=0)
    B.iconv_check(stream())


@pytest.mark.parametrize("into", ["x", "r"])
@pytest.mark.parametrize("d", [513, 2049, 4001])
def test_rows_that_start_anywhere_in_place(d, into):
    gen = generator(d)
    x, r = (_anywhere(gen, 300, d, d, first, "bf16")[0] for first in (0, 3))
    g = torch.randn(d, generator=gen, device="cuda").bfloat16()
    q = lambda: torch.empty(300, -(-d // 16) * 16, dtype=torch.int8, device="cuda")[:, :d]
    want = rms_call(x, r, g, q=q())
    x2, r2 = (torch.empty(300 * d + 3, dtype=torch.bfloat16, device="cuda").as_strided((300, d), (d, 1), first).copy_(t) for first, t in ((0, x), (3, r)))
    q2, scales, total = rms_call(x2, r2, g, q=q(), total=x2 if into == "x" else r2)
    assert torch.equal(q2, want[0]) and torch.equal(scales, want[1]) and torch.equal(total, want[2])


@pytest.mark.parametrize("dtype", list(TYPES))
def test_bad_values_beside_a_row_do_not_reach_it(dtype):
    """What a vector's words hold besides its own elements: NaN in the rows before and behind, and between rows."""
    m, d, stride = 7, 517, 521
    x, store = _anywhere(generator(5), m, d, stride, 1, dtype)
    clean = rms_call(x.clone(), q=torch.empty(m, 528, dtype=torch.int8, device="cuda")[:, :d])
    keep = torch.zeros_like(store, dtype=torch.bool)
    keep.as_strided((m, d), (stride, 1), 1)[::2].fill_(True)
    store[~keep] = float("nan")
    q, scales, total = rms_call(x, q=torch.empty(m, 528, dtype=torch.int8, device="cuda")[:, :d])
    assert torch.equal(q[::2], clean[0][::2]) and torch.equal(total[::2], clean[2][::2]) and torch.isnan(scales[1::2]).all()
    assert ((scales - clean[1]).abs()[::2] <= 40 * 2.0 ** -24 * scales[::2]).all()


@pytest.mark.parametrize("d", [1 << 24, (1 << 24) - 3])
def test_the_widest_row(d):
    x, _, g = _data(d, 1, d, "bf16", residual=False)
    rms_check(x, None, g, *rms_call(x, None, g))
    with pytest.raises(B.IconvError):
        B.irms_quant(ptr(x), None, None, None, ptr(x), ptr(x), stream(), rows=1, width=(1 << 24) + 1, dtype=B.BF16)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [40, 333, 700, 4104, 40000, 40001])
@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-12])
def test_squares_too_small_to_hold(dtype, d, eps):
    """Rows whose squares vanish in float, in part or all, beside an eps that does not cover them."""
    size = torch.tensor([1e-34, 1e-30, 1e-25, 1e-21, 1e-18, 1e-14, 1e-10, 1e-8], device="cuda")[:, None]
    x = (torch.randn(8, d, generator=generator(1), device="cuda") * size).to(TYPES[dtype])
    x[4:6, ::3] *= 1e-7                                     # (large and small ones in a row)
    for g in (None, (1e4 * torch.rand(d, generator=generator(2), device="cuda")).to(TYPES[dtype]), torch.full((d,), 1e30, device="cuda").to(TYPES[dtype])):
        q, scales, total = rms_call(x, None, g, eps=eps)
        rms_check(x, None, g, q, scales, total, eps=float(torch.tensor(eps)))      # (eps is a float)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 333, 700, 40000])
def test_large_rows_times_small_weights(dtype, d):
    x = (torch.randn(3, d, generator=generator(1), device="cuda") * torch.tensor([1e19, 1e25, 1e37], device="cuda")[:, None]).to(TYPES[dtype])
    g = torch.full((d,), 2e-31, device="cuda").to(TYPES[dtype])
    q, scales, total = rms_call(x, None, g)
    rms_check(x, None, g, q, scales, total)


def test_many_small_wide_rows():
    m, d = 148 * 4 + 3, 8192
    x = (torch.randn(m, d, generator=generator(1), device="cuda") * 10.0 ** -torch.randint(10, 35, (m, 1), generator=generator(2), device="cuda")).bfloat16()
    rms_check(x, None, None, *rms_call(x, eps=0.0), eps=0.0)


FIRST = """
import torch
from paper_2006_11735_b200 import binding as B
x = torch.randn(%(m)d, %(d)d, device="cuda").bfloat16()
q, scales = torch.empty(%(m)d, %(d)d, dtype=torch.int8, device="cuda"), torch.empty(%(m)d, device="cuda")
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    B.irms_quant(x.data_ptr(), None, None, None, q.data_ptr(), scales.data_ptr(), torch.cuda.current_stream().cuda_stream, rows=%(m)d, width=%(d)d, dtype=B.BF16)
graph.replay()
torch.cuda.synchronize()
got = q.float() * scales[:, None]
want = x.float() * (x.float().pow(2).mean(1, keepdim=True) + 1e-5).rsqrt()
assert ((got - want).abs() <= 0.51 * scales[:, None]).all()
print("captured first")
"""


@pytest.mark.parametrize("m,d", [(3, 64), (3, 333), (700, 8192)])
def test_the_first_call_of_a_process_is_captured(m, d):
    import subprocess
    import sys
    done = subprocess.run([sys.executable, "-c", FIRST % dict(m=m, d=d)], capture_output=True, text=True, timeout=120, cwd=B.__file__.rsplit("/", 2)[0])
    assert done.returncode == 0 and "captured first" in done.stdout, done.stderr[-2000:]


@pytest.mark.parametrize("m,d,step", [(5, 4000, (1 << 30) + 1), (5, 20001, (1 << 30) + 1), (700, 8192, 1 << 23)])
def test_far_rows_of_every_kind(m, d, step):
    """Cut out of words, single elements, streams: more than 4 GB from the first row to the last, in q too."""
    gen = generator(d)
    x = torch.empty(m * step, dtype=torch.bfloat16, device="cuda").view(m, step)[:, :d]
    x.copy_(torch.randn(m, d, generator=gen, device="cuda"))
    q = torch.empty(m * step, dtype=torch.int8, device="cuda").view(m, step)[:, :d]
    q, scales, total = rms_call(x, q=q, total=x)
    rms_check(x, None, None, q, scales, total)


def test_very_many_rows():
    x, r, g = _data(5, (1 << 25) + 1, 3, "bf16")
    rms_check(x, r, g, *rms_call(x, r, g))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [1, 8, 9, 64, 333, 1024, 4104, 40000, 40001])
@pytest.mark.parametrize("eps", [1e30, 1e36, 1e38, 3e38])
def test_large_rows_beside_a_large_eps(dtype, d, eps):
    """Squares whose sum, or whose mean with eps, a float cannot hold, and an eps of their size."""
    size = torch.tensor([1e15, 1e17, 3e17, 1e18, 3e18, 1e19, 1.8e19, 1e20], device="cuda")[:, None]
    sign = torch.where(torch.rand(8, d, generator=generator(1), device="cuda") < 0.5, -1.0, 1.0)
    x = (sign * (0.5 + 0.5 * torch.rand(8, d, generator=generator(2), device="cuda")) * size).to(TYPES[dtype])
    for g in (None, torch.rand(d, generator=generator(3), device="cuda").to(TYPES[dtype])):
        q, scales, total = rms_call(x, None, g, eps=eps)
        rms_check(x, None, g, q, scales, total, eps=float(torch.tensor(eps)))


def test_many_large_wide_rows_beside_a_large_eps():
    m, d = 148 * 4 + 3, 8192
    x = (torch.randn(m, d, generator=generator(1), device="cuda") * 10.0 ** torch.randint(14, 22, (m, 1), generator=generator(2), device="cuda")).bfloat16()
    for eps in (1e36, 3e38):
        rms_check(x, None, None, *rms_call(x, eps=eps), eps=float(torch.tensor(eps)))
