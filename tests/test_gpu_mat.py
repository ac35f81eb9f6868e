"""``imat_forward`` against its definition in 64 bits."""
import pytest
import torch

from ff_util import TYPES, Filter, Plan, generator, ptr, rms_call, rms_check, rows8, stream
from paper_2006_11735_b200 import binding as B

pytestmark = pytest.mark.gpu

ACTS = ["none", "relu", "silu", "gelu", "gelu_tanh"]


def _case(seed, m, k, n, dtype="bf16", act="none", gated=False, bias=True, residual=False):
    gen = generator(seed)
    plan = Plan(dtype, Filter(gen, n, k, bias), Filter(gen, n, k, bias) if gated else None, act)
    x, sx = rows8(gen, m, k)
    r = torch.randn(m, n, generator=gen, device="cuda").to(TYPES[dtype]) if residual else None
    return plan, x, sx, r


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("k", [1, 16, 100, 128, 129, 1000, 4096])
@pytest.mark.parametrize("n", [1, 63, 65, 128, 300])
def test_sizes(gated, k, n):
    for m in (1, 3, 17, 130):
        plan, x, sx, _ = _case(m + n + k, m, k, n, "f32", gated=gated)
        plan.check(x, sx, plan(x, sx))
    B.iconv_check(stream())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("m,k,kernel", [(2, 640, "stream"), (11, 640, "stream"), (40, 640, "few"), (100, 4096, "few"), (2100, 640, "bulk")])
def test_epilogues(dtype, act, gated, m, k, kernel):
    """Every kernel (of the few-tile one the forms that share a reduction and that do not) with every activation, type and form."""
    plan, x, sx, r = _case(1, m, k, 2336, dtype, act, gated, residual=not gated)
    assert plan.describe(m).startswith(kernel)
    if kernel == "few" and not gated:
        assert ("split 1," in plan.describe(m)) == (m == 40)
    plan.check(x, sx, plan(x, sx, r), r)
    if not gated:
        plan.check(x, sx, plan(x, sx))
    B.iconv_check(stream())


@pytest.mark.parametrize("m", list(range(1, 34)) + [47, 48, 49, 63, 64, 65, 96, 127, 128, 129, 160, 200, 255, 256, 257, 383, 385])
def test_rows(m):
    """Every number of rows on the way through the tile sizes, with the reduction shared among a cluster's blocks (few channels) and not."""
    for k, n in ((2048, 200), (96, 4000)):
        plan, x, sx, r = _case(m, m, k, n, "bf16", residual=True)
        plan.check(x, sx, plan(x, sx, r), r)
    plan, x, sx, _ = _case(m, m, 1100, 130, "f16", "silu", gated=True)
    plan.check(x, sx, plan(x, sx))
    B.iconv_check(stream())


@pytest.mark.parametrize("m,k,n,gated", [(4096, 512, 2048, False), (2049, 1000, 5000, False), (5000, 130, 2600, False), (3000, 384, 2500, True), (2300, 256, 1990, True),
                                         (70000, 128, 256, False)])
def test_many_rows(m, k, n, gated):
    """The bulk kernel: whole and ragged tiles, an odd number of channel tiles, more than one group of token tiles, several tiles a pair."""
    plan, x, sx, r = _case(m, m, k, n, "bf16", "silu" if gated else "none", gated, residual=not gated)
    assert plan.describe(m).startswith("bulk")
    plan.check(x, sx, plan(x, sx, r), r)
    B.iconv_check(stream())


def test_largest_sums():
    """131071 products of -128 and -128: the largest sum that the plan admits."""
    k = 131071
    gen = generator(3)
    f = Filter(gen, 130, k, bias=False, w=torch.full((130, k), -128, device="cuda", dtype=torch.int16))
    plan = Plan("f32", f)
    for m in (2, 20):
        x, sx = rows8(gen, m, k)
        x.fill_(-128)
        out = plan(x, sx)
        assert (f.sums(x) == 128.0 * 128 * k).all()
        plan.check(x, sx, out)


@pytest.mark.parametrize("m", [3, 2200])
def test_strides_leave_what_is_between_rows(m):
    k, n, gen = 200, 1003, generator(4)
    plan = Plan("bf16", Filter(gen, n, k, w_stride=k + 5), act="relu")
    if m > 3:
        plan = Plan("bf16", Filter(gen, 2700, k, w_stride=k + 8), act="relu")
        n = 2700
    x, sx = rows8(gen, m, k, stride=k + 24)
    sx = torch.cat([sx, torch.full((5,), float("nan"), device="cuda")])      # nobody's scales
    store = torch.full((m + 1, n + 9), 3.0, dtype=torch.bfloat16, device="cuda")
    r_store = torch.randn(m, n + 3, generator=gen, device="cuda").bfloat16()
    out, r = store[:m, 1:n + 1], r_store[:, 2:n + 2]
    plan(x, sx, r, out)
    plan.check(x, sx[:m], out, r)
    assert (store[:, 0] == 3).all() and (store[:, n + 1:] == 3).all() and (store[m] == 3).all()


@pytest.mark.parametrize("m", [5, 2200])
def test_residual_in_place(m):
    plan, x, sx, r = _case(6, m, 256, 2500, "bf16", "gelu", residual=True)
    want = plan(x, sx, r)
    out = r.clone()
    plan(x, sx, out, out)
    assert torch.equal(out, want)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_a_row_is_the_same_in_any_call(gated, dtype):
    plan, x, sx, r = _case(7, 2500, 1030, 2500, dtype, "silu", gated, residual=not gated)
    whole = plan(x, sx, r)
    assert plan.describe(2500).startswith("bulk")
    for m, kernel in ((1, "stream"), (9, "stream"), (64, "few"), (100, "few")):
        assert plan.describe(m).startswith(kernel)
        for at in (0, 1200):
            some = plan(x[at:at + m], sx[at:at + m].clone(), r[at:at + m] if r is not None else None)
            assert torch.equal(some, whole[at:at + m]), (m, at)


@pytest.mark.parametrize("m", [4, 2400])
@pytest.mark.parametrize("gated", [False, True])
def test_bad_scales_and_residuals_stay_where_they_are(m, gated):
    plan, x, sx, r = _case(8, m, 300, 2300, "f32", gated=gated, residual=not gated)
    clean = plan(x, sx, r)
    sx[1], sx[2] = float("nan"), float("inf")
    plan.f.scales[7] = float("nan")
    spoilt = Plan("f32", plan.f, plan.up)
    if r is not None:
        r[3, 11] = float("-inf")
    out = spoilt(x, sx, r)
    assert torch.isnan(out[1]).all() and torch.isnan(out[:, 7]).all() and not torch.isfinite(out[2]).any()
    rows = torch.tensor([i for i in range(m) if i not in (1, 2)], device="cuda")
    same = out[rows] == clean[rows]
    same[:, 7] = True
    if r is not None:
        assert out[3, 11] == float("-inf")
        same[1, 11] = True
    assert same.all()


def test_steep_activations():
    """Arguments from one end of float to the other: the exponentials run out of range on either side."""
    n = 64
    f = Filter(generator(0), n, 16, bias=False, w=torch.zeros(n, 16, device="cuda", dtype=torch.int16))
    at = [0.0, 1e-30, 1e-5, 0.5, 3, 10, 40, 80, 86, 87.5, 88, 89, 100, 200, 1e4, 1e18, 1e30, 3e38]
    f.bias = torch.tensor([s * v for v in at for s in (1, -1)] + [1.0] * (n - 2 * len(at)), device="cuda")
    x, sx = rows8(generator(1), 2, 16)
    for act in ACTS:
        plan = Plan("f32", f, act=act)
        out = plan(x, sx)
        assert torch.isfinite(out).all(), act
        plan.check(x, sx, out)


def test_two_plans_and_streams_at_once():
    a, xa, sa, ra = _case(11, 3000, 512, 2500, "bf16", residual=True)
    b, xb, sb, _ = _case(12, 16, 4096, 1000, "bf16", "silu", gated=True)
    wa, wb = a(xa, sa, ra), b(xb, sb)
    streams = [torch.cuda.Stream() for _ in range(3)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = []
    for i in range(12):
        with torch.cuda.stream(streams[i % 3]):
            got.append((a(xa, sa, ra), wa) if i % 2 else (b(xb, sb), wb))
    torch.cuda.synchronize()
    for out, want in got:
        assert torch.equal(out, want)
    B.iconv_check(stream())


@pytest.mark.parametrize("m", [1, 24, 2100])
def test_the_sublayer_as_it_is_used(m):
    """norm -> gated product -> 8-bit rows -> product with the residual, step by step against the definitions on the very inputs of
    each, directly and as a captured graph replayed on new inputs."""
    d, f, gen = 520, 1160, generator(13)
    gated = Plan("bf16", Filter(gen, f, d, bias=False), Filter(gen, f, d, bias=False), "silu")
    down = Plan("bf16", Filter(gen, d, f))
    x, r = (torch.randn(m, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    g = (1 + 0.1 * torch.randn(d, generator=gen, device="cuda")).bfloat16()
    q, q2 = torch.empty(m, 528, dtype=torch.int8, device="cuda")[:, :d], torch.empty(m, 1168, dtype=torch.int8, device="cuda")[:, :f]
    s1, s2 = torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
    total, h, out = torch.empty_like(x), torch.empty(m, f, dtype=torch.bfloat16, device="cuda"), torch.empty_like(x)

    def run():
        rms_call(x, r, g, q=q, total=total, scales=s1)
        gated(q, s1, out=h)
        rms_call(h, norm=0, with_sum=False, q=q2, scales=s2)
        down(q2, s2, total, out)

    def check():
        rms_check(x, r, g, q, s1, total)
        gated.check(q, s1, h)
        rms_check(h, None, None, q2, s2, None, norm=0)
        down.check(q2, s2, out, total)

    run()
    check()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        run()
    for seed in (14, 15):
        x.copy_(torch.randn(m, d, generator=generator(seed), device="cuda"))
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        check()
    B.iconv_check(stream())


def test_outputs_past_32_bits():
    """The last row of x and out starts more than 4 GB behind the first."""
    gen = generator(16)
    plan = Plan("bf16", Filter(gen, 96, 64))
    m, step = 5, 1 << 30
    store = torch.zeros(m * step, dtype=torch.int8, device="cuda")
    x = store.view(m, step)[:, :64]
    x.copy_(rows8(gen, m, 64)[0])
    sx = torch.rand(m, generator=gen, device="cuda")
    out = torch.zeros(m * step, dtype=torch.bfloat16, device="cuda").view(m, step)[:, :96]
    plan(x, sx, out=out)
    plan.check(x, sx, out)


def test_no_rows_and_refusals_with_a_plan():
    plan, x, sx, r = _case(17, 4, 64, 32, "bf16", residual=True)
    out = plan(x, sx, r)
    call = lambda **o: B.imat_forward(*[{**dict(p=plan.handle, rows=4, x=ptr(x), xs=64, sx=ptr(sx), r=None, rs=0, out=ptr(out), os=32, st=stream()), **o}[i]
                                        for i in ("p", "rows", "x", "xs", "sx", "r", "rs", "out", "os", "st")])
    call(rows=0, x=None, sx=None, out=None)
    for over, status in [(dict(p=None), B.ERR_ARG), (dict(rows=-1), B.ERR_ARG), (dict(rows=(1 << 30) + 1), B.ERR_ARG), (dict(x=None), B.ERR_ARG),
                         (dict(sx=None), B.ERR_ARG), (dict(out=None), B.ERR_ARG), (dict(xs=63), B.ERR_SHAPE), (dict(os=31), B.ERR_SHAPE),
                         (dict(r=ptr(r), rs=31), B.ERR_SHAPE), (dict(x=ptr(x) + 8), B.ERR_ALIGN), (dict(xs=72), B.ERR_ALIGN), (dict(sx=ptr(sx) + 4), B.ERR_ALIGN),
                         (dict(out=ptr(out) + 1), B.ERR_ALIGN), (dict(xs=1 << 50), B.ERR_SHAPE)]:
        with pytest.raises(B.IconvError) as e:
            call(**over)
        assert e.value.status == status, over
    gated, *_ = _case(18, 4, 64, 32, "bf16", gated=True)
    with pytest.raises(B.IconvError) as e:
        call(p=gated.handle, r=ptr(r), rs=32)
    assert e.value.status == B.ERR_UNSUPPORTED
    for rows in (0, (1 << 30) + 1):
        with pytest.raises(B.IconvError):
            plan.describe(rows)


def test_a_plan_is_refused_inside_a_capture_and_leaves_it_whole():
    gen = generator(1)
    f = Filter(gen, 64, 128)
    x, sx = rows8(gen, 4, 128)
    plan = Plan("f32", f)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph, out = torch.cuda.CUDAGraph(), torch.zeros(4, 64, device="cuda")
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        with pytest.raises(B.IconvError) as e:
            Plan("f32", f)
        assert e.value.status == B.ERR_CUDA and "capturing" in B.iconv_last_error()
        plan(x, sx, out=out)
    graph.replay()
    torch.cuda.synchronize()
    plan.check(x, sx, out)


@pytest.mark.parametrize("m,step,n,gated,k", [(40, 1 << 27, 4000, False, 144), (40, 1 << 27, 300, True, 144), (2100, 1 << 22, 2600, False, 144), (2100, 1 << 22, 2600, True, 144),
                                              (2100, 1 << 22, 5000, False, 1000), (2100, 1 << 22, 5000, True, 1000)])
def test_far_rows_on_the_other_kernels(m, step, n, gated, k):
    """x and out more than 4 GB from their first row to their last, the residual more than 2^31 elements."""
    gen = generator(19)
    plan = Plan("bf16", Filter(gen, n, k), Filter(gen, n, k) if gated else None)
    assert k == 144 or plan.describe(m).startswith("bulk")
    x = torch.empty(m * step, dtype=torch.int8, device="cuda").view(m, step)[:, :k]
    x.copy_(rows8(gen, m, k)[0])
    sx = torch.rand(m, generator=gen, device="cuda")
    out = torch.empty(m * step, dtype=torch.bfloat16, device="cuda").view(m, step)[:, 1:n + 1]
    r = None
    if not gated:
        r = torch.empty(m * step, dtype=torch.bfloat16, device="cuda").view(m, step)[:, :n]
        r.copy_(torch.randn(m, n, generator=gen, device="cuda"))
    plan(x, sx, r, out)
    plan.check(x, sx, out.contiguous(), r)


def test_very_many_rows():
    plan, x, sx, _ = _case(20, (1 << 24) + 3, 16, 3, "f32")
    plan.check(x, sx, plan(x, sx))
    B.iconv_check(stream())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("form", ["gated", "residual", "neither"])
def test_a_row_is_the_same_in_any_call_whatever_the_activation(form, act, dtype):
    """Products and sums behind one another, in kernels that are compiled apart."""
    plan, x, sx, r = _case(21, 2500, 1030, 2500, dtype, act, form == "gated", residual=form == "residual")
    whole = plan(x, sx, r)
    assert plan.describe(2500).startswith("bulk")
    forms = set()
    for m, kernel in ((1, "stream"), (9, "stream"), (20, "few"), (64, "few"), (100, "few")):
        assert plan.describe(m).startswith(kernel)
        forms.add(kernel + (" alone" if "split 1," in plan.describe(m) else ""))
        some = plan(x[1000:1000 + m], sx[1000:1000 + m].clone(), r[1000:1000 + m] if r is not None else None)
        assert torch.equal(some, whole[1000:1000 + m]), m
    small, x, sx, r = _case(22, 700, 4096, 70, dtype, act, form == "gated", residual=form == "residual")     # (few channels: a reduction in parts)
    whole = small(x, sx, r)
    forms.add("few" if "split 1," not in small.describe(40) else "")
    some = small(x[300:340], sx[300:340].clone(), r[300:340] if r is not None else None)
    assert torch.equal(some, whole[300:340]) and {"stream", "few"} <= forms
    B.iconv_check(stream())
