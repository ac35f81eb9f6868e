"""What ``irms_quant`` and ``imat_plan`` refuse, before anything touches a GPU (addresses are never read here), and how their kernels, which
come up while the kernel before them still runs, read their tensors."""
import os
import re

import pytest

from paper_2006_11735_b200 import binding as B
from paper_2006_11735_b200.build import CSRC

A = 1 << 20         # a well-aligned address that nothing reads


def _rms(x=A, r=None, g=None, total=None, q=A, scales=A, **over):
    B.irms_quant(x, r, g, total, q, scales, 0, **{**dict(rows=2, width=64, dtype=B.BF16), **over})


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), B.ERR_ARG), (dict(width=0), B.ERR_ARG), (dict(dtype=B.S8), B.ERR_ARG), (dict(dtype=7), B.ERR_ARG),
    (dict(g=A, weight_dtype=B.F16), B.ERR_ARG), (dict(eps=-1.0), B.ERR_ARG), (dict(eps=float("nan")), B.ERR_ARG), (dict(eps=float("inf")), B.ERR_ARG),
    (dict(norm=2), B.ERR_ARG), (dict(x=None), B.ERR_ARG), (dict(q=None), B.ERR_ARG), (dict(scales=None), B.ERR_ARG),
    (dict(x_stride=63), B.ERR_SHAPE), (dict(q_stride=63), B.ERR_SHAPE), (dict(r=A, residual_stride=63), B.ERR_SHAPE), (dict(total=A, sum_stride=63), B.ERR_SHAPE),
    (dict(rows=1 << 31), B.ERR_SHAPE), (dict(x_stride=1 << 46), B.ERR_SHAPE), (dict(q_stride=1 << 62), B.ERR_SHAPE),
    (dict(x=A + 1), B.ERR_ALIGN), (dict(r=A + 1), B.ERR_ALIGN), (dict(total=A + 1), B.ERR_ALIGN), (dict(g=A + 1), B.ERR_ALIGN),
    (dict(g=A + 2, weight_dtype=B.F32), B.ERR_ALIGN), (dict(scales=A + 2), B.ERR_ALIGN), (dict(x=A + 2, dtype=B.F32), B.ERR_ALIGN),
])
def test_rms_refuses(kw, status):
    with pytest.raises(B.IconvError) as e:
        _rms(**kw)
    assert e.value.status == status and "irms_quant" in B.iconv_last_error()


def test_null_descriptors():
    assert B.lib.irms_quant(None, A, None, None, None, A, A, None) == B.ERR_ARG
    assert B.lib.imat_plan(None, None, None) == B.ERR_ARG
    assert B.lib.imat_plan_destroy(None) == B.OK
    assert B.lib.imat_forward(None, 1, A, 16, A, None, 0, A, 16, None) == B.ERR_ARG


@pytest.mark.parametrize("kw,status", [
    (dict(n=0), B.ERR_ARG), (dict(k=0), B.ERR_ARG), (dict(k=-4), B.ERR_ARG), (dict(out_dtype=B.S8), B.ERR_ARG), (dict(out_dtype=B.I32), B.ERR_ARG),
    (dict(act=-1), B.ERR_ARG), (dict(act=5), B.ERR_ARG), (dict(weights=None), B.ERR_ARG), (dict(scales=None), B.ERR_ARG),
    (dict(up_weights=A), B.ERR_ARG), (dict(up_scales=A), B.ERR_ARG), (dict(up_bias=A), B.ERR_ARG),
    (dict(w_stride=99), B.ERR_SHAPE), (dict(k=131072), B.ERR_OVERFLOW), (dict(n=1 << 25), B.ERR_SHAPE), (dict(n=1 << 24, k=131071), B.ERR_SHAPE),
    (dict(scales=A + 2), B.ERR_ALIGN), (dict(bias=A + 1), B.ERR_ALIGN), (dict(up_weights=A, up_scales=A + 2), B.ERR_ALIGN),
    (dict(up_weights=A, up_scales=A, up_bias=A + 3), B.ERR_ALIGN),
])
def test_plan_refuses(kw, status):
    with pytest.raises(B.IconvError) as e:
        B.imat_plan(**{**dict(n=64, k=100, out_dtype=B.BF16, weights=A, scales=A), **kw})
    assert e.value.status == status and "imat_plan" in B.iconv_last_error()


def test_no_rows_need_no_memory():
    _rms(x=None, q=None, scales=None, rows=0)


@pytest.mark.parametrize("file", ["kernel_rms.cu", "mat_device.cuh"])
def test_tensors_are_read_by_plain_loads(file):
    """The read-only path is for the plan's constants alone."""
    text = open(os.path.join(CSRC, file)).read()
    assert "__restrict__" not in text and not re.search(r"\.nc\b", text) and "grid_dep_wait()" in text
    assert all(m.group(1).startswith("a.row_params") for m in re.finditer(r"__ldg\((.*)", text))


def test_wider_rows_than_any():
    """Indexes within a row are 32-bit numbers."""
    for width in ((1 << 24) + 1, (1 << 31) - 1):
        with pytest.raises(B.IconvError) as e:
            _rms(rows=1, width=width)
        assert e.value.status == B.ERR_SHAPE and "width" in B.iconv_last_error()


def test_weights_further_apart_than_any():
    with pytest.raises(B.IconvError) as e:
        B.imat_plan(n=64, k=100, out_dtype=B.BF16, weights=A, scales=A, w_stride=1 << 60)
    assert e.value.status == B.ERR_SHAPE


def test_the_streaming_product_kernel_reads_its_tensors_by_plain_loads():
    """It comes up early too, and reads rows, scales and residual; its weights are the plan's constants, past L1 but coherent."""
    text = open(os.path.join(CSRC, "mat_stream.cuh")).read()
    assert "__restrict__" not in text and not re.search(r"\.nc\b", text) and "grid_dep_wait()" in text
    assert [m.group(1).startswith("a.row_params") for m in re.finditer(r"__ldg\((.*)", text)] == [True]


def test_many_wide_rows_are_counted_by_the_devices_sms():
    """No SM count stands in the rules that choose a kernel."""
    for file in ("kernel_rms.cu", "kernel_mat.cu"):
        text = re.sub(r"//.*", "", open(os.path.join(CSRC, file)).read())
        assert not re.search(r"\b(148|74|132)\b", text), file
