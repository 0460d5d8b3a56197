"""Expert products without a GPU: the C layout of the argument struct, and the argument
checks, which come before any CUDA call."""
import ctypes
import os
import subprocess

import pytest

from paper_2606_00539_gb300 import GnmrError
from paper_2606_00539_gb300 import _native as N
from paper_2606_00539_gb300 import build as native_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def lib():
    native_build.build()
    return N.load()


def test_struct_layout_matches_c(tmp_path):
    fields = [f for f, _ in N.gnmr_product._fields_]
    prints = "\n".join(f'printf("{f} %zu\\n", offsetof(gnmr_product, {f}));' for f in fields)
    src, exe = tmp_path / "probe.c", tmp_path / "probe"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "gnmr.h"\nint main(void) {\n'
                   f'printf("sizeof %zu\\n", sizeof(gnmr_product));\n{prints}\nreturn 0; }}\n')
    subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    said = dict(line.split() for line in subprocess.check_output([str(exe)], text=True).splitlines())
    assert int(said["sizeof"]) == ctypes.sizeof(N.gnmr_product)
    for f in fields:
        assert int(said[f]) == getattr(N.gnmr_product, f).offset, f


def product(**over):
    """A forward product that passes the checks; nothing here is dereferenced."""
    p = N.gnmr_product()
    kw = dict(op=N.GNMR_PRODUCT_FORWARD, groups=2, rows=10, n_out=16, n_in=8, dtype=N.GNMR_DTYPE_BF16,
              out_dtype=N.GNMR_DTYPE_BF16, d_offsets=4096, d_x=4096, x_stride=8, d_dy=4096, dy_stride=16, d_w=4096,
              w_stride=8, w_group_stride=128, d_x_scale=4096, d_w_scale=4096, d_out=4096, out_stride=16,
              out_group_stride=16 * 16)
    kw.update(over)
    for key, v in kw.items():
        setattr(p, key, v)
    return p


def test_operands_read_in_place_need_no_scratch():
    assert N.gnmr_products_scratch_bytes(product()) == 0
    assert N.gnmr_products_scratch_bytes(product(op=N.GNMR_PRODUCT_INPUT_GRAD)) == 0
    assert N.gnmr_products_scratch_bytes(product(op=N.GNMR_PRODUCT_WEIGHT_GRAD)) == 0


def test_other_operands_are_copied_to_scratch():
    """An odd start, row stride or group stride, and 8-bit codes: rows of 16-bit
    elements in multiples of eight, each operand's copy in whole 256 bytes."""
    assert N.gnmr_products_scratch_bytes(product(d_x=4098)) == 256            # 10 x 8
    assert N.gnmr_products_scratch_bytes(product(n_in=9, x_stride=9, w_stride=16)) == 512          # 10 x 16
    assert N.gnmr_products_scratch_bytes(product(w_group_stride=129)) == 512  # 2 x 16 x 8
    assert N.gnmr_products_scratch_bytes(product(w_group_stride=0, d_w=4098)) == 256
    i8 = dict(op=N.GNMR_PRODUCT_FORWARD_I8, n_in=32, x_stride=32, w_stride=32, w_group_stride=512)
    assert N.gnmr_products_scratch_bytes(product(**i8)) == 0
    assert N.gnmr_products_scratch_bytes(product(**i8, rows=64)) == 0
    assert N.gnmr_products_scratch_bytes(product(**i8, rows=65)) == 65 * 128 + 128    # widened, to whole 128 bytes
    assert N.gnmr_products_scratch_bytes(product(**i8, rows=65, groups=1)) == 0       # few tiles
    assert N.gnmr_products_scratch_bytes(product(**i8, rows=48 * 64 + 1, groups=1)) == 3073 * 128 + 128
    assert N.gnmr_products_scratch_bytes(product(**{**i8, "w_stride": 33, "w_group_stride": 528})) == 2 * 16 * 32


INVALID, LAYOUT = N.GNMR_ERR_INVALID_ARG, N.GNMR_ERR_LAYOUT
WG, I8 = N.GNMR_PRODUCT_WEIGHT_GRAD, N.GNMR_PRODUCT_FORWARD_I8


@pytest.mark.parametrize("status,over", [
    (INVALID, dict(op=-1)), (INVALID, dict(op=4)), (INVALID, dict(groups=0)), (INVALID, dict(groups=2049)),
    (INVALID, dict(rows=-1)), (INVALID, dict(rows=1 << 30)), (INVALID, dict(n_out=0)), (INVALID, dict(n_in=0)),
    (INVALID, dict(dtype=N.GNMR_DTYPE_F32)), (INVALID, dict(dtype=7)), (INVALID, dict(out_dtype=N.GNMR_DTYPE_F16)),
    (INVALID, dict(op=I8, out_dtype=7)), (INVALID, dict(op=I8, n_in=131072, x_stride=131072, w_stride=131072)),
    (INVALID, dict(d_offsets=None)), (INVALID, dict(d_x=None)), (INVALID, dict(d_w=None)), (INVALID, dict(d_out=None)),
    (INVALID, dict(op=N.GNMR_PRODUCT_INPUT_GRAD, d_dy=None)), (INVALID, dict(op=I8, d_x_scale=None)),
    (INVALID, dict(op=I8, d_w_scale=None)), (INVALID, dict(op=WG, d_x=None)),
    (LAYOUT, dict(x_stride=7)), (LAYOUT, dict(w_stride=7)), (LAYOUT, dict(w_group_stride=-1)),
    (LAYOUT, dict(out_stride=15)), (LAYOUT, dict(op=N.GNMR_PRODUCT_INPUT_GRAD, dy_stride=15)),
    (LAYOUT, dict(op=WG, out_group_stride=16 * 15 + 7)), (LAYOUT, dict(d_x=4097)), (LAYOUT, dict(d_out=4097)),
    (LAYOUT, dict(d_offsets=4100)), (LAYOUT, dict(out_dtype=N.GNMR_DTYPE_F32, d_out=4098)),
    (LAYOUT, dict(x_stride=(1 << 36) + 1)), (LAYOUT, dict(op=WG, out_stride=(1 << 62), out_group_stride=(1 << 62))),
    (LAYOUT, dict(op=WG, n_out=1 << 29, dy_stride=1 << 29, out_stride=1 << 36, out_group_stride=1 << 36)),
    (LAYOUT, dict(n_out=1 << 29, n_in=1 << 29, groups=2048, x_stride=1 << 29, w_stride=1 << 29, out_stride=1 << 29)),
    (LAYOUT, dict(d_mask=4096, mask_stride=0)), (LAYOUT, dict(op=I8, d_x_scale=4098)),
])
def test_refusals(status, over):
    with pytest.raises(GnmrError) as e:
        N.gnmr_products_scratch_bytes(product(**over))
    assert e.value.status == status and "products:" in e.value.detail


def test_refusals_without_arguments(lib):
    n = ctypes.c_int64(0)
    assert lib.gnmr_products_scratch_bytes(None, ctypes.addressof(n)) == INVALID
    p = product()
    assert lib.gnmr_products_scratch_bytes(ctypes.addressof(p), None) == INVALID
    assert lib.gnmr_products_run(None, ctypes.addressof(p), None) == INVALID
    assert lib.gnmr_products_create(0, None) == INVALID
    assert lib.gnmr_products_destroy(None) == N.GNMR_OK


@pytest.mark.parametrize("columns", [False, True])
@pytest.mark.parametrize("status,over", [
    (INVALID, dict(dtype=3)), (INVALID, dict(groups=0)), (INVALID, dict(rows=-1)), (INVALID, dict(cols=-1)),
    (INVALID, dict(x=None)), (INVALID, dict(q=None)), (INVALID, dict(scale=None)), (LAYOUT, dict(x_stride=7)),
    (LAYOUT, dict(q_stride=6)), (LAYOUT, dict(x_group_stride=-1)), (LAYOUT, dict(x=4097)), (LAYOUT, dict(scale=4098)),
    (LAYOUT, dict(rows=1 << 40, x_stride=1 << 40, q_stride=1 << 40)), (LAYOUT, dict(groups=2, mask=4096, mask_stride=0)),
])
def test_quantize_refusals(columns, status, over):
    kw = dict(x=4096, dtype=N.GNMR_DTYPE_BF16, groups=1, rows=8, cols=8, x_stride=8, x_group_stride=64, mask=None,
              mask_stride=1, q=4096, q_stride=8, q_group_stride=64, scale=4096)
    kw.update(over)
    fn = N.gnmr_quantize_columns if columns else N.gnmr_quantize_rows
    with pytest.raises(GnmrError) as e:
        fn(*kw.values())
    assert e.value.status == status and "quantize:" in e.value.detail


def test_quantize_of_nothing_is_no_work():
    N.gnmr_quantize_rows(None, N.GNMR_DTYPE_F32, 1, 0, 8, 8, 0, None, 1, None, 8, 0, None)
    N.gnmr_quantize_columns(None, N.GNMR_DTYPE_F32, 1, 8, 0, 8, 0, None, 1, None, 8, 0, None)
