"""Refusals and sizes of the group norm, 4-bit matrices and linear layers that need no device."""
import pytest

from paper_2001_00138_b200 import binding as B

E_NULL, E_SHAPE, E_DTYPE = 1, 2, 9


def refused(status, call, *args, **kw):
    with pytest.raises(B.PatdnnError) as e:
        call(*args, **kw)
    assert e.value.status == status


@pytest.mark.parametrize("kw", [dict(N=-1), dict(N=65536), dict(P=0), dict(C=0), dict(groups=0), dict(groups=5), dict(eps=-1.0),
                                dict(eps=float("nan")), dict(eps=float("inf")), dict(x_pixel=31), dict(y_pixel=16), dict(x_image=100),
                                dict(y_image=9 * 32 - 1), dict(P=2 ** 31), dict(C=2 ** 21), dict(x_pixel=-64)])
def test_group_norm_refuses_sizes_and_strides(kw):
    args = dict(N=2, P=9, C=32, groups=8) | kw
    refused(E_SHAPE, B.GroupNorm, **args)


@pytest.mark.parametrize("kw", [dict(dtype=3), dict(dtype=-1), dict(act=3), dict(act=-1)])
def test_group_norm_refuses_types(kw):
    refused(E_DTYPE, B.GroupNorm, 2, 9, 32, 8, **kw)


def test_an_empty_batch_makes_a_handle_without_a_device():
    norm = B.GroupNorm(0, 9, 32, 8)
    norm.run(0, 0, 0, 0)
    norm.free()


def test_mx4_sizes():
    # row tiles of 128 rows; column tiles of 64, 128 or 256 columns; 512 scale bytes per 128 columns
    assert B.mx4_bytes(0, 32) == 0
    assert B.mx4_bytes(1, 1) == B.mx4_bytes(128, 64) == 128 * 32 + 512
    assert B.mx4_bytes(129, 64) == 2 * (128 * 32 + 512)
    assert B.mx4_bytes(1, 65) == B.mx4_bytes(1, 128) == 128 * 64 + 512
    assert B.mx4_bytes(1, 129) == B.mx4_bytes(1, 256) == 128 * 128 + 1024
    assert B.mx4_bytes(1, 257) == 2 * (128 * 128 + 1024)
    refused(E_SHAPE, B.mx4_bytes, -1, 32)
    refused(E_SHAPE, B.mx4_bytes, 1, 0)
    refused(E_SHAPE, B.mx4_bytes, 1, 2 ** 20 + 1)
    refused(E_SHAPE, B.mx4_bytes, 2 ** 31, 1)


@pytest.mark.parametrize("call", [B.mx4_quantize, B.mx4_dequantize])
def test_mx4_refusals(call):
    refused(E_DTYPE, call, 64, 64, 1, 32, dtype=7)
    refused(E_SHAPE, call, 64, 64, 1, 32, ld=31)
    refused(E_SHAPE, call, 64, 64, -1, 32)
    refused(E_SHAPE, B.mx4_quantize, 64, 72, 1, 32)           # the 4-bit buffer is not 16-byte aligned
    refused(E_SHAPE, B.mx4_dequantize, 72, 64, 1, 32)
    refused(E_SHAPE, B.mx4_quantize, 66, 64, 1, 32)           # a tensor that is not aligned to its elements
    refused(E_SHAPE, B.mx4_dequantize, 64, 66, 1, 32)
    refused(E_NULL, call, 0, 0, 1, 32)
    call(0, 0, 0, 32)                                         # no rows: nothing to do


@pytest.mark.parametrize("status, kw", [(E_SHAPE, dict(F=0)), (E_SHAPE, dict(K=0)), (E_SHAPE, dict(max_rows=-1)), (E_SHAPE, dict(ldw=63)),
                                        (E_SHAPE, dict(K=2 ** 21)), (E_SHAPE, dict(F=2 ** 21)), (E_DTYPE, dict(dtype=5)), (E_DTYPE, dict(act=9)),
                                        (E_NULL, dict(weights=0))])
def test_linear_refusals(status, kw):
    args = dict(weights=64, F=32, K=64, max_rows=4) | kw
    refused(status, B.Linear, **args)
