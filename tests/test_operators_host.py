"""The operators of the 8-bit layer without a GPU: sizes of workspaces, records, refusals that come before any device is touched."""
import ctypes as C
import os

import pytest

import paper_2604_06836_amd as stq


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(stq.library_path()):
        from paper_2604_06836_amd.build import build
        build()
    return stq.load_library()


def test_matrix_record_is_the_headers(lib):
    # 2 pointers, 3 sizes, 2 words, in the order of include/stq.h
    assert C.sizeof(stq.Matrix) == 48
    assert [getattr(stq.Matrix, n).offset for n in ("data", "scales", "rows", "cols", "stride", "dtype", "block")] == [0, 8, 16, 24, 32, 40, 44]
    m = stq.make_matrix(4096, 3, 5, stq.STQ_BF16)
    assert (m.data, m.rows, m.cols, m.stride, m.dtype, m.block) == (4096, 3, 5, 5, 1, 0)
    m = stq.make_matrix(4096, 3, 5, stq.STQ_Q8, stride=9, scales=64, block=128)
    assert (m.scales, m.stride, m.dtype, m.block) == (64, 9, 2, 128)


def test_constants_are_the_headers(lib):
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "stq.h")).read()
    for name in ("STQ_F32", "STQ_BF16", "STQ_Q8", "STQ_MAX_INNER"):
        assert "#define %s %du" % (name, getattr(stq, name)) in header
    assert "sizes" in stq.strerror(-9) and "type" in stq.strerror(-10)


def test_workspace_sizes(lib):
    assert stq.rms_norm_grad_bytes(0, 100) == 0
    assert stq.rms_norm_grad_bytes(1, 100) >= 400
    assert stq.rms_norm_grad_bytes(1 << 20, 100) <= 4 * 100 * 4096
    assert stq.matmul_grad_weight_bytes(0, 10, 10) == 0
    for bad in ((1, 0), (1, 1 << 31), (1 << 31, 1)):
        with pytest.raises(stq.StqError) as e:
            stq.rms_norm_grad_bytes(*bad)
        assert e.value.code == -9
    for bad in ((1, 0, 1), (1, 1, 0), (1 << 31, 1, 1), (1, 1 << 31, 1)):
        with pytest.raises(stq.StqError) as e:
            stq.matmul_grad_weight_bytes(*bad)
        assert e.value.code == -9
    assert lib.stq_rms_norm_grad_bytes(1, 1, None) == -1 and lib.stq_matmul_grad_weight_bytes(1, 1, 1, None) == -1


def test_no_context(lib):
    m = stq.make_matrix(4096, 1, 1, stq.STQ_F32)
    q = stq.make_matrix(4096, 1, 1, stq.STQ_Q8, scales=4096)
    assert lib.stq_quantize_rows(None, m, q, None) == -1
    assert lib.stq_dequantize_rows(None, q, m, None) == -1
    assert lib.stq_rms_norm(None, m, None, 4096, 1e-6, None, q, None, None, None) == -1
    assert lib.stq_rms_norm_grad(None, m, 4096, 4096, m, None, m, 4096, 4096, 1 << 20, None) == -1
    assert lib.stq_gated_silu(None, m, m, q, None, None, None) == -1
    assert lib.stq_gated_silu_grad(None, m, m, m, m, m, None) == -1
    assert lib.stq_matmul(None, q, q, m, None) == -1
    assert lib.stq_matmul_grad_input(None, m, q, m, None) == -1
    assert lib.stq_matmul_grad_weight(None, m, q, m, 4096, 1 << 30, None) == -1
