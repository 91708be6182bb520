"""The cross entropy, the gradients' norm and clipping without a GPU: sizes of workspaces, records, refusals that come before any device is touched."""
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


def test_gradient_record_is_the_headers(lib):
    # 2 pointers, a size, a word, in the order of include/stq.h
    assert C.sizeof(stq.Grad) == 32
    assert [getattr(stq.Grad, n).offset for n in ("grad", "out", "numel", "dtype")] == [0, 8, 16, 24]
    a = stq.make_grads([dict(grad=4096, numel=5, dtype=stq.STQ_BF16), dict(grad=64, out=128, numel=0, dtype=stq.STQ_F32)])
    assert [(g.grad, g.out, g.numel, g.dtype) for g in a] == [(4096, None, 5, 1), (64, 128, 0, 0)]
    assert len(stq.make_grads([])) == 0


@pytest.mark.parametrize("size", [stq.cross_entropy_bytes, stq.cross_entropy_grad_bytes])
def test_workspace_sizes(lib, size):
    assert size(0, 10, 10) == 0
    assert size(1, 1, 1) > 0
    # far below the logits of all classes, 4 bytes each
    assert size(65536, 200000, 64) < 65536 * 200000 * 4 / 8
    # sizes that no card has do not overflow
    assert size((1 << 31) - 1, (1 << 31) - 1, 131071) > 0
    for bad in ((1, 0, 1), (1, 1, 0), (1 << 31, 1, 1), (1, 1 << 31, 1), (1, 1, 131072)):
        with pytest.raises(stq.StqError) as e:
            size(*bad)
        assert e.value.code == -9


def test_no_context(lib):
    n = C.c_uint64()
    q = stq.make_matrix(4096, 1, 1, stq.STQ_Q8, scales=4096)
    f = stq.make_matrix(4096, 1, 1, stq.STQ_F32)
    g = stq.make_grads([dict(grad=4096, numel=5, dtype=0)])
    assert lib.stq_cross_entropy_bytes(1, 1, 1, None) == -1 and lib.stq_cross_entropy_grad_bytes(1, 1, 1, None) == -1
    assert lib.stq_cross_entropy_bytes(1, 1, 1, C.byref(n)) == 0
    assert lib.stq_cross_entropy(None, q, q, 4096, 4096, 4096, 4096, 1 << 30, None) == -1
    assert lib.stq_cross_entropy_grad(None, q, q, 4096, 4096, 4096, 4096, None, f, f, 4096, 1 << 30, None) == -1
    assert lib.stq_grad_norm(None, g, 1, 4096, None) == -1
    assert lib.stq_clip_grads(None, g, 1, 4096, 1.0, None) == -1
