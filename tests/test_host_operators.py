"""What hag_embedding, hag_layer_norm and hag_clip_gradients refuse, by the status they return before anything is launched (no GPU)."""
import ctypes

import pytest

from paper_1906_03707_amd import binding as B

P = 1 << 20                                                # an address that nothing reads
BIG = 1 << 31


def refused(rc):
    assert rc == B.HAG_EINVAL and B.lib().hag_last_error()


@pytest.mark.parametrize("n,rows,d,dtype,stride,ids", [(-1, 3, 4, 0, 4, 4), (2, -1, 4, 0, 4, 4), (2, 3, 0, 0, 4, 4), (BIG, 3, 4, 0, 4, 4), (2, BIG, 4, 0, 4, 4), (2, 3, (1 << 20) + 1, 0, 4, 4),
                                                       (2, 3, 4, 1, 4, 4), (2, 3, 4, 4, 4, 4), (2, 3, 4, 0, -1, 4), (2, 3, 4, 0, 4, 0), (2, 3, 4, 7, 4, 4)])
def test_embedding_refusals(n, rows, d, dtype, stride, ids):
    L = B.lib()
    refused(L.hag_embedding(n, rows, d, dtype, P, stride, ids, P, -1, 1.0, P, None))
    refused(L.hag_embedding_grad(n, rows, d, dtype, P, stride, ids, P, -1, 1.0, dtype, P, P, None))


def test_embedding_refuses_null_pointers_and_types():
    L = B.lib()
    refused(L.hag_embedding(2, 3, 4, 0, None, 4, 4, P, -1, 1.0, P, None))
    refused(L.hag_embedding(2, 3, 4, 0, P, 4, 4, None, -1, 1.0, P, None))
    refused(L.hag_embedding(2, 3, 4, 0, P, 4, 4, P, -1, 1.0, None, None))
    for gy, ids, out, ws in ((None, P, P, P), (P, None, P, P), (P, P, None, P), (P, P, P, None), (P, P, P, P + 8)):
        refused(L.hag_embedding_grad(2, 3, 4, 0, gy, 4, 4, ids, -1, 1.0, 0, out, ws, None))
    refused(L.hag_embedding_grad(2, 3, 4, 0, P, 4, 4, P, -1, 1.0, 2, P, P, None))                       # fp32 gradients into a bf16 table
    refused(L.hag_embedding_grad(2, 3, 4, 2, P, 4, 4, P, -1, 1.0, 3, P, P, None))
    assert L.hag_embedding(0, 3, 4, 0, None, 4, 4, None, -1, 1.0, None, None) == B.HAG_OK               # nothing to do
    assert L.hag_embedding_grad(5, 0, 4, 0, None, 4, 4, None, -1, 1.0, 0, None, None, None) == B.HAG_OK
    assert L.hag_embedding_grad_workspace_bytes(-1, 2, 3) == 0 and L.hag_embedding_grad_workspace_bytes(1000, 50, 8) > 0


@pytest.mark.parametrize("n,d,dtype,param,stride,eps", [(-1, 4, 0, 0, 4, 1e-5), (BIG, 4, 0, 0, 4, 1e-5), (2, 0, 0, 0, 4, 1e-5), (2, (1 << 20) + 1, 0, 0, 4, 1e-5), (2, 4, 1, 0, 4, 1e-5),
                                                        (2, 4, 2, 3, 4, 1e-5), (2, 4, 0, 2, 4, 1e-5), (2, 4, 0, 0, -4, 1e-5), (2, 4, 0, 0, 4, -1e-5), (2, 4, 0, 0, 4, float("nan"))])
def test_layer_norm_refusals(n, d, dtype, param, stride, eps):
    L = B.lib()
    refused(L.hag_layer_norm(n, d, dtype, P, stride, param, P, P, eps, P, P, P, None))
    if eps == 1e-5:
        refused(L.hag_layer_norm_grad(n, d, dtype, P, stride, P, 4, param, P, P, P, P, P, P, P, None))


def test_layer_norm_refuses_null_pointers():
    L = B.lib()
    refused(L.hag_layer_norm(2, 4, 0, None, 4, 0, P, P, 1e-5, P, P, P, None))
    refused(L.hag_layer_norm(2, 4, 0, P, 4, 0, P, P, 1e-5, None, P, P, None))
    for gy, x, mean, rstd, gx, ws in ((None, P, P, P, P, P), (P, None, P, P, P, P), (P, P, None, P, P, P), (P, P, P, None, P, P), (P, P, P, P, None, P), (P, P, P, P, P, None), (P, P, P, P, P, P + 4)):
        refused(L.hag_layer_norm_grad(2, 4, 0, gy, 4, x, 4, 0, P, mean, rstd, gx, P, P, ws, None))
    assert L.hag_layer_norm(0, 4, 0, None, 4, 0, None, None, 1e-5, None, None, None, None) == B.HAG_OK
    assert L.hag_layer_norm_grad(0, 4, 0, None, 4, None, 4, 0, None, None, None, None, None, None, None, None) == B.HAG_OK
    assert L.hag_layer_norm_grad_workspace_bytes(5, 0) == 0 and L.hag_layer_norm_grad_workspace_bytes(5, 7) > 0


def test_clip_refusals():
    L = B.lib()

    def entry(*fields):
        return (ctypes.c_int64 * 4)(*fields)

    good = entry(P, P, 5, 0)
    for max_norm in (0.0, -1.0, float("nan")):
        refused(L.hag_clip_gradients(1, good, max_norm, P, P, None))
    refused(L.hag_clip_gradients(-1, good, 1.0, P, P, None))
    refused(L.hag_clip_gradients(1, None, 1.0, P, P, None))
    refused(L.hag_clip_gradients(1, good, 1.0, None, P, None))
    refused(L.hag_clip_gradients(1, good, 1.0, P, None, None))
    refused(L.hag_clip_gradients(1, good, 1.0, P, P + 8, None))
    for fields in ((P, P, -1, 0), (P, P, 5, 1), (P, P, 5, 4), (0, P, 5, 0), (P, 0, 5, 0), (P, P, 1 << 50, 0)):
        refused(L.hag_clip_gradients(1, entry(*fields), 1.0, P, P, None))
    assert L.hag_clip_workspace_bytes(-1) == 0 and L.hag_clip_workspace_bytes(3) > 0


def test_wide_tokens_of_fewer_rows_are_shared():
    """One workgroup takes the few tokens of 32 rows by itself; where that is much and there are fewer rows than tokens, these are put in order and shared, which takes a workspace."""
    size = B.lib().hag_embedding_grad_workspace_bytes
    for n, rows, d in ((2000, 16, 1024), (2000, 74, 1024), (2048, 16, 100), (300, 200, 1030), (2, 1, 1 << 20)):
        assert size(n, rows, d) >= 16 * n + 4 * rows
    for n, rows, d in ((777, 4096, 37), (74, 74, 64), (2000, 74, 64), (0, 5, 1 << 20), (2000, 2000, 1024)):
        assert size(n, rows, d) == 16


def test_sizes_at_their_limits():
    """n and rows are below 2^31: the largest are not refused (nothing is launched: a NULL pointer comes after the sizes), the next are."""
    L = B.lib()
    for n, rows in ((2, BIG - 1), (BIG - 1, 2)):
        refused(L.hag_embedding(n, rows, 4, 0, None, 4, 4, P, -1, 1.0, P, None))
        assert L.hag_last_error() == b"NULL pointer"
        refused(L.hag_embedding_grad(n, rows, 4, 0, None, 4, 4, P, -1, 1.0, 0, P, P, None))
        assert L.hag_last_error() == b"NULL pointer"
        assert L.hag_embedding_grad_workspace_bytes(n, rows, 4) > 0
        assert L.hag_embedding_grad_workspace_bytes(n + (n > 2), rows + (rows > 2), 4) == 0
