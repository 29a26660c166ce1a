"""Sizes past 2^31 that the library takes as 32-bit integers: refused by the wrappers, not cut (2^32 + 5 to 5)."""
import pytest

from paper_2405_19509_amd import gcx

torch = pytest.importorskip("torch")
BIG = 2 ** 32 + 5


def t(*shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="meta")


def i(*shape):
    return t(*shape, dtype=torch.int32)


@pytest.mark.parametrize("call", [
    lambda: gcx.gc_assign(gcx.GC_ASSIGN_CYCLIC, BIG, 6, 1),
    lambda: gcx.gc_chunk_grads(t(1, BIG, 1), t(1, BIG), t(1), gcx.GC_LOSS_LINEAR),
    lambda: gcx.gc_chunk_grads(t(BIG, 1, 1), t(BIG, 1), t(1), gcx.GC_LOSS_LINEAR),
    lambda: gcx.gc_chunk_grads(t(1, 1, 1), t(1, 1), t(BIG, 1), gcx.GC_LOSS_LINEAR),
    lambda: gcx.gc_sum_chunks(t(BIG, 1)),
    lambda: gcx.gc_decode_coeffs(i(1, 6), i(6, 2), i(BIG, 2), i(BIG, 2), t(1, 6)),
    lambda: gcx.gc_decode_coeffs(i(1, BIG), i(BIG, 2), i(6, 2), i(6, 2), t(1, BIG)),
    lambda: gcx.gc_encode(t(BIG, 1), i(1, 6), i(6, 2), t(1, 6, 2, 1)),
    lambda: gcx.gc_encode(t(6, 1), i(1, 6), i(6, BIG), t(1, 6, BIG, 1)),
    lambda: gcx.gc_reconstruct(t(1, BIG, 1), t(1, BIG), 1, i(1, BIG)),
    lambda: gcx.gc_reconstruct_noalloc(t(1, BIG, 1), t(1, BIG), 1, i(1, BIG), t(1, 1)),
    lambda: gcx.gc_decode_direct(t(BIG, 1), i(1, 6), i(6, 2), i(BIG, 2), i(BIG, 2), t(1, 6)),
    lambda: gcx.gc_progress(t(1, 6, 2, dtype=torch.float64), t(BIG, dtype=torch.float64)),
    lambda: gcx.gc_completion_times(t(1, 6, 2, dtype=torch.float64), i(BIG, 2), i(BIG, 2), 1),
    lambda: gcx.gc_original_ls(i(1, 6), i(6, 2), i(BIG, 2)),
    lambda: gcx.gc_original_ls(i(1, 6), i(6, 2), i(6, 2), max_iter=BIG),
    lambda: gcx.gc_chunk_grads_workspace_size(5, BIG, 8, 1), lambda: gcx.gc_reconstruct_workspace_size(5, BIG, 8, 1),
    lambda: gcx.gc_decode_direct_workspace_size(5, BIG, 8, 1)])
def test_refused(call):
    with pytest.raises(ValueError, match="32 bits"):
        call()
