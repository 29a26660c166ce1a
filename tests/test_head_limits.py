"""Sizes at which the language-model head's launches reach their limits, on the CPU: which calls are taken (a workspace
has a size) and which are refused, the queries and the calls alike."""
import pytest

from paper_2405_19509_amd import gcx

P = 1 << 12  # an address that is never used
F32, BF16 = gcx.GC_F32, gcx.GC_BF16


@pytest.mark.parametrize("rows,V,d,dtype,taken", [
    (2 ** 21 + 5, 2 ** 18 + 3, 8, BF16, True),  # 2^39 logits
    (2 ** 27 + 5, 300, 8, BF16, True),
    (2 ** 31, 128, 8, BF16, True),
    (2 ** 28, 300, 8, F32, True),
    (2 ** 31 + 1, 128, 8, BF16, False),
    (2 ** 24, 2 ** 24, 8, BF16, False),  # 2^36 tiles
    (2 ** 30, 300, 8, F32, False),
    (2 ** 27, 128, 2 ** 20, BF16, False),  # 2^35 tiles of dH, were there one
])
def test_forward(rows, V, d, dtype, taken):
    assert (gcx.gc_softmax_xent_workspace_size(rows, V, d, dtype) > 0) == taken
    st = gcx.load().gc_softmax_xent(P, P, P, rows, V, d, dtype, P, P, P, 16, None)
    assert st == gcx.GC_EINVAL  # refused, or its workspace too small


@pytest.mark.parametrize("N,n,V,d,dtype,taken", [
    (2 ** 24 + 3, 9, 2, 1, BF16, True),
    (2 ** 24 + 3, 1, 2, 1, BF16, True),
    (2 ** 23, 4, 256, 8, F32, True),  # few rows a chunk: no kernels over columns
    (2 ** 18, 17, 300, 8, F32, True),
    (2 ** 24, 17, 300, 8, F32, False),  # 2^27 blocks over columns
    (2 ** 30, 2, 300, 8, BF16, False),
    (2 ** 31 - 1, 1, 2 ** 20, 1, BF16, False),
])
def test_gradients(N, n, V, d, dtype, taken):
    assert (gcx.gc_softmax_xent_grads_workspace_size(N, n, V, d, dtype) > 0) == taken
    st = gcx.load().gc_softmax_xent_grads(P, P, P, P, None, N, n, V, d, dtype, P, P, P, 16, None)
    assert st == gcx.GC_EINVAL


def test_sizes_that_do_not_fit_32_bits():
    """2^32 + 5 is not taken for 5."""
    torch = pytest.importorskip("torch")
    big = 2 ** 32 + 5

    def t(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="meta")

    i32 = torch.int32
    for call in (lambda: gcx.gc_layer_norm_grads(t(1, big, 8), t(1, big, 8), None, t(1, big), t(1, big)),
                 lambda: gcx.gc_layer_norm_grads(t(big, 1, 8), t(big, 1, 8), None, t(big, 1), t(big, 1)),
                 lambda: gcx.gc_softmax_xent_grads(t(1, big, 8), t(9, 8), t(1, big, dtype=i32), t(1, big)),
                 lambda: gcx.gc_softmax_xent_grads(t(big, 1, 8), t(9, 8), t(big, 1, dtype=i32), t(big, 1)),
                 lambda: gcx.gc_softmax_xent_grads(t(1, 5, 8), t(big, 8), t(1, 5, dtype=i32), t(1, 5)),
                 lambda: gcx.gc_softmax_xent(t(5, 8), t(big, 8), t(5, dtype=i32)),
                 lambda: gcx.gc_layer_norm_grads_workspace_size(big, 5, 8), lambda: gcx.gc_layer_norm_grads_workspace_size(5, big, 8),
                 lambda: gcx.gc_softmax_xent_workspace_size(5, big, 8, F32),
                 lambda: gcx.gc_softmax_xent_grads_workspace_size(big, 5, 9, 8, F32),
                 lambda: gcx.gc_softmax_xent_grads_workspace_size(5, big, 9, 8, BF16),
                 lambda: gcx.gc_softmax_xent_grads_workspace_size(5, 5, big, 8, BF16)):
        with pytest.raises(ValueError, match="32 bits"):
            call()
