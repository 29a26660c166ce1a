"""Gradients where values are finite but near the largest float: past the largest bf16, which fp32 operands and the
probabilities are split into or rounded to.  Reference and bars are those of test_softmax_xent_gpu."""
import pytest

torch = pytest.importorskip("torch")

from paper_2405_19509_amd import gcx  # noqa: E402
from test_softmax_xent_gpu import CORES, check, everything, problem, reference  # noqa: E402

pytestmark = pytest.mark.gpu
SIZES = [(2, 30, 300, 64), (1, 5, 300, 33), (1, 400, 2000, 180), tuple(CORES.values())]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,n,V,d", SIZES)
def test_entries_ruled_out_by_the_lowest_value(N, n, V, d, dtype):
    """Their probability is 0 and their weights are finite: every gradient is that of the other entries alone."""
    H, W, label, dloss = problem(N, n, V, d, dtype, masked=0.1)
    H[..., 0] = 1.0
    W[:, 0] = 0.0
    ruled = slice(64, 192)
    label[(label >= 64) & (label < 192)] = 5
    W[ruled] = 0.0
    W[ruled, 0] = torch.finfo(dtype).min
    label1 = torch.where((label >= 192) & (label < V), label - 128, label)
    ref, bar = reference(H, torch.cat([W[:64], W[192:]]).contiguous(), torch.where(label1 >= V - 128, -1, label1), dloss)
    got = everything(H, W, label, dloss)
    assert not got["G"][:, ruled].any()
    got["G"] = torch.cat([got["G"][:, :64], got["G"][:, 192:]], 1)
    check(got, ref, bar, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,n,V,d", SIZES)
def test_weights_of_losses_near_the_largest_float(N, n, V, d, dtype):
    """Weights up to the largest float: gradients of up to 1e37, as exact as others."""
    H, W, label, dloss = problem(N, n, V, d, dtype, masked=0.1)
    H *= 2.0 ** -10
    top = torch.finfo(torch.float32).max
    dloss = torch.where(dloss.abs() < 0.2, dloss * 1e30, torch.where(dloss > 0, top, -top))
    ref, bar = reference(H, W, label, dloss)
    assert bool(ref["dH"].isfinite().all()) and float(ref["G"].abs().max()) < 1e38
    got = everything(H, W, label, dloss)
    check(got, ref, bar, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("N,n,V,d", SIZES)
def test_weights_of_losses_that_are_not_finite(N, n, V, d, bad, dtype):
    """They reach their own row of dH and their chunk's G, and no other."""
    H, W, label, dloss = problem(N, n, V, d, dtype, masked=0.0)
    _, lse = gcx.gc_softmax_xent(H, W, label)
    clean = gcx.gc_softmax_xent_grads(H, W, label, lse, dloss=dloss)
    dloss[0, 3] = bad
    dH, G = gcx.gc_softmax_xent_grads(H, W, label, lse, dloss=dloss)
    others = torch.ones((N, n), dtype=torch.bool)
    others[0, 3] = False
    assert not bool(dH[0, 3].isfinite().any()) and torch.equal(dH[others], clean[0][others])
    assert not bool(G[0].isfinite().any()) and torch.equal(G[1:], clean[1][1:])
