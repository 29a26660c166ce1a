"""Losses and log-sum-exps at logits that are known exactly: W has one column that is not zero, H is 1 there.

Bars, u = 2^-24.  The target's logit is taken from the largest exactly where they are the same, and to a rounding
else; the sum of exponentials (each to 2 u of itself and to the rounding of its logit's difference to the largest,
which its own smallness makes up for) and its logarithm add 4 u where the sum is near 1 and 16 u of the loss
elsewhere.  None of that grows with the logits."""
import pytest

torch = pytest.importorskip("torch")

from paper_2405_19509_amd import gcx  # noqa: E402

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
# fp32 as it is and in parts, one tile of entries and several, one size of tiles and two
SIZES = [(1, 1, 7, 8), (3, 20, 100, 24), (2, 40, 1000, 37), (4, 151, 1000, 264), (1, 300, 256, 2000), (1, 1030, 20001, 136)]


def known(N, n, V, d, dtype, logits):
    """H, W whose logits are `logits` [V], values of the type, in every row."""
    H, W = torch.zeros((N, n, d), dtype=dtype, device="cuda"), torch.zeros((V, d), dtype=dtype, device="cuda")
    H[..., d // 2] = 1.0
    W[:, d // 2] = logits.to(dtype)
    assert torch.equal(W[:, d // 2].double(), logits.double())
    return H, W


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("z", [-1000.0, 0.0, 50.0, 100.0, 1000.0, 2.0 ** 50])
@pytest.mark.parametrize("n", [1, 5, 300])
def test_the_only_entry_has_no_loss(n, z, dtype):
    H, W = known(2, n, 1, 24, dtype, torch.full((1,), z, device="cuda"))
    loss, lse = gcx.gc_softmax_xent(H, W, torch.zeros((2, n), dtype=torch.int32, device="cuda"))
    assert not loss.any() and bool((lse == z).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("z,gap", [(50.0, 16.0), (100.0, 16.0), (1000.0, 16.0), (1000.0, 8.0), (-992.0, 32.0)])
@pytest.mark.parametrize("N,n,V,d", SIZES)
def test_losses_of_sure_rows(N, n, V, d, z, gap, dtype):
    """The target far above all others: log(1 + (V - 1) exp(-gap)), never below 0, whatever the logits' size."""
    logits = torch.full((V,), z - gap, device="cuda")
    y = 2 * V // 3
    logits[y] = z
    H, W = known(N, n, V, d, dtype, logits)
    loss, lse = gcx.gc_softmax_xent(H, W, torch.full((N, n), y, dtype=torch.int32, device="cuda"))
    want = torch.log1p((V - 1) * torch.exp(torch.tensor(-gap, dtype=torch.float64))).item()
    assert float(loss.min()) >= 0.0
    assert float((loss.double() - want).abs().max()) <= 4 * U + 16 * U * want
    assert float((lse.double() - (z + want)).abs().max()) <= U * abs(z + want) + 4 * U + 16 * U * want


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,n,V,d", SIZES)
def test_logits_near_the_largest_float(N, n, V, d, dtype):
    """Finite logits up to 3e38 have finite losses and gradients: the largest of a row, and one at the other end."""
    big = 2.0 ** 127 * 1.75  # 2.98e38; log2(e) times it is no float
    logits = torch.linspace(-50, 50, V, device="cuda").round()
    logits[0], logits[V - 1] = -big, big
    H, W = known(N, n, V, d, dtype, logits)
    label = torch.full((N, n), V - 1, dtype=torch.int32, device="cuda")
    label[:, -1] = -1
    loss, lse = gcx.gc_softmax_xent(H, W, label)
    assert not loss.any() and bool((lse == big).all())
    dH, G = gcx.gc_softmax_xent_grads(H, W, label, lse)
    assert not dH.any() and not G.any()
    W[V - 1] = 0.0  # the lowest logit is the only large one left, and no row's largest
    rest = torch.where(logits.abs() < 1e3, logits, 0.0).double()
    want = torch.logsumexp(rest[1:], 0).item()
    loss, lse = gcx.gc_softmax_xent(H, W, label)
    assert float((lse.double() - want).abs().max()) <= 32 * U * max(abs(want), 1.0)
    there = label >= 0
    assert float((loss[there].double() - want).abs().max() if there.any() else 0.0) <= 32 * U * max(abs(want), 1.0)
