"""bf16 gradients where nearly all of them is in the targets: as exact as their own rounding to bf16.

With flat logits over V entries a row's P is -w at its target and w / V elsewhere.  Let r be the 2-norm of what rounding
the exact gradient to bf16 leaves.  P rounded to bf16 alone would add an error of the same size, independent of it: 1.41 r
in all.  With what that leaves of the target added, only the other entries' roundings remain, 1 / sqrt(V) of it: below
1.01 r for V >= 100, and 1.15 r is the bar.  That the bar would see the target's rounding is checked on the definition, where rows are
many enough for their roundings' mean square."""
import pytest

torch = pytest.importorskip("torch")

from paper_2405_19509_amd import gcx  # noqa: E402
from test_softmax_xent_gpu import problem  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,n,V,d", [
    (2, 5, 1000, 96), (40, 8, 300, 93),  # chunks of few tokens
    (3, 40, 700, 64), (1, 9, 30011, 60), (2, 300, 1333, 264),  # one split of the vocabulary and many
    (1, 700, 300, 33), (1, 3000, 100, 40), (2, 2500, 200, 128),  # more targets in a tile than are listed at once
    (1, 1030, 8192, 1024), (2, 2048, 4096, 512), (3, 2500, 20011, 24)])  # large tiles; several pieces of the vocabulary
def test_targets_keep_their_digits(N, n, V, d):
    H, W, label, dloss = problem(N, n, V, d, torch.bfloat16, scale=0.1)
    _, lse = gcx.gc_softmax_xent(H, W, label)
    got = gcx.gc_softmax_xent_grads(H, W, label, lse, dloss=dloss)
    there = (label >= 0) & (label < V)
    y = torch.where(there, label, 0).long()[..., None]
    P = torch.softmax(H.double() @ W.double().t(), -1)
    P.scatter_add_(2, y, torch.full_like(y, -1.0, dtype=torch.float64))
    P *= torch.where(there, dloss.double(), 0.0)[..., None]

    def gradients(P):
        return P @ W.double(), torch.stack([p.t().contiguous() @ h for p, h in zip(P, H.double())])

    for a, want, rounded in zip(got, gradients(P), gradients(P.bfloat16().double())):
        r = float((want.bfloat16().double() - want).norm())
        assert N * n < 100 or float((rounded.bfloat16().double() - want).norm()) > 1.3 * r
        assert float((a.double() - want).norm()) <= 1.15 * r
