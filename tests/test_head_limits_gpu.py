"""The language-model head's operators at sizes whose launches have more than 2^32 threads.  Bars: each result is some
ten roundings of terms of its own size, or the bars that the operators' own tests derive."""
import pytest

torch = pytest.importorskip("torch")

from paper_2405_19509_amd import gcx  # noqa: E402

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def test_layer_norm_gradients_of_more_than_2_26_chunks():
    """A wave per chunk of one row: dgamma = dy h, dbeta = dy, dx = rstd (a - mean a - h mean(a h))."""
    N, d = 2 ** 26 + 3, 8
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn((N, 1, d), generator=g, device="cuda")
    dy = torch.randn((N, 1, d), generator=g, device="cuda")
    gamma = 1 + 0.2 * torch.randn(d, generator=g, device="cuda")
    _, mean, rstd = gcx.gc_layer_norm(x, gamma)
    dx, dgamma, dbeta = gcx.gc_layer_norm_grads(x, dy, gamma, mean, rstd)
    assert torch.equal(dbeta, dy[:, 0])
    for rows in (slice(0, 1 << 20), slice(2 ** 21 - 5, 2 ** 21 + 5), slice(2 ** 25 - 5, 2 ** 25 + 5), slice(N - (1 << 20), N)):
        m, rs, v = mean[rows].double()[..., None], rstd[rows].double()[..., None], dy[rows].double()
        h, a = (x[rows].double() - m) * rs, v * gamma.double()
        e = 4 * U * (h.abs() + m.abs() * rs)  # of h
        assert bool(((dgamma[rows].double() - (v * h)[:, 0]).abs() <= (v.abs() * (e + 2 * U * h.abs()))[:, 0] + 1e-30).all())
        ah = (a * h).abs().mean(-1, keepdim=True)
        want = rs * (a - a.mean(-1, keepdim=True) - h * (a * h).mean(-1, keepdim=True))
        bar = rs * (16 * U * (a.abs() + a.abs().mean(-1, keepdim=True) + h.abs() * ah) + e * ah + h.abs() * (a.abs() * e).mean(-1, keepdim=True))
        assert bool(((dx[rows].double() - want).abs() <= bar + 1e-30).all())


def words(shape, seed):
    return torch.randint(-4, 5, shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda", dtype=torch.int32)


def check_losses(H, W, label, loss, lse):
    """Small whole numbers: logits are exact in fp32.  Exponentials to 4 U of themselves, sums of V of them."""
    z = H.double() @ W.double().t()
    want = torch.logsumexp(z, 1)
    bar = (4 * len(W) ** 0.5 + 16) * U * (1 + want.abs())
    assert bool(((lse.double() - want).abs() <= bar).all())
    there = label >= 0
    target = z.gather(1, label.clamp(min=0).long()[:, None])[:, 0]
    assert bool(((loss.double() - torch.where(there, want - target, 0.0)).abs() <= bar).all())


def test_softmax_xent_of_more_than_2_39_logits():
    """2^21 + 5 tokens against 2^18 + 3 entries: more than 2^23 tiles of 512 threads."""
    rows, V, d = 2 ** 21 + 5, 2 ** 18 + 3, 8
    H, W = words((rows, d), 1).bfloat16(), (words((V, d), 2) / 8).bfloat16()
    label = torch.randint(-1, V, (rows,), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda", dtype=torch.int32)
    label[-3:] = torch.tensor([0, V - 1, V - 2], dtype=torch.int32)
    loss, lse = gcx.gc_softmax_xent(H, W, label)
    for part in (slice(0, 40), slice(2 ** 20 - 20, 2 ** 20 + 20), slice(rows - 300, rows)):
        check_losses(H[part], W, label[part], loss[part], lse[part])
    assert bool(lse.isfinite().all()) and float(lse.min()) >= 12.0


def test_softmax_xent_of_more_than_2_27_rows():
    """Rows whose log-sum-exps come from three tiles, joined by 2^24 blocks and more."""
    rows, V, d = 2 ** 27 + 5, 300, 8
    H = torch.randint(-4, 5, (rows, d), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda", dtype=torch.int8).bfloat16()
    W = (words((V, d), 2) / 8).bfloat16()
    label = torch.randint(-1, V, (rows,), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda", dtype=torch.int32)
    loss, lse = gcx.gc_softmax_xent(H, W, label)
    for part in (slice(0, 100000), slice(2 ** 24 - 999, 2 ** 24 + 999), slice(rows - 100000, rows)):
        check_losses(H[part], W, label[part], loss[part], lse[part])
    assert bool(lse.isfinite().all()) and float(lse.min()) >= 5.0


@pytest.mark.parametrize("n", [1, 9])
def test_softmax_xent_gradients_of_more_than_2_24_chunks(n):
    """Chunks whose G is formed by the vector units, and by the matrix cores; rows off 16 bytes, so that all of H is laid
    out (n = 9: by more than 2^25 blocks).  P and what its rounding to bf16 leaves are 2^-16 of the targets' P, the rest 2^-8."""
    N, V, d = 2 ** 24 + 3, 2, 1
    g = torch.Generator(device="cuda").manual_seed(4)
    H = torch.randint(-4, 5, (N, n, d), generator=g, device="cuda", dtype=torch.int8).bfloat16()
    W = torch.tensor([[0.5], [-0.25]], device="cuda").bfloat16()
    label = torch.randint(-1, V, (N, n), generator=g, device="cuda", dtype=torch.int32)
    loss, lse = gcx.gc_softmax_xent(H, W, label)
    dH, G = gcx.gc_softmax_xent_grads(H, W, label, lse)
    for part in (slice(0, 1 << 20), slice(2 ** 21 - 99, 2 ** 21 + 99), slice(N - (1 << 20), N)):
        check_losses(H[part].view(-1, d), W, label[part].reshape(-1), loss[part].reshape(-1), lse[part].reshape(-1))
        h, y = H[part].double(), label[part].long()
        z = h * W[:, 0].double()
        P = torch.softmax(z, -1)
        P.scatter_add_(2, y.clamp(min=0)[..., None], torch.full_like(P[..., :1], -1.0))
        P = torch.where((y >= 0)[..., None], P, 0.0)
        want = P @ W.double()
        bar = 2.0 ** -8 * (P.abs() @ W.double().abs()) + 2.0 ** -18
        assert bool(((dH[part].double() - want).abs() <= bar + 2.0 ** -8 * (want.abs() + bar)).all())
        want = (P * h).sum(1)
        bar = 2.0 ** -8 * (P * h).abs().sum(1) + 2.0 ** -18 * h.abs().sum(1)
        assert bool(((G[part, :, 0].double() - want).abs() <= bar + 2.0 ** -8 * (want.abs() + bar)).all())
    del P, z, h
    assert bool(dH.isfinite().all()) and bool(G.isfinite().all())
