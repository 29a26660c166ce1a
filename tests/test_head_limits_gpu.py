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
