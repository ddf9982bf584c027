"""GPU: the root-mean-square norm where its statistics are hard to hold: mean squares
below float32's normal numbers, against a plain implementation in 64 bits.

Tolerances are bounds, not measured values. Squares of float32 values and their sums
are held in 64 bits, so a mean is off by some 2^-47 of its size at the most (32 additions in a
thread, 21 behind it). The root starts from float32's: m, its root and the reciprocal are
rounded, 2.5 steps of 2^-24, and one step of Newton's iteration leaves 1.5 times that
squared, 2^-44.7. Then rstd, and y in float32, are rounded once: 2^-24 (1 + 2^-16) of the value,
2^-150 at the least."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

STEP = 2.0 ** -24
ONCE = STEP * (1 + 2.0 ** -16)


def _native():
    from paper_1809_02839_amd import native
    return native


def _randn(shape, seed, scale=1.0):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * scale


def _statistics(h, eps):
    eps = float(torch.tensor(eps, dtype=torch.float32).double())       # as the call takes it
    return 1 / torch.sqrt(h.double().square().mean(1, keepdim=True) + eps)


def _close(got, want, tol, what):
    off = (got.double() - want).abs()
    assert bool((off <= tol + 2.0 ** -150).all()), (what, float((off / (tol + 2.0 ** -150)).max()))


@pytest.mark.parametrize("eps", [2.0 ** -149, 3e-45, 1e-44, 1e-41, 1e-38, 1.2e-38, 1e-30])
@pytest.mark.parametrize("cols", [1, 200, 1531, 8200])
def test_mean_squares_below_the_normal_numbers(cols, eps):
    native = _native()
    print(f"[norm range] {cols} {eps}", flush=True)
    size = torch.tensor([0.0, 1e-30, 1e-23, 3e-23, 1e-22, 1e-21, 1e-20, 1e-19, 1e-12], device="cuda")[:, None]
    h = _randn((9, cols), cols) * size
    w = 1 + 0.2 * _randn((cols,), 7)
    y, rstd = torch.empty_like(h), torch.empty(9, device="cuda")
    norm = native.RmsNorm(cols, eps=eps)
    norm.forward(h, w, y, rstd=rstd)
    r = _statistics(h, eps)
    assert math.isfinite(float(r.max()))
    _close(rstd[:, None], r, ONCE * r, "rstd")
    want = h.double() * r * w.double()
    _close(y, want, ONCE * want.abs(), "y")
