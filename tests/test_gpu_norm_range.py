"""GPU: the root-mean-square norm where its statistics are hard to hold (mean squares
below float32's normal numbers, rows of unlike values) and over many rows, against a
plain implementation in 64 bits.

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


# Rows by the thousand. The forward takes up to 65536 blocks of one row (past 1024 columns), then each
# block another; the backward 512 blocks at most, of four waves that take rows by
# themselves (up to 1024 columns) or one group of threads: they walk three rows and more here.
ROWS = [(65600, 1032, torch.bfloat16), (1700, 1531, torch.float32), (5000, 512, torch.bfloat16),
        (2600, 8192, torch.bfloat16), (1541, 8200, torch.bfloat16)]


@pytest.mark.parametrize("shape", ROWS, ids=lambda s: f"{s[0]}x{s[1]}-{str(s[2])[6:]}")
def test_many_rows_match_the_definition(shape):
    """The backward's bounds are those of few rows (dx: 256 steps of 2^-24); dweight adds up a group's rows, up to
    seven other groups', then 16 partial rows of a run and 32 runs, of terms that are 52 steps off."""
    native = _native()
    R, C, dtype = shape
    print(f"[norm rows] {shape}", flush=True)
    half = torch.finfo(dtype).eps / 2
    x, dy = _randn((R, C), 1).to(dtype), _randn((R, C), 2).to(dtype)
    w = 1 + 0.2 * _randn((C,), 3)
    norm = native.RmsNorm(C, eps=1e-5)
    y, rstd = torch.empty_like(x), torch.empty(R, device="cuda")
    codes, scales = native.blocks_empty(R, C)
    norm.forward(x, w, y, codes=codes, scales=scales, rstd=rstd)
    dx, dw, ws = torch.empty_like(x), torch.empty(C, device="cuda"), norm.workspace(R)
    ws.fill_(255)
    norm.backward(dy, x, w, rstd, dx, dw, workspace=ws)
    total, size = torch.zeros(C, dtype=torch.float64, device="cuda"), torch.zeros(C, dtype=torch.float64, device="cuda")
    back = torch.empty_like(x)
    native.blocks_restore(codes, scales, back)
    unit = torch.exp2(scales.double() - 127).repeat_interleave(128, 0)[:C]
    for r in range(0, R, 8192):                                # float64 by the piece
        s = slice(r, r + 8192)
        h, d, i = x[s].double(), dy[s].double(), _statistics(x[s], 1e-5)
        _close(rstd[s, None], i, ONCE * i, "rstd")
        z = h * i
        want = z * w.double()
        _close(y[s], want, want.abs() * (ONCE + half * (1 + ONCE)) if dtype != torch.float32 else want.abs() * ONCE, "y")
        _close(back[s], want, torch.maximum(want.abs() * 2.0 ** -4, unit[:, s].t() * 2.0 ** -10) + 2 * ONCE * want.abs(), "codes")
        u = d * w.double()
        mean = (u * z).mean(1, keepdim=True)
        want = i * (u - z * mean)
        tol = 256 * STEP * i * (u.abs() + z.abs() * (u * z).abs().mean(1, keepdim=True))
        _close(dx[s], want, tol + half * (want.abs() + tol), "dx")
        total += (d * z).sum(0)
        size += (d * z).abs().sum(0)
    _close(dw, total, (R / 512 + 1 + 7 + 16 + 32 + 52) * STEP * size, "dweight")
    again, dw2 = torch.empty_like(dx), torch.empty_like(dw)
    ws.fill_(255)
    norm.backward(dy, x, w, rstd, again, dw2, workspace=ws)
    assert torch.equal(again, dx) and torch.equal(dw2, dw)


@pytest.mark.parametrize("shape", [(7, 1531), (33, 512), (3, 8200), (2, 30000)])
def test_statistics_are_held_in_64_bits(shape):
    """Rows whose squares differ by far, where sums in float32 lose steps: rstd and y are rounded once, and codes are
    those of the float32 y."""
    native = _native()
    R, C = shape
    h = _randn(shape, R) * torch.exp(2 * _randn((R, 1), 5)) * torch.exp(_randn((1, C), 6))
    w = 1 + 0.2 * _randn((C,), 7)
    norm = native.RmsNorm(C, eps=1e-6)
    y, rstd = torch.empty_like(h), torch.empty(R, device="cuda")
    codes, scales = native.blocks_empty(R, C)
    norm.forward(h, w, y, codes=codes, scales=scales, rstd=rstd)
    r = _statistics(h, 1e-6)
    _close(rstd[:, None], r, ONCE * r, "rstd")
    want = h.double() * r * w.double()
    _close(y, want, ONCE * want.abs(), "y")
    packed = native.blocks_empty(R, C)
    native.blocks_pack(y, *packed)
    assert torch.equal(packed[0], codes) and torch.equal(packed[1], scales)
