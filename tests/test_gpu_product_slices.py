"""GPU: products in slices of k, in every tile that takes them, how exactly a float32
result is summed, and everything that may become of the sums at once, against a plain
implementation in 64 bits.

Tolerances are bounds, not measured values.
  element  as for products in one piece: (k / 16 + 64 + 16 + 3) 2^-23 sum |a b|, for a
           bf16 out 7 2^-13 sum |a b| more, then bias and the result's rounding.
  norm     of a float32 result's error, which that bound leaves too wide: it would let an
           8-bit instruction's sums pass (1.5e-5 of the norm, 252 steps of 2^-24). Products are
           exact in float32. A matrix instruction adds 16 to a running sum, with at
           most four roundings of half a step, 2^-24 of that sum. Terms are centred, so
           after i of k / 16 instructions the sum's norm is sqrt(16 i / k) of the result's, and
           the roundings, of either sign, add as squares: 2^-24 sqrt(4 sum_i 16 i / k) =
           2^-24 sqrt(2 k / 16) of the norm. Slices shorten the sums that round and add one
           rounding of each plane's sum, at most 16 more, of sums no larger than the
           result: 2^-24 (sqrt(k / 8) + 4) in all, and the result's own.
"""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from product_shapes import KINDS, SLICED, WHOLE                                          # noqa: E402
from test_gpu_blocks import BF, F32, HALF, STEP, _close, _expected, _gen, _native, _operand, _randn, _scale, _tolerance   # noqa: E402


def _norm_bound(k):
    return STEP * ((k / 8) ** 0.5 + 5)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", SLICED)
def test_slices_match_the_definition(shape, kind):
    native = _native()
    m, n, k = shape
    print(f"[slices] {shape} {kind}", flush=True)
    g = _gen(m + 3 * n + 7 * k)
    a, sa, A = _operand(m, k, g)
    b, sb, B = _operand(n, k, g, tiles=kind != "float32", scale=k ** -0.5)
    out_t = BF if kind in ("bf16", "masked") else F32
    bias = {"bf16": _randn((n,), g, BF), "masked": _randn((n,), g, F32)}.get(kind)
    mask = _randn((m, n + 3), g, out_t)[:, :n] if kind == "masked" else None
    p = native.Product(m, n, k, relu=kind == "masked", accumulate=kind == "added")
    room = torch.full((m + 2, n + 5), 3.0, dtype=out_t, device="cuda")
    out, ws = room[1:-1, 3:3 + n], p.workspace()
    ws.fill_(255)                                              # planes of NaN
    p.apply(a, sa, b, sb, out, bias=bias, mask=mask, workspace=ws)
    want = _expected(A, B, bias, kind == "masked", mask)
    tol = _tolerance(out_t, k, A, B, _scale(a, sa), _scale(b, sb), bias)
    if out_t == F32:
        old = 3.0 if kind == "added" else 0.0                  # one more rounding, of the sum with it
        off = (out.double() - old - want).norm()
        assert float(off) <= _norm_bound(k) * float(want.norm()) + STEP * float((want + old).norm()), float(off / want.norm())
        want, tol = want + old, tol + STEP * (want.abs() + old)
    _close(out, want, tol + HALF[out_t] * (want.abs() + tol) + 1e-300, "out")
    got = out.clone()
    for _ in range(2):                                         # the same bits again
        out.fill_(3.0)
        ws.fill_(255)
        p.apply(a, sa, b, sb, out, bias=bias, mask=mask, workspace=ws)
        assert torch.equal(out, got)
    out.fill_(3.0)
    assert bool((room == 3.0).all()), "values around out were written"


@pytest.mark.parametrize("shape", [(16, 1000, 1531), (31, 500, 2049), (33, 300, 4096), (64, 64, 8192), (300, 16, 6000),
                                   (777, 500, 333), (1531, 3001, 272), (1000, 130, 5000), (4090, 4081, 1003),
                                   (4090, 4081, 6001), (20, 16401, 700)])
def test_a_float32_result_is_summed_in_float32(shape):
    native = _native()
    m, n, k = shape
    g = _gen(m + n + k)
    (a, sa, A), (b, sb, B) = _operand(m, k, g), _operand(n, k, g, tiles=True)
    p = native.Product(m, n, k)
    out = torch.empty(m, n, device="cuda")
    p.apply(a, sa, b, sb, out, workspace=p.workspace())
    want = A @ B.t()
    off = float((out.double() - want).norm() / want.norm())
    print(f"[float32] {shape} {off:.2e} of the norm", flush=True)
    assert off <= _norm_bound(k)


@pytest.mark.parametrize("out_t", [F32, BF], ids=["float32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 33, 7), (31, 500, 300), *WHOLE, (300, 301, 6001), (69, 2883, 11031)])
def test_bias_relu_mask_and_what_was_there_together(shape, out_t):
    """A bias of the other type, ReLU, a mask in rows that start at odd elements; into float32 also added."""
    native = _native()
    m, n, k = shape
    print(f"[together] {shape} {out_t}", flush=True)
    g = _gen(m + n + 5 * k)
    (a, sa, A), (b, sb, B) = _operand(m, k, g), _operand(n, k, g, tiles=True, scale=k ** -0.5)
    bias = _randn((n,), g, BF if out_t == F32 else F32)
    mask = _randn((m, n + 5), g, out_t)[:, 3:3 + n]
    mask[0, 0], mask[-1, -1], mask[m // 2, n // 2] = float("nan"), 0.0, -0.0
    p = native.Product(m, n, k, relu=True, accumulate=out_t == F32)
    room = _randn((m + 2, n + 7), g, out_t)
    before, out, ws = room.clone(), room[1:-1, 5:5 + n], p.workspace()
    ws.fill_(255)
    old = out.double() if out_t == F32 else torch.zeros(m, n, dtype=torch.float64, device="cuda")
    p.apply(a, sa, b, sb, out, bias=bias, mask=mask, workspace=ws)
    want = _expected(A, B, bias, True, mask)
    tol = _tolerance(out_t, k, A, B, _scale(a, sa), _scale(b, sb), bias)
    tol = torch.where(mask.double() > 0, tol, torch.zeros_like(tol))         # a masked element is 0, or what was there
    if out_t == F32:
        want, tol = want + old, tol + STEP * (want.abs() + old.abs() + tol)
    _close(out, want, tol + HALF[out_t] * (want.abs() + tol) + 1e-300, "out")
    assert torch.equal(out[~(mask > 0)].double(), old[~(mask > 0)])
    out.copy_(before[1:-1, 5:5 + n])
    assert torch.equal(room, before), "values around out were written"
