"""GPU: tensors in blocks of 128, the root-mean-square norm and the product of
tensors in blocks, against plain implementations in 64 bits.

Tolerances are bounds, not measured values (half a step: fp32 2^-24, bf16 2^-8,
e4m3 2^-4, all relative).
  blocks   exact: a scale is a power of two, the code's rounding is the definition.
  norm     a row's sum of squares in float32 would take at most 64 additions in a
           thread, 6 in a wave and 15 between waves: 85 roundings, half of that on the
           root; the mean, eps, root and reciprocal 5 more, y two: 50 steps of 2^-24
           and y's own rounding. An 8-bit y is a code of such a value.
  dx       u, z and the mean of u z (at most 64 + 21 additions of terms that are 53
           steps off): below 256 steps of 2^-24 of r (|u| + |z| mean|u z|).
  dweight  at most rows / 256 + 1 additions in a thread, 128 in a run of partial
           rows, 8 runs; each term 52 steps off.
  product  every product is exact in float32; a matrix instruction adds up to 64 of
           them, each no further off than 2^-23 of the largest partial sum, k / 16 such
           sums follow each other, at most 16 slices of k are added: below
           (k / 16 + 64 + 16 + 3) 2^-23 of sum |a b|, bias and the result's rounding.
           A bf16 out is summed by the 8-bit instruction, which cuts seven of eight
           consecutive products 2^-13 below the largest power of two that codes of
           their exponents have (small codes count as 2^-6): 7 2^-13 sum |a b| more,
           |a| and |b| at least 2^-6 of their scale.
"""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

STEP = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
BF, F32 = torch.bfloat16, torch.float32


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(shape, g, dtype=BF, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _native():
    from paper_1809_02839_amd import native
    return native


# ------------------------------------------------------------- definitions ----

def _powers():
    return torch.tensor([2.0 ** i for i in range(-300, 301)], dtype=torch.float64, device="cuda")


def _two(e):
    return _powers()[e.long() + 300]


def _exponents(top):
    """Smallest e in [-117, 120] with top <= 448 * 2^e, by trial of each."""
    e = torch.full(top.shape, -117, dtype=torch.int64, device=top.device)
    for s in range(-116, 121):
        e = torch.where(top > 448 * 2.0 ** (s - 1), torch.full_like(e, s), e)
    return e


def _nearest(z):
    """Nearest e4m3 number of float64 z within +-448, ties to even."""
    step = _two(torch.frexp(z.abs().clamp(min=2.0 ** -6))[1] - 4)
    return torch.round(z / step) * step


def _packed(x, tiles=False):
    """Float64 definition: values, and scale bytes [block columns, rows]."""
    R, C = x.shape
    x = x.double()
    out = torch.empty_like(x)
    byte = torch.empty(-(-C // 128), R, dtype=torch.uint8, device=x.device)
    high = 128 if tiles else R
    for r in range(0, R, high):
        for n in range(byte.shape[0]):
            y = x[r:r + high, 128 * n:128 * n + 128]
            size = torch.where(y.isfinite(), y.abs(), torch.zeros_like(y))
            e = _exponents(size.amax().expand(y.shape[0]) if tiles else size.amax(1))
            byte[n, r:r + high] = (e + 127).to(torch.uint8)
            limit = torch.where(e == 120, 240.0, 448.0).double()[:, None]
            z = torch.minimum(torch.maximum(y * _two(-e)[:, None], -limit), limit)
            value = _nearest(torch.where(y.isfinite(), z, torch.zeros_like(z))) * _two(e)[:, None]
            out[r:r + high, 128 * n:128 * n + 128] = torch.where(y.isfinite(), value, torch.full_like(z, math.nan))
    return out, byte


def _same(a, b):
    return torch.equal(a.double().nan_to_num(nan=12345.0), b.double().nan_to_num(nan=12345.0))


def _table():
    code = torch.arange(256, device="cuda")
    power, part = (code >> 3) & 15, (code & 7).double() / 8
    size = torch.where(power == 0, part * 2.0 ** -6, (1 + part) * _two(power - 7))
    size = torch.where((code & 127) == 127, torch.full_like(size, math.nan), size)
    return torch.where(code >= 128, -size, size)


def _value(codes, scales):
    """Float64 values of codes and scales, from their bits."""
    e = scales.long() - 127
    return _table()[codes.long()] * _two(e).repeat_interleave(128, 0)[:codes.shape[1]].t()


def _guarded(rows, cols):
    """Codes and scales inside larger tensors of 0xab bytes, and those."""
    room = torch.full((rows + 2, -(-cols // 16) * 16 + 32), 0xab, dtype=torch.uint8, device="cuda")
    side = torch.full((-(-cols // 128) + 2, -(-rows // 16) * 16 + 32), 0xab, dtype=torch.uint8, device="cuda")
    return room[1:-1, 16:16 + cols], side[1:-1, 16:16 + rows], (room, side)


def _untouched(codes, scales, rooms):
    for t, room in ((codes, rooms[0]), (scales, rooms[1])):
        kept = t.clone()
        t.fill_(0xab)
        assert bool((room == 0xab).all()), "bytes around a tensor were written"
        t.copy_(kept)


# ------------------------------------------------------------------ blocks ----

SHAPES = [(1, 1), (1, 128), (3, 129), (7, 95), (128, 128), (130, 256), (5, 8), (2, 1000), (257, 72), (1, 4096),
          (131, 385), (129, 16), (300, 7)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tiles", [False, True], ids=["rows", "tiles"])
@pytest.mark.parametrize("shape", SHAPES)
def test_blocks_match_the_definition(shape, tiles, dtype):
    native = _native()
    print(f"[blocks] {shape} {tiles} {dtype}", flush=True)
    g = _gen(shape[0] + 3 * shape[1])
    R, C = shape
    big = torch.exp2(torch.randint(-140, 125, (R, 1), generator=g, device="cuda").float())   # rows over the whole range
    for scale in (1.0, big):
        x = (torch.randn(shape, generator=g, device="cuda") * scale * 4.0 ** torch.randint(
            -9, 1, shape, generator=g, device="cuda").float()).to(dtype)
        x[torch.rand(shape, generator=g, device="cuda") < 0.1] = 0.0
        want, byte = _packed(x, tiles)
        want_t, byte_t = _packed(x.t().contiguous(), tiles)
        codes, scales, rooms = _guarded(R, C)
        tcodes, tscales, trooms = _guarded(C, R)
        native.blocks_pack(x, codes, scales, tcodes, tscales, tiles=tiles)
        _untouched(codes, scales, rooms)
        _untouched(tcodes, tscales, trooms)
        assert torch.equal(scales, byte) and torch.equal(tscales, byte_t)
        for back in (BF, F32):
            for c, s, w in ((codes, scales, want), (tcodes, tscales, want_t)):
                out = torch.empty(w.shape, dtype=back, device="cuda")
                native.blocks_restore(c, s, out)
                assert torch.equal(out.double(), w)
                assert torch.equal(_value(c, s), w)
        if tiles:
            assert torch.equal(tcodes.t(), codes)
        for one in ((codes, scales, None, None), (None, None, tcodes, tscales)):      # either orientation by itself
            before = [None if t is None else t.clone() for t in one]
            for t in one:
                if t is not None:
                    t.zero_()
            native.blocks_pack(x, *one, tiles=tiles)
            assert all(t is None or torch.equal(t, b) for t, b in zip(one, before))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tiles", [False, True], ids=["rows", "tiles"])
def test_blocks_special_values_and_strides(dtype, tiles):
    native = _native()
    top, inf, nan = torch.finfo(dtype).max, math.inf, math.nan
    x = torch.zeros(6, 200, dtype=dtype, device="cuda")
    x[0, :4] = torch.tensor([top, -top, top * 0.5, 1.0])           # the largest: no infinity comes back
    x[1, 126:131] = torch.tensor([inf, -inf, nan, 3.0, -448.0])    # not finite: NaN, and no part of the scale
    x[2, :3] = torch.tensor([1e-38, -1e-38, -0.0])
    x[3, :4] = torch.tensor([448.0, 0.4, -0.6, 9.0])               # far below the largest: may become zero
    x[4, :] = nan
    x = x[:5] if tiles else x
    for bad in (range(5) if tiles else [None]):                    # a tile's largest is one: rows by themselves
        part = x if bad is None else x[bad:bad + 1]
        R = part.shape[0]
        want, byte = _packed(part, tiles)
        room = torch.full((R, 217), 5.0, dtype=dtype, device="cuda")    # rows that start at odd elements
        view = room[:, 9:209]
        view.copy_(part)
        codes, scales = native.blocks_empty(R, 200)
        tcodes, tscales = native.blocks_empty(200, R)
        native.blocks_pack(view, codes, scales, tcodes, tscales, tiles=tiles)
        assert torch.equal(scales, byte) and _same(_value(codes, scales), want)
        assert _same(_value(tcodes, tscales), _packed(part.t().contiguous(), tiles)[0])
        room.fill_(5.0)
        native.blocks_restore(codes, scales, view)
        assert _same(view, want) and bool((room[:, :9] == 5.0).all()) and bool((room[:, 209:] == 5.0).all())


def test_blocks_of_nothing_and_offsets_past_32_bits():
    native = _native()
    for R, C in ((0, 5), (5, 0), (0, 0)):
        x = torch.empty(R, C, dtype=BF, device="cuda")
        native.blocks_pack(x, *native.blocks_empty(R, C), *native.blocks_empty(C, R))
        native.blocks_restore(*native.blocks_empty(R, C), x)
    R, wide = 70001, 1 << 16
    room = torch.empty(R * wide, dtype=BF, device="cuda").view(R, wide)        # 9 GB: the last rows lie past 2^32 bytes
    x = room[:, wide - 200:]
    x.copy_(_randn((R, 200), _gen(3)))
    codes = torch.zeros(R, wide, dtype=torch.uint8, device="cuda")[:, :200]
    scales = native.blocks_empty(R, 200)[1]
    tcodes, tscales = native.blocks_empty(200, R)
    native.blocks_pack(x, codes, scales, tcodes, tscales)
    last = slice(R // 128 * 128 - 256, R)
    want, byte = _packed(x[last])
    assert torch.equal(scales[:, last], byte) and torch.equal(_value(codes[last], scales[:, last]), want)
    want = _packed(x[last].t().contiguous())[0]
    assert torch.equal(_value(tcodes[:, last], tscales[last.start // 128:]), want)
    x.zero_()
    native.blocks_restore(codes, scales, x)
    assert torch.equal(x[last].double(), _packed(_randn((R, 200), _gen(3))[last])[0])


# -------------------------------------------------------------------- norm ----

def _normed(h, w, eps):
    """z, r and y in float64."""
    r = 1 / torch.sqrt(h.square().mean(1, keepdim=True) + eps)
    return h * r, r, h * r * w


def _close(got, want, tol, what):
    off = (got.double() - want).abs()
    assert bool((off <= tol).all()), (what, float((off / tol.clamp(min=1e-300)).max()))


TYPES = [(BF, BF, F32), (F32, F32, F32), (F32, BF, BF)]
NORMS = [(1, 1), (3, 7), (5, 64), (2, 513), (9, 1000), (130, 512), (67, 1531), (33, 2048), (3, 4096), (2, 8200),
         (1100, 128), (5, 16384), (2, 30000), (1, 32768), (3, 17001)]


def _views(shape, g, dtype, odd, scale=1.0):
    """A tensor by itself, or inside a larger one whose rows start at odd elements."""
    t = _randn(shape, g, dtype, scale)
    if not odd:
        return t
    room = torch.full((shape[0], shape[1] + 13), 3.0, dtype=dtype, device="cuda")
    room[:, 5:5 + shape[1]] = t
    return room[:, 5:5 + shape[1]]


@pytest.mark.parametrize("odd", [False, True], ids=["whole", "views"])
@pytest.mark.parametrize("types", TYPES, ids=lambda t: "-".join(str(x)[6:] for x in t))
@pytest.mark.parametrize("shape", NORMS)
def test_norm_and_gradients_match_the_definition(shape, types, odd):
    native = _native()
    T, Y, W = types
    print(f"[norm] {shape} {types} {odd}", flush=True)
    g = _gen(shape[0] * 7 + shape[1])
    R, C = shape
    x, res = _views(shape, g, T, odd), _views(shape, g, T, odd, 0.5)
    w = (1 + 0.2 * torch.randn(C, generator=g, device="cuda")).to(W)
    norm = native.RmsNorm(C, eps=1e-5)
    total, y = _views(shape, g, T, odd), _views(shape, g, Y, odd)
    rstd = torch.empty(R, device="cuda")
    codes, scales, rooms = _guarded(R, C)
    norm.forward(x, w, y, residual=res, sum=total, codes=codes, scales=scales, rstd=rstd)
    _untouched(codes, scales, rooms)
    exact = x.double() + res.double()
    _close(total, exact, exact.abs() * (HALF[T] + STEP), "sum")
    h = total.double()
    z, r, want = _normed(h, w.double(), 1e-5)
    _close(rstd[:, None], r, r * 48 * STEP, "rstd")
    _close(y, want, want.abs() * (50 * STEP + HALF[Y] * (1 + 50 * STEP)), "y")
    # the 8-bit output: a code of a value that is 50 steps from y, under the scale of such a largest one
    e = scales.long() - 127
    for n in range(scales.shape[0]):
        top = want[:, 128 * n:128 * n + 128].abs().amax(1)
        assert bool(((e[n] >= _exponents(top * (1 - 50 * STEP))) & (e[n] <= _exponents(top * (1 + 50 * STEP)))).all())
    unit = _two(e).repeat_interleave(128, 0)[:C].t()
    near = torch.maximum(want.abs() * 2.0 ** -4, unit * 2.0 ** -10)
    _close(_value(codes, scales), want, near + want.abs() * 60 * STEP, "codes")
    # no residual, blocks alone, y alone
    again, y2 = native.blocks_empty(R, C), torch.empty(shape, dtype=Y, device="cuda")
    norm.forward(total, w, codes=again[0], scales=again[1])
    norm.forward(total, w, y2)
    assert torch.equal(again[0], codes) and torch.equal(again[1], scales) and torch.equal(y2, y)

    dy, dsum = _views(shape, g, Y, odd), _views(shape, g, T, odd)
    for d in (dsum, None):
        dx, dw = _views(shape, g, T, odd), torch.empty(C, device="cuda")
        ws = norm.workspace(R)
        ws.fill_(255)
        norm.backward(dy, total, w, rstd, dx, dw, dsum=d, workspace=ws)
        u = dy.double() * w.double()
        mean = (u * z).mean(1, keepdim=True)
        want = r * (u - z * mean)
        tol = 256 * STEP * r * (u.abs() + z.abs() * (u * z).abs().mean(1, keepdim=True))
        if d is not None:
            want, tol = want + d.double(), tol + 2 * STEP * d.double().abs()
        _close(dx, want, tol + HALF[T] * (want.abs() + tol), "dx")
        terms = dy.double() * z
        _close(dw, terms.sum(0), (R / 256 + 1 + 128 + 8 + 52) * STEP * terms.abs().sum(0) + 1e-300, "dweight")


def test_norm_in_place_and_repeats_bitwise():
    native = _native()
    g = _gen(5)
    for R, C in ((37, 512), (5, 1531), (6, 8192)):
        x, res, w = _randn((R, C), g), _randn((R, C), g), _randn((C,), g, F32)
        norm = native.RmsNorm(C)
        want = [torch.empty_like(x), torch.empty_like(x), torch.empty(R, device="cuda")]
        norm.forward(x, w, want[1], residual=res, sum=want[0], rstd=want[2])
        for place in (x.clone(), res.clone()):
            other = res if torch.equal(place, x) else x
            y = torch.empty_like(x)
            norm.forward(place, w, y, residual=other, sum=place)
            assert torch.equal(place, want[0]) and torch.equal(y, want[1])
            place = other.clone()
            norm.forward(x if torch.equal(other, res) else res, w, y, residual=place, sum=place)
            assert torch.equal(place, want[0]) and torch.equal(y, want[1])
        dy, dsum = _randn((R, C), g), _randn((R, C), g)
        dx, dw, ws = torch.empty_like(x), torch.empty(C, device="cuda"), norm.workspace(R)
        norm.backward(dy, want[0], w, want[2], dx, dw, dsum=dsum, workspace=ws)
        for which in ("dsum", "dy"):
            a, b, dw2 = dy.clone(), dsum.clone(), torch.empty_like(dw)
            norm.backward(a, want[0], w, want[2], b if which == "dsum" else a, dw2, dsum=b, workspace=ws)
            assert torch.equal(b if which == "dsum" else a, dx) and torch.equal(dw2, dw)


def test_norm_special_rows():
    native = _native()
    for dtype in (BF, F32):
        h = torch.zeros(5, 300, dtype=dtype, device="cuda")
        h[1, 7] = math.inf
        h[2, 290] = math.nan
        h[3] = 2.0 ** 70                                    # squares past float32: rstd 0
        h[4, 5] = 1e-30
        w = torch.full((300,), 2.0, device="cuda")
        y, rstd = torch.empty_like(h), torch.empty(5, device="cuda")
        norm = native.RmsNorm(300, eps=1e-6)
        codes, scales = native.blocks_empty(5, 300)
        norm.forward(h, w, y, codes=codes, scales=scales, rstd=rstd)
        got = _value(codes, scales)
        for out in (y.double(), got):
            assert bool((out[0] == 0).all()) and bool((out[3] == 0).all())
            assert bool(out[1, 7].isnan()) and int(out[1].isnan().sum()) == 1 and bool(out[2].isnan().all())
        assert rstd[1] == 0 and bool(rstd[2].isnan()) and rstd[3] == 0 and abs(float(rstd[0]) - 1000) < 1e-2
        assert abs(float(y[4, 5]) / 2e-27 - 1) < 0.01
        dx, dw = torch.empty_like(h), torch.empty(300, device="cuda")
        dy = torch.ones_like(h)
        keep = [0, 3, 4]
        norm.backward(dy[keep], h[keep], w, rstd[keep], dx[:3], dw, workspace=norm.workspace(3))
        assert bool((dx[1] == 0).all()) and bool(dx[:3].isfinite().all()) and bool(dw.isfinite().all())
        norm.backward(dy[:0], h[:0], w, rstd[:0], dx[:0], dw, workspace=norm.workspace(0))
        assert bool((dw == 0).all())                        # a sum over no rows
        norm.forward(h[:0], w, y[:0])


def test_norm_gradients_match_differences():
    native = _native()
    g = _gen(11)
    R, C = 9, 200
    x, w, dy = _randn((R, C), g, F32), 1 + 0.2 * _randn((C,), g, F32), _randn((R, C), g, F32)
    norm = native.RmsNorm(C, eps=1e-3)
    y, rstd = torch.empty_like(x), torch.empty(R, device="cuda")
    norm.forward(x, w, y, rstd=rstd)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    norm.backward(dy, x, w, rstd, dx, dw, workspace=norm.workspace(R))

    def loss(h, v):
        out = torch.empty_like(h)
        norm.forward(h, v, out)
        return (out.double() * dy.double()).sum()

    def loss64(h, v):
        return (_normed(h.double(), v.double(), 1e-3)[2] * dy.double()).sum()

    for seed in range(4):
        gd = _gen(seed)
        a, b, s = _randn((R, C), gd, F32), _randn((C,), gd, F32), 2.0 ** -6
        ends = (x + s * a, w + s * b), (x - s * a, w - s * b)          # rounded steps: differences of what was asked
        da, db = ends[0][0].double() - ends[1][0].double(), ends[0][1].double() - ends[1][1].double()
        slope = (loss(*ends[0]) - loss(*ends[1]))
        want = (dx.double() * da).sum() + (dw.double() * db).sum()
        exact = loss64(*ends[0]) - loss64(*ends[1])
        h = x.double().requires_grad_(True)
        v = w.double().requires_grad_(True)
        gh, gv = torch.autograd.grad((_normed(h, v, 1e-3)[2] * dy.double()).sum(), (h, v))
        curved = (exact - (gh * da).sum() - (gv * db).sum()).abs()     # what the difference itself is off by
        z, r, _ = _normed(x.double(), w.double(), 1e-3)
        u = dy.double() * w.double()
        size = r * (u.abs() + z.abs() * (u * z).abs().mean(1, keepdim=True))
        rounding = 2 * 52 * STEP * sum((_normed(e.double(), f.double(), 1e-3)[2] * dy.double()).abs().sum() for e, f in ends)
        rounding += 257 * STEP * ((size * da.abs()).sum() + ((dy.double() * z).abs().sum(0) * db.abs()).sum())
        assert abs(float(slope - want)) <= float(curved + rounding)


# ----------------------------------------------------------------- product ----

def _operand(rows, cols, g, tiles=False, scale=1.0):
    """Codes and scales in tensors whose other bytes are NaN codes, and their values."""
    native = _native()
    codes, scales, rooms = _guarded(rows, cols)
    x = torch.randn(rows, cols, generator=g, device="cuda") * scale
    x *= torch.exp2(torch.randint(-3, 4, (rows, 1), generator=g, device="cuda").float())
    native.blocks_pack(x, codes, scales, tiles=tiles)
    for t, room in ((codes, rooms[0]), (scales, rooms[1])):
        kept = t.clone()
        room.fill_(0xff)
        t.copy_(kept)
    return codes, scales, _value(codes, scales)


PRODUCTS = [(1, 1, 1), (1, 40, 128), (3, 33, 7), (5, 2048, 512), (16, 1000, 1531), (17, 129, 64), (31, 500, 2049),
            (33, 300, 4096), (64, 64, 8192), (65, 127, 129), (100, 1, 777), (128, 128, 128), (130, 257, 384),
            (256, 512, 1024), (300, 16, 6000), (777, 500, 333), (1000, 130, 5000), (513, 769, 640), (256, 256, 16),
            (2000, 1030, 2056), (1531, 3001, 272), (20, 16401, 700), (32, 16384, 130),
            (9, 9001, 1500), (16, 17000, 64), (4090, 4081, 1003), (4096, 4096, 4000), (4090, 4081, 6001)]


def _scale(codes, scales):
    """Float64 scale of every code."""
    return _two(scales.long() - 127).repeat_interleave(128, 0)[:codes.shape[1]].t()


def _tolerance(out_t, k, A, B, a_scale, b_scale, bias=None):
    """Of the sums before the result's rounding."""
    tol = (k / 16 + 64 + 16 + 3) * 2 * STEP * (A.abs() @ B.abs().t() + (0 if bias is None else bias.double().abs()))
    if out_t == BF:
        tol = tol + 7 * 2.0 ** -13 * (torch.maximum(A.abs(), a_scale * 2.0 ** -6)
                                      @ torch.maximum(B.abs(), b_scale * 2.0 ** -6).t())
    return tol


def _expected(A, B, bias, relu, mask):
    v = A @ B.t()
    if bias is not None:
        v = v + bias.double()
    if relu:
        v = torch.relu(v)
    if mask is not None:
        v = torch.where(mask.double() > 0, v, torch.zeros_like(v))
    return v


@pytest.mark.parametrize("kind", ["plain", "bf16", "epilogue", "accumulate"])
@pytest.mark.parametrize("shape", PRODUCTS)
def test_product_matches_the_definition(shape, kind):
    native = _native()
    m, n, k = shape
    print(f"[product] {shape} {kind}", flush=True)
    g = _gen(m + 3 * n + 7 * k)
    a, sa, A = _operand(m, k, g)
    b, sb, B = _operand(n, k, g, tiles=kind != "plain", scale=k ** -0.5)
    out_t = F32 if kind in ("plain", "accumulate") else BF
    bias = {"plain": None, "bf16": _randn((n,), g, BF), "epilogue": _randn((n,), g, F32), "accumulate": None}[kind]
    mask = _randn((m, n + 3), g, out_t)[:, :n] if kind == "epilogue" else None
    if mask is not None:
        mask[0, 0] = math.nan
    p = native.Product(m, n, k, relu=kind == "epilogue", accumulate=kind == "accumulate")
    room = torch.full((m + 2, n + 5), 3.0, dtype=out_t, device="cuda")
    out = room[1:-1, 3:3 + n] if kind in ("plain", "bf16") else torch.full((m, n), 3.0, dtype=out_t, device="cuda")
    ws = p.workspace()
    ws.fill_(255)
    assert p.apply(a, sa, b, sb, out, bias=bias, mask=mask, workspace=ws) is out
    want = _expected(A, B, bias, kind == "epilogue", mask)
    tol = _tolerance(out_t, k, A, B, _scale(a, sa), _scale(b, sb), bias)
    if kind == "accumulate":
        want, tol = want + 3.0, tol + STEP * (want.abs() + 3.0)
    _close(out, want, tol + HALF[out_t] * (want.abs() + tol) + 1e-300, "out")
    if out.data_ptr() != room[1:, 3:].data_ptr():
        return
    got = out.clone()
    out.fill_(3.0)
    assert bool((room == 3.0).all()), "values around out were written"
    # an element does not depend on the rows and columns beside it
    if m > 40 and n > 40:
        q = native.Product(m, n, k)
        other = torch.empty(m, n, dtype=out_t, device="cuda")
        a2, b2 = a.clone(), b.clone()
        keep_m, keep_n = torch.rand(m, device="cuda", generator=g) < 0.5, torch.rand(n, device="cuda", generator=g) < 0.5
        wide = torch.zeros(m, -(-k // 16) * 16, dtype=torch.uint8, device="cuda")[:, :k]
        wide_b = torch.zeros(n, -(-k // 16) * 16, dtype=torch.uint8, device="cuda")[:, :k]
        wide.copy_(torch.where(keep_m[:, None], a2, torch.full_like(a2, 0x7f)))
        wide_b.copy_(torch.where(keep_n[:, None], b2, torch.full_like(b2, 0x7f)))
        q.apply(wide, sa, wide_b, sb, other, bias=bias, workspace=ws)
        assert torch.equal(other[keep_m][:, keep_n], got[keep_m][:, keep_n])
        assert bool(other[~keep_m].isnan().all()) and bool(other[:, ~keep_n].isnan().all())


def test_product_of_nothing():
    native = _native()
    for m, n, k in ((0, 5, 7), (5, 0, 7), (0, 0, 0)):
        p = native.Product(m, n, k)
        p.apply(*native.blocks_empty(m, k), *native.blocks_empty(n, k), torch.empty(m, n, device="cuda"),
                workspace=p.workspace())
    for m, n in ((3, 5), (200, 300)):                          # no terms: the bias alone
        p = native.Product(m, n, 0)
        bias = torch.arange(n, device="cuda").float()
        out = torch.full((m, n), 9.0, device="cuda")
        p.apply(*native.blocks_empty(m, 0), *native.blocks_empty(n, 0), out, bias=bias, workspace=p.workspace())
        assert torch.equal(out, bias.expand(m, n))


@pytest.mark.parametrize("out_t", [F32, BF])
@pytest.mark.parametrize("shape", [(9, 70, 300), (200, 300, 520), (300, 520, 1100)])
def test_product_scales_over_their_range(shape, out_t):
    """Sums of blocks whose scales lie anywhere in the format's range, some past float32: infinite as in float32."""
    native = _native()
    m, n, k = shape
    g = _gen(k)
    a, sa, _ = _operand(m, k, g)
    b, sb, _ = _operand(n, k, g)
    for spread in ((10, 130), (117, 137), (120, 248)):
        sa.copy_(torch.randint(*spread, sa.shape, generator=g, device="cuda"))
        sb.copy_(torch.randint(*spread, sb.shape, generator=g, device="cuda"))
        A, B = _value(a, sa), _value(b, sb)
        p = native.Product(m, n, k)
        out = torch.empty(m, n, dtype=out_t, device="cuda")
        p.apply(a, sa, b, sb, out, workspace=p.workspace())
        want, size = _expected(A, B, None, False, None), A.abs() @ B.abs().t()
        sure = size < 2.0 ** 127                               # no partial sum leaves float32
        tol = _tolerance(out_t, k, A, B, _scale(a, sa), _scale(b, sb)) + 2.0 ** -126 * (k + 1)
        off = (out.double() - want).abs()
        assert bool((off <= tol + HALF[out_t] * (want.abs() + tol))[sure].all())
        never = (want.abs() > 2.0 ** 130) & (want.abs() > 0.01 * size)
        assert not bool(out[never].isfinite().any())


def test_product_offsets_past_32_bits():
    native = _native()
    m, n, k = 70001, 200, 300
    g = _gen(2)
    room = torch.empty(m * (1 << 16), dtype=torch.uint8, device="cuda").view(m, 1 << 16)
    A = torch.randn(m, k, generator=g, device="cuda")
    a, sa = room[:, -304:][:, :k], native.blocks_empty(m, k)[1]
    native.blocks_pack(A, a, sa)
    b, sb, B = _operand(n, k, g)
    out = torch.empty(m * (1 << 16), dtype=BF, device="cuda").view(m, 1 << 16)[:, 777:777 + n]
    p = native.Product(m, n, k)
    p.apply(a, sa, b, sb, out, workspace=p.workspace())
    for rows in (slice(0, 300), slice(m - 300, m)):
        A = _value(a[rows], sa[:, rows])
        want = _expected(A, B, None, False, None)
        tol = _tolerance(BF, k, A, B, _scale(a[rows], sa[:, rows]), _scale(b, sb))
        _close(out[rows], want, tol + HALF[BF] * (want.abs() + tol), "out")
    # the long operand second
    out2 = torch.empty(n, m, device="cuda")
    q = native.Product(n, m, k)
    q.apply(b, sb, a, sa, out2, workspace=q.workspace())
    for rows in (slice(0, 300), slice(m - 300, m)):
        A = _value(a[rows], sa[:, rows])
        want, tol = _expected(B, A, None, False, None), _tolerance(F32, k, B, A, None, None)
        _close(out2[:, rows], want, tol + STEP * want.abs(), "out")


# --------------------------------------------------- a layer, as it is used ----

class Layer:
    """A sub-layer h = x + r, y = relu(norm(h) W^T + b) in 8 bits with its gradients, by the library's calls."""

    def __init__(self, T, K, N, seed, stream=None):
        native = _native()
        g = _gen(seed)
        self.x, self.r = _randn((T, K), g), _randn((T, K), g)
        self.gain, self.bias = 1 + 0.1 * _randn((K,), g, F32), 0.1 * _randn((N,), g, F32)
        self.W, self.dy, self.dsum = _randn((N, K), g, F32, K ** -0.5), _randn((T, N), g, BF, 1e-3), _randn((T, K), g)
        e, empty = native.blocks_empty, torch.empty
        self.norm = native.RmsNorm(K)
        self.sum, self.h, self.rstd = empty(T, K, dtype=BF, device="cuda"), empty(T, K, dtype=BF, device="cuda"), empty(T, device="cuda")
        self.h8, self.ht8, self.w8, self.wt8 = e(T, K), e(K, T), e(N, K), e(K, N)
        self.d8, self.dt8 = e(T, N), e(N, T)
        self.products = native.Product(T, N, K, relu=True), native.Product(T, K, N), native.Product(N, K, T)
        self.y, self.dh = empty(T, N, dtype=BF, device="cuda"), empty(T, K, dtype=BF, device="cuda")
        self.dz = torch.zeros(T, N, dtype=BF, device="cuda")
        self.dW, self.dx, self.dgain = empty(N, K, device="cuda"), empty(T, K, dtype=BF, device="cuda"), empty(K, device="cuda")
        self.ws = [p.workspace() for p in self.products] + [self.norm.workspace(T)]

    def outputs(self):
        return [self.sum, self.y, self.dx, self.dW, self.dgain, self.dh]

    def run(self, stream=None):
        native = _native()
        n, s = self.norm, dict(stream=stream)
        native.blocks_pack(self.W, *self.w8, *self.wt8, tiles=True, **s)
        n.forward(self.x, self.gain, self.h, residual=self.r, sum=self.sum, codes=self.h8[0], scales=self.h8[1],
                  rstd=self.rstd, **s)
        f, d, g = self.products
        f.apply(*self.h8, *self.w8, self.y, bias=self.bias, workspace=self.ws[0], **s)
        self.dz.copy_(self.dy * (self.y > 0))
        native.blocks_pack(self.dz, *self.d8, *self.dt8, **s)
        native.blocks_pack(self.h, None, None, *self.ht8, **s)
        d.apply(*self.d8, *self.wt8, self.dh, workspace=self.ws[1], **s)
        g.apply(*self.dt8, *self.ht8, self.dW, workspace=self.ws[2], **s)
        n.backward(self.dh, self.sum, self.gain, self.rstd, self.dx, self.dgain, dsum=self.dsum, workspace=self.ws[3], **s)
        return [t.clone() for t in self.outputs()]

    def check(self):
        """Each call against its definition on what the calls before it left."""
        for out, a, b, bias in ((self.y, self.h8, self.w8, self.bias), (self.dh, self.d8, self.wt8, None),
                                (self.dW, self.dt8, self.ht8, None)):
            A, B = _value(*a), _value(*b)
            want = _expected(A, B, bias, bias is not None, None)
            tol = _tolerance(out.dtype, A.shape[1], A, B, _scale(*a), _scale(*b), bias)
            _close(out, want, tol + HALF[out.dtype] * (want.abs() + tol) + 1e-300, "product")
        assert torch.equal(_value(*self.w8), _value(*self.wt8).t())
        # and all of it against the layer without 8 bits: a term of a sum is off by 2^-4 + 2^-4 at most
        h = self.sum.double()
        z, r, norm = _normed(h, self.gain.double(), 1e-6)
        full = norm @ self.W.double().t() + self.bias.double()
        slack = (2 * 2.0 ** -4 + 2.0 ** -8 + 0.01) * (norm.abs() @ self.W.double().abs().t())
        _close(self.y, torch.relu(full), slack + HALF[BF] * full.abs() * 1.1, "layer")


@pytest.mark.parametrize("shape", [(1, 64, 48), (65, 200, 130), (300, 512, 260), (1024, 512, 512)])
def test_layer_as_it_is_used(shape):
    layer = Layer(*shape, seed=1)
    layer.run()
    layer.check()


@pytest.mark.parametrize("shape", [(7, 200, 130), (300, 512, 260)])
def test_layer_repeats_on_another_stream_and_in_a_graph(shape):
    a, b = Layer(*shape, seed=1), Layer(*shape, seed=2)
    want = a.run(), b.run()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = a.run(stream=stream)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want[0]))
    graphs = []
    for layer in (a, b):                                     # two graphs that share no workspace
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            layer.run()
        graphs.append(graph)
    for replay in range(3):
        for layer, seed in ((a, replay), (b, replay + 10)):
            for t in layer.outputs():
                t.zero_()
            for w in layer.ws:
                w.fill_(255)
            fresh = _randn(layer.x.shape, _gen(seed + 50))
            layer.x.copy_(fresh)
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for layer in (a, b):
            got = [t.clone() for t in layer.outputs()]
            assert all(torch.equal(x, y) for x, y in zip(got, layer.run()))


def test_norm_of_no_rows_takes_no_tensors():
    """A backward of no rows reads nothing, the weight neither: its pointers may be null."""
    import ctypes
    native = _native()
    d = native.RmsNormDesc(native.ABI_VERSION, native.FP32, native.FP32, native.FP32, 1e-6, 0, 0, 100)
    dw, ws = torch.ones(100, device="cuda"), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    rc = native.lib().spectrain_rms_norm_backward(ctypes.byref(d), None, None, None, None, None, None, dw.data_ptr(),
                                                  ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert rc == native.OK and bool((dw == 0).all())
