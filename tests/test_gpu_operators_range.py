"""GPU: the stand-alone operators at the far ends of what they accept, against
plain implementations in 64 bits. The bounds are those of test_gpu_operators.py,
but for capped scores, whose bound does not grow with the cap: tanh as
1 - 2 / (1 + e^(2u)) is off by 2^-22.6 and a score by that times the cap, up to
2^-16 at caps of 64; past them a score is off relative to itself, below 2^-21 of it
(z by the roundings of its sum, tanh(u) / u by 2^-23 up to |u| = 1/2, and beyond
2^-22.6 is 2^-21.5 of a value of 0.46 or more).
"""
import pytest

from test_gpu_operators import Reference, _attention, _case, _close, _gen, _randn, _run, _see, _turned

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


class Capped(Reference):
    """The definition with bounds that no cap above 64 makes larger."""

    def __init__(self, q, k, v, scale, cap, slopes, see, offset, dout):
        super().__init__(q, k, v, scale, cap, slopes, see, offset, dout)
        (B, Sq, H, D), Sk, Hk, BF = q.shape, k.shape[1], k.shape[2], 2.0 ** -8
        T, back = (lambda t: t.transpose(2, 3)), (lambda t: t.transpose(1, 2))
        Q, dO = back(q.double()), back(dout.double())
        K, V = (back(t.double()).repeat_interleave(H // Hk, 1) for t in (k, v))
        z = scale * Q @ T(K)
        s = cap * torch.tanh(z / cap)
        if slopes is not None:
            far = (torch.arange(Sq, device="cuda")[:, None] + offset - torch.arange(Sk, device="cuda")[None]).abs()
            s = s - slopes.double()[None, :, None, None] * far
        hidden, empty = ~see[:, None], self.empty[..., None]
        lse = self.lse[..., None].masked_fill(empty, 0.0)
        P = torch.exp(s.masked_fill(hidden, -float("inf")) - lse).masked_fill(empty, 0.0)
        sums = (D + 8) * 2.0 ** -24                       # of `dim` products in float32, relative to their magnitudes
        Ez = sums * (abs(scale) * Q.abs() @ T(K.abs())).masked_fill(hidden, 0.0).amax((1, 2, 3), keepdim=True)
        E = Ez + 2.0 ** -21 * (1 + s.masked_fill(hidden, 0.0).abs().amax()) + 2.0 ** -22 * min(cap, 64.0)
        out = back(self.out)
        out_tol = (BF + 2 * E) * (P @ V.abs()) * (1 + 2 * BF) + BF * out.abs()
        self.out_tol, self.lse_tol = back(out_tol), (E + 2.0 ** -22 * lse.abs())[..., 0]
        dP, delta = dO @ T(V), (out * dO).sum(3, keepdim=True)
        delta_tol = (out_tol * dO.abs()).sum(3, keepdim=True) + sums * (out.abs() * dO.abs()).sum(3, keepdim=True)
        # the cap's slope 1 - tanh^2 by at most 0.77 of the error of z / cap, and twice tanh's own
        slope_tol = 0.77 * Ez / cap + 2.0 ** -20
        dS_tol = P * (delta_tol + sums * dO.abs() @ T(V.abs())) + (BF + 2 * E + slope_tol) * P * (dP.abs() + delta.abs())
        dS_tol = dS_tol * abs(scale) * (1 + 2 * BF)
        group = lambda t: back(t.reshape(B, Hk, H // Hk, Sk, D).sum(2))
        self.dq_tol = back(dS_tol @ K.abs()) + BF * self.dq.abs()
        self.dk_tol = group(T(dS_tol) @ Q.abs()) + BF * self.dk.abs()
        self.dv_tol = group(T(P) @ dO.abs()) * (BF + 2 * E) * (1 + 2 * BF) + BF * self.dv.abs()


@pytest.mark.parametrize("cap", [1e-3, 0.7, 4.0, 64.0, 65.0, 1e3, 1e4, 1e6, 1e9, 1e30])
@pytest.mark.parametrize("shape", [
    # B, H, Hk, D, Sq, Sk, offset, causal, masks, slopes
    (2, 8, 2, 64, 1, 300, 299, True, "len", False),        # single tokens
    (1, 4, 4, 128, 200, 200, 0, True, "doc", False),       # eight waves of dK and dV
    (2, 6, 2, 80, 130, 130, 0, True, "prefix", True),
    (1, 2, 2, 32, 70, 150, 80, False, "len", False),
    (1, 2, 1, 64, 1100, 1100, 0, True, "", True),          # walks in pieces
], ids=lambda s: "-".join(str(v) for v in s))
def test_capped_scores_over_the_range_of_caps(shape, cap):
    from paper_1809_02839_amd import native
    B, H, Hk, D, Sq, Sk, offset, causal, kind, biased = shape
    print(f"[capped] {shape} cap {cap}", flush=True)
    c = (B, H, Hk, D, Sq, Sk, offset, causal, kind, cap, biased)
    q, k, v, dout, m = _case(c)
    scale = D ** -0.5
    r = Capped(q, k, v, scale, cap, m.get("slopes"), _see(c, m), offset, dout)
    a = native.Attention(B, H, Hk, D, Sq, Sk, causal=causal, q_offset=offset, cap=cap)
    out, lse, dq, dk, dv = _run(a, q, k, v, dout, m)
    _close(out, r.out, r.out_tol, "out")
    _close(lse.masked_fill(r.empty, 0.0), r.lse.masked_fill(r.empty, 0.0), r.lse_tol, "lse")
    for got, name in ((dq, "dq"), (dk, "dk"), (dv, "dv")):
        _close(got, getattr(r, name), getattr(r, name + "_tol"), name)


def test_capped_scores_at_the_ends_of_cap_and_scale():
    """Scales of 0 and near it, caps of single steps, and scores far past a cap: finite, and as defined."""
    from paper_1809_02839_amd import native
    c = (1, 2, 2, 64, 90, 90, 0, True, "", 0.0, False)
    q, k, v, dout, m = _case(c)
    for scale, cap in ((0.0, 1e-45), (0.0, 5.0), (1e-38, 1e-40), (1e-38, 1e30), (-0.3, 1e30), (1e30, 1.0),
                       (1e30, 1e30), (-2.0, 3.0)):
        print(f"[cap and scale] {scale} {cap}", flush=True)
        a = native.Attention(1, 2, 2, 64, 90, 90, causal=True, scale=scale, cap=cap)
        # the operator takes scale and cap in 32 bits
        scale, cap = (float(torch.tensor(x, dtype=torch.float32)) for x in (scale, cap))
        r = Capped(q, k, v, scale, cap, None, _see(c, m), 0, dout)
        got = _run(a, q, k, v, dout, m)
        assert all(bool(t.isfinite().all()) for t in got)
        if cap < 1e29 or scale < 1.0:      # else scores are far past what a softmax resolves
            _close(got[0], r.out, r.out_tol, "out")
            _close(got[1], r.lse, r.lse_tol, "lse")
            for x, name in zip(got[2:], ("dq", "dk", "dv")):
                _close(x, getattr(r, name), getattr(r, name + "_tol"), name)


@pytest.mark.parametrize("D", [64, 128])
def test_what_nothing_sees_may_hold_anything(D):
    """NaN in the unwritten end of a cache (no lengths given), in a document no query row belongs to, and in rows
    that see no key (before the first key; in a document past the valid keys) changes nothing."""
    nan = float("nan")

    def same(c, m, spoil):
        q, k, v, dout, _ = _case(c)
        clean = _run(_attention(c), q, k, v, dout, m)
        for t in clean:
            assert not bool(t.isnan().any())
        spoil(q, k, v, dout)
        for name, x, y in zip(("out", "lse", "dq", "dk", "dv"), clean, _run(_attention(c), q, k, v, dout, m)):
            assert torch.equal(x, y), name

    for Sq in (1, 9, 100, 150):            # a cache of 333 keys of which 70 + Sq are written
        print(f"[unseen] {D} {Sq}", flush=True)

        def end_of_cache(q, k, v, dout):
            k[:, 70 + Sq:], v[:, 70 + Sq:] = nan, nan

        same((2, 4, 2, D, Sq, 333, 70, True, "", 0.0, False), {}, end_of_cache)

    docs = torch.cat([torch.zeros(77), torch.ones(83)]).int().cuda().expand(2, -1).contiguous()

    def other_document(q, k, v, dout):
        k[:, :77], v[:, :77] = nan, nan

    for Sq in (1, 60):
        same((2, 4, 2, D, Sq, 160, 160 - Sq, True, "", 0.0, False), {"documents": docs}, other_document)

    def early_rows(q, k, v, dout):
        q[:, :30], dout[:, :30] = nan, nan

    same((2, 4, 2, D, 130, 100, -30, True, "", 0.0, False), {}, early_rows)
    lengths = torch.tensor([77, 40], dtype=torch.int32, device="cuda")

    def late_rows(q, k, v, dout):          # the second document lies past the valid keys
        q[:, 77:], dout[:, 77:] = nan, nan
        k[0, 77:], v[0, 77:], k[1, 40:], v[1, 40:] = nan, nan, nan, nan

    same((2, 4, 2, D, 160, 160, 0, False, "", 0.0, False), {"documents": docs, "kv_lengths": lengths}, late_rows)


def test_no_query_rows_leave_zero_gradients_of_keys():
    for D in (64, 128):
        c = (2, 4, 2, D, 0, 300, 0, True, "len", 0.0, False)
        q, k, v, dout, m = _case(c)
        out, lse, dq, dk, dv = _run(_attention(c), q, k, v, dout, m)
        assert dk.shape == k.shape and not bool(dk.any()) and not bool(dv.any())


def test_rotary_first_positions_up_to_the_last():
    """first_position + token past 2^31 - 1 and below 0. A float64 angle of 2^31 radians is off by 2^-22 (the
    position's, and the power's 2 x 2^-53 where it is largest), here and in the reference."""
    from paper_1809_02839_amd import native
    x = _randn((2, 40, 3, 64), _gen(21), torch.float32)
    for first in ((1 << 31) - 5, -(1 << 31), 0):
        pos = torch.arange(first, first + 40, device="cuda", dtype=torch.int64).expand(2, 40)
        want, size = _turned(x, pos, 64, "half", 1e4, "none", 1.0, 0, False)
        out = native.Rotary(64).apply(x, torch.empty_like(x), first_position=first)
        assert bool(((out.double() - want).abs() <= (8e-7 + 4 * 2.0 ** -22) * size).all())


@pytest.mark.parametrize("D", [40, 64, 128])
@pytest.mark.parametrize("S,doc,cap,biased", [(2, 0, 0.0, False), (3, 0, 4.0, True), (16, 0, 0.0, False),
                                              (100, 0, 0.0, True), (128, 0, 4.0, False), (1000, 16, 0.0, False),
                                              (1000, 37, 4.0, True)])
def test_gradients_of_few_keys_do_not_carry_the_rounding_of_out(S, doc, cap, biased, D):
    """delta = sum of P dP in float32, not of the rounded out: dS = P (dP - delta) is off by float32 errors of its
    terms and its own rounding, 2^-8 |dS|, and by nothing that is relative to out."""
    BF, B, H, Hk = 2.0 ** -8, 3, 4, 2
    c = (B, H, Hk, D, S, S, 0, True, "", cap, biased)
    q, k, v, dout, m = _case(c)
    see = torch.ones(S, S, dtype=torch.bool, device="cuda").tril()
    if doc:
        ids = (torch.arange(S, device="cuda") // doc).int()
        m["documents"], see = ids.expand(B, S).contiguous(), see & (ids[:, None] == ids[None])
    _, _, dq, dk, _ = _run(_attention(c), q, k, v, dout, m)
    T, back = (lambda t: t.transpose(2, 3)), (lambda t: t.transpose(1, 2))
    Q, dO = back(q.double()), back(dout.double())
    K, V = (back(t.double()).repeat_interleave(H // Hk, 1) for t in (k, v))
    scale = D ** -0.5
    z = scale * Q @ T(K)
    t = torch.tanh(z / cap) if cap else torch.zeros_like(z)
    s = cap * t if cap else z
    if biased:
        i = torch.arange(S, device="cuda")
        s = s - m["slopes"].double()[None, :, None, None] * (i[:, None] - i[None]).abs()
    s = s.masked_fill(~see, -float("inf"))
    P, one = torch.softmax(s, 3), 1 - t * t
    sums = (D + 8) * 2.0 ** -24
    Ez = sums * (scale * Q.abs() @ T(K.abs())).masked_fill(~see, 0.0).amax()
    E = Ez + 2.0 ** -21 * (1 + s.masked_fill(~see, 0.0).abs().amax()) + 2.0 ** -22 * cap
    dP = dO @ T(V)
    delta, size = (P * dP).sum(3, keepdim=True), dO.abs() @ T(V.abs())
    dP_tol = sums * size
    delta_tol = (P * (dP_tol + (2 * E + 200 * 2.0 ** -24) * dP.abs())).sum(3, keepdim=True)   # up to 192 keys
    slope_tol = 0.77 * Ez / cap + 2.0 ** -20 if cap else 0.0
    dS = P * (dP - delta) * one
    tol = P * (delta_tol + dP_tol) + (2 * E + slope_tol) * P * (dP - delta).abs()
    tol = (tol + BF * dS.abs()) * (1 + 2 * BF) * scale
    group = lambda x: back(x.reshape(B, Hk, H // Hk, S, D).sum(2))
    want = {"dq": back(scale * dS @ K), "dk": group(scale * T(dS) @ Q)}
    tols = {"dq": back(tol @ K.abs()), "dk": group(T(tol) @ Q.abs())}
    for got, name in ((dq, "dq"), (dk, "dk")):
        _close(got, want[name], tols[name] + BF * want[name].abs(), name)


@pytest.mark.parametrize("D", [64, 128])
def test_gradients_with_offsets_past_32_bits(D):
    """Every tensor of a forward and a backward with its last tokens beyond 2^32 elements."""
    step, S, H, Hk = 1 << 20, 4200, 2, 1
    c = (1, H, Hk, D, S, S, 0, True, "len", 0.0, False)
    q, k, v, dout, m = _case(c)
    store = torch.empty(step * S, dtype=torch.bfloat16, device="cuda")
    place = iter(range(0, step, 1024))

    def strided(t):
        return store.as_strided(t.shape, (8, step, D, 1), next(place))

    far = [strided(t) for t in (q, k, v, q, dout, q, k, v)]
    for x, t in zip(far, (q, k, v, None, dout)):
        if t is not None:
            x.copy_(t)
    qf, kf, vf, of, dof, *grads = far
    a = _attention(c)
    ws, lse = a.workspace(backward=True), torch.empty(1, H, S, device="cuda")
    a.forward(qf, kf, vf, of, lse, workspace=ws, **m)
    a.backward(qf, kf, vf, of, lse, dof, *grads, workspace=ws, **m)
    # the bits of the same call on contiguous tensors, which are tested against the definition
    for x, t in zip((of, lse, *grads), _run(a, q, k, v, dout, m)):
        assert torch.equal(x, t)
    r = Reference(q[:, -200:], k, v, D ** -0.5, 0.0, None, _see((1, H, Hk, D, 200, S, S - 200, True, "len", 0.0, False), m),
                  S - 200)
    _close(of[:, -200:], r.out, r.out_tol, "out")
