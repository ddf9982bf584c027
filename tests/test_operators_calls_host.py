"""Host-side checks of how the binding calls the operators (no GPU needed)."""
import pytest

from paper_1809_02839_amd import native

torch = pytest.importorskip("torch")


def _heads(*shape):
    return torch.zeros(*shape, dtype=torch.bfloat16)


def _interrupt(monkeypatch, other):
    """The descriptors that two calls hand to the library, the second made (by `other`) while the first is inside."""
    seen, depth = [], []

    def on(device, stream, entry, *args):
        depth.append(args[0])
        if len(depth) == 1:
            other()
        seen.append(type(args[0]._obj).from_buffer_copy(args[0]._obj))

    monkeypatch.setattr(native, "_on", on)
    return seen


def test_rotary_calls_do_not_share_a_descriptor(monkeypatch):
    """Another thread's call on the same object, with its own layout and position, changes nothing of this one's."""
    r = native.Rotary(64)
    seen = _interrupt(monkeypatch, lambda: r.apply(_heads(1, 7, 2, 64), first_position=9))
    for x, first in ((_heads(2, 3, 4, 64), 5), (_heads(1, 7, 2, 64), 0)):   # another layout; another position only
        seen.clear()
        r.apply(x, first_position=first)
        d = seen[-1]
        assert (d.batch, d.tokens, d.heads, d.first_position) == (*x.shape[:3], first)
        assert (d.x.token, d.x.head) == x.stride()[1:3]


def test_attention_calls_do_not_share_a_descriptor(monkeypatch):
    a = native.Attention(2, 4, 2, 64, 3, 3)
    q, k, ws = _heads(2, 3, 4, 64), _heads(2, 3, 2, 64), torch.empty(256, dtype=torch.uint8)
    wide = _heads(2, 3, 5, 64)[:, :, :4]
    lse = torch.zeros(2, 4, 3)
    seen = _interrupt(monkeypatch, lambda: a.forward(wide, k, k, wide, workspace=ws))
    a.forward(q, k, k, q, workspace=ws)
    assert (seen[0].q.token, seen[0].out.token) == (320, 320) and (seen[1].q.token, seen[1].out.token) == (256, 256)
    seen = _interrupt(monkeypatch, lambda: a.backward(wide, k, k, q, lse, q, wide, k, k, workspace=ws))
    a.backward(q, k, k, q, lse, wide, q, k, k, workspace=ws)
    assert (seen[0].q.token, seen[0].dout.token, seen[0].dq.token) == (320, 256, 320)
    assert (seen[1].q.token, seen[1].dout.token, seen[1].dq.token) == (256, 320, 256)


P = 4096          # an aligned address that these calls never touch


def test_a_backward_of_nothing_is_no_error_whatever_the_heads():
    """batch * kv_heads of 2^32 with no row and no key: nothing is divided by it."""
    import ctypes
    d = native.Attention(1 << 16, 1 << 16, 1 << 16, 8, 0, 0)._d
    for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv"):
        setattr(d, n, native.Strides(8, 8, 8))
    assert native.lib().spectrain_attention_backward(ctypes.byref(d), None, *[None] * 9, None, 0, None) == native.OK
    assert native.lib().spectrain_attention_forward(ctypes.byref(d), None, *[None] * 6, 0, None) == native.OK


def test_checkpoint_refuses_what_a_grid_does_not_hold():
    lib = native.lib()
    for rows in ((1 << 30) - 1, (1 << 30) - 63):
        assert lib.spectrain_checkpoint_pack(1, rows, 32, P, 32, P, P, None) == native.EINVAL
        assert "2^30" in lib.spectrain_last_error().decode()


def test_strides_of_single_elements_do_not_matter(monkeypatch):
    """A dimension of size 1 may have any stride (torch keeps odd ones there)."""
    calls = []

    def on(device, stream, entry, *args):
        calls.append(type(args[0]._obj).from_buffer_copy(args[0]._obj))

    monkeypatch.setattr(native, "_on", on)
    q = torch.zeros(2, 4, 64, 1, dtype=torch.bfloat16).permute(0, 3, 1, 2)     # strides 256, 1, 64, 1
    assert q.shape == (2, 1, 4, 64) and q.stride(1) == 1
    k = _heads(2, 3, 2, 64)
    a = native.Attention(2, 4, 2, 64, 1, 3)
    a.forward(q, k, k, torch.empty_like(q), workspace=torch.empty(256, dtype=torch.uint8))
    native.Rotary(64).apply(q)
    assert (calls[0].q.batch, calls[0].q.token, calls[0].q.head) == (256, 0, 64)
    assert (calls[1].x.batch, calls[1].x.token, calls[1].x.head) == (256, 0, 64)
