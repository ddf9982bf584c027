"""Host-side checks of the stand-alone operators (no GPU needed): every call
the interface refuses is refused before any device work, with a message that
names the argument, and the workspace sizes follow from the shape alone."""
import ctypes

import pytest

from paper_1809_02839_amd import native

P = 4096          # an aligned address that a refused call never touches


def _err():
    return native.lib().spectrain_last_error().decode()


def _rotary(**change):
    d = native.Rotary(64)._d
    d.dtype, d.batch, d.tokens, d.heads = native.BF16, 2, 3, 4
    d.x = d.out = native.Strides(3 * 4 * 64, 4 * 64, 64)
    for k, v in change.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("change,needle", [
    (dict(abi_version=2), "abi_version"),
    (dict(dtype=7), "dtype"),
    (dict(batch=-1), "must be >= 0"),
    (dict(tokens=1 << 24), "2^24"),
    (dict(heads=1 << 16), "2^16"),
    (dict(head_dim=0), "head_dim"),
    (dict(head_dim=258), "head_dim"),
    (dict(rotary_dim=63), "rotary_dim"),
    (dict(rotary_dim=66), "rotary_dim"),
    (dict(rotary_dim=0), "rotary_dim"),
    (dict(layout=2), "layout"),
    (dict(scaling=4), "scaling"),
    (dict(reserved=1), "reserved"),
    (dict(base=1.0), "base"),
    (dict(base=float("nan")), "base"),
    (dict(scaling=1, factor=0.5), "factor"),
    (dict(scaling=2, factor=float("inf")), "factor"),
    (dict(scaling=3, factor=2.0), "original_length"),
    (dict(out=native.Strides(3 * 4 * 64, 4 * 64, 32)), "overlap"),
    (dict(out=native.Strides(0, 4 * 64, 64)), "overlap"),
    (dict(x=native.Strides(-1, 4 * 64, 64)), "strides"),
])
def test_rotary_refusals(change, needle):
    rc = native.lib().spectrain_rotary(ctypes.byref(_rotary(**change)), P, None, 0, 2 * P, None)
    assert rc == native.EINVAL and needle in _err(), _err()


def test_rotary_refuses_null_and_unlike_strides_in_place():
    lib = native.lib()
    assert lib.spectrain_rotary(None, P, None, 0, P, None) == native.EINVAL
    assert lib.spectrain_rotary(ctypes.byref(_rotary()), None, None, 0, P, None) == native.EINVAL
    assert lib.spectrain_rotary(ctypes.byref(_rotary()), P + 1, None, 0, 2 * P, None) == native.EINVAL
    d = _rotary(x=native.Strides(3 * 8 * 64, 8 * 64, 64))
    assert lib.spectrain_rotary(ctypes.byref(d), P, None, 0, P, None) == native.EINVAL and "in place" in _err()
    assert lib.spectrain_rotary(ctypes.byref(_rotary(batch=0)), None, None, 0, None, None) == native.OK


def _attention(**change):
    d = native.Attention(2, 4, 2, 64, 16, 16, causal=True)._d
    big = native.Strides(16 * 4 * 64, 4 * 64, 64)
    for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv"):
        setattr(d, n, big)
    for k, v in change.items():
        setattr(d, k, v)
    return d


def _call(d, masks=None, ws=P, ws_bytes=1 << 20, out=3 * P, q=P, dq=4 * P, dk=5 * P, backward=False, lse=P):
    lib = native.lib()
    m = ctypes.byref(masks) if masks is not None else None
    if not backward:
        return lib.spectrain_attention_forward(ctypes.byref(d), m, q, 2 * P, 2 * P, out, lse, ws, ws_bytes, None)
    return lib.spectrain_attention_backward(ctypes.byref(d), m, q, 2 * P, 2 * P, out, lse, 7 * P, dq, dk, 6 * P, ws,
                                            ws_bytes, None)


@pytest.mark.parametrize("change,needle", [
    (dict(abi_version=0), "abi_version"),
    (dict(dtype=native.FP32), "bf16 only"),
    (dict(batch=-1), "must be >= 0"),
    (dict(q_len=-1), "must be >= 0"),
    (dict(heads=3), "multiple of kv_heads"),
    (dict(heads=0), "multiple of kv_heads"),
    (dict(head_dim=136), "head_dim"),
    (dict(head_dim=60), "head_dim"),
    (dict(causal=2), "causal"),
    (dict(scale=float("nan")), "scale"),
    (dict(cap=-1.0), "cap"),
    (dict(cap=float("inf")), "cap"),
    (dict(scale=3e38), "2^100"),
    (dict(cap=1e-37), "2^100"),
    (dict(cap=2e30), "2^100"),
    (dict(k=native.Strides(1 << 34, 1 << 26, 64)), "2^29"),
    (dict(q=native.Strides(0, 64, 1 << 29)), "2^29"),
    (dict(q_offset=(1 << 30) + 1), "2^30"),
    (dict(kv_len=(1 << 30) + 1), "2^30"),
    (dict(batch=1 << 20, q_len=1 << 10), "2^23"),
    (dict(q=native.Strides(4096, 256, 60)), "multiples of 8"),
    (dict(k=native.Strides(4096, -8, 64)), "strides"),
    (dict(out=native.Strides(4096, 256, 32)), "overlap"),
])
@pytest.mark.parametrize("backward", [False, True])
def test_attention_refusals(change, needle, backward):
    assert _call(_attention(**change), backward=backward) == native.EINVAL
    assert needle in _err(), _err()


def test_attention_refuses_masks_and_buffers():
    lib = native.lib()
    masks = native.AttentionMasks
    assert _call(_attention(causal=0), masks(None, P, None, None)) == native.EINVAL and "prefix" in _err()
    assert _call(_attention(q_offset=1), masks(P, None, None, None)) == native.EINVAL and "documents" in _err()
    assert _call(_attention(q_offset=-1), masks(P, None, None, None)) == native.EINVAL and "documents" in _err()
    assert _call(_attention(), masks(P + 2, None, None, None)) == native.EINVAL and "aligned" in _err()
    need = ctypes.c_size_t()
    assert lib.spectrain_attention_workspace(ctypes.byref(_attention()), 1, ctypes.byref(need)) == native.OK
    assert need.value > 0
    assert _call(_attention(), ws_bytes=need.value - 1, backward=True) == native.EINVAL and "workspace" in _err()
    assert _call(_attention(), ws=None, backward=True) == native.EINVAL and "workspace" in _err()
    assert _call(_attention(), ws=P + 16) == native.EINVAL and "256-byte" in _err()
    assert _call(_attention(), q=P + 8) == native.EINVAL and "16-byte" in _err()
    assert _call(_attention(), q=None) == native.EINVAL and "NULL" in _err()
    assert _call(_attention(), out=P) == native.EINVAL and "input" in _err()
    assert _call(_attention(), dq=P, backward=True) == native.EINVAL and "input" in _err()
    assert _call(_attention(), dk=4 * P, backward=True) == native.EINVAL and "overlap" in _err()
    assert _call(_attention(), lse=None, backward=True) == native.EINVAL and "lse" in _err()
    assert _call(_attention(dk=native.Strides(4096, 0, 64)), backward=True) == native.EINVAL and "overlap" in _err()
    assert lib.spectrain_attention_forward(None, None, P, P, P, P, P, P, 1 << 20, None) == native.EINVAL
    assert lib.spectrain_attention_workspace(ctypes.byref(_attention()), 0, None) == native.EINVAL
    # nothing to do is no error, and touches nothing
    assert _call(_attention(batch=0), q=None, out=None, backward=False) == native.OK
    assert _call(_attention(q_len=0), q=None, out=None, backward=False) == native.OK


@pytest.mark.parametrize("args,needle", [
    ((5, 4, 64, P, 64, P, P), "dtype"),
    ((1, -1, 64, P, 64, P, P), ">= 0"),
    ((1, 4, 64, P, 63, P, P), "ld"),
    ((1, 4, 64, None, 64, P, P), "NULL"),
    ((1, 4, 64, P, 64, None, P), "NULL"),
    ((1, 4, 64, P, 64, P, None), "NULL"),
    ((1, 4, 64, P + 1, 64, P, P), "aligned"),
    ((1, 1 << 30, 64, P, 64, P, P), "2^30"),
    ((1, 4, 1 << 30, P, 1 << 30, P, P), "2^30"),
])
def test_checkpoint_refusals(args, needle):
    dt, rows, cols, x, ld, codes, scales = args
    lib = native.lib()
    assert lib.spectrain_checkpoint_pack(dt, rows, cols, x, ld, codes, scales, None) == native.EINVAL
    assert needle in _err(), _err()
    assert lib.spectrain_checkpoint_restore(dt, rows, cols, codes, scales, x, ld, None) == native.EINVAL
    assert needle in _err(), _err()
    assert lib.spectrain_checkpoint_pack(1, 0, 64, None, 64, None, None, None) == native.OK


def test_binding_refuses_host_tensors_and_unlike_shapes():
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        native.Rotary(64).apply(x)
    with pytest.raises(ValueError, match="batch, token, head"):
        native.Rotary(32).apply(x)
    with pytest.raises(ValueError, match="positions"):
        native.Rotary(64).apply(x, positions=torch.zeros(2, 4, dtype=torch.int32))
    a = native.Attention(2, 4, 2, 64, 3, 3)
    k = x[:, :, :2]
    ws = torch.empty(256, dtype=torch.uint8)
    with pytest.raises(ValueError, match="shape"):
        a.forward(x, x, k, torch.empty_like(x), workspace=ws)
    with pytest.raises(ValueError, match="kv_lengths"):
        a.forward(x, k, k, torch.empty_like(x), workspace=ws, kv_lengths=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="GPU"):
        a.forward(x, k, k, torch.empty_like(x), workspace=ws)
    with pytest.raises(ValueError, match="codes"):
        native.checkpoint_pack(x[0, 0], torch.zeros(4, 63, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8))
