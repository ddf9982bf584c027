"""Host-side checks of blocks, norm and product (no GPU needed): what the
interface refuses is refused before any device work, with a message that names
the argument, and calls of nothing are no errors."""
import ctypes

import pytest

from paper_1809_02839_amd import native

P = 4096          # an aligned address that a refused call never touches


def _err():
    return native.lib().spectrain_last_error().decode()


def _refused(rc, needle):
    assert rc == native.EINVAL and needle in _err(), (rc, _err())


def _set(d, change):
    for k, v in change.items():
        setattr(d, k, v)
    return d


# ------------------------------------------------------------------ blocks ----

def _blocks(**change):
    return _set(native.BlocksDesc(native.ABI_VERSION, native.BF16, 0, 0, 200, 300, 300, 304, 208, 208, 304), change)


def _pack(d, x=P, codes=2 * P, scales=3 * P, t=4 * P, ts=5 * P):
    return native.lib().spectrain_blocks_pack(ctypes.byref(d), x, codes, scales, t, ts, None)


def _restore(d, codes=2 * P, scales=3 * P, out=P):
    return native.lib().spectrain_blocks_restore(ctypes.byref(d), codes, scales, out, None)


@pytest.mark.parametrize("change,needle", [
    (dict(abi_version=2), "abi_version"),
    (dict(dtype=7), "dtype"),
    (dict(reserved=1), "reserved"),
    (dict(rows=-1), ">= 0"),
    (dict(rows=1 << 31), "2^31"),
    (dict(rows=1 << 30, cols=1 << 14, ld=1 << 14, codes_ld=1 << 14), "2^23"),
    (dict(ld=299), "ld"),
    (dict(ld=(1 << 40) + 8), "ld"),
    (dict(codes_ld=288), "codes_ld"),
    (dict(codes_ld=305), "codes_ld"),
    (dict(codes_ld=(1 << 22) + 16), "codes_ld"),
    (dict(scales_ld=192), "codes scales_ld"),
    (dict(scales_ld=201), "codes scales_ld"),
])
def test_blocks_refusals(change, needle):
    _refused(_pack(_blocks(**change)), needle)
    _refused(_restore(_blocks(**change)), needle)


def test_blocks_refuses_buffers():
    _refused(_pack(_blocks(shape=2)), "shape")
    _refused(_pack(_blocks(transposed_ld=192)), "transposed_ld")
    _refused(_pack(_blocks(transposed_scales_ld=288)), "transposed scales_ld")
    _refused(_pack(_blocks(), x=None), "NULL")
    _refused(_pack(_blocks(), x=P + 1), "aligned")
    _refused(_pack(_blocks(), codes=2 * P + 8), "16-byte")
    _refused(_pack(_blocks(), ts=5 * P + 8), "16-byte")
    _refused(_pack(_blocks(), scales=None), "scales")
    _refused(_pack(_blocks(), t=None), "scales")
    _refused(_pack(_blocks(), codes=None, scales=None, t=None, ts=None), "NULL")
    _refused(_pack(_blocks(), t=2 * P), "overlap")
    _refused(_pack(_blocks(), ts=3 * P), "overlap")
    _refused(_pack(_blocks(), scales=2 * P), "overlap")
    _refused(_pack(_blocks(), codes=P), "x")
    _refused(_restore(_blocks(), codes=None, scales=None), "NULL")
    _refused(_restore(_blocks(), out=None), "NULL")
    _refused(_restore(_blocks(), out=2 * P), "input")
    lib = native.lib()
    _refused(lib.spectrain_blocks_pack(None, P, P, P, P, P, None), "desc")
    _refused(lib.spectrain_blocks_restore(None, P, P, P, None), "desc")
    for change in (dict(rows=0), dict(cols=0)):           # nothing to do is no error, and touches nothing
        assert _pack(_blocks(**change), x=None, codes=None, scales=None, t=None, ts=None) == native.OK
        assert _restore(_blocks(**change), codes=None, scales=None, out=None) == native.OK


# -------------------------------------------------------------------- norm ----

def _norm(**change):
    d = native.RmsNormDesc(native.ABI_VERSION, native.FP32, native.FP32, native.FP32, 1e-6, 0, 20, 300)
    for n in ("x_ld", "residual_ld", "sum_ld", "y_ld", "dy_ld", "dsum_ld", "dx_ld"):
        setattr(d, n, 300)
    d.codes_ld, d.scales_ld = 304, 32
    return _set(d, change)


def _forward(d, x=P, res=2 * P, w=3 * P, total=4 * P, y=5 * P, codes=6 * P, scales=7 * P, rstd=8 * P):
    return native.lib().spectrain_rms_norm_forward(ctypes.byref(d), x, res, w, total, y, codes, scales, rstd, None)


def _backward(d, dy=P, h=2 * P, w=3 * P, rstd=4 * P, dsum=5 * P, dx=6 * P, dw=7 * P, ws=8 * P, n=1 << 30):
    return native.lib().spectrain_rms_norm_backward(ctypes.byref(d), dy, h, w, rstd, dsum, dx, dw, ws, n, None)


@pytest.mark.parametrize("change,needle", [
    (dict(abi_version=0), "abi_version"),
    (dict(dtype=2), "dtype"),
    (dict(out_dtype=-1), "out_dtype"),
    (dict(weight_dtype=5), "weight_dtype"),
    (dict(dtype=native.BF16), "out_dtype"),
    (dict(eps=0.0), "eps"),
    (dict(eps=float("nan")), "eps"),
    (dict(eps=float("inf")), "eps"),
    (dict(reserved=3), "reserved"),
    (dict(rows=-1), "rows"),
    (dict(rows=1 << 31), "rows"),
    (dict(cols=0), "cols"),
    (dict(cols=32769), "cols"),
    (dict(sum_ld=299), "sum_ld"),
])
def test_norm_refusals(change, needle):
    _refused(_forward(_norm(**change)), needle)
    _refused(_backward(_norm(**change)), needle)
    if "ld" not in needle:
        n = ctypes.c_size_t()
        _refused(native.lib().spectrain_rms_norm_workspace(ctypes.byref(_norm(**change)), ctypes.byref(n)), needle)


def test_norm_refuses_buffers():
    for name, entry in (("x", _forward), ("residual", _forward), ("y", _forward), ("dy", _backward),
                        ("dsum", _backward), ("dx", _backward)):
        _refused(entry(_norm(**{name + "_ld": 12})), name + "_ld")
    _refused(_forward(_norm(codes_ld=296)), "codes_ld")
    _refused(_forward(_norm(scales_ld=16)), "scales_ld")
    _refused(_forward(_norm(), codes=6 * P + 8), "16-byte")
    _refused(_forward(_norm(), scales=None), "scales")
    _refused(_forward(_norm(), x=P + 2), "aligned")
    _refused(_forward(_norm(), w=P + 2), "aligned")
    _refused(_forward(_norm(), rstd=8 * P + 2), "aligned")
    _refused(_forward(_norm(), res=None), "residual")
    for k in ("x", "w"):
        _refused(_forward(_norm(), **{k: None}), "NULL")
    _refused(_forward(_norm(), y=None, codes=None, scales=None), "NULL")
    _refused(_forward(_norm(x_ld=304), total=P), "same ld")
    _refused(_forward(_norm(residual_ld=304), total=2 * P), "same ld")
    for k in ("y", "codes", "scales", "rstd"):
        for at in (P, 2 * P, 3 * P, 4 * P):
            _refused(_forward(_norm(), **{k: at}), "input")
    _refused(_forward(_norm(), total=3 * P), "input")
    _refused(_forward(_norm(), codes=5 * P), "overlap")
    need = ctypes.c_size_t()
    assert native.lib().spectrain_rms_norm_workspace(ctypes.byref(_norm()), ctypes.byref(need)) == native.OK
    assert need.value > 0
    _refused(_backward(_norm(), n=need.value - 1), "workspace")
    _refused(_backward(_norm(), ws=None), "workspace")
    _refused(_backward(_norm(), ws=8 * P + 16), "256-byte")
    for k in ("dy", "h", "w", "rstd", "dx", "dw"):
        _refused(_backward(_norm(), **{k: None}), "NULL")
    for at in (2 * P, 3 * P, 4 * P, 7 * P):
        _refused(_backward(_norm(), dx=at), "dx")
    for at in (P, 2 * P, 3 * P, 4 * P, 5 * P):
        _refused(_backward(_norm(), dw=at), "dweight")
    _refused(_backward(_norm(dsum_ld=304), dx=5 * P), "same ld")
    _refused(_backward(_norm(dy_ld=304), dx=P), "same ld")
    _refused(_backward(_norm(out_dtype=native.BF16), dx=P), "type")
    lib = native.lib()
    _refused(lib.spectrain_rms_norm_forward(None, P, P, P, P, P, P, P, P, None), "desc")
    _refused(lib.spectrain_rms_norm_backward(None, P, P, P, P, P, P, P, P, 8, None), "desc")
    _refused(lib.spectrain_rms_norm_workspace(ctypes.byref(_norm()), None), "bytes")
    assert _forward(_norm(rows=0), x=None, res=None, w=None, total=None, y=None, codes=None, scales=None,
                    rstd=None) == native.OK


# ----------------------------------------------------------------- product ----

def _product(**change):
    d = native.ProductDesc(native.ABI_VERSION, native.FP32, native.FP32, 0, 0, 0, 200, 300, 500, 512, 208, 512, 304,
                           300, 300)
    return _set(d, change)


def _apply(d, a=P, sa=2 * P, b=3 * P, sb=4 * P, bias=5 * P, mask=6 * P, out=7 * P, ws=8 * P, n=1 << 40):
    return native.lib().spectrain_product(ctypes.byref(d), a, sa, b, sb, bias, mask, out, ws, n, None)


@pytest.mark.parametrize("change,needle", [
    (dict(abi_version=4), "abi_version"),
    (dict(out_dtype=2), "out_dtype"),
    (dict(bias_dtype=2), "bias_dtype"),
    (dict(relu=2), "relu"),
    (dict(accumulate=-1), "accumulate"),
    (dict(accumulate=1, out_dtype=native.BF16), "accumulate"),
    (dict(reserved=1), "reserved"),
    (dict(m=-1), ">= 0"),
    (dict(k=-1), ">= 0"),
    (dict(n=1 << 31), "2^31"),
    (dict(k=(1 << 22) + 1), "2^22"),
    (dict(m=1 << 20, n=1 << 17), "at most 2^22"),
    (dict(a_ld=496), "a_ld"),
    (dict(b_ld=504), "b_ld"),
    (dict(a_ld=(1 << 22) + 16), "a_ld"),
    (dict(a_scales_ld=192), "a scales_ld"),
    (dict(b_scales_ld=300), "b scales_ld"),
    (dict(a_scales_ld=1 << 29), "2^31"),
    (dict(b_scales_ld=1 << 29), "2^31"),
    (dict(out_ld=299), "out_ld"),
    (dict(mask_ld=299), "mask_ld"),
])
def test_product_refusals(change, needle):
    _refused(_apply(_product(**change)), needle)
    if "ld" not in needle and not any(k.endswith("_ld") for k in change):
        n = ctypes.c_size_t()
        _refused(native.lib().spectrain_product_workspace(ctypes.byref(_product(**change)), ctypes.byref(n)), needle)


def test_product_refuses_buffers():
    for k in ("a", "sa", "b", "sb"):
        _refused(_apply(_product(), **{k: P * 9 + 8}), "16-byte")
        _refused(_apply(_product(), **{k: None}), "scales")
    _refused(_apply(_product(), a=None, sa=None), "NULL")
    _refused(_apply(_product(), out=None), "NULL")
    for k in ("bias", "mask", "out"):
        _refused(_apply(_product(), **{k: P * 9 + 2}), "aligned")
    for at in range(1, 7):
        _refused(_apply(_product(), out=at * P), "input")
    _refused(_apply(_product(), ws=8 * P + 16), "256-byte")
    lib = native.lib()
    need = ctypes.c_size_t()
    d = _product(m=128, n=128, k=1 << 20, a_ld=1 << 20, b_ld=1 << 20)
    assert lib.spectrain_product_workspace(ctypes.byref(d), ctypes.byref(need)) == native.OK
    if need.value:
        _refused(_apply(d, n=need.value - 1), "workspace")
        _refused(_apply(d, ws=None), "workspace")
    _refused(lib.spectrain_product(None, P, P, P, P, P, P, P, P, 0, None), "desc")
    _refused(lib.spectrain_product_workspace(ctypes.byref(_product()), None), "bytes")
    for change in (dict(m=0), dict(n=0)):
        assert _apply(_product(**change), a=None, sa=None, b=None, sb=None, bias=None, mask=None,
                      out=None) == native.OK


# ----------------------------------------------------------------- binding ----

def test_binding_refuses_what_the_library_would_misread():
    torch = pytest.importorskip("torch")
    x, w = torch.zeros(4, 200), torch.ones(200)
    codes, scales = native.blocks_empty(4, 200, device="cpu")
    assert codes.stride(0) == 208 and scales.shape == (2, 4) and scales.stride(0) == 16
    with pytest.raises(ValueError, match="GPU"):
        native.blocks_pack(x, codes, scales)
    with pytest.raises(ValueError, match="codes"):
        native.blocks_pack(x, codes[:, :100], scales)
    with pytest.raises(ValueError, match="scales"):
        native.blocks_pack(x, codes, scales.t().contiguous())
    with pytest.raises(ValueError, match="together"):
        native.blocks_pack(x, codes)
    with pytest.raises(ValueError, match="transposed"):
        native.blocks_pack(x, None, None, codes, scales)
    with pytest.raises(ValueError, match="rows, cols"):
        native.blocks_restore(codes, scales, x[0])
    with pytest.raises(ValueError, match="contiguous"):
        native.blocks_restore(codes, scales, torch.zeros(200, 4).t())
    norm = native.RmsNorm(200)
    with pytest.raises(ValueError, match="rows, 200"):
        norm.forward(x[:, :100], w, x)
    with pytest.raises(ValueError, match="weight"):
        norm.forward(x, w[:100], x)
    with pytest.raises(ValueError, match="residual"):
        norm.forward(x, w, x, residual=x.to(torch.bfloat16))
    with pytest.raises(ValueError, match="rstd"):
        norm.forward(x, w, x, rstd=torch.zeros(5))
    with pytest.raises(ValueError, match="GPU"):
        norm.forward(x, w, x)
    with pytest.raises(ValueError, match="dweight"):
        norm.backward(x, x, w, torch.zeros(4), x, torch.zeros(100), workspace=torch.zeros(256, dtype=torch.uint8))
    p, ws = native.Product(4, 4, 200), torch.zeros(256, dtype=torch.uint8)
    with pytest.raises(ValueError, match="out"):
        p.apply(codes, scales, codes, scales, torch.zeros(4, 5), workspace=ws)
    with pytest.raises(ValueError, match="bias"):
        p.apply(codes, scales, codes, scales, torch.zeros(4, 4), bias=torch.zeros(5), workspace=ws)
    with pytest.raises(ValueError, match="mask"):
        p.apply(codes, scales, codes, scales, torch.zeros(4, 4), mask=torch.zeros(4, 4, dtype=torch.bfloat16), workspace=ws)
    with pytest.raises(ValueError, match="together"):
        p.apply(codes, scales, codes, None, torch.zeros(4, 4), workspace=ws)
    with pytest.raises(ValueError, match="GPU"):
        p.apply(codes, scales, codes, scales, torch.zeros(4, 4), workspace=ws)
