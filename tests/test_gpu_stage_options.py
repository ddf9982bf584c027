"""GPU: the options of transformer stages (attention, masks, stash) in orders of
calls and sizes that the other tests do not make."""
import pytest

import synth

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def _stage(layers=2, S=40, k=1, n=4, d=128, batch=3, ffn=256):
    from paper_1809_02839_amd import native
    spec = synth.StageSpec("transformer", "bf16", "none", k, n, batch, layers, (d, 4, ffn, S), 5e-5, 0.9)
    return spec, native.Stage(native.desc_from_spec(spec), synth.initial_params(spec))


def _refused(code, f, *args, **kw):
    from paper_1809_02839_amd import native
    with pytest.raises(native.SpecTrainError) as e:
        f(*args, **kw)
    assert e.value.code == code, e.value


def test_waiting_masks_outlive_a_new_attention_only_where_it_takes_them():
    """A prefix that waits for its forward refuses an attention without causal when it is set, not in the forward."""
    from paper_1809_02839_amd import native
    spec, st = _stage()
    _, other = _stage()
    x = torch.from_numpy(synth.stage_input(spec, 0)).cuda().bfloat16()
    prefix = torch.tensor([3, 0, 39], dtype=torch.int32, device="cuda")
    st.set_attention(causal=True)
    st.set_masks(0, prefix=prefix)
    _refused(native.ESTATE, st.set_attention, causal=False)
    st.set_attention(causal=True, rotary_dim=32)         # takes them
    other.set_attention(causal=True, rotary_dim=32)
    other.set_masks(0, prefix=prefix)
    y = [torch.empty_like(x) for _ in range(2)]
    st.forward(0, x, y[0])
    other.forward(0, x, y[1])
    torch.cuda.synchronize()
    assert torch.equal(*y)
    st.backward(0, x, None)
    st.update(0, 0)
    st.set_masks(1, prefix=prefix)
    _refused(native.ESTATE, st.set_attention, causal=False)
    st.set_masks(1)                                      # replaced by none
    st.set_attention(causal=False)
    st.forward(1, x, y[0])
    torch.cuda.synchronize()
    for s in (st, other):
        s.destroy()


@pytest.mark.parametrize("layers", [1, 3])
def test_an_8_bit_stash_adds_one_layer_of_activations_to_the_workspace(layers):
    """Device memory of a stage with one slot: what the slot saves, against one layer's restored activations."""
    spec, st = _stage(layers=layers, S=1024, k=0, n=1, d=512, batch=32, ffn=2048)
    T, d, F = 32 * 1024, 512, 2048

    def held():
        torch.cuda.synchronize()
        free, total = torch.cuda.mem_get_info()
        return total - free

    plain = held()
    st.set_stash("e4m3")
    packed = held() - plain
    st.set_stash("bf16")
    assert abs(held() - plain) <= 8 << 20                # as before, up to the allocator's granules
    kept = T * (3 * d + F) * layers + T * d * (layers - 1)   # r1, h, r2, f1, and the outputs between layers
    saved = kept * 2 - kept * 33 // 32
    assert packed <= T * (F + 4 * d) * 2 - saved + (8 << 20)
    st.destroy()
