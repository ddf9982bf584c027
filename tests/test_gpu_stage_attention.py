"""GPU: transformer stages with rotary positions, masked attention and an 8-bit
stash, the operators run together as training uses them. Every forward and
backward of a few mini-batches is held against the oracle's recomputation from
the stage's own state, at the stepwise bound for bf16 stages: the output or loss
of the whole stage, the backward from the stage's own stashed activations (as
the stepwise tests explain), and every stashed activation from the stashed ones
that it was formed from. The last are not compared through the layers: two
correct stages round a few values of q and k one bf16 step (2^-8) apart, which
moves a score by 2^-7 of its size; scores reach the cap of 20 here, so their
probabilities, and a row of ctx with them, may differ by exp(0.16)."""
import dataclasses

import numpy as np
import pytest

import synth
from oracle import attention as At
from oracle import layers as Lr
from oracle import method, stages
from oracle.numerics import to_bf16
from parity import TOL, Worst
from stepwise import oracle_stash_from_gpu, read_gpu_stash

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

LM = synth.AttentionSpec(causal=True, rotary_dim=32, rotary_base=500.0)
FULL = synth.AttentionSpec(causal=True, cap=20.0, slopes=True, rotary_dim=16, rotary_layout="interleaved",
                           rotary_scaling="parts", rotary_factor=4.0, rotary_original_length=16)
BIDIRECTIONAL = synth.AttentionSpec(rotary_dim=64)


def _spec(heads=4, S=40, head="none", layers=2, attention=LM, stash="bf16", d=128, batch=3, k=1):
    dims = (d, heads, 2 * d, S) + ((104,) if head == "ce" else ())
    return synth.StageSpec("transformer", "bf16", head, k, 4, batch, layers, dims, 5e-5, 0.9, attention=attention,
                           stash=stash)


def _masks(spec, m, kind):
    g = np.random.default_rng(100 + m)
    B, S = spec.batch, spec.dims[3]
    out = {}
    if "doc" in kind:
        out["documents"] = np.cumsum(g.random((B, S)) < 3 / S, axis=1).astype(np.int32)
    if "prefix" in kind:
        out["prefix"] = g.integers(0, S, B).astype(np.int32)
    if "len" in kind:
        out["kv_lengths"] = g.integers(S // 2, S + 1, B).astype(np.int32)
    return out


CASES = {
    "causal": (_spec(), ""),
    "documents": (_spec(heads=2, S=128), "doc"),
    "vocabulary": (_spec(head="ce", k=3, S=72), "doc prefix"),
    "capped": (_spec(attention=FULL, S=104, heads=8), "prefix len"),
    "bidirectional": (_spec(attention=BIDIRECTIONAL, heads=2, S=24), "len"),
    "packed": (_spec(stash="e4m3"), "doc"),
    "packed_vocabulary": (_spec(head="ce", k=3, stash="e4m3", attention=FULL, heads=8), ""),
    "packed_unmasked": (_spec(attention=None, stash="e4m3", heads=2, S=128), ""),
    "packed_gemm": (_spec(attention=None, stash="e4m3", heads=8, S=16), ""),
}


def _inputs(spec, m):
    ce = spec.head == "ce"
    return (synth.stage_input(spec, m), None if ce else synth.upstream_grad(spec, m),
            synth.labels(spec, m) if ce else None)


def _recomputed(spec, P, l, c, masks):
    """(name, value) of each activation of layer l, from the stashed ones before it."""
    d, H, _, S = spec.dims[:4]
    B, p = spec.batch, f"layer{l}."
    lin = lambda x, n: Lr.linear(x, P[p + n + ".weight"], P[p + n + ".bias"])
    norm = lambda x, n: Lr.layernorm_forward(x, P[p + n + ".weight"], P[p + n + ".bias"], stages.LN_EPS)[0]
    qkv = to_bf16(lin(c["a"], "attn.qkv"))
    if spec.attention is not None:
        qkv = At.turn_heads(spec.attention, qkv, B, S, H)
    q, k, v = (Lr.split_heads(c["qkv"][:, i * d:(i + 1) * d], B, S, H) for i in range(3))
    probs = Lr.attention_probs(q, k) if spec.attention is None else At.probs(spec.attention, q, k, masks)[0]
    return [("qkv", qkv), ("ctx", Lr.merge_heads(probs @ v)), ("r1", c["a"] + lin(c["ctx"], "attn.out")),
            ("h", norm(c["r1"], "ln1")), ("f1", Lr.relu(lin(c["h"], "ffn1"))), ("r2", c["h"] + lin(c["f1"], "ffn2"))]


@pytest.mark.parametrize("name", list(CASES))
def test_stage_matches_the_oracle(name):
    from paper_1809_02839_amd.pipeline import Pipeline, stage_task_order
    spec, kind = CASES[name]
    print(f"[stage attention] {name}", flush=True)
    k, N, steps = spec.stage_index, spec.num_stages, 5
    W0 = synth.initial_params(spec)
    states, stash = {}, {}
    masks = {m: _masks(spec, m, kind) for m in range(steps)}
    device = {m: {n: torch.from_numpy(a).cuda() for n, a in masks[m].items()} for m in range(steps)}
    pipe = Pipeline((spec,), [W0])
    out = pipe.run(steps, _inputs, keep_io=True, masks=(lambda s, m: device[m]) if spec.attention else None,
                   on_forward=lambda k_, m, st: stash.__setitem__(m, read_gpu_stash(spec, st, m)),
                   on_update=lambda k_, u, st: states.__setitem__(u, st.get_state()))
    torch.cuda.synchronize()
    f32 = lambda t: t.float().cpu().numpy()
    worst, tol = Worst(name), TOL["bf16"]
    lr, gamma = float(np.float32(spec.lr)), float(np.float32(spec.momentum))
    sf, sb = method.staleness_versions("spectrain", k, N)
    rnd = stages.weight_rounder(spec)
    W, v = W0.astype(np.float64), np.zeros(W0.size)
    u, mine = 0, {}
    for task, m in stage_task_order(k, N, steps):
        x, dy, lab = _inputs(spec, m)
        if task == "F":
            P = stages.unpack(spec, rnd(method.predict(W, v, sf, lr)))
            y, loss, st = stages.forward(spec, P, x, lab, masks=masks[m])
            yg = None if spec.head == "ce" else f32(out["y"][(k, m)])
            if spec.head == "ce":
                worst.check2("loss", [out["loss"][m].item()], [loss], tol, f"m{m}")
            else:
                worst.check2("y", yg, y, tol, f"m{m}")
            bufs = stash.pop(m)
            mine[m] = oracle_stash_from_gpu(spec, bufs, x, yg)
            if spec.stash == "e4m3":     # the backward's layer norms keep the statistics of the unrounded rows
                for l, c in enumerate(mine[m]["layers"]):
                    for ln, i in (("ln1", 5), ("ln2", 10)):
                        c[ln] = tuple(bufs[13 * l + j].view(np.float32).astype(np.float64)[:, None] for j in (i, i + 1))
            if spec.stash == "bf16":     # an 8-bit buffer is tested against its bf16 original below
                for l, c in enumerate(mine[m]["layers"]):
                    for n, want in _recomputed(spec, P, l, c, masks[m]):
                        worst.check2("fwd " + n, c[n], want, tol, f"m{m} layer {l}")
        else:
            P = stages.unpack(spec, rnd(method.predict(W, v, sb, lr)))
            dx, grads = stages.backward(spec, P, mine.pop(m), dy, masks=masks[m])
            W1, v1 = method.momentum_sgd_step(W, v, stages.pack(spec, grads), lr, gamma)
            u += 1
            Wg, vg = states[u]
            worst.check2("v", vg, v1, tol, f"u{u}")
            worst.check2("W", Wg, W1, tol, f"u{u}")
            worst.check2("dx", f32(out["dx"][(k, m)]), dx, tol, f"m{m}")
            W, v = Wg.astype(np.float64), vg.astype(np.float64)
    pipe.destroy()
    print(f"[stage attention] {name}: {worst.report()}", flush=True)


def _bf16(raw, cols):
    return torch.from_numpy(raw.copy()).view(torch.bfloat16).reshape(-1, cols)


@pytest.mark.parametrize("head", ["none", "ce"])
def test_packed_stash_holds_the_checkpoints_of_the_plain_one(head):
    """The forward does not change by a bit, and every packed buffer reads back as the packed and restored
    original."""
    from paper_1809_02839_amd import native
    spec = _spec(head=head, k=2, S=56)
    W0 = synth.initial_params(spec)
    st = [native.Stage(native.desc_from_spec(spec), W0) for _ in range(2)]
    for s in st:
        s.configure(spec)
    st[1].set_stash("e4m3")
    x, dy, lab = _inputs(spec, 0)
    x = torch.from_numpy(x).cuda().bfloat16()
    y = [torch.empty(spec.output_shape(), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    loss = [torch.empty(1, device="cuda") for _ in range(2)]
    for i, s in enumerate(st):
        if head == "ce":
            s.forward(0, x, None, torch.from_numpy(lab).int().cuda(), loss[i])
        else:
            s.forward(0, x, y[i])
    torch.cuda.synchronize()
    assert torch.equal(*(loss if head == "ce" else y))
    plain, packed = (read_gpu_stash(spec, s, 0) for s in st)
    d, F = spec.dims[0], spec.dims[2]
    for i in plain:
        assert plain[i].size == packed[i].size
        if i < 13 * spec.num_layers and i % 13 in (4, 7, 8, 9, 12) and plain[i].size:
            t = _bf16(plain[i], F if i % 13 == 8 else d).cuda()
            codes = torch.empty(t.shape, dtype=torch.uint8, device="cuda")
            scales = torch.empty(t.shape[0], t.shape[1] // 32, dtype=torch.uint8, device="cuda")
            want = torch.empty_like(t)
            native.checkpoint_pack(t, codes, scales)
            native.checkpoint_restore(codes, scales, want)
            assert torch.equal(want.cpu(), _bf16(packed[i], t.shape[1])), i
        else:
            assert np.array_equal(plain[i], packed[i]), i
    for s in st:
        s.destroy()


@pytest.mark.parametrize("stash", ["bf16", "e4m3"])
def test_combined_noalloc_and_captured_calls_give_the_separate_calls_bits(stash):
    from paper_1809_02839_amd import native
    spec = _spec(stash=stash, S=64, k=1)
    W0 = synth.initial_params(spec)
    stream = torch.cuda.Stream()
    st = [native.Stage(native.desc_from_spec(spec), W0, stream) for _ in range(3)]
    for s in st:
        s.configure(spec)
    n = 4
    with torch.cuda.stream(stream):
        xs = [torch.from_numpy(synth.stage_input(spec, m)).cuda().bfloat16() for m in range(n)]
        dys = [torch.from_numpy(synth.upstream_grad(spec, m)).cuda().bfloat16() for m in range(n)]
        docs = [torch.from_numpy(_masks(spec, m, "doc")["documents"]).cuda() for m in range(n)]
        ys = [[torch.zeros_like(x) for x in xs] for _ in st]
        dxs = [[torch.zeros_like(x) for x in xs] for _ in st]
    torch.cuda.synchronize()

    def separate(s, i, back):
        s.set_masks(0, documents=docs[0])
        s.forward(0, xs[0], ys[i][0])
        for m in range(n):
            if m + 1 < n:
                s.set_masks(m + 1, documents=docs[m + 1])
                s.forward(m + 1, xs[m + 1], ys[i][m + 1])
            back(m, dys[m], dxs[i][m])
            s.update(2, 0)

    def combined(s, i):
        s.set_masks(0, documents=docs[0])
        s.forward(0, xs[0], ys[i][0])
        for m in range(n):
            if m + 1 < n:
                s.set_masks(m + 1, documents=docs[m + 1])
                s.forward_backward(m + 1, xs[m + 1], ys[i][m + 1], m, dys[m], dxs[i][m])
            else:
                s.backward(m, dys[m], dxs[i][m])
            s.update(2, 0)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        combined(st[1], 1)
    for replay in range(3):
        separate(st[0], 0, st[0].backward)
        separate(st[2], 2, st[2].backward_noalloc)
        with torch.cuda.stream(stream):
            graph.replay()
        torch.cuda.synchronize()
        states = [s.get_state() for s in st]
        for i in (1, 2):
            for m in range(n):
                assert torch.equal(ys[0][m], ys[i][m]) and torch.equal(dxs[0][m], dxs[i][m]), (replay, i, m)
            assert all(np.array_equal(a, b) for a, b in zip(states[0], states[i])), (replay, i)
    for s in st:
        s.destroy()


def test_options_are_refused_where_they_do_not_belong():
    from paper_1809_02839_amd import native
    fc = synth.StageSpec("fc", "bf16", "none", 1, 3, 64, 1, (64, 64, 64), 0.01, 0.9)
    s = native.Stage(native.desc_from_spec(fc), synth.initial_params(fc))

    def refused(code, f, *a, **kw):
        with pytest.raises(native.SpecTrainError) as e:
            f(*a, **kw)
        assert e.value.code == code, e.value

    refused(native.EINVAL, s.set_attention, causal=True)
    refused(native.EINVAL, s.set_stash, "e4m3")
    refused(native.ESTATE, lambda: native._check(native.lib().spectrain_stage_set_masks(s.h, 0, None)))
    s.destroy()

    spec = _spec(attention=None)
    s = native.Stage(native.desc_from_spec(spec), synth.initial_params(spec))
    docs = torch.zeros(3, 40, dtype=torch.int32, device="cuda")
    refused(native.ESTATE, s.set_masks, 0, documents=docs)
    for bad in (dict(cap=-1.0), dict(rotary_dim=5), dict(rotary_dim=34), dict(rotary_dim=-2),
                dict(rotary_dim=32, rotary_base=0.5), dict(rotary_dim=32, rotary_scaling="linear", rotary_factor=0.1),
                dict(slopes=[float("nan")] * 4)):
        refused(native.EINVAL, s.set_attention, **bad)
    assert native.lib().spectrain_stage_set_stash(s.h, 7) == native.EINVAL
    s.set_attention(causal=False)
    refused(native.EINVAL, s.set_masks, 0, prefix=docs[:, 0].contiguous())
    x = torch.zeros(spec.input_shape(), dtype=torch.bfloat16, device="cuda")
    y = torch.empty_like(x)
    s.set_masks(7, documents=docs)
    s.forward(7, x, y)
    refused(native.ESTATE, s.set_masks, 7, documents=docs)
    refused(native.ESTATE, s.set_attention, causal=True)
    refused(native.ESTATE, s.set_stash, "e4m3")
    s.backward(7, x, None)
    s.set_stash("e4m3")              # the gradient of mini-batch 7 still waits: it is kept
    s.update(0, 0)
    s.destroy()
    wide = synth.StageSpec("transformer", "bf16", "none", 0, 1, 2, 1, (256, 1, 64, 16), 5e-5, 0.9)
    s = native.Stage(native.desc_from_spec(wide), synth.initial_params(wide))
    refused(native.EINVAL, s.set_attention, causal=True)      # a head of 256
    s.destroy()


def test_options_come_and_go_without_a_trace():
    """A stage whose options were set and cleared gives the bits of one that never had any."""
    from paper_1809_02839_amd import native
    spec = _spec(attention=None, S=128, heads=2)
    W0 = synth.initial_params(spec)
    st = [native.Stage(native.desc_from_spec(spec), W0) for _ in range(2)]
    st[1].set_attention(causal=True, rotary_dim=64)
    st[1].set_stash("e4m3")
    st[1].clear_attention()
    st[1].set_stash("bf16")
    x = torch.from_numpy(synth.stage_input(spec, 0)).cuda().bfloat16()
    dy = torch.from_numpy(synth.upstream_grad(spec, 0)).cuda().bfloat16()
    y, dx = ([torch.empty_like(x) for _ in st] for _ in range(2))
    for i, s in enumerate(st):
        s.forward(0, x, y[i])
        s.backward(0, dy, dx[i])
        s.update(1, 0)
    torch.cuda.synchronize()
    assert torch.equal(*y) and torch.equal(*dx)
    (Wa, va), (Wb, vb) = (s.get_state() for s in st)
    assert np.array_equal(Wa, Wb) and np.array_equal(va, vb)
    for s in st:
        s.destroy()
