"""Positions and masked attention of a transformer stage in float64 (test
infrastructure only): rotary positions of the query and key heads, scores
capped by tanh, a bias that grows with distance, and causal, prefix, document
and length masks, with the gradients."""
import math

import numpy as np

from . import layers as Lr


def frequencies(at):
    rot, base = at.rotary_dim, at.rotary_base
    if at.rotary_scaling == "ntk" and rot > 2:
        base = base * at.rotary_factor ** (rot / (rot - 2))
    w = base ** (-np.arange(0, rot, 2) / rot)
    if at.rotary_scaling == "linear":
        w = w / at.rotary_factor
    if at.rotary_scaling == "parts":
        keep = np.clip((at.rotary_original_length * w / (2 * math.pi) - 1) / 31, 0, 1)
        w = w * (keep + (1 - keep) / at.rotary_factor)
    return w


def turn(at, x, inverse=False):
    """x [B, H, S, dh] turned by token index."""
    rot = at.rotary_dim
    if rot == 0:
        return x
    m = 0.1 * math.log(at.rotary_factor) + 1 if at.rotary_scaling == "parts" else 1.0
    t = np.arange(x.shape[2])[:, None] * frequencies(at) * (-1 if inverse else 1)
    c, s = m * np.cos(t), m * np.sin(t)
    first, second = ((slice(0, rot // 2), slice(rot // 2, rot)) if at.rotary_layout == "half"
                     else (slice(0, rot, 2), slice(1, rot, 2)))
    a, b = x[..., first], x[..., second]
    y = x.copy()
    y[..., first], y[..., second] = a * c - b * s, a * s + b * c
    return y


def turn_heads(at, qkv, B, S, H, inverse=False):
    """The query and key heads of a packed [B*S, 3 d] turned."""
    dm = qkv.shape[1] // 3
    parts = [turn(at, Lr.split_heads(qkv[:, i * dm:(i + 1) * dm], B, S, H), inverse) for i in (0, 1)]
    return np.concatenate([Lr.merge_heads(p) for p in parts] + [qkv[:, 2 * dm:]], axis=1)


def visible(at, B, S, masks):
    """[B, S, S]: whether a row (second axis) sees a key (third)."""
    masks = masks or {}
    i, j = np.arange(S)[:, None], np.arange(S)[None]
    see = np.ones((B, S, S), bool)
    if at.causal:
        see &= j <= i
        if masks.get("prefix") is not None:
            see |= j < np.asarray(masks["prefix"])[:, None, None]
    if masks.get("documents") is not None:
        ids = np.asarray(masks["documents"])
        run = np.cumsum(np.concatenate([np.zeros((B, 1), int), ids[:, 1:] != ids[:, :-1]], axis=1), axis=1)
        see &= run[:, :, None] == run[:, None, :]
    if masks.get("kv_lengths") is not None:
        see &= j < np.asarray(masks["kv_lengths"])[:, None, None]
    return see


def probs(at, q, k, masks):
    """Softmax over the visible keys (rows without one: zero) and tanh of the
    capped scores (None without a cap); q, k [B, H, S, dh]."""
    B, H, S, dh = q.shape
    z = q @ k.transpose(0, 1, 3, 2) / np.sqrt(dh)
    t = np.tanh(z / at.cap) if at.cap else None
    s = at.cap * t if at.cap else z
    if at.slopes:
        far = np.abs(np.arange(S)[:, None] - np.arange(S)[None])
        s = s - at.slope_values(H).astype(np.float64)[:, None, None] * far
    see = visible(at, B, S, masks)[:, None]
    s = np.where(see, s, -np.inf)
    top = s.max(axis=-1, keepdims=True)
    e = np.exp(s - np.where(np.isinf(top), 0.0, top))
    total = e.sum(axis=-1, keepdims=True)
    return e / np.where(total == 0, 1.0, total), t


def backward(at, dctx, qkv, B, S, H, masks, r):
    """Gradient of the packed qkv before its heads were turned; r rounds
    operands (bf16) or is the identity."""
    dm = qkv.shape[1] // 3
    q, k, v = (Lr.split_heads(qkv[:, i * dm:(i + 1) * dm], B, S, H) for i in range(3))
    p, t = probs(at, q, k, masks)
    do = Lr.split_heads(dctx, B, S, H)
    dv = r(r(p).transpose(0, 1, 3, 2) @ do)
    dp = do @ v.transpose(0, 1, 3, 2)
    ds = p * (dp - (p * dp).sum(axis=-1, keepdims=True))
    if t is not None:
        ds = ds * (1 - t * t)
    ds = r(ds)
    scale = 1.0 / np.sqrt(q.shape[-1])
    dq, dk = r(ds @ k * scale), r(ds.transpose(0, 1, 3, 2) @ q * scale)
    dqkv = np.concatenate([Lr.merge_heads(g) for g in (dq, dk, dv)], axis=1)
    return r(turn_heads(at, dqkv, B, S, H, inverse=True)) if at.rotary_dim else dqkv
