"""Oracle of the cache held in 4 bits, the attention over it and the
verification of drafted tokens (test infrastructure; numpy, float64 where the
format does not state a narrower step).
"""
from __future__ import annotations

import numpy as np

LIMIT = np.float32(16384.0)


def quantise(x, group: int):
    """Codes [..., D] uint8, scales and offsets [..., D / group] float16 of rows x (float32 values)."""
    x = np.asarray(x, np.float32)
    x = np.clip(np.where(np.isnan(x), np.float32(0), x), -LIMIT, LIMIT)
    x = x.reshape(*x.shape[:-1], x.shape[-1] // group, group)
    z = x.min(-1).astype(np.float16)
    span = x.max(-1) - z.astype(np.float32)
    s = np.where(span > 0, span * (np.float32(1) / np.float32(15)), np.float32(0)).astype(np.float16)
    s32 = s.astype(np.float32)
    inv = np.divide(np.float32(1), s32, out=np.zeros_like(s32), where=s32 > 0)
    n = np.rint((x - z.astype(np.float32)[..., None]) * inv[..., None])
    n = np.clip(n, 0, 15).astype(np.uint8)
    return n.reshape(*n.shape[:-2], n.shape[-2] * group), s, z


def value(n, s, z) -> np.ndarray:
    """The values that codes stand for, float64."""
    g = n.shape[-1] // s.shape[-1]
    n = n.reshape(*s.shape, g).astype(np.float64)
    v = z.astype(np.float64)[..., None] + s.astype(np.float64)[..., None] * n
    return v.reshape(*v.shape[:-2], v.shape[-2] * g)


def stand_for(x, group: int) -> np.ndarray:
    return value(*quantise(x, group))


def attend(k, v, q, scale: float) -> np.ndarray:
    """k, v [N][D] (all tokens, oldest first), q [G][nq][D] of the last nq of them -> [G][nq][D]."""
    G, nq, D = q.shape
    out = np.zeros((G, nq, D))
    for t in range(nq):
        see = k.shape[0] - (nq - 1 - t)
        if see <= 0:
            continue
        x = q[:, t].astype(np.float64) @ k[:see].T * scale
        w = np.exp(x - x.max(-1, keepdims=True))
        out[:, t] = (w / w.sum(-1, keepdims=True)) @ v[:see]
    return out


def distribution(logits, temperature: float, top_k: int, top_p: float):
    """The sampler's tokens, by falling logit (ties to the lower id), and their probabilities."""
    x = np.asarray(logits, np.float64)
    at = np.nonzero(~np.isnan(x))[0]
    at = at[np.lexsort((at, -x[at]))][:top_k]
    w = np.exp((x[at] - x[at[0]]) / float(np.float32(temperature)))
    cum = np.cumsum(w)
    keep = int(np.argmax(cum >= float(np.float32(top_p)) * cum[-1])) + 1
    return at[:keep], w[:keep] / w[:keep].sum()


def verify(logits, draft_logits, tok, n_draft: int, u_accept, u_draw: float, sampler, draft_sampler=None):
    """One sequence: logits [T + 1][V], draft_logits [T][Vd] or None; sampler = (temperature, top_k, top_p).
    Returns (tokens, margin): the tokens that stand and the next one, and the least distance of a decision from its
    border, relative to the mass it is taken in."""
    draft_sampler = draft_sampler or sampler
    res, margin = [], np.inf
    for t in range(n_draft + 1):
        ids, p = distribution(logits[t], *sampler)
        r = p
        if t < n_draft:
            x = int(tok[t])
            q = {x: 1.0}
            if draft_logits is not None:
                q = dict(zip(*(a.tolist() for a in distribution(draft_logits[t], *draft_sampler))))
            px = dict(zip(ids.tolist(), p.tolist())).get(x, 0.0)
            lhs = float(u_accept[t]) * q.get(x, 0.0)
            if lhs != px:
                margin = min(margin, abs(lhs - px))
            if lhs < px:
                res.append(x)
                continue
            r = np.maximum(p - np.array([q.get(i, 0.0) for i in ids.tolist()]), 0.0)
            if not r.sum() > 0:
                r = p
        cum = np.cumsum(r)
        target = float(u_draw) * cum[-1]
        over = np.nonzero(cum > target)[0]
        margin = min(margin, np.abs(cum - target).min() / cum[-1])
        res.append(int(ids[over[0]]) if len(over) else int(ids[np.nonzero(r)[0][-1]]))
        break
    return res, margin
