"""Plain 64-bit forms of the operators on heads, from their definitions, for the tests: rotation, norm, a batch over a paged
cache and its attention.  Everything is numpy on the host."""
import math

import numpy as np
import torch


def to64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def frequencies(dim, theta, scaling="none", factor=1.0, original_context=0.0, low=1.0, high=4.0):
    f = []
    for i in range(dim // 2):
        fi = theta ** (-2.0 * i / dim)
        if scaling == "linear":
            fi /= factor
        if scaling == "bands":
            keep = min(1.0, max(0.0, (original_context * fi / (2 * math.pi) - low) / (high - low)))
            fi = keep * fi + (1 - keep) * fi / factor
        f.append(fi)
    return np.array(f)


def rotate(x, positions, spec, layout="half", attention_scale=1.0, inverse=False):
    """x[T, heads, dim] float64; spec = arguments of `frequencies` (dim first)."""
    rot = spec["dim"]
    ang = np.asarray(positions, np.float64)[:, None, None] * frequencies(**spec)
    c, s = np.cos(ang) * attention_scale, np.sin(ang) * attention_scale * (-1 if inverse else 1)
    y = x.copy()
    a, b = (x[..., :rot // 2], x[..., rot // 2:rot]) if layout == "half" else (x[..., 0:rot:2], x[..., 1:rot:2])
    ya, yb = a * c - b * s, b * c + a * s
    if layout == "half":
        y[..., :rot // 2], y[..., rot // 2:rot] = ya, yb
    else:
        y[..., 0:rot:2], y[..., 1:rot:2] = ya, yb
    return y


def pair_size(x, spec, layout="half"):
    """|a| + |b| of every entry's pair (an entry that passes through stands for itself)."""
    rot = spec["dim"]
    m = np.abs(x).copy()
    a, b = (m[..., :rot // 2], m[..., rot // 2:rot]) if layout == "half" else (m[..., 0:rot:2], m[..., 1:rot:2])
    t = a + b
    if layout == "half":
        m[..., :rot // 2], m[..., rot // 2:rot] = t, t
    else:
        m[..., 0:rot:2], m[..., 1:rot:2] = t, t
    return m


def norm(x, gain, eps):
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def places(batch, t):
    """(sequence, own place) of token t, or None: batch = dict(B, cu or None, lengths)."""
    cu = batch["cu"]
    if cu is None:
        b = t if t < len(batch["lengths"]) else None
        first = t
    else:
        b = next((i for i in range(len(cu) - 1) if cu[i] <= t < cu[i + 1]), None)
        first = cu[b] if b is not None else 0
    if b is None or batch["lengths"][b] < 0:
        return None
    return b, batch["lengths"][b] + t - first


def page_entry(pages, i, page_size, n_pages):
    """(page, entry) of the i-th token of a list of pages, None where there is none."""
    slot = i // page_size
    if slot >= len(pages) or not 0 <= pages[slot] < n_pages:
        return None
    return pages[slot], i % page_size


def attention(q, kc, vc, batch, scale):
    """Row by row: (out, lse, A, B, D, n) with A = sum of w |v - out|, B = sum of w |v|, D = largest sum |q||k|, n = keys.
    Rows of tokens without a sequence are NaN.  q[T, heads, dim], caches [pages, kv heads, page, dim], float64."""
    T, H, D = q.shape
    n_pages, kv, page, _ = kc.shape
    out, A, B = np.full((T, H, D), np.nan), np.zeros((T, H, D)), np.zeros((T, H, D))
    lse, size, count = np.full((T, H), np.nan), np.zeros((T, H)), np.zeros((T, H))
    for t in range(T):
        at = places(batch, t)
        if at is None:
            continue
        b, i = at
        where = [page_entry(batch["prefix_pages"], j, page, n_pages) for j in range(batch["prefix_len"])]
        where += [page_entry(batch["table"][b], j, page, n_pages) for j in range(i + 1)]
        where = [w for w in where if w is not None]
        if not where:
            out[t], lse[t] = 0.0, -np.inf
            continue
        p, e = np.array([w[0] for w in where]), np.array([w[1] for w in where])
        for h in range(H):
            k, v = kc[p, h // (H // kv), e], vc[p, h // (H // kv), e]
            s = k @ q[t, h] * scale
            top = s.max()
            w = np.exp(s - top)
            total = w.sum()
            w = w / total
            out[t, h] = w @ v
            lse[t, h] = top + np.log(total)
            A[t, h], B[t, h] = w @ np.abs(v - out[t, h]), w @ np.abs(v)
            size[t, h], count[t, h] = (np.abs(k) @ np.abs(q[t, h])).max() * abs(scale), len(p)
    return out, lse, A, B, size, count
