"""Attention where every worker of every kernel goes through many tiles and units: its rings several times around, the running
maximum moving tile by tile, units that start and end inside a share.  A sample of rows against the definition in 64 bits, with
the bounds of test_gpu_prefix_attention.py."""
import math

import numpy as np
import pytest
import torch

from paper_2405_13053_b200 import binding as mb
from tests import heads_util as hu

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def make(new, held, page, prefix, H, K, D, dtype, grow, seed=0):
    """Keys grow (or, grow < 0, shrink) to four times their size along the prefix and again along the own tokens."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    B, T = len(new), sum(new)
    width, n_prefix = max((n + h + page - 1) // page for n, h in zip(new, held)), (prefix + page - 1) // page
    order = torch.randperm(B * width + n_prefix, device="cuda", generator=g)
    table, prefix_pages = order[:B * width].view(B, width), order[B * width:]
    kc, vc = (rand(B * width + n_prefix, K, page, D) for _ in range(2))
    for pages in (table, prefix_pages[None]):
        n = pages.shape[1] * page
        size = 1 + 3 * torch.arange(n, device="cuda") / max(n - 1, 1)
        if grow:
            kc[pages] *= (size if grow > 0 else size.flip(0)).view(1, -1, 1, page, 1)
    to32 = lambda x: torch.as_tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    return dict(q=rand(T, H, D).to(dtype), kc=kc.to(dtype), vc=vc.to(dtype), table=to32(table), prefix_pages=to32(prefix_pages), prefix=prefix,
                lengths=to32(held), cu=to32(np.concatenate([[0], np.cumsum(new)])), new=new, held=held)


def token(s, b, j):
    """Row of the definition for the j-th new token of sequence b, all heads, in 64 bits: out, lse and the sizes the bounds go by."""
    page, K = s["kc"].shape[2], s["kc"].shape[1]
    t, n = int(s["cu"][b]) + j, s["held"][b] + j + 1
    i, p = torch.arange(n, device="cuda"), torch.arange(s["prefix"], device="cuda")
    slot = torch.cat([s["prefix_pages"].long()[p // page], s["table"].long()[b][i // page]])
    at = torch.cat([p, i]) % page
    k, v = (c[slot, :, at].double().transpose(0, 1) for c in (s["kc"], s["vc"]))             # [K, keys, D]
    q = s["q"][t].double().view(K, -1, s["q"].shape[2])
    x = q @ k.transpose(1, 2) / math.sqrt(q.shape[2])
    w = torch.softmax(x, -1)
    out = w @ v
    spread = torch.stack([torch.einsum("kn,knd->kd", w[:, r], (v - out[:, r, None]).abs()) for r in range(w.shape[1])], 1)
    size = (q.abs() @ k.abs().transpose(1, 2)).amax(-1) / math.sqrt(q.shape[2])
    flat = lambda y: y.flatten(0, 1).cpu().numpy()  # noqa: E731
    return t, flat(out), flat(torch.logsumexp(x, -1)), flat(spread), flat(w @ v.abs()), flat(size), k.shape[1]


# new, held, page, prefix, H, K, D, dtype: by the kernel that the own tokens take (and the prefix, where it is long)
CASES = {
    "warps": ([1] * 128, [1000 - 3 * b for b in range(128)], 64, 0, 32, 8, 128, BF16),
    "warps_64": ([1] * 64, [2000 - 7 * b for b in range(64)], 8, 0, 32, 8, 64, BF16),
    "warps_wide": ([1] * 32, [900 - 5 * b for b in range(32)], 32, 600, 32, 8, 256, BF16),
    "warps_places": ([1] * 40, [800 - 5 * b for b in range(40)], 20, 700, 24, 8, 80, BF16),          # keys looked up one by one
    "chunks": ([40 - b for b in range(32)], [1000 + b for b in range(32)], 16, 3000, 8, 8, 128, BF16),
    "chunks_64": ([24] * 64, [1500] * 64, 32, 0, 8, 8, 64, BF16),
    "chunks_wide": ([100, 70, 90, 120, 33, 64], [1500, 1600, 40, 900, 1700, 1200], 64, 1000, 4, 4, 256, BF16),
    "chunks_places": ([40] * 16, [900 - b for b in range(16)], 20, 800, 12, 4, 80, BF16),
    "own_tc": ([100 - b for b in range(16)], [300 + 11 * b for b in range(16)], 32, 0, 40, 40, 128, BF16),
    "own_tc_long": ([300] * 4, [5000, 4000, 10, 3001], 64, 0, 16, 4, 128, BF16),
    "own_tc_units": ([300 if b % 3 else 70 for b in range(48)], [b for b in range(48)], 16, 0, 64, 64, 64, BF16),
    "prefix": ([1] * 128, [5 * b % 90 for b in range(128)], 64, 32768, 32, 8, 128, BF16),
    "prefix_64": ([9] * 64, [40] * 64, 128, 16001, 12, 6, 64, BF16),
    "fp32": ([1] * 32, [900 - 9 * b for b in range(32)], 16, 0, 16, 8, 64, F32),
    "fp32_chunks": ([64, 50, 61, 1, 64, 9, 64, 64], [2000, 1000, 1500, 10, 1800, 2000, 3, 1900], 24, 500, 8, 8, 64, F32),
    "fp32_wide": ([20] * 8, [1200 - 30 * b for b in range(8)], 16, 900, 4, 2, 256, F32),
    "odd_heads": ([30, 2, 64], [2500, 2500, 2000], 5, 700, 12, 6, 33, BF16),
}


@pytest.mark.parametrize("grow", [1, 0, -1])
@pytest.mark.parametrize("name", CASES)
def test_long_shares(name, grow):
    new, held, page, prefix, H, K, D, dtype = CASES[name]
    s = make(new, held, page, prefix, H, K, D, dtype, grow)
    cu = None if max(new) == 1 else s["cu"]
    ws = mb.meteora_prefix_attention_workspace(s["q"], s["kc"], s["table"], prefix)
    call = lambda **kw: mb.meteora_prefix_attention(s["q"], s["kc"], s["vc"], s["table"], s["lengths"], s["prefix_pages"], prefix, cu_tokens=cu,  # noqa: E731
                                                    workspace=ws, **kw)
    y, lse = call(return_lse=True)
    assert torch.equal(call(), y) and mb.meteora_workspace_status(ws) == 0 and torch.isfinite(y).all()
    B = len(new)
    for b in sorted({0, 1, B // 3, B // 2, B - 2, B - 1}):
        for j in sorted({0, new[b] // 2, new[b] - 1}):
            t, ref, ref_lse, A, V, S, n = token(s, b, j)
            moved = 2 * (D + 4) * 2.0 ** -24 * S + 2.0 ** -20
            tol = (moved + (n + 130) * 2.0 ** -24)[:, None] * V
            if dtype == BF16:
                tol = tol + 2.0 ** -8 * (1 + 2.0 ** -7) * A
                tol = tol + hu.half_step(BF16) * (np.abs(ref) + tol)
            else:
                tol = tol + hu.half_step(F32) * np.abs(ref)
            worst = float((np.abs(hu.to64(y[t]) - ref) - tol).max())
            assert worst <= 0.0, (b, j, worst)
            off = moved + (n + 130) * 2.0 ** -24 + (2.0 ** -8 if dtype == BF16 else 0.0) + 2.0 ** -22 * (1 + np.abs(ref_lse))
            assert (np.abs(hu.to64(lse[t]) - ref_lse) <= off).all(), (b, j)
