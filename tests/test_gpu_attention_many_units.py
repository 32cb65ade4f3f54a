"""Attention whose workers have very many units each: thousands of sequences of thousands of key heads."""
import pytest
import torch

from paper_2405_13053_b200 import binding as mb

pytestmark = pytest.mark.gpu


def test_more_than_8192_units_of_a_warp():
    """19.7 M units of one row on the 2368 warps of the 16-row kernel.  All sequences read one page, so a row's result follows from
    its length and head alone.  Bound: weights off by 2^-8 (1 + 2^-7) of themselves, their sum alike, move an average of
    values up to m by at most that times their mean distance from it, which is m at most; the result's half step is 2^-8 of it;
    2^-7 m for the first leaves 2^-8 m for sums in fp32 and the second order."""
    B, K, D, page = 4096, 4800, 8, 16
    g = torch.Generator(device="cuda").manual_seed(0)
    kc, vc = (torch.randn(1, K, page, D, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    q = torch.randn(B, K, D, device="cuda", generator=g).to(torch.bfloat16)
    lengths = (torch.arange(B, dtype=torch.int32, device="cuda") * 7) % 15
    table = torch.zeros(B, 1, dtype=torch.int32, device="cuda")
    ws = mb.meteora_prefix_attention_workspace(q, kc, table)
    out = mb.meteora_prefix_attention(q, kc, vc, table, lengths, workspace=ws)
    assert mb.meteora_workspace_status(ws) == 0
    for b0 in range(0, B, 64):                                       # every row, 64 sequences at a time
        x, n = q[b0:b0 + 64].double(), lengths[b0:b0 + 64, None, None]
        s = torch.einsum("bkd,kpd->bkp", x, kc[0].double()) * D ** -0.5
        s = s.masked_fill(torch.arange(page, device="cuda") > n, -float("inf"))
        want = torch.einsum("bkp,kpd->bkd", torch.softmax(s, -1), vc[0].double())
        off = (out[b0:b0 + 64].double() - want).abs()
        assert bool((off <= 2.0 ** -8 * want.abs() + 2.0 ** -7 * vc.double().abs().max()).all())
