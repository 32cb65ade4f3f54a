"""Own tokens on the tensor cores where a CTA goes through many units: tiles of 256 rows followed by short ones, in which only
one of its two groups of 128 rows has work, and values that are no numbers on the way."""
import pytest
import torch

from paper_2405_13053_b200 import binding as mb

pytestmark = pytest.mark.gpu


def run(B, n, K, D, bad, page=64, seed=0):
    """B prompts of n tokens and K heads without and with the values `bad`, (key, entry, value) in every head of every sequence:
    results, and which entries see one."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    width = (n + page - 1) // page
    kc, vc = (torch.randn(B * width, K, page, D, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    q = torch.randn(B * n, K, D, device="cuda", generator=g).to(torch.bfloat16)
    table = torch.arange(B * width, dtype=torch.int32, device="cuda").view(B, width)
    lengths, cu = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.arange(B + 1, dtype=torch.int32, device="cuda") * n
    ws = mb.meteora_prefix_attention_workspace(q, kc, table)
    call = lambda v: mb.meteora_prefix_attention(q, kc, v, table, lengths, cu_tokens=cu, workspace=ws)  # noqa: E731
    want = call(vc)
    vb, hit = vc.clone(), torch.zeros(n, D, dtype=torch.bool, device="cuda")
    for key, e, value in bad:
        vb.view(B, width, K, page, D)[:, key // page, :, key % page, e] = value
        hit[key:, e] = True
    got = [call(vb) for _ in range(4)]
    assert mb.meteora_workspace_status(ws) == 0 and torch.isfinite(want).all()
    return want.view(B, n, K, D), [y.view(B, n, K, D) for y in got], hit[None, :, None].expand(B, n, K, D)


def check(B, n, K, D, bad):
    want, got, hit = run(B, n, K, D, bad)
    for y in got:
        assert not torch.isfinite(y[hit]).any()                      # the rows that see it, and they alone
        assert torch.equal(y[~hit], want[~hit])


@pytest.mark.parametrize("D", [64, 128])
def test_a_long_tile_before_forty_short_ones(D):
    """A bad value that only the long tiles' rows add by themselves: the second group is at that while more units than the ring
    describes pass by in which it has no rows."""
    check(80, 300, 40, D, [(100, 5, float("nan")), (101, D - 1, float("inf"))])


@pytest.mark.parametrize("B,n,K,D", [(200, 300, 1, 128), (200, 300, 1, 64), (90, 380, 2, 128), (80, 300, 40, 64)])
def test_bad_values_in_a_long_tile_and_in_the_short_one_behind_it(B, n, K, D):
    """The first group finds the short tile's bad value while the second one still adds the long tile's."""
    check(B, n, K, D, [(60, 7, float("nan")), (250, D - 1, float("-inf")), (270, 2, float("inf")), (n - 2, 11, float("nan"))])
