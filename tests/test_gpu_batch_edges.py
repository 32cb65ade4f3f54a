"""Batches at the edges of their tables: starts of sequences far outside the tokens, and what append and attention make of them."""
import pytest
import torch

from paper_2405_13053_b200 import binding as mb
from tests.test_gpu_prefix_attention import BF16, F32, call, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new,held,prefix,D,dtype", [([9, 5, 30], [10, 200, 3], 100, 128, BF16), ([300, 40, 200], [0, 130, 20], 0, 64, BF16),
                                                     ([2, 1, 1], [10, 90, 3], 40, 128, BF16), ([9, 5, 30], [10, 70, 3], 33, 64, F32)])
def test_a_start_far_below_zero_has_no_tokens(new, held, prefix, D, dtype):
    """The lowest start behind a positive one: their difference is past 32 bits.  Out of contract, but no memory beside the
    tensors is read or written, and later calls on the workspace are as they were."""
    s = make(B=3, new=new, held=held, page=16, prefix=prefix, H=8, K=2, D=D, dtype=dtype)
    T, low = sum(new), -2 ** 31
    ws = mb.meteora_prefix_attention_workspace(s["q"], s["kc"], s["table"], s["prefix"])
    want = call(s, workspace=ws)
    for cu in ([T - 1, low, low, T], [1, low + 1, low, 2 ** 31 - 1], [T, low, T, low], [3, low, T, T]):
        around = torch.full((T + 8, 8, D), 3.0, dtype=dtype, device="cuda")
        call(dict(s, cu=torch.tensor(cu, dtype=torch.int32, device="cuda")), out=around[4:-4], workspace=ws)
        assert (around[:4] == 3).all() and (around[-4:] == 3).all()
    assert torch.equal(call(s, workspace=ws), want) and mb.meteora_workspace_status(ws) == 0


@pytest.mark.parametrize("low", [-3, -2 ** 31])
def test_a_start_below_zero_counts_as_zero(low):
    """The first of the tokens that the call has is the first new one of its sequence, in the append as in the attention."""
    B, K, H, D, page = 2, 2, 4, 64, 16
    g = torch.Generator(device="cuda").manual_seed(4)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g).to(BF16)  # noqa: E731
    T, r = 9, mb.meteora_rotary_init(D, 10000.0)
    k, v, q = rand(T, K, D), rand(T, K, D), rand(T, H, D)
    table = torch.arange(2 * B, dtype=torch.int32, device="cuda").view(B, 2) + 1         # page 0 is nobody's
    lengths = torch.tensor([14, 3], dtype=torch.int32, device="cuda")
    got = []
    for first, end in ((low, T), (0, 2 ** 31 - 1)):
        kc, vc = (torch.zeros(2 * B + 2, K, page, D, dtype=BF16, device="cuda") for _ in range(2))
        cu = torch.tensor([first, 6, end], dtype=torch.int32, device="cuda")
        y = mb.meteora_cache_append(k, v, kc, vc, table, lengths, r, cu_tokens=cu, q=q)
        got.append((y, kc, vc, mb.meteora_prefix_attention(y, kc, vc, table, lengths, cu_tokens=cu)))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert torch.equal(vc[1, :, 14:], v[:2].transpose(0, 1)) and torch.equal(vc[2, :, :4], v[2:6].transpose(0, 1))
    assert torch.equal(vc[3, :, 3:6], v[6:].transpose(0, 1)) and int((vc != 0).any(-1).sum()) == T * K
