"""The norm's gradient with strided, shared and overwritten tensors, through the C entry point, which takes results of any strides
and in place; against the call with contiguous tensors, bit for bit, or the definition in 64 bits with test_gpu_heads.py's bounds."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2405_13053_b200 import binding as mb
from tests import heads_util as hu
from tests.test_gpu_heads import BF16, F32, close, randn

pytestmark = pytest.mark.gpu
EPS = 1e-5


def view(t):
    return ctypes.byref(mb.MeteoraHeads(t.data_ptr(), t.stride(0), t.stride(1), t.shape[1])) if t is not None else None


def backward(dq_out, dk_out, q, k, gq, gk, dq, dk, pos, rot):
    T, _, D = q.shape
    lib = mb.load_library()
    n = lib.meteora_head_norm_rotary_backward_workspace_bytes(T, q.shape[1], k.shape[1], D)
    ws, sums = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.full((2, D), 7.0, device="cuda")
    rc = lib.meteora_head_norm_rotary_backward(view(dq_out), view(dk_out), view(q), view(k), gq.data_ptr(), gk.data_ptr(), view(dq), view(dk), sums[0].data_ptr(),
                                               sums[1].data_ptr(), pos.data_ptr(), 1, T, D, mb._dtype_code(q), ctypes.byref(rot), EPS, ws.data_ptr(), n,
                                               torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    return sums


def inputs(T, H, K, D, dtype):
    q, dq = randn(T, H, D, dtype=dtype), randn(T, H, D, dtype=dtype, seed=1)
    k, dk = randn(T, K, D, dtype=dtype, seed=2), randn(T, K, D, dtype=dtype, seed=3)
    gq, gk = ((1 + 0.3 * randn(D, dtype=F32, seed=s)).to(dtype) for s in (4, 5))
    return q, k, dq, dk, gq, gk, torch.arange(T, device="cuda") + 9


def definition(x, g, dy, pos, spec, layout, dx, dgain):
    p, dtype = pos.cpu().numpy(), x.dtype
    x, g, dy = hu.to64(x), hu.to64(g), hu.to64(dy)
    rs = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + EPS)
    n, dn, mag = x * rs, hu.rotate(dy, p, spec, layout, inverse=True), hu.pair_size(dy, spec, layout)
    close(dx, rs * (g * dn - n * (g * dn * n).mean(-1, keepdims=True)), rs * (np.abs(g) * mag + np.abs(n) * (np.abs(g) * mag * np.abs(n)).mean(-1, keepdims=True)),
          dtype, 2.0 ** -17)
    bound = (2.0 ** -18 + (min(x.shape[0] * x.shape[1], 4096) + 100) * 2.0 ** -24) * (mag * np.abs(n)).sum((0, 1))
    assert (np.abs(hu.to64(dgain) - (dn * n).sum((0, 1))) <= bound).all()


SIZES = [(77, 6, 2, 128, 128, "half", BF16), (700, 5, 3, 64, 32, "interleaved", BF16), (33, 4, 4, 80, 40, "half", BF16), (50, 3, 1, 256, 256, "half", F32),
         (9, 2, 1, 33, 32, "interleaved", F32)]


@pytest.mark.parametrize("T,H,K,D,rot,layout,dtype", SIZES)
@pytest.mark.parametrize("over", ["inputs", "gradients"])
def test_results_in_place(T, H, K, D, rot, layout, dtype, over):
    q, k, dq, dk, gq, gk, pos = inputs(T, H, K, D, dtype)
    r = mb.meteora_rotary_init(rot, 10000.0, layout)
    want = mb.meteora_head_norm_rotary_backward(dq, dk, q, k, gq, gk, pos, r, eps=EPS)
    to = (q, k) if over == "inputs" else (dq, dk)
    sums = backward(dq, dk, q, k, gq, gk, *to, pos, r)
    assert torch.equal(to[0], want[0]) and torch.equal(to[1], want[1]) and torch.equal(sums[0], want[2]) and torch.equal(sums[1], want[3])


@pytest.mark.parametrize("T,H,K,D,rot,layout,dtype", SIZES)
@pytest.mark.parametrize("shift", [0, 1, 4])
def test_slices_of_fused_tensors_and_heads_first(T, H, K, D, rot, layout, dtype, shift):
    """q, k and their gradients as slices of fused products from bases that allow 16-, 8- and 2- or 4-byte loads, results into such slices and into
    [heads, tokens]; what lies beside them stays."""
    q, k, dq, dk, gq, gk, pos = inputs(T, H, K, D, dtype)
    r = mb.meteora_rotary_init(rot, 10000.0, layout)

    def fused(a, b, fill):
        buf = torch.full((T, (H + K) * D + 8), fill, dtype=dtype, device="cuda")
        x, y = buf[:, shift:shift + H * D].unflatten(1, (H, D)), buf[:, shift + H * D:shift + (H + K) * D].unflatten(1, (K, D))
        if a is not None:
            x.copy_(a)
            y.copy_(b)
        return buf, x, y
    (_, fq, fk), (_, fdq, fdk), (to, tq, tk) = fused(q, k, 0.0), fused(dq, dk, 0.0), fused(None, None, 3.0)
    sums = backward(fdq, fdk, fq, fk, gq, gk, tq, tk, pos, r)
    got = mb.meteora_head_norm_rotary_backward(fdq, fdk, fq, fk, gq, gk, pos, r, eps=EPS)
    assert torch.equal(tq, got[0]) and torch.equal(tk, got[1]) and torch.equal(sums[0], got[2]) and torch.equal(sums[1], got[3])
    for i, (x, g, dy) in enumerate(((q, gq, dq), (k, gk, dk))):
        definition(x, g, dy, pos, dict(dim=rot, theta=10000.0), layout, got[i], got[2 + i])
    assert (to[:, :shift] == 3).all() and (to[:, shift + (H + K) * D:] == 3).all()
    first = torch.full((H + K + 2, T, D), 3.0, dtype=dtype, device="cuda")
    backward(fdq, fdk, fq, fk, gq, gk, first[1:H + 1].transpose(0, 1), first[H + 1:-1].transpose(0, 1), pos, r)
    assert torch.equal(first[1:H + 1].transpose(0, 1), got[0]) and torch.equal(first[H + 1:-1].transpose(0, 1), got[1])
    assert (first[0] == 3).all() and (first[-1] == 3).all()


@pytest.mark.parametrize("T,H,K,D,rot,layout,dtype", SIZES)
def test_a_gradient_that_all_tokens_or_heads_share(T, H, K, D, rot, layout, dtype):
    """Strides of 0, as sums and means hand their gradients back."""
    q, k, dq, dk, gq, gk, pos = inputs(T, H, K, D, dtype)
    r = mb.meteora_rotary_init(rot, 10000.0, layout)
    for a, b in ((dq[:1, :1], dk[:1, :1]), (dq[:1], dk[:1]), (dq[:, :1], dk[:, :1])):
        a, b = a.expand_as(q), b.expand_as(k)
        want = mb.meteora_head_norm_rotary_backward(a.contiguous(), b.contiguous(), q, k, gq, gk, pos, r, eps=EPS)
        got = mb.meteora_head_norm_rotary_backward(a, b, q, k, gq, gk, pos, r, eps=EPS)
        assert all(torch.equal(x, y) for x, y in zip(got, want))
