"""The norm of heads and its gradients at sizes of the entries far from 1, against their definitions in 64 bits; bounds as in
test_gpu_heads.py, whose arithmetic does not depend on the sizes as long as no step leaves the range of fp32 normal numbers."""
import numpy as np
import pytest
import torch

from paper_2405_13053_b200 import binding as mb
from tests import heads_util as hu
from tests.test_gpu_heads import BF16, F32, close, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size,eps", [(1e-15, 0.0), (1e-13, 1e-30), (1e12, 1e-5), (1e14, 1e-5), (1e15, 0.0), (1e16, 1e-5), (1e17, 1e-5)])
@pytest.mark.parametrize("D,rot,layout,dtype", [(128, 128, "half", F32), (128, 64, "interleaved", BF16), (80, 40, "half", F32), (7, 0, "half", F32)])
def test_gradients_of_heads_of_any_size(size, eps, D, rot, layout, dtype):
    T, H = 5, 3
    spec = dict(dim=rot, theta=10000.0)
    r = mb.meteora_rotary_init(rot, 10000.0, layout) if rot else None
    x, gain, dy = (randn(T, H, D, dtype=F32) * size).to(dtype), (1 + 0.3 * randn(D, dtype=F32, seed=1)).to(dtype), randn(T, H, D, dtype=dtype, seed=2)
    pos = torch.arange(T, device="cuda") + 3 if rot else None
    y, _ = mb.meteora_head_norm_rotary(x, None, gain, None, pos, r, eps=eps)
    dx, _, dg, _ = mb.meteora_head_norm_rotary_backward(dy, None, x, None, gain, None, pos, r, eps=eps)
    a, g, d = hu.to64(x), hu.to64(gain), hu.to64(dy)
    turn = (lambda v, inv: hu.rotate(v, pos.cpu().numpy(), spec, layout, inverse=inv)) if rot else (lambda v, inv: v)
    pair = (lambda v: hu.pair_size(v, spec, layout)) if rot else np.abs
    rs = 1 / np.sqrt((a * a).mean(-1, keepdims=True) + eps)
    n, dn, mag = a * rs, turn(d, True), pair(d)
    close(y, turn(n * g, False), pair(n * g), dtype, 2.0 ** -18)
    close(dx, rs * (g * dn - n * (g * dn * n).mean(-1, keepdims=True)), rs * (np.abs(g) * mag + np.abs(n) * (np.abs(g) * mag * np.abs(n)).mean(-1, keepdims=True)),
          dtype, 2.0 ** -17)
    bound = (2.0 ** -18 + (T * H + 100) * 2.0 ** -24) * (mag * np.abs(n)).sum((0, 1))
    assert (np.abs(hu.to64(dg) - (dn * n).sum((0, 1))) <= bound).all()
