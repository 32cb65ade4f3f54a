"""Infinities and NaN in queries, keys and values of attention where the definition has an answer for them: against softmax in 64
bits, which entries are finite.  Each of the kernels: one token (16 rows), a chunk (64), prompts on the tensor cores, fp32."""
import numpy as np
import pytest
import torch

from tests import heads_util as hu
from tests.test_gpu_prefix_attention import BF16, F32, call, check, make

pytestmark = pytest.mark.gpu
SHAPES = {"tokens": dict(B=3, new=[1, 1, 1], held=[40, 3, 70], page=16, H=8, K=2, D=128, dtype=BF16), "chunk": dict(B=2, new=[9, 20], held=[40, 3], page=16, H=8, K=2, D=256, dtype=BF16),
          "prompts": dict(B=2, new=[300, 40], held=[0, 70], page=16, H=4, K=2, D=64, dtype=BF16), "fp32": dict(B=2, new=[3, 1], held=[40, 70], page=16, H=4, K=2, D=64, dtype=F32)}


@pytest.mark.parametrize("name", SHAPES)
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_a_value_that_is_no_number_under_a_weight_next_to_nothing(name, value):
    """An own token's value where the prefix's keys have scores some 400 above: its weight is below 2^-500, and the average with
    it is no finite number all the same."""
    s = make(**SHAPES[name], prefix=100, nan=False)
    s["q"][..., 0] = 16.0
    s["kc"][..., 0] = 0.0
    at = s["prefix_pages"].tolist()
    s["kc"][at, :, :, 0] = 25.0 * s["q"].shape[2] ** 0.5
    clean = call(s)
    bad = dict(s, vc=s["vc"].clone())
    for b in range(len(s["lengths"])):                               # the sequences' first own token
        bad["vc"][int(s["table"][b, 0]), :, 0, 3] = value
    y, lse = call(bad, return_lse=True)
    assert torch.isfinite(lse).all() and torch.isfinite(clean).all()
    assert not torch.isfinite(y[..., 3]).any()
    rest = torch.arange(y.shape[2], device="cuda") != 3
    assert torch.equal(y[..., rest], clean[..., rest])


@pytest.mark.parametrize("name", SHAPES)
@pytest.mark.parametrize("prefix", [0, 100])
def test_scores_that_are_all_minus_infinity(name, prefix):
    """Keys of -inf in one entry under queries above 0 there: softmax over scores of -inf alone is 0 / 0.  Other heads stay, and a row
    whose pages are all gone is still zero."""
    s = make(**SHAPES[name], prefix=prefix, nan=False, seed=2)
    gone, H, K = len(s["lengths"]) - 1, s["q"].shape[1], s["kc"].shape[1]
    s["table"][gone] = -1                                            # the last sequence has its prefix alone
    clean = call(s)
    bad = dict(s, kc=s["kc"].clone(), q=s["q"].clone())
    bad["q"][:, :H // K, 5] = 0.5
    bad["kc"][:, 0, :, 5] = float("-inf")
    y, lse = call(bad, return_lse=True)
    assert torch.equal(y[:, H // K:], clean[:, H // K:]) and torch.isfinite(lse[:, H // K:]).all() == (prefix > 0)
    seen = torch.tensor([prefix > 0 or hu.places(dict(cu=None if s["cu"] is None else s["cu"].tolist(), lengths=s["lengths"].tolist()), t)[0] != gone
                         for t in range(y.shape[0])], device="cuda")
    assert torch.isnan(y[seen, :H // K]).all() and (y[~seen] == 0).all() and (lse[:, :H // K] == -float("inf")).all()
    part = dict(bad, kc=bad["kc"].clone())                           # one key of the first sequence with a score of its own
    part["kc"][int(s["table"][0, 0]), 0, 0] = 0.0
    y = call(part)
    v = s["vc"][int(s["table"][0, 0]), 0, 0]
    first = int(s["cu"][1]) if s["cu"] is not None else 1
    assert torch.equal(y[:first, :H // K], v.expand(first, H // K, -1))


@pytest.mark.parametrize("name", SHAPES)
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("prefix", [0, 200])
def test_no_numbers_under_a_scale_of_zero(name, value, prefix):
    """scale = 0 makes every score 0 and the row an average of what it sees; a query or a key that is no finite number makes its
    scores NaN, 0 times it, and the rows with it."""
    s = make(**SHAPES[name], prefix=prefix, nan=False, seed=3)
    clean, lse = call(s, scale=0.0, return_lse=True)
    check(s, clean, lse, scale=0.0)
    t, h, H, K = s["q"].shape[0] - 1, 1, s["q"].shape[1], s["kc"].shape[1]
    bad = dict(s, q=s["q"].clone())
    bad["q"][t, h, 9] = value
    y = call(bad, scale=0.0)
    hit = torch.zeros(y.shape[:2], dtype=torch.bool, device="cuda")
    hit[t, h] = True
    assert torch.isnan(y[hit]).all() and torch.equal(y[~hit], clean[~hit])
    bad = dict(s, kc=s["kc"].clone())
    bad["kc"][int(s["table"][0, 0]), 0, 0, 9] = value                # seen by the first sequence, through one kv head
    y = call(bad, scale=0.0)
    hit[:] = False
    hit[:int(s["cu"][1]), :H // K] = True
    assert torch.isnan(y[hit]).all() and torch.equal(y[~hit], clean[~hit])
