"""Token counts next to 2^31 at the C entry points of the operators on heads: refused on the host (every call here returns there)."""
import ctypes

import pytest

from paper_2405_13053_b200 import binding as mb
from paper_2405_13053_b200 import build
from tests.test_heads_cpu import UNSUPPORTED, cache, heads

MOST = 2 ** 31 - 4096                                                # the first count that is too large


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return mb.load_library()


@pytest.mark.parametrize("T", [MOST, 2 ** 31 - 600, 2 ** 31 - 1])
def test_more_tokens_than_indexes_hold(lib, T):
    """The launches' rounding up of a token count would wrap."""
    rot = ctypes.byref(mb.meteora_rotary_init(2))
    one = heads(st=2, sh=2, n=1)
    assert lib.meteora_rotary(one, None, one, None, 4096, 1, T, 2, 1, rot, 0, None) == UNSUPPORTED
    assert lib.meteora_head_norm_rotary(one, None, 4096, None, one, None, 4096, 1, T, 2, 1, rot, 1e-5, None) == UNSUPPORTED
    assert lib.meteora_head_norm_rotary_backward_workspace_bytes(T, 1, 0, 2) == 0
    assert lib.meteora_head_norm_rotary_backward_workspace_bytes(MOST - 1, 1, 0, 2) > 0
    assert lib.meteora_head_norm_rotary_backward(one, None, one, None, 4096, None, one, None, 4096, None, 4096, 1, T, 2, 1, rot, 1e-5, 4096, 1 << 30,
                                                 None) == UNSUPPORTED
    batch = ctypes.byref(mb.MeteoraBatch(1, T, 4096, 4096, 4096, 4, 0, None))
    assert lib.meteora_cache_append(one, one, None, None, None, None, 1e-5, rot, cache(kv=1, D=2), batch, None) == UNSUPPORTED
    assert lib.meteora_prefix_attention(one, cache(kv=1, D=2), batch, 0.1, one, None, 4096, 1 << 40, None) == UNSUPPORTED
