"""The operators on heads without a GPU: the frequencies of rotary embeddings and what the C entry points refuse before any
launch (every call here returns on the host)."""
import ctypes
from fractions import Fraction

import numpy as np
import pytest

from paper_2405_13053_b200 import binding as mb
from paper_2405_13053_b200 import build
from tests import heads_util as hu

INVALID, UNSUPPORTED, MISALIGNED, SMALL = -1, -2, -3, -4


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return mb.load_library()


@pytest.mark.parametrize("dim,theta,scaling", [(128, 500000.0, {}), (2, 10000.0, {}), (256, 1e6, dict(scaling="linear", factor=4.0)),
                                               (64, 10000.0, dict(scaling="bands", factor=8.0, original_context=8192.0, low=1.0, high=4.0)),
                                               (8, 0.01, {})])
def test_frequencies_as_fractions_of_a_turn(lib, dim, theta, scaling):
    """turns[i] / 2^64 is f_i / (2 pi) modulo 1, to the double's own 2^-52 of f_i (frequencies above a turn lose whole turns)."""
    rot = mb.meteora_rotary_init(dim, theta, **scaling)
    f = hu.frequencies(dim, theta, **scaling)
    for i in range(dim // 2):
        want = f[i] / (2 * np.pi)
        got = float(Fraction(rot.turns[i], 2 ** 64))
        diff = abs((want - got + 0.5) % 1.0 - 0.5)
        assert diff <= 2.0 ** -50 * max(want, 1e-300) + 2.0 ** -64
    assert all(rot.turns[i] == 0 for i in range(dim // 2, 128)) and rot.dim == dim and rot.scale == 1.0


def test_rotary_init_refuses(lib):
    for bad in (dict(dim=0), dict(dim=3), dict(dim=258), dict(theta=0.0), dict(theta=float("inf")), dict(theta=float("nan")), dict(attention_scale=float("inf")),
                dict(scaling="linear", factor=0.0), dict(scaling="bands", factor=8.0), dict(scaling="bands", factor=8.0, original_context=8192.0, low=4.0, high=4.0)):
        with pytest.raises(mb.MeteoraError):
            mb.meteora_rotary_init(**dict(dict(dim=64, theta=10000.0), **bad))
    for bad in (dict(layout="quarter"), dict(scaling="cubic")):
        with pytest.raises(ValueError):
            mb.meteora_rotary_init(64, **bad)
    assert lib.meteora_rotary_init(None, None) == INVALID


def heads(data=4096, st=512, sh=64, n=4):
    return ctypes.byref(mb.MeteoraHeads(data, st, sh, n))


def test_rotary_and_norm_refuse(lib):
    rot = mb.meteora_rotary_init(64)
    ok = dict(q=heads(), k=heads(n=2), qo=heads(), ko=heads(n=2), pos=4096, p64=1, T=8, D=64, dt=1, rot=ctypes.byref(rot), inv=0)

    def rotary(**kw):
        a = dict(ok, **kw)
        return lib.meteora_rotary(a["q"], a["k"], a["qo"], a["ko"], a["pos"], a["p64"], a["T"], a["D"], a["dt"], a["rot"], a["inv"], None)

    def norm(**kw):
        a = dict(ok, gq=4096, gk=4096, eps=1e-5, **kw) if not {"gq", "gk", "eps"} & set(kw) else dict(dict(ok, gq=4096, gk=4096, eps=1e-5), **kw)
        return lib.meteora_head_norm_rotary(a["q"], a["k"], a["gq"], a["gk"], a["qo"], a["ko"], a["pos"], a["p64"], a["T"], a["D"], a["dt"], a["rot"],
                                            a["eps"], None)
    narrow = mb.meteora_rotary_init(66)
    broken = mb.meteora_rotary_init(64)
    broken.layout = 5
    for f in (rotary, norm):
        assert f(T=0) == 0                                           # no tokens: nothing to do
        assert f(T=-1) == INVALID and f(D=0) == INVALID and f(D=257) == UNSUPPORTED and f(dt=2) == INVALID
        assert f(q=None) == INVALID and f(qo=None) == INVALID and f(ko=None) == INVALID and f(k=None) == INVALID
        assert f(q=heads(data=None)) == INVALID and f(qo=heads(data=None)) == INVALID and f(pos=None) == INVALID
        assert f(q=heads(data=4097)) == MISALIGNED and f(pos=4100) == MISALIGNED
        assert f(qo=heads(n=3)) == INVALID and f(q=heads(n=0)) == INVALID and f(q=heads(st=-1)) == INVALID
        assert f(qo=heads(st=0)) == INVALID and f(qo=heads(sh=63)) == INVALID and f(qo=heads(st=255)) == INVALID     # entries that coincide
        assert f(rot=ctypes.byref(narrow)) == INVALID and f(rot=ctypes.byref(broken)) == INVALID
    assert rotary(rot=None) == INVALID
    assert norm(eps=-1.0) == INVALID and norm(eps=float("nan")) == INVALID and norm(gq=None) == INVALID and norm(gk=None) == INVALID and norm(gq=4097) == MISALIGNED


def test_norm_gradient_refuses(lib):
    rot = mb.meteora_rotary_init(64)
    size = lib.meteora_head_norm_rotary_backward_workspace_bytes
    need = size(8, 4, 2, 64)
    assert need > 0 and size(-1, 4, 2, 64) == 0 and size(8, 0, 2, 64) == 0 and size(8, 4, 2, 257) == 0 and size(0, 4, 0, 64) > 0

    def grad(dy=heads(), dyk=heads(n=2), q=heads(), k=heads(n=2), gq=4096, gk=4096, dx=heads(), dxk=heads(n=2), dgq=4096, dgk=4096, pos=4096, T=8, eps=1e-5, ws=4096,
             n=need):
        return lib.meteora_head_norm_rotary_backward(dy, dyk, q, k, gq, gk, dx, dxk, dgq, dgk, pos, 1, T, 64, 1, ctypes.byref(rot), eps, ws, n, None)
    assert grad(n=need - 1) == SMALL and grad(ws=None) == INVALID and grad(ws=4104) == MISALIGNED
    assert grad(dyk=None) == INVALID and grad(dgk=None) == INVALID and grad(gq=None) == INVALID and grad(dgq=None) == INVALID and grad(pos=None) == INVALID
    assert grad(dx=heads(st=100)) == INVALID and grad(dy=heads(n=5)) == INVALID and grad(T=-1) == INVALID and grad(eps=-1.0) == INVALID


def cache(k=4096, v=4096, n=10, kv=2, page=16, D=64, dt=1):
    return ctypes.byref(mb.MeteoraCache(k, v, n, kv, page, D, dt))


def batch(B=8, T=8, cu=None, lengths=4096, table=4096, width=4, prefix=0, pages=None):
    return ctypes.byref(mb.MeteoraBatch(B, T, cu, lengths, table, width, prefix, pages))


def test_append_and_attention_refuse(lib):
    rot = mb.meteora_rotary_init(64)

    def append(k=heads(n=2), v=heads(n=2), q=None, qo=None, gq=None, gk=None, eps=1e-5, r=rot, c=cache(), b=batch()):
        return lib.meteora_cache_append(k, v, q, qo, gq, gk, eps, ctypes.byref(r) if r else None, c, b, None)
    size = lib.meteora_prefix_attention_workspace_bytes

    def attend(q=heads(), c=cache(), b=batch(), scale=0.1, out=heads(), lse=None, ws=4096, n=1 << 30):
        return lib.meteora_prefix_attention(q, c, b, scale, out, lse, ws, n, None)
    for f in (append, attend):
        assert f(c=None) == INVALID and f(b=None) == INVALID
        assert f(c=cache(n=-1)) == INVALID and f(c=cache(page=0)) == INVALID and f(c=cache(D=0)) == INVALID and f(c=cache(dt=7)) == INVALID
        assert f(c=cache(k=None)) == INVALID and f(c=cache(k=4104)) == MISALIGNED and f(c=cache(D=257)) == UNSUPPORTED and f(c=cache(n=1 << 31)) == UNSUPPORTED
        assert f(b=batch(B=-1)) == INVALID and f(b=batch(T=7)) == INVALID and f(b=batch(width=-1)) == INVALID and f(b=batch(prefix=-1)) == INVALID
        assert f(b=batch(lengths=None)) == INVALID and f(b=batch(table=None)) == INVALID and f(b=batch(lengths=4098)) == MISALIGNED
        assert f(b=batch(B=4097, T=4097)) == UNSUPPORTED
        assert f(b=batch(B=0, T=0)) == 0
    assert append(k=heads(n=3)) == INVALID and append(v=None) == INVALID and append(q=heads()) == INVALID and append(gq=4096) == INVALID
    assert append(q=heads(), qo=heads(n=3)) == INVALID and append(eps=-1.0) == INVALID and append(gk=4097) == MISALIGNED
    assert attend(q=None) == INVALID and attend(out=None) == INVALID and attend(q=heads(n=3), out=heads(n=3)) == INVALID and attend(out=heads(n=6)) == INVALID
    assert attend(scale=float("inf")) == INVALID and attend(ws=None) == INVALID and attend(ws=4104) == MISALIGNED and attend(lse=4097) == MISALIGNED
    assert attend(b=batch(prefix=5)) == INVALID and attend(out=heads(st=0)) == INVALID
    need = size(cache(), batch(prefix=5, pages=4096), 4)
    assert need > 4096 and attend(b=batch(prefix=5, pages=4096), n=need - 1) == SMALL
    assert size(cache(), batch(B=0, T=0, width=0), 4) >= 4096 and size(cache(), batch(T=0, cu=4096, prefix=9), 4) >= 4096   # (T = 0: sizes only)
    assert size(cache(), batch(), 3) == 0 and size(None, batch(), 4) == 0 and size(cache(), batch(width=1 << 26), 4) == 0
    assert attend(b=batch(width=1 << 26)) == UNSUPPORTED and attend(b=batch(prefix=1 << 29, pages=4096)) == UNSUPPORTED
