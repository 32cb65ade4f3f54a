"""Rotary positions, norms of heads with the rotation and their gradients, and the append to a paged cache, against their
definitions in 64 bits.

Bounds, from the arithmetic (u = 2^-24): cos and sin come within two steps of their last place (2^-22) of an angle that is
exact to 2^-24, one product and one FMA follow, so a turned entry is off by less than 2^-21 (|a| + |b|); a norm's sum has
at most 24 additions in a row, which its square root halves, and five more roundings, so a normed and turned entry is off by
less than 2^-18 (|a| + |b|).  bf16 results add half a step of their own, finfo.eps / 2.
"""
import numpy as np
import pytest
import torch

from tests import heads_util as hu
from paper_2405_13053_b200 import binding as mb

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
BANDS = dict(scaling="bands", factor=8.0, original_context=8192.0, low=1.0, high=4.0)


def randn(*shape, dtype=BF16, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, device="cuda", generator=g).to(dtype)


def close(y, ref, size, dtype, ulp=2.0 ** -21):
    y = hu.to64(y)
    tol = ulp * size + (hu.half_step(dtype) * (np.abs(ref) + ulp * size) if dtype == BF16 else 0.0)
    worst = float(np.max(np.abs(y - ref) - tol)) if y.size else 0.0
    assert np.isfinite(y).all() and worst <= 0.0, worst


# T, q heads, kv heads, dim, rot, layout, dtype, scaling, first position
ROTARY = [(1, 32, 8, 128, 128, "half", BF16, {}, 2048), (5, 3, 1, 128, 64, "interleaved", BF16, BANDS, 120000),
          (33, 40, 40, 128, 128, "interleaved", BF16, {}, 0), (7, 12, 4, 80, 40, "half", BF16, {}, 999999),
          (7, 12, 4, 80, 80, "interleaved", BF16, {}, 17), (9, 2, 2, 256, 256, "half", BF16, BANDS, 5),
          (3, 5, 0, 64, 32, "half", BF16, dict(scaling="linear", factor=4.0), 77), (64, 32, 8, 128, 128, "half", F32, {}, 2 ** 31),
          (11, 16, 1, 256, 128, "interleaved", F32, BANDS, 3), (4, 3, 2, 7, 6, "half", F32, {}, 100), (4, 3, 2, 255, 2, "interleaved", BF16, {}, 100),
          (2, 1, 1, 2, 2, "half", BF16, {}, 1), (2, 1, 1, 1, 0, "half", BF16, {}, 1), (1100, 4, 2, 64, 64, "half", BF16, {}, 0)]


@pytest.mark.parametrize("T,H,K,D,rot,layout,dtype,scaling,start", ROTARY)
@pytest.mark.parametrize("inverse", [False, True])
def test_rotary(T, H, K, D, rot, layout, dtype, scaling, start, inverse):
    if rot == 0:
        with pytest.raises(mb.MeteoraError):
            mb.meteora_rotary_init(rot, 10000.0)
        return
    spec = dict(dim=rot, theta=500000.0, **scaling)
    r = mb.meteora_rotary_init(spec["dim"], spec["theta"], layout, attention_scale=1.25, **scaling)
    q, k = randn(T, H, D, dtype=dtype, seed=1), randn(T, K, D, dtype=dtype, seed=2) if K else None
    pos = start + torch.arange(T, device="cuda") * 3
    if start < 2 ** 30 and T % 2:
        pos = (-pos).to(torch.int32)                                 # 32-bit positions, backwards
    yq, yk = mb.meteora_rotary(q, k, pos, r, inverse=inverse)
    for x, y in ((q, yq), (k, yk)):
        if x is None:
            assert y is None
            continue
        x = hu.to64(x)
        ref = hu.rotate(x, pos.cpu().numpy(), spec, layout, 1.25, inverse)
        # the double's own angle is off by 2^-52 of itself, which counts for positions past 2^30
        close(y, ref, 1.25 * hu.pair_size(x, spec, layout) * (1 + 2 ** -10), dtype, 2.0 ** -21 + start * 2.0 ** -51)
        if layout == "half" and rot < D:
            assert np.array_equal(hu.to64(y)[..., rot:], x[..., rot:])


def test_rotary_turns_back_and_runs_in_place():
    r = mb.meteora_rotary_init(128, 10000.0)
    q, k, pos = randn(50, 8, 128, dtype=F32), randn(50, 2, 128, dtype=F32, seed=1), torch.arange(50, device="cuda")
    a, b = mb.meteora_rotary(q, k, pos, r)
    q2, k2 = q.clone(), k.clone()
    same = mb.meteora_rotary(q2, k2, pos, r, out_q=q2, out_k=k2)
    assert torch.equal(q2, a) and torch.equal(k2, b) and same[0].data_ptr() == q2.data_ptr()
    back, _ = mb.meteora_rotary(a, b, pos, r, inverse=True)
    close(back, hu.to64(q), hu.pair_size(hu.to64(q), dict(dim=128)), F32, 2.0 ** -19)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shift", [0, 1, 4])
def test_strided_heads_read_and_write(dtype, shift):
    """q, k, v as slices of one fused product, from bases that allow 16-, 8- and 2- or 4-byte loads."""
    T, H, K, D = 19, 6, 2, 64
    buf = randn(T, (H + 2 * K) * D + shift + 3, dtype=dtype)
    q = buf[:, shift:shift + H * D].unflatten(1, (H, D))
    k = buf[:, shift + H * D:shift + (H + K) * D].unflatten(1, (K, D))
    pos = torch.arange(T, device="cuda")
    r = mb.meteora_rotary_init(D, 10000.0, "interleaved")
    base = mb.meteora_rotary(q.contiguous(), k.contiguous(), pos, r)
    got = mb.meteora_rotary(q, k, pos, r)
    assert torch.equal(got[0], base[0]) and torch.equal(got[1], base[1])
    heads_first = torch.full((H, T, D), 7.0, dtype=dtype, device="cuda")
    mb.meteora_rotary(q, None, pos, r, out_q=heads_first.transpose(0, 1))
    assert torch.equal(heads_first.transpose(0, 1), base[0])
    before = buf.clone()
    mb.meteora_rotary(q, k, pos, r, out_q=q, out_k=k)
    assert torch.equal(q, base[0]) and torch.equal(k, base[1])
    rest = torch.ones(buf.shape[1], dtype=torch.bool)
    rest[shift:shift + (H + K) * D] = False
    assert torch.equal(buf[:, rest.cuda()], before[:, rest.cuda()])


@pytest.mark.parametrize("heads_first", [False, True])
def test_strides_past_31_bits(heads_first):
    """Two tokens (or heads) 2^31 entries apart."""
    n, D, eps = 2, 64, 1e-5
    buf = torch.zeros(2 ** 31 + 2 * D, dtype=BF16, device="cuda")
    near, dy = (randn(n, n, D, dtype=BF16, seed=i) for i in range(2))
    gain = (1 + 0.3 * randn(D, dtype=F32, seed=2)).to(BF16)
    far = torch.as_strided(buf, (n, n, D), (D, 2 ** 31, 1) if heads_first else (2 ** 31, D, 1))
    far.copy_(near)
    pos, r, spec = torch.arange(n, device="cuda") + 7, mb.meteora_rotary_init(D, 10000.0), dict(dim=D, theta=10000.0)
    assert torch.equal(mb.meteora_rotary(far, None, pos, r)[0], mb.meteora_rotary(near, None, pos, r)[0])
    x, g, d, p = hu.to64(near), hu.to64(gain), hu.to64(dy), pos.cpu().numpy()
    rs = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    close(mb.meteora_head_norm_rotary(far, None, gain, None, pos, r, eps=eps)[0], hu.rotate(x * rs * g, p, spec), hu.pair_size(x * rs * g, spec), BF16, 2.0 ** -18)
    dx = mb.meteora_head_norm_rotary_backward(dy, None, far, None, gain, None, pos, r, eps=eps)[0]
    dn, mag, m = hu.rotate(d, p, spec, inverse=True), hu.pair_size(d, spec), x * rs
    close(dx, rs * (g * dn - m * (g * dn * m).mean(-1, keepdims=True)), rs * (np.abs(g) * mag + np.abs(m) * (np.abs(g) * mag * np.abs(m)).mean(-1, keepdims=True)),
          BF16, 2.0 ** -17)
    mb.meteora_rotary(far, None, pos, r, out_q=far)
    assert torch.equal(far, mb.meteora_rotary(near, None, pos, r)[0])
    far.zero_()
    assert not buf.any()                                             # nothing was written beside them


NORM = [(1, 32, 8, 128, 128, "half", BF16), (64, 32, 8, 128, 64, "interleaved", BF16), (5, 12, 4, 80, 40, "half", BF16), (257, 3, 1, 128, 128, "half", F32),
        (3, 40, 40, 256, 256, "interleaved", BF16), (2, 5, 3, 7, 4, "half", F32), (700, 4, 4, 64, 64, "half", BF16), (9, 1, 1, 1, 0, "half", F32),
        (1300, 2, 1, 255, 254, "interleaved", BF16), (130, 7, 0, 128, 0, "half", F32), (0, 4, 2, 64, 64, "half", BF16)]


@pytest.mark.parametrize("T,H,K,D,rot,layout,dtype", NORM)
def test_head_norm_rotary_and_its_gradient(T, H, K, D, rot, layout, dtype):
    eps, theta = 1e-5, 10000.0
    spec = dict(dim=rot, theta=theta)
    r = mb.meteora_rotary_init(rot, theta, layout) if rot else None
    tensors = []
    for heads, seed in ((H, 1), (K, 4)):
        if heads:
            x = randn(T, heads, D, dtype=dtype, seed=seed)
            if T > 1:
                x[1, 0] = 0                                          # a head of zeros: eps alone
                x[0, heads - 1] *= 1000
            tensors.append((x, (1 + 0.3 * randn(D, dtype=F32, seed=seed + 1)).to(dtype), randn(T, heads, D, dtype=dtype, seed=seed + 2)))
    pos = torch.arange(T, device="cuda") + 41
    q, gq, dq = tensors[0]
    k, gk, dk = tensors[1] if K else (None, None, None)
    out = mb.meteora_head_norm_rotary(q, k, gq, gk, pos if rot else None, r, eps=eps)
    back = mb.meteora_head_norm_rotary_backward(dq, dk, q, k, gq, gk, pos if rot else None, r, eps=eps)
    again = mb.meteora_head_norm_rotary_backward(dq, dk, q, k, gq, gk, pos if rot else None, r, eps=eps)
    for a, b in zip(back, again):
        assert a is None or torch.equal(a, b)                        # same order of sums every time
    p = pos.cpu().numpy()
    for i, (x, g, dy) in enumerate(tensors):
        x, g, dy = hu.to64(x), hu.to64(g), hu.to64(dy)
        rs = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        n = x * rs
        turn = (lambda v, inv: hu.rotate(v, p, spec, layout, inverse=inv)) if rot else (lambda v, inv: v)
        size = (lambda v: hu.pair_size(v, spec, layout)) if rot else np.abs
        close(out[i], turn(n * g, False), size(n * g), dtype, 2.0 ** -18)
        dn, mag = turn(dy, True), size(dy)
        mean = (g * dn * n).mean(-1, keepdims=True)
        ref = rs * (g * dn - n * mean)
        close(back[i], ref, rs * (np.abs(g) * mag + np.abs(n) * (np.abs(g) * mag * np.abs(n)).mean(-1, keepdims=True)), dtype, 2.0 ** -17)
        # the gain's sum: every term off by 2^-18 of |dn| |n|, at most all T * heads of them and 100 partial sums in a row
        bound = (2.0 ** -18 + (min(T * x.shape[1], 4096) + 100) * 2.0 ** -24) * (mag * np.abs(n)).sum((0, 1))
        assert (np.abs(hu.to64(back[2 + i]) - (dn * n).sum((0, 1))) <= bound).all()


def test_norm_gradient_against_differences():
    """Directional differences of the forward in fp32: (L(x + h d) - L(x - h d)) / 2h against the gradient's product with d.
    L is O(100) and known to 2^-18 of the sum of its 768 terms, the difference is over 2 h = 2^-5, and the cubic term is
    of the order h^2 times L's third derivative along d, below 1e-3 of the sum of sizes here."""
    T, H, D, eps = 6, 2, 64, 1e-5
    r = mb.meteora_rotary_init(32, 10000.0, "interleaved")
    q, g, dy, d = (randn(T, H, D, dtype=F32, seed=i) for i in range(4))
    g, dg = 1 + 0.2 * g[0, 0], d[0, 1].contiguous()
    pos, h = torch.arange(T, device="cuda"), 2.0 ** -6

    def loss(x, gain):
        y, _ = mb.meteora_head_norm_rotary(x, None, gain.contiguous(), None, pos, r, eps=eps)
        return float((hu.to64(y) * hu.to64(dy)).sum())
    dx, _, dgain, _ = mb.meteora_head_norm_rotary_backward(dy, None, q, None, g, None, pos, r, eps=eps)
    size = float((np.abs(hu.to64(dx)) * np.abs(hu.to64(d))).sum())
    diff = (loss(q + h * d, g) - loss(q - h * d, g)) / (2 * h)
    assert abs(diff - float((hu.to64(dx) * hu.to64(d)).sum())) <= 2e-3 * size
    size = float((np.abs(hu.to64(dgain)) * np.abs(hu.to64(dg))).sum())
    diff = (loss(q, g + h * dg) - loss(q, g - h * dg)) / (2 * h)
    assert abs(diff - float((hu.to64(dgain) * hu.to64(dg)).sum())) <= 2e-3 * size


# B, cu or None, lengths, page, width, prefix_len, H, K, D, rot, layout, dtype, normed, with q
APPEND = [
    (4, None, [0, 15, 16, 31], 16, 3, 2048, 32, 8, 128, 128, "half", BF16, False, True),
    (3, [0, 5, 5, 40], [3, 100, 0], 16, 8, 0, 4, 4, 128, 64, "interleaved", BF16, True, True),
    (3, [2, 9, 30, 33], [1, -1, 60], 24, 3, 100000, 12, 4, 80, 40, "half", BF16, False, True),    # padding; tokens of none
    (2, [0, 70, 71], [0, 7], 64, 1, 5, 16, 1, 64, 64, "half", F32, True, True),                   # past the table's end
    (1, None, [5], 1, 9, 0, 1, 1, 7, 6, "interleaved", F32, False, False),
    (5, None, [0, 1, 2, 3, 4], 128, 1, 17, 2, 2, 256, 256, "half", BF16, True, False),
]


@pytest.mark.parametrize("B,cu,lengths,page,width,prefix,H,K,D,rot,layout,dtype,normed,with_q", APPEND)
def test_cache_append(B, cu, lengths, page, width, prefix, H, K, D, rot, layout, dtype, normed, with_q):
    T = B if cu is None else cu[-1] + 3                              # three tokens behind the last sequence
    n_pages, eps = B * width + 2, 1e-5
    g = np.random.default_rng(5)
    table = g.permutation(n_pages)[:B * width].reshape(B, width).astype(np.int32)
    if width > 2:
        table[-1, 1] = -1                                            # a page that is not there
        table[0, 2] = n_pages
    spec, r = dict(dim=rot, theta=500000.0), mb.meteora_rotary_init(rot, 500000.0, layout)
    q, k, v = randn(T, H, D, dtype=dtype), randn(T, K, D, dtype=dtype, seed=1), randn(T, K, D, dtype=dtype, seed=2)
    v[0, 0, 0] = float("nan")
    gq, gk = ((1 + 0.2 * randn(D, dtype=F32, seed=s)).to(dtype) if normed else None for s in (8, 9))
    kc, vc = randn(n_pages, K, page, D, dtype=dtype, seed=3), randn(n_pages, K, page, D, dtype=dtype, seed=4)
    want_k, want_v = hu.to64(kc), vc.clone()
    out = torch.full((T, H, D), 9.0, dtype=dtype, device="cuda")
    got = mb.meteora_cache_append(k, v, kc, vc, torch.from_numpy(table).cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda"), r,
                                  cu_tokens=None if cu is None else torch.tensor(cu, dtype=torch.int32, device="cuda"), prefix_len=prefix,
                                  q=q if with_q else None, q_gain=gq if with_q else None, k_gain=gk, eps=eps, out_q=out if with_q else None)
    assert (got is None) != with_q
    batch = dict(cu=cu, lengths=lengths)
    place = [hu.places(batch, t) for t in range(T)]
    pos = np.array([0 if p is None else prefix + p[1] for p in place])
    nk = hu.norm(hu.to64(k), hu.to64(gk), eps) if normed else hu.to64(k)
    nq = hu.norm(hu.to64(q), hu.to64(gq), eps) if normed else hu.to64(q)
    ref_k, size_k, size = hu.rotate(nk, pos, spec, layout), hu.pair_size(nk, spec, layout), np.zeros(want_k.shape)
    written = 0
    for t, p in enumerate(place):
        e = None if p is None else hu.page_entry(table[p[0]], p[1], page, n_pages)
        if e is None:
            continue
        want_k[e[0], :, e[1]], size[e[0], :, e[1]] = ref_k[t], size_k[t]
        want_v[e[0], :, e[1]] = v[t]
        written += 1
    assert written > 0
    untouched = np.broadcast_to((size.sum(-1, keepdims=True) == 0), size.shape)
    assert np.array_equal(hu.to64(kc)[untouched], want_k[untouched])
    close(kc, want_k, size, dtype, 2.0 ** -18)
    bits = torch.int16 if dtype == BF16 else torch.int32
    assert torch.equal(vc.view(bits), want_v.view(bits))             # values bit for bit, NaN too
    if with_q:
        mine = np.array([p is not None for p in place])
        ref_q, size_q = hu.rotate(nq, pos, spec, layout), hu.pair_size(nq, spec, layout)
        close(got[torch.from_numpy(mine).cuda()], ref_q[mine], size_q[mine], dtype, 2.0 ** -18)
        assert (got[torch.from_numpy(~mine).cuda()] == 9.0).all()    # rows of no sequence: as they were


def test_append_offsets_past_32_bits():
    """A cache of more than 2^31 entries: the last page's rows are found."""
    page, K, D = 512, 8, 128
    n_pages = 2 ** 31 // (page * K * D) + 2
    kc = torch.zeros(n_pages, K, page, D, dtype=BF16, device="cuda")
    vc = torch.zeros(n_pages, K, page, D, dtype=BF16, device="cuda")
    k, v = randn(1, K, D), randn(1, K, D, seed=1)
    table = torch.tensor([[n_pages - 1]], dtype=torch.int32, device="cuda")
    mb.meteora_cache_append(k, v, kc, vc, table, torch.tensor([511], dtype=torch.int32, device="cuda"), None)
    assert torch.equal(kc[-1, :, 511], k[0]) and torch.equal(vc[-1, :, 511], v[0])
    assert int((kc != 0).sum()) == int((k != 0).sum())


def test_refusals():
    r = mb.meteora_rotary_init(64, 10000.0)
    q, k, pos = randn(4, 2, 64), randn(4, 1, 64), torch.arange(4, device="cuda")
    gain = torch.ones(64, dtype=BF16, device="cuda")
    for bad in (dict(q=q.half()), dict(q=q[:, :, ::2]), dict(q=q[0]), dict(k=k[:3]), dict(k=k.float()), dict(positions=pos[:3]), dict(positions=pos.float()),
                dict(positions=pos.cpu()), dict(q=q.cpu()), dict(rot=b"short"), dict(out_q=q[:, :1].expand(4, 2, 64)), dict(q=randn(4, 2, 32))):
        args = dict(dict(q=q, k=k, positions=pos, rot=r), **bad)
        with pytest.raises((ValueError, TypeError, mb.MeteoraError)):
            mb.meteora_rotary(args["q"], args["k"], args["positions"], args["rot"], out_q=args.get("out_q"))
    with pytest.raises(mb.MeteoraError):
        mb.meteora_head_norm_rotary(q, k, gain, gain, pos, r, eps=-1.0)
    with pytest.raises(ValueError):
        mb.meteora_head_norm_rotary(q, k, gain[:32], gain, pos, r)
    with pytest.raises((TypeError, ValueError)):
        mb.meteora_head_norm_rotary(q, k, gain, None, pos, r)
    with pytest.raises(mb.MeteoraError):
        mb.meteora_head_norm_rotary_backward(q, k, q, k, gain, gain, pos, r, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    cache = randn(4, 1, 16, 64)
    table, lengths = torch.zeros(4, 1, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad in (dict(v=k[:, :, :32]), dict(kc=cache.transpose(1, 2)), dict(vc=cache.float()), dict(table=table.long()), dict(lengths=lengths[:2]),
                dict(cu=lengths), dict(prefix=-1), dict(k=randn(4, 2, 64)), dict(k=randn(3, 1, 64), v=randn(3, 1, 64))):
        a = dict(dict(k=k, v=k, kc=cache, vc=cache.clone(), table=table, lengths=lengths, cu=None, prefix=0), **bad)
        with pytest.raises((ValueError, TypeError, mb.MeteoraError)):
            mb.meteora_cache_append(a["k"], a["v"], a["kc"], a["vc"], a["table"], a["lengths"], r, cu_tokens=a["cu"], prefix_len=a["prefix"])
    with pytest.raises(ValueError):
        mb.meteora_cache_append(k, k, cache, cache.clone(), table, lengths, r, q_gain=gain)


def test_captured_call_follows_its_inputs():
    r = mb.meteora_rotary_init(64, 10000.0)
    q, k, pos = randn(30, 4, 64), randn(30, 2, 64, seed=1), torch.arange(30, device="cuda")
    kc, vc = (torch.zeros(8, 2, 16, 64, dtype=BF16, device="cuda") for _ in range(2))
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4)
    lengths, cu = torch.tensor([0, 3], dtype=torch.int32, device="cuda"), torch.tensor([0, 20, 30], dtype=torch.int32, device="cuda")
    gain = torch.ones(64, dtype=BF16, device="cuda")
    out_q, out_k = torch.empty_like(q), torch.empty_like(k)

    def step():
        mb.meteora_rotary(q, k, pos, r, out_q=out_q, out_k=out_k)
        mb.meteora_cache_append(out_k, k, kc, vc, table, lengths, r, cu_tokens=cu, k_gain=gain)
        return mb.meteora_head_norm_rotary_backward(out_q, out_k, q, k, gain, gain, pos, r)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            back = step()
    torch.cuda.synchronize()
    q.copy_(randn(30, 4, 64, seed=7))
    pos += 1000
    lengths += 5
    kc.zero_()
    vc.zero_()                                                       # (the warm-up wrote at other places)
    graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in (out_q, out_k, kc, vc, *back)]
    kc.zero_()
    vc.zero_()
    want = step()
    for a, b in zip(got, (out_q, out_k, kc, vc, *want)):
        assert torch.equal(a, b)
