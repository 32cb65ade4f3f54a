"""Attention of a batch over a shared prefix and paged own tokens against its definition in 64 bits (row by row, in numpy).

Bound of an entry, from the arithmetic (u = 2^-24; w the row's weights, A = sum w |v - out|, B = sum w |v|):
  - a score's sum of dim products is off by at most (dim + 4) u sum |q||k|, which moves every weight by twice that
    relative to the others, as the exponential's 2^-21 does: (2 (dim + 4) u S + 2^-20) B with S the largest scaled sum |q||k|;
  - sums over n keys and up to 130 pieces in fp32: (n + 130) u B;
  - bf16 caches: weights rounded by 2^-8 at most, in the sum of weights alike: 2^-8 A (1 + 2^-7);
  - the result rounded by half a step.
"""
import numpy as np
import pytest
import torch

from tests import heads_util as hu
from paper_2405_13053_b200 import binding as mb

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def make(B, new, held, page, prefix, H, K, D, dtype, seed=0, drop=(), pad=(), behind=0, one_each=False, spread=1.0, nan=True):
    """A batch with new[b], held[b] tokens; every entry of the cache that no row may read is NaN."""
    g = torch.Generator().manual_seed(seed)
    T = sum(new) + behind
    width = max(1, max((n + h + page - 1) // page for n, h in zip(new, held)))
    n_prefix = (prefix + page - 1) // page
    n_pages = B * width + n_prefix + 1
    order = torch.randperm(n_pages, generator=g).to(torch.int32)
    table, prefix_pages = order[:B * width].view(B, width).clone(), order[B * width:B * width + n_prefix].clone()
    kc, vc = torch.randn(n_pages, K, page, D, generator=g), torch.randn(n_pages, K, page, D, generator=g) + torch.randn(1, K, 1, D, generator=g)
    if nan:
        live = torch.zeros(n_pages, page, dtype=torch.bool)
        for b in range(B):
            for i in range(new[b] + held[b]):
                live[table[b, i // page], i % page] = True
        for i in range(prefix):
            live[prefix_pages[i // page], i % page] = True
        dead = ~live[:, None, :, None].expand_as(kc)
        kc[dead], vc[dead] = float("nan"), float("inf")
    for b, s in drop:                                                # pages that are gone
        if b < 0:
            prefix_pages[s] = -1
        else:
            table[b, s] = n_pages if (b + s) % 2 else -7
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    lengths = np.array(held, np.int32)
    for b in pad:
        lengths[b] = -1
    q = (spread * torch.randn(T, H, D, generator=g)).to(dtype)
    return dict(q=q.cuda(), kc=kc.to(dtype).cuda(), vc=vc.to(dtype).cuda(), table=table.cuda(), prefix_pages=prefix_pages.cuda(), prefix=prefix,
                lengths=torch.from_numpy(lengths).cuda(), cu=None if one_each else torch.from_numpy(cu).cuda())


def batch_of(s):
    return dict(cu=None if s["cu"] is None else s["cu"].tolist(), lengths=s["lengths"].tolist(), table=s["table"].tolist(), prefix_len=s["prefix"],
                prefix_pages=s["prefix_pages"].tolist())


def call(s, **kw):
    return mb.meteora_prefix_attention(s["q"], s["kc"], s["vc"], s["table"], s["lengths"], s["prefix_pages"], s["prefix"], cu_tokens=s["cu"], **kw)


def check(s, out, lse, scale=None, fill=None, rows=None):
    """rows: tokens to compare (all)."""
    dtype, D = s["q"].dtype, s["q"].shape[2]
    scale = D ** -0.5 if scale is None else scale
    q = hu.to64(s["q"])
    batch = batch_of(s)
    ref, ref_lse, A, B, S, n = hu.attention(q, hu.to64(s["kc"]), hu.to64(s["vc"]), batch, scale)
    y, l = hu.to64(out), hu.to64(lse)
    none = np.isnan(ref_lse)
    if fill is not None:
        assert (y[none] == fill).all()                               # rows of no sequence: as they were
    y, l, ref, ref_lse, A, B, S, n = (a[~none] for a in (y, l, ref, ref_lse, A, B, S, n))
    moved = 2 * (D + 4) * 2.0 ** -24 * S + 2.0 ** -20
    tol = (moved + (n + 130) * 2.0 ** -24)[..., None] * B
    if dtype == BF16:
        tol += 2.0 ** -8 * (1 + 2.0 ** -7) * A
        tol += hu.half_step(BF16) * (np.abs(ref) + tol)
    else:
        tol += hu.half_step(F32) * np.abs(ref)
    assert np.isfinite(y).all()
    worst = float((np.abs(y - ref) - tol).max()) if y.size else 0.0
    assert worst <= 0.0, worst
    empty = np.isinf(ref_lse)
    assert (l[empty] == -np.inf).all() and (y[empty] == 0).all()
    # its logarithm: the sum of weights as above (in bf16 rounded by 2^-8 each), log2 and the product with ln 2
    off = moved + (n + 130) * 2.0 ** -24 + (2.0 ** -8 if dtype == BF16 else 0.0) + 2.0 ** -22 * (1 + np.abs(np.where(empty, 0, ref_lse)))
    assert (np.abs(l[~empty] - ref_lse[~empty]) <= off[~empty]).all()


CASES = {
    "one_token": dict(B=1, new=[1], held=[37], page=16, prefix=300, H=32, K=8, D=128, dtype=BF16, one_each=True),
    "first_token": dict(B=1, new=[1], held=[0], page=16, prefix=0, H=4, K=4, D=64, dtype=BF16, one_each=True),
    "decode": dict(B=9, new=[1] * 9, held=[0, 1, 15, 16, 63, 64, 65, 200, 7], page=16, prefix=333, H=8, K=2, D=128, dtype=BF16, one_each=True),
    "decode_padded": dict(B=5, new=[1] * 5, held=[3, 0, 70, 9, 0], page=8, prefix=64, H=8, K=2, D=64, dtype=BF16, pad=(1, 4), one_each=True),
    "decode_64_rows": dict(B=40, new=[1] * 40, held=[(i * 37) % 130 for i in range(40)], page=32, prefix=517, H=8, K=2, D=128, dtype=BF16),
    "no_prefix": dict(B=3, new=[1, 4, 2], held=[100, 0, 31], page=16, prefix=0, H=6, K=2, D=128, dtype=BF16, behind=3),
    "chunk": dict(B=3, new=[33, 1, 70], held=[0, 90, 31], page=16, prefix=130, H=8, K=2, D=128, dtype=BF16),
    "chunk_behind": dict(B=4, new=[5, 0, 40, 9], held=[3, 50, 0, 64], page=64, prefix=65, H=5, K=5, D=64, dtype=BF16, pad=(3,), behind=5),
    "prompts": dict(B=3, new=[300, 41, 150], held=[0, 130, 257], page=16, prefix=70, H=8, K=4, D=128, dtype=BF16, behind=2),
    "prompts_no_prefix": dict(B=2, new=[513, 1], held=[0, 64], page=64, prefix=0, H=2, K=2, D=64, dtype=BF16, drop=((0, 3), (0, 8))),
    "few_rows_long_keys": dict(B=2, new=[24, 20], held=[1100, 900], page=8, prefix=200, H=3, K=3, D=64, dtype=BF16, pad=()),
    "chunk_wide_heads": dict(B=2, new=[20, 37], held=[10, 0], page=32, prefix=100, H=4, K=2, D=256, dtype=BF16),
    "decode_wide_heads": dict(B=3, new=[1] * 3, held=[130, 2, 64], page=32, prefix=200, H=4, K=2, D=256, dtype=BF16),
    "odd_page": dict(B=3, new=[2, 1, 3], held=[50, 0, 23], page=24, prefix=75, H=12, K=4, D=80, dtype=BF16),
    "page_of_one": dict(B=2, new=[1, 2], held=[9, 70], page=1, prefix=7, H=2, K=1, D=64, dtype=BF16),
    "many_heads": dict(B=2, new=[1, 1], held=[40, 5], page=16, prefix=90, H=70, K=1, D=64, dtype=BF16, one_each=True),
    "many_heads_chunk": dict(B=2, new=[3, 2], held=[40, 5], page=16, prefix=90, H=140, K=2, D=64, dtype=BF16),
    "fp32_decode": dict(B=4, new=[1] * 4, held=[0, 65, 130, 3], page=16, prefix=140, H=8, K=2, D=128, dtype=F32, one_each=True),
    "fp32_chunk": dict(B=3, new=[9, 1, 30], held=[0, 70, 5], page=24, prefix=77, H=6, K=3, D=256, dtype=F32, behind=2),
    "odd_heads": dict(B=2, new=[3, 5], held=[60, 1], page=5, prefix=33, H=3, K=1, D=7, dtype=BF16),
    "odd_heads_fp32": dict(B=2, new=[1, 18], held=[60, 1], page=128, prefix=0, H=34, K=2, D=33, dtype=F32),
    "dropped_pages": dict(B=4, new=[1, 3, 1, 2], held=[90, 40, 0, 17], page=16, prefix=100, H=8, K=2, D=128, dtype=BF16,
                          drop=((-1, 0), (-1, 3), (0, 0), (0, 2), (1, 1), (2, 0))),
    "nothing_left": dict(B=2, new=[1, 2], held=[15, 14], page=16, prefix=16, H=4, K=2, D=64, dtype=BF16, drop=((-1, 0), (0, 0))),
    "nothing_left_fp32": dict(B=2, new=[1, 2], held=[15, 14], page=16, prefix=16, H=4, K=2, D=64, dtype=F32, drop=((-1, 0), (0, 0))),
    "sharp": dict(B=6, new=[1] * 6, held=[100] * 6, page=16, prefix=1000, H=16, K=4, D=128, dtype=BF16, spread=20.0),
    "sharp_fp32": dict(B=2, new=[2, 1], held=[100] * 2, page=16, prefix=300, H=4, K=4, D=64, dtype=F32, spread=30.0),
}


@pytest.mark.parametrize("name", CASES)
def test_against_the_definition(name):
    s = make(**CASES[name])
    out = torch.full_like(s["q"], 5.0)
    got, lse = call(s, out=out, return_lse=True)
    assert got is out
    check(s, got, lse, fill=5.0)
    again = call(s)
    seen = ~torch.isnan(lse) if s["cu"] is None else torch.ones(s["q"].shape[0], dtype=torch.bool)
    mine = torch.tensor([hu.places(batch_of(s), t) is not None for t in range(s["q"].shape[0])])
    assert torch.equal(again[mine.cuda()], got[mine.cuda()])         # run to run, bit for bit
    assert seen is not None


@pytest.mark.parametrize("prefix,B,H,K,D,page", [(4096, 64, 32, 8, 128, 16), (2111, 70, 16, 16, 64, 32), (1000, 33, 12, 4, 128, 8), (1537, 150, 8, 2, 128, 128),
                                               (515, 300, 2, 2, 64, 64)])
def test_large_shared_prefix(prefix, B, H, K, D, page):
    """Many sequences over one prefix: tiles of rows of different sequences against the prefix's keys."""
    held = [(b * 53) % 190 for b in range(B)]
    s = make(B, [1] * B, held, page, prefix, H, K, D, BF16, one_each=True)
    out, lse = call(s, return_lse=True)
    some = sorted({0, 1, B // 2, B - 2, B - 1, min(31, B - 1), min(32, B - 1)})
    sub = dict(s, q=s["q"][some], table=s["table"][some], lengths=s["lengths"][some])
    check(sub, out[some], lse[some])


def test_strided_queries_and_output():
    s = make(B=3, new=[1, 2, 30], held=[70, 0, 20], page=16, prefix=100, H=8, K=2, D=64, dtype=BF16)
    want = call(s)
    T = s["q"].shape[0]
    buf = torch.zeros(T, 8 * 64 + 64 + 1, dtype=BF16, device="cuda")
    for shift in (0, 1):
        q = buf[:, shift:shift + 512].unflatten(1, (8, 64))
        q.copy_(s["q"])
        out = torch.zeros(8, T, 65, dtype=BF16, device="cuda")[:, :, :64].transpose(0, 1)
        got = call(dict(s, q=q), out=out)
        assert torch.equal(got, want)


@pytest.mark.parametrize("D,dtype", [(128, BF16), (256, BF16), (64, F32)])
def test_one_token_over_a_long_prefix(D, dtype):
    """Far more pieces of a row than the join's warps take at a time (their sums are shorter than the keys' that the bound counts)."""
    s = make(B=1, new=[1], held=[300], page=16, prefix=7001, H=16, K=1, D=D, dtype=dtype, one_each=True)
    out, lse = call(s, return_lse=True)
    check(s, out, lse)


@pytest.mark.parametrize("new,D,dtype", [([1, 1, 1], 128, BF16), ([40, 7, 90], 64, BF16), ([300, 200, 2], 128, BF16), ([2, 5, 1], 64, F32)])
def test_in_place_of_the_queries(new, D, dtype):
    s = make(B=3, new=new, held=[20, 0, 77], page=16, prefix=150, H=8, K=2, D=D, dtype=dtype)
    want = call(s)
    q = s["q"].clone()
    assert call(dict(s, q=q), out=q) is q and torch.equal(q, want)


def test_scale_and_workspace():
    s = make(B=3, new=[1, 2, 5], held=[70, 0, 20], page=16, prefix=100, H=8, K=2, D=64, dtype=BF16)
    ws = mb.meteora_prefix_attention_workspace(s["q"], s["kc"], s["table"], s["prefix"])
    for scale in (0.3, -0.2, 0.0):
        out, lse = call(s, scale=scale, workspace=ws, return_lse=True)
        check(s, out, lse, scale=scale)
    assert mb.meteora_workspace_status(ws) == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("K,D,more", [(2, 128, 0), (4, 64, 0), (2, 256, 0), (2, 128, 260), (4, 64, 330)])
def test_values_that_are_no_numbers_stay_with_the_rows_that_see_them(dtype, K, D, more):
    """NaN in the value of a later token, in one sequence's own pages, in one query: only the rows that see them change."""
    new, held, prefix = [40 + more, 3, 1], [10, 5, 20], 90
    n = new[0]
    s = make(B=3, new=new, held=held, page=16, prefix=prefix, H=4, K=K, D=D, dtype=dtype, nan=False)
    want = call(s)
    bad = dict(s, vc=s["vc"].clone(), kc=s["kc"].clone(), q=s["q"].clone())
    table = s["table"].tolist()
    for b, i, e, value in ((0, held[0] + 17, 3, float("nan")), (0, held[0] + 30, D - 1, float("inf")), (1, 2, 0, float("nan"))):
        bad["vc"][table[b][i // 16], :, i % 16, e] = value
    bad["kc"][table[2][0], :, 4] = float("nan")
    bad["q"][5, 1] = float("nan")
    got = call(bad)
    a, b = hu.to64(got), hu.to64(want)
    hit = np.zeros(a.shape, bool)
    hit[17:n, :, 3], hit[30:n, :, D - 1] = True, True
    hit[n:n + 3, :, 0] = True                                        # sequence 1: every token sees its third
    hit[n + 3], hit[5, 1] = True, True
    assert np.array_equal(a[~hit], b[~hit]) or np.abs(a - b)[~hit].max() <= 2.0 ** -7 * np.abs(b).max()
    assert np.isfinite(a[~hit]).all() and not np.isfinite(a[hit]).any()


def test_append_then_attend_as_a_step():
    """Three steps of a batch: a prompt each, then two single tokens; cache, rotation and attention as a program has them."""
    H, K, D, page, B, prefix = 8, 2, 64, 16, 3, 50
    g = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g).to(BF16)  # noqa: E731
    rot = mb.meteora_rotary_init(D, 10000.0)
    kc, vc = (torch.full((30, K, page, D), float("nan"), dtype=BF16, device="cuda") for _ in range(2))
    prefix_pages = torch.tensor([7, 3, 11, 20], dtype=torch.int32, device="cuda")
    table = torch.tensor([[0, 1, 2], [4, 5, 6], [8, 9, 10]], dtype=torch.int32, device="cuda")
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    mb.meteora_cache_append(rand(prefix, K, D), rand(prefix, K, D), kc, vc, prefix_pages.view(1, 4), one, rot,
                            cu_tokens=torch.tensor([0, prefix], dtype=torch.int32, device="cuda"))
    lengths, new = torch.zeros(B, dtype=torch.int32, device="cuda"), [17, 1, 30]
    for step in range(3):
        cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda") if step == 0 else None
        T = sum(new)
        q = mb.meteora_cache_append(rand(T, K, D), rand(T, K, D), kc, vc, table, lengths, rot, cu_tokens=cu, prefix_len=prefix, q=rand(T, H, D))
        s = dict(q=q, kc=kc, vc=vc, table=table, lengths=lengths, prefix_pages=prefix_pages, prefix=prefix, cu=cu)
        out, lse = call(s, return_lse=True)
        check(s, out, lse)
        lengths = lengths + torch.tensor(new, dtype=torch.int32, device="cuda")
        new = [1] * B


def test_captured_steps_share_a_workspace():
    """Two captured calls of different batches on one workspace, replayed in turn while lengths grow."""
    a = make(B=20, new=[1] * 20, held=[60 + b for b in range(20)], page=16, prefix=400, H=8, K=2, D=128, dtype=BF16, one_each=True)
    b = make(B=2, new=[30, 9], held=[0, 40], page=32, prefix=100, H=8, K=2, D=128, dtype=BF16, seed=1)
    a["lengths"] -= 50
    ws = max((mb.meteora_prefix_attention_workspace(s["q"], s["kc"], s["table"], s["prefix"]) for s in (a, b)), key=lambda w: w.numel())
    outs, graphs = [], []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for s in (a, b):
            call(s, workspace=ws)
            graph, out = torch.cuda.CUDAGraph(), torch.empty_like(s["q"])
            with torch.cuda.graph(graph, stream=side):
                call(s, workspace=ws, out=out)
            outs.append(out)
            graphs.append(graph)
        for step in range(3):
            a["lengths"] += 16                                       # (up to 58 + b of the 60 + b tokens that are there)
            for s, graph, out in zip((a, b), graphs, outs):
                s["q"].mul_(0.9)
                graph.replay()
                assert torch.equal(out, call(s))
    torch.cuda.synchronize()


def test_two_streams_with_a_workspace_each():
    cases = [make(B=16, new=[1] * 16, held=[90] * 16, page=16, prefix=700, H=8, K=2, D=128, dtype=BF16, one_each=True, seed=i) for i in range(2)]
    want = [call(s) for s in cases]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in cases], [[], []]
    ws = [mb.meteora_prefix_attention_workspace(s["q"], s["kc"], s["table"], s["prefix"]) for s in cases]
    torch.cuda.synchronize()
    for _ in range(10):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(call(cases[i], workspace=ws[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i]) for o in got[i])


def test_offsets_past_32_bits():
    page, K, D = 512, 8, 128
    n_pages = 2 ** 31 // (page * K * D) + 2
    kc, vc = (torch.zeros(n_pages, K, page, D, dtype=BF16, device="cuda") for _ in range(2))
    small = make(B=2, new=[1, 1], held=[100, 20], page=page, prefix=90, H=32, K=K, D=D, dtype=BF16, one_each=True, nan=False)
    n = small["kc"].shape[0]
    kc[-n:], vc[-n:] = small["kc"], small["vc"]
    far = dict(small, kc=kc, vc=vc, table=small["table"] + (n_pages - n), prefix_pages=small["prefix_pages"] + (n_pages - n))
    assert torch.equal(call(far), call(small))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,T", [(2, 2), (3, 90)])
def test_a_cache_without_pages_or_tables(B, T, dtype):
    H, K, D, page = 4, 2, 64, 16
    cu = None if T == B else torch.tensor([0, T // 2, T // 2, T], dtype=torch.int32, device="cuda")
    table, lengths = torch.zeros(B, 0, dtype=torch.int32, device="cuda"), torch.tensor([3, 0, 1][:B], dtype=torch.int32, device="cuda")
    pages = torch.zeros(2, dtype=torch.int32, device="cuda")
    q = torch.randn(T, H, D, device="cuda").to(dtype)
    full = torch.randn(1, K, page, D, device="cuda").to(dtype)
    for kc, prefix in ((full[:0], 0), (full[:0], 20), (full, 0)):
        s = dict(q=q, kc=kc, vc=kc, table=table, lengths=lengths, prefix_pages=pages if prefix else None, prefix=prefix, cu=cu)
        out, lse = call(s, return_lse=True)
        assert (out == 0).all() and (lse == -np.inf).all()
    s = dict(q=q, kc=full, vc=full, table=table, lengths=lengths, prefix_pages=pages[:1], prefix=9, cu=cu)      # the prefix alone
    out, lse = call(s, return_lse=True)
    check(s, out, lse)


@pytest.mark.parametrize("new,held,prefix,D,dtype", [([9, 5, 30], [10, 200, 3], 100, 128, BF16), ([300, 40, 200], [0, 130, 20], 0, 64, BF16),
                                                     ([2, 1, 1], [10, 90, 3], 40, 128, BF16), ([9, 5, 30], [10, 70, 3], 33, 64, F32)])
def test_starts_that_do_not_ascend_stay_inside_the_tensors(new, held, prefix, D, dtype):
    """Out of contract but checked: other rows, the cache and later calls on the workspace are as they would be."""
    s = make(B=3, new=new, held=held, page=16, prefix=prefix, H=8, K=2, D=D, dtype=dtype)
    T = sum(new)
    ws = mb.meteora_prefix_attention_workspace(s["q"], s["kc"], s["table"], s["prefix"])
    want, kc, vc = call(s, workspace=ws), s["kc"].clone(), s["vc"].clone()
    for cu in ([0, T, 0, T], [T, 0, T, T], [-7, T + 9, -7, T + 9], [5, 0, -2 ** 31, 2 ** 31 - 1], [2 ** 31 - 1, -1, T, 0], [0, T, T - 1, T]):
        around = torch.full((T + 8, 8, D), 3.0, dtype=dtype, device="cuda")
        call(dict(s, cu=torch.tensor(cu, dtype=torch.int32, device="cuda")), out=around[4:-4], workspace=ws)
        assert (around[:4] == 3).all() and (around[-4:] == 3).all()
    assert torch.equal(kc.view(torch.uint8), s["kc"].view(torch.uint8)) and torch.equal(vc.view(torch.uint8), s["vc"].view(torch.uint8))
    assert torch.equal(call(s, workspace=ws), want)


def test_refusals():
    s = make(B=2, new=[1, 1], held=[10, 3], page=16, prefix=20, H=4, K=2, D=64, dtype=BF16, one_each=True)
    ws = mb.meteora_prefix_attention_workspace(s["q"], s["kc"], s["table"], s["prefix"])
    for bad in (dict(q=s["q"][:1]), dict(q=s["q"].float()), dict(q=s["q"][:, :3]), dict(q=s["q"][..., :32]), dict(q=s["q"].cpu()), dict(vc=s["vc"][:1]),
                dict(kc=s["kc"].transpose(1, 2)), dict(table=s["table"].long()), dict(lengths=s["lengths"][:1]), dict(prefix=-1), dict(prefix=33),
                dict(prefix_pages=None), dict(cu=s["lengths"]), dict(q=s["q"].half(), kc=s["kc"].half(), vc=s["vc"].half())):
        with pytest.raises((ValueError, TypeError, mb.MeteoraError)):
            call(dict(s, **bad))
    for kw in (dict(workspace=ws[:-256]), dict(out=s["q"][:, :1].expand_as(s["q"])), dict(scale=float("nan")), dict(out=s["q"].float()), dict(workspace=ws.cpu())):
        with pytest.raises((ValueError, TypeError, mb.MeteoraError)):
            call(s, **kw)
    assert call(dict(s, q=s["q"][:0], lengths=s["lengths"][:0], table=s["table"][:0])).shape == (0, 4, 64)
