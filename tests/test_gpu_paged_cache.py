"""The workspaces of a decoder layer's paged cache: steps of any number of tokens, captured ones, layers that share."""
import pytest
import torch

from paper_2405_13053_b200 import binding as mb
from paper_2405_13053_b200 import decoder_layer as dl

pytestmark = pytest.mark.gpu
B = 6


def step(T, seed):
    """q, k, v of T new tokens of the B sequences, dealt unevenly, and their starts."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, k, v = (torch.randn(T, n, dl.HEAD_DIM, device="cuda", generator=g).to(torch.bfloat16) for n in (dl.N_HEADS, dl.N_KV_HEADS, dl.N_KV_HEADS))
    return q, k, v, torch.tensor([T * b * b // (B * B) for b in range(B + 1)], dtype=torch.int32, device="cuda")


def fill(cache):
    g = torch.Generator(device="cuda").manual_seed(99)
    for c in (cache.k, cache.v):
        c.copy_(torch.randn(c.shape, device="cuda", generator=g))
    cache.lengths += 50
    return cache


def need(cache, T):
    return mb.meteora_prefix_attention_workspace(step(T, 0)[0], cache.k, cache.page_table, cache.prefix_len).numel()


def test_steps_of_many_sizes_keep_one_workspace():
    cache, fresh = fill(dl.PagedCache(B, 700, prefix_len=90)), fill(dl.PagedCache(B, 700, prefix_len=90))
    sizes, most = [6, 301, 40, 7, 1000, 333, 64, 8], 0
    for T in sizes:
        x, most = step(T, T), max(most, need(cache, T))
        got = cache.attend(*x)
        assert sum(w.numel() for w in cache.workspaces.values()) == most
        want = mb.meteora_prefix_attention(mb.meteora_cache_append(x[1], x[2], fresh.k, fresh.v, fresh.page_table, fresh.lengths, fresh.rot, cu_tokens=x[3],
                                                                   prefix_len=90, q=x[0]),
                                           fresh.k, fresh.v, fresh.page_table, fresh.lengths, fresh.prefix_pages, 90, cu_tokens=x[3])
        assert torch.equal(got, want)
    assert all(mb.meteora_workspace_status(w) == 0 for w in cache.workspaces.values())


def test_a_captured_step_keeps_the_workspace_that_it_was_captured_with():
    cache = fill(dl.PagedCache(B, 700, prefix_len=90))
    x = step(12, 1)
    want = cache.attend(*x)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = cache.attend(*x)
    small = list(cache.workspaces.values())
    big = cache.attend(*step(900, 2))                                # outgrows it
    lent = [torch.full_like(w, 255) for w in small]                  # (where it had been given back, these would lie in its place)
    assert len(small) == 1 and len(cache.workspaces) == 2 and all(a is b for a, b in zip(small, cache.workspaces.values()))
    for _ in range(2):
        cache.attend(*x)                                             # (the same tokens' places as they were)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    assert all(bool((w == 255).all()) for w in lent) and torch.equal(cache.attend(*step(900, 2)), big)
    more = cache.attend(*step(1500, 3))                              # this one is in no graph: it goes
    assert len(cache.workspaces) == 2 and max(cache.workspaces) == need(cache, 1500) and torch.isfinite(more).all()
    assert cache.status() == 0


def test_a_step_that_is_captured_first_leaves_no_workspace_of_the_graph_behind():
    cache, other = fill(dl.PagedCache(B, 700)), fill(dl.PagedCache(B, 700))
    x = step(300, 4)
    other.attend(*x)                                                 # (the library's own first use of these kernels)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = cache.attend(*x)
    assert not cache.workspaces
    graph.replay()
    torch.cuda.synchronize()
    want = out.clone()
    assert torch.equal(want, other.attend(*x)) and torch.equal(want, cache.attend(*x)) and len(cache.workspaces) == 1
    del graph
    assert torch.equal(want, cache.attend(*x)) and cache.status() == 0


def test_layers_share_a_workspace_and_report_its_status():
    one = fill(dl.PagedCache(B, 300))
    two = fill(dl.PagedCache(B, 300, scratch=one.scratch))
    x = step(200, 5)
    assert torch.equal(one.attend(*x), two.attend(*x)) and len(one.workspaces) == 1 and two.workspaces is one.workspaces
    assert one.status() == two.status() == 0
    next(iter(one.workspaces.values()))[:4].view(torch.int32).fill_(1)       # what a kernel leaves whose wait has run out
    assert two.status() == -6
