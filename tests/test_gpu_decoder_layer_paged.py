"""The decoder layer over a paged cache against the same layer in its other modes, which the oracle's layer is compared with: a
prompt against the prefill of one sequence, a decode batch behind a shared prefix against the batch with a cache per
sequence.  Every intermediate of either side is rounded to bf16 (about ten roundings of 2^-9 along the path, some of them
elsewhere): relative L2 of the output <= 2e-2, the bound of those comparisons.
"""
import pytest
import torch

from paper_2405_13053_b200 import decoder_layer as dl

pytestmark = pytest.mark.gpu


def rel(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm())


@pytest.fixture(scope="module")
def layer():
    return dl.random_layer(torch.device("cuda"), b_std=0.2)


def test_prompts_then_single_tokens(layer):
    """Two prompts of different lengths in one call, then a token of each; every sequence alone through the prefill mode."""
    weights, norms = layer
    g = torch.Generator(device="cuda").manual_seed(1)
    lens, lin = [301, 70], dl.LibraryLinears(weights, k=2)
    xs = [torch.randn(n + 1, dl.HIDDEN, device="cuda", generator=g).to(torch.bfloat16) for n in lens]
    cache = dl.PagedCache(2, 400, page_size=32)
    cu = torch.tensor([0, lens[0], sum(lens)], dtype=torch.int32, device="cuda")
    y = dl.layer_forward(torch.cat([x[:-1] for x in xs]), norms, lin, paged=cache, cu_tokens=cu)
    cache.advance(torch.tensor(lens, dtype=torch.int32, device="cuda"))
    z = dl.layer_forward(torch.stack([x[-1] for x in xs]), norms, lin, paged=cache)
    assert lin.status() == 0
    for b, x in enumerate(xs):
        want = dl.layer_forward(x, norms, lin, torch.arange(lens[b] + 1, device="cuda"))
        assert rel(y[int(cu[b]):int(cu[b + 1])], want[:-1]) <= 2e-2
        assert rel(z[b], want[-1]) <= 2e-2


def test_decode_batch_behind_a_shared_prefix(layer):
    weights, norms = layer
    g = torch.Generator(device="cuda").manual_seed(2)
    B, prefix, own, lin = 24, 150, 45, dl.LibraryLinears(weights, k=2)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g).to(torch.bfloat16)  # noqa: E731
    kp, vp = rand(prefix, dl.N_KV_HEADS, dl.HEAD_DIM), rand(prefix, dl.N_KV_HEADS, dl.HEAD_DIM)
    ko, vo = rand(B, own, dl.N_KV_HEADS, dl.HEAD_DIM), rand(B, own, dl.N_KV_HEADS, dl.HEAD_DIM)
    x = rand(B, dl.HIDDEN)
    cache = dl.PagedCache(B, 64, prefix_len=prefix, page_size=16)
    cache.append_prefix(kp, vp)
    cu = torch.arange(B + 1, dtype=torch.int32, device="cuda") * own
    cache.attend(rand(B * own, dl.N_HEADS, dl.HEAD_DIM), ko.flatten(0, 1), vo.flatten(0, 1), cu)
    cache.advance(own)
    # the other mode: the rotated keys of prefix and own tokens in one contiguous cache per sequence
    kp, ko = dl.rotary(kp, torch.arange(prefix, device="cuda")), dl.rotary(ko, torch.arange(prefix, prefix + own, device="cuda"))
    flat = lambda p, o: torch.cat([p.expand(B, *p.shape), o], dim=1).transpose(1, 2).contiguous()  # noqa: E731
    want = dl.layer_forward(x, norms, lin, torch.full((B,), prefix + own, device="cuda"), flat(kp, ko), flat(vp, vo))
    got = dl.layer_forward(x, norms, lin, paged=cache)
    assert rel(got, want) <= 2e-2
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(got)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):                                    # the same step, captured
        out.copy_(dl.layer_forward(x, norms, lin, paged=cache))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, got) and lin.status() == 0
    assert all(cache.mb.meteora_workspace_status(w) == 0 for w in cache.workspaces.values())
