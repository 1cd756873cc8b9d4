"""Calls on a given stream: what they allocate, workspaces among it, belongs to that stream."""
import pytest
import torch

from gpu_util import device, note
from paper_2606_00535_amd import dreams

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    d = device()
    dreams.lib()
    return d


def stream_of(t):
    """The stream that the caching allocator gives a tensor's memory to."""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not the allocator's memory")


def calls(dev):
    """name, a call that takes stream=."""
    g = torch.Generator(device=dev)
    g.manual_seed(5)
    normal = lambda *s, dt=torch.float32: torch.empty(s, dtype=dt, device=dev).normal_(generator=g)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
    B, H, T, D, S, V = 2, 4, 6, 128, 2100, 300
    q, k, v = normal(B, H, T, D, dt=torch.bfloat16), normal(B, 2, S, D, dt=torch.bfloat16), normal(B, 2, S, D, dt=torch.bfloat16)
    kv, par = ints([2000, 77]), ints([[-1, 0, 0, 1, 1, 2]] * B)
    logits, draft, tokens = normal(B, T, V), normal(B, T, V), ints([[3, 1, 4, 1, 5, 9]] * B)
    hidden, weight = normal(B, T, 256, dt=torch.bfloat16), normal(V, 256, dt=torch.bfloat16)
    uniforms = torch.empty((B, T), device=dev).uniform_(generator=g)
    entropy, lse, long = normal(B, H, T).abs(), normal(B, H, T), normal(B, H, 40, D, dt=torch.bfloat16)
    plen, scores = ints([40, 17]), normal(B, 50).abs()
    path, alen = ints([[0, 2, 5, -1, -1, -1]] * B), ints([2, 0])
    kept, k2, v2 = ints([[0, 2, 9], [1, 5, 6]]), k.clone(), v.clone()
    long_lse = dreams.prefill_attn_stats(long, k, plen)[0]
    return [
        ("tree_verify_attn", lambda **kw: dreams.tree_verify_attn(q, k, v, kv, par, num_splits=4, **kw)),
        ("tree_verify_attn_entropy", lambda **kw: dreams.tree_verify_attn_entropy(q, k, v, kv, par, num_splits=4, **kw)),
        ("tree_verify_attn_noalloc", lambda **kw: dreams.tree_verify_attn_noalloc(q, k, v, kv, par, num_splits=4, **kw)),
        ("attn_entropy_mean", lambda **kw: (dreams.attn_entropy_mean(entropy, **kw),)),
        ("attn_entropy_select", lambda **kw: (dreams.attn_entropy_select(scores[0], **kw),)),
        ("visual_importance", lambda **kw: (dreams.visual_importance(q, k, kv, lse, 5, 60, **kw),)),
        ("prefill_attn_stats", lambda **kw: dreams.prefill_attn_stats(long, k, plen, **kw)),
        ("prefill_attn_entropy_mean", lambda **kw: (dreams.prefill_attn_entropy_mean(long_lse, plen, **kw),)),
        ("prefill_visual_importance", lambda **kw: (dreams.prefill_visual_importance(long, k, plen, long_lse, 0, 16, **kw),)),
        ("visual_topk", lambda **kw: (dreams.visual_topk(scores, 7, **kw),)),
        ("visual_gather", lambda **kw: dreams.visual_gather(k, v, 3, kept, **kw)),
        ("tree_accept", lambda **kw: dreams.tree_accept(logits, tokens, par, True, **kw)),
        ("tree_accept_sampled", lambda **kw: dreams.tree_accept_sampled(logits, draft, tokens, par, uniforms, **kw)),
        ("tree_accept_lm_head", lambda **kw: dreams.tree_accept_lm_head(hidden, weight, tokens, par, True, **kw)),
        ("kv_commit", lambda **kw: (dreams.kv_commit(k2, v2, kv, path, alen, **kw),)),
        ("stream_read", lambda **kw: (dreams.stream_read(k, **kw),)),
    ]


def test_memory_of_calls_on_a_given_stream(dev):
    side = torch.cuda.Stream()
    for name, call in calls(dev):
        note(name)
        want = call()
        torch.cuda.synchronize()
        before = {id(w) for w in dreams.cached_workspaces()}
        got = call(stream=side)
        torch.cuda.synchronize()
        for x in got + tuple(w for w in dreams.cached_workspaces() if id(w) not in before):
            assert x is None or stream_of(x) == side.cuda_stream, name
        for x, y in zip(got, want):
            assert (x is None and y is None) or torch.equal(x, y) or name == "stream_read", name
