"""Where the memory of a call on a given stream comes from."""
import numpy as np
import pytest
import torch

import paged_ref as R
from gpu_util import device
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


@pytest.mark.parametrize("given", [False, True])
def test_outputs_belong_to_the_stream_that_writes_them(dev, given):
    """Memory of another stream's pool may still be in use there when the call writes it."""
    rng = np.random.default_rng(41)
    D, T, lens, ps = 64, 9, [100, 30], 16
    c = R.Cache(rng, dev, np.array(lens) + T, 2, ps, D, True)
    q, qh = R.rounded(rng, (2, 4, T, D), True, dev)
    par, kv = R.tree(rng, 2, T), R.ints(lens, dev)
    pard = R.ints(par, dev)
    path, alen = R.ints([[0] + [-1] * (T - 1)] * 2, dev), R.ints([0, 0], dev)
    t = R.Tables(3, 8, 20, ps)
    t.reserve([40, 0, 0])
    t.kv_len[0] = 40
    table, count, kv_len, ref = t.on(dev)
    k = torch.zeros((20, 1, ps, D), device=dev)
    v, want, src, dst = k.clone(), R.ints([48, 16, 0], dev), R.ints([0], dev), R.ints([2], dev)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    kw = dict(stream=side) if given else {}
    with torch.cuda.stream(torch.cuda.current_stream() if given else side):
        verify = dreams.paged_verify_attn(q, c.kd, c.vd, c.tabled, kv, pard, **kw)
        prompt = dreams.paged_prompt_attn(q, c.kd, c.vd, c.tabled, kv, **kw)
        kept = dreams.paged_kv_commit(c.kd, c.vd, c.tabled, kv, path, alen, **kw)
        forked = dreams.pages_fork(k, v, table, count, kv_len, ref, src, dst, **kw)
        room = dreams.pages_reserve(table, count, ref, want, ps, **kw)
    torch.cuda.synchronize()
    for x in (*verify, *prompt, kept, forked, room):
        assert stream_of(x) == side.cuda_stream != stream_of(q)
    R.check(*verify, R.verify(qh, c.k, c.v, c.table, lens, par, R.ancestors(par), 0, 0, 1 / np.sqrt(D)), True, "verify")
    R.check(*prompt, R.prompt(qh, c.k, c.v, c.table, lens, [T, T], 0, 0, 1 / np.sqrt(D)), True, "prompt")
    assert kept.tolist() == [101, 31] and forked.tolist() == t.fork([0], [2])[0] and room.tolist() == t.reserve([48, 16, 0])


def test_eager_calls_on_another_stream_than_the_captured_one(dev):
    """They would take memory for their outputs while a graph is captured: refused, and the graph is whole."""
    table, count, kv_len, ref = R.Tables(2, 4, 9, 16).on(dev)
    want, granted = R.ints([20, 0], dev), R.ints([7, 7], dev)
    k = torch.zeros((9, 1, 16, 64), device=dev)
    side, captured = torch.cuda.Stream(), torch.cuda.Stream()
    dreams.pages_reserve(table, count, ref, R.ints([0, 0], dev), 16, granted=granted)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=captured):
        with pytest.raises(ValueError, match="captured"):
            dreams.pages_reserve(table, count, ref, want, 16, stream=side)
        with pytest.raises(ValueError, match="captured"):
            dreams.pages_fork(k, k, table, count, kv_len, ref, want[:1], want[1:], stream=side)
        room = dreams.pages_reserve(table, count, ref, want, 16)
    for rep in range(3):
        room.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert room.tolist() == [1, 1] and count.tolist() == [2, 0] and table[0].tolist() == [0, 1, -1, -1]
