"""The calls that keep the cache of chunks, on a side stream behind work that has not finished: whatever they read is read after it.  (The
attention's test of this is with those of its kernels.)"""
import pytest
import torch

import paper_2509_15763_b200 as ug

from chunk_util import DEV, Cache, attn_ref, cu_of

pytestmark = pytest.mark.gpu
BASE = 500000.0


def late_copies(values):
    """Buffers that hold something else until a side stream has slept, -> the stream, the buffers."""
    side, bufs = torch.cuda.Stream(), []
    for v in values:
        b = torch.empty_like(v)
        b.fill_(float("nan") if v.is_floating_point() else 0)
        bufs.append(b)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)
        for b, v in zip(bufs, values):
            b.copy_(v)
    return side, bufs


def both(values, outs, call):
    """call(values, outs, stream) on the current stream and behind late copies of the values on a side stream: the same outputs."""
    first = [x.clone() for x in outs]
    call(values, first, None)
    torch.cuda.synchronize()
    second = [x.clone() for x in outs]
    side, late = late_copies(values)
    call(late, second, side)
    side.synchronize()
    for a, b in zip(first, second):
        assert torch.equal(torch.nan_to_num(a.float(), 77.0), torch.nan_to_num(b.float(), 77.0))
    ug.unigist_device_status()


def rows_of(n, heads, dim, seed=1):
    return torch.randn(n, heads, dim, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).to(DEV)


@pytest.mark.parametrize("n", [3, 500])
def test_rotation(n):
    x, pos = rows_of(n, 9, 128), torch.arange(2 * n, dtype=torch.int32, device=DEV).reshape(2, n)
    both([x, pos], [torch.zeros_like(x)], lambda v, o, s: ug.unigist_rope_axes(v[0], o[0], v[1], [j % 2 for j in range(64)], BASE, stream=s))


@pytest.mark.parametrize("rows", [[3, 1], [100, 70]])
def test_append(rows):
    n, cache = sum(rows), Cache([70, 200], 2, 64, room=max(rows), waste=3.0)
    d = cache.device()
    pos = torch.arange(n, dtype=torch.int32, device=DEV)[None]
    both([rows_of(n, 2, 64), rows_of(n, 2, 64, 2), cu_of(rows).to(DEV), d["table"], d["lens"], pos],
         [d["k"], d["v"], d["w"], torch.zeros_like(d["lens"])],
         lambda v, o, s: ug.unigist_chunk_append(v[0], v[1], v[2], o[0], o[1], v[3], v[4], o[3], o[2], v[5], [0] * 32, BASE, stream=s))


@pytest.mark.parametrize("rows", [[3, 1], [100, 70]])
def test_weights(rows):
    cache = Cache([700, 200], 2, 64, waste=1.0)
    d, q = cache.device(), rows_of(sum(rows), 8, 64)
    lse = attn_ref(cache, q.cpu(), rows, 0.125)[1].float().to(DEV)
    both([q, cu_of(rows).to(DEV), lse, d["k"], d["table"], d["lens"], d["w"]], [torch.zeros_like(d["w"])],
         lambda v, o, s: ug.unigist_cache_weigh(*v, o[0], 0.5, stream=s))


@pytest.mark.parametrize("lens", [[700, 200], [30000, 60]])
@pytest.mark.parametrize("in_place", [False, True])
def test_eviction(lens, in_place):
    keep = 100
    cache = Cache(lens, 2, 64, waste=1.0, spare=5)
    d = cache.device()
    held = {int(p) for b, n in enumerate(lens) for p in cache.table[b, : -(-n // 64)]}
    to = torch.tensor([p for p in range(cache.blocks) if p not in held][:4], dtype=torch.int32, device=DEV).reshape(2, 2)

    def call(v, o, s):
        ug.unigist_cache_evict(o[0], o[1], o[2], v[0], v[1], v[0] if in_place else v[2], o[3], o[4], keep, 3, 5, stream=s)

    both([d["table"], d["lens"], to], [d["k"], d["v"], d["w"], torch.zeros_like(d["lens"]), torch.zeros(2, 2, keep, dtype=torch.int32, device=DEV)], call)


@pytest.mark.parametrize("rows,dim,wide", [([5, 1, 3], 128, 0), ([5, 1, 3], 128, 400), ([3, 1, 2], 64, 400), ([90, 1, 40], 64, 0), ([90, 1, 40], 128, 0)])
def test_a_whole_step_in_a_graph(rows, dim, wide):
    """Rotation, append, attention, weights and eviction in place, one behind the other in a graph (whose kernels start before the one before
    has ended): replayed three times, on what the last replay left, it is what the calls do by themselves."""
    hq, hkv, keep, n = 8, 2, 150, sum(rows)
    cache = Cache([500, 64, 170], hkv, dim, room=200, waste=1.0)
    if wide:
        table = torch.full((3, wide), -7, dtype=torch.int32)
        table[:, : cache.width] = cache.table
        cache.table, cache.width = table, wide
    qkv, cu = rows_of(n, hq + 2 * hkv, dim), cu_of(rows).to(DEV)
    pos = torch.arange(n, dtype=torch.int32, device=DEV)[None]
    axes = [0] * (dim // 2)
    states = []
    for _ in range(2):
        s = {**cache.device(), "q": torch.empty(n, hq, dim, dtype=torch.bfloat16, device=DEV), "lse": torch.empty(n, hq, device=DEV)}
        s.update(o=torch.empty_like(s["q"]), longer=torch.zeros_like(s["lens"]), kept=torch.zeros(3, hkv, keep, dtype=torch.int32, device=DEV),
                 ws=torch.empty(ug.unigist_chunk_attn_workspace_bytes(3, n, hq, hkv, dim, cache.width), dtype=torch.uint8, device=DEV))
        states.append(s)

    def step(s):
        ug.unigist_rope_axes(qkv[:, :hq], s["q"], pos, axes, BASE)
        ug.unigist_chunk_append(qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], cu, s["k"], s["v"], s["table"], s["lens"], s["longer"], s["w"], pos, axes, BASE)
        ug.unigist_chunk_attn(s["q"], cu, s["k"], s["v"], s["table"], s["longer"], s["o"], s["lse"], s["ws"])
        ug.unigist_cache_weigh(s["q"], cu, s["lse"], s["k"], s["table"], s["longer"], s["w"], s["w"], 0.9)
        ug.unigist_cache_evict(s["k"], s["v"], s["w"], s["table"], s["longer"], s["table"], s["lens"], s["kept"], keep, 4, 20)

    eager, captured = states
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(captured)
    for _ in range(3):
        step(eager)
        graph.replay()
        torch.cuda.synchronize()
        for name in ("q", "o", "lse", "longer", "kept", "lens", "k", "v", "w"):
            assert torch.equal(eager[name], captured[name]), name
        assert torch.isfinite(eager["o"].float()).all() and eager["lens"].max() <= keep
    ug.unigist_device_status()
