"""The calls on chunks where offsets pass 32 bits: caches, row tensors and outputs of more than 2^31 elements; the largest number of sequences.
What a call makes of far pages and rows is, bit for bit, what it makes of the same content in small tensors."""
import pytest
import torch

import paper_2509_15763_b200 as ug

from chunk_routes import launched
from chunk_util import DEV, PG, Cache, attn_ref, attn_workspace, check_attn, cu_of, evict_ref

pytestmark = pytest.mark.gpu
BASE = 500000.0


@pytest.fixture(autouse=True)
def free():
    yield
    torch.cuda.empty_cache()


class Far:
    """A cache's content in the last pages of pools that hold more than 2^31 elements (the first pages hold NaN)."""

    def __init__(self, cache, dim):
        self.blocks = 2 ** 31 // (cache.hkv * PG * dim) + cache.blocks + 7
        self.first = self.blocks - cache.blocks
        assert self.first * cache.hkv * PG * dim >= 2 ** 31
        shape = (self.blocks, cache.hkv, PG, dim)
        self.d = {"k": torch.empty(shape, dtype=torch.bfloat16, device=DEV), "v": torch.empty(shape, dtype=torch.bfloat16, device=DEV),
                  "w": torch.empty(shape[:3], device=DEV), "lens": torch.tensor(cache.lens, dtype=torch.int32, device=DEV)}
        for n in ("k", "v", "w"):
            self.d[n][: cache.blocks] = float("nan")
            self.d[n][self.first:] = getattr(cache, n).to(DEV)
        real = (cache.table >= 0) & (cache.table < cache.blocks)
        self.d["table"] = torch.where(real, cache.table + self.first, cache.table).to(DEV)

    def same(self, name, small):
        return torch.equal(torch.nan_to_num(self.d[name][self.first:].float(), 77.0), torch.nan_to_num(small.float(), 77.0))


@pytest.mark.parametrize("rows,lens,hq,hkv,dim,width", [([4, 1, 3], [700, 64, 130], 32, 8, 128, 0), ([8, 3], [900, 65], 32, 8, 128, 400), ([70, 1, 90], [500, 300, 90], 32, 8, 128, 0),
                                                        ([3, 2], [900, 65], 32, 8, 64, 400), ([70, 1, 90], [500, 300, 90], 32, 8, 64, 0)])
def test_far_pages(rows, lens, hq, hkv, dim, width):
    """Append, attention, weights and eviction, in place and into other pages, by one loop over a small and a far cache."""
    n, keep = sum(rows), 60
    before = [L - r for L, r in zip(lens, rows)]
    cache = Cache(before, hkv, dim, room=max(rows), waste=2.0, spare=1 + len(rows))
    if width:
        wide = torch.full((len(rows), width), -7, dtype=torch.int32)
        wide[:, : cache.width] = cache.table
        cache.table, cache.width = wide, width
    g = torch.Generator().manual_seed(2)
    qkv = torch.randn(n, hq + 2 * hkv, dim, generator=g).to(torch.bfloat16).to(DEV)
    cu = cu_of(rows).to(DEV)
    results = []
    far = Far(cache, dim)
    held = {int(p) for b, L in enumerate(before) for p in cache.table[b, : -(-(L + max(rows)) // PG)]}
    free_pages = [p for p in range(cache.blocks) if p not in held][: len(rows)]
    for d, first in ((cache.device(), 0), (far.d, far.first)):
        new_lens = torch.zeros_like(d["lens"])
        pos = torch.arange(n, dtype=torch.int32, device=DEV)[None]
        ug.unigist_chunk_append(qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], cu, d["k"], d["v"], d["table"], d["lens"], new_lens, d["w"], pos, [0] * (dim // 2), BASE)
        q = qkv[:, :hq].contiguous()
        o, lse = torch.empty_like(q), torch.empty(n, hq, device=DEV)
        ug.unigist_chunk_attn(q, cu, d["k"], d["v"], d["table"], new_lens, o, lse, attn_workspace(len(rows), n, hq, hkv, dim, d["table"].shape[1]))
        ug.unigist_cache_weigh(q, cu, lse, d["k"], d["table"], new_lens, d["w"], d["w"], 0.5)
        ug.unigist_device_status()
        kept = torch.zeros(len(rows), hkv, keep, dtype=torch.int32, device=DEV)
        cut = torch.zeros_like(new_lens)
        to = torch.tensor(free_pages, dtype=torch.int32, device=DEV)[:, None] + first
        ug.unigist_cache_evict(d["k"], d["v"], d["w"], d["table"], new_lens, to, cut, kept, keep, 4, 8)       # into other pages
        kept2, cut2 = torch.zeros_like(kept), torch.zeros_like(cut)
        ug.unigist_cache_evict(d["k"], d["v"], d["w"], d["table"], new_lens, d["table"], cut2, kept2, keep, 4, 8)   # in place
        assert torch.equal(kept, kept2) and torch.equal(cut, cut2) and cut.tolist() == [min(L, keep) for L in lens]
        results.append((o, lse, kept, d))
    (o, lse, kept, small), (o2, lse2, kept2, _) = results
    assert torch.isfinite(o.float()).all() and torch.equal(o, o2) and torch.equal(lse, lse2) and torch.equal(kept, kept2)
    for name in ("k", "v", "w"):
        assert far.same(name, small[name]), name
        assert torch.isnan(far.d[name][: cache.blocks].float()).all()


def test_a_rotated_tensor_of_more_than_two_to_the_31_elements():
    tokens, heads = 16500, 1024
    x = torch.empty(tokens, heads, 128, dtype=torch.bfloat16, device=DEV)
    assert x[:-1].numel() > 2 ** 31
    x.normal_(generator=torch.Generator(DEV).manual_seed(1))
    pos = torch.arange(2 * tokens, dtype=torch.int32, device=DEV).reshape(2, tokens)
    axes, y = [j % 2 for j in range(64)], torch.empty_like(x)
    ug.unigist_rope_axes(x, y, pos, axes, BASE)
    for part in (slice(0, 3), slice(tokens // 2, tokens // 2 + 2), slice(tokens - 50, tokens)):
        want = torch.empty_like(x[part])
        ug.unigist_rope_axes(x[part], want, pos[:, part].contiguous(), axes, BASE)
        assert torch.equal(y[part], want)
    ug.unigist_rope_axes(x, x, pos, axes, BASE)
    assert torch.equal(x, y)


@pytest.mark.parametrize("rows,lens", [([5, 1], [300, 64]), ([100, 90], [300, 90])])
def test_rows_far_apart(rows, lens):
    """Rows that lie 2^24 elements from each other in a tensor of more than 2^31."""
    n, hq, hkv, dim = sum(rows), 8, 2, 128
    apart = 2 ** 32 // n // 8 * 8
    whole = torch.empty(n, apart // dim, dim, dtype=torch.bfloat16, device=DEV)
    qkv = whole[:, 3: 3 + hq + 2 * hkv]
    near = torch.randn(n, hq + 2 * hkv, dim, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).to(DEV)
    qkv.copy_(near)
    assert qkv.stride(0) * (n - 1) > 2 ** 31
    cache, cu, results = Cache(lens, hkv, dim, waste=1.0, room=max(rows)), cu_of(rows).to(DEV), []
    pos = torch.arange(n, dtype=torch.int32, device=DEV)[None]
    for x in (near, qkv):
        d = cache.device()
        q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
        ug.unigist_rope_axes(q, q, pos, [0] * 64, BASE)
        new_lens, w = torch.zeros_like(d["lens"]), torch.zeros_like(d["w"])
        ug.unigist_chunk_append(k, v, cu, d["k"], d["v"], d["table"], d["lens"], new_lens, None, pos, [0] * 64, BASE)
        o, lse = torch.empty(n, hq, dim, dtype=torch.bfloat16, device=DEV), torch.empty(n, hq, device=DEV)
        ug.unigist_chunk_attn(q, cu, d["k"], d["v"], d["table"], new_lens, o, lse, attn_workspace(2, n, hq, hkv, dim, cache.width))
        ug.unigist_cache_weigh(q, cu, lse, d["k"], d["table"], new_lens, None, w, 0.0)
        ug.unigist_device_status()
        results.append((q.clone(), d["k"], d["v"], o, lse, w))
    assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("per,kernel", [(8, "chunk_few_kernel"), (9, "chunk_attn_sm100_kernel")])
def test_the_largest_number_of_sequences_and_more_than_two_to_the_31_outputs(per, kernel):
    S, hq, hkv, dim, L = 65535, 40, 10, 128, 50
    cache = Cache([L] * 3, hkv, dim)
    d, n = cache.device(), S * per
    q = torch.empty(n, hq, dim, dtype=torch.bfloat16, device=DEV).normal_(generator=torch.Generator(DEV).manual_seed(1))
    assert q.numel() > 2 ** 31
    o, lse = torch.full_like(q, 7.0), torch.full((n, hq), 7.0, device=DEV)
    table, lens = d["table"].repeat(S // 3, 1).contiguous(), torch.full((S,), L, dtype=torch.int32, device=DEV)   # (pages that are only read may be shared)
    cu = torch.arange(0, n + 1, per, dtype=torch.int32, device=DEV)
    ws = attn_workspace(S, n, hq, hkv, dim, 1)
    names = launched(lambda: ug.unigist_chunk_attn(q, cu, d["k"], d["v"], table, lens, o, lse, ws))
    assert names[0] == kernel
    ug.unigist_device_status()
    assert torch.isfinite(lse).all()
    for b in (0, 1, 21844, 43691, S - 3):   # three neighbours at a time, which read the three pages
        b -= b % 3
        part = slice(b * per, (b + 3) * per)
        check_attn(o[part], lse[part], attn_ref(cache, q[part].cpu(), [per] * 3, dim ** -0.5), f"from sequence {b}")
    del o, lse
    new_lens = torch.zeros_like(lens)
    ug.unigist_chunk_append(q[:, :hkv], q[:, hkv:2 * hkv], cu, d["k"], d["v"], torch.full_like(table, -1), lens, new_lens)   # (no page to write to)
    assert (new_lens == L + per).all()


def test_the_largest_number_of_sequences_weighed_and_evicted():
    S, hkv, dim, L, keep = 65535, 2, 64, 64, 20
    pools = torch.randn(S, hkv, PG, dim, device=DEV, generator=torch.Generator(DEV).manual_seed(1)).to(torch.bfloat16)
    w = torch.rand(S, hkv, PG, device=DEV, generator=torch.Generator(DEV).manual_seed(2))
    table = torch.arange(S, dtype=torch.int32, device=DEV)[:, None].contiguous()
    lens = torch.full((S,), L, dtype=torch.int32, device=DEV)
    lens[7::11] = 13
    q = torch.randn(S, 4, dim, device=DEV, generator=torch.Generator(DEV).manual_seed(3)).to(torch.bfloat16)
    cu, lse = torch.arange(S + 1, dtype=torch.int32, device=DEV), torch.full((S, 4), 5.0, device=DEV)
    out = torch.full_like(w, 5.0)
    ug.unigist_cache_weigh(q, cu, lse, pools, table, lens, w, out, 0.5)
    ug.unigist_device_status()
    z = torch.einsum("shgd,shjd->shgj", q.double().unflatten(1, (2, 2)), pools.double()) / 8 - 5.0
    want = 0.5 * w.double() + z.exp().sum(2)
    live = torch.arange(PG, device=DEV) < lens[:, None, None]
    assert (((out.double() - want).abs() - 1e-4 * want)[live.expand_as(w)] <= 0).all() and (out[~live.expand_as(w)] == 5.0).all()
    new_lens, kept = torch.zeros_like(lens), torch.zeros(S, hkv, keep, dtype=torch.int32, device=DEV)
    ug.unigist_cache_evict(pools, pools.clone(), w, table, lens, table, new_lens, kept, keep, 2, 3)
    assert torch.equal(new_lens, lens.clamp(max=keep))
    w0 = torch.rand(S, hkv, PG, device=DEV, generator=torch.Generator(DEV).manual_seed(2)).cpu()
    for b in (0, 1, 7, 32767, 32768, S - 1, S - 2):
        for h in range(hkv):
            slots = evict_ref(w0[b, h, : int(lens[b])], int(lens[b]), keep, 2, 3)
            assert kept[b, h].tolist() == slots + [-1] * (keep - len(slots))
            assert torch.equal(w[b, h, : len(slots)].cpu(), w0[b, h][slots])


@pytest.mark.parametrize("n,hq,dim,kernel", [(1, 8, 64, "chunk_few_kernel"), (3, 8, 128, "chunk_thin_sm100_kernel"), (70, 4, 64, "chunk_attn_sm100_kernel"),
                                             (70, 4, 128, "chunk_attn_sm100_kernel")])
def test_a_very_long_cache(n, hq, dim, kernel):
    """400003 slots: attention and weights.  (Fewer bits than the slots have would show: the values of the far ones are large.)"""
    L, scale = 400003, dim ** -0.5
    cache = Cache([L], 1, dim, seed=1)
    far = torch.zeros(cache.width * PG)
    far[: L] = 1.0
    far[: 700], far[L - 900: L - 100] = 30.0, 30.0
    pages = cache.table[0, : cache.width].long()
    cache.v[pages] = (cache.v[pages].float() * far.reshape(-1, 1, PG, 1)).to(torch.bfloat16)
    q = (0.3 * torch.randn(n, hq, dim, generator=torch.Generator().manual_seed(2))).to(torch.bfloat16)
    d, cu = cache.device(), cu_of([n]).to(DEV)
    o, lse = torch.empty(n, hq, dim, dtype=torch.bfloat16, device=DEV), torch.empty(n, hq, device=DEV)
    ws = attn_workspace(1, n, hq, 1, dim, cache.width)
    names = launched(lambda: ug.unigist_chunk_attn(q.to(DEV), cu, d["k"], d["v"], d["table"], d["lens"], o, lse, ws))
    assert names[0] == kernel
    k, v = cache.rows(cache.k, 0).to(DEV)[0], cache.rows(cache.v, 0).to(DEV)[0]
    want, want_lse, size = (torch.zeros(n, hq, dim, dtype=torch.float64), torch.zeros(n, hq, dtype=torch.float64), torch.zeros(n, hq, dim, dtype=torch.float64))
    total = torch.zeros(L, dtype=torch.float64, device=DEV)
    for i in range(n):
        see = L - n + i + 1
        z = q[i].double().to(DEV) @ k[:see].T * scale
        l = torch.logsumexp(z, -1)
        p = torch.exp(z - l[:, None])
        total[:see] += p.sum(0)
        want[i], want_lse[i], size[i] = (p @ v[:see]).cpu(), l.cpu(), (p @ v[:see].abs()).cpu()
    check_attn(o, lse, (want, want_lse, size), kernel)
    w = torch.zeros_like(d["w"])
    ug.unigist_cache_weigh(q.to(DEV), cu, lse, d["k"], d["table"], d["lens"], None, w, 0.0)
    ug.unigist_device_status()
    got = cache.rows(w, 0)[0].to(DEV)
    assert ((got - total).abs() - 3e-4 * total).max() <= 1e-30   # (1e-4 of the call itself, 2e-4 of the log-sum-exps that it was given)


@pytest.mark.parametrize("keep,first,last", [(700, 4, 64), (150001, 0, 0), (1, 0, 0), (200002, 1, 1)])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("weights", ["random", "ties"])
def test_eviction_from_a_cache_whose_weights_fit_no_cluster(keep, first, last, in_place, weights):
    """More slots than the blocks of a cluster hold weights of: they are read again in every pass."""
    L = 200003
    cache = Cache([L, 100], 1, 64, seed=keep, waste=2.0, spare=1 + 2 * -(-keep // PG))
    if weights == "ties":
        cache.w = (cache.w * 3).round()
    d = cache.device()
    held = set(cache.table[0].tolist()) | {int(cache.table[1, 0]), int(cache.table[1, 1])}
    width = -(-keep // PG)
    fresh = torch.tensor([p for p in range(cache.blocks) if p not in held][: 2 * width], dtype=torch.int32).reshape(2, width)
    to = d["table"] if in_place else fresh.to(DEV)
    new_lens, kept = torch.zeros(2, dtype=torch.int32, device=DEV), torch.zeros(2, 1, keep, dtype=torch.int32, device=DEV)
    names = launched(lambda: ug.unigist_cache_evict(d["k"], d["v"], d["w"], d["table"], d["lens"], to, new_lens, kept, keep, first, last))
    assert names == ["evict_select_kernel", "evict_move_kernel"]
    for b, n in enumerate((L, 100)):
        m, w0 = min(n, keep), cache.rows(cache.w, b, n)[0]
        number = torch.where(w0 > 0, w0, 0.0)
        number[:first], number[n - last:] = float("inf"), float("inf")
        want = torch.sort(number, descending=True, stable=True).indices[:m].sort().values if n > keep else torch.arange(n)
        assert int(new_lens[b]) == m and torch.equal(kept[b, 0, :m].cpu().long(), want) and (kept[b, 0, m:] == -1).all()
        for name in ("k", "v", "w"):
            pages = to[b, : -(-m // PG)].cpu().long()
            got = d[name].cpu()[pages, 0].flatten(0, 1)[:m]
            assert torch.equal(got, getattr(cache, name)[cache.table[b, : -(-n // PG)].long(), 0].flatten(0, 1)[want])
