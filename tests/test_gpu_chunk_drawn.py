"""Weights, appends and evictions of batches drawn at random, against their definitions."""
import random

import pytest
import torch

import paper_2509_15763_b200 as ug

from chunk_routes import launched, widened
from chunk_util import DEV, PG, Cache, attn_ref, cu_of, evict_ref, weigh_ref

pytestmark = pytest.mark.gpu


def drawn_lens(rng, seqs, top):
    return [rng.choice([0, 1, 63, 64, 65, 127, 128, 129, rng.randint(0, top), rng.randint(0, top), -rng.randint(1, 9)]) for _ in range(seqs)]


@pytest.mark.parametrize("seed", range(6))
def test_weights(seed):
    rng = random.Random(seed)
    for i in range(12):
        G, hkv, dim, seqs = rng.choice([1, 2, 3, 4, 7, 8, 16, 31, 32, 33, 43, 64, 65, 127, 128]), rng.choice([1, 2, 3]), rng.choice([64, 128]), rng.choice([1, 2, 5, 12])
        top = rng.choice([1, 9, 70, 300])
        rows = [rng.choice([0, 1, rng.randint(0, top)]) for _ in range(seqs)]
        rows[0] = max(rows[0], 1)
        lens = [max(0, n + rng.choice([-5, 0, 0, 1, 64, 200, rng.randint(0, 1500)])) for n in rows]
        cache = Cache(lens, hkv, dim, seed=i)
        cache = widened(cache, cache.width + rng.choice([0, 1, 30]))
        q = torch.randn(sum(rows), G * hkv, dim, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16)
        lse = attn_ref(cache, q, rows, dim ** -0.5)[1].float()
        decay = rng.choice([0.0, 0.3, 1.0])
        d = cache.device()
        out = torch.full_like(d["w"], 5.0)
        ug.unigist_cache_weigh(q.to(DEV), cu_of(rows).to(DEV), lse.to(DEV), d["k"], d["table"], d["lens"], d["w"] if decay else None, out, decay)
        ug.unigist_device_status()
        out = out.cpu()
        rest = torch.ones_like(out, dtype=torch.bool)
        for b, want in weigh_ref(cache, q, rows, lse, dim ** -0.5, decay, cache.w).items():
            got = cache.rows(out, b)
            assert (((got - want).abs() - 1e-4 * want) <= 1e-30).all(), (rows, lens, G, hkv, dim, b)   # (the bound of the tests of that call)
            for j0 in range(0, lens[b], PG):
                rest[int(cache.table[b, j0 // PG]), :, : min(PG, lens[b] - j0)] = False
        assert (out[rest] == 5.0).all()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("seed", range(6))
def test_eviction(seed, in_place):
    """Short and long tables: one kernel or two, blocks alone and in clusters of any size."""
    rng = random.Random(seed)
    for i in range(8):
        hkv, dim, seqs = rng.choice([1, 2, 5]), rng.choice([64, 128]), rng.choice([1, 1, 2, 9, 30])
        lens = drawn_lens(rng, seqs, rng.choice([200, 3000, 60000 // seqs]))
        keep = rng.choice([1, 2, 63, 64, 65, 500, rng.randint(1, 5000)])
        first = rng.randint(0, keep)
        last = rng.choice([0, keep - first, rng.randint(0, keep - first)])
        fresh = [-(-min(max(n, 0), keep) // PG) for n in lens]
        cache = Cache(lens, hkv, dim, seed=i, waste=2.0, spare=1 + sum(fresh))
        kind = rng.choice(["spread", "few values", "equal"])
        if kind != "spread":
            cache.w = (cache.w * (3 if kind == "few values" else 0)).round()
        cache = widened(cache, cache.width + rng.choice([0, 1, 400]))
        d = cache.device()
        if in_place:
            to = d["table"]
        else:
            held = {int(p) for b, n in enumerate(lens) for p in cache.table[b, : -(-max(n, 0) // PG)]}
            free = iter([p for p in range(cache.blocks) if p not in held])
            to = torch.full((seqs, -(-keep // PG) + rng.choice([0, 3])), -3, dtype=torch.int32)
            for b, n in enumerate(fresh):
                to[b, :n] = torch.tensor([next(free) for _ in range(n)], dtype=torch.int32)
            to = to.to(DEV)
        new_lens = torch.full((seqs,), 99, dtype=torch.int32, device=DEV)
        kept = torch.full((seqs, hkv, keep), 99, dtype=torch.int32, device=DEV)
        names = launched(lambda: ug.unigist_cache_evict(d["k"], d["v"], d["w"], d["table"], d["lens"], to, new_lens, kept, keep, first, last))
        assert names in (["evict_fused_kernel"], ["evict_select_kernel", "evict_move_kernel"])
        what = f"{lens} keep {keep} {first} {last} {hkv} {dim} {names}"
        assert new_lens.tolist() == [min(n, keep) for n in lens], what
        pools, to, kept = {n: d[n].cpu() for n in ("k", "v", "w")}, to.cpu(), kept.cpu()
        touched = torch.zeros(cache.blocks, PG, dtype=torch.bool)
        for b, n in enumerate(lens):
            L, pages = max(n, 0), cache.table[b, : -(-max(n, 0) // PG)].long()
            m = min(L, keep)
            for j in range(m):
                touched[int(to[b, j // PG]), j % PG] = True
            for h in range(hkv):
                want = evict_ref(cache.w[pages, h].flatten()[:L], L, keep, first, last)
                assert kept[b, h].tolist() == want + [-1] * (keep - m), what
                for name in ("k", "v", "w"):
                    got = pools[name][to[b, : fresh[b]].long(), h].flatten(0, 1)[:m]
                    assert torch.equal(got, getattr(cache, name)[pages, h].flatten(0, 1)[want] if m else got), (what, name)
        rest = ~touched[:, None].expand(-1, hkv, -1)   # every other slot is as it was
        for name in ("k", "v", "w"):
            assert torch.equal(pools[name][rest], getattr(cache, name)[rest]), (what, name)


@pytest.mark.parametrize("seed", range(6))
def test_append(seed):
    rng = random.Random(seed)
    for i in range(10):
        hkv, dim, seqs = rng.choice([1, 2, 7, 8, 9, 17]), rng.choice([64, 128]), rng.choice([1, 2, 33, 40, 1100])
        rows = [rng.choice([0, 1, 2, rng.randint(0, 200 if seqs < 10 else 5)]) for _ in range(seqs)]
        lens = drawn_lens(rng, seqs, 300)
        cache = Cache(lens, hkv, dim, seed=i, room=rng.choice([0, 64, max(rows)]), waste=3.0)   # (some chunks do not fit)
        first, n = rng.choice([0, 3]), sum(rows)
        new = torch.randn(first + n + 2, 2 * hkv, dim, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16)
        d, nd = cache.device(), new.to(DEV)
        new_lens = torch.full((seqs,), 99, dtype=torch.int32, device=DEV)
        ug.unigist_chunk_append(nd[:, :hkv], nd[:, hkv:], cu_of(rows, first).to(DEV), d["k"], d["v"], d["table"], d["lens"], new_lens, d["w"])
        k, v, w, want, at = cache.k.clone(), cache.v.clone(), cache.w.clone(), [], first
        for b, (L, m) in enumerate(zip(lens, rows)):
            fits = L >= 0 and L + m <= cache.width * PG
            want.append(L + m if fits else -1)
            for j in range(m if fits else 0):
                page, slot = int(cache.table[b, (L + j) // PG]), (L + j) % PG
                if 0 <= page < cache.blocks:
                    k[page, :, slot], v[page, :, slot], w[page, :, slot] = new[at + j, :hkv], new[at + j, hkv:], 0.0
            at += m
        assert new_lens.tolist() == want
        assert torch.equal(d["k"].cpu(), k) and torch.equal(d["v"].cpu(), v) and torch.equal(d["w"].cpu(), w), (rows, lens, hkv, dim)
