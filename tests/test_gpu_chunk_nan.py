"""A score that is no number shows in what it reaches, and nowhere else: the query's output and log-sum-exp, and from there the weights of
the slots that it sees.  (Zeros and a log-sum-exp of minus infinity are for queries that see nothing.)"""
import math

import pytest
import torch

import paper_2509_15763_b200 as ug

from chunk_routes import ROUTES, cache_of, launched
from chunk_util import DEV, PG, Cache, attn_ref, attn_workspace, check_attn, cu_of, weigh_ref

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")
every_route = pytest.mark.parametrize("route", sorted(ROUTES))


def queries(n, hq, dim, seed=1):
    return torch.randn(n, hq, dim, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


def attend(cache, q, rows, kernels=None):
    d, (n, hq, dim) = cache.device(), q.shape
    o, lse = torch.full((n, hq, dim), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((n, hq), 7.0, device=DEV)
    ws = attn_workspace(len(rows), n, hq, cache.hkv, dim, cache.width)
    args = q.to(DEV), cu_of(rows).to(DEV), d["k"], d["v"], d["table"], d["lens"], o, lse, ws
    names = launched(lambda: ug.unigist_chunk_attn(*args))
    assert kernels is None or names == kernels
    ug.unigist_device_status()
    return o.cpu(), lse.cpu()


def check(o, lse, ref, bad, what=""):
    """Rows [n, heads] that `bad` names hold NaN in every feature, the others their results."""
    assert torch.isnan(o[bad].float()).all(), f"{what}: an output hides a score that is no number"
    assert torch.isnan(lse[bad]).all() or (lse[bad][~torch.isnan(lse[bad])] == INF).all(), f"{what}: {lse[bad]}"
    want, want_lse, size = (x.clone() for x in ref)
    o, lse = o.clone(), lse.clone()
    for x in (o, lse, want, want_lse, size):
        x[bad] = 0
    check_attn(o, lse, (want, want_lse, size), what)


@every_route
@pytest.mark.parametrize("x", [NAN, INF])
def test_queries_that_are_none(route, x):
    """One head of each of a few queries: the first of a chunk that sees the first slot alone, and others."""
    kernels, hq, _, dim, _, per = ROUTES[route]
    rows, lens = [per, max(1, per - 1), per], [700, 300, per]    # the last one's cache is its own chunk
    cache = cache_of(route, lens)
    q = queries(sum(rows), hq, dim)
    ref = attn_ref(cache, q, rows, dim ** -0.5)
    bad = torch.zeros(q.shape[:2], dtype=torch.bool)
    for i in {0, per, 2 * per - 1 if per > 1 else 2, q.shape[0] - 1}:
        for h in (i % hq, 5):
            bad[i, h] = True
            q[i, h, (3 * i) % dim:] = x
    o, lse = attend(cache, q, rows, kernels)
    check(o, lse, ref, bad, f"{route} {x}")


@every_route
@pytest.mark.parametrize("slot", [0, 1, 2, 8, 77, 449, 639, 640, 690, 691])
def test_keys_that_are_none(route, slot):
    """The queries that see the slot show it, those of the same chunk before it and the other KV head do not; wherever in the walk it comes."""
    kernels, hq, hkv, dim, _, per = ROUTES[route]
    L = 692
    rows, lens = [per, 1], [L, 130]
    cache = cache_of(route, lens)
    q = queries(sum(rows), hq, dim)
    ref = attn_ref(cache, q, rows, dim ** -0.5)
    cache.k[int(cache.table[0, slot // PG]), 1, slot % PG, 5:] = NAN
    o, lse = attend(cache, q, rows, kernels)
    bad = torch.zeros(q.shape[:2], dtype=torch.bool)
    for i in range(per):
        bad[i, hq // 2:] = L - per + i >= slot
    check(o, lse, ref, bad, f"{route} {slot}")


@pytest.mark.parametrize("dim", [64, 128])
def test_keys_that_are_none_in_walks_that_are_cut(dim):
    """A part of a cut unit may hold nothing but such scores for a row."""
    for rows, hq, hkv, L in (([300], 8, 2, 7000), ([5], 8, 2, 20000), ([70], 4, 1, 12000)):
        for slot in (0, 3000, L - rows[0] - 1):
            cache = Cache([L], hkv, dim, seed=slot)
            q = queries(rows[0], hq, dim)
            ref = attn_ref(cache, q, rows, dim ** -0.5)
            cache.k[int(cache.table[0, slot // PG]), 0, slot % PG] = NAN
            bad = torch.zeros(q.shape[:2], dtype=torch.bool)
            bad[:, : hq // hkv] = True
            check(*attend(cache, q, rows), ref, bad, f"{rows} {slot}")
            q[-1, 0] = NAN                      # every score of the row, in every part
            bad[:] = False
            bad[-1, 0] = True
            cache = Cache([L], hkv, dim, seed=slot)
            check(*attend(cache, q, rows), ref, bad, f"{rows} all")


@pytest.mark.parametrize("rows,lens,hq,hkv", [([1, 1], [300, 700], 8, 2), ([8, 4], [300, 700], 32, 1), ([100, 90], [400, 700], 8, 2), ([200, 64], [900, 64], 12, 4), ([40], [300], 7, 1)])
@pytest.mark.parametrize("dim", [64, 128])
def test_weights_of_queries_that_are_none(rows, lens, hq, hkv, dim):
    """Each query in turn: the slots that it sees get no number, in its head's KV head; all others theirs."""
    cache, n, G = Cache(lens, hkv, dim, seed=hq), sum(rows), hq // hkv
    q = queries(n, hq, dim)
    lse = attn_ref(cache, q, rows, dim ** -0.5)[1].float()
    for i in sorted({0, 1 % n, 2 % n, n // 2, n // 2 + 5 if n > 12 else 0, n - 1}):
        head = (3 * i + 1) % hq
        q2, lse2 = q.clone(), lse.clone()
        q2[i, head], lse2[i, head] = NAN, NAN
        d = cache.device()
        out = torch.full_like(d["w"], 5.0)
        ug.unigist_cache_weigh(q2.to(DEV), cu_of(rows).to(DEV), lse2.to(DEV), d["k"], d["table"], d["lens"], d["w"], out)
        ug.unigist_device_status()
        b = 0 if i < rows[0] else 1
        seen = lens[b] - rows[b] + (i - (0 if b == 0 else rows[0]))   # the last slot that it sees
        for c, want in weigh_ref(cache, q, rows, lse, dim ** -0.5, 1.0, cache.w).items():
            got = cache.rows(out, c)
            none = torch.zeros_like(got, dtype=torch.bool)
            if c == b:
                none[head // G, : seen + 1] = True
            assert torch.isnan(got[none]).all(), f"query {i} of {rows}: a weight hides it"
            assert (((got - want).abs() - 1e-4 * want)[~none] <= 1e-30).all(), (i, c)   # (the bound of the tests of that call)
