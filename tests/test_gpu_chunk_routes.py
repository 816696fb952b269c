"""What the attention of chunks promises holds for each of the kernels that a call may take, named by the test: the sizes alone choose
among them, and a case that a change of the choice leads to another kernel fails."""
import math
import random

import pytest
import torch

import paper_2509_15763_b200 as ug

from chunk_routes import ROUTES, cache_of, launched, widened
from chunk_util import BF16_HALF, DEV, PG, Cache, attn_ref, attn_workspace, check_attn, cu_of, weigh_ref

pytestmark = pytest.mark.gpu
LEAST = -2 ** 31
every_route = pytest.mark.parametrize("route", sorted(ROUTES))


def queries(n, hq, dim, seed=1):
    return torch.randn(n, hq, dim, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


def attend(route, cache, q, cu, dev=None, scale=0.0):
    """-> o, lse; the call's kernels are the route's (its name, or theirs)."""
    kernels = ROUTES[route][0] if isinstance(route, str) else route
    d = dev or cache.device()
    (n, hq, dim), (S, width) = q.shape, d["table"].shape
    o = torch.full((n, hq, dim), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((n, hq), 7.0, device=DEV)
    ws = attn_workspace(S, n, hq, cache.hkv, dim, width)
    args = q.to(DEV), cu.to(DEV), d["k"], d["v"], d["table"], d["lens"], o, lse, ws, scale
    assert launched(lambda: ug.unigist_chunk_attn(*args)) == kernels
    ug.unigist_device_status()
    return o, lse


def case(kernels, rows, lens, hq, hkv, dim, seed=0, width=0):
    cache = Cache(lens, hkv, dim, seed=seed)
    cache = widened(cache, width or cache.width)
    q, cu = queries(sum(rows), hq, dim, seed + 1), cu_of(rows)
    o, lse = attend(kernels, cache, q, cu)
    check_attn(o, lse, attn_ref(cache, q, rows, dim ** -0.5), f"{rows} {lens} {hq}/{hkv} {dim}")
    for x, y in zip(attend(kernels, cache, q, cu), (o, lse)):
        assert torch.equal(x, y)


SHARES, THIN = ROUTES["shares64"][0], ROUTES["thin128"][0]


@pytest.mark.parametrize("rows,lens,hq,hkv,width", [
    ([1] * 40, [3000 + 61 * i for i in range(40)], 16, 4, 0),      # one tile of 16 rows a unit
    ([1] * 20, [4000 + 61 * i for i in range(20)], 32, 2, 0),      # a group that fills it
    ([4, 0, 0, 0], [700, 5000, 1, 64], 10, 2, 400),                # two units of three tokens and one
    ([0, 1, 1, 2], [700, 5000, 1, 65], 6, 2, 400),
    ([4], [20011], 32, 8, 0),                                      # two tiles; one sequence, cut many times
    ([12, 0, 1, 3], [9000, 300, 9001, 8000], 64, 16, 0),           # a sequence of two units
    ([16], [30000], 4, 4, 0), ([40, 1, 1, 1], [30000, 70, 5, 1], 2, 2, 600),   # groups of one
    ([5, 3, 0, 1], [5000, 200, 40, 64], 6, 2, 400), ([1, 0, 0, 1], [9000, 1, 1, 77], 20, 1, 1000), ([0, 1, 0], [10, 30000, 10], 32, 1, 1000),
    ([7, 2] * 8, [2 ** (i % 13) + 7 for i in range(16)], 4, 2, 500),
    ([3] * 90, [130 + 37 * i for i in range(90)], 8, 8, 0),
])
def test_shared_out_walks_of_few_rows(rows, lens, hq, hkv, width):
    """Heads of 64, short chunks over long caches: all pages dealt out in equal shares, cut units added up."""
    case(SHARES, rows, lens, hq, hkv, 64, seed=hq, width=width)


@pytest.mark.parametrize("rows,lens,hq,hkv,width", [
    ([8], [20011], 32, 8, 0), ([1] * 40, [3000 + 61 * i for i in range(40)], 16, 4, 0), ([20, 0, 1, 8], [9000, 300, 9001, 8000], 64, 16, 0),
    ([32], [30000], 4, 4, 0), ([70, 1, 1, 1], [30000, 70, 5, 1], 2, 2, 600), ([5, 3, 0, 1], [5000, 200, 40, 64], 6, 2, 400),
    ([11, 0, 0, 1], [700, 5000, 1, 64], 10, 1, 1000), ([0, 1, 0], [10, 30000, 10], 32, 1, 1000), ([1, 1], [9000, 1], 32, 1, 1000),
    ([7, 2] * 8, [2 ** (i % 13) + 7 for i in range(16)], 4, 2, 500), ([3] * 90, [130 + 37 * i for i in range(90)], 8, 8, 0),
])
def test_few_rows_as_columns(rows, lens, hq, hkv, width):
    """Heads of 128, short chunks over long caches: the kernel that has the keys as the rows of its products."""
    case(THIN, rows, lens, hq, hkv, 128, seed=hq, width=width)


def drawn_rows(rng, seqs, most):
    """Rows of the sequences, empty chunks and long ones beside each other, `most` in all."""
    rows = [rng.choice([0, 1, 1, rng.randint(0, 6), rng.randint(0, 40)]) for _ in range(seqs)]
    while sum(rows) > most:
        rows[rng.randrange(seqs)] = 0
    return rows if sum(rows) else [1] + rows[1:]


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("name", ["shares64", "thin128", "clusters64", "clusters128"])
def test_drawn_batches(name, seed):
    rng = random.Random(name + str(seed))
    dim = ROUTES[name][3]
    for i in range(10):
        G, seqs = rng.choice([1, 2, 3, 4, 5, 7, 8, 11, 16, 32]), rng.choice([1, 2, 3, 5, 9, 20])
        hkv = rng.choice([1, 2, 4])
        per = 16 if name == "shares64" and G <= 16 else 32
        if per * seqs < G:
            continue
        if name == "shares64" and G > 16:   # (a unit of 32 rows, no more than 16 on average)
            seqs = max(seqs, 2)
            per = 16
        rows = drawn_rows(rng, seqs, per * seqs // G)
        if sum(rows) * G > per * seqs:
            continue
        short = name.startswith("clusters")
        lens = [max(0, n + rng.choice([0, -3, 1, rng.randint(0, 200), 63, 64, 65, 127, 128, rng.randint(0, 700 if short else 4000)])) for n in rows]
        width = 12 if short else 64 * 19
        lens = [min(L, width * PG) for L in lens]
        case(ROUTES[name][0], rows, lens, G * hkv, hkv, dim, seed=i, width=width)


def steep(cache, rise, hq):
    """Keys that follow one direction, more so towards slot 0 (whence walks come: from the last slot down), so that the scores of a
    query along it rise by `rise` in all, and values that fall as the weights rise: whatever a maximum outgrown on the way does to what
    had been added up before shows in the result.  -> queries along the direction by 1, 0.5, 0.1 and -1."""
    g = torch.Generator().manual_seed(5)
    u = torch.randint(0, 2, (cache.dim,), generator=g).double() * 2 - 1
    for b, L in enumerate(cache.lens):
        for j in range(L):
            page, at = int(cache.table[b, j // PG]), j % PG
            z = rise * (1 - j / L)
            cache.k[page, :, at] = (0.3 * torch.randn(cache.hkv, cache.dim, generator=g) + u.float() * (z / math.sqrt(cache.dim))).to(torch.bfloat16)
            cache.v[page, :, at] = (torch.randn(cache.hkv, cache.dim, generator=g) * 2.0 ** round(-z * math.log2(math.e))).to(torch.bfloat16)

    def along(n):
        c = torch.tensor([(1.0, 0.5, 0.1, -1.0)[i % 4] for i in range(n * hq)]).reshape(n, hq, 1)
        return (0.05 * torch.randn(n, hq, cache.dim, generator=g) + c * u.float()).to(torch.bfloat16)
    return along


@every_route
@pytest.mark.parametrize("rise", [60.0, 25.0])
def test_maxima_that_are_outgrown_on_the_way(route, rise):
    """Scores: fp32 dot products of `dim` terms, off by at most dim 2^-24 times the sum of the terms' sizes; a weight and the sum that it is
    divided by are off by that much, relative, and by 7.5e-5 (a quarter of the exponentials) each."""
    _, hq, hkv, dim, _, per = ROUTES[route]
    short = route.startswith("clusters")
    cache = cache_of(route, [760, 700] if short else [3000, 2000])
    along = steep(cache, rise, hq)
    rows = [per, max(1, per - 1)]
    q = along(sum(rows))
    o, lse = attend(route, cache, q, cu_of(rows))
    scale = dim ** -0.5
    want, want_lse, size = attn_ref(cache, q, rows, scale)
    terms = max(float(torch.einsum("ihd,hjd->ihj", q[:, ::hq // hkv].double().abs(), cache.rows(cache.k, b).abs()).max()) for b in range(2))
    slack = dim * 2.0 ** -24 * terms * scale + 7.5e-5 + 1e-5
    assert torch.isfinite(o.float()).all()
    over = (o.cpu().double() - want).abs() - ((BF16_HALF + 2 * slack) * size + BF16_HALF * want.abs())
    assert (over / size).max() <= 0, f"O off by {float((over / size).max()):.3g} of the sum of its terms' sizes more than allowed"
    assert ((lse.cpu().double() - want_lse).abs() - slack - want_lse.abs() * 2.0 ** -22).max() <= 0


@every_route
@pytest.mark.parametrize("waste", [float("inf"), float("-inf"), 3e38])
def test_what_lies_behind_the_end_does_not_matter(route, waste):
    """(The other tests hold NaN there.)"""
    _, hq, _, dim, _, per = ROUTES[route]
    lens, rows = [65, 100, 64, 700], [per, max(1, per - 1), 0, per]
    q, results = queries(sum(rows), hq, dim), []
    for w in (waste, 0.0):
        results.append(attend(route, cache_of(route, lens, seed=3, waste=w), q, cu_of(rows)))
    assert all(torch.equal(x, y) for x, y in zip(*results))


@every_route
def test_rows_of_no_sequence_are_left_as_they_were(route):
    _, hq, _, dim, _, per = ROUTES[route]
    rows, lens, first = [per - 1, 0, max(1, per - 1), 1], [50, 20, 300, 64], 2
    if per == 1:
        rows = [0, 0, 1, 0]
    n = sum(rows)
    cache = cache_of(route, lens)
    q = queries(n + 3, hq, dim)
    q[:first], q[first + n:] = float("nan"), float("nan")
    o, lse = attend(route, cache, q, cu_of(rows, first))
    for x in (o, lse):
        assert (x[:first] == 7).all() and (x[first + n:] == 7).all()
    check_attn(o[first:first + n], lse[first:first + n], attn_ref(cache, q[first:first + n], rows, dim ** -0.5))


@every_route
def test_pages_and_lengths_that_are_none(route):
    """Of a sequence with pages outside the cache, and of one whose length exceeds the table, every result is some number; the third's are its own."""
    _, hq, _, dim, _, per = ROUTES[route]
    cache = cache_of(route, [300, 70, 200], waste=1.0)
    rows = [per] * 3
    q = queries(sum(rows), hq, dim)
    want = attn_ref(cache, q, rows, dim ** -0.5)
    d = cache.device()
    d["table"][0, 1], d["table"][0, 3], d["lens"][1] = 10 ** 6, -5, 2 ** 31 - 1
    o, lse = attend(route, cache, q, cu_of(rows), dev=d)
    assert torch.isfinite(o.float()).all() and torch.isfinite(lse).all()
    check_attn(o[2 * per:], lse[2 * per:], tuple(x[2 * per:] for x in want))


@every_route
def test_empty_caches_and_queries_that_see_nothing(route):
    """Chunks longer than their cache, and of caches that hold nothing or say less than nothing."""
    _, hq, hkv, dim, _, per = ROUTES[route]
    rows, lens = [per, per, 0, per], [0, -1, 40, max(1, per // 2)]
    case_lens = [max(0, x) for x in lens]
    cache = cache_of(route, case_lens)
    cache.lens = lens
    q = queries(sum(rows), hq, dim)
    o, lse = attend(route, cache, q, cu_of(rows))
    check_attn(o, lse, attn_ref(cache, q, rows, dim ** -0.5), route)


@every_route
def test_in_a_graph_with_other_lengths_and_on_a_side_stream(route):
    kernels, hq, hkv, dim, width, per = ROUTES[route]
    rows, lens = [per, max(1, per - 1), per], [700, 300, 250]
    cache = cache_of(route, lens)
    n = sum(rows)
    d, q, cu = cache.device(), queries(n, hq, dim).to(DEV), cu_of(rows).to(DEV)
    ws = attn_workspace(3, n, hq, hkv, dim, width)
    late, o, lse = torch.full_like(q, float("nan")), torch.empty_like(q), torch.empty(n, hq, device=DEV)

    def call(x, stream=None):
        ug.unigist_chunk_attn(x, cu, d["k"], d["v"], d["table"], d["lens"], o, lse, ws, stream=stream)

    assert launched(lambda: call(q)) == kernels
    want = o.clone(), lse.clone()
    check_attn(*want, attn_ref(cache, q.cpu(), rows, dim ** -0.5))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)
        late.copy_(q)
    call(late, side)
    side.synchronize()
    assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(q)
    for _ in range(3):
        o.zero_(), lse.zero_(), ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
    d["lens"].copy_(torch.tensor([64, 299, 1], dtype=torch.int32))
    graph.replay()
    cache.lens = [64, 299, 1]
    check_attn(o, lse, attn_ref(cache, q.cpu(), rows, dim ** -0.5))
    ug.unigist_device_status()


@pytest.mark.parametrize("route", [r for r in sorted(ROUTES) if not r.startswith("rows")])   # (which never take one token of a group of four)
def test_one_token_over_caches_around_pages_and_tiles(route):
    _, hq, _, dim, _, _ = ROUTES[route]
    lens = [1, 2, 63, 64, 65, 127, 128, 129, 191, 192, 193, 256, 257, 700]
    cache = cache_of(route, lens)
    for b, L in enumerate(lens):
        rows = [int(i == b) for i in range(len(lens))]
        q = queries(1, hq, dim, L)
        o, lse = attend(route, cache, q, cu_of(rows))
        check_attn(o, lse, attn_ref(cache, q, rows, dim ** -0.5), f"{route} {L}")


@every_route
def test_boundaries_of_any_value(route):
    """Ends below the start, past the rows and down to the least int: such a sequence has no rows, the others have theirs."""
    _, hq, hkv, dim, _, per = ROUTES[route]
    lens, n = [200, 130, 300, 90], 4 * per
    m = max(1, n // 3)
    cache = cache_of(route, lens, waste=1.0)
    q = queries(n, hq, dim)
    cu = torch.tensor([n - 1, LEAST, m, 2 ** 31 - 1, LEAST + 3], dtype=torch.int32)   # rows: none, 0 .. m, m .. n, none
    rows = [0, m, n - m, 0]
    want = attn_ref(cache, q, rows, dim ** -0.5)
    o, lse = attend(route, cache, q, cu)
    check_attn(o, lse, want, route)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n", [4, 200])
def test_weights_and_append_with_boundaries_of_any_value(dim, n):
    from chunk_util import Cache

    lens, hq, hkv, m = [200, 130, 300, 90], 8, 2, max(1, n // 3)
    cache = Cache(lens, hkv, dim, waste=1.0, room=n)
    q = queries(n, hq, dim)
    cu = torch.tensor([n - 1, LEAST, m, 2 ** 31 - 1, LEAST + 3], dtype=torch.int32)
    rows = [0, m, n - m, 0]
    lse = attn_ref(cache, q, rows, dim ** -0.5)[1].float()
    lse[lse == -float("inf")] = 0.0
    d = cache.device()
    out = torch.full_like(d["w"], 5.0)
    ug.unigist_cache_weigh(q.to(DEV), cu.to(DEV), lse.to(DEV), d["k"], d["table"], d["lens"], d["w"], out)
    ug.unigist_device_status()
    for b, w in weigh_ref(cache, q, rows, lse, dim ** -0.5, 1.0, cache.w).items():
        assert ((cache.rows(out, b) - w).abs() - 1e-4 * w).max() <= 1e-30, b   # (the bound of the tests of that call)
    new_lens = torch.zeros(4, dtype=torch.int32, device=DEV)
    new = torch.randn(n, hkv, dim, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).to(DEV)
    ug.unigist_chunk_append(new, new, cu.to(DEV), d["k"], d["v"], d["table"], d["lens"], new_lens, d["w"])
    torch.cuda.synchronize()
    assert new_lens.tolist() == [a + b for a, b in zip(lens, rows)]
    for b, L in enumerate(lens):   # what was there is there
        assert torch.equal(cache.rows(d["k"], b, L), cache.rows(cache.k, b, L)) and torch.equal(cache.rows(d["w"], b, L), cache.rows(cache.w, b, L))
