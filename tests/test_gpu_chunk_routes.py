"""What the attention of chunks promises holds for each of the kernels that a call may take, named by the test: the sizes alone choose
among them, and a case that a change of the choice leads to another kernel fails."""
import pytest
import torch

import paper_2509_15763_b200 as ug

from chunk_routes import ROUTES, cache_of, launched
from chunk_util import DEV, PG, attn_ref, attn_workspace, check_attn, cu_of, weigh_ref

pytestmark = pytest.mark.gpu
LEAST = -2 ** 31
every_route = pytest.mark.parametrize("route", sorted(ROUTES))


def queries(n, hq, dim, seed=1):
    return torch.randn(n, hq, dim, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


def attend(route, cache, q, cu, dev=None, scale=0.0):
    """-> o, lse; the call's kernels are the route's."""
    kernels, hq, hkv, dim, width, _ = ROUTES[route]
    d = dev or cache.device()
    n, S = q.shape[0], d["table"].shape[0]
    o = torch.full((n, hq, dim), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((n, hq), 7.0, device=DEV)
    ws = attn_workspace(S, n, hq, hkv, dim, width)
    args = q.to(DEV), cu.to(DEV), d["k"], d["v"], d["table"], d["lens"], o, lse, ws, scale
    assert launched(lambda: ug.unigist_chunk_attn(*args)) == kernels
    ug.unigist_device_status()
    return o, lse


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
