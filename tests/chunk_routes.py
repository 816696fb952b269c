"""Calls of the attention of chunks that each of its kernels takes, by sizes alone (the widths of the tables among them, so that short
sequences will do), and the names of the kernels that a call has launched."""
from __future__ import annotations

import torch

import paper_2509_15763_b200 as ug

from chunk_util import Cache

# name: (kernels launched, query heads, KV heads, head size, pages of a table row, tokens per sequence that fit the route)
ROUTES = {
    "rows64": (["chunk_attn_sm100_kernel", "chunk_combine_kernel"], 8, 2, 64, 60, 40),
    "rows128": (["chunk_attn_sm100_kernel", "chunk_combine_kernel"], 8, 2, 128, 60, 40),
    "clusters64": (["chunk_few_kernel"], 8, 2, 64, 12, 4),
    "clusters128": (["chunk_few_kernel"], 8, 2, 128, 12, 4),
    "shares64": (["chunk_few_kernel", "chunk_combine_kernel"], 8, 2, 64, 400, 4),
    "shares64_one": (["chunk_few_kernel", "chunk_combine_kernel"], 8, 2, 64, 400, 1),
    "thin128": (["chunk_thin_sm100_kernel", "chunk_combine_kernel"], 8, 2, 128, 400, 8),
}


def launched(call):
    """-> names of the kernels that call() launches, in order."""
    torch.cuda.synchronize()
    ug.unigist_kernel_timing(True)
    call()
    torch.cuda.synchronize()
    names = [ug.unigist_kernel_timing_get(i)[0] for i in range(ug.unigist_kernel_timing_count())]
    ug.unigist_kernel_timing(False)
    return names


def cache_of(route, lens, seed=0, **kw):
    """A cache whose table is as wide as the route wants it: the entries behind a sequence's pages name no page."""
    _, _, hkv, dim, width, _ = ROUTES[route]
    return widened(Cache(lens, hkv, dim, seed=seed, **kw), width)


def widened(cache, width):
    assert cache.width <= width, "the sequences outgrow the table"
    wide = torch.full((len(cache.lens), width), -7, dtype=torch.int32)
    wide[:, ::2] = 2 ** 30
    wide[:, : cache.width] = cache.table
    cache.table, cache.width = wide, width
    return cache
