"""The calls on chunks from several threads at once, each on a stream and with buffers of its own; the first CUDA call of each thread is one of
them (tensor maps want a context, and the driver's function that makes them is looked up by whoever comes first)."""
import subprocess
import sys
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu
ROOT = Path(__file__).resolve().parent.parent

SRC = """
import sys, threading
sys.path[:0] = [{root!r}, {tests!r}]
import torch
import paper_2509_15763_b200 as ug
from chunk_util import DEV, Cache, attn_ref, check_attn, cu_of

SIZES = [([5, 90], [300, 500], 8, 2, 128), ([1, 1], [700, 64], 8, 2, 64), ([40, 3], [200, 130], 4, 4, 64), ([2, 2], [1500, 90], 16, 4, 128)]
work = []
for i in range(8):
    rows, lens, hq, hkv, dim = SIZES[i % 4]
    n, cache = sum(rows), Cache(lens, hkv, dim, seed=i)
    d, q = cache.device(), torch.randn(n, hq, dim, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16)
    ws = torch.empty(ug.unigist_chunk_attn_workspace_bytes(2, n, hq, hkv, dim, cache.width), dtype=torch.uint8, device=DEV)
    pos = torch.arange(n, dtype=torch.int32, device=DEV)[None] * 0
    work.append(dict(rows=rows, cache=cache, d=d, q=q, qd=q.to(DEV), cu=cu_of(rows).to(DEV), ws=ws, pos=pos, rot=torch.empty_like(q, device=DEV),
                     o=torch.empty_like(q, device=DEV), lse=torch.empty(n, hq, device=DEV), w=torch.empty_like(d["w"]), stream=torch.cuda.Stream()))
torch.cuda.synchronize()
start, failed = threading.Barrier(8), []

def run(x):
    try:
        start.wait(60)
        d, s = x["d"], x["stream"]
        for _ in range(20):
            ug.unigist_rope_axes(x["qd"], x["rot"], x["pos"], [0] * (x["q"].shape[2] // 2), 10000.0 + len(x["rows"]), stream=s)   # (positions of zero: q itself)
            ug.unigist_chunk_attn(x["rot"], x["cu"], d["k"], d["v"], d["table"], d["lens"], x["o"], x["lse"], x["ws"], stream=s)
            ug.unigist_cache_weigh(x["rot"], x["cu"], x["lse"], d["k"], d["table"], d["lens"], None, x["w"], 0.0, stream=s)
    except BaseException as e:
        failed.append(e)

threads = [threading.Thread(target=run, args=(x,)) for x in work]
[t.start() for t in threads]
[t.join() for t in threads]
assert not failed, failed
ug.unigist_device_status()
for x in work:
    dim, c = x["q"].shape[2], x["cache"]
    check_attn(x["o"], x["lse"], attn_ref(c, x["q"], x["rows"], dim ** -0.5))
    for b, n in enumerate(x["rows"]):   # every query head gives its KV head's slots a weight of one in all, up to the bounds of either call
        total = c.rows(x["w"], b).sum(1)
        assert (total / (n * x["q"].shape[1] // c.hkv) - 1).abs().max() < 4e-4
print("done")
"""


def test_calls_of_several_threads_at_once():
    src = SRC.format(root=str(ROOT), tests=str(ROOT / "tests"))
    out = subprocess.run([sys.executable, "-c", src], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and out.stdout.strip() == "done", out.stdout + out.stderr
