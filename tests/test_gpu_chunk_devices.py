"""Every tensor of a call on chunks has to lie on the current device.  There is one device here: tensors of another are stood in for by tensors
without storage, which are refused by their device before anything asks for their address."""
import pytest
import torch

import paper_2509_15763_b200 as ug

from chunk_util import DEV

pytestmark = pytest.mark.gpu
BF16, I32, F32 = torch.bfloat16, torch.int32, torch.float32


class Elsewhere(torch.Tensor):
    @staticmethod
    def __new__(cls, size, dtype):
        return torch.Tensor._make_wrapper_subclass(cls, size, dtype=dtype, device="cuda:1")

    @classmethod
    def __torch_dispatch__(cls, func, types, args=(), kwargs=None):
        raise NotImplementedError


# S 2, 3 rows, 4 / 2 heads of 64, 4 pages, tables of 2
X = {"q": ((3, 4, 64), BF16), "k": ((3, 2, 64), BF16), "cu": ((3,), I32), "cache": ((4, 2, 64, 64), BF16), "table": ((2, 2), I32), "lens": ((2,), I32),
     "o": ((3, 4, 64), BF16), "lse": ((3, 4), F32), "ws": ((1 << 20,), torch.uint8), "w": ((4, 2, 64), F32), "pos": ((1, 3), I32), "kept": ((2, 2, 10), I32)}
CALLS = {
    "rope_axes": (["q", "q", "pos"], lambda t: ug.unigist_rope_axes(*t, [0] * 32, 10000.0)),
    "chunk_append": (["k", "k", "cu", "cache", "cache", "table", "lens", "lens", "w", "pos"], lambda t: ug.unigist_chunk_append(*t, [0] * 32, 10000.0)),
    "chunk_attn": (["q", "cu", "cache", "cache", "table", "lens", "o", "lse", "ws"], lambda t: ug.unigist_chunk_attn(*t)),
    "cache_weigh": (["q", "cu", "lse", "cache", "table", "lens", "w", "w"], lambda t: ug.unigist_cache_weigh(*t)),
    "cache_evict": (["cache", "cache", "w", "table", "lens", "table", "lens", "kept"], lambda t: ug.unigist_cache_evict(*t, 10)),
}


@pytest.mark.parametrize("call,i", [(c, i) for c, (names, _) in CALLS.items() for i in range(len(names))])
def test_a_tensor_of_another_device(call, i):
    names, run = CALLS[call]
    tensors = [torch.zeros(X[n][0], dtype=X[n][1], device=DEV) for n in names]
    tensors[i] = Elsewhere(*X[names[i]])
    before = ug.unigist_launch_count()
    with pytest.raises(ValueError, match="not on the current device"):
        run(tensors)
    assert ug.unigist_launch_count() == before
