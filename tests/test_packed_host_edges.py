"""Host side of the operators on packed tokens: sizes of workspaces, sizes and strides that the binding is given.  None of these needs a GPU."""
import ctypes as C
import random

import pytest

import paper_2107_05377_amd as mt
from paper_2107_05377_amd import binding


def attention_work(n_seqs, total_q, total_k, heads, kv_heads, width, precision=mt.MT_BF16):
    op = binding.mt_packed_attention(precision=precision, n_seqs=n_seqs, heads=heads, kv_heads=kv_heads, width=width, total_q=total_q, total_k=total_k,
                                     causal=1, scale=0.125)
    return mt.lib().mt_op_packed_attention_work(C.byref(op), 0)


# a workgroup's partial sums: 32 rows of 128 columns and two statistics (and two floats for their alignment)
PARTIAL = 32 * (128 + 4) * 4


@pytest.mark.parametrize("n_seqs,queries,keys,heads,kv_heads", [(500, 1, 2000, 32, 1), (800, 1, 1000, 8, 1), (256, 1, 2000, 32, 2), (256, 1, 4096, 32, 1),
                                                                (256, 4, 2600, 8, 1), (200, 1, 4096, 32, 4)])
def test_attention_workspace_of_many_sequences(n_seqs, queries, keys, heads, kv_heads):
    """Partial sums of a few thousand workgroups, not of the product of all rows and all keys."""
    need = attention_work(n_seqs, n_seqs * queries, n_seqs * keys, heads, kv_heads, 128)
    assert 0 < need <= 5120 * PARTIAL


def test_attention_workspace_over_the_whole_range():
    """At least what the chunks of equal sequences need (two workgroups a compute unit: 512), at most 5120 partial sums."""
    rng = random.Random(4)
    some = 0
    for _ in range(3000):
        kv_heads = rng.randint(1, 64)
        heads = kv_heads * rng.choice([1, 2, 3, 4, 8, 32])
        n_seqs = int(2 ** rng.uniform(0, 14))
        total_q, total_k = int(n_seqs * 2 ** rng.uniform(0, 6)), int(n_seqs * 2 ** rng.uniform(0, 15))
        if total_k > 1 << 29 or total_q * (heads // kv_heads) > 1 << 29:
            continue
        need = attention_work(n_seqs, total_q, total_k, heads, kv_heads, 128, rng.choice([mt.MT_BF16, mt.MT_FP32_CHECK]))
        assert need <= 5120 * PARTIAL
        some += need > 0
    assert some > 100


class Tensor:
    """What the binding looks at of a tensor on GPU 0, without its memory."""

    def __init__(self, *shape, dtype):
        self.shape, self.dtype, self.device = shape, dtype, "cuda:0"

    def get_device(self):
        return 0

    def stride(self, i=None):
        step = [1]
        for n in self.shape[:0:-1]:
            step.insert(0, step[0] * n)
        return tuple(step) if i is None else step[i]

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x10000


def test_binding_refuses_sizes_beyond_32_bits():
    """A size that the entry points' integers cannot hold is refused, not cut: 2^32 + 5 rows are not 5."""
    torch = pytest.importorskip("torch")
    far, bf, i32, f32 = (1 << 32) + 5, torch.bfloat16, torch.int32, torch.float32
    table, ids, rows = Tensor(far, 64, dtype=bf), Tensor(3, dtype=i32), Tensor(3, 64, dtype=bf)
    q, k, st = Tensor(3, 2, 64, dtype=bf), Tensor(far, 2, 64, dtype=bf), Tensor(2, dtype=i32)
    for call in (lambda: mt.op_embedding(mt.MT_BF16, table, ids, out=rows), lambda: mt.op_embedding(mt.MT_BF16, rows, Tensor(far, dtype=i32), out=table),
                 lambda: mt.op_embedding_grad(mt.MT_BF16, rows, ids, far), lambda: mt.op_embedding_grad(mt.MT_BF16, rows, ids, -1),
                 lambda: mt.op_embedding_grad(mt.MT_BF16, table, Tensor(far, dtype=i32), 10),
                 lambda: mt.op_embedding_grad(mt.MT_BF16, rows, ids, far, add_to=Tensor(far, 64, dtype=f32)),
                 lambda: mt.op_vocab_loss(mt.MT_BF16, rows, table, ids), lambda: mt.op_vocab_loss(mt.MT_BF16, table, rows, Tensor(far, dtype=i32)),
                 lambda: mt.op_vocab_loss_grad(mt.MT_BF16, rows, table, ids, Tensor(3, dtype=f32), Tensor(3, dtype=f32)),
                 lambda: mt.op_packed_attention(mt.MT_BF16, q, k, k, st, st, out=q), lambda: mt.op_packed_attention(mt.MT_BF16, q, q, q, Tensor(far, dtype=i32), out=q),
                 lambda: mt.op_packed_attention_grad(mt.MT_BF16, q, q, k, k, q, Tensor(2, 3, dtype=f32), st, st, out=(q, k, k))):
        with pytest.raises(mt.MTError):
            call()


@pytest.mark.parametrize("scale", [1e39, float("inf"), float("nan"), 0.0, -1.0])
def test_binding_refuses_scales(scale):
    torch = pytest.importorskip("torch")
    q, st = Tensor(3, 2, 64, dtype=torch.bfloat16), Tensor(2, dtype=torch.int32)
    with pytest.raises(mt.MTError):
        mt.op_packed_attention(mt.MT_BF16, q, q, q, st, scale=scale, out=q)
