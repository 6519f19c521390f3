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
