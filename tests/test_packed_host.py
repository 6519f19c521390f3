"""Refusals of the operators on packed tokens: every check is made on the host before anything is enqueued, so none of these needs a GPU."""
import ctypes as C

import pytest

import paper_2107_05377_amd as mt
from paper_2107_05377_amd import binding

FAKE = 0x10000


def attention(**change):
    """A call that would be accepted, but for `change`."""
    f = dict(precision=mt.MT_BF16, n_seqs=2, heads=4, kv_heads=2, width=64, total_q=10, total_k=12, causal=1, scale=0.125, work_bytes=1 << 40)
    for n, rows, heads in (("q", 10, 4), ("k", 12, 2), ("v", 12, 2), ("ctx", 10, 4), ("grad_ctx", 10, 4), ("grad_q", 10, 4), ("grad_k", 12, 2), ("grad_v", 12, 2)):
        f.update({n + "_row": heads * 64, n + "_head": 64, "d_" + n: FAKE})
    f.update(d_lse=FAKE, d_q_start=FAKE, d_k_start=FAKE, d_work=FAKE)
    f.update(change)
    return binding.mt_packed_attention(**f)


@pytest.mark.parametrize("grad", [0, 1])
@pytest.mark.parametrize("change,code", [
    ({"d_q": None}, mt.MT_ERR_NULL), ({"d_v": None}, mt.MT_ERR_NULL), ({"d_ctx": None}, mt.MT_ERR_NULL), ({"d_q_start": None}, mt.MT_ERR_NULL),
    ({"precision": mt.MT_FP8_FFN}, mt.MT_ERR_CONFIG), ({"precision": 9}, mt.MT_ERR_CONFIG), ({"n_seqs": 0}, mt.MT_ERR_SHAPE), ({"n_seqs": 16385}, mt.MT_ERR_SHAPE),
    ({"heads": 5}, mt.MT_ERR_SHAPE), ({"kv_heads": 0}, mt.MT_ERR_SHAPE), ({"width": 0}, mt.MT_ERR_SHAPE), ({"width": 60}, mt.MT_ERR_SHAPE),
    ({"width": 136}, mt.MT_ERR_SHAPE), ({"total_q": 0}, mt.MT_ERR_SHAPE), ({"total_k": -1}, mt.MT_ERR_SHAPE), ({"total_k": (1 << 29) + 1}, mt.MT_ERR_SHAPE),
    ({"total_q": (1 << 28) + 1}, mt.MT_ERR_SHAPE), ({"scale": 0.0}, mt.MT_ERR_SHAPE), ({"scale": -1.0}, mt.MT_ERR_SHAPE), ({"scale": float("nan")}, mt.MT_ERR_SHAPE),
    ({"scale": float("inf")}, mt.MT_ERR_SHAPE), ({"d_k": FAKE + 8}, mt.MT_ERR_SHAPE), ({"k_row": 132}, mt.MT_ERR_SHAPE), ({"v_head": -64}, mt.MT_ERR_SHAPE)])
def test_attention_refusals(change, code, grad):
    L = mt.lib()
    call = L.mt_op_packed_attention_grad if grad else L.mt_op_packed_attention
    assert call(C.byref(attention(**change)), None) == code
    if code != mt.MT_ERR_NULL and not any(n.startswith("d_") or n.endswith(("_row", "_head")) for n in change):
        assert L.mt_op_packed_attention_work(C.byref(attention(**change)), grad) == 0


def test_attention_results_and_workspaces():
    L = mt.lib()
    assert L.mt_op_packed_attention(None, None) == L.mt_op_packed_attention_grad(None, None) == mt.MT_ERR_NULL
    for change in ({"ctx_row": 0}, {"ctx_head": 0}, {"ctx_row": 128, "ctx_head": 64}):           # heads of one row over those of the next
        assert L.mt_op_packed_attention(C.byref(attention(**change)), None) == mt.MT_ERR_SHAPE
    for field in ("d_lse", "d_grad_ctx", "d_grad_q", "d_grad_k", "d_grad_v"):
        assert L.mt_op_packed_attention_grad(C.byref(attention(**{field: None})), None) == mt.MT_ERR_NULL
    for change in ({"grad_q_head": 0}, {"grad_k_row": 64}, {"grad_v_head": 0}, {"d_grad_k": FAKE + 4}, {"grad_ctx_row": 7}):
        assert L.mt_op_packed_attention_grad(C.byref(attention(**change)), None) == mt.MT_ERR_SHAPE
    need = L.mt_op_packed_attention_work(C.byref(attention()), 1)
    assert need >= 10 * 4 * 4                                                                    # a float per head and query
    for change in ({"work_bytes": need - 1}, {"d_work": None}, {"d_work": FAKE + 16}):
        assert L.mt_op_packed_attention_grad(C.byref(attention(**change)), None) == mt.MT_ERR_SHAPE


@pytest.mark.parametrize("change,code", [
    ({"x": None}, mt.MT_ERR_NULL), ({"W": None}, mt.MT_ERR_NULL), ({"labels": None}, mt.MT_ERR_NULL), ({"lse": None}, mt.MT_ERR_NULL),
    ({"precision": mt.MT_FP8_LAYER}, mt.MT_ERR_CONFIG), ({"tokens": 0}, mt.MT_ERR_SHAPE), ({"hidden": 96}, mt.MT_ERR_SHAPE), ({"hidden": 0}, mt.MT_ERR_SHAPE),
    ({"vocab": 0}, mt.MT_ERR_SHAPE), ({"vocab": (1 << 22) + 1}, mt.MT_ERR_SHAPE), ({"tokens": (1 << 23) + 1}, mt.MT_ERR_SHAPE), ({"x": FAKE + 2}, mt.MT_ERR_SHAPE), ({"ldx": 120}, mt.MT_ERR_SHAPE),
    ({"ldw": 132}, mt.MT_ERR_SHAPE), ({"work": None}, mt.MT_ERR_SHAPE), ({"work": FAKE + 128}, mt.MT_ERR_SHAPE), ({"bytes": -1}, mt.MT_ERR_SHAPE)])
def test_vocab_loss_refusals(change, code):
    L = mt.lib()
    a = dict(precision=mt.MT_BF16, x=FAKE, ldx=128, W=FAKE, ldw=128, labels=FAKE, loss=FAKE, lse=FAKE, weight=FAKE, dx=FAKE, dw=FAKE, tokens=5, hidden=128,
             vocab=100, work=FAKE, bytes=0)
    a.update({k: v for k, v in change.items() if k != "bytes"})
    for grad in (0, 1):
        size = L.mt_op_vocab_loss_work(a["precision"], a["tokens"], a["hidden"], a["vocab"], grad) + change.get("bytes", 0)
        if size < 0:
            size = 0
        if grad:
            rc = L.mt_op_vocab_loss_grad(a["precision"], a["x"], a["ldx"], a["W"], a["ldw"], a["labels"], a["lse"], a["weight"], a["dx"], a["dw"], 0, a["tokens"],
                                         a["hidden"], a["vocab"], a["work"], size, None)
        else:
            rc = L.mt_op_vocab_loss(a["precision"], a["x"], a["ldx"], a["W"], a["ldw"], a["labels"], a["loss"], a["lse"], a["tokens"], a["hidden"], a["vocab"],
                                    a["work"], size, None)
        assert rc == code, grad


def test_embedding_refusals():
    L = mt.lib()

    def look(precision=mt.MT_BF16, table=FAKE, ldt=64, ids=FAKE, scale=1.0, out=FAKE, ldo=64, n=3, vocab=10, hidden=64):
        return L.mt_op_embedding(precision, table, ldt, ids, scale, out, ldo, n, vocab, hidden, None)

    def grad(precision=mt.MT_BF16, grad=FAKE, ldg=64, ids=FAKE, scale=1.0, out=FAKE, ldt=64, f32=0, add=0, n=3, vocab=10, hidden=64, work=FAKE, size=1 << 40):
        return L.mt_op_embedding_grad(precision, grad, ldg, ids, scale, out, ldt, f32, add, n, vocab, hidden, work, size, None)

    assert look(table=None) == look(ids=None) == look(out=None) == grad(grad=None) == grad(ids=None) == grad(out=None) == mt.MT_ERR_NULL
    assert look(precision=mt.MT_FP8_FFN) == grad(precision=7) == mt.MT_ERR_CONFIG
    for bad in (dict(n=0), dict(vocab=0), dict(hidden=60), dict(hidden=0), dict(scale=float("nan"))):
        assert look(**bad) == grad(**bad) == mt.MT_ERR_SHAPE
    assert look(ldt=56) == look(ldo=68) == look(table=FAKE + 4) == look(out=FAKE + 8) == mt.MT_ERR_SHAPE
    assert grad(n=(1 << 24) + 1) == grad(ldg=0) == grad(ldt=68) == grad(out=FAKE + 4) == grad(add=1) == mt.MT_ERR_SHAPE            # (adding needs float32)


def test_work_sizes_of_the_largest_calls_fit_their_type():
    L = mt.lib()
    assert 0 < L.mt_op_vocab_loss_work(mt.MT_BF16, 1 << 20, 4096, 1 << 18, 1) < 1 << 40
    assert L.mt_op_vocab_loss_work(mt.MT_BF16, 0, 4096, 1 << 18, 1) == L.mt_op_embedding_grad_work(mt.MT_BF16, 4, 10, 60) == 0
