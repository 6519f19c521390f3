"""The operators on packed tokens at the edges of what their description allows.  Formulas, bounds and helpers are those of test_gpu_packed."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2107_05377_amd as mt  # noqa: E402
import test_gpu_packed as base  # noqa: E402
from test_gpu_packed import PRECISIONS, normal, starts, within  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    mt.lib()


@pytest.mark.parametrize("precision", ["bf16", "fp32"])
@pytest.mark.parametrize("heads,kv_heads,d,length", [(2, 1, 64, 50), (2, 1, 80, 50), (3, 1, 8, 70), (2, 2, 24, 300), (4, 1, 72, 200), (1, 1, 120, 33)])
def test_attention_key_of_minus_infinity_at_any_width(precision, heads, kv_heads, d, length):
    """A key whose score is -infinity has weight 0: the result is that without the key, at whatever width.  (0 times -infinity makes the column of dq NaN in
    which the key is infinite, by the formula.)"""
    p, dt, u = PRECISIONS[precision]
    print(f"attention {precision} {heads}/{kv_heads} x {d}, a key of -infinity among {length}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(d + length)
    q, g = normal(gen, length, heads, d, dtype=dt), normal(gen, length, heads, d, dtype=dt)
    k, v = normal(gen, length, kv_heads, d, dtype=dt), normal(gen, length, kv_heads, d, dtype=dt)
    q[:, :, 0] = q[:, :, 0].abs() + 0.5
    bad = length // 3
    rest = [i for i in range(length) if i != bad]
    k[bad, :, 0] = -math.inf
    scale = 1 / math.sqrt(d)
    want, bound = base.attention_formula(q, k[rest].contiguous(), v[rest].contiguous(), g, [0, length], [0, length - 1], False, scale, u)
    qs = starts([length])
    ctx, lse = mt.op_packed_attention(p, q, k, v, qs, causal=False, want_lse=True)
    within(ctx, want["ctx"], bound["ctx"], "ctx")
    assert ((lse.double() - want["lse"]).abs() <= bound["lse"]).all()
    dq, dk, dv = mt.op_packed_attention_grad(p, g, q, k, v, ctx, lse, qs, causal=False)
    within(dq[..., 1:], want["dq"][..., 1:], bound["dq"][..., 1:], "dq")
    assert torch.isnan(dq[..., 0]).all()
    for name, got in (("dk", dk), ("dv", dv)):
        within(got[rest], want[name], bound[name], name)
        assert (got[bad] == 0).all(), name


@pytest.mark.parametrize("precision", ["bf16", "fp32"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("heads,d,length", [(1, 8, 50), (5, 24, 150), (3, 80, 150), (2, 104, 70)])
def test_attention_keys_not_seen_reach_nothing_at_any_width(precision, value, heads, d, length):
    base.test_attention_keys_not_seen_reach_nothing(precision, value, heads, d, length)


@pytest.mark.parametrize("precision", ["bf16", "fp32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,count", [(64, 100), (128, 300)])
def test_attention_of_long_prompts_among_single_tokens(precision, causal, d, count):
    """Keys dealt out to workgroups where two sequences have many tiles of rows, whose chunks are then fewer and longer than those of the others (3 of 1536 keys and
    1 of all 4000 instead of 8 of 512), and sequences without keys or queries."""
    seqs = [(1, 300 + 41 * (i % 23)) for i in range(count)]
    seqs[count // 2], seqs[count - 20], seqs[3], seqs[70] = (160, 4000), (48, 4000), (1, 0), (0, 600)
    base.check_attention(base.run_attention(precision, 8, 1, d, seqs, causal, before=2, behind=3))


@pytest.mark.parametrize("precision", ["bf16", "fp32"])
@pytest.mark.parametrize("heads,kv_heads,d,seqs", [
    (1, 1, 64, [(i % 5, i % 5) for i in range(1100)]), (2, 1, 128, [(i % 7, i % 6) for i in range(300)]), (1, 1, 80, [(i % 40, i % 45) for i in range(300)]),
    (2, 1, 64, [(1, 1 + 37 * i % 1500) for i in range(600)]), (2, 2, 128, [(1, 1 + 37 * i % 900) for i in range(300)]), (1, 1, 16, [(1, i % 3) for i in range(1025)])])
def test_attention_of_more_sequences_than_a_workgroup_looks_at_once(precision, heads, kv_heads, d, seqs):
    base.check_attention(base.run_attention(precision, heads, kv_heads, d, seqs, True, before=1, behind=1))


@pytest.mark.parametrize("precision", ["bf16", "fp32"])
@pytest.mark.parametrize("heads,kv_heads,d,length", [(96, 32, 24, 700), (80, 16, 64, 850), (48, 8, 128, 700)])
def test_attention_of_groups_that_do_not_divide_a_tile(precision, heads, kv_heads, d, length):
    """Groups of 3, 5 and 6 heads in calls large enough for 128 rows a workgroup."""
    base.check_attention(base.run_attention(precision, heads, kv_heads, d, [(length, length), (33, 40)], True))


@pytest.mark.parametrize("precision", ["bf16", "fp32"])
@pytest.mark.parametrize("n,v", [(5, 300), (64, 30), (200, 1000), (2048, 8200)])
def test_vocab_loss_of_tokens_that_are_sure(precision, n, v):
    """Large logits that float32 holds exactly, the label's often the largest: the loss has no error of the size of the logits' rounding steps (2^-7 here).

    With D the distance of a logit from its token's largest, a weight is off by D (2^-26 for the constant log2e + 2^-24 for its argument) + 2^-23 for exp2, and the
    label's argument by as much without exp2; the sum of v weights by (v / 64 + 72) 2^-24 and its logarithm by 2^-23 of itself.  D is at most 2 x 31.875 here."""
    p, dt, _ = PRECISIONS[precision]
    print(f"vocab loss {precision} {n} x 64 x {v}, sure", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(n + v)
    x, w = torch.zeros(n, 64, device="cuda"), torch.zeros(v, 64, device="cuda")
    x[:, 0], w[:, 0] = 1024.0, 125.0
    x[:, 5] = 2.0 ** torch.randint(-1, 2, (n,), generator=gen, device="cuda")
    w[:, 5] = -torch.randint(1, 256, (v,), generator=gen, device="cuda") / 8
    w[v // 2, 5] = 0.0
    labels = torch.randint(0, v, (n,), generator=gen, device="cuda", dtype=torch.int32)
    labels[::2] = v // 2
    loss, lse = mt.op_vocab_loss(p, x.to(dt), w.to(dt), labels)
    z = x.double() @ w.double().t()
    want = torch.logsumexp(z - 128000.0, 1) - z[torch.arange(n, device="cuda"), labels.long()] + 128000.0
    d = 63.75
    bound = (v / 64 + 72) * 2.0 ** -24 + 2 * d * (2.0 ** -26 + 2.0 ** -24) + 2.0 ** -23 + 2.0 ** -22 * want
    assert ((loss.double() - want).abs() <= bound).all(), (loss.double() - want).abs().max().item()
    assert (loss >= 0).all()
    assert ((lse.double() - torch.logsumexp(z, 1)).abs() <= 4 * 2.0 ** -24 * 128000).all()


def test_strides_of_dimensions_of_one():
    """The stride of a dimension of one says nothing: whatever it is, the result is that of the same tensor laid out anew."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    p, dt = mt.MT_BF16, torch.bfloat16

    def odd(t):                                              # the same values, 3 where a dimension is one
        return t.as_strided(t.shape, [3 if n == 1 else s for s, n in zip(t.stride(), t.shape)])

    for heads, kv_heads, n, m in ((4, 1, 1, 20), (1, 1, 1, 1), (1, 1, 9, 9), (4, 2, 1, 1)):
        q, k, v, g = (normal(gen, r, h, 64, dtype=dt) for r, h in ((n, heads), (m, kv_heads), (m, kv_heads), (n, heads)))
        qs, ks = starts([n]), starts([m])
        ctx, lse = mt.op_packed_attention(p, q, k, v, qs, ks, want_lse=True)
        grads = mt.op_packed_attention_grad(p, g, q, k, v, ctx, lse, qs, ks)
        assert torch.equal(mt.op_packed_attention(p, odd(q), odd(k), odd(v), qs, ks, out=odd(torch.empty_like(ctx))), ctx)
        got = mt.op_packed_attention_grad(p, odd(g), odd(q), odd(k), odd(v), odd(ctx), lse, qs, ks, out=[odd(torch.empty_like(t)) for t in grads])
        assert all(torch.equal(a, b) for a, b in zip(got, grads))
    ids, label, weight = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.ones(1, device="cuda")
    for v in (1, 30):
        x, w = normal(gen, 1, 64, dtype=dt), normal(gen, v, 64, dtype=dt)
        loss, lse = mt.op_vocab_loss(p, x, w, label)
        assert all(torch.equal(a, b) for a, b in zip(mt.op_vocab_loss(p, odd(x), odd(w), label), (loss, lse)))
        grads = mt.op_vocab_loss_grad(p, x, w, label, lse, weight)
        assert all(torch.equal(a, b) for a, b in zip(mt.op_vocab_loss_grad(p, odd(x), odd(w), label, lse, weight), grads))
        assert torch.equal(mt.op_embedding(p, odd(w), ids, out=odd(torch.empty_like(x))), w[:1])
        total = torch.zeros(v, 64, device="cuda")
        mt.op_embedding_grad(p, odd(x), ids, v, add_to=odd(total))
        assert torch.equal(total[:1], x.float())


@pytest.mark.parametrize("precision,n,h,v", [("bf16", 4160, 64, 70001), ("fp32", 4160, 128, 70001), ("fp32", 61, 64, 2100001), ("bf16", 70001, 64, 4111)])
def test_vocab_loss_gradient_in_several_pieces(precision, n, h, v):
    """More than 512 MB of dz: the vocabulary in pieces, whose dx is added up and whose last one is narrower."""
    p, dt, u = PRECISIONS[precision]
    assert -(-n // 64) * 64 * v * (2 if precision == "bf16" else 4) > 1 << 29
    print(f"vocab loss in pieces {precision} {n} x {h} x {v}", flush=True)
    x, w, labels, weight = base.make_loss(precision, n, h, v, 0.9)
    want, bound = base.loss_formula(x, w, labels, weight, u)
    loss, lse = mt.op_vocab_loss(p, x, w, labels)
    within(loss, want["loss"], bound["loss"], "loss")
    dx, dw = mt.op_vocab_loss_grad(p, x, w, labels, lse, weight)
    within(dx, want["dx"], bound["dx"], "dx")
    within(dw, want["dw"], bound["dw"] + 1.01 * (u + 2 * base.E) * want["dw"].abs(), "dw")
