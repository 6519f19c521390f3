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


# ---- offsets that 32 bits do not hold

def test_attention_of_keys_beyond_4_gb():
    """A sequence whose keys lie more than 4 GB (and 2^31 elements) into the cache: forward pass and gradient are those of the same sequence alone."""
    p, dt = mt.MT_BF16, torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(9)
    far, n = (1 << 24) + 77, 700
    q, g = normal(gen, 3, 4, 64, dtype=dt), normal(gen, 3, 4, 64, dtype=dt)
    k, v = (torch.zeros(far + n, 2, 64, dtype=dt, device="cuda") for _ in range(2))
    k[far:], v[far:] = normal(gen, n, 2, 64, dtype=dt), normal(gen, n, 2, 64, dtype=dt)
    qs, ks = torch.tensor([0, 0, 3], dtype=torch.int32, device="cuda"), torch.tensor([0, far, far + n], dtype=torch.int32, device="cuda")
    want = mt.op_packed_attention(p, q, k[far:].clone(), v[far:].clone(), starts([3]), starts([n]), want_lse=True)
    got = mt.op_packed_attention(p, q, k, v, qs, ks, want_lse=True)
    # (keys may be dealt out otherwise: sums of 700 terms in another order, weights rounded about another reference)
    assert ((got[0].double() - want[0].double()).abs() <= 2.0 ** -7 * (1 + want[0].double().abs())).all()
    assert ((got[1] - want[1]).abs() <= 2.0 ** -20 * (1 + want[1].abs())).all()
    alone = mt.op_packed_attention_grad(p, g, q, k[far:].clone(), v[far:].clone(), *want, starts([3]), starts([n]))
    grads = mt.op_packed_attention_grad(p, g, q, k, v, *want, qs, ks)
    assert torch.equal(grads[0], alone[0])
    for a, b in zip(grads[1:], alone[1:]):
        assert torch.equal(a[far:], b) and (a[:far:4099] == 0).all()


def test_embedding_beyond_4_gb():
    p, dt = mt.MT_BF16, torch.bfloat16
    v, h = (1 << 22) + 9, 1024
    table = torch.zeros(v, h, dtype=dt, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(3)
    table[-5:] = normal(gen, 5, h, dtype=dt)
    ids = torch.tensor([v - 1, 0, v - 5, v - 3, v - 1], dtype=torch.int32, device="cuda")
    assert torch.equal(mt.op_embedding(p, table, ids), table[ids.long()])
    grad = normal(gen, 5, h, dtype=dt)
    out = mt.op_embedding_grad(p, grad, ids, v)
    assert torch.equal(out[v - 5], grad[2]) and torch.equal(out[v - 3], grad[3]) and torch.equal(out[v - 1], (grad[0].float() + grad[4].float()).to(dt))
    assert (out[v - 2] == 0).all() and (out[1:v - 5:4099] == 0).all() and torch.equal(out[0], grad[1])


def test_vocab_loss_of_weights_beyond_4_gb():
    """Columns of zeros but for the last rows of the weights: their logits, gradients of x and of these rows are those of a small vocabulary with as many zeros
    reckoned in."""
    p, dt, u = PRECISIONS["bf16"]
    gen = torch.Generator(device="cuda").manual_seed(4)
    n, h, v, last = 70, 1024, (1 << 21) + 300, 299
    x = normal(gen, n, h, dtype=dt)
    w = torch.zeros(v, h, dtype=dt, device="cuda")
    w[-last:] = (normal(gen, last, h, dtype=torch.float32) / 4).to(dt)            # logits of +-8
    labels = torch.randint(v - last, v, (n,), generator=gen, device="cuda", dtype=torch.int32)
    weight = torch.randn(n, generator=gen, device="cuda") / n
    z = x.double() @ w[-last:].double().t()
    lse = torch.logsumexp(torch.cat([z, torch.full((n, 1), math.log(v - last), dtype=torch.float64, device="cuda")], 1), 1)
    at = (labels.long() - (v - last))[:, None]
    loss, got_lse = mt.op_vocab_loss(p, x, w, labels)
    # z to (h + 8) 2^-24 of its terms (sum of 1024 terms of 0.2: 1.3e-2), the sums of 2^21 equal weights in ranges of 128 and then in slices: 2^-24 x (128 + 2^21 / 128 / 16)
    e = 2 * (h + 8) * 2.0 ** -24 * (x.double().abs() @ w[-last:].double().abs().t()).amax(1) + (128 + 1100) * 2.0 ** -24 + 2.0 ** -21 * (1 + z.abs().amax(1))
    assert ((got_lse.double() - lse).abs() <= e + 2.0 ** -22 * lse).all()
    assert ((loss.double() - (lse - z.gather(1, at)[:, 0])).abs() <= 2 * e + 2.0 ** -22 * lse).all()
    dx, dw = mt.op_vocab_loss_grad(p, x, w, labels, got_lse, weight)
    dz = torch.exp(z - lse[:, None])
    dz.scatter_add_(1, at, torch.full((n, 1), -1.0, dtype=torch.float64, device="cuda"))
    dz *= weight.double()[:, None]
    ez = (2 * e[:, None] + u) * (dz.abs() + (torch.exp(z - lse[:, None]) * weight.double().abs()[:, None]))
    within(dx, dz @ w[-last:].double(), 1.01 * (ez @ w[-last:].double().abs() + (u + 4 * base.E) * (dz @ w[-last:].double()).abs()), "dx")
    want = dz.t() @ x.double()
    within(dw[-last:], want, 1.01 * (ez.t() @ x.double().abs() + (u + 4 * base.E) * want.abs()) + (n + 8) * base.E * (dz.abs().t() @ x.double().abs()), "dw")
    zero = (torch.exp(-lse) * weight.double()) @ x.double()
    size = (torch.exp(-lse) * weight.double().abs()) @ x.double().abs()
    within(dw[:v - last:40961], zero.expand(len(dw[:v - last:40961]), h), ((u + 2 * e.amax() + (n + 8) * base.E) * size + u * zero.abs()).expand(len(dw[:v - last:40961]), h), "dw of zeros")


def test_captured_single_tokens_whose_lengths_change():
    """Two graphs of dealt-out keys in one pool, each replayed over other lengths than those it was captured with: the bits of the eager calls."""
    p, dt = mt.MT_BF16, torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(6)
    heads, kv_heads, total = 16, 4, 20000
    lengths = [[5000, 1, 0, 700, 9000, 64, 300, 1200], [0, 0, 19000, 1, 1, 1, 500, 497], [2500] * 8, [1] * 8]
    q, k, v = normal(gen, 8, heads, 128, dtype=dt), normal(gen, total, kv_heads, 128, dtype=dt), normal(gen, total, kv_heads, 128, dtype=dt)
    qs, tables = starts([1] * 8), [starts(n) for n in lengths]
    eager = [[t.clone() for t in mt.op_packed_attention(p, q, k, v, qs, t, want_lse=True)] for t in tables]
    live = [tables[0].clone(), tables[1].clone()]
    graphs, outs = [], []
    for t in live:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=graphs[0].pool() if graphs else None):
            outs.append(mt.op_packed_attention(p, q, k, v, qs, t, want_lse=True))
        graphs.append(graph)
    for turn in range(6):
        for i in (0, 1):
            live[i].copy_(tables[(turn + i) % 4])
            graphs[i].replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs[i], eager[(turn + i) % 4])), (turn, i)
            mt.op_packed_attention(p, q, k, v, qs, tables[turn % 4])
