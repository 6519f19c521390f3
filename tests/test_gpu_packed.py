"""The operators on packed tokens against their formulas in float64, at the sizes and masks where tiles, remainders and empty rows can go wrong.

Bounds.  U is half a rounding step of the tensors' type (bfloat16 2^-8, float32 2^-24, relative).  A float32 sum of n products is off by at most
(n + 8) 2^-24 times the sum of their magnitudes.  A score is such a sum, so a weight exp(score - lse) is off by the factor exp(e), e <= 2 (error of the
scores of its row) + the error of the row's sum + 2^-21 (1 + largest |score|) for exp2, log2 and the scaled arguments.  bfloat16 rounds weights and
score gradients once more (U each), and results by U of their value.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2107_05377_amd as mt  # noqa: E402

E = 2.0 ** -24
PRECISIONS = {"bf16": (mt.MT_BF16, torch.bfloat16, 2.0 ** -8), "fp32": (mt.MT_FP32_CHECK, torch.float32, 2.0 ** -24)}


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    mt.lib()


def normal(gen, *shape, dtype):
    return torch.randn(*shape, generator=gen, device="cuda").to(dtype)


def within(got, want, bound, what):
    got = got.double()
    assert torch.isfinite(got).all(), what
    # below 2^-126 = 1.2e-38 float32 and bfloat16 keep no relative precision (weights and products there may be flushed to 0): up to 10^4 such terms, times
    # factors up to 10, are 1.2e-33
    off = ((got - want).abs() - bound).max().item() - 1.2e-33 if got.numel() else 0.0
    assert off <= 0, (what, off, (got - want).abs().max().item())


# ---- attention

def starts(lengths, first=0):
    out = [first]
    for n in lengths:
        out.append(out[-1] + n)
    return torch.tensor(out, dtype=torch.int32, device="cuda")


def attention_formula(q, k, v, g, qs, ks, causal, scale, u):
    """Results and their bounds, in float64, sequence by sequence and head by head."""
    r = {n: torch.zeros_like(t, dtype=torch.float64) for n, t in (("ctx", q), ("dq", q), ("dk", k), ("dv", v))}
    r["lse"] = torch.full((q.shape[1], q.shape[0]), -math.inf, dtype=torch.float64, device=q.device)
    b = {n: torch.zeros_like(t) for n, t in r.items()}
    group, d = q.shape[1] // k.shape[1], q.shape[2]
    for s in range(len(qs) - 1):
        iq, ik = slice(qs[s], qs[s + 1]), slice(ks[s], ks[s + 1])
        lq, lk = qs[s + 1] - qs[s], ks[s + 1] - ks[s]
        if lq == 0 or lk == 0:
            continue
        see = torch.ones(lq, lk, dtype=torch.bool, device=q.device)
        if causal:
            see = see.tril(lk - lq)
        for a in range(q.shape[1]):
            qa, ka, va = q[iq, a].double(), k[ik, a // group].double(), v[ik, a // group].double()
            z = (qa @ ka.t() * scale).masked_fill(~see, -math.inf)
            lse = torch.logsumexp(z, -1)
            some = see.any(-1)
            p = torch.where(see & some[:, None], torch.exp(z - lse[:, None]), torch.zeros_like(z))
            zmax = torch.where(see, z.abs(), torch.zeros_like(z)).amax(-1)
            ez = torch.where(see, (d + 8) * E * scale * (qa.abs() @ ka.abs().t()), torch.zeros_like(z)).amax(-1)
            e = (2 * ez + (lk + 8) * E + 2.0 ** -21 * (1 + zmax))[:, None]
            c = p @ va
            r["ctx"][iq, a], r["lse"][a, iq] = c, lse
            bc = (u + e + (lk + 8) * E) * (p @ va.abs()) + (u + 2 * E) * c.abs()
            b["ctx"][iq, a], b["lse"][a, iq] = 1.01 * bc, e[:, 0] + 2 * E * lse.abs().nan_to_num(posinf=0.0)
            if g is None:
                continue
            ga = g[iq, a].double()
            dp, delta = ga @ va.t(), (ga * c).sum(-1, keepdim=True)
            ds = p * (dp - delta)
            ed = (d + 8) * E * (ga.abs() @ va.abs().t()) + (ga.abs() * (bc + (d + 8) * E * c.abs())).sum(-1, keepdim=True)
            es = (e + u + 2 * E) * ds.abs() + p * ed
            r["dq"][iq, a] = scale * ds @ ka
            b["dq"][iq, a] = 1.01 * (scale * (es + (lk + 8) * E * ds.abs()) @ ka.abs() + (u + 2 * E) * r["dq"][iq, a].abs())
            n = group * lq + 8
            r["dk"][ik, a // group] += scale * ds.t() @ qa
            b["dk"][ik, a // group] += 1.01 * scale * (es + n * E * ds.abs()).t() @ qa.abs()
            r["dv"][ik, a // group] += p.t() @ ga
            b["dv"][ik, a // group] += 1.01 * (p * (u + e + n * E)).t() @ ga.abs()
    for n in ("dk", "dv"):
        b[n] += 1.01 * (u + 2 * E) * r[n].abs()
    return r, b


def run_attention(precision, heads, kv_heads, d, seqs, causal, layout="apart", before=0, behind=0, scale=None, spoil=None, seed=0):
    """All of the operator on one set of sequences [(queries, keys)]; `before`, `behind`: rows of no sequence, filled with NaN."""
    p, dt, u = PRECISIONS[precision]
    print(f"attention {precision} {heads}/{kv_heads} x {d} {seqs[:6]} causal {causal} {layout}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(1000 + seed + heads + d + len(seqs))
    nq, nk = before + sum(s[0] for s in seqs) + behind, before + sum(s[1] for s in seqs) + behind
    nq, nk = max(nq, 1), max(nk, 1)
    if layout == "fused":
        x = normal(gen, nq, heads + 2 * kv_heads, d, dtype=dt)
        q, k, v = x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]
    elif layout == "heads":
        q = normal(gen, heads, nq, d, dtype=dt).transpose(0, 1)
        k, v = (normal(gen, kv_heads, nk, d, dtype=dt).transpose(0, 1) for _ in range(2))
    else:
        q, k, v = normal(gen, nq, heads, d, dtype=dt), normal(gen, nk, kv_heads, d, dtype=dt), normal(gen, nk, kv_heads, d, dtype=dt)
    g = normal(gen, nq, heads, d, dtype=dt)
    qs, ks = starts([s[0] for s in seqs], before), starts([s[1] for s in seqs], before)
    for t, st in ((q, qs), (g, qs), (k, ks), (v, ks)):
        t[:int(st[0])] = math.nan
        t[int(st[-1]):] = math.nan
    hq, hk = qs.tolist(), ks.tolist()
    keys = None if layout == "fused" else ks
    scale_ = 1 / math.sqrt(d) if scale is None else scale
    want, bound = attention_formula(q, k, v, g, hq, hk, causal, scale_, u)
    if spoil:
        spoil(q, k, v, g)
    out = torch.full((nq, heads, d), 7.0, dtype=dt, device="cuda")
    ctx, lse = mt.op_packed_attention(p, q, k, v, qs, keys, causal=causal, scale=scale, out=out, want_lse=True)
    grads = [torch.full(t.shape, 7.0, dtype=dt, device="cuda") for t in (q, k, v)]
    mt.op_packed_attention_grad(p, g, q, k, v, ctx, lse, qs, keys, causal=causal, scale=scale, out=grads)
    return dict(q=q, k=k, v=v, g=g, qs=qs, ks=keys, hq=hq, hk=hk, want=want, bound=bound, got=dict(ctx=ctx, dq=grads[0], dk=grads[1], dv=grads[2]), lse=lse)


def check_attention(r, rows=None):
    for n, st in (("ctx", r["hq"]), ("dq", r["hq"]), ("dk", r["hk"]), ("dv", r["hk"])):
        at = slice(st[0], st[-1])
        within(r["got"][n][at], r["want"][n][at], r["bound"][n][at], n)
        rest = torch.cat([r["got"][n][:st[0]], r["got"][n][st[-1]:]])
        assert (rest == 7).all(), n                                  # rows of no sequence are left as they were
    lse, want = r["lse"][:, r["hq"][0]:r["hq"][-1]].double(), r["want"]["lse"][:, r["hq"][0]:r["hq"][-1]]
    assert torch.equal(torch.isinf(lse), torch.isinf(want)) and not torch.isnan(lse).any()
    some = torch.isfinite(want)
    assert ((lse - want).abs()[some] <= r["bound"]["lse"][:, r["hq"][0]:r["hq"][-1]][some]).all()


MIXED = [(33, 33), (0, 0), (1, 1), (64, 64), (31, 31), (129, 129), (200, 200)]
CACHED = [(1, 61), (1, 1), (3, 130), (40, 200), (0, 9), (1, 300), (7, 7)]
EMPTY = [(5, 0), (70, 3), (1, 0), (0, 0), (140, 139)]                # causal: rows that see nothing


@pytest.mark.parametrize("precision", ["bf16", "fp32"])
@pytest.mark.parametrize("heads,kv_heads,d,seqs,causal,layout", [
    (2, 2, 64, [(1, 1)], True, "apart"), (3, 1, 64, MIXED, True, "fused"), (2, 2, 64, MIXED, False, "fused"), (8, 2, 128, MIXED, True, "heads"),
    (4, 4, 128, MIXED, False, "apart"), (6, 2, 64, CACHED, True, "heads"), (4, 1, 128, CACHED, False, "apart"), (2, 1, 64, EMPTY, True, "apart"),
    (2, 1, 128, EMPTY, False, "apart"), (1, 1, 8, MIXED, True, "apart"), (5, 5, 80, CACHED, True, "apart"), (8, 1, 24, MIXED, True, "fused"),
    (16, 2, 32, CACHED, True, "heads"), (3, 3, 104, EMPTY, True, "apart")])
def test_attention(precision, heads, kv_heads, d, seqs, causal, layout):
    check_attention(run_attention(precision, heads, kv_heads, d, seqs, causal, layout, before=3, behind=5))


@pytest.mark.parametrize("precision", ["bf16", "fp32"])
def test_attention_of_many_sequences(precision):
    check_attention(run_attention(precision, 2, 1, 64, [(i % 5, i % 5) for i in range(150)], True))
    check_attention(run_attention(precision, 2, 2, 64, [(1, 1 + i % 9) for i in range(65)], True))
    check_attention(run_attention(precision, 64, 64, 16, [(1, 1 + i % 40) for i in range(40)], True, "heads"))
    check_attention(run_attention(precision, 128, 64, 16, [(1, 150 + 70 * (i % 9)) for i in range(20)], True))


@pytest.mark.parametrize("precision", ["bf16", "fp32"])
@pytest.mark.parametrize("heads,kv_heads,d,seqs,causal", [(128, 64, 64, MIXED, True), (64, 64, 40, MIXED, False), (256, 64, 128, CACHED, True), (256, 64, 24, EMPTY, True)])
def test_attention_of_many_heads(precision, heads, kv_heads, d, seqs, causal):
    check_attention(run_attention(precision, heads, kv_heads, d, seqs, causal, before=2, behind=1))


@pytest.mark.parametrize("precision,heads,kv_heads,d,seqs,causal", [
    ("bf16", 4, 1, 64, [(1, 9001)], True), ("bf16", 4, 2, 128, [(2, 4097), (1, 100)], True), ("fp32", 2, 1, 64, [(1, 5003)], False),
    ("bf16", 2, 1, 64, [(1111, 1111), (90, 1500)], True), ("bf16", 1, 1, 128, [(700, 1300)], False),
    ("bf16", 128, 128, 16, [(2060, 2060)], True), ("bf16", 128, 128, 72, [(1700, 1701), (400, 400)], True), ("fp32", 128, 128, 8, [(2060, 2060)], False)])
def test_attention_of_long_sequences(precision, heads, kv_heads, d, seqs, causal):
    check_attention(run_attention(precision, heads, kv_heads, d, seqs, causal))


@pytest.mark.parametrize("precision", ["bf16", "fp32"])
def test_attention_of_starts_that_fall(precision):
    """Starts that fall name more chunks of keys than the workspace holds: those are left out, the first sequence is as if it were alone."""
    p, dt, _ = PRECISIONS[precision]
    gen = torch.Generator(device="cuda").manual_seed(11)
    q, k, v = normal(gen, 1, 4, 64, dtype=dt), normal(gen, 9001, 1, 64, dtype=dt), normal(gen, 9001, 1, 64, dtype=dt)
    qs, ks = torch.tensor([0, 1, 0, 1, 0, 1], dtype=torch.int32, device="cuda"), torch.tensor([0, 9001, 0, 9001, 0, 9001], dtype=torch.int32, device="cuda")
    got, alone = mt.op_packed_attention(p, q, k, v, qs, ks), mt.op_packed_attention(p, q, k, v, qs[:2], ks[:2])
    assert torch.equal(got, alone)


@pytest.mark.parametrize("precision", ["bf16", "fp32"])
def test_attention_of_large_scores(precision):
    """Scores of +-100 and more: weights of 0 and 1, a maximum that rises from tile to tile."""
    p, dt, _ = PRECISIONS[precision]
    n = 300
    k = torch.zeros(n, 1, 64, device="cuda")
    k[:, 0, 0] = torch.linspace(-40, 40, n, device="cuda")
    q = torch.zeros(n, 1, 64, device="cuda")
    q[:, 0, 0] = 8.0
    gen = torch.Generator(device="cuda").manual_seed(3)
    v, g = normal(gen, n, 1, 64, dtype=dt), normal(gen, n, 1, 64, dtype=dt)
    q, k = q.to(dt), k.to(dt)
    for order in (torch.arange(n), torch.arange(n - 1, -1, -1)):
        kk, qs = k[order.cuda()].contiguous(), starts([n])
        want, bound = attention_formula(q, kk, v, g, [0, n], [0, n], False, 0.5, PRECISIONS[precision][2])
        ctx, lse = mt.op_packed_attention(p, q, kk, v, qs, causal=False, scale=0.5, want_lse=True)
        grads = mt.op_packed_attention_grad(p, g, q, kk, v, ctx, lse, qs, causal=False, scale=0.5)
        for name, got in zip(("ctx", "dq", "dk", "dv"), (ctx,) + grads):
            within(got, want[name], bound[name], name)


@pytest.mark.parametrize("precision", ["bf16", "fp32"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("heads,d,length", [(1, 64, 50), (3, 128, 150)])
def test_attention_keys_not_seen_reach_nothing(precision, value, heads, d, length):
    """A key that only the queries behind it see spoils those alone, and a query's gradient none of the keys behind it."""
    bad = length - 7

    def spoil(q, k, v, g):
        k[bad], v[bad], q[bad], g[bad] = value, value, value, value

    r = run_attention(precision, heads, 1, d, [(length, length)], True, spoil=spoil)
    for n in ("ctx", "dq"):
        within(r["got"][n][:bad], r["want"][n][:bad], r["bound"][n][:bad], n)
        assert not torch.isfinite(r["got"][n][bad:]).all(-1).any(), n
    for n in ("dk", "dv"):                                   # (row `bad` sees all keys in front of it)
        assert not torch.isfinite(r["got"][n][:bad]).any(), n
    # an infinite value in front of finite ones stays what it is, with its sign
    if math.isinf(value):
        p = PRECISIONS[precision][0]
        q, k, v = r["q"].clone(), r["k"].clone(), r["v"].clone()
        q[bad], k[bad] = 1.0, 1.0
        ctx = mt.op_packed_attention(p, q, k, v, r["qs"])
        assert (ctx[bad:].float() == value).all() and torch.isfinite(ctx[:bad]).all()


def test_attention_gradient_against_differences():
    """d(sum of g ctx) along a direction, by central differences of the formula in float64."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    seqs = [(9, 9), (3, 20)]
    qs, ks = [0, 9, 12], [0, 9, 29]
    q, k, v, g = (normal(gen, n, h, 32, dtype=torch.float32) for n, h in ((12, 4), (29, 2), (29, 2), (12, 4)))
    sq, sk = starts([s[0] for s in seqs]), starts([s[1] for s in seqs])
    ctx, lse = mt.op_packed_attention(mt.MT_FP32_CHECK, q, k, v, sq, sk, want_lse=True)
    grads = mt.op_packed_attention_grad(mt.MT_FP32_CHECK, g, q, k, v, ctx, lse, sq, sk)

    def value(*x):
        return (attention_formula(x[0], x[1], x[2], None, qs, ks, True, 1 / math.sqrt(32), E)[0]["ctx"] * g.double()).sum()

    for i in range(3):
        way = torch.randn((q, k, v)[i].shape, generator=gen, device="cuda").double()
        h = 1e-5
        at = [t.double() for t in (q, k, v)]
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + h * way, at[i] - h * way
        slope = (value(*up) - value(*down)) / (2 * h)
        got = (grads[i].double() * way).sum()
        # the differences are good to h^2 and rounding / h, the gradient to about 100 sums of 2^-24
        assert abs(got - slope) <= 1e-4 * (grads[i].double() * way).abs().sum()


# ---- loss over the vocabulary

def loss_formula(x, w, labels, weight, u):
    n, h = x.shape
    v = w.shape[0]
    xd, wd = x.double(), w.double()
    has = (labels >= 0) & (labels < v)
    rows = torch.nonzero(has)[:, 0]
    r = {"loss": torch.zeros(n, dtype=torch.float64, device=x.device), "lse": torch.zeros(n, dtype=torch.float64, device=x.device), "dx": torch.zeros_like(xd),
         "dw": torch.zeros_like(wd)}
    b = {k: torch.zeros_like(t) for k, t in r.items()}
    xs, ls = xd[rows], labels[rows].long()
    z = xs @ wd.t()
    ez = ((h + 8) * E * (xs.abs() @ wd.abs().t())).amax(1, keepdim=True) if len(rows) else z[:, :1]
    lse = torch.logsumexp(z, 1, keepdim=True)
    e = 2 * ez + (v / 64 + 72) * E + 2.0 ** -21 * (1 + z.abs().amax(1, keepdim=True)) if len(rows) else ez
    at = torch.arange(len(rows), device=x.device)
    r["lse"][rows], r["loss"][rows] = lse[:, 0], lse[:, 0] - z[at, ls]
    b["lse"][rows], b["loss"][rows] = e[:, 0] + 2 * E * lse[:, 0].abs(), (2 * e)[:, 0] + 4 * E * lse[:, 0].abs()
    p = torch.exp(z - lse)
    g = weight[rows].double()[:, None]
    dz = p.clone()
    dz[at, ls] -= 1
    ed = (e * p + 2 * E * (p + dz.abs()) + u * dz.abs()) * g.abs()
    dz = dz * g
    m = len(rows) + 8
    r["dx"][rows] = dz @ wd
    b["dx"][rows] = 1.01 * ((ed + (v + 8) * E * dz.abs()) @ wd.abs() + (u + 2 * E) * r["dx"][rows].abs())
    r["dw"] = dz.t() @ xs
    b["dw"] = 1.01 * ((ed + m * E * dz.abs()).t() @ xs.abs())
    return r, b


def make_loss(precision, n, h, v, labelled, seed=0):
    p, dt, u = PRECISIONS[precision]
    gen = torch.Generator(device="cuda").manual_seed(77 + n + h + v + seed)
    x, w = normal(gen, n, h, dtype=dt), (normal(gen, v, h, dtype=torch.float32) / math.sqrt(h)).to(dt)
    labels = torch.randint(0, v, (n,), generator=gen, device="cuda", dtype=torch.int32)
    drop = torch.rand(n, generator=gen, device="cuda") >= labelled
    labels[drop] = torch.where(torch.rand(n, generator=gen, device="cuda") < 0.5, -100, v + 3).int()[drop]
    weight = torch.randn(n, generator=gen, device="cuda") / n
    return x, w, labels, weight


@pytest.mark.parametrize("precision", ["bf16", "fp32"])
@pytest.mark.parametrize("n,h,v,labelled", [(1, 64, 1, 1.0), (1, 768, 1000, 1.0), (5, 64, 127, 1.0), (33, 128, 129, 0.5), (64, 192, 2051, 1.0), (129, 320, 500, 0.9),
                                            (17, 64, 300, 0.5), (300, 768, 5003, 0.15), (1000, 64, 40, 0.7), (2100, 128, 8301, 0.9), (257, 1024, 4096, 1.0), (40, 64, 70, 0.0),
                                            (64, 128, 1000, 0.8), (34, 64, 515, 1.0), (65, 64, 700, 0.9)])
def test_vocab_loss(precision, n, h, v, labelled):
    print(f"vocab loss {precision} {n} x {h} x {v}", flush=True)
    p, dt, u = PRECISIONS[precision]
    x, w, labels, weight = make_loss(precision, n, h, v, labelled)
    want, bound = loss_formula(x, w, labels, weight, u)
    none = (labels < 0) | (labels >= v)
    x[none] = math.nan                                       # rows without a label are not read
    loss, lse = mt.op_vocab_loss(p, x, w, labels)
    within(loss, want["loss"], bound["loss"], "loss")
    within(lse, want["lse"], bound["lse"], "lse")
    for f32 in (False, True):
        dx, dw = mt.op_vocab_loss_grad(p, x, w, labels, lse, weight, out_f32=f32)
        within(dx, want["dx"], bound["dx"], "dx")
        r = 2.0 ** -24 if f32 else u
        within(dw, want["dw"], bound["dw"] + 1.01 * (r + 2 * E) * want["dw"].abs(), "dw")
        assert (dx[none] == 0).all()


@pytest.mark.parametrize("precision", ["bf16", "fp32"])
def test_vocab_loss_strided_rows_and_large_logits(precision):
    p, dt, u = PRECISIONS[precision]
    x, w, labels, weight = make_loss(precision, 70, 128, 900, 1.0)
    wide_x, wide_w = torch.full((70, 192), math.nan, dtype=dt, device="cuda"), torch.full((900, 256), math.nan, dtype=dt, device="cuda")
    wide_x[:, :128], wide_w[:, 64:192] = x * 30, w
    xs, ws = wide_x[:, :128], wide_w[:, 64:192]
    want, bound = loss_formula(xs, ws, labels, weight, u)
    loss, lse = mt.op_vocab_loss(p, xs, ws, labels)
    within(loss, want["loss"], bound["loss"], "loss")
    dx, dw = mt.op_vocab_loss_grad(p, xs, ws, labels, lse, weight)
    within(dx, want["dx"], bound["dx"], "dx")
    within(dw, want["dw"], bound["dw"] + 1.01 * (u + 2 * E) * want["dw"].abs(), "dw")


def test_vocab_loss_gradient_against_differences():
    x, w, labels, weight = make_loss("fp32", 21, 64, 333, 0.8)
    _, lse = mt.op_vocab_loss(mt.MT_FP32_CHECK, x, w, labels)
    grads = mt.op_vocab_loss_grad(mt.MT_FP32_CHECK, x, w, labels, lse, weight)
    gen = torch.Generator(device="cuda").manual_seed(8)
    for i in range(2):
        way = torch.randn((x, w)[i].shape, generator=gen, device="cuda").double()
        at = [x.double(), w.double()]
        sides = []
        for s in (1e-5, -1e-5):
            t = list(at)
            t[i] = at[i] + s * way
            sides.append((loss_formula(t[0], t[1], labels, weight, E)[0]["loss"] * weight.double()).sum())
        got = (grads[i].double() * way).sum()
        assert abs(got - (sides[0] - sides[1]) / 2e-5) <= 1e-4 * (grads[i].double() * way).abs().sum()


# ---- embedding

@pytest.mark.parametrize("precision", ["bf16", "fp32"])
@pytest.mark.parametrize("n,h,v,kind", [(1, 8, 1, "any"), (61, 768, 30522, "words"), (500, 64, 37, "any"), (1025, 520, 300, "one"), (3000, 24, 5000, "words"),
                                        (5000, 136, 100, "words"), (20011, 64, 1000, "one"), (33000, 72, 4000, "words"), (40000, 16, 70000, "any"), (140001, 8, 900, "words")])
def test_embedding(precision, n, h, v, kind):
    print(f"embedding {precision} {n} x {h} of {v}, {kind}", flush=True)
    p, dt, u = PRECISIONS[precision]
    gen = torch.Generator(device="cuda").manual_seed(n + h + v)
    table, grad = normal(gen, v, h, dtype=dt), normal(gen, n, h, dtype=dt)
    x = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    ids = {"any": x * v, "words": torch.exp(x * math.log(v)) - 1, "one": torch.full_like(x, v // 2)}[kind].long().clamp(0, v - 1).int()
    if n > 3:
        ids[1], ids[n - 1] = -1, v                           # outside the table
    scale = 1.7
    inside = (ids >= 0) & (ids < v)
    want = torch.where(inside[:, None], (table[ids.long().clamp(0, v - 1)].float() * scale).to(dt), torch.zeros_like(grad))
    assert torch.equal(mt.op_embedding(p, table, ids, scale=scale), want)
    assert torch.equal(mt.op_embedding(p, table, ids)[inside], table[ids[inside].long()])
    at = ids[inside].long()
    exact = torch.zeros(v, h, dtype=torch.float64, device="cuda").index_add_(0, at, grad[inside].double()) * scale
    size = torch.zeros(v, h, dtype=torch.float64, device="cuda").index_add_(0, at, grad[inside].double().abs()) * scale
    count = torch.bincount(at, minlength=v)[:, None]
    grad[~inside] = math.nan
    for f32 in (False, True):
        got = mt.op_embedding_grad(p, grad, ids, v, scale=scale, out_f32=f32)
        assert got.dtype == (torch.float32 if f32 else dt)
        within(got, exact, (count + 2) * E * size + (2.0 ** -24 if f32 else u) * exact.abs() * 1.01, "grad")
        assert (got[count[:, 0] == 0] == 0).all()
        assert torch.equal(got, mt.op_embedding_grad(p, grad, ids, v, scale=scale, out_f32=f32))
    start = normal(gen, v, h, dtype=torch.float32)
    total = start.clone()
    assert mt.op_embedding_grad(p, grad, ids, v, scale=scale, add_to=total) is total
    within(total, start.double() + exact, (count + 4) * E * (size + start.double().abs()), "sum")
    assert torch.equal(total[count[:, 0] == 0], start[count[:, 0] == 0])


def test_embedding_strided_rows():
    gen = torch.Generator(device="cuda").manual_seed(2)
    wide = normal(gen, 50, 96, dtype=torch.bfloat16)
    ids = torch.arange(49, -1, -1, device="cuda", dtype=torch.int32)
    out = torch.full((50, 80), 7.0, dtype=torch.bfloat16, device="cuda")
    mt.op_embedding(mt.MT_BF16, wide[:, 16:80], ids, out=out[:, :64])
    assert torch.equal(out[:, :64], wide[:, 16:80].flip(0)) and (out[:, 64:] == 7).all()
    got = mt.op_embedding_grad(mt.MT_BF16, wide[:, 16:80], ids, 60)
    assert torch.equal(got[:50], wide[:, 16:80].flip(0)) and (got[50:] == 0).all()


# ---- as they are used

def language_model_step(precision, p):
    """Loss and gradients of a one-layer language model with tied embeddings on packed sequences, by the operators."""
    ids, labels, weight, qs = p["ids"], p["labels"], p["weight"], p["starts"]
    heads, kv_heads, d = p["shape"]
    n, h = len(ids), p["table"].shape[1]
    scale = math.sqrt(h)
    lin = lambda a, w, **kw: mt.op_linear(precision, a.contiguous(), w.contiguous(), **kw)  # noqa: E731
    x = mt.op_embedding(precision, p["table"], ids, scale=scale)
    qkv = lin(x, p["wqkv"]).view(n, heads + 2 * kv_heads, d)
    q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
    ctx, lse_a = mt.op_packed_attention(precision, q, k, v, qs, want_lse=True)
    y = lin(ctx.view(n, -1), p["wo"])
    loss, lse = mt.op_vocab_loss(precision, y, p["table"], labels)
    dy, dtable = mt.op_vocab_loss_grad(precision, y, p["table"], labels, lse, weight, out_f32=True)
    dctx = lin(dy, p["wo"].t()).view(n, heads, d)
    dwo = dy.float().t() @ ctx.view(n, -1).float()
    dqkv = torch.empty_like(qkv)
    mt.op_packed_attention_grad(precision, dctx, q, k, v, ctx, lse_a, qs, out=(dqkv[:, :heads], dqkv[:, heads:heads + kv_heads], dqkv[:, heads + kv_heads:]))
    dwqkv = dqkv.view(n, -1).float().t() @ x.float()
    dx = lin(dqkv.view(n, -1), p["wqkv"].t())
    mt.op_embedding_grad(precision, dx, ids, len(p["table"]), scale=scale, add_to=dtable)
    return loss, dtable, dwqkv, dwo


def language_model(dtype, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    heads, kv_heads, d, h, v = 4, 2, 32, 128, 517
    lengths = [40, 1, 77, 0, 19]
    n = sum(lengths)
    ids = torch.randint(0, v, (n,), generator=gen, device="cuda", dtype=torch.int32)
    labels = torch.cat([ids[1:], ids[:1]])
    labels[torch.cumsum(torch.tensor([m for m in lengths if m]), 0).cuda() - 1] = -1       # the last token of a sequence predicts nothing
    has = labels >= 0
    return dict(ids=ids, labels=labels, weight=has.float() / has.sum(), starts=starts(lengths), shape=(heads, kv_heads, d), lengths=lengths,
                table=(normal(gen, v, h, dtype=torch.float32) / math.sqrt(h)).to(dtype),
                wqkv=(normal(gen, (heads + 2 * kv_heads) * d, h, dtype=torch.float32) / math.sqrt(h)).to(dtype),
                wo=(normal(gen, h, heads * d, dtype=torch.float32) / math.sqrt(heads * d)).to(dtype))


def language_model_reference(p):
    table, wqkv, wo = (p[n].double().requires_grad_() for n in ("table", "wqkv", "wo"))
    heads, kv_heads, d = p["shape"]
    x = table[p["ids"].long()] * math.sqrt(table.shape[1])
    qkv = (x @ wqkv.t()).view(len(x), -1, d)
    parts = []
    at = 0
    for m in p["lengths"]:
        q, k, v = (t.transpose(0, 1) for t in qkv[at:at + m].split([heads, kv_heads, kv_heads], 1))
        k, v = k.repeat_interleave(heads // kv_heads, 0), v.repeat_interleave(heads // kv_heads, 0)
        z = q @ k.transpose(1, 2) / math.sqrt(d)
        z = z.masked_fill(torch.ones(m, m, dtype=torch.bool, device=z.device).triu(1), -math.inf)
        parts.append((torch.softmax(z, -1) @ v).transpose(0, 1).reshape(m, heads * d))
        at += m
    y = torch.cat(parts) @ wo.t()
    has = p["labels"] >= 0
    loss = torch.nn.functional.cross_entropy(y @ table.t(), p["labels"].long().clamp(min=0), reduction="none") * has
    (loss * p["weight"].double()).sum().backward()
    return loss.detach(), table.grad, wqkv.grad, wo.grad


@pytest.mark.parametrize("precision", ["bf16", "fp32"])
def test_language_model_step(precision):
    """Embedding, attention and loss one after another with their gradients, against differentiation of the whole in float64.

    float32: six products of up to 517 terms one behind another, 525 x 2^-24 = 3e-5 of their size each, 2e-4 in all.  bfloat16: about ten roundings of
    2^-8 in a row between the table and its gradient, each of independent sign per element, against sums of as many terms as they spoil: 10 x 2^-8 = 4e-2
    of the norm."""
    p, dt, _ = PRECISIONS[precision]
    m = language_model(dt)
    got, want = language_model_step(p, m), language_model_reference(m)
    for name, a, b in zip(("loss", "table", "wqkv", "wo"), got, want):
        off = (a.double() - b).norm() / b.norm()
        assert off <= (2e-4 if precision == "fp32" else 4e-2), (name, off.item())


def test_captured_and_replayed():
    """The whole step in a graph, replayed with other inputs and eager work in between: the bits of the eager calls."""
    m, other = language_model(torch.bfloat16), language_model(torch.bfloat16, seed=1)
    eager = [[t.clone() for t in language_model_step(mt.MT_BF16, x)] for x in (m, other)]
    live = {k: (v.clone() if torch.is_tensor(v) else v) for k, v in m.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        language_model_step(mt.MT_BF16, live)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = language_model_step(mt.MT_BF16, live)
    for turn in range(4):
        src = (m, other)[turn % 2]
        for n, t in live.items():
            if torch.is_tensor(t):
                t.copy_(src[n])
        graph.replay()
        again = language_model_step(mt.MT_BF16, src)
        torch.cuda.synchronize()
        for i, (a, b, c) in enumerate(zip(out, eager[turn % 2], again)):
            same = torch.equal(a, b) and torch.equal(b, c) if i < 2 else torch.allclose(a, b, rtol=1e-3, atol=1e-5)     # (wqkv, wo: the library's products)
            assert same, (turn, i)


def test_two_calls_at_once():
    """Two streams, the same operators, workspaces of their own."""
    a, b = language_model(torch.bfloat16), language_model(torch.bfloat16, seed=1)
    want = [[t.clone() for t in language_model_step(mt.MT_BF16, x)[:2]] for x in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = []
        for s, x in zip(streams, (a, b)):
            with torch.cuda.stream(s):
                got.append(language_model_step(mt.MT_BF16, x)[:2])
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(g, w))


def test_binding_refuses_tensors_of_another_kind():
    q = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    st = starts([4])
    for bad in (lambda: mt.op_packed_attention(mt.MT_BF16, q, q.float(), q, st), lambda: mt.op_packed_attention(mt.MT_FP32_CHECK, q, q, q, st),
                lambda: mt.op_packed_attention(mt.MT_BF16, q, q.cpu(), q, st), lambda: mt.op_packed_attention(mt.MT_BF16, q, q, q, st.long()),
                lambda: mt.op_packed_attention(mt.MT_BF16, q.transpose(0, 2), q, q, st), lambda: mt.op_packed_attention(mt.MT_BF16, q, q, q[:3], st),
                lambda: mt.op_packed_attention(mt.MT_BF16, q, q, q, st, out=q[:1].expand(4, 2, 64)),
                lambda: mt.op_vocab_loss(mt.MT_BF16, q[:, 0], q[:, 0].cpu(), st[:1].expand(4)), lambda: mt.op_vocab_loss(mt.MT_BF16, q[:, 0], q[:, 0], st),
                lambda: mt.op_embedding(mt.MT_BF16, q[:, 0], st.long()), lambda: mt.op_embedding_grad(mt.MT_BF16, q[:, 0], st, 9),
                lambda: mt.op_embedding_grad(mt.MT_BF16, q[:2, 0], st, 9, add_to=q[:, 0])):
        with pytest.raises(mt.MTError):
            bad()
