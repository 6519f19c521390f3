"""The operators of one language-model step on single buffers, for timing: embedding, attention over packed sequences, vocabulary loss.

A case names an operator, what is asked of it ("forward": the result; "train": the result and the gradients of its inputs) and its
sizes.  Prepared once is what a program has in hand before the call: the tensors on the device, the table that says where the packed
sequences start, and the buffers that receive an attention's results.

Lengths of packed sequences belong to the case (spread evenly over the logarithm of their range, in a mixed order), values to the seed:
activations and cached keys are N(0, 1), embedding rows N(0, 1), classifier weights N(0, 1 / width) so that logits are N(0, 1) as a
trained head's are, token ids and labels follow a 1 / rank law as words do, upstream gradients are N(0, 1) (attention, embedding) or one
over the number of labelled tokens (the mean of the loss).
"""
from __future__ import annotations

import math

import torch

own = False

# elements that the padded scores of a drawn attention may have, and the contraction of a drawn loss: those of the largest listed cases
MOST_SCORES = 32 * 8192 * 8192
MOST_LOSS = 4099 * 1024 * 128000
MOST_EMBED = 8 * 32 * 128 * 768


def _attention(name, call, precision, heads, kv_heads, width, seqs, q_len, k_len, causal=True, layout="fused"):
    """q_len, k_len: (shortest, longest) queries and keys of a sequence, k_len None: the queries' own tokens are the keys.
    layout: "fused": q | k | v are columns of one matrix; "apart": tensors of their own; "heads": keys and values head after head."""
    return {"name": name, "op": "attention", "call": call, "precision": precision, "heads": heads, "kv_heads": kv_heads, "width": width, "seqs": seqs,
            "q_lo": q_len[0], "q_hi": q_len[1], "k_lo": k_len[0] if k_len else 0, "k_hi": k_len[1] if k_len else 0, "causal": causal, "layout": layout}


def _loss(name, call, precision, tokens, hidden, vocab, labelled):
    """labelled: share of the tokens that have a label (the others are marked -100)."""
    return {"name": name, "op": "loss", "call": call, "precision": precision, "tokens": tokens, "hidden": hidden, "vocab": vocab, "labelled": labelled}


def _embedding(name, call, precision, tokens, hidden, vocab, scale, grad_f32=False):
    return {"name": name, "op": "embedding", "call": call, "precision": precision, "tokens": tokens, "hidden": hidden, "vocab": vocab, "scale": scale,
            "grad_f32": grad_f32}


def listed():
    return [
        # one user's next token against a short history: latency
        _attention("attn_token_b1", "forward", "bf16", 12, 12, 64, 1, (1, 1), (61, 61), layout="apart"),
        # the next tokens of 32 conversations of very different lengths, grouped heads, keys kept head after head
        _attention("attn_token_ragged_b32", "forward", "bf16", 16, 4, 128, 32, (1, 1), (100, 8191), layout="heads"),
        # eight request batches of padding-free utterances through an encoder layer
        _attention("attn_encoder_8x32", "forward", "bf16", 12, 12, 64, 256, (16, 128), None, causal=False),
        # one long document as a prompt: the largest forward call
        _attention("attn_prompt_8192", "forward", "bf16", 32, 8, 128, 1, (8192, 8192), None),
        # a training batch of packed documents, grouped heads
        _attention("attn_train_packed", "train", "bf16", 16, 4, 64, 9, (300, 4001), None),
        # the same step of the validation precision, sentence pairs up to the model's longest input
        _attention("attn_train_fp32", "train", "fp32", 12, 12, 64, 7, (60, 509), None),
        # scoring a handful of candidate tokens: every weight is read for few rows
        _loss("loss_score_b5", "forward", "bf16", 5, 768, 30522, 1.0),
        # masked language modelling on a batch of 64 x 128 tokens, 15 % of them predicted
        _loss("loss_masked_64x128", "train", "bf16", 8192, 768, 30522, 0.15),
        # next-token training with a large vocabulary: the largest call
        _loss("loss_wide", "train", "bf16", 4099, 1024, 128000, 0.97),
        # validation precision
        _loss("loss_fp32", "train", "fp32", 509, 768, 30522, 1.0),
        # the tokens of one short request
        _embedding("embed_b1", "forward", "bf16", 61, 768, 30522, 1.0),
        # eight request batches' worth of training tokens, rows scaled by the root of the width, master gradients in float32
        _embedding("embed_train_8x32x128", "train", "bf16", 8 * 32 * 128, 768, 30522, math.sqrt(768.0), grad_f32=True),
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attention", "attention", "loss", "loss", "embedding"])
    precision = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    call = rng.choice(["forward", "train"])
    if op == "attention":
        while True:
            width = rng.choice([32, 64, 64, 80, 128, 128])
            kv_heads = rng.randint(1, 12)
            heads = kv_heads * rng.choice([1, 1, 2, 3, 4, 8])
            seqs = _spread(rng, 1, 256)
            if call == "forward" and rng.random() < 0.4:        # tokens against a cache
                q_hi = rng.choice([1, 1, rng.randint(2, 7)])
                k_hi = _spread(rng, q_hi + 1, 8192)
                k_len, q_len, layout = (max(q_hi, k_hi // rng.randint(1, 20)), k_hi), (1, q_hi), rng.choice(["apart", "heads"])
            else:
                q_hi = _spread(rng, 2, 8192 if call == "forward" else 4096)
                k_len, q_len, layout = None, (max(1, q_hi // rng.randint(1, 20)), q_hi), rng.choice(["fused", "apart", "heads"])
            scores = seqs * heads * q_len[1] * (k_len or q_len)[1]
            rows = seqs * max(heads * q_len[1], kv_heads * (k_len or q_len)[1]) * width
            if heads <= 32 and scores * (3 if call == "train" else 1) <= MOST_SCORES and rows <= 1 << 28:
                return _attention("", call, precision, heads, kv_heads, width, seqs, q_len, k_len, rng.random() < 0.7, layout)
    if op == "loss":
        while True:
            tokens, hidden, vocab = _spread(rng, 1, 16384), 64 * rng.randint(2, 32), _spread(rng, 1000, 128000)
            cost = tokens * hidden * vocab * (4 if call == "train" else 1) * (3 if precision == "fp32" else 1)
            if cost <= 4 * MOST_LOSS and tokens * vocab <= 4099 * 128000:
                return _loss("", call, precision, tokens, hidden, vocab, rng.choice([1.0, round(rng.uniform(0.1, 1.0), 3)]))
    while True:
        tokens, hidden, vocab = _spread(rng, 1, 65536), 8 * rng.randint(8, 256), _spread(rng, 100, 128000)
        if tokens * hidden <= MOST_EMBED and vocab * hidden <= 2 * 30522 * 768:
            return _embedding("", call, precision, tokens, hidden, vocab, rng.choice([1.0, math.sqrt(hidden)]), rng.random() < 0.5)


def _lengths(count, lo, hi):
    """`count` lengths, even over the logarithm of [lo, hi], the longest among them, in an order that mixes long and short."""
    at = [math.modf(i * 0.6180339887498949)[0] for i in range(count)]
    top = max(at) or 1.0
    return [max(lo, min(hi, int(round(lo * (hi / lo) ** (a / top))))) if count > 1 else hi for a in at]


def _sequences(case):
    """Lengths of a case's sequences: (queries, keys)."""
    q = _lengths(case["seqs"], case["q_lo"], case["q_hi"])
    return q, (_lengths(case["seqs"], case["k_lo"], case["k_hi"]) if case["k_hi"] else q)


def _starts(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def _type(case):
    return torch.bfloat16 if case["precision"] == "bf16" else torch.float32


def _words(count, vocab, gen):
    """Token ids with a 1 / rank law."""
    u = torch.rand(count, generator=gen, device="cuda", dtype=torch.float64)
    return (torch.exp(u * math.log(vocab)) - 1).long().clamp(0, vocab - 1).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = _type(case)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=gen, device="cuda").mul_(std).to(dt)

    s = {"case": case}
    if case["op"] == "attention":
        hq, hk, d = case["heads"], case["kv_heads"], case["width"]
        nq, nk = _sequences(case)
        tq, tk = sum(nq), sum(nk)
        if case["layout"] == "fused":
            x = normal(tq, hq + 2 * hk, d)
            s["q"], s["k"], s["v"] = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
        elif case["layout"] == "heads":
            s["q"], s["k"], s["v"] = normal(tq, hq, d), normal(hk, tk, d).transpose(0, 1), normal(hk, tk, d).transpose(0, 1)
        else:
            s["q"], s["k"], s["v"] = normal(tq, hq, d), normal(tk, hk, d), normal(tk, hk, d)
        s["q_start"] = torch.tensor(_starts(nq), dtype=torch.int32, device="cuda")
        s["k_start"] = torch.tensor(_starts(nk), dtype=torch.int32, device="cuda") if case["k_hi"] else None
        s["longest"] = (max(nq), max(nk))
        s["ctx"] = torch.empty(tq, hq, d, dtype=dt, device="cuda")
        if case["call"] == "train":
            s["grad"] = normal(tq, hq, d)
            s["grads"] = (torch.empty_like(s["ctx"]), torch.empty(tk, hk, d, dtype=dt, device="cuda"), torch.empty(tk, hk, d, dtype=dt, device="cuda"))
    elif case["op"] == "loss":
        n, h, v = case["tokens"], case["hidden"], case["vocab"]
        s["x"], s["w"] = normal(n, h), normal(v, h, std=1.0 / math.sqrt(h))
        labels = _words(n, v, gen)
        with_label = torch.arange(n, device="cuda") < max(1, round(n * case["labelled"]))
        with_label = with_label[torch.randperm(n, generator=gen, device="cuda")]
        s["labels"] = torch.where(with_label, labels, torch.full_like(labels, -100))
        s["weight"] = with_label.float() / with_label.sum()
    else:
        s["table"], s["ids"] = normal(case["vocab"], case["hidden"]), _words(case["tokens"], case["vocab"], gen)
        if case["call"] == "train":
            s["grad"] = normal(case["tokens"], case["hidden"])
    return s


def work(case):
    size = 2 if case["precision"] == "bf16" else 4
    train = case["call"] == "train"
    if case["op"] == "attention":
        nq, nk = _sequences(case)
        # query i of a sequence sees the keys up to its own distance from the end
        pairs = sum(sum(max(0, min(k, i + 1 + k - q)) for i in range(q)) if case["causal"] else q * k for q, k in zip(nq, nk))
        q_el, k_el = sum(nq) * case["heads"] * case["width"], sum(nk) * case["kv_heads"] * case["width"]
        lse = sum(nq) * case["heads"] * 4
        moved = (2 * q_el + 2 * k_el) * size
        if train:
            moved += (2 * q_el + 2 * k_el) * size + lse         # the upstream gradient and dq, dk, dv; the statistics as an output
        return {"bytes": moved, "flops": pairs * case["heads"] * case["width"] * (14 if train else 4)}
    if case["op"] == "loss":
        n, h, v = max(1, round(case["tokens"] * case["labelled"])), case["hidden"], case["vocab"]
        moved = (n * h + v * h) * size + case["tokens"] * 12
        if train:
            moved += (case["tokens"] * h + v * h) * size + case["tokens"] * 4
        return {"bytes": moved, "flops": n * h * v * (6 if train else 2)}
    n, h, v = case["tokens"], case["hidden"], case["vocab"]
    moved = n * 4 + 2 * n * h * size
    if train:
        moved += n * h * size + v * h * (4 if case["grad_f32"] else size)
    return {"bytes": moved, "flops": n * h * (2 if train else 1)}


# ---- plain forms: padded batches in float32

def _padded(x, start, longest):
    """[sequences, heads, longest, width] in float32 of packed rows [rows, heads, width], and which places hold a row."""
    rows = start[:-1, None].long() + torch.arange(longest, device=x.device)
    held = rows < start[1:, None]
    p = x[rows.clamp(max=x.shape[0] - 1)].float().masked_fill(~held[:, :, None, None], 0.0)
    return p.transpose(1, 2).contiguous(), held


def _packed(p, start, rows):
    """The rows [rows, heads, width] of a padded batch."""
    row = torch.arange(rows, device=p.device)
    seq = torch.searchsorted(start[1:].long(), row, right=True)
    return p[seq, :, row - start[seq].long()]


def _plain_attention(s):
    case = s["case"]
    hq, hk, d = case["heads"], case["kv_heads"], case["width"]
    group, scale = hq // hk, 1.0 / math.sqrt(d)
    k_start = s["q_start"] if s["k_start"] is None else s["k_start"]
    lq, lk = s["longest"]
    q, _ = _padded(s["q"], s["q_start"], lq)
    k, held = _padded(s["k"], k_start, lk)
    v, _ = _padded(s["v"], k_start, lk)
    n = q.shape[0]
    see = held[:, None, :].expand(n, lq, lk)
    if case["causal"]:
        behind = (k_start[1:] - k_start[:-1] - s["q_start"][1:] + s["q_start"][:-1])[:, None, None]
        see = see & (torch.arange(lk, device=q.device) <= torch.arange(lq, device=q.device)[:, None] + behind)
    q = q.view(n, hk, group * lq, d)
    score = (torch.matmul(q, k.transpose(2, 3)) * scale).view(n, hk, group, lq, lk)
    score.masked_fill_(~see[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp_(score.sub_(top))
    total = p.sum(-1, keepdim=True)
    p = p.div_(total).view(n, hk, group * lq, lk)
    ctx = torch.matmul(p, v)
    pack = lambda x: _packed(x.reshape(n, hq, lq, -1), s["q_start"], s["q"].shape[0])  # noqa: E731
    out = pack(ctx).to(s["q"].dtype)
    if case["call"] == "forward":
        return out
    lse = pack(top + torch.log(total))[..., 0].t().contiguous()
    g = _padded(s["grad"], s["q_start"], lq)[0].view(n, hk, group * lq, d)
    dv = torch.matmul(p.transpose(2, 3), g)
    ds = torch.matmul(g, v.transpose(2, 3)).sub_((g * ctx).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(2, 3), q)
    rows = s["k"].shape[0]
    return out, lse, pack(dq).to(out.dtype), _packed(dk, k_start, rows).to(out.dtype), _packed(dv, k_start, rows).to(out.dtype)


def _plain_loss(s):
    x, w, labels = s["x"].float(), s["w"].float(), s["labels"].long()
    has = labels >= 0
    z = torch.matmul(x, w.t())
    top = z.amax(1, keepdim=True)
    lse = (top + torch.log(torch.exp(z - top).sum(1, keepdim=True)))[:, 0]
    at = labels.clamp(min=0)[:, None]
    zero = torch.zeros_like(lse)
    loss = torch.where(has, lse - z.gather(1, at)[:, 0], zero)
    if s["case"]["call"] == "forward":
        return loss, torch.where(has, lse, zero)
    dz = torch.exp_(z.sub_(lse[:, None]))
    dz.scatter_add_(1, at, torch.full_like(dz[:, :1], -1.0)).mul_(s["weight"][:, None])
    return loss, torch.where(has, lse, zero), torch.matmul(dz, w).to(s["x"].dtype), torch.matmul(dz.t(), x).to(s["w"].dtype)


def _plain_embedding(s):
    case, ids = s["case"], s["ids"].long()
    out = (s["table"][ids].float() * case["scale"]).to(s["table"].dtype)
    if case["call"] == "forward":
        return out
    sums = torch.zeros(case["vocab"], case["hidden"], device=ids.device).index_add_(0, ids, s["grad"].float())
    return out, (sums * case["scale"]).to(torch.float32 if case["grad_f32"] else s["table"].dtype)


# ---- the framework's calls

def _own_attention(s):
    import paper_2107_05377_amd as mt
    case = s["case"]
    precision = mt.MT_BF16 if case["precision"] == "bf16" else mt.MT_FP32_CHECK
    if case["call"] == "forward":
        return mt.op_packed_attention(precision, s["q"], s["k"], s["v"], s["q_start"], s["k_start"], causal=case["causal"], out=s["ctx"])
    ctx, lse = mt.op_packed_attention(precision, s["q"], s["k"], s["v"], s["q_start"], s["k_start"], causal=case["causal"], out=s["ctx"], want_lse=True)
    grads = mt.op_packed_attention_grad(precision, s["grad"], s["q"], s["k"], s["v"], ctx, lse, s["q_start"], s["k_start"], causal=case["causal"],
                                        out=s["grads"])
    return (ctx, lse) + tuple(grads)


def _own_loss(s):
    import paper_2107_05377_amd as mt
    precision = mt.MT_BF16 if s["case"]["precision"] == "bf16" else mt.MT_FP32_CHECK
    loss, lse = mt.op_vocab_loss(precision, s["x"], s["w"], s["labels"])
    if s["case"]["call"] == "forward":
        return loss, lse
    dx, dw = mt.op_vocab_loss_grad(precision, s["x"], s["w"], s["labels"], lse, s["weight"])
    return loss, lse, dx, dw


def _own_embedding(s):
    import paper_2107_05377_amd as mt
    case = s["case"]
    precision = mt.MT_BF16 if case["precision"] == "bf16" else mt.MT_FP32_CHECK
    out = mt.op_embedding(precision, s["table"], s["ids"], scale=case["scale"])
    if case["call"] == "forward":
        return out
    return out, mt.op_embedding_grad(precision, s["grad"], s["ids"], case["vocab"], scale=case["scale"], out_f32=case["grad_f32"])


def run(state):
    op = state["case"]["op"]
    if own:
        return {"attention": _own_attention, "loss": _own_loss, "embedding": _own_embedding}[op](state)
    return {"attention": _plain_attention, "loss": _plain_loss, "embedding": _plain_embedding}[op](state)


# ---- from the definitions, in float64, sequence by sequence

def _exact_attention(case, s):
    nq, nk = _sequences(case)
    qs, ks = _starts(nq), _starts(nk)
    train, group, scale = case["call"] == "train", case["heads"] // case["kv_heads"], 1.0 / math.sqrt(case["width"])
    q, k, v = (s[n].transpose(0, 1).double() for n in ("q", "k", "v"))
    ctx, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], dtype=torch.float64, device=q.device)
    g = s["grad"].transpose(0, 1).double() if train else None
    dq, dk, dv = (torch.zeros_like(t) for t in (q, k, v))
    for b in range(case["seqs"]):
        iq, ik = slice(qs[b], qs[b + 1]), slice(ks[b], ks[b + 1])
        hidden = torch.ones(nq[b], nk[b], dtype=torch.bool, device=q.device).triu(nk[b] - nq[b] + 1) if case["causal"] else None
        for h in range(case["kv_heads"]):
            heads = slice(h * group, (h + 1) * group)
            kb, vb = k[h, ik], v[h, ik]
            step = max(1, (1 << 28) // (nq[b] * nk[b]))
            for a in range(heads.start, heads.stop, step):
                at = slice(a, min(a + step, heads.stop))
                z = q[at, iq] @ kb.t() * scale
                if hidden is not None:
                    z.masked_fill_(hidden, -math.inf)
                l = torch.logsumexp(z, -1)
                p = torch.exp_(z.sub_(l[..., None]))
                c = p @ vb
                ctx[at, iq], lse[at, iq] = c, l
                if train:
                    gb = g[at, iq]
                    dv[h, ik] += (p.transpose(1, 2) @ gb).sum(0)
                    dz = (gb @ vb.t()).sub_((gb * c).sum(-1, keepdim=True)).mul_(p).mul_(scale)
                    dq[at, iq] = dz @ kb
                    dk[h, ik] += (dz.transpose(1, 2) @ q[at, iq]).sum(0)
    back = lambda t: t.transpose(0, 1).contiguous()  # noqa: E731
    return (back(ctx), lse, back(dq), back(dk), back(dv)) if train else back(ctx)


def _exact_loss(case, s):
    x, w = s["x"].double(), s["w"].double()
    n, train = case["tokens"], case["call"] == "train"
    loss, lse = torch.zeros(n, dtype=torch.float64, device=x.device), torch.zeros(n, dtype=torch.float64, device=x.device)
    dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    rows = torch.nonzero(s["labels"] >= 0)[:, 0]
    for part in rows.split(1024):
        xb, lb = x[part], s["labels"][part].long()
        z = xb @ w.t()
        l = torch.logsumexp(z, 1)
        loss[part], lse[part] = l - z[torch.arange(len(part), device=x.device), lb], l
        if train:
            p = torch.softmax(z, 1)
            p[torch.arange(len(part), device=x.device), lb] -= 1.0
            p *= s["weight"][part].double()[:, None]
            dx[part] = p @ w
            dw += p.t() @ xb
    return (loss, lse, dx, dw) if train else (loss, lse)


def _exact_embedding(case, s):
    out = s["table"].double()[s["ids"].long()] * case["scale"]
    if case["call"] == "forward":
        return out
    order = torch.argsort(s["ids"], stable=True)
    held, count = torch.unique_consecutive(s["ids"][order], return_counts=True)
    total = torch.cat([torch.zeros_like(out[:1]), s["grad"].double()[order].cumsum(0)])
    end = count.cumsum(0)
    grad = torch.zeros(case["vocab"], case["hidden"], dtype=torch.float64, device=out.device)
    grad[held.long()] = (total[end] - total[end - count]) * case["scale"]
    return out, grad


def exact(case, seed):
    s = prepare(case, seed)
    return {"attention": _exact_attention, "loss": _exact_loss, "embedding": _exact_embedding}[case["op"]](case, s)
