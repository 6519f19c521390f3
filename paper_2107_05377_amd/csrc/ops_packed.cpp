// C entry points of the operators on packed tokens (include/mt.h): argument checks, then the launches.
#include <cmath>
#include <cstdint>

#include "../../include/mt.h"
#include "packed.h"

using namespace mt;

namespace {

int result(hipError_t e) { return e == hipSuccess ? MT_OK : e == hipErrorInvalidValue ? MT_ERR_SHAPE : MT_ERR_HIP; }
bool known(int32_t precision) { return precision == MT_BF16 || precision == MT_FP32_CHECK; }
bool at16(const void* p) { return ((uintptr_t)p & 15) == 0; }
// a row stride of whole 16-byte pieces whose products with a row number stay far inside 63 bits
bool rows16(int64_t stride, int size) { return stride >= 0 && stride < (1ll << 40) && stride * size % 16 == 0; }
// strides under which no two (row, head) pairs of an output share an element in one of the two directions
bool apart(int64_t row, int64_t head, int32_t rows, int32_t heads, int32_t width)
{
    if (rows > 1 && row < width) return false;
    if (heads > 1 && head < width) return false;
    return rows <= 1 || heads <= 1 || row >= (int64_t)heads * head || head >= (int64_t)rows * row;
}
bool fits(const void* work, size_t have, size_t need) { return need == 0 || (work && ((uintptr_t)work & 255) == 0 && have >= need); }

// sizes alone: MT_OK or what is wrong.  (Every workgroup looks through the sequences for its own: at 16384 of them for a tenth of a millisecond.)
int attention_sizes(const mt_packed_attention* op)
{
    if (!known(op->precision)) return MT_ERR_CONFIG;
    if (op->n_seqs < 1 || op->n_seqs > 16384 || op->heads < 1 || op->kv_heads < 1 || op->kv_heads > 65535 || op->heads % op->kv_heads != 0 || op->width < 8 ||
        op->width > 128 || op->width % 8 != 0 || op->total_q < 1 || op->total_k < 1 || !(op->scale > 0.f) || !std::isfinite(op->scale))
        return MT_ERR_SHAPE;
    // rows are numbered with 31 bits: a group's heads of all queries, and the keys, with room for a tile and for the longest shift between the two
    if ((int64_t)op->total_q * (op->heads / op->kv_heads) > 1 << 29 || op->total_k > 1 << 29 || (int64_t)op->total_q * op->heads > 1ll << 34) return MT_ERR_SHAPE;
    return MT_OK;
}

PackedAttn attention_args(const mt_packed_attention* op)
{
    PackedAttn p{};
    p.q = op->d_q;
    p.k = op->d_k;
    p.v = op->d_v;
    p.q_start = op->d_q_start;
    p.k_start = op->d_k_start ? op->d_k_start : op->d_q_start;
    p.q_row = op->q_row;
    p.q_head = op->q_head;
    p.k_row = op->k_row;
    p.k_head = op->k_head;
    p.v_row = op->v_row;
    p.v_head = op->v_head;
    p.o_row = op->ctx_row;
    p.o_head = op->ctx_head;
    p.n_seqs = op->n_seqs;
    p.heads = op->heads;
    p.kv_heads = op->kv_heads;
    p.group = op->heads / op->kv_heads;
    p.d = op->width;
    p.total_q = op->total_q;
    p.total_k = op->total_k;
    p.causal = op->causal != 0;
    p.scale = op->scale;
    p.work = op->d_work;
    p.work_bytes = op->work_bytes;
    return p;
}

size_t attention_work(const mt_packed_attention* op, bool grad)
{
    if (grad) return packed_attention_grad_work(op->total_q, op->heads);
    return packed_attention_work(op->n_seqs, op->total_q, op->total_k, op->heads, op->kv_heads, op->width);
}

}  // namespace

extern "C" {

size_t mt_op_packed_attention_work(const mt_packed_attention* op, int32_t grad)
{
    return op && attention_sizes(op) == MT_OK ? attention_work(op, grad != 0) : 0;
}

int mt_op_packed_attention(const mt_packed_attention* op, void* hip_stream)
{
    if (!op || !op->d_q || !op->d_k || !op->d_v || !op->d_ctx || !op->d_q_start) return MT_ERR_NULL;
    const int bad = attention_sizes(op);
    if (bad != MT_OK) return bad;
    const int size = op->precision == MT_BF16 ? 2 : 4;
    for (const void* t : {op->d_q, op->d_k, op->d_v, (const void*)op->d_ctx})
        if (!at16(t)) return MT_ERR_SHAPE;
    for (const int64_t s : {op->q_row, op->q_head, op->k_row, op->k_head, op->v_row, op->v_head, op->ctx_row, op->ctx_head})
        if (!rows16(s, size)) return MT_ERR_SHAPE;
    if (!apart(op->ctx_row, op->ctx_head, op->total_q, op->heads, op->width) || !fits(op->d_work, op->work_bytes, attention_work(op, false))) return MT_ERR_SHAPE;
    PackedAttn p = attention_args(op);
    p.out = op->d_ctx;
    p.lse = op->d_lse;
    return result(launch_packed_attention(p, size == 4, static_cast<hipStream_t>(hip_stream)));
}

int mt_op_packed_attention_grad(const mt_packed_attention* op, void* hip_stream)
{
    if (!op || !op->d_q || !op->d_k || !op->d_v || !op->d_ctx || !op->d_lse || !op->d_q_start || !op->d_grad_ctx || !op->d_grad_q || !op->d_grad_k || !op->d_grad_v)
        return MT_ERR_NULL;
    const int bad = attention_sizes(op);
    if (bad != MT_OK) return bad;
    const int size = op->precision == MT_BF16 ? 2 : 4;
    for (const void* t : {op->d_q, op->d_k, op->d_v, (const void*)op->d_ctx, op->d_grad_ctx, (const void*)op->d_grad_q, (const void*)op->d_grad_k, (const void*)op->d_grad_v})
        if (!at16(t)) return MT_ERR_SHAPE;
    for (const int64_t s : {op->q_row, op->q_head, op->k_row, op->k_head, op->v_row, op->v_head, op->ctx_row, op->ctx_head, op->grad_ctx_row, op->grad_ctx_head,
                            op->grad_q_row, op->grad_q_head, op->grad_k_row, op->grad_k_head, op->grad_v_row, op->grad_v_head})
        if (!rows16(s, size)) return MT_ERR_SHAPE;
    if (!apart(op->grad_q_row, op->grad_q_head, op->total_q, op->heads, op->width) || !apart(op->grad_k_row, op->grad_k_head, op->total_k, op->kv_heads, op->width) ||
        !apart(op->grad_v_row, op->grad_v_head, op->total_k, op->kv_heads, op->width) || !fits(op->d_work, op->work_bytes, attention_work(op, true)))
        return MT_ERR_SHAPE;
    PackedAttn p = attention_args(op);
    p.ctx = op->d_ctx;
    p.lse_in = op->d_lse;
    p.dctx = op->d_grad_ctx;
    p.dq = op->d_grad_q;
    p.dk = op->d_grad_k;
    p.dv = op->d_grad_v;
    p.g_row = op->grad_ctx_row;
    p.g_head = op->grad_ctx_head;
    p.dq_row = op->grad_q_row;
    p.dq_head = op->grad_q_head;
    p.dk_row = op->grad_k_row;
    p.dk_head = op->grad_k_head;
    p.dv_row = op->grad_v_row;
    p.dv_head = op->grad_v_head;
    return result(launch_packed_attention_grad(p, size == 4, static_cast<hipStream_t>(hip_stream)));
}

static int loss_sizes(int32_t precision, int32_t tokens, int32_t hidden, int32_t vocab)
{
    if (!known(precision)) return MT_ERR_CONFIG;
    if (tokens < 1 || tokens > 1 << 23 || hidden < 64 || hidden > 1 << 20 || hidden % 64 != 0 || vocab < 1 || vocab > 1 << 22) return MT_ERR_SHAPE;
    return MT_OK;
}

size_t mt_op_vocab_loss_work(int32_t precision, int32_t tokens, int32_t hidden, int32_t vocab, int32_t grad)
{
    if (loss_sizes(precision, tokens, hidden, vocab) != MT_OK) return 0;
    return grad ? vocab_loss_grad_work(precision != MT_BF16, tokens, hidden, vocab) : vocab_loss_work(tokens, vocab);
}

int mt_op_vocab_loss(int32_t precision, const void* d_x, int64_t ldx, const void* d_W, int64_t ldw, const int32_t* d_labels, float* d_loss, float* d_lse,
                     int32_t tokens, int32_t hidden, int32_t vocab, void* d_work, size_t work_bytes, void* hip_stream)
{
    if (!d_x || !d_W || !d_labels || !d_loss || !d_lse) return MT_ERR_NULL;
    const int bad = loss_sizes(precision, tokens, hidden, vocab);
    if (bad != MT_OK) return bad;
    const int size = precision == MT_BF16 ? 2 : 4;
    if (!at16(d_x) || !at16(d_W) || ldx < hidden || ldw < hidden || !rows16(ldx, size) || !rows16(ldw, size) ||
        !fits(d_work, work_bytes, mt_op_vocab_loss_work(precision, tokens, hidden, vocab, 0)))
        return MT_ERR_SHAPE;
    VocabLoss p{};
    p.x = d_x;
    p.w = d_W;
    p.ldx = ldx;
    p.ldw = ldw;
    p.labels = d_labels;
    p.loss = d_loss;
    p.lse = d_lse;
    p.tokens = tokens;
    p.hidden = hidden;
    p.vocab = vocab;
    p.work = d_work;
    p.work_bytes = work_bytes;
    return result(launch_vocab_loss(p, size == 4, static_cast<hipStream_t>(hip_stream)));
}

int mt_op_vocab_loss_grad(int32_t precision, const void* d_x, int64_t ldx, const void* d_W, int64_t ldw, const int32_t* d_labels, const float* d_lse,
                          const float* d_weight, void* d_grad_x, void* d_grad_W, int32_t grad_W_f32, int32_t tokens, int32_t hidden, int32_t vocab,
                          void* d_work, size_t work_bytes, void* hip_stream)
{
    if (!d_x || !d_W || !d_labels || !d_lse || !d_weight || !d_grad_x || !d_grad_W) return MT_ERR_NULL;
    const int bad = loss_sizes(precision, tokens, hidden, vocab);
    if (bad != MT_OK) return bad;
    const int size = precision == MT_BF16 ? 2 : 4;
    if (!at16(d_x) || !at16(d_W) || !at16(d_grad_x) || !at16(d_grad_W) || ldx < hidden || ldw < hidden || !rows16(ldx, size) || !rows16(ldw, size) ||
        !fits(d_work, work_bytes, mt_op_vocab_loss_work(precision, tokens, hidden, vocab, 1)))
        return MT_ERR_SHAPE;
    VocabLoss p{};
    p.x = d_x;
    p.w = d_W;
    p.ldx = ldx;
    p.ldw = ldw;
    p.labels = d_labels;
    p.lse = const_cast<float*>(d_lse);
    p.weight = d_weight;
    p.dx = d_grad_x;
    p.dw = d_grad_W;
    p.dw_f32 = grad_W_f32 != 0;
    p.tokens = tokens;
    p.hidden = hidden;
    p.vocab = vocab;
    p.work = d_work;
    p.work_bytes = work_bytes;
    return result(launch_vocab_loss_grad(p, size == 4, static_cast<hipStream_t>(hip_stream)));
}

// tokens of a gradient: each workgroup of the sort adds up the counts of all, a quarter of a million loads at this many
constexpr int32_t kMostSorted = 1 << 24;

static int embedding_sizes(int32_t precision, int32_t n, int32_t vocab, int32_t hidden)
{
    if (!known(precision)) return MT_ERR_CONFIG;
    if (n < 1 || n > 1 << 28 || vocab < 1 || vocab > 1 << 28 || hidden < 4 || hidden > 1 << 16 || hidden % (precision == MT_BF16 ? 8 : 4) != 0) return MT_ERR_SHAPE;
    return MT_OK;
}

int mt_op_embedding(int32_t precision, const void* d_table, int64_t ldt, const int32_t* d_ids, float scale, void* d_out, int64_t ldo, int32_t n,
                    int32_t vocab, int32_t hidden, void* hip_stream)
{
    if (!d_table || !d_ids || !d_out) return MT_ERR_NULL;
    const int bad = embedding_sizes(precision, n, vocab, hidden);
    if (bad != MT_OK) return bad;
    const int size = precision == MT_BF16 ? 2 : 4;
    if (!at16(d_table) || !at16(d_out) || ldt < hidden || ldo < hidden || !rows16(ldt, size) || !rows16(ldo, size) || !std::isfinite(scale)) return MT_ERR_SHAPE;
    Embedding p{};
    p.table = d_table;
    p.ids = d_ids;
    p.out = d_out;
    p.ld_in = ldt;
    p.ld_out = ldo;
    p.n = n;
    p.vocab = vocab;
    p.hidden = hidden;
    p.scale = scale;
    return result(launch_embedding(p, size == 4, static_cast<hipStream_t>(hip_stream)));
}

size_t mt_op_embedding_grad_work(int32_t precision, int32_t n, int32_t vocab, int32_t hidden)
{
    return embedding_sizes(precision, n, vocab, hidden) == MT_OK && n <= kMostSorted ? embedding_grad_work(n, vocab, hidden) : 0;
}

int mt_op_embedding_grad(int32_t precision, const void* d_grad, int64_t ldg, const int32_t* d_ids, float scale, void* d_grad_table, int64_t ldt,
                         int32_t out_f32, int32_t accumulate, int32_t n, int32_t vocab, int32_t hidden, void* d_work, size_t work_bytes, void* hip_stream)
{
    if (!d_grad || !d_ids || !d_grad_table) return MT_ERR_NULL;
    const int bad = embedding_sizes(precision, n, vocab, hidden);
    if (bad != MT_OK) return bad;
    if (n > kMostSorted) return MT_ERR_SHAPE;
    const int size = precision == MT_BF16 ? 2 : 4, out_size = size == 4 || out_f32 ? 4 : 2;
    if (!at16(d_grad) || !at16(d_grad_table) || ldg < hidden || ldt < hidden || !rows16(ldg, size) || !rows16(ldt, out_size) || !std::isfinite(scale) ||
        (accumulate && out_size != 4) || !fits(d_work, work_bytes, embedding_grad_work(n, vocab, hidden)))
        return MT_ERR_SHAPE;
    Embedding p{};
    p.grad = d_grad;
    p.ids = d_ids;
    p.out = d_grad_table;
    p.ld_in = ldg;
    p.ld_out = ldt;
    p.n = n;
    p.vocab = vocab;
    p.hidden = hidden;
    p.out_f32 = out_size == 4;
    p.accumulate = accumulate != 0;
    p.scale = scale;
    p.work = d_work;
    p.work_bytes = work_bytes;
    return result(launch_embedding_grad(p, size == 4, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
