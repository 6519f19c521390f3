// Launch interface of the operators on packed tokens: attention over packed sequences, loss over the vocabulary, embedding rows.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mt {

// a launch has less than 2^32 threads
inline bool fits_launch(int64_t groups, int threads) { return groups >= 0 && groups * threads < 1ll << 32; }

// bytes of a workspace's part
inline size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

// ---- attention over packed sequences.  Strides in elements; rows of a head are `d` contiguous elements.
struct PackedAttn {
    const void *q, *k, *v;
    const void *ctx, *dctx;             // gradient: the result and what comes back through it
    void *out;                          // forward: the result
    void *dq, *dk, *dv;
    const float* lse_in;
    float* lse;                         // [heads][total_q], natural logarithm; forward: may be null
    const int32_t *q_start, *k_start;   // [n_seqs + 1]
    int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head, g_row, g_head;      // o: ctx / out, g: dctx
    int64_t dq_row, dq_head, dk_row, dk_head, dv_row, dv_head;
    int32_t n_seqs, heads, kv_heads, group, d, total_q, total_k, causal;     // group: heads / kv_heads
    float scale;
    void* work;
    size_t work_bytes;
};
size_t packed_attention_work(int n_seqs, int total_q, int total_k, int heads, int kv_heads, int d);
size_t packed_attention_grad_work(int total_q, int heads);
hipError_t launch_packed_attention(const PackedAttn& p, int f32, hipStream_t stream);
hipError_t launch_packed_attention_grad(const PackedAttn& p, int f32, hipStream_t stream);

// ---- softmax cross entropy of x W^T over the vocabulary
struct VocabLoss {
    const void *x, *w;                  // [tokens][hidden], [vocab][hidden]
    int64_t ldx, ldw;                   // row strides in elements
    const int32_t* labels;              // [tokens], outside [0, vocab): no label
    float *loss, *lse;                  // [tokens]; gradient: lse is read
    const float* weight;                // gradient: [tokens], what comes back through each token's loss
    void *dx, *dw;                      // gradient: [tokens][hidden], [vocab][hidden], dense
    int32_t dw_f32;
    int32_t tokens, hidden, vocab;
    void* work;
    size_t work_bytes;
};
size_t vocab_loss_work(int tokens, int vocab);
size_t vocab_loss_grad_work(int f32, int tokens, int hidden, int vocab);
hipError_t launch_vocab_loss(const VocabLoss& p, int f32, hipStream_t stream);
hipError_t launch_vocab_loss_grad(const VocabLoss& p, int f32, hipStream_t stream);

// ---- rows of an embedding table
struct Embedding {
    const void* table;                  // lookup: [vocab][hidden]
    const void* grad;                   // gradient: [n][hidden]
    const int32_t* ids;                 // [n], outside [0, vocab): no row
    void* out;                          // lookup: [n][hidden]; gradient: [vocab][hidden]
    int64_t ld_in, ld_out;              // row strides in elements
    int32_t n, vocab, hidden, out_f32, accumulate;
    float scale;
    void* work;
    size_t work_bytes;
};
size_t embedding_grad_work(int n, int vocab, int hidden);
hipError_t launch_embedding(const Embedding& p, int f32, hipStream_t stream);
hipError_t launch_embedding_grad(const Embedding& p, int f32, hipStream_t stream);

}  // namespace mt
