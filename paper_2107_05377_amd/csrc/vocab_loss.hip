// Softmax cross entropy over a large vocabulary and its gradient (bfloat16 and float32); the logits are never stored.
//   z = x W^T,  lse_i = log sum_v exp z_iv,  loss_i = lse_i - z_i,label
//   dz = weight_i (exp(z_iv - lse_i) - [v = label_i]),  dx = dz W,  dW = dz^T x
//
// Tokens without a label are dropped on the device before anything is multiplied: `index` lists the labelled ones in order, and every product
// has as many rows (dW: as long a sum) as there are.  Forward: blocks of z are multiplied, reduced to a maximum and a sum of exponentials per
// token and range of the vocabulary, and the ranges are joined.  Gradient: for a piece of the vocabulary at a time dz is formed from z multiplied
// again (bfloat16: rounded to bfloat16, half a step of 2^-8 per term, as any operand of these products) and used for both gradients.
#include "packed_tile.h"
#include "packed.h"

#include <cmath>

namespace mt {

namespace {

constexpr int kTok = 128, kVoc = 128;       // tile of the products
constexpr int kPieceGrain = 256;

// ---- the labelled tokens, in order: index[0 .. *count)
__global__ __launch_bounds__(1024) void label_index_kernel(const int32_t* labels, int tokens, int vocab, int32_t* count, int32_t* index)
{
    __shared__ int wave_n[16];
    __shared__ int base;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (threadIdx.x == 0) base = 0;
    for (int t0 = 0; t0 < tokens; t0 += 1024) {
        const int t = t0 + threadIdx.x;
        const bool has = t < tokens && (uint32_t)labels[t] < (uint32_t)vocab;
        const uint64_t b = __ballot(has);
        if (lane == 0) wave_n[wave] = __popcll(b);
        __syncthreads();
        int before = base, all = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            before += i < wave ? wave_n[i] : 0;
            all += wave_n[i];
        }
        if (has) index[before + __popcll(b & ((1ull << lane) - 1))] = t;
        __syncthreads();
        if (threadIdx.x == 0) base += all;
    }
    __syncthreads();
    if (threadIdx.x == 0) *count = base;
}

// ---- a product's operands.  A "row" operand has the sum along its rows (contiguous), a "column" operand down its columns.
struct Operand {
    const void* base;
    int64_t ld;                 // elements
    const int32_t* rows;        // row operand: row i is row rows[i] of the matrix (null: i)
    int32_t n;                  // rows (row operand) or columns (column operand) that exist; copies stand in for those beyond
    int32_t k_n;                // column operand: rows that exist; the last one stands in for those beyond, which must meet zeros
};

template <typename E, int B, int NW, bool COLS>
struct Stager {
    static constexpr int BK = 128 / E::SIZE;                        // elements of the sum per slice
    static constexpr int WIDTH = COLS ? B : BK, ROWS = COLS ? BK : B;
    using T = Tile<E, WIDTH>;
    static constexpr int BYTES = ROWS * T::ROWB, N = BYTES / 1024 / NW;
    const typename E::elem* at[N];
    int64_t ld;
    int row[N];
    int k_n;

    __device__ __forceinline__ void init(const Operand& o, int first)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        ld = o.ld;
        k_n = o.k_n;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            row[i] = (wave + i * NW) * T::RPI + lane / T::CH;
            const int chunk = (lane % T::CH) ^ T::key(row[i]);
            const auto* b = static_cast<const typename E::elem*>(o.base);
            if constexpr (COLS) {
                const int col = first + chunk * E::EPC;
                at[i] = b + (col < o.n ? col : 0);
            } else {
                int r = min(first + row[i], o.n - 1);
                if (o.rows) r = o.rows[r];
                at[i] = b + r * o.ld + chunk * E::EPC;
            }
        }
    }
    __device__ __forceinline__ void issue(int k0, unsigned char* t) const
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const typename E::elem* p;
            if constexpr (COLS) p = at[i] + (int64_t)min(k0 + row[i], k_n - 1) * ld;
            else p = at[i] + k0;
            __builtin_amdgcn_global_load_lds((gptr_t)p, (lptr_t)(t + (wave + i * NW) * 1024), 16, 0, 0);
        }
    }
};

// acc[i][j]: block i of the first operand's rows (registers) and j of the second's (lanes); 4 wavefronts, 64 x 64 each
template <typename E, bool ACOL, bool BCOL>
struct Product {
    static constexpr int B = 128, NW = 4;
    using SA = Stager<E, B, NW, ACOL>;
    using SB = Stager<E, B, NW, BCOL>;
    static constexpr int BK = SA::BK, STEPS = BK / E::KS, LDS = 2 * (SA::BYTES + SB::BYTES);

    // sums over [k0, k1): k0 a multiple of BK; row operands hold whole slices
    static __device__ __forceinline__ void run(f32x16 (&acc)[2][2], const Operand& a, int a0, const Operand& b, int b0, int k0, int k1, unsigned char* lds)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, half = lane >> 5;
        const int wm = (wave >> 1) * 64, wn = (wave & 1) * 64;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
        SA sa;
        SB sb;
        sa.init(a, a0);
        sb.init(b, b0);
        if (k0 < k1) {
            sa.issue(k0, lds);
            sb.issue(k0, lds + SA::BYTES);
        }
        int stage = 0;
        for (int k = k0; k < k1; k += BK, stage ^= 1) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            unsigned char* ta = lds + stage * (SA::BYTES + SB::BYTES);
            unsigned char* tb = ta + SA::BYTES;
            if (k + BK < k1) {
                unsigned char* next = lds + (stage ^ 1) * (SA::BYTES + SB::BYTES);
                sa.issue(k + BK, next);
                sb.issue(k + BK, next + SA::BYTES);
            }
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                typename E::frag fa[2], fb[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if constexpr (ACOL) fa[i] = SA::T::template col_frag<true>(ta, 0, wm / 32 + i, s, lane);
                    else fa[i] = SA::T::row_frag(ta, wm + 32 * i + l32, s, half);
                    if constexpr (BCOL) fb[i] = SB::T::template col_frag<true>(tb, 0, wn / 32 + i, s, lane);
                    else fb[i] = SB::T::row_frag(tb, wn + 32 * i + l32, s, half);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc[i][j] = E::mma(fa[i], fb[j], acc[i][j]);
            }
        }
    }
};

struct Stat {
    float top, sum;         // sum of exp2(log2e (z - top))
};

// ---- forward: one 128 x 128 block of z (vocabulary in registers, tokens in lanes) -> a Stat per token and 64 entries of the vocabulary
template <typename E>
__global__ __launch_bounds__(256) void vocab_stats_kernel(VocabLoss p, const int32_t* count, const int32_t* index, Stat* stats, float* at_label)
{
    using P = Product<E, false, false>;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const int n = *count, t0 = blockIdx.x * kTok, v0 = blockIdx.y * kVoc;
    if (t0 >= n) return;
    f32x16 acc[2][2];
    P::run(acc, Operand{p.w, p.ldw, nullptr, p.vocab, 0}, v0, Operand{p.x, p.ldx, index, n, 0}, t0, 0, p.hidden, lds);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, half = lane >> 5;
    const int vb = v0 + (wave >> 1) * 64, tb = t0 + (wave & 1) * 64;
    if (vb >= p.vocab) return;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int t = tb + j * 32 + l32;
        const int label = t < n ? p.labels[index[t]] : -1;
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int v = vb + i * 32 + 8 * (e >> 2) + 4 * half + (e & 3);
                if (v == label) at_label[t] = acc[i][j][e];
                if (v >= p.vocab) acc[i][j][e] = -INFINITY;
                top = fmaxf(top, acc[i][j][e]);
            }
        top = lane_pair_max<32>(top);
        const float from = top == -INFINITY ? 0.f : top * kLog2e;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) sum += __builtin_amdgcn_exp2f(fmaf(acc[i][j][e], kLog2e, -from));
        sum = lane_pair_sum<32>(sum);
        if (t < n && half == 0) stats[(int64_t)(vb / 64) * p.tokens + t] = Stat{top, sum};
    }
}

// one wavefront a token: the ranges joined; tokens without a label get zeros
__global__ __launch_bounds__(256) void vocab_join_kernel(VocabLoss p, const int32_t* count, const int32_t* index, const Stat* stats, const float* at_label, int ranges)
{
    const int t = blockIdx.x * 256 + threadIdx.x;
    if (t < p.tokens && (uint32_t)p.labels[t] >= (uint32_t)p.vocab) p.loss[t] = p.lse[t] = 0.f;
    if (t >= *count) return;
    float top = -INFINITY;
    for (int r = 0; r < ranges; ++r) top = fmaxf(top, stats[(int64_t)r * p.tokens + t].top);
    const float from = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    for (int r = 0; r < ranges; ++r) {
        const Stat s = stats[(int64_t)r * p.tokens + t];
        sum = fmaf(s.sum, __builtin_amdgcn_exp2f((s.top - from) * kLog2e), sum);
    }
    const float lse = top + __builtin_amdgcn_logf(sum) * kLn2;
    const int at = index[t];
    p.lse[at] = lse;
    p.loss[at] = lse - at_label[t];
}

// ---- gradient
// the labelled rows of x behind one another
template <typename E>
__global__ __launch_bounds__(256) void labelled_rows_kernel(VocabLoss p, const int32_t* count, const int32_t* index, typename E::elem* out)
{
    const int per = p.hidden / E::EPC, n = *count;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int row = (int)(at / per), c = (int)(at - (int64_t)row * per) * E::EPC;
    if (row >= n) return;
    *reinterpret_cast<typename E::frag*>(out + (int64_t)row * p.hidden + c) =
        *reinterpret_cast<const typename E::frag*>(static_cast<const typename E::elem*>(p.x) + index[row] * p.ldx + c);
}

// dz of one piece of the vocabulary [piece0, piece0 + width) (columns beyond the vocabulary: 0), rows beyond the labelled ones up to a whole slice: 0
template <typename E>
__global__ __launch_bounds__(256) void vocab_dz_kernel(VocabLoss p, const int32_t* count, const int32_t* index, const typename E::elem* xc, int piece0, int width,
                                                       typename E::elem* dz)
{
    using P = Product<E, false, false>;
    typedef typename E::elem out4 __attribute__((ext_vector_type(4)));
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const int n = *count, t0 = blockIdx.x * kTok, v0 = piece0 + blockIdx.y * kVoc;
    if (t0 >= n) return;
    f32x16 acc[2][2];
    // (a tile behind the vocabulary, whose columns of dz are zeros, multiplies nothing)
    P::run(acc, Operand{p.w, p.ldw, nullptr, p.vocab, 0}, v0, Operand{xc, p.hidden, nullptr, n, 0}, t0, 0, v0 < p.vocab ? p.hidden : 0, lds);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, half = lane >> 5;
    const int vb = v0 + (wave >> 1) * 64, tb = t0 + (wave & 1) * 64;
    const int n_pad = (n + 63) & ~63;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int t = tb + j * 32 + l32;
        if (t >= n_pad) continue;
        const bool real = t < n;
        const int at = real ? index[t] : 0, label = real ? p.labels[at] : -1;
        const float lse = real ? p.lse[at] * kLog2e : 0.f, g = real ? p.weight[at] : 0.f;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int v = vb + i * 32 + 8 * q + 4 * half;
                out4 o;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float w = __builtin_amdgcn_exp2f(fmaf(acc[i][j][4 * q + e], kLog2e, -lse)) - (v + e == label ? 1.f : 0.f);
                    o[e] = (typename E::elem)(real && v + e < p.vocab ? w * g : 0.f);
                }
                *reinterpret_cast<out4*>(dz + (int64_t)t * width + v - piece0) = o;
            }
    }
}

// dx += dz W over one piece, float32 sums in memory; the piece is cut into `splits` ranges with sums of their own
template <typename E>
__global__ __launch_bounds__(256) void vocab_dx_kernel(VocabLoss p, const int32_t* count, const typename E::elem* dz, int piece0, int width, int splits, float* part)
{
    using P = Product<E, true, false>;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const int n = *count, t0 = blockIdx.x * 128, h0 = blockIdx.y * 128, split = blockIdx.z;
    if (t0 >= n) return;
    const int slices = width / P::BK, k0 = (int)((int64_t)slices * split / splits) * P::BK, k1 = (int)((int64_t)slices * (split + 1) / splits) * P::BK;
    f32x16 acc[2][2];
    const auto* w = static_cast<const typename E::elem*>(p.w) + (int64_t)piece0 * p.ldw;
    P::run(acc, Operand{w, p.ldw, nullptr, p.hidden, p.vocab - piece0}, h0, Operand{dz, width, nullptr, n, 0}, t0, k0, k1, lds);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, half = lane >> 5;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int t = t0 + (wave & 1) * 64 + j * 32 + l32;
        if (t >= n) continue;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int h = h0 + (wave >> 1) * 64 + i * 32 + 8 * q + 4 * half;
                if (h >= p.hidden) continue;
                f32x4* at = reinterpret_cast<f32x4*>(part + ((int64_t)split * p.tokens + t) * p.hidden + h);
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = acc[i][j][4 * q + e];
                if (piece0 > 0) v += *at;
                *at = v;
            }
    }
}

// dW of one piece: the sum over the labelled tokens
template <typename E, typename Out>
__global__ __launch_bounds__(256) void vocab_dw_kernel(VocabLoss p, const int32_t* count, const typename E::elem* dz, const typename E::elem* xc, int piece0, int width)
{
    using P = Product<E, true, true>;
    typedef Out out4 __attribute__((ext_vector_type(4)));
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const int n = *count, h0 = blockIdx.x * 128, v0 = blockIdx.y * 128;
    f32x16 acc[2][2];
    P::run(acc, Operand{xc, p.hidden, nullptr, p.hidden, n}, h0, Operand{dz, width, nullptr, width, (n + 63) & ~63}, v0, 0, (n + P::BK - 1) / P::BK * P::BK, lds);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, half = lane >> 5;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int v = piece0 + v0 + (wave & 1) * 64 + j * 32 + l32;
        if (v >= p.vocab) continue;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int h = h0 + (wave >> 1) * 64 + i * 32 + 8 * q + 4 * half;
                if (h >= p.hidden) continue;
                out4 o;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = (Out)acc[i][j][4 * q + e];
                *reinterpret_cast<out4*>(static_cast<Out*>(p.dw) + (int64_t)v * p.hidden + h) = o;
            }
    }
}

// dx: the ranges' sums put together and rounded, in the tokens' places; zeros for tokens without a label
template <typename E>
__global__ __launch_bounds__(256) void vocab_dx_rows_kernel(VocabLoss p, const int32_t* count, const int32_t* index, const float* part, int splits)
{
    const int per = p.hidden / 4;
    typedef typename E::elem out4 __attribute__((ext_vector_type(4)));
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int row = (int)(at / per), c = (int)(at - (int64_t)row * per) * 4;
    if (row >= p.tokens) return;
    auto* dx = static_cast<typename E::elem*>(p.dx);
    out4 o;
    if ((uint32_t)p.labels[row] >= (uint32_t)p.vocab) {
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (typename E::elem)0.f;
        *reinterpret_cast<out4*>(dx + (int64_t)row * p.hidden + c) = o;
    }
    if (row >= *count) return;
    f32x4 v{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < splits; ++s) v += *reinterpret_cast<const f32x4*>(part + ((int64_t)s * p.tokens + row) * p.hidden + c);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (typename E::elem)v[e];
    *reinterpret_cast<out4*>(dx + (int64_t)index[row] * p.hidden + c) = o;
}

size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

struct Plan {
    int piece, splits;
    size_t index, xc, dz, part, bytes;
};
Plan grad_plan(int f32, int tokens, int hidden, int vocab)
{
    const size_t es = f32 ? 4 : 2;
    const size_t rows = (size_t)(tokens + 127) / 128 * 128;
    Plan p;
    // pieces whose dz (at most 128 MB) stays in the last-level cache until both products have read it
    const size_t fit = (size_t)(128u << 20) / (rows * es) / kPieceGrain * kPieceGrain;
    const size_t whole = ((size_t)vocab + kPieceGrain - 1) / kPieceGrain * kPieceGrain;
    p.piece = (int)std::min(whole, std::max<size_t>(fit, 1024));
    // enough workgroups for dx, whose tiles are few
    const long tiles = (long)(rows / 128) * ((hidden + 127) / 128);
    p.splits = (int)std::max<long>(1, std::min<long>({8, 512 / tiles, p.piece / 512}));
    p.index = 256;
    p.xc = p.index + up256((size_t)tokens * 4);
    p.dz = p.xc + up256(rows * hidden * es);
    p.part = p.dz + up256(rows * p.piece * es);
    p.bytes = p.part + up256((size_t)p.splits * tokens * hidden * 4);
    return p;
}

template <typename K>
hipError_t with_lds(K* kernel, int bytes, std::atomic<uint64_t>& done)
{
    return ensure_dynamic_lds(reinterpret_cast<const void*>(kernel), bytes, done);
}

template <typename E>
hipError_t forward_of(const VocabLoss& p, hipStream_t stream)
{
    static std::atomic<uint64_t> done{0};
    constexpr int lds = Product<E, false, false>::LDS;
    hipError_t e = with_lds(vocab_stats_kernel<E>, lds, done);
    if (e != hipSuccess) return e;
    unsigned char* ws = static_cast<unsigned char*>(p.work);
    const int ranges = (p.vocab + 63) / 64;
    int32_t* count = reinterpret_cast<int32_t*>(ws);
    int32_t* index = reinterpret_cast<int32_t*>(ws + 256);
    float* at_label = reinterpret_cast<float*>(ws + 256 + up256((size_t)p.tokens * 4));
    Stat* stats = reinterpret_cast<Stat*>(ws + 256 + 2 * up256((size_t)p.tokens * 4));
    label_index_kernel<<<1, 1024, 0, stream>>>(p.labels, p.tokens, p.vocab, count, index);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    vocab_stats_kernel<E><<<dim3((p.tokens + kTok - 1) / kTok, (p.vocab + kVoc - 1) / kVoc), 256, lds, stream>>>(p, count, index, stats, at_label);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    vocab_join_kernel<<<(p.tokens + 255) / 256, 256, 0, stream>>>(p, count, index, stats, at_label, ranges);
    return hipGetLastError();
}

template <typename E>
hipError_t gradient_of(const VocabLoss& p, hipStream_t stream)
{
    typedef typename E::elem elem;
    static std::atomic<uint64_t> done_dz{0}, done_dx{0}, done_dw{0}, done_dwf{0};
    constexpr int lds_dz = Product<E, false, false>::LDS, lds_dx = Product<E, true, false>::LDS, lds_dw = Product<E, true, true>::LDS;
    hipError_t e;
    if ((e = with_lds(vocab_dz_kernel<E>, lds_dz, done_dz)) != hipSuccess || (e = with_lds(vocab_dx_kernel<E>, lds_dx, done_dx)) != hipSuccess ||
        (e = with_lds(vocab_dw_kernel<E, elem>, lds_dw, done_dw)) != hipSuccess || (e = with_lds(vocab_dw_kernel<E, float>, lds_dw, done_dwf)) != hipSuccess)
        return e;
    const Plan pl = grad_plan(E::SIZE == 4, p.tokens, p.hidden, p.vocab);
    unsigned char* ws = static_cast<unsigned char*>(p.work);
    int32_t* count = reinterpret_cast<int32_t*>(ws);
    int32_t* index = reinterpret_cast<int32_t*>(ws + pl.index);
    elem* xc = reinterpret_cast<elem*>(ws + pl.xc);
    elem* dz = reinterpret_cast<elem*>(ws + pl.dz);
    float* part = reinterpret_cast<float*>(ws + pl.part);
    const unsigned t_tiles = (p.tokens + 127) / 128, h_tiles = (p.hidden + 127) / 128;
    label_index_kernel<<<1, 1024, 0, stream>>>(p.labels, p.tokens, p.vocab, count, index);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    labelled_rows_kernel<E><<<(unsigned)(((int64_t)p.tokens * (p.hidden / E::EPC) + 255) / 256), 256, 0, stream>>>(p, count, index, xc);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    for (int v0 = 0; v0 < p.vocab; v0 += pl.piece) {
        const int width = std::min(pl.piece, (p.vocab - v0 + kPieceGrain - 1) / kPieceGrain * kPieceGrain);
        vocab_dz_kernel<E><<<dim3(t_tiles, width / kVoc), 256, lds_dz, stream>>>(p, count, index, xc, v0, width, dz);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        vocab_dx_kernel<E><<<dim3(t_tiles, h_tiles, pl.splits), 256, lds_dx, stream>>>(p, count, dz, v0, width, pl.splits, part);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        if (p.dw_f32) vocab_dw_kernel<E, float><<<dim3(h_tiles, width / 128), 256, lds_dw, stream>>>(p, count, dz, xc, v0, width);
        else vocab_dw_kernel<E, elem><<<dim3(h_tiles, width / 128), 256, lds_dw, stream>>>(p, count, dz, xc, v0, width);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    vocab_dx_rows_kernel<E><<<(unsigned)(((int64_t)p.tokens * (p.hidden / 4) + 255) / 256), 256, 0, stream>>>(p, count, index, part, pl.splits);
    return hipGetLastError();
}

}  // namespace

size_t vocab_loss_work(int tokens, int vocab) { return 256 + 2 * up256((size_t)tokens * 4) + (size_t)((vocab + 63) / 64) * tokens * sizeof(Stat); }
size_t vocab_loss_grad_work(int f32, int tokens, int hidden, int vocab) { return grad_plan(f32, tokens, hidden, vocab).bytes; }

hipError_t launch_vocab_loss(const VocabLoss& p, int f32, hipStream_t stream) { return f32 ? forward_of<F32>(p, stream) : forward_of<B16>(p, stream); }
hipError_t launch_vocab_loss_grad(const VocabLoss& p, int f32, hipStream_t stream) { return f32 ? gradient_of<F32>(p, stream) : gradient_of<B16>(p, stream); }

}  // namespace mt
