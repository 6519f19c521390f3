// Softmax cross entropy over a large vocabulary and its gradient (bfloat16 and float32); the logits are never stored.
//   z = x W^T,  lse_i = log sum_v exp z_iv,  loss_i = lse_i - z_i,label
//   dz = weight_i (exp(z_iv - lse_i) - [v = label_i]),  dx = dz W,  dW = dz^T x
//
// Tokens without a label are dropped on the device before anything is multiplied: `index` lists the labelled ones in order, and every product
// has as many rows (dW: as long a sum) as there are.  Forward: blocks of z are multiplied, reduced to a maximum and a sum of exponentials per
// token and range of the vocabulary, and the ranges are joined.  Gradient: for a piece of the vocabulary at a time dz is formed from z multiplied
// again (bfloat16: rounded to bfloat16, half a step of 2^-8 per term, as any operand of these products) and used for both gradients.  Multiplying again costs a
// quarter of the work and holds nothing between the two calls; keeping z in float32 would move 4 bytes for every 2 x hidden operations, twice, and hold
// tokens x vocab x 4 bytes: more time in bfloat16 up to a hidden size of about 1000, less in float32 (at 768 10 ps of products a logit against 2 of memory).
//
// What bounds it (MI355X).  Many tokens: the matrix rate; 4099 x 1024 x 128000, 97 % labelled, 4.2 ms for 4 products, 0.98 PFLOP/s (a library's product of
// 8192^3: 1.21), matrix instructions 41 to 66 % of the kernels' cycles.  8192 tokens of which 15 % are labelled, 768 x 30522: 339 us; 600 blocks of 256 x 256 on 256
// compute units leave the last round a third full.  5 tokens: one pass over the weights, 47 MB in 10 us, 4.5 TB/s, and a join of 4 us.  float32, 509 tokens,
// 768 x 30522: 825 us, 116 TFLOP/s (a library's 8192^3: 153).
#include "packed_tile.h"
#include "packed.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace mt {

namespace {

// ---- the labelled tokens, in order: index[0 .. *count).  One workgroup, 8 tokens a thread at a time (8192 tokens: one round).
__global__ __launch_bounds__(1024) void label_index_kernel(const int32_t* labels, int tokens, int vocab, int32_t* count, int32_t* index)
{
    __shared__ int wave_n[2][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int base = 0, turn = 0;
    for (int t0 = 0; t0 < tokens; t0 += 8192, turn ^= 1) {
        // a wavefront's 512 tokens as 8 rows of 64
        const int first = t0 + wave * 512 + lane;
        uint64_t has[8];
        int l[8], mine = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) l[k] = first + k * 64 < tokens ? labels[first + k * 64] : -1;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            has[k] = __ballot((uint32_t)l[k] < (uint32_t)vocab);
            mine += __popcll(has[k]);
        }
        if (lane == 0) wave_n[turn][wave] = mine;
        __syncthreads();
        int at = base;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            at += i < wave ? wave_n[turn][i] : 0;
            base += wave_n[turn][i];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if ((has[k] >> lane) & 1) index[at + __popcll(has[k] & ((1ull << lane) - 1))] = first + k * 64;
            at += __popcll(has[k]);
        }
    }
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

template <typename E, int B, int BK, int NW, bool COLS>
struct Stager {
    static constexpr int WIDTH = COLS ? B : BK, ROWS = COLS ? BK : B;
    using T = Tile<E, WIDTH>;
    static constexpr int BYTES = ROWS * T::ROWB, N = BYTES / 1024 / NW;
    static_assert(N * NW * 1024 == BYTES, "a tile must split evenly over wavefront loads");
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
    __device__ __forceinline__ void issue(int k0, uint32_t t) const
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const typename E::elem* p;
            if constexpr (COLS) p = at[i] + (int64_t)min(k0 + row[i], k_n - 1) * ld;
            else p = at[i] + k0;
            load_to_lds(p, t + (wave + i * NW) * 1024);
        }
    }
};

// A workgroup's BM x BN block of a product: WM x WN wavefronts of TMI x TNI blocks of 32 x 32; acc[i][j]: block i of the first operand's rows (registers),
// j of the second's (lanes).  Slices of BK elements of the sum go through a ring of STAGES in LDS, straight from memory; the barrier of a slice stands in
// its last step, when its operands are in registers, so that the next slice's first operands are read behind that step's matrix instructions.
template <typename E, bool ACOL, bool BCOL, int WM, int WN, int TMI, int TNI, int BK, int STAGES>
struct Product {
    static constexpr int BM = WM * TMI * 32, BN = WN * TNI * 32, NW = WM * WN, NT = NW * 64;
    using SA = Stager<E, BM, BK, NW, ACOL>;
    using SB = Stager<E, BN, BK, NW, BCOL>;
    static constexpr int STAGE = SA::BYTES + SB::BYTES, STEPS = BK / E::KS, LDS = STAGES * STAGE, LPS = SA::N + SB::N;
    static constexpr int kBK = BK, tmi = TMI, tni = TNI;
    static_assert(LDS <= 160 * 1024 && STAGES >= 2 && LPS * (STAGES - 2) < 64, "");

    static __device__ __forceinline__ void wait_slices(int n)       // all but the last n slices issued have landed
    {
        if (STAGES >= 4 && n >= 2) wait_loads<2 * LPS>();
        else if (STAGES >= 3 && n >= 1) wait_loads<LPS>();
        else wait_loads<0>();
    }
    static __device__ __forceinline__ int wave_m() { return (threadIdx.x >> 6) / WN * TMI * 32; }
    static __device__ __forceinline__ int wave_n() { return (threadIdx.x >> 6) % WN * TNI * 32; }

    // sums over [k0, k1): k0 a multiple of BK; row operands hold whole slices
    static __device__ __forceinline__ void run(f32x16 (&acc)[TMI][TNI], const Operand& a, int a0, const Operand& b, int b0, int k0, int k1, unsigned char* lds)
    {
        static_assert(STAGES <= 4, "wait_slices");
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, half = lane >> 5;
        const int wm = wave / WN * TMI * 32, wn = wave % WN * TNI * 32;
#pragma unroll
        for (int i = 0; i < TMI; ++i)
#pragma unroll
            for (int j = 0; j < TNI; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
        const int slices = (k1 - k0 + BK - 1) / BK;
        if (slices <= 0) return;
        SA sa;
        SB sb;
        sa.init(a, a0);
        sb.init(b, b0);
        const auto fill = [&](int s) {
            const uint32_t t = lds_address(lds) + s % STAGES * STAGE;
            sa.issue(k0 + s * BK, t);
            sb.issue(k0 + s * BK, t + SA::BYTES);
        };
        typename E::frag fa[2][TMI], fb[2][TNI];
        const auto read = [&](int buf, int s, int step) {
            const unsigned char* t = lds + s % STAGES * STAGE;
#pragma unroll
            for (int i = 0; i < TMI; ++i) {
                if constexpr (ACOL) fa[buf][i] = SA::T::template col_frag<true>(t, 0, wm / 32 + i, step, lane);
                else fa[buf][i] = SA::T::row_frag(t, wm + 32 * i + l32, step, half);
            }
#pragma unroll
            for (int j = 0; j < TNI; ++j) {
                if constexpr (BCOL) fb[buf][j] = SB::T::template col_frag<true>(t + SA::BYTES, 0, wn / 32 + j, step, lane);
                else fb[buf][j] = SB::T::row_frag(t + SA::BYTES, wn + 32 * j + l32, step, half);
            }
        };
        const auto multiply = [&](int buf) {
#pragma unroll
            for (int i = 0; i < TMI; ++i)
#pragma unroll
                for (int j = 0; j < TNI; ++j) acc[i][j] = E::mma(fa[buf][i], fb[buf][j], acc[i][j]);
        };
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s)
            if (s < slices) fill(s);
        wait_slices(min(STAGES - 2, slices - 1));
        __builtin_amdgcn_s_barrier();
        read(0, 0, 0);
        static_assert(STEPS % 2 == 0, "the operands' two buffers alternate by step");
        // slices whose refill exists: no branch inside, which would cut the reads off from the matrix instructions that cover them
        int s = 0;
        for (; s + STAGES - 1 < slices; ++s) {
#pragma unroll
            for (int step = 0; step < STEPS; ++step) {
                if (step + 1 < STEPS) {
                    read((step + 1) & 1, s, step + 1);
                    if (step == 0) fill(s + STAGES - 1);
                } else {
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    wait_loads<(STAGES - 2) * LPS>();
                    __builtin_amdgcn_s_barrier();
                    read(0, s + 1, 0);
                }
                multiply(step & 1);
                interleave();
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        for (; s < slices; ++s) {
#pragma unroll
            for (int step = 0; step < STEPS; ++step) {
                if (step + 1 < STEPS) read((step + 1) & 1, s, step + 1);
                else if (s + 1 < slices) {
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    wait_slices(slices - 2 - s);
                    __builtin_amdgcn_s_barrier();
                    read(0, s + 1, 0);
                }
                multiply(step & 1);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }

    // a step's LDS reads one or two behind each of its first matrix instructions
    static __device__ __forceinline__ void interleave()
    {
        constexpr int M = TMI * TNI * (E::SIZE == 2 ? 1 : 4), R = E::SIZE == 2 ? (ACOL ? 2 : 1) * TMI + (BCOL ? 2 : 1) * TNI : (ACOL ? 4 : 1) * TMI + (BCOL ? 4 : 1) * TNI;
        constexpr int EACH = (R + M - 2) / (M > 1 ? M - 1 : 1) > 0 ? (R + M - 2) / (M > 1 ? M - 1 : 1) : 1;
#pragma unroll
        for (int i = 0; i < (R + EACH - 1) / EACH; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, M, 0);
    }
};

// A workgroup's block to memory, row b (a lane's) of the block at row_at(b) (null: nowhere), its first `cols` columns.  The accumulators hold 4 columns of 32
// rows per instruction, which memory would see as 32 pieces of 16 bytes; through the idle ring they become whole rows, 16 bytes a lane.
template <typename P, typename Out, bool ADD, typename RowAt>
__device__ __forceinline__ void store_rows(const f32x16 (&acc)[P::tmi][P::tni], unsigned char* lds, int cols, RowAt row_at)
{
    typedef Out out4 __attribute__((ext_vector_type(4)));
    typedef Out out16 __attribute__((ext_vector_type(16 / sizeof(Out))));
    constexpr int ROWB = P::BM * sizeof(Out), LANES = ROWB / 16, ROWS = P::BN / P::tni, PER = 16 / sizeof(Out);
    static_assert(ROWS * ROWB <= P::LDS && P::NT % LANES == 0 && LANES >= 16, "");
    const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5, c = threadIdx.x % LANES;
    const int mine = P::wave_n() / P::tni + l32;
#pragma unroll
    for (int j = 0; j < P::tni; ++j) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < P::tmi; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int at = (P::wave_m() + i * 32 + 8 * q + 4 * half) * (int)sizeof(Out);
                out4 o;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = (Out)acc[i][j][4 * q + e];
                *reinterpret_cast<out4*>(lds + mine * ROWB + (((at >> 4) ^ (mine & 15)) << 4) + (at & 15)) = o;
            }
        __syncthreads();
#pragma unroll 4
        for (int r = threadIdx.x / LANES; r < ROWS; r += P::NT / LANES) {
            Out* row = row_at((r >> 5) * (P::tni * 32) + j * 32 + (r & 31));
            if (!row || c * PER >= cols) continue;
            out16 v = *reinterpret_cast<const out16*>(lds + r * ROWB + ((c ^ (r & 15)) << 4));
            out16* to = reinterpret_cast<out16*>(row + c * PER);
            if constexpr (ADD) v += *to;
            *to = v;
        }
    }
}

// Workgroup id -> block of a grid of m x n: consecutive ids go to the 8 XCDs in turn, so each gets a run of blocks of its own, which walks bands of
// kBand blocks of m and shares their operands in that XCD's L2.
constexpr int kBand = 8;
__device__ __forceinline__ void block_of(int id, int m, int n, int& bm, int& bn)
{
    const int total = m * n, x = id & 7, q = total >> 3, r = total & 7;
    const int t = x * q + min(x, r) + (id >> 3);
    const int band = t / (kBand * n), in_band = min(kBand, m - band * kBand), tb = t - band * kBand * n;
    bn = tb / in_band;
    bm = band * kBand + tb % in_band;
}

// Blocks of a launch (weights' side x tokens): FEW 128 x 32 of four wavefronts with one 32 x 32 block each (a stream of weights), MID 128 x 128, BIG 256 x 256
// of 8 wavefronts (bfloat16).
enum { FEW, MID, BIG };
constexpr int kFewTokens = 64;
template <typename E, bool ACOL, bool BCOL, int C>
struct Pick;
template <bool A, bool B>
struct Pick<B16, A, B, FEW> { typedef Product<B16, A, B, 4, 1, 1, 1, 64, 4> P; };
template <bool A, bool B>
struct Pick<B16, A, B, MID> { typedef Product<B16, A, B, 2, 2, 2, 2, 32, 4> P; };
template <bool A, bool B>
struct Pick<B16, A, B, BIG> { typedef Product<B16, A, B, 2, 4, 4, 2, 32, 4> P; };
template <bool A, bool B>
struct Pick<F32, A, B, FEW> { typedef Product<F32, A, B, 4, 1, 1, 1, 32, 4> P; };
template <bool A, bool B>
struct Pick<F32, A, B, MID> { typedef Product<F32, A, B, 2, 2, 2, 2, 32, 2> P; };

// The reference is log2e times the largest z, as rounded, and nothing rounds between it and the exponents log2e z - ref (one fused operation): the loss, which is
// their sum's logarithm less the label's exponent, is then good to a few 2^-24, where lse - z would be good to as many of lse, of which little is left over for
// a token that the model is sure of.
struct Stat {
    float ref, sum;         // sum of exp2(log2e z - ref)
};

// ---- forward: a block of z (vocabulary in registers, tokens in lanes) -> a Stat per token and wavefront's range of the vocabulary
template <typename E, int C>
__global__ __launch_bounds__((Pick<E, false, false, C>::P::NT)) void vocab_stats_kernel(VocabLoss p, const int32_t* count, const int32_t* index, Stat* stats, float* at_label)
{
    typedef typename Pick<E, false, false, C>::P P;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const int n = count ? *count : p.tokens, t_blocks = (n + P::BN - 1) / P::BN, v_blocks = (p.vocab + P::BM - 1) / P::BM;
    if ((int)blockIdx.x >= t_blocks * v_blocks) return;
    int bt, bv;
    block_of(blockIdx.x, t_blocks, v_blocks, bt, bv);
    const int t0 = bt * P::BN, v0 = bv * P::BM;
    f32x16 acc[P::tmi][P::tni];
    P::run(acc, Operand{p.w, p.ldw, nullptr, p.vocab, 0}, v0, Operand{p.x, p.ldx, index, n, 0}, t0, 0, p.hidden, lds);
    const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
    const int vb = v0 + P::wave_m(), tb = t0 + P::wave_n();
    if (vb >= p.vocab) return;
#pragma unroll
    for (int j = 0; j < P::tni; ++j) {
        const int t = tb + j * 32 + l32;
        const int label = t < n ? p.labels[index ? index[t] : t] : -1;
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int i = 0; i < P::tmi; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int v = vb + i * 32 + 8 * (e >> 2) + 4 * half + (e & 3);
                if (v == label) at_label[t] = acc[i][j][e];
                if (v >= p.vocab) acc[i][j][e] = -INFINITY;
                top = fmaxf(top, acc[i][j][e]);
            }
        top = lane_pair_max<32>(top);
        const float ref = top * kLog2e, from = top == -INFINITY ? 0.f : ref;
#pragma unroll
        for (int i = 0; i < P::tmi; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) sum += __builtin_amdgcn_exp2f(fmaf(acc[i][j][e], kLog2e, -from));
        sum = lane_pair_sum<32>(sum);
        if (t < n && half == 0) stats[(int64_t)(vb / (P::tmi * 32)) * p.tokens + t] = Stat{ref, sum};
    }
}

// the ranges joined: TOK tokens a workgroup, 256 / TOK threads each; tokens without a label get zeros
template <int TOK>
__global__ __launch_bounds__(256) void vocab_join_kernel(VocabLoss p, const int32_t* count, const int32_t* index, const Stat* stats, const float* at_label, int ranges)
{
    constexpr int SLICES = 256 / TOK;
    __shared__ Stat part[SLICES][TOK];
    const int slice = threadIdx.x / TOK, t = blockIdx.x * TOK + threadIdx.x % TOK;
    const bool in = t < p.tokens, none = in && (uint32_t)p.labels[t] >= (uint32_t)p.vocab;
    if (slice == 0 && none) p.loss[t] = p.lse[t] = 0.f;
    const int n = count ? *count : p.tokens;
    if ((int)blockIdx.x * TOK >= n) return;
    const bool mine = t < n && (index || !none);
    Stat s{-INFINITY, 0.f};
    for (int r0 = slice; r0 < ranges; r0 += 8 * SLICES) {
        Stat v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = stats[(int64_t)min(r0 + k * SLICES, ranges - 1) * p.tokens + min(t, n - 1)];
        float ref = s.ref;
#pragma unroll
        for (int k = 0; k < 8; ++k) ref = fmaxf(ref, v[k].ref);
        const float from = ref == -INFINITY ? 0.f : ref;
        s.sum *= __builtin_amdgcn_exp2f(s.ref - from);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (r0 + k * SLICES < ranges) s.sum = fmaf(v[k].sum, __builtin_amdgcn_exp2f(v[k].ref - from), s.sum);
        s.ref = ref;
    }
    part[slice][threadIdx.x % TOK] = s;
    __syncthreads();
    if (slice != 0 || !mine) return;
    float ref = -INFINITY;
#pragma unroll
    for (int k = 0; k < SLICES; ++k) ref = fmaxf(ref, part[k][threadIdx.x].ref);
    const float from = ref == -INFINITY ? 0.f : ref;
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < SLICES; ++k) sum = fmaf(part[k][threadIdx.x].sum, __builtin_amdgcn_exp2f(part[k][threadIdx.x].ref - from), sum);
    const float log_sum = __builtin_amdgcn_logf(sum), loss = (log_sum - fmaf(at_label[t], kLog2e, -ref)) * kLn2;
    const int at = index ? index[t] : t;
    p.lse[at] = fmaf(ref, kLn2, log_sum * kLn2);
    p.loss[at] = loss < 0.f ? 0.f : loss;
}

// ---- gradient
// the labelled rows of x behind one another: a workgroup a row
template <typename E>
__global__ __launch_bounds__(256) void labelled_rows_kernel(VocabLoss p, const int32_t* count, const int32_t* index, typename E::elem* out)
{
    const int row = blockIdx.x;
    if (row >= *count) return;
    const typename E::elem* from = static_cast<const typename E::elem*>(p.x) + index[row] * p.ldx;
    for (int c = threadIdx.x * E::EPC; c < p.hidden; c += blockDim.x * E::EPC)
        *reinterpret_cast<typename E::frag*>(out + (int64_t)row * p.hidden + c) = *reinterpret_cast<const typename E::frag*>(from + c);
}

// dz of one piece of the vocabulary [piece0, piece0 + width) (columns beyond the vocabulary: 0), rows beyond the labelled ones up to a whole slice: 0
template <typename E, int C>
__global__ __launch_bounds__((Pick<E, false, false, C>::P::NT)) void vocab_dz_kernel(VocabLoss p, const int32_t* count, const int32_t* index, const typename E::elem* xc,
                                                                                     int piece0, int width, typename E::elem* dz)
{
    typedef typename Pick<E, false, false, C>::P P;
    typedef typename E::elem out4 __attribute__((ext_vector_type(4)));
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const int n = *count, t_blocks = (n + P::BN - 1) / P::BN, v_blocks = width / P::BM;
    if ((int)blockIdx.x >= t_blocks * v_blocks) return;
    int bt, bv;
    block_of(blockIdx.x, t_blocks, v_blocks, bt, bv);
    const int t0 = bt * P::BN, v0 = piece0 + bv * P::BM;
    f32x16 acc[P::tmi][P::tni];
    // (a block behind the vocabulary, whose columns of dz are zeros, multiplies nothing)
    P::run(acc, Operand{p.w, p.ldw, nullptr, p.vocab, 0}, v0, Operand{xc, p.hidden, nullptr, n, 0}, t0, 0, v0 < p.vocab ? p.hidden : 0, lds);
    const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
    const int vb = v0 + P::wave_m(), tb = t0 + P::wave_n();
    const int n_pad = (n + 63) & ~63;
    // straight from the accumulators, 8 bytes a lane: the exponentials between the stores leave them time (through LDS as whole rows: 3 % slower)
#pragma unroll
    for (int j = 0; j < P::tni; ++j) {
        const int t = tb + j * 32 + l32;
        if (t >= n_pad) continue;
        const bool real = t < n;
        const int at = real ? index[t] : 0, label = (real ? p.labels[at] : -1) - vb - 4 * half;
        const float lse = real ? p.lse[at] * kLog2e : 0.f, g = real ? p.weight[at] : 0.f;
        typename E::elem* row = dz + (int64_t)t * width + vb - piece0 + 4 * half;
#pragma unroll
        for (int i = 0; i < P::tmi; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int v = i * 32 + 8 * q;
                out4 o;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float w = __builtin_amdgcn_exp2f(fmaf(acc[i][j][4 * q + e], kLog2e, -lse));
                    w = v + e == label ? w - 1.f : w;
                    o[e] = (typename E::elem)(real && vb + 4 * half + v + e < p.vocab ? w * g : 0.f);
                }
                *reinterpret_cast<out4*>(row + v) = o;
            }
    }
}

// How many ranges of the vocabulary dx is summed in: as many as fill the chip with the blocks that n labelled tokens have.
struct Ranges {
    int most, blocks;       // most ranges; workgroups wanted
    __host__ __device__ int of(int64_t tiles) const
    {
        const int64_t r = blocks / (tiles > 0 ? tiles : 1);
        return (int)(r < 1 ? 1 : r < most ? r : most);
    }
};

// dx += dz W over one piece, float32 sums in memory, one per range
template <typename E, int C>
__global__ __launch_bounds__((Pick<E, true, false, C>::P::NT)) void vocab_dx_kernel(VocabLoss p, const int32_t* count, const typename E::elem* dz, int piece0, int width,
                                                                                    Ranges ranges, float* part)
{
    typedef typename Pick<E, true, false, C>::P P;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const int n = *count, t_blocks = (n + P::BN - 1) / P::BN, h_blocks = (p.hidden + P::BM - 1) / P::BM, tiles = t_blocks * h_blocks, split_n = ranges.of(tiles);
    if ((int)blockIdx.x >= tiles * split_n) return;
    // (an XCD's workgroups share ranges, whose part of W and dz its L2 then holds)
    int bt, split;
    block_of(blockIdx.x, tiles, split_n, bt, split);
    const int t0 = bt / h_blocks * P::BN, h0 = bt % h_blocks * P::BM;
    const int slices = width / P::kBK, k0 = (int)((int64_t)slices * split / split_n) * P::kBK, k1 = (int)((int64_t)slices * (split + 1) / split_n) * P::kBK;
    f32x16 acc[P::tmi][P::tni];
    const auto* w = static_cast<const typename E::elem*>(p.w) + (int64_t)piece0 * p.ldw;
    P::run(acc, Operand{w, p.ldw, nullptr, p.hidden, p.vocab - piece0}, h0, Operand{dz, width, nullptr, n, 0}, t0, k0, k1, lds);
    const auto row_at = [&](int b) { return t0 + b < n ? part + ((int64_t)split * n + t0 + b) * p.hidden + h0 : nullptr; };
    if (piece0 > 0) store_rows<P, float, true>(acc, lds, p.hidden - h0, row_at);
    else store_rows<P, float, false>(acc, lds, p.hidden - h0, row_at);
}

// dW of one piece: the sum over the labelled tokens
template <typename E, typename Out, int C>
__global__ __launch_bounds__((Pick<E, true, true, C>::P::NT)) void vocab_dw_kernel(VocabLoss p, const int32_t* count, const typename E::elem* dz,
                                                                                   const typename E::elem* xc, int piece0, int width)
{
    typedef typename Pick<E, true, true, C>::P P;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const int n = *count, h_blocks = (p.hidden + P::BM - 1) / P::BM, v_blocks = (width + P::BN - 1) / P::BN;
    int bh, bv;
    block_of(blockIdx.x, h_blocks, v_blocks, bh, bv);
    const int h0 = bh * P::BM, v0 = bv * P::BN;
    f32x16 acc[P::tmi][P::tni];
    P::run(acc, Operand{xc, p.hidden, nullptr, p.hidden, n}, h0, Operand{dz, width, nullptr, width, (n + 63) & ~63}, v0, 0, n, lds);
    const int rows = min(p.vocab - piece0, width) - v0;
    store_rows<P, Out, false>(acc, lds, p.hidden - h0, [&](int b) { return b < rows ? static_cast<Out*>(p.dw) + (int64_t)(piece0 + v0 + b) * p.hidden + h0 : nullptr; });
}

// dx: the ranges' sums put together and rounded, in the tokens' places; zeros for tokens without a label.  A workgroup a row.
template <typename E>
__global__ __launch_bounds__(256) void vocab_dx_rows_kernel(VocabLoss p, const int32_t* count, const int32_t* index, const float* part, Ranges ranges, int bm, int bn)
{
    typedef typename E::elem out4 __attribute__((ext_vector_type(4)));
    const int row = blockIdx.x, n = *count;
    auto* dx = static_cast<typename E::elem*>(p.dx);
    if ((uint32_t)p.labels[row] >= (uint32_t)p.vocab)
        for (int c = threadIdx.x * 4; c < p.hidden; c += blockDim.x * 4) {
            out4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = (typename E::elem)0.f;
            *reinterpret_cast<out4*>(dx + (int64_t)row * p.hidden + c) = o;
        }
    if (row >= n) return;
    const int splits = ranges.of((int64_t)((n + bn - 1) / bn) * ((p.hidden + bm - 1) / bm)), to = index[row];
    for (int c = threadIdx.x * 4; c < p.hidden; c += blockDim.x * 4) {
        f32x4 v{0.f, 0.f, 0.f, 0.f};
        for (int s0 = 0; s0 < splits; s0 += 8) {
            f32x4 x[8];
#pragma unroll
            for (int s = 0; s < 8; ++s) x[s] = *reinterpret_cast<const f32x4*>(part + ((int64_t)min(s0 + s, splits - 1) * n + row) * p.hidden + c);
#pragma unroll
            for (int s = 0; s < 8; ++s)
                if (s0 + s < splits) v += x[s];
        }
        out4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (typename E::elem)v[e];
        *reinterpret_cast<out4*>(dx + (int64_t)to * p.hidden + c) = o;
    }
}

// The kind of blocks, by the bound on the tokens (the count of the labelled ones is known on the device alone).  Measured on both sides (30522 x 768, us):
//   FEW instead of MID: 5 tokens 15.3, not 20.1; 64 tokens 16.8, not 21.9 (float32 39, not 66; gradient 71.9, not 78.5).  128 tokens 22.7, not 23.0, but
//   with the gradient 93.8, not 89.6.
//   BIG instead of MID, where its blocks are as many as the chip has compute units: 600 tokens with gradient 210, not 220; 2048 491, not 563; 8192 of which
//   15 % are labelled 326, not 352.  With fewer blocks than that some compute units would have none.
template <typename E>
int blocks_for(int tokens, int other)
{
    if (tokens <= kFewTokens) return FEW;
    if (E::SIZE == 2 && (int64_t)((tokens + 255) / 256) * ((other + 255) / 256) >= 256) return BIG;
    return MID;
}
template <typename E, typename F>
hipError_t with_blocks(int kind, F&& f)
{
    if (kind == FEW) return f(std::integral_constant<int, FEW>());
    if constexpr (E::SIZE == 2) {
        if (kind == BIG) return f(std::integral_constant<int, BIG>());
    }
    return f(std::integral_constant<int, MID>());
}
int range_of(int kind) { return kind == FEW ? 32 : kind == MID ? 64 : 128; }        // vocabulary entries of a Stat

struct Plan {
    int piece;
    Ranges ranges;
    size_t index, xc, dz, part, bytes;
};
template <typename E>
Plan grad_plan(int tokens, int hidden, int vocab)
{
    const size_t es = E::SIZE, rows = (size_t)(tokens + 63) / 64 * 64;
    Plan p;
    // pieces of the vocabulary: dz of at most 512 MB, or of 1024 entries where those are more (from 2^18 tokens on in bfloat16, 2^17 in float32; then 2 or 4 KB a token)
    const size_t fit = (size_t)(512u << 20) / (rows * es) / 256 * 256, whole = ((size_t)vocab + 255) / 256 * 256;
    p.piece = (int)std::min(whole, std::max<size_t>(fit, 1024));
    const int kind = blocks_for<E>(tokens, vocab), bm = kind == BIG ? 256 : 128, bn = kind == BIG ? 256 : kind == MID ? 128 : 32, h_blocks = (hidden + bm - 1) / bm;
    p.ranges = Ranges{std::max(1, std::min(64, p.piece / 256)), kind == BIG ? 256 : 512};
    const size_t part_rows = std::max<size_t>(tokens, std::min<size_t>((size_t)p.ranges.most * tokens, (size_t)p.ranges.blocks * bn / h_blocks));
    p.index = 256;
    p.xc = p.index + up256((size_t)tokens * 4);
    p.dz = p.xc + up256(rows * hidden * es);
    p.part = p.dz + up256(rows * p.piece * es);
    p.bytes = p.part + up256(part_rows * hidden * 4);
    return p;
}

template <typename E>
hipError_t forward_of(const VocabLoss& p, hipStream_t stream)
{
    const int kind = blocks_for<E>(p.tokens, p.vocab), ranges = (p.vocab + range_of(kind) - 1) / range_of(kind);
    unsigned char* ws = static_cast<unsigned char*>(p.work);
    const size_t list = up256((size_t)p.tokens * 4);
    int32_t* count = reinterpret_cast<int32_t*>(ws);
    int32_t* index = reinterpret_cast<int32_t*>(ws + 256);
    float* at_label = reinterpret_cast<float*>(ws + 256 + list);
    Stat* stats = reinterpret_cast<Stat*>(ws + 256 + 2 * list);
    hipError_t e;
    if (kind == FEW) count = index = nullptr;           // a block takes all the tokens: nothing to gain by listing the labelled ones
    else {
        label_index_kernel<<<1, 1024, 0, stream>>>(p.labels, p.tokens, p.vocab, count, index);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    e = with_blocks<E>(kind, [&](auto c) {
        typedef typename Pick<E, false, false, c.value>::P P;
        static std::atomic<uint64_t> done{0};
        const hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void*>(vocab_stats_kernel<E, c.value>), P::LDS, done);
        if (e != hipSuccess) return e;
        const int64_t grid = (int64_t)((p.tokens + P::BN - 1) / P::BN) * ((p.vocab + P::BM - 1) / P::BM);
        if (!fits_launch(grid, P::NT)) return hipErrorInvalidValue;
        vocab_stats_kernel<E, c.value><<<(unsigned)grid, P::NT, P::LDS, stream>>>(p, count, index, stats, at_label);
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    // few tokens: more threads each (a workgroup of 4 tokens instead of 16: 5 tokens 15.3 us, not 17.7; 64 21.2, not 21.9; 256 30.4, not 30.5; 1000 65.8, not 63.4)
    if (p.tokens <= 256) vocab_join_kernel<4><<<(p.tokens + 3) / 4, 256, 0, stream>>>(p, count, index, stats, at_label, ranges);
    else vocab_join_kernel<16><<<(p.tokens + 15) / 16, 256, 0, stream>>>(p, count, index, stats, at_label, ranges);
    return hipGetLastError();
}

template <typename E>
hipError_t gradient_of(const VocabLoss& p, hipStream_t stream)
{
    typedef typename E::elem elem;
    hipError_t e;
    const Plan pl = grad_plan<E>(p.tokens, p.hidden, p.vocab);
    unsigned char* ws = static_cast<unsigned char*>(p.work);
    int32_t* count = reinterpret_cast<int32_t*>(ws);
    int32_t* index = reinterpret_cast<int32_t*>(ws + pl.index);
    elem* xc = reinterpret_cast<elem*>(ws + pl.xc);
    elem* dz = reinterpret_cast<elem*>(ws + pl.dz);
    float* part = reinterpret_cast<float*>(ws + pl.part);
    label_index_kernel<<<1, 1024, 0, stream>>>(p.labels, p.tokens, p.vocab, count, index);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    labelled_rows_kernel<E><<<p.tokens, std::min(256, (p.hidden / E::EPC + 63) / 64 * 64), 0, stream>>>(p, count, index, xc);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    return with_blocks<E>(blocks_for<E>(p.tokens, p.vocab), [&](auto c) {
        constexpr int C = c.value, CW = C == FEW ? MID : C;      // (dW has no tokens among its blocks)
        typedef typename Pick<E, false, false, C>::P PZ;
        typedef typename Pick<E, true, false, C>::P PX;
        typedef typename Pick<E, true, true, CW>::P PW;
        static std::atomic<uint64_t> done_z{0}, done_x{0}, done_w{0}, done_wf{0};
        hipError_t e;
        if ((e = ensure_dynamic_lds(reinterpret_cast<const void*>(vocab_dz_kernel<E, C>), PZ::LDS, done_z)) != hipSuccess ||
            (e = ensure_dynamic_lds(reinterpret_cast<const void*>(vocab_dx_kernel<E, C>), PX::LDS, done_x)) != hipSuccess ||
            (e = ensure_dynamic_lds(reinterpret_cast<const void*>(vocab_dw_kernel<E, elem, CW>), PW::LDS, done_w)) != hipSuccess ||
            (e = ensure_dynamic_lds(reinterpret_cast<const void*>(vocab_dw_kernel<E, float, CW>), PW::LDS, done_wf)) != hipSuccess)
            return e;
        for (int v0 = 0; v0 < p.vocab; v0 += pl.piece) {
            const int width = std::min(pl.piece, (p.vocab - v0 + 255) / 256 * 256);
            const int64_t grid_z = (int64_t)((p.tokens + PZ::BN - 1) / PZ::BN) * (width / PZ::BM);
            const int64_t tiles_x = (int64_t)((p.tokens + PX::BN - 1) / PX::BN) * ((p.hidden + PX::BM - 1) / PX::BM), grid_x = std::max<int64_t>(tiles_x, pl.ranges.blocks);
            const int64_t grid_w = (int64_t)((p.hidden + PW::BM - 1) / PW::BM) * ((width + PW::BN - 1) / PW::BN);
            if (!fits_launch(std::max({grid_z, grid_x, grid_w}), 512)) return hipErrorInvalidValue;
            vocab_dz_kernel<E, C><<<(unsigned)grid_z, PZ::NT, PZ::LDS, stream>>>(p, count, index, xc, v0, width, dz);
            if ((e = hipGetLastError()) != hipSuccess) return e;
            vocab_dx_kernel<E, C><<<(unsigned)grid_x, PX::NT, PX::LDS, stream>>>(p, count, dz, v0, width, pl.ranges, part);
            if ((e = hipGetLastError()) != hipSuccess) return e;
            if (p.dw_f32) vocab_dw_kernel<E, float, CW><<<(unsigned)grid_w, PW::NT, PW::LDS, stream>>>(p, count, dz, xc, v0, width);
            else vocab_dw_kernel<E, elem, CW><<<(unsigned)grid_w, PW::NT, PW::LDS, stream>>>(p, count, dz, xc, v0, width);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
        vocab_dx_rows_kernel<E><<<p.tokens, std::min(256, (p.hidden / 4 + 63) / 64 * 64), 0, stream>>>(p, count, index, part, pl.ranges, PX::BM, PX::BN);
        return hipGetLastError();
    });
}

}  // namespace

size_t vocab_loss_work(int tokens, int vocab)
{
    const int range = range_of(tokens <= kFewTokens ? FEW : MID);
    return 256 + 2 * up256((size_t)tokens * 4) + (size_t)((vocab + range - 1) / range) * tokens * sizeof(Stat);
}
size_t vocab_loss_grad_work(int f32, int tokens, int hidden, int vocab)
{
    return f32 ? grad_plan<F32>(tokens, hidden, vocab).bytes : grad_plan<B16>(tokens, hidden, vocab).bytes;
}

hipError_t launch_vocab_loss(const VocabLoss& p, int f32, hipStream_t stream) { return f32 ? forward_of<F32>(p, stream) : forward_of<B16>(p, stream); }
hipError_t launch_vocab_loss_grad(const VocabLoss& p, int f32, hipStream_t stream) { return f32 ? gradient_of<F32>(p, stream) : gradient_of<B16>(p, stream); }

}  // namespace mt
