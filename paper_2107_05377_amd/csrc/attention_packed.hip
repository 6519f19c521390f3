// Attention over packed sequences, causal or not, with grouped heads, and its gradient (bfloat16 and float32).
//
// Sequence b owns query rows q_start[b] .. q_start[b+1]-1 and key rows k_start[b] .. ; with Lq and Lk of them, query i sees the keys
// j <= i + Lk - Lq (causal: the last query sees the last key) or all Lk.  Query head a reads key head a / group.
//   S = scale q k^T,  lse = log sum_visible exp S,  P = exp(S - lse),  ctx = P v
//   delta = sum P (dctx v^T) = dctx . ctx,  dS = P (dctx v^T - delta),  dv = P^T dctx,  dq = scale dS k,  dk = scale dS^T q
//
// Rows.  The query heads of a group share keys and values, so their rows are one list: row r of a (sequence, key head) is query r / group
// of head r % group.  A group of 4 heads then needs its keys once, a single token has `group` rows, and dk, dv come out summed over the group.
//
// Matrix instructions: 32x32 blocks with float32 sums.  The forward pass and dq hold rows fixed and compute S^T = k q^T: a lane then holds ONE
// row's scores of 16 of 32 keys, so that the softmax needs one exchange per block (with the other half of the wavefront), and P^T is in the
// registers that the next product takes as its second operand.  The order of a sum is free, so the first operand (v^T or k^T, rows = head
// columns) is read from the row-major LDS tile in the key order in which P^T lies: bfloat16 by transposing LDS reads, float32 by plain ones.
// dk and dv hold keys fixed and compute S = q k^T, with the same step from S to the product over rows.
//
// Nothing that a row does not see reaches it: scores are replaced, not multiplied by zero, and in blocks that a mask cuts, a non-finite first
// operand is kept out of the product and put back for the rows that see it.
//
// What bounds it (MI355X, bfloat16 unless said otherwise; times of whole calls among others, shares of a call and busy pipes from a profiler).  Forward, 8192
// tokens, 32 heads on 8 of D = 128, causal: 548 us, 1.00 PFLOP/s, matrix and vector instructions (exp, maximum, rounding of P) in turn, 48 % of the cycles each.
// D = 64 has half the matrix work for the same softmax: 16 heads on 4 over 9 documents of 300..4001 tokens, forward and gradient 451 us, of which the forward
// pass is 22 % (vector instructions 66 %, matrix 33 % of its cycles), dq 30 % (56 and 36), dk and dv 45 % (37 and 31, with two
// wavefronts per SIMD), delta 4 %.  256 sentences of 16..128 tokens, twelve heads: 35 us, start-up of a workgroup that has one or two key blocks (matrix 8 %).
// Single tokens against a cache of 100..8191 keys: 39 us for 125 MB, 3.2 TB/s, where a copy of that size reaches 4.7.  float32: its matrix instructions have
// a sixteenth of the rate; forward and gradient of 7 sequences of 60..509 tokens, a few hundred workgroups: 121 us.
// Heads between 64 and 128 columns do the matrix work of 128, those below 64 that of 64: the documents with D = 128 845 us, 80 785, 32 390 on a card
// where D = 64 takes 434.
#include "packed_tile.h"
#include "packed.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace mt {

namespace {

// the accumulators of a 32x32 block as the second operand of a product over its rows, step c
__device__ __forceinline__ bf16x8 acc_frag(const f32x16& s, int c, B16)
{
    bf16x8 f;
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = (__bf16)s[8 * c + j];
    return f;
}
__device__ __forceinline__ f32x4 acc_frag(const f32x16& s, int c, F32)
{
    f32x4 f;
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = s[4 * c + j];
    return f;
}

// ---- non-finite operands of a block that a mask cuts
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <typename E>
__device__ __forceinline__ bool any_bad(const typename E::frag& f)
{
    constexpr uint32_t FULL = E::SIZE == 2 ? 0x7F807F80u : 0x7F800000u, CARRY = E::SIZE == 2 ? 0x00800080u : 0x00800000u, SIGN = E::SIZE == 2 ? 0x80008000u : 0x80000000u;
    const u32x4 v = __builtin_bit_cast(u32x4, f);       // (of the whole vector: a bit cast of one element reads element 0)
    uint32_t t = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) t |= (v[j] & FULL) + CARRY;         // a full exponent carries into the sign's place
    return (t & SIGN) != 0;
}
// non-finite elements replaced by 0
template <typename E>
__device__ __forceinline__ void drop_bad(typename E::frag& f)
{
    u32x4 v = __builtin_bit_cast(u32x4, f);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (E::SIZE == 2) {
            const uint32_t t = (v[j] & 0x7F807F80u) + 0x00800080u;
            v[j] &= ((t & 0x8000u) ? 0u : 0xFFFFu) | ((t >> 31) ? 0u : 0xFFFF0000u);
        } else v[j] = ((v[j] & 0x7F800000u) + 0x00800000u) >> 31 ? 0u : v[j];
    }
    f = __builtin_bit_cast(typename E::frag, v);
}

// acc += (columns of the tile) x w, w the accumulators of a block of 32 rows (of the sum), 0 in row k of a lane that does not see it (sees(k)); `cut`:
// there are such.  What is not seen must not reach the result, but 0 times a non-finite operand is NaN: where a cut block's operands hold such
// (which a few instructions tell), they are taken out, and put back one by one for the lanes that see them.  w carries a sign (dS) or not (P):
// an infinity is put back with its own sign only for P, as NaN for dS.
template <typename E, int DP, bool SIGNED, typename Sees>
__device__ __forceinline__ void add_product(f32x16 (&acc)[DP / 32], const unsigned char* t, int row0, const f32x16& w, bool cut, Sees sees, int lane)
{
    using T = Tile<E, DP>;
    constexpr int STEPS = 32 / E::KS;
    typename E::frag wf[STEPS];
#pragma unroll
    for (int c = 0; c < STEPS; ++c) wf[c] = acc_frag(w, c, E{});
    // 64 columns at a time: their operands are read at once, and there is one branch for the rare case
#pragma unroll
    for (int d0 = 0; d0 < DP / 32; d0 += 2) {
        typename E::frag a[2][STEPS];
#pragma unroll
        for (int db = 0; db < 2; ++db)
#pragma unroll
            for (int c = 0; c < STEPS; ++c) a[db][c] = T::col_frag(t, row0, d0 + db, c, lane);
        if (cut) {
            bool bad = false;
#pragma unroll
            for (int db = 0; db < 2; ++db)
#pragma unroll
                for (int c = 0; c < STEPS; ++c) bad |= any_bad<E>(a[db][c]);
            if (__any(bad)) {
#pragma unroll
                for (int db = 0; db < 2; ++db)
#pragma unroll
                    for (int c = 0; c < STEPS; ++c) drop_bad<E>(a[db][c]);
#pragma unroll 1
                for (int k = 0; k < 32; ++k) {
                    const int r = row0 + k, at = (d0 * 32 + lane) * E::SIZE;       // a lane reads one of the 64 columns of row k
                    const unsigned char* e = t + r * T::ROWB + (((at >> 4) ^ T::key(r)) << 4) + (at & 15);
                    const uint32_t v = E::SIZE == 2 ? (uint32_t)*reinterpret_cast<const uint16_t*>(e) << 16 : *reinterpret_cast<const uint32_t*>(e);
                    uint64_t m = __ballot((v & 0x7F800000u) == 0x7F800000u);
                    const bool mine = sees(k);
                    while (m) {
                        const int col = __ffsll((unsigned long long)m) - 1, i_at = (col >> 5) * 16 + ((col >> 3) & 3) * 4 + (col & 3);
                        m &= m - 1;
                        float put = __builtin_bit_cast(float, __builtin_amdgcn_readlane((int)v, col));
                        put = SIGNED ? NAN : put;
                        put = mine && (lane >> 5) == ((col >> 2) & 1) ? put : 0.f;
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (i == i_at) acc[d0 + (i >> 4)][i & 15] += put;
                    }
                }
            }
        }
#pragma unroll
        for (int c = 0; c < STEPS; ++c)
#pragma unroll
            for (int db = 0; db < 2; ++db) acc[d0 + db] = E::mma(a[db][c], wf[c], acc[d0 + db]);
    }
}

// ---- sequences
constexpr int kTilesFree = 4;       // tiles of a sequence whose keys are dealt out without regard to the others'
struct Seq {
    int q0, lq, k0, lk, tile;
    int chunk, chunks, first;       // of keys: this one's, how many the sequence has, the number of the tile's first item
};
__device__ __forceinline__ int clamp_start(int v, int total) { return min(max(v, 0), total); }

// Chunks of a sequence's keys: of `each` keys (a multiple of 256), but no more than the sequence's part of the workgroups that there are (Deal::items) gives each
// of its tiles; then they are longer.
__device__ __forceinline__ int chunks_of(int lk, int tiles, int each)
{
    const int n = max(1, (lk + each - 1) / each);
    return tiles > kTilesFree ? min(n, 1 + lk / (each / kTilesFree) / tiles) : n;       // (up to kTilesFree tiles the part is never less than n)
}
__device__ __forceinline__ int chunk_keys(int lk, int chunks, int each) { return chunks * each >= lk ? each : ((lk + chunks - 1) / chunks + 255) / 256 * 256; }

// Workgroups: key heads first, so that the tiles of a sequence, whose cost falls from the first to the last, end a launch with the cheapest, and a key head's
// workgroups share an XCD where there are 8 key heads or a part of 8.
// What is found is the same in all lanes; the compiler is told, so that what is reckoned from it is scalar work.
__device__ __forceinline__ Seq same_in_all(const Seq& s)
{
    const auto u = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    return Seq{u(s.q0), u(s.lq), u(s.k0), u(s.lk), u(s.tile), u(s.chunk), u(s.chunks), u(s.first)};
}

// Item w of a list: for every sequence its tiles (`tile` rows each, `per` rows per token, of the queries or of the keys), and for every tile with
// keys_each > 0 its sequence's chunks of about that many keys.  BY_TILE: w counts tiles, chunk is 0.  False behind the last.  Starts outside the arrays are
// brought inside, a sequence that would end before it starts is empty.  A workgroup looks through 64 sequences for each of its wavefronts at a time:
// one load and a prefix sum, about a microsecond in which nothing else happens.
template <int NW, bool KEYS, bool BY_TILE = false>
__device__ __forceinline__ bool find_tile(const PackedAttn& p, int w, int per, int tile, int keys_each, Seq& s)
{
    __shared__ int wave_sum[NW][2], found[8];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int base = 0, base_items = 0;
    for (int b0 = 0; b0 < p.n_seqs; b0 += 64 * NW) {
        const bool one = p.n_seqs - b0 <= 64;               // every wavefront looks at the same sequences: nothing to exchange
        const int mine_b = b0 + (one ? lane : (int)threadIdx.x), b = min(mine_b, p.n_seqs - 1);
        const int q0 = clamp_start(p.q_start[b], p.total_q), lq = max(clamp_start(p.q_start[b + 1], p.total_q) - q0, 0);
        const int k0 = clamp_start(p.k_start[b], p.total_k), lk = max(clamp_start(p.k_start[b + 1], p.total_k) - k0, 0);
        const int tiles = mine_b < p.n_seqs ? (int)(((int64_t)(KEYS ? lk : lq) * per + tile - 1) / tile) : 0;
        const int chunks = keys_each > 0 ? chunks_of(lk, tiles, keys_each) : 1;
        if (!BY_TILE && keys_each == 0 && p.n_seqs > 1 && p.n_seqs <= 64) {
            // few sequences: the tiles that are followed by most others of their sequence first, in all sequences (the longest sequence last in the
            // list would otherwise end the launch with its longest tiles).  behind(d): tiles followed by d others or more.
            const auto behind = [&](int d) { return wave_sum_int(max(tiles - d, 0)); };
            if (w >= behind(0)) return false;
            int lo = 1, hi = (int)wave_max((float)tiles);           // (less than 2^24 tiles: rows are numbered with 29 bits, 32 a tile)
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (behind(mid) <= w) hi = mid;
                else lo = mid + 1;
            }
            const int nth = w - behind(lo);
            const uint64_t have = __ballot(tiles >= lo);
            const int l = __ffsll((unsigned long long)__ballot(tiles >= lo && __popcll(have & ((1ull << lane) - 1)) == nth)) - 1;
            s.chunk = s.first = 0;
            s.chunks = 1;
            s.tile = __shfl(tiles, l) - lo;
            s.q0 = __shfl(q0, l);
            s.lq = __shfl(lq, l);
            s.k0 = __shfl(k0, l);
            s.lk = __shfl(lk, l);
            return true;
        }
        const int n = BY_TILE ? tiles : tiles * chunks;
        int sum = n, items = tiles * chunks;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int up = __shfl_up(sum, o), up_items = BY_TILE ? __shfl_up(items, o) : 0;
            if (lane >= o) {
                sum += up;
                items += up_items;
            }
        }
        int all = __shfl(sum, 63), all_items = __shfl(items, 63);
        if (!one) {
            if (lane == 63) {
                wave_sum[wave][0] = sum;
                wave_sum[wave][1] = items;
            }
            __syncthreads();
            int before = 0, before_items = 0;
            all = all_items = 0;
#pragma unroll
            for (int k = 0; k < NW; ++k) {
                before += k < wave ? wave_sum[k][0] : 0;
                before_items += k < wave ? wave_sum[k][1] : 0;
                all += wave_sum[k][0];
                all_items += wave_sum[k][1];
            }
            sum += before;
            items += before_items;
        }
        if (w < base + all) {
            int mine, first_items;
            if (one) {
                const int l = __ffsll((unsigned long long)__ballot(base + sum > w)) - 1;
                mine = w - (base + __shfl(sum, l) - __shfl(n, l));
                s.chunks = __shfl(chunks, l);
                first_items = base_items + __shfl(items, l) - __shfl(tiles, l) * s.chunks;
                s.q0 = __shfl(q0, l);
                s.lq = __shfl(lq, l);
                s.k0 = __shfl(k0, l);
                s.lk = __shfl(lk, l);
            } else {
                if (w >= base + sum - n && w < base + sum) {
                    const int put[7] = {w - (base + sum - n), chunks, base_items + items - tiles * chunks, q0, lq, k0, lk};
#pragma unroll
                    for (int i = 0; i < 7; ++i) found[i] = put[i];
                }
                __syncthreads();
                mine = found[0];
                s.chunks = found[1];
                first_items = found[2];
                s.q0 = found[3];
                s.lq = found[4];
                s.k0 = found[5];
                s.lk = found[6];
            }
            s.tile = BY_TILE ? mine : mine / s.chunks;
            s.chunk = BY_TILE ? 0 : mine - s.tile * s.chunks;
            s.first = BY_TILE ? first_items + s.tile * s.chunks : w - s.chunk;
            return true;
        }
        base += all;
        base_items += all_items;
        __syncthreads();
    }
    return false;
}

// A matrix whose tiles of ROWS rows go into LDS, 16 bytes a lane straight from memory.  Row r is row r / group of its head r % group.  A lane's place inside
// a tile is an offset that stays the same from tile to tile (32 bits, from the tile's first row on: where a tile is whole tokens and spans less than
// 4 GB), so a whole tile costs scalar instructions only; the last tile, beyond whose rows copies of the last one stand in, is reckoned out.
// Columns beyond a width that is not DP (!FULL) are zeros, which the other operand's zeros meet (copies of real columns would not do: 0 times an infinity is
// NaN): the kernel writes them once (clear_columns), and the lanes of a load that would fetch them are off.  A load spans whole rows, so some are always on.
template <typename E, int DP, int ROWS, int NW, bool FULL>
struct Rows {
    using T = Tile<E, DP>;
    static constexpr int N = ROWS / T::RPI / NW;
    static_assert(N * NW * T::RPI == ROWS, "rows must split evenly over wavefront loads");
    const char* base;
    int64_t row_bytes, head_bytes, step;
    uint32_t off[N];
    uint64_t on[N];             // the lanes of a load (!FULL)
    int group, d;
    bool even;

    __device__ __forceinline__ uint32_t column(int row) const
    {
        const int lane = threadIdx.x & 63;
        return ((lane % T::CH) ^ T::key(row)) * 16;
    }
    __device__ __forceinline__ bool held(uint32_t column) const { return FULL || (int)column < d * E::SIZE; }
    __device__ __forceinline__ void init(const typename E::elem* from, int64_t row, int64_t head, int group_, int d_)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        base = reinterpret_cast<const char*>(from);
        row_bytes = row * E::SIZE;
        head_bytes = head * E::SIZE;
        group = group_;
        d = d_;
        step = ROWS / group * row_bytes;
        even = ROWS % group == 0 && step + group * head_bytes < (1ll << 32);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = (wave + i * NW) * T::RPI + lane / T::CH, tok = r / group;
            off[i] = (uint32_t)(tok * row_bytes + (r - tok * group) * head_bytes) + column(r);
            if constexpr (!FULL) on[i] = __ballot(held(column(r)));
        }
    }
    __device__ __forceinline__ void fetch(int tile, int last, uint32_t to) const
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        if (even && (tile + 1) * ROWS - 1 <= last) {
            const char* at = uniform(base + tile * step);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if constexpr (FULL) load_to_lds(at, off[i], to + (wave + i * NW) * 1024);
                else load_to_lds_of(on[i], at, off[i], to + (wave + i * NW) * 1024);
            }
            return;
        }
        const int lane = threadIdx.x & 63;
#pragma unroll 1
        for (int i = 0; i < N; ++i) {
            const int in = (wave + i * NW) * T::RPI + lane / T::CH, r = min(tile * ROWS + in, last), tok = r / group;
            const char* at = base + tok * row_bytes + (r - tok * group) * head_bytes + column(in);
            if constexpr (FULL) load_to_lds(at, to + (wave + i * NW) * 1024);
            else load_to_lds_of(__ballot(held(column(in))), at, to + (wave + i * NW) * 1024);
        }
    }
};

// The columns beyond the width `d` of `rows` tile rows from t on (the first of a tile) become zeros.  A barrier stands between this and their first use.
template <typename E, int DP, int NT, bool FULL>
__device__ __forceinline__ void clear_columns(unsigned char* t, int rows, int d)
{
    using T = Tile<E, DP>;
    if constexpr (!FULL)
        for (int r = threadIdx.x; r < rows; r += NT)
            for (int c = d / E::EPC; c < T::CH; ++c) *reinterpret_cast<f32x4*>(t + r * T::ROWB + ((c ^ T::key(r)) << 4)) = f32x4{0.f, 0.f, 0.f, 0.f};
}

// The tiles that pass by go through a ring in LDS: one is used while up to STAGES - 1 are under way.  All loads of a loop are those of its ring, LPS of each
// wavefront per tile, so that a wait can leave the last tiles under way.
template <int STAGES, int LPS>
__device__ __forceinline__ void tile_landed(int behind)         // tiles behind this one that have been asked for
{
    static_assert(STAGES >= 2 && STAGES <= 4 && (STAGES - 2) * LPS < 64, "");
    if (STAGES >= 4 && behind >= 2) wait_loads<(STAGES >= 4 ? 2 : 0) * LPS>();
    else if (STAGES >= 3 && behind >= 1) wait_loads<(STAGES >= 3 ? 1 : 0) * LPS>();
    else wait_loads<0>();
    __syncthreads();
}

template <typename E, int DP>
__device__ __forceinline__ void load_row(typename E::frag (&f)[DP / E::KS], const typename E::elem* row, int d, int half)
{
#pragma unroll
    for (int ks = 0; ks < DP / E::KS; ++ks) {
        const int c = ks * E::KS + half * E::EPC;
#pragma unroll
        for (int j = 0; j < E::EPC; ++j) f[ks][j] = (typename E::elem)0.f;
        if (c < d) f[ks] = *reinterpret_cast<const typename E::frag*>(row + c);
    }
}

// Registers loaded from memory are used here: the compiler's wait for them stands here too, and not in the loop behind, where it would be one for the
// tiles under way.
template <typename F, int N>
__device__ __forceinline__ void loaded(const F (&f)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" ::"v"(f[i]));
}

template <typename E, int DP>
__device__ __forceinline__ void store_cols(const f32x16 (&acc)[DP / 32], float by, typename E::elem* row, int d, int half)
{
    typedef typename E::elem out4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int c = db * 32 + g * 8 + half * 4;
            if (c >= d) continue;
            out4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = (typename E::elem)(acc[db][g * 4 + j] * by);
            *reinterpret_cast<out4*>(row + c) = v;
        }
}

// wavefronts per SIMD that a kernel is compiled for: `narrow` for bfloat16 rows of up to 64 columns, 2 for wider ones and float32 ones of up to 64, 1 for the rest
template <typename E, int DP>
constexpr int waves_of(int narrow)
{
    return Tile<E, DP>::ROWB == 128 ? narrow : Tile<E, DP>::ROWB == 256 ? 2 : 1;
}

// RW x KW wavefronts: RW blocks of 32 rows, each with KW wavefronts that take UB blocks of 32 keys of a tile in turn and put their sums together at the
// end.  p.work: with keys_each > 0 a tile's keys are dealt out to workgroups as well, whose sums a second launch puts together.
// Keys and values pass through a ring of tiles in LDS (loads straight from memory, a tile or two ahead); q stays in registers.  Steps that paid, on 8192 tokens of D = 128: loads
// that the compiler does not wait for in front of every transposing read, two wavefronts per SIMD 1044 -> 672 us; the rare non-finite operands handled
// behind one branch 697 -> 607; key heads as the fastest index of the launch, so that an XCD's L2 keeps one head's keys 607 -> 578; deepest rows first 498 -> 478.
template <typename E, int DP, int RW, int KW, int UB, int STAGES>
struct Forward {
    using T = Tile<E, DP>;
    static constexpr int BM = RW * 32, TK = KW * UB * 32, NW = RW * KW, BYTES = TK * T::ROWB, LDS = STAGES * 2 * BYTES, LPS = 2 * BYTES / 1024 / NW;
    static constexpr int ROW = DP + 4;                      // floats of a partial row: sums, then reference and sum of the weights
    static_assert(LDS <= 160 * 1024 && (KW - 1) * RW * (DP / 2 + 2) * 64 * 4 <= LDS, "");
};

template <typename E, int DP, int RW, int KW, int UB, int STAGES, bool FULL>
__global__ __launch_bounds__(RW * KW * 64, (waves_of<E, DP>(UB == 1 ? 3 : 2))) void packed_forward_kernel(PackedAttn p, int keys_each)
{
    using F = Forward<E, DP, RW, KW, UB, STAGES>;
    using T = Tile<E, DP>;
    typedef typename E::elem elem;
    constexpr int BM = F::BM, TK = F::TK, NW = F::NW, BYTES = F::BYTES;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];      // the ring of keys and values
    const uint32_t lds0 = lds_address(lds);
    const int group = p.group, item = __builtin_amdgcn_readfirstlane(blockIdx.x / p.kv_heads), kvh = blockIdx.x - item * p.kv_heads;
    Seq s;
    if (!find_tile<NW, false>(p, item, group, BM, keys_each, s)) return;
    s = same_in_all(s);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, half = lane >> 5;
    const int rw = wave / KW, kw = wave % KW;
    const int rows = s.lq * group, tiles = (rows + BM - 1) / BM;
    const int r0 = (tiles - 1 - s.tile) * BM;                                 // the rows that see most first
    const int shift = p.causal ? s.lk - s.lq : 0x40000000;                    // query i sees keys up to i + shift
    const auto limit_of = [&](int r) { return min(min(r, rows - 1) / group + shift, s.lk - 1); };
    const auto limit_all = [&](int r) { return __builtin_amdgcn_readfirstlane(limit_of(r)); };         // of a row that is the same in all lanes
    const int my_row = min(r0 + rw * 32 + l32, rows - 1);
    const int tok = my_row / group, head = kvh * group + my_row - tok * group;
    const int limit = limit_of(my_row), wave_min = limit_all(r0 + rw * 32), wave_max = limit_all(r0 + rw * 32 + 31);
    int n_keys = limit_all(r0 + BM - 1) + 1, t0 = 0;
    if (keys_each > 0) {
        const int each = chunk_keys(s.lk, s.chunks, keys_each);
        t0 = s.chunk * (each / TK);
        n_keys = min(n_keys, (s.chunk + 1) * each);
    }
    const int n_tiles = n_keys > 0 ? (n_keys + TK - 1) / TK : 0;

    const elem* K = static_cast<const elem*>(p.k) + (int64_t)s.k0 * p.k_row + kvh * p.k_head;
    const elem* V = static_cast<const elem*>(p.v) + (int64_t)s.k0 * p.v_row + kvh * p.v_head;
    Rows<E, DP, TK, NW, FULL> rows_k, rows_v;
    rows_k.init(K, p.k_row, 0, 1, p.d);
    rows_v.init(V, p.v_row, 0, 1, p.d);
    const auto fetch = [&](int kt, int stage_at) {
        const uint32_t to = lds0 + stage_at * 2 * BYTES;
        rows_k.fetch(kt, s.lk - 1, to);
        rows_v.fetch(kt, s.lk - 1, to + BYTES);
    };
    clear_columns<E, DP, NW * 64, FULL>(lds, STAGES * 2 * TK, p.d);
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i)
        if (t0 + i < n_tiles) fetch(t0 + i, i);
    typename E::frag qf[DP / E::KS];
    load_row<E, DP>(qf, static_cast<const elem*>(p.q) + (int64_t)(s.q0 + tok) * p.q_row + head * p.q_head, p.d, half);

    f32x16 acc[DP / 32];
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[db][i] = 0.f;
    const float c = p.scale * kLog2e;
    float ref = -INFINITY, sum = 0.f;       // weights are exp2(c (score - ref))

    loaded(qf);
    int at = 0;
    for (int kt = t0; kt < n_tiles; ++kt, at = at + 1 == STAGES ? 0 : at + 1) {
        tile_landed<STAGES, F::LPS>(n_tiles - 1 - kt);
        if (kt + STAGES - 1 < n_tiles) fetch(kt + STAGES - 1, at == 0 ? STAGES - 1 : at - 1);
        const unsigned char* tk = lds + at * 2 * BYTES + kw * UB * 32 * T::ROWB;
        const unsigned char* tv = tk + BYTES;
        const int key0 = kt * TK + kw * UB * 32;
        if (key0 > wave_max) continue;
        f32x16 sc[UB];
#pragma unroll
        for (int u = 0; u < UB; ++u) {
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[u][i] = 0.f;
#pragma unroll
            for (int ks = 0; ks < DP / E::KS; ++ks) sc[u] = E::mma(T::row_frag(tk, u * 32 + l32, ks, half), qf[ks], sc[u]);
        }
        const bool cut = key0 + UB * 32 - 1 > wave_min;
        if (cut) {
#pragma unroll
            for (int u = 0; u < UB; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[u][i] = key0 + u * 32 + 8 * (i >> 2) + 4 * half + (i & 3) <= limit ? sc[u][i] : -INFINITY;
        }
        float top = sc[0][0];
#pragma unroll
        for (int u = 0; u < UB; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[u][i]);
        top = lane_pair_max<32>(top);
        // the reference follows the maximum only when that has grown by 2^8: the weights' sums stay far from overflow and the accumulators are
        // rescaled a few times per row instead of once per tile
        if (__any((top - ref) * c > 8.f || ref == -INFINITY)) {
            const float to = fmaxf(ref, top);
            const float by = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((ref - to) * c);
            ref = to;
            sum *= by;
#pragma unroll
            for (int db = 0; db < DP / 32; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[db][i] *= by;
        }
        const float rc = ref == -INFINITY ? 0.f : ref * c;
#pragma unroll
        for (int u = 0; u < UB; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                sc[u][i] = __builtin_amdgcn_exp2f(fmaf(sc[u][i], c, -rc));
                sum += sc[u][i];
            }
#pragma unroll
        for (int u = 0; u < UB; ++u) add_product<E, DP, false>(acc, tv, u * 32, sc[u], cut, [&](int k) { return key0 + u * 32 + k <= limit; }, lane);
    }
    sum = lane_pair_sum<32>(sum);
    if constexpr (KW > 1) {
        // the wavefronts of a block of rows, in order
        float* const other = reinterpret_cast<float*>(lds) + rw * (KW - 1) * (DP / 2 + 2) * 64 + lane;
        __syncthreads();
        if (kw > 0) {
            float* at = other + (kw - 1) * (DP / 2 + 2) * 64;
#pragma unroll
            for (int db = 0; db < DP / 32; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) at[(db * 16 + i) * 64] = acc[db][i];
            at[DP / 2 * 64] = ref;
            at[(DP / 2 + 1) * 64] = sum;
        }
        __syncthreads();
        if (kw > 0) return;
#pragma unroll 1
        for (int o = 0; o < KW - 1; ++o) {
            const float* at = other + o * (DP / 2 + 2) * 64;
            const float ref_o = at[DP / 2 * 64], to = fmaxf(ref, ref_o), from = to == -INFINITY ? 0.f : to;
            const float by = __builtin_amdgcn_exp2f((ref - from) * c), by_o = __builtin_amdgcn_exp2f((ref_o - from) * c);
            ref = to;
            sum = fmaf(at[(DP / 2 + 1) * 64], by_o, sum * by);
#pragma unroll
            for (int db = 0; db < DP / 32; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[db][i] = fmaf(at[(db * 16 + i) * 64], by_o, acc[db][i] * by);
        }
    }
    if (r0 + rw * 32 + l32 >= rows) return;
    if (s.chunks > 1) {
        float* at = static_cast<float*>(p.work) + (((int64_t)(s.first + s.chunk) * p.kv_heads + kvh) * BM + rw * 32 + l32) * F::ROW;
#pragma unroll
        for (int db = 0; db < DP / 32; ++db)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f32x4 v;
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = acc[db][g * 4 + j];
                *reinterpret_cast<f32x4*>(at + db * 32 + g * 8 + half * 4) = v;
            }
        if (half == 0) {
            at[DP] = ref;
            at[DP + 1] = sum;
        }
        return;
    }
    if (limit < 0) {
#pragma unroll
        for (int db = 0; db < DP / 32; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[db][i] = 0.f;
    }
    store_cols<E, DP>(acc, limit < 0 ? 0.f : 1.f / sum, static_cast<elem*>(p.out) + (int64_t)(s.q0 + tok) * p.o_row + head * p.o_head, p.d, half);
    if (p.lse && half == 0) p.lse[(int64_t)head * p.total_q + s.q0 + tok] = limit < 0 ? -INFINITY : fmaf(ref, p.scale, __builtin_amdgcn_logf(sum) * kLn2);
}

// the chunks of a tile's keys put together, one workgroup per 4 rows of a tile and key head: 64 lanes a row
template <typename E, int DP, int BM>
__global__ __launch_bounds__(256) void packed_join_kernel(PackedAttn p, int keys_each, int items)
{
    typedef typename E::elem elem;
    constexpr int ROW = DP + 4, COLS = DP / 64;
    const int group = p.group, item = __builtin_amdgcn_readfirstlane(blockIdx.x / p.kv_heads), kvh = blockIdx.x - item * p.kv_heads;
    Seq s;
    if (!find_tile<4, false, true>(p, item, group, BM, keys_each, s) || s.chunks == 1) return;
    if (s.first < 0 || (int64_t)s.first + s.chunks > items) return;        // starts that fall name more items than there are
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int rows = s.lq * group, tiles = (rows + BM - 1) / BM, r = blockIdx.y * 4 + wave, row = (tiles - 1 - s.tile) * BM + r;
    if (row >= rows) return;
    const int tok = row / group, head = kvh * group + row - tok * group;
    const int limit = min(tok + (p.causal ? s.lk - s.lq : 0x40000000), s.lk - 1);
    const float c = p.scale * kLog2e;
    const float* at = static_cast<const float*>(p.work) + (((int64_t)s.first * p.kv_heads + kvh) * BM + r) * ROW;
    const int64_t step = (int64_t)p.kv_heads * BM * ROW;
    float ref = -INFINITY;
    for (int k = lane; k < s.chunks; k += 64) ref = fmaxf(ref, at[k * step + DP]);
    ref = wave_max(ref);
    const float from = ref == -INFINITY ? 0.f : ref;
    float sum = 0.f, v[COLS];
#pragma unroll
    for (int i = 0; i < COLS; ++i) v[i] = 0.f;
    for (int k0 = 0; k0 < s.chunks; k0 += 8) {
        float x[8][COLS], ro[8], so[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float* from_k = at + min(k0 + k, s.chunks - 1) * step;
            ro[k] = from_k[DP];
            so[k] = from_k[DP + 1];
#pragma unroll
            for (int i = 0; i < COLS; ++i) x[k][i] = from_k[lane * COLS + i];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float by = k0 + k < s.chunks ? __builtin_amdgcn_exp2f((ro[k] - from) * c) : 0.f;
            if (k0 + k >= s.chunks) continue;
            sum = fmaf(so[k], by, sum);
#pragma unroll
            for (int i = 0; i < COLS; ++i) v[i] = fmaf(x[k][i], by, v[i]);
        }
    }
    const float by = limit < 0 ? 0.f : 1.f / sum;
    elem* out = static_cast<elem*>(p.out) + (int64_t)(s.q0 + tok) * p.o_row + head * p.o_head;
#pragma unroll
    for (int i = 0; i < COLS; ++i)
        if (lane * COLS + i < p.d) out[lane * COLS + i] = (elem)(limit < 0 ? 0.f : v[i] * by);
    if (p.lse && lane == 0) p.lse[(int64_t)head * p.total_q + s.q0 + tok] = limit < 0 ? -INFINITY : fmaf(ref, p.scale, __builtin_amdgcn_logf(sum) * kLn2);
}

// What the gradient needs of a row, in the order of the packed rows (key head, query, head of the group): lse log2e and -delta.
// delta = dctx . ctx = sum_j P_ij (dctx_i . v_j).  ctx has been rounded, which delta hardly notices where a row averages many values, but rows of few keys
// have the largest gradients: in bfloat16, tiles whose rows see at most kFewKeys keys take the second form, from the weights themselves.  Against float64, dq
// and dk of sequences of a few tens of tokens are off by 0.0024 (2-norm, relative) instead of 0.0032, of 300 to 4001 tokens 0.0024 instead of 0.0025; what
// is left is the rounding of dS and of the results.
constexpr int kFewKeys = 128;
template <typename E, int DP, bool FULL>
__global__ __launch_bounds__(256) void packed_stat_kernel(PackedAttn p, float* stat)
{
    using T = Tile<E, DP>;
    typedef typename E::elem elem;
    constexpr int NW = 4, BM = NW * 32, TK = 32, BYTES = TK * T::ROWB, LPS = 2 * BYTES / 1024 / NW;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[4 * BYTES];
    const uint32_t lds0 = lds_address(lds);
    const int group = p.group, item = __builtin_amdgcn_readfirstlane(blockIdx.x / p.kv_heads), kvh = blockIdx.x - item * p.kv_heads;
    Seq s;
    if (!find_tile<NW, false>(p, item, group, BM, 0, s)) return;
    s = same_in_all(s);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, half = lane >> 5;
    const int rows = s.lq * group, tiles = (rows + BM - 1) / BM, r0 = (tiles - 1 - s.tile) * BM;
    const int shift = p.causal ? s.lk - s.lq : 0x40000000;
    const auto limit_of = [&](int r) { return min(min(r, rows - 1) / group + shift, s.lk - 1); };
    const auto limit_all = [&](int r) { return __builtin_amdgcn_readfirstlane(limit_of(r)); };
    const int my_row = min(r0 + wave * 32 + l32, rows - 1);
    const int tok = my_row / group, head = kvh * group + my_row - tok * group;
    const int limit = limit_of(my_row), n_keys = limit_all(r0 + BM - 1) + 1;

    typename E::frag gf[DP / E::KS], of[DP / E::KS];
    load_row<E, DP>(gf, static_cast<const elem*>(p.dctx) + (int64_t)(s.q0 + tok) * p.g_row + head * p.g_head, p.d, half);
    const float lse = p.lse_in[(int64_t)head * p.total_q + s.q0 + tok] * kLog2e;
    float sum = 0.f;
    if (E::SIZE == 4 || n_keys > kFewKeys) {
        load_row<E, DP>(of, static_cast<const elem*>(p.ctx) + (int64_t)(s.q0 + tok) * p.o_row + head * p.o_head, p.d, half);
#pragma unroll
        for (int ks = 0; ks < DP / E::KS; ++ks)
#pragma unroll
            for (int j = 0; j < E::EPC; ++j) sum = fmaf((float)gf[ks][j], (float)of[ks][j], sum);
    } else {
        load_row<E, DP>(of, static_cast<const elem*>(p.q) + (int64_t)(s.q0 + tok) * p.q_row + head * p.q_head, p.d, half);
        loaded(gf);
        loaded(of);
        asm volatile("" ::"v"(lse));
        const float c = p.scale * kLog2e;
        Rows<E, DP, TK, NW, FULL> rows_k, rows_v;
        rows_k.init(static_cast<const elem*>(p.k) + (int64_t)s.k0 * p.k_row + kvh * p.k_head, p.k_row, 0, 1, p.d);
        rows_v.init(static_cast<const elem*>(p.v) + (int64_t)s.k0 * p.v_row + kvh * p.v_head, p.v_row, 0, 1, p.d);
        const auto fetch = [&](int kt) {
            rows_k.fetch(kt, s.lk - 1, lds0 + (kt & 1) * 2 * BYTES);
            rows_v.fetch(kt, s.lk - 1, lds0 + (kt & 1) * 2 * BYTES + BYTES);
        };
        const int n_tiles = n_keys > 0 ? (n_keys + TK - 1) / TK : 0;
        clear_columns<E, DP, NW * 64, FULL>(lds, 4 * TK, p.d);
        if (n_tiles > 0) fetch(0);
        for (int kt = 0; kt < n_tiles; ++kt) {
            tile_landed<2, LPS>(0);
            if (kt + 1 < n_tiles) fetch(kt + 1);
            const unsigned char* tk = lds + (kt & 1) * 2 * BYTES;
            const unsigned char* tv = tk + BYTES;
            f32x16 sc, dp;
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[i] = dp[i] = 0.f;
#pragma unroll
            for (int ks = 0; ks < DP / E::KS; ++ks) {
                sc = E::mma(T::row_frag(tk, l32, ks, half), of[ks], sc);
                dp = E::mma(T::row_frag(tv, l32, ks, half), gf[ks], dp);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float w = __builtin_amdgcn_exp2f(fmaf(sc[i], c, -lse)) * dp[i];
                sum += kt * TK + 8 * (i >> 2) + 4 * half + (i & 3) <= limit ? w : 0.f;
            }
        }
    }
    sum = lane_pair_sum<32>(sum);
    if (half != 0 || r0 + wave * 32 + l32 >= rows) return;
    float* to = stat + ((int64_t)kvh * p.total_q + s.q0) * group + my_row;
    to[0] = lse;
    to[(int64_t)p.total_q * p.heads] = -sum;
}

// dq: rows fixed, keys pass by.  RW blocks of 32 rows, each with KW wavefronts that take a block of 32 keys of a tile each.  Three products (S, dP, dq) for one
// exp: documents of 300..4001 tokens, 16 heads on 4 of D = 64, 147 us under the profiler; vector and matrix instructions.
// Rounding: in bfloat16 dS is rounded to the operands' type before the last product (half a step, 2^-9 .. 2^-8 of each term), as P is in the forward pass.
template <typename E, int DP, int RW, int KW, int STAGES>
struct RowGrad {
    using T = Tile<E, DP>;
    static constexpr int BM = RW * 32, TK = KW * 32, NW = RW * KW, BYTES = TK * T::ROWB, LDS = STAGES * 2 * BYTES, LPS = 2 * BYTES / 1024 / NW;
    static_assert(LDS <= 160 * 1024 && (KW - 1) * RW * DP / 2 * 64 * 4 <= LDS, "");
};

template <typename E, int DP, int RW, int KW, int STAGES, bool FULL>
__global__ __launch_bounds__(RW * KW * 64, (waves_of<E, DP>(3))) void packed_dq_kernel(PackedAttn p, const float* stat)
{
    using R = RowGrad<E, DP, RW, KW, STAGES>;
    using T = Tile<E, DP>;
    typedef typename E::elem elem;
    constexpr int BM = R::BM, TK = R::TK, NW = R::NW, BYTES = R::BYTES;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const uint32_t lds0 = lds_address(lds);
    const int group = p.group, item = __builtin_amdgcn_readfirstlane(blockIdx.x / p.kv_heads), kvh = blockIdx.x - item * p.kv_heads;
    Seq s;
    if (!find_tile<NW, false>(p, item, group, BM, 0, s)) return;
    s = same_in_all(s);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, half = lane >> 5;
    const int rw = wave / KW, kw = wave % KW;
    const int rows = s.lq * group, tiles = (rows + BM - 1) / BM;
    const int r0 = (tiles - 1 - s.tile) * BM;
    const int shift = p.causal ? s.lk - s.lq : 0x40000000;
    const auto limit_of = [&](int r) { return min(min(r, rows - 1) / group + shift, s.lk - 1); };
    const auto limit_all = [&](int r) { return __builtin_amdgcn_readfirstlane(limit_of(r)); };         // of a row that is the same in all lanes
    const int my_row = min(r0 + rw * 32 + l32, rows - 1);
    const int tok = my_row / group, head = kvh * group + my_row - tok * group;
    const int limit = limit_of(my_row), wave_min = limit_all(r0 + rw * 32), wave_max = limit_all(r0 + rw * 32 + 31);
    const int n_keys = limit_all(r0 + BM - 1) + 1, n_tiles = n_keys > 0 ? (n_keys + TK - 1) / TK : 0;

    const elem* K = static_cast<const elem*>(p.k) + (int64_t)s.k0 * p.k_row + kvh * p.k_head;
    const elem* V = static_cast<const elem*>(p.v) + (int64_t)s.k0 * p.v_row + kvh * p.v_head;
    Rows<E, DP, TK, NW, FULL> rows_k, rows_v;
    rows_k.init(K, p.k_row, 0, 1, p.d);
    rows_v.init(V, p.v_row, 0, 1, p.d);
    const auto fetch = [&](int kt, int stage_at) {
        const uint32_t to = lds0 + stage_at * 2 * BYTES;
        rows_k.fetch(kt, s.lk - 1, to);
        rows_v.fetch(kt, s.lk - 1, to + BYTES);
    };
    clear_columns<E, DP, NW * 64, FULL>(lds, STAGES * 2 * TK, p.d);
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i)
        if (i < n_tiles) fetch(i, i);
    typename E::frag qf[DP / E::KS], gf[DP / E::KS];
    load_row<E, DP>(qf, static_cast<const elem*>(p.q) + (int64_t)(s.q0 + tok) * p.q_row + head * p.q_head, p.d, half);
    load_row<E, DP>(gf, static_cast<const elem*>(p.dctx) + (int64_t)(s.q0 + tok) * p.g_row + head * p.g_head, p.d, half);
    const float c = p.scale * kLog2e;
    const float* my_stat = stat + ((int64_t)kvh * p.total_q + s.q0) * group + my_row;
    const float lse = my_stat[0], less = my_stat[(int64_t)p.total_q * p.heads];

    f32x16 acc[DP / 32];
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[db][i] = 0.f;
    loaded(qf);
    loaded(gf);
    asm volatile("" ::"v"(lse), "v"(less));
    int at = 0;
    for (int kt = 0; kt < n_tiles; ++kt, at = at + 1 == STAGES ? 0 : at + 1) {
        tile_landed<STAGES, R::LPS>(n_tiles - 1 - kt);
        if (kt + STAGES - 1 < n_tiles) fetch(kt + STAGES - 1, at == 0 ? STAGES - 1 : at - 1);
        const unsigned char* tk = lds + at * 2 * BYTES;
        const unsigned char* tv = tk + BYTES;
        const int key0 = kt * TK + kw * 32;
        if (key0 > wave_max) continue;
        f32x16 sc, dp;
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = dp[i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < DP / E::KS; ++ks) {
            sc = E::mma(T::row_frag(tk, kw * 32 + l32, ks, half), qf[ks], sc);
            dp = E::mma(T::row_frag(tv, kw * 32 + l32, ks, half), gf[ks], dp);
        }
        const bool cut = key0 + 31 > wave_min;
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = __builtin_amdgcn_exp2f(fmaf(sc[i], c, -lse)) * (dp[i] + less);
        if (cut) {
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[i] = key0 + 8 * (i >> 2) + 4 * half + (i & 3) <= limit ? sc[i] : 0.f;
        }
        add_product<E, DP, true>(acc, tk, kw * 32, sc, cut, [&](int k) { return key0 + k <= limit; }, lane);
    }
    if constexpr (KW > 1) {
        float* const other = reinterpret_cast<float*>(lds) + rw * (KW - 1) * DP / 2 * 64 + lane;
        __syncthreads();
        if (kw > 0) {
#pragma unroll
            for (int db = 0; db < DP / 32; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) other[((kw - 1) * DP / 2 + db * 16 + i) * 64] = acc[db][i];
        }
        __syncthreads();
        if (kw > 0) return;
#pragma unroll 1
        for (int o = 0; o < KW - 1; ++o)
#pragma unroll
            for (int db = 0; db < DP / 32; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[db][i] += other[(o * DP / 2 + db * 16 + i) * 64];
    }
    if (r0 + rw * 32 + l32 < rows)
        store_cols<E, DP>(acc, p.scale, static_cast<elem*>(p.dq) + (int64_t)(s.q0 + tok) * p.dq_row + head * p.dq_head, p.d, half);
}

// dk, dv: keys fixed, the rows of all heads of the group pass by.  KW blocks of 32 keys, each with RW wavefronts that take one block of 32 rows of a tile
// each and put their sums together at the end.  Four products (S, dP, dv, dk): the documents above 220 us.  For D = 64 one block of keys with four wavefronts of rows
// (each with a quarter of the rows and all sums of its keys in registers) instead of two by two: whole gradient and forward pass 566 -> 519 us.
// Rounding: P and dS to the operands' type, as above; the sums over the heads of a group stay in float32.
template <typename E, int DP, int KW, int RW, int STAGES>
struct KeyGrad {
    using T = Tile<E, DP>;
    // a stage: rows of q, rows of dctx, 256 bytes of every wavefront's: lse and delta of 64 rows, of the next 64 ..
    static constexpr int NW = KW * RW, BN = KW * 32, TQ = RW * 32, BYTES = TQ * T::ROWB, STAGE = 2 * BYTES + NW * 256, LPS = 2 * BYTES / 1024 / NW + 1;
    static constexpr int LDS = std::max(STAGES * STAGE, KW * (RW - 1) * DP * 64 * 4);
    static_assert(LDS <= 160 * 1024 && TQ <= NW * 32, "");
};

template <typename E, int DP, int KW, int RW, int STAGES, bool FULL>
__global__ __launch_bounds__(KW * RW * 64, (Tile<E, DP>::ROWB == 128 ? 2 : 1)) void packed_dkv_kernel(PackedAttn p, const float* stat)
{
    using G = KeyGrad<E, DP, KW, RW, STAGES>;
    using T = Tile<E, DP>;
    typedef typename E::elem elem;
    constexpr int BN = G::BN, TQ = G::TQ, NW = G::NW, BYTES = G::BYTES;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    const uint32_t lds0 = lds_address(lds);
    const int group = p.group, item = __builtin_amdgcn_readfirstlane(blockIdx.x / p.kv_heads), kvh = blockIdx.x - item * p.kv_heads;
    Seq s;
    if (!find_tile<NW, true>(p, item, 1, BN, 0, s)) return;
    s = same_in_all(s);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, half = lane >> 5;
    const int kw = wave / RW, rw = wave % RW;
    const int rows = s.lq * group, n0 = s.tile * BN;
    const int shift = p.causal ? s.lk - s.lq : 0x40000000;
    const int my_key = n0 + kw * 32 + l32, key = min(my_key, s.lk - 1);
    const int wave_last = min(n0 + kw * 32 + 31, s.lk - 1), wave_first = n0 + kw * 32;
    // the first rows that see the wavefront's first key, all its keys, the lane's key
    const auto first_of = [&](int k) { return p.causal ? min(max(k - shift, 0), s.lq) * group : 0; };
    const int row_first = first_of(wave_first), row_all = first_of(wave_last), my_first = first_of(key);
    const int rt0 = first_of(n0) / TQ, n_tiles = (rows + TQ - 1) / TQ;

    typename E::frag kf[DP / E::KS], vf[DP / E::KS];
    load_row<E, DP>(kf, static_cast<const elem*>(p.k) + (int64_t)(s.k0 + key) * p.k_row + kvh * p.k_head, p.d, half);
    load_row<E, DP>(vf, static_cast<const elem*>(p.v) + (int64_t)(s.k0 + key) * p.v_row + kvh * p.v_head, p.d, half);
    const elem* Q = static_cast<const elem*>(p.q) + (int64_t)s.q0 * p.q_row + (int64_t)kvh * group * p.q_head;
    const elem* O = static_cast<const elem*>(p.dctx) + (int64_t)s.q0 * p.g_row + (int64_t)kvh * group * p.g_head;
    const float c = p.scale * kLog2e;

    f32x16 ak[DP / 32], av[DP / 32];
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) ak[db][i] = av[db][i] = 0.f;

    // wavefronts 0, 2 .. fetch lse, 1, 3 .. delta
    const float* my_stat = stat + ((int64_t)kvh * p.total_q + s.q0) * group + (wave & 1) * (int64_t)p.total_q * p.heads;
    Rows<E, DP, TQ, NW, FULL> rows_q, rows_g;
    rows_q.init(Q, p.q_row, p.q_head, group, p.d);
    rows_g.init(O, p.g_row, p.g_head, group, p.d);
    const auto fetch = [&](int rt, int stage_at) {
        const uint32_t to = lds0 + stage_at * G::STAGE;
        rows_q.fetch(rt, rows - 1, to);
        rows_g.fetch(rt, rows - 1, to + BYTES);
        load_to_lds_4(my_stat + min(rt * TQ + (wave >> 1) * 64 + lane, rows - 1), to + 2 * BYTES + wave * 256);
    };
#pragma unroll
    for (int i = 0; i < STAGES; ++i) clear_columns<E, DP, NW * 64, FULL>(lds + i * G::STAGE, 2 * TQ, p.d);
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i)
        if (rt0 + i < n_tiles) fetch(rt0 + i, i);
    loaded(kf);
    loaded(vf);
    int at = 0;
    for (int rt = rt0; rt < n_tiles; ++rt, at = at + 1 == STAGES ? 0 : at + 1) {
        tile_landed<STAGES, G::LPS>(n_tiles - 1 - rt);
        if (rt + STAGES - 1 < n_tiles) fetch(rt + STAGES - 1, at == 0 ? STAGES - 1 : at - 1);
        const unsigned char* tq = lds + at * G::STAGE;
        const unsigned char* tg = tq + BYTES;
        const float* in_lse = reinterpret_cast<const float*>(tg + BYTES) + (rw >> 1) * 128 + (rw & 1) * 32;
        const float* in_delta = in_lse + 64;      // (-delta)
        const int b0 = rt * TQ + rw * 32;
        if (b0 < rows && b0 + 31 >= row_first) {
            // dctx v^T is added to -delta, whose rows are the accumulators' as they lie in LDS
            f32x16 sc, dp;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 less = *reinterpret_cast<const f32x4*>(in_delta + 8 * g + 4 * half);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    sc[4 * g + j] = 0.f;
                    dp[4 * g + j] = less[j];
                }
            }
#pragma unroll
            for (int ks = 0; ks < DP / E::KS; ++ks) {
                sc = E::mma(T::row_frag(tq, rw * 32 + l32, ks, half), kf[ks], sc);
                dp = E::mma(T::row_frag(tg, rw * 32 + l32, ks, half), vf[ks], dp);
            }
            const bool cut = b0 < row_all || b0 + 32 > rows;
            const auto sees = [&](int k) { return b0 + k >= my_first && b0 + k < rows; };
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 l = *reinterpret_cast<const f32x4*>(in_lse + 8 * g + 4 * half);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int i = 4 * g + j;
                    sc[i] = __builtin_amdgcn_exp2f(fmaf(sc[i], c, -l[j]));
                    dp[i] = sc[i] * dp[i];
                }
            }
            if (cut) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const bool see = sees(8 * (i >> 2) + 4 * half + (i & 3));
                    sc[i] = see ? sc[i] : 0.f;
                    dp[i] = see ? dp[i] : 0.f;
                }
            }
            add_product<E, DP, false>(av, tg, rw * 32, sc, cut, sees, lane);
            add_product<E, DP, true>(ak, tq, rw * 32, dp, cut, sees, lane);
        }
    }
    if constexpr (RW > 1) {
        float* const other = reinterpret_cast<float*>(lds) + kw * (RW - 1) * DP * 64 + lane;
        __syncthreads();
        if (rw > 0) {
            float* to = other + (rw - 1) * DP * 64;
#pragma unroll
            for (int db = 0; db < DP / 32; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    to[(db * 16 + i) * 64] = ak[db][i];
                    to[(DP / 2 + db * 16 + i) * 64] = av[db][i];
                }
        }
        __syncthreads();
        if (rw > 0) return;
#pragma unroll 1
        for (int o = 0; o < RW - 1; ++o) {
            const float* from = other + o * DP * 64;
#pragma unroll
            for (int db = 0; db < DP / 32; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    ak[db][i] += from[(db * 16 + i) * 64];
                    av[db][i] += from[(DP / 2 + db * 16 + i) * 64];
                }
        }
    }
    if (my_key < s.lk) {
        store_cols<E, DP>(ak, p.scale, static_cast<elem*>(p.dk) + (int64_t)(s.k0 + key) * p.dk_row + kvh * p.dk_head, p.d, half);
        store_cols<E, DP>(av, 1.f, static_cast<elem*>(p.dv) + (int64_t)(s.k0 + key) * p.dv_row + kvh * p.dv_head, p.d, half);
    }
}

// ---- launches
// How the rows of the forward pass are dealt out, by what is known on the host: the sums of the lengths, not the lengths.  Measured on both sides (bfloat16,
// us; q: queries of a sequence, k: its keys, D: columns of a head):
//   32 rows, four wavefronts (D = 128: two) that share the keys, for rows of one query.  With 64 rows and two of them instead: 128 x 12 heads of D = 64 with
//     20..61 keys 14.2, not 19.8; 200..500 keys 30.4, not 32.3; 1000..2000 keys 111, not 110; 300 x 4 key heads of D = 128 with 1000..3000 keys 222, not 218;
//     float32 with 200..500 keys 111, not 101.  Hence from 256 keys per sequence on, for both types: bfloat16 alone would have 64 rows up to about 1000 keys, where
//     they gain 6 per cent at most, float32 alone 32 rows from fewer keys on.  Always with few workgroups, whose keys may be dealt out (below), because a
//     long sequence among short ones would hold up the launch: short ones alone (64 sequences of 8..28 keys) would take 10.3, not 12.5.
//   64 rows, two wavefronts of rows by two that share the keys, for short sequences (20..60 tokens 9.8; 128 rows 10.8) and few tiles (512 tokens x 4, four
//     key heads 12.1; 14.2.  1000 tokens, twelve 16.7; 21.0.  1000 tokens, eight of D = 128 with groups of 4 23.6; 30.6).
//   128 rows, four wavefronts, each with its own rows and all the keys, so that each key block is read from LDS for twice the rows: 512 tokens x 8, four key
//     heads 16.0; 64 rows 19.4.  256 x 64 tokens, twelve heads 31.4; 35.1, 256 x 30..80 36; 38.  64 x 128 tokens, twelve heads, 15.1; 19.6.  9 sequences of 300..4001 tokens 111; 131.  8192 tokens, D = 128 560; 698.
//   Keys dealt out to several workgroups, whose sums a second launch joins: one token over 8192 keys, eight heads 17.5; not dealt out 114.
//     32 tokens over 100..8191 keys 33.8; 115.  Only for 32 rows: what has more rows a sequence walks all keys in each workgroup, however few those are.
struct Deal {
    int rows_each;          // rows of a workgroup: 32, 64 or 128
    int keys_each;          // > 0: keys of a workgroup
    int64_t items, tiles;   // workgroups per key head; tiles
};
Deal deal_of(int n_seqs, int total_q, int total_k, int heads, int kv_heads)
{
    const int64_t group = heads / kv_heads, rows = total_q * group;
    Deal d{128, 0, 0, 0};
    const auto tiles = [&](int bm) { return rows / bm + n_seqs; };
    const bool few = tiles(32) * kv_heads < 1024;
    if (rows <= 32ll * n_seqs && (few || total_k > 256ll * n_seqs)) d.rows_each = 32;
    else if (rows <= 40ll * n_seqs || tiles(128) * kv_heads < 512) d.rows_each = 64;
    d.tiles = tiles(d.rows_each);
    d.items = d.tiles;
    if (d.rows_each == 32 && few) {
        // about 1024 workgroups of 512 keys each at least (what a workgroup needs to get going costs as much as 256 keys)
        const int64_t each = std::max<int64_t>(512, ((int64_t)total_k * kv_heads / 1024 + 255) / 256 * 256);
        if (total_k > each) {
            d.keys_each = (int)each;
            // The host knows sums alone.  A sequence's tiles are t <= rows / 32 + 1, its chunks c <= 1 + keys / each, and t (c - 1) <= keys / (each / 4), which
            // chunks_of sees to: without that only the product of the sums would bound them, half a million workgroups and 8 GB for 500 tokens of 32 heads
            // on one, of which 1000 had anything to do.  So there are at most 5120, and 87 MB.
            const int64_t c = total_k / each;
            d.items = d.tiles + std::min((rows / 32 + 1) * c, total_k / (each / kTilesFree));
        }
    }
    return d;
}

template <typename E, int DP, bool FULL, int RW, int KW, int UB, int STAGES>
hipError_t forward_with(const PackedAttn& p, const Deal& d, hipStream_t stream)
{
    using F = Forward<E, DP, RW, KW, UB, STAGES>;
    static std::atomic<uint64_t> done{0};
    hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void*>(packed_forward_kernel<E, DP, RW, KW, UB, STAGES, FULL>), F::LDS, done);
    if (e != hipSuccess) return e;
    if (!fits_launch(d.items * p.kv_heads, F::NW * 64)) return hipErrorInvalidValue;
    packed_forward_kernel<E, DP, RW, KW, UB, STAGES, FULL><<<(unsigned)(d.items * p.kv_heads), F::NW * 64, F::LDS, stream>>>(p, d.keys_each);
    if ((e = hipGetLastError()) != hipSuccess || d.keys_each == 0) return e;
    const int rows = std::min<int64_t>(F::BM, (int64_t)p.total_q * (p.heads / p.kv_heads));
    packed_join_kernel<E, DP, F::BM><<<dim3((unsigned)(d.tiles * p.kv_heads), (unsigned)((rows + 3) / 4)), 256, 0, stream>>>(p, d.keys_each, (int)d.items);
    return hipGetLastError();
}
// (rings of at most 64 KB, of which a compute unit holds two, as long as that leaves two stages)
template <typename E, int DP, bool FULL>
hipError_t forward_of(const PackedAttn& p, hipStream_t stream)
{
    const Deal d = deal_of(p.n_seqs, p.total_q, p.total_k, p.heads, p.kv_heads);
    constexpr int ROWB = Tile<E, DP>::ROWB;
    if (d.rows_each == 32) {
        if constexpr (ROWB == 128) return forward_with<E, DP, FULL, 1, 4, 1, 2>(p, d, stream);
        else return forward_with<E, DP, FULL, 1, 2, 1, 2>(p, d, stream);
    }
    if (d.rows_each == 64) return forward_with<E, DP, FULL, 2, 2, 1, ROWB == 128 ? 3 : 2>(p, d, stream);
    return forward_with<E, DP, FULL, 4, 1, 2, ROWB == 128 ? 3 : 2>(p, d, stream);
}

template <typename E, int DP, bool FULL>
hipError_t gradient_of(const PackedAttn& p, hipStream_t stream)
{
    constexpr int ROWB = Tile<E, DP>::ROWB, SQ = ROWB == 128 ? 3 : 2, SK = ROWB == 512 || ROWB == 128 ? 2 : 3, A = ROWB == 128 ? 1 : 2, B = ROWB == 128 ? 4 : 2;
    using G = KeyGrad<E, DP, A, B, SK>;
    using R = RowGrad<E, DP, 2, 2, SQ>;
    static std::atomic<uint64_t> done_q{0}, done_k{0};
    hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void*>(packed_dq_kernel<E, DP, 2, 2, SQ, FULL>), R::LDS, done_q);
    if (e != hipSuccess) return e;
    e = ensure_dynamic_lds(reinterpret_cast<const void*>(packed_dkv_kernel<E, DP, A, B, SK, FULL>), G::LDS, done_k);
    if (e != hipSuccess) return e;
    float* stat = static_cast<float*>(p.work);
    const int64_t tiles_s = (int64_t)p.total_q * p.group / 128 + p.n_seqs, tiles_q = (int64_t)p.total_q * p.group / R::BM + p.n_seqs, tiles_k = (int64_t)p.total_k / G::BN + p.n_seqs;
    if (!fits_launch(std::max({tiles_s, tiles_q, tiles_k}) * p.kv_heads, 256)) return hipErrorInvalidValue;
    packed_stat_kernel<E, DP, FULL><<<(unsigned)(tiles_s * p.kv_heads), 256, 0, stream>>>(p, stat);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    packed_dkv_kernel<E, DP, A, B, SK, FULL><<<(unsigned)(tiles_k * p.kv_heads), G::NW * 64, G::LDS, stream>>>(p, stat);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    packed_dq_kernel<E, DP, 2, 2, SQ, FULL><<<(unsigned)(tiles_q * p.kv_heads), R::NW * 64, R::LDS, stream>>>(p, stat);
    return hipGetLastError();
}

// f(columns of a tile, whether they are the width itself): kernels of their own, because one that asks costs full heads 1 to 2 per cent.  Narrower ones, with the
// lanes off and with copies of real columns instead: width 80, 256 sentences 57.5 and 55.6 us, 9 packed documents with gradient 785 and 798.
template <typename F>
hipError_t with_width(int d, F&& f)
{
    if (d <= 64) return d == 64 ? f(std::integral_constant<int, 64>(), std::true_type()) : f(std::integral_constant<int, 64>(), std::false_type());
    return d == 128 ? f(std::integral_constant<int, 128>(), std::true_type()) : f(std::integral_constant<int, 128>(), std::false_type());
}

}  // namespace

size_t packed_attention_work(int n_seqs, int total_q, int total_k, int heads, int kv_heads, int d)
{
    const Deal deal = deal_of(n_seqs, total_q, total_k, heads, kv_heads);
    return deal.keys_each ? (size_t)deal.items * kv_heads * deal.rows_each * ((d <= 64 ? 64 : 128) + 4) * 4 : 0;
}
size_t packed_attention_grad_work(int total_q, int heads) { return (size_t)total_q * heads * 8; }

hipError_t launch_packed_attention(const PackedAttn& p, int f32, hipStream_t stream)
{
    return with_width(p.d, [&](auto dp, auto full) { return f32 ? forward_of<F32, dp.value, full.value>(p, stream) : forward_of<B16, dp.value, full.value>(p, stream); });
}

hipError_t launch_packed_attention_grad(const PackedAttn& p, int f32, hipStream_t stream)
{
    return with_width(p.d, [&](auto dp, auto full) { return f32 ? gradient_of<F32, dp.value, full.value>(p, stream) : gradient_of<B16, dp.value, full.value>(p, stream); });
}

}  // namespace mt
