// Rows of an embedding table, scaled, and the table's gradient.
//   out_i = scale table[id_i] (an id outside the vocabulary: zeros),  dtable_v = scale sum over i with id_i = v of grad_i, in the order of i
// Both move memory and little else: 32768 tokens of width 768 in bfloat16 are looked up in 13.7 us (50 MB read, most of it from caches, and 50 MB written), and
// their gradient over 30522 rows in float32 takes 70 us: the sort's launches 21, sums and cleared rows 25 (144 MB, 5.7 TB/s), the join of cut runs 5, and the gaps between.
//
// Gradient.  The tokens are sorted by id, keeping their order (radix sort of (id, place) pairs, 8 bits or fewer a pass, no atomics whose order could
// show), and cut into chunks of kChunk sorted tokens, whatever ids they have: words follow a 1 / rank law, so a workgroup per table row would leave
// one with thousands of rows to add and most with none.  A workgroup adds its chunk's runs of equal ids in registers (float32); a run that lies
// inside the chunk is a finished row, the first and the last run of a chunk may go on in its neighbours and are left as partial sums, which a second
// launch puts together in order.  Rows without a token are found by a search in the sorted ids and cleared by further workgroups of the same launch.
#include "device_util.h"
#include "packed.h"

namespace mt {

namespace {

template <typename T>
struct Chunk;
template <>
struct Chunk<__bf16> {
    typedef bf16x8 vec;
    static constexpr int N = 8;
};
template <>
struct Chunk<float> {
    typedef f32x4 vec;
    static constexpr int N = 4;
};

template <typename T>
__global__ __launch_bounds__(256) void embedding_rows_kernel(Embedding p)
{
    typedef typename Chunk<T>::vec vec;
    constexpr int N = Chunk<T>::N;
    const uint32_t per = p.hidden / N;
    const uint32_t at = blockIdx.x * 256 + threadIdx.x, row = at / per;
    if (row >= (uint32_t)p.n) return;
    const uint32_t c = (at - row * per) * N;
    const int id = p.ids[row];
    vec v;
    if ((uint32_t)id < (uint32_t)p.vocab) {
        v = *reinterpret_cast<const vec*>(static_cast<const T*>(p.table) + id * p.ld_in + c);
        if (p.scale != 1.f) {
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = (T)((float)v[e] * p.scale);
        }
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = (T)0.f;
    }
    *reinterpret_cast<vec*>(static_cast<T*>(p.out) + row * p.ld_out + c) = v;
}

// ---- stable sort of (id, place) by id; ids outside the vocabulary become `vocab` and end up last
struct SortPass {
    const int32_t *ids;             // first pass: the ids as given; else null
    const uint32_t *key_in, *place_in;
    uint32_t *key_out, *place_out;
    int32_t* hist;                  // [workgroups][256]
    int n, vocab, shift, bits;
};
// up to 4096 tokens (what one workgroup's LDS holds twice) are sorted by one launch: 1000 tokens of width 768, whole gradient 25.7 us, with the launches of the long
// sort 31.5; 4096 tokens 28.7 and 34.0
constexpr int kSmallSort = 4096;

__device__ __forceinline__ uint32_t sort_key(const SortPass& p, int i)
{
    if (!p.ids) return p.key_in[i];
    const int id = p.ids[i];
    return (uint32_t)id < (uint32_t)p.vocab ? id : p.vocab;
}

// lanes of the wavefront that hold the same digit (idle lanes hold none)
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, int bits, bool held)
{
    uint64_t m = __ballot(held);
    for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot((digit >> b) & 1);
        m &= (digit >> b) & 1 ? set : ~set;
    }
    return m;
}

template <int ITEMS>
__global__ __launch_bounds__(256) void sort_count_kernel(SortPass p)
{
    __shared__ int count[256];
    count[threadIdx.x] = 0;
    __syncthreads();
    const int n0 = blockIdx.x * 256 * ITEMS;
    uint32_t key[ITEMS];
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
        const int i = n0 + j * 256 + threadIdx.x;
        key[j] = i < p.n ? sort_key(p, i) : 0;
    }
#pragma unroll
    for (int j = 0; j < ITEMS; ++j)
        if (n0 + j * 256 + (int)threadIdx.x < p.n) atomicAdd(&count[(key[j] >> p.shift) & ((1u << p.bits) - 1)], 1);
    __syncthreads();
    p.hist[blockIdx.x * 256 + threadIdx.x] = count[threadIdx.x];
}

// inclusive sum over the 256 threads of the workgroup's first 4 wavefronts; sums: 4 ints of LDS
__device__ __forceinline__ int sum_before_256(int v, int* sums)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int s = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int up = __shfl_up(s, o);
        if (lane >= o) s += up;
    }
    if (lane == 63 && wave < 4) sums[wave] = s;
    __syncthreads();
    for (int w = 0; w < 4; ++w) s += w < wave ? sums[w] : 0;
    return s - v;
}

// A wavefront's keys are consecutive, so that ranks keep their order: rank = keys with the digit in front, in the wavefront, in the wavefronts before and
// in the workgroups before.
template <int ITEMS>
__global__ __launch_bounds__(256) void sort_place_kernel(SortPass p)
{
    __shared__ int count[4][256], base[256], sums[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
#pragma unroll
    for (int w = 0; w < 4; ++w) count[w][tid] = 0;
    const int n0 = blockIdx.x * 256 * ITEMS + wave * 64 * ITEMS;
    uint32_t key[ITEMS], place[ITEMS];
    int rank[ITEMS];
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
        const int i = n0 + j * 64 + lane;
        key[j] = i < p.n ? sort_key(p, i) : 0;
        place[j] = i < p.n ? (p.ids ? (uint32_t)i : p.place_in[i]) : 0;
    }
    int all = 0, before = 0;
    for (int b0 = 0; b0 < (int)gridDim.x; b0 += 16) {
        int c[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) c[j] = p.hist[min(b0 + j, (int)gridDim.x - 1) * 256 + tid];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            all += b0 + j < (int)gridDim.x ? c[j] : 0;
            before += b0 + j < (int)blockIdx.x ? c[j] : 0;
        }
    }
    base[tid] = sum_before_256(all, sums) + before;
    const uint32_t mask = (1u << p.bits) - 1;
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
        const bool held = n0 + j * 64 + lane < p.n;
        const uint32_t d = (key[j] >> p.shift) & mask;
        const uint64_t same = same_digit(d, p.bits, held);
        const int first = __ffsll((unsigned long long)same) - 1;
        int had = 0;
        if (held && lane == first) {
            had = count[wave][d];
            count[wave][d] = had + __popcll(same);
        }
        rank[j] = __shfl(had, first) + __popcll(same & ((1ull << lane) - 1));
    }
    __syncthreads();
    int sum = base[tid];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int c = count[w][tid];
        count[w][tid] = sum;
        sum += c;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
        if (n0 + j * 64 + lane >= p.n) continue;
        const int to = count[wave][(key[j] >> p.shift) & mask] + rank[j];
        p.key_out[to] = key[j];
        p.place_out[to] = place[j];
    }
}

// the whole sort of up to kSmallSort tokens in one workgroup: one launch instead of two a pass
__global__ __launch_bounds__(1024) void sort_small_kernel(SortPass p, int passes)
{
    __shared__ uint32_t key[2][kSmallSort];
    __shared__ uint16_t place[2][kSmallSort], count[16][256];
    __shared__ int sums[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int i = tid + j * 1024;
        if (i < p.n) {
            key[0][i] = sort_key(p, i);
            place[0][i] = (uint16_t)i;
        }
    }
    const uint32_t mask = (1u << p.bits) - 1;
    for (int pass = 0; pass < passes; ++pass) {
        const int shift = pass * p.bits, from = pass & 1;
        for (int i = tid; i < 16 * 256; i += 1024) (&count[0][0])[i] = 0;
        __syncthreads();
        uint32_t k[4], at[4];
        int rank[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = wave * 256 + j * 64 + lane;
            const bool held = i < p.n;
            k[j] = held ? key[from][i] : 0;
            at[j] = held ? place[from][i] : 0;
            const uint32_t d = (k[j] >> shift) & mask;
            const uint64_t same = same_digit(d, p.bits, held);
            const int first = __ffsll((unsigned long long)same) - 1;
            int had = 0;
            if (held && lane == first) {
                had = count[wave][d];
                count[wave][d] = (uint16_t)(had + __popcll(same));
            }
            rank[j] = __shfl(had, first) + __popcll(same & ((1ull << lane) - 1));
        }
        __syncthreads();
        int all = 0;
        if (tid < 256)
            for (int w = 0; w < 16; ++w) all += count[w][tid];
        int sum = sum_before_256(all, sums);
        if (tid < 256)
            for (int w = 0; w < 16; ++w) {
                const int c = count[w][tid];
                count[w][tid] = (uint16_t)sum;
                sum += c;
            }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (wave * 256 + j * 64 + lane >= p.n) continue;
            const int to = count[wave][(k[j] >> shift) & mask] + rank[j];
            if (pass + 1 < passes) {
                key[from ^ 1][to] = k[j];
                place[from ^ 1][to] = (uint16_t)at[j];
            } else {
                p.key_out[to] = k[j];
                p.place_out[to] = at[j];
            }
        }
        __syncthreads();
    }
}

// ---- sums
constexpr int kChunk = 32, kClear = 64;         // sorted tokens, table rows of a workgroup

struct Sums {
    const uint32_t *key, *place;
    float* part;            // [chunks][2][hidden]: the run that came in from the chunk before, the run that goes on into the next
    int chunks;
};

template <typename Out, int N>
__device__ __forceinline__ void put_row(const Embedding& p, uint32_t row, int c, const float (&s)[N])
{
    typedef Out outv __attribute__((ext_vector_type(N)));
    outv* at = reinterpret_cast<outv*>(static_cast<Out*>(p.out) + row * p.ld_out + c);
    outv v;
    if constexpr (sizeof(Out) == 4) {
        if (p.accumulate) {
            v = *at;
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] += s[e] * p.scale;
            *at = v;
            return;
        }
    }
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = (Out)(s[e] * p.scale);
    *at = v;
}

template <typename T, typename Out>
__global__ __launch_bounds__(128) void embedding_sums_kernel(Embedding p, Sums s)
{
    constexpr int N = Chunk<T>::N;
    typedef typename Chunk<T>::vec vec;
    __shared__ uint32_t key[kChunk + 2], place[kChunk];
    __shared__ int absent[kClear];
    const int tid = threadIdx.x, c = (blockIdx.y * 128 + tid) * N;
    if ((int)blockIdx.x >= s.chunks) {
        // rows without a token
        const int v0 = ((int)blockIdx.x - s.chunks) * kClear;
        if (tid < kClear) {
            const uint32_t v = v0 + tid;
            int lo = 0, hi = p.n;
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (s.key[mid] < v) lo = mid + 1;
                else hi = mid;
            }
            absent[tid] = (int)v < p.vocab && (lo == p.n || s.key[lo] != v);
        }
        __syncthreads();
        if (c >= p.hidden) return;
        typedef Out outv __attribute__((ext_vector_type(N)));
        for (int r = 0; r < kClear; ++r)
            if (absent[r]) {
                outv z;
#pragma unroll
                for (int e = 0; e < N; ++e) z[e] = (Out)0.f;
                *reinterpret_cast<outv*>(static_cast<Out*>(p.out) + (v0 + r) * p.ld_out + c) = z;
            }
        return;
    }
    const int n0 = blockIdx.x * kChunk, held = min(kChunk, p.n - n0);
    if (tid < kChunk + 2) {
        const int i = n0 + tid - 1;
        key[tid] = i >= 0 && i < p.n ? s.key[i] : 0xFFFFFFFFu;      // (no id)
    }
    if (tid < held) place[tid] = s.place[n0 + tid];
    __syncthreads();
    if (c >= p.hidden) return;
    const auto* g = static_cast<const T*>(p.grad) + c;
    float sum[N];
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] = 0.f;
    bool from_before = key[0] == key[1];
    for (int k0 = 0; k0 < held; k0 += 8) {
        vec v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = *reinterpret_cast<const vec*>(g + place[min(k0 + k, held - 1)] * p.ld_in);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int i = k0 + k;
            if (i >= held) break;
            const uint32_t id = key[i + 1];
            if (id >= (uint32_t)p.vocab) return;                      // tokens outside the vocabulary are the last
#pragma unroll
            for (int e = 0; e < N; ++e) sum[e] += (float)v[k][e];
            if (id == key[i + 2] && i + 1 < held) continue;
            const bool goes_on = id == key[i + 2];
            if (from_before || goes_on) {
                float* to = s.part + ((int64_t)blockIdx.x * 2 + (from_before ? 0 : 1)) * p.hidden + c;
#pragma unroll
                for (int e = 0; e < N; ++e) to[e] = sum[e];
            } else put_row<Out, N>(p, id, c, sum);
            from_before = false;
#pragma unroll
            for (int e = 0; e < N; ++e) sum[e] = 0.f;
        }
    }
}

// Runs of more than one chunk: the workgroup of the chunk where a run begins adds up its partial sums.  Four wavefronts share them, 8 chunks each in turn, and
// their sums are added in order.
template <typename Out>
__global__ __launch_bounds__(256) void embedding_join_kernel(Embedding p, Sums s)
{
    constexpr int N = 4;
    __shared__ f32x4 other[3][64];
    const int chunk = blockIdx.x, n0 = chunk * kChunk, end = n0 + kChunk, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (end >= p.n) return;
    const uint32_t id = s.key[end - 1], after = s.key[end], at0 = s.key[n0], before = n0 > 0 ? s.key[n0 - 1] : 0xFFFFFFFFu;
    if (id >= (uint32_t)p.vocab || after != id || (at0 == id && before == id)) return;      // ends here; began before
    // the last chunk that the run reaches: the first one that it does not fill
    int last = chunk + 1;
    for (;;) {
        const int next = (last + lane + 1) * kChunk;
        const uint64_t on = __ballot(next < p.n && s.key[min(next, p.n - 1)] == id);
        if (~on == 0) {
            last += 64;
            continue;
        }
        last += __ffsll((unsigned long long)~on) - 1;
        break;
    }
    const int c = (blockIdx.y * 64 + lane) * N;
    f32x4 sum{0.f, 0.f, 0.f, 0.f};
    if (c < p.hidden) {
        if (wave == 0) sum = *reinterpret_cast<const f32x4*>(s.part + ((int64_t)chunk * 2 + 1) * p.hidden + c);
        for (int k = chunk + 1 + wave * 8; k <= last; k += 32) {
            f32x4 v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = *reinterpret_cast<const f32x4*>(s.part + (int64_t)min(k + j, last) * 2 * p.hidden + c);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (k + j <= last) sum += v[j];
        }
    }
    if (wave > 0) other[wave - 1][lane] = sum;
    __syncthreads();
    if (wave > 0 || c >= p.hidden) return;
    sum += other[0][lane];
    sum += other[1][lane];
    sum += other[2][lane];
    float out[N];
#pragma unroll
    for (int e = 0; e < N; ++e) out[e] = sum[e];
    put_row<Out, N>(p, id, c, out);
}

int chunks_of(int n) { return (n + kChunk - 1) / kChunk; }
// keys of a thread of the sort: 4 spread the work over more workgroups, but each adds up the counts of all.  Whole gradient with 4 and with 16: 32768 tokens 39.3 and
// 60.6 us, 131072 60.2 and 76.6, 400000 128.7 and 122.6
int items_of(int n) { return n <= 1 << 17 ? 4 : 16; }
int sort_groups(int n) { return (n + 256 * items_of(n) - 1) / (256 * items_of(n)); }

hipError_t sort(const Embedding& p, uint32_t* const (&key)[2], uint32_t* const (&place)[2], int32_t* hist, int& result, hipStream_t stream)
{
    int bits = 1;
    while (bits < 31 && (1u << bits) <= (uint32_t)p.vocab) ++bits;
    const int passes = (bits + 7) / 8;
    SortPass s{p.ids, nullptr, nullptr, key[0], place[0], hist, p.n, p.vocab, 0, (bits + passes - 1) / passes};
    result = 0;
    if (p.n <= kSmallSort) {
        sort_small_kernel<<<1, 1024, 0, stream>>>(s, passes);
        return hipGetLastError();
    }
    const unsigned grid = sort_groups(p.n);
    for (int i = 0; i < passes; ++i) {
        s.shift = i * s.bits;
        if (items_of(p.n) == 4) {
            sort_count_kernel<4><<<grid, 256, 0, stream>>>(s);
            sort_place_kernel<4><<<grid, 256, 0, stream>>>(s);
        } else {
            sort_count_kernel<16><<<grid, 256, 0, stream>>>(s);
            sort_place_kernel<16><<<grid, 256, 0, stream>>>(s);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        result = i & 1;
        s.ids = nullptr;
        s.key_in = key[i & 1];
        s.place_in = place[i & 1];
        s.key_out = key[(i & 1) ^ 1];
        s.place_out = place[(i & 1) ^ 1];
    }
    return hipSuccess;
}

template <typename T, typename Out>
hipError_t gradient_of(const Embedding& p, hipStream_t stream)
{
    unsigned char* ws = static_cast<unsigned char*>(p.work);
    const size_t list = up256((size_t)p.n * 4);
    uint32_t* const key[2] = {reinterpret_cast<uint32_t*>(ws), reinterpret_cast<uint32_t*>(ws + list)};
    uint32_t* const place[2] = {reinterpret_cast<uint32_t*>(ws + 2 * list), reinterpret_cast<uint32_t*>(ws + 3 * list)};
    int32_t* hist = reinterpret_cast<int32_t*>(ws + 4 * list);
    float* part = reinterpret_cast<float*>(ws + 4 * list + (size_t)sort_groups(p.n) * 1024);
    int at;
    hipError_t e = sort(p, key, place, hist, at, stream);
    if (e != hipSuccess) return e;
    const Sums s{key[at], place[at], part, chunks_of(p.n)};
    const int clear = p.accumulate ? 0 : (p.vocab + kClear - 1) / kClear;
    constexpr int cols = 128 * Chunk<T>::N;
    embedding_sums_kernel<T, Out><<<dim3(s.chunks + clear, (p.hidden + cols - 1) / cols), 128, 0, stream>>>(p, s);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    embedding_join_kernel<Out><<<dim3(s.chunks, (p.hidden + 255) / 256), 256, 0, stream>>>(p, s);
    return hipGetLastError();
}

}  // namespace

size_t embedding_grad_work(int n, int, int hidden)
{
    return 4 * up256((size_t)n * 4) + (size_t)sort_groups(n) * 1024 + up256((size_t)chunks_of(n) * 2 * hidden * 4);
}

hipError_t launch_embedding(const Embedding& p, int f32, hipStream_t stream)
{
    const int64_t n = (int64_t)p.n * (p.hidden / (f32 ? 4 : 8));
    if (n > 0xFFFFFF00ll) return hipErrorInvalidValue;
    const unsigned grid = (unsigned)((n + 255) / 256);
    if (f32) embedding_rows_kernel<float><<<grid, 256, 0, stream>>>(p);
    else embedding_rows_kernel<__bf16><<<grid, 256, 0, stream>>>(p);
    return hipGetLastError();
}

hipError_t launch_embedding_grad(const Embedding& p, int f32, hipStream_t stream)
{
    if (f32) return gradient_of<float, float>(p, stream);
    return p.out_f32 ? gradient_of<__bf16, float>(p, stream) : gradient_of<__bf16, __bf16>(p, stream);
}

}  // namespace mt
