// Rows of an embedding table, scaled, and the table's gradient.
//   out_i = scale table[id_i] (an id outside the vocabulary: zeros),  dtable_v = scale sum over i with id_i = v of grad_i, in the order of i
// Both move memory and little else.  The gradient has no atomics: a workgroup owns some rows of the table and some columns, goes through all ids in
// order, lists those that are its own and adds their rows, so the sums (float32) do not depend on the launch.
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
    const int per = p.hidden / N;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = at / per;
    if (row >= p.n) return;
    const int c = (int)(at - row * per) * N, id = p.ids[row];
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

constexpr int kRows = 16, kCols = 512;

template <typename T, typename Out>
__global__ __launch_bounds__(256) void embedding_grad_kernel(Embedding p)
{
    __shared__ float acc[kRows][kCols];
    __shared__ int list[1024], wave_n[4];
    __shared__ bool used[kRows];
    const int v0 = blockIdx.x * kRows, c0 = blockIdx.y * kCols, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int i = tid; i < kRows * kCols; i += 256) (&acc[0][0])[i] = 0.f;
    if (tid < kRows) used[tid] = false;
    const int c = c0 + tid * 2;
    for (int n0 = 0; n0 < p.n; n0 += 1024) {
        __syncthreads();
        int total = 0;
        for (int part = 0; part < 4; ++part) {
            const int i = n0 + part * 256 + tid;
            const int id = i < p.n ? p.ids[i] : -1;
            const bool mine = id >= v0 && id < min(v0 + kRows, p.vocab);
            const uint64_t b = __ballot(mine);
            if (lane == 0) wave_n[wave] = __popcll(b);
            __syncthreads();
            int before = total;
            for (int w = 0; w < 4; ++w) {
                before += w < wave ? wave_n[w] : 0;
                total += wave_n[w];
            }
            if (mine) {
                list[before + __popcll(b & ((1ull << lane) - 1))] = (i - n0) << 8 | (id - v0);
                used[id - v0] = true;
            }
            __syncthreads();
        }
        if (c < p.hidden)
            for (int k = 0; k < total; ++k) {
                const int row = list[k] & 255;
                const T* g = static_cast<const T*>(p.grad) + (int64_t)(n0 + (list[k] >> 8)) * p.ld_in + c;
                acc[row][tid * 2] += (float)g[0];
                acc[row][tid * 2 + 1] += (float)g[1];
            }
    }
    __syncthreads();
    if (c >= p.hidden) return;
    for (int r = 0; r < kRows && v0 + r < p.vocab; ++r) {
        Out* o = static_cast<Out*>(p.out) + (int64_t)(v0 + r) * p.ld_out + c;
        for (int e = 0; e < 2; ++e) {
            const float s = acc[r][tid * 2 + e] * p.scale;
            if (!p.accumulate) o[e] = (Out)(used[r] ? s : 0.f);
            else if (used[r]) o[e] = (Out)((float)o[e] + s);
        }
    }
}

}  // namespace

size_t embedding_grad_work(int, int, int) { return 0; }

hipError_t launch_embedding(const Embedding& p, int f32, hipStream_t stream)
{
    const int64_t n = (int64_t)p.n * (p.hidden / (f32 ? 4 : 8));
    if ((n + 255) / 256 > 0x7FFFFFFF) return hipErrorInvalidValue;
    const unsigned grid = (unsigned)((n + 255) / 256);
    if (f32) embedding_rows_kernel<float><<<grid, 256, 0, stream>>>(p);
    else embedding_rows_kernel<__bf16><<<grid, 256, 0, stream>>>(p);
    return hipGetLastError();
}

hipError_t launch_embedding_grad(const Embedding& p, int f32, hipStream_t stream)
{
    const dim3 grid((p.vocab + kRows - 1) / kRows, (p.hidden + kCols - 1) / kCols);
    if (f32) embedding_grad_kernel<float, float><<<grid, 256, 0, stream>>>(p);
    else if (p.out_f32) embedding_grad_kernel<__bf16, float><<<grid, 256, 0, stream>>>(p);
    else embedding_grad_kernel<__bf16, __bf16><<<grid, 256, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace mt
