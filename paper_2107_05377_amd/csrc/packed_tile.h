// 32x32 matrix-core blocks fed from LDS tiles of rows, in bfloat16 and float32, for the operators on packed tokens.
#pragma once

#include "device_util.h"

namespace mt {

typedef __attribute__((address_space(1))) const void* gptr_t;
typedef __attribute__((address_space(3))) void* lptr_t;
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;
typedef __attribute__((address_space(3))) s16x4* l16x4_t;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ uint32_t lds_address(const unsigned char* p) { return (uint32_t)(uintptr_t)(lptr_t)p; }

// 16 bytes a lane straight from memory to LDS, lane l's at address `to` + 16 l (`to` the same in all lanes).  As assembly, because the compiler would make every
// transposing LDS read wait for all such loads under way, the next tiles' among them; the waits are the callers' (s_waitcnt vmcnt, then a barrier), and
// there is no result in a register that could be used too early.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"        // (that m0 is a reserved register: it is told that this changes it)
__device__ __forceinline__ void load_to_lds(const void* from, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(__builtin_amdgcn_readfirstlane(to)), "v"(from) : "m0");
}
// A pointer that is the same in all lanes, in scalar registers.  Behind a vector instruction that writes one, a load has to wait 5 states before it reads it, which
// the compiler sees to in its own code only: here the wait is part of the value (where that is scalar work already, as in all kernels so far, 5 cycles a tile).
__device__ __forceinline__ const char* uniform(const char* p)
{
    const uint64_t v = (uint64_t)(uintptr_t)p;
    uint64_t s = (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(v >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)v);
    asm("s_nop 4" : "+s"(s));
    return reinterpret_cast<const char*>((uintptr_t)s);
}
// the same from a place that all lanes share and a lane's offset in bytes
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t offset, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(__builtin_amdgcn_readfirstlane(to)), "v"(offset), "s"(base) : "m0");
}
// both with the lanes of `on` alone (one at least), which the compiler need not know: what it has to do about other lanes would cost it a branch a load
__device__ __forceinline__ void load_to_lds_of(uint64_t on, const void* from, uint32_t to)
{
    uint64_t all;
    asm volatile("s_mov_b64 %0, exec\n\ts_mov_b64 exec, %3\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off\n\ts_mov_b64 exec, %0"
                 : "=&s"(all) : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(from), "s"(on) : "m0");
}
__device__ __forceinline__ void load_to_lds_of(uint64_t on, const void* base, uint32_t offset, uint32_t to)
{
    uint64_t all;
    asm volatile("s_mov_b64 %0, exec\n\ts_mov_b64 exec, %4\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b64 exec, %0"
                 : "=&s"(all) : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(offset), "s"(base), "s"(on) : "m0");
}
// the same with 4 bytes a lane
__device__ __forceinline__ void load_to_lds_4(const void* from, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(__builtin_amdgcn_readfirstlane(to)), "v"(from) : "m0");
}
#pragma clang diagnostic pop

// all but the wavefront's last N loads have landed
template <int N>
__device__ __forceinline__ void wait_loads()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// ---- element types: what 16 bytes of a row mean to the matrix instructions
struct B16 {
    typedef __bf16 elem;
    typedef bf16x8 frag;
    static constexpr int SIZE = 2, EPC = 8, KS = 16;      // elements per 16 bytes; elements of a sum per product step (both halves of the wavefront)
    static __device__ __forceinline__ f32x16 mma(frag a, frag b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
struct F32 {
    typedef float elem;
    typedef f32x4 frag;
    static constexpr int SIZE = 4, EPC = 4, KS = 8;
    static __device__ __forceinline__ f32x16 mma(frag a, frag b, f32x16 c)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
};

// ---- a tile of rows in LDS: rows of DP elements, 16-byte chunks exchanged within a row by the row's number so that reading one chunk of 16 rows,
// and reading a few chunks of 8 rows transposed, both reach all banks
template <typename E, int DP>
struct Tile {
    static constexpr int ROWB = DP * E::SIZE, CH = ROWB / 16, RPI = 1024 / ROWB;
    static __device__ __forceinline__ int key(int row)
    {
        if constexpr (CH == 4) return (row >> 2) & 3;
        else if constexpr (CH == 8) return ((row >> 3) & 1) | ((row >> 1) & 2) | ((row << 1) & 4);       // the row pair's three bits reversed
        else if constexpr (E::SIZE == 2) return ((row & 3) << 2) | ((row >> 2) & 3);
        else return (row & 3) | ((row << 1) & 8) | ((row >> 1) & 4);
    }
    // 16 bytes (a product step's operand) of row `row` (a lane's own) at step ks
    static __device__ __forceinline__ typename E::frag row_frag(const unsigned char* t, int row, int ks, int half)
    {
        return *reinterpret_cast<const typename E::frag*>(t + row * ROWB + (((ks * 2 + half) ^ key(row)) << 4));
    }
    // the operand "columns 32 db .. +31 as rows": lane l32 its column, the rows in the order in which accumulators hold them.
    // step c of 32 rows: bfloat16 rows 16 c + 4 half + {0..3, 8..11}, float32 rows 8 c + 4 half + {0..3}
    // (IN_ORDER: bfloat16 rows 16 c + 8 half + {0..7}, the order of row_frag; float32 has only one)
    template <bool IN_ORDER = false>
    static __device__ __forceinline__ typename E::frag col_frag(const unsigned char* t, int row0, int db, int c, int lane)
    {
        const int half = lane >> 5;
        if constexpr (E::SIZE == 2) {
            constexpr int NEXT = IN_ORDER ? 4 : 8;
            const int r = row0 + 16 * c + (IN_ORDER ? 8 : 4) * half + ((lane & 15) >> 2), chunk = db * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1), in = (lane & 1) * 8;
            union {
                s16x4 h[2];
                bf16x8 f;
            } u;
            u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((l16x4_t)(t + r * ROWB + ((chunk ^ key(r)) << 4) + in));
            u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((l16x4_t)(t + (r + NEXT) * ROWB + ((chunk ^ key(r + NEXT)) << 4) + in));
            return u.f;
        } else {
            f32x4 f;
            const int col = db * 32 + (lane & 31);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = row0 + 8 * c + 4 * half + i;
                f[i] = *reinterpret_cast<const float*>(t + r * ROWB + (((col >> 2) ^ key(r)) << 4) + (col & 3) * 4);
            }
            return f;
        }
    }
};

}  // namespace mt
