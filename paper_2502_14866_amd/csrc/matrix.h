// What the kernels on the matrix cores share: operand types, direct-to-LDS loads, the transposing LDS read, quantised rows.
#pragma once

#include <type_traits>

#include "common.h"

namespace lserve {

typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf168_t __attribute__((ext_vector_type(8)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef float float16_t __attribute__((ext_vector_type(16)));

// Tiles reach LDS through direct-to-LDS loads, which place the 64 lanes of an instruction at 64
// consecutive 16-byte slots, so rows cannot be padded.  Bank conflicts are avoided by permuting the
// chunks inside a row instead.  Chunk c of K row r sits at position c ^ (r % 16): sixteen consecutive rows
// then hit sixteen different 16-byte bank groups for any fixed c, which is what the K operand reads (one
// row per lane) need.  Chunk c of V row r sits at position c ^ 4 (r % 4): a transposing read takes, from
// each of four consecutive rows, the same 64 bytes (32 channels), and the four stretches then fall into
// the four 64-byte quarters of the 256 bytes the banks serve per cycle.
__device__ __forceinline__ int k_chunk_pos(int row, int c) { return c ^ (row % 16); }
__device__ __forceinline__ int v_chunk_pos(int row, int c) { return c ^ (4 * (row % 4)); }

// The load itself is written in assembly: left to the compiler it is treated as an access that may
// touch both memory and LDS, and while one is in flight every LDS operand read in the loop waits with
// lgkmcnt(0), exposing the LDS latency in front of the products.  The source address is a wave-uniform
// 64-bit base (scalar registers) plus a 32-bit lane offset; `lds_base` is the wave-uniform LDS byte
// address of the 1 KiB destination and lane l lands at lds_base + 16 l.  Completion is tracked by
// vmcnt only, which dma_wait() drains before the workgroup barrier.
__device__ __forceinline__ void dma_load16(unsigned long long src_base, unsigned lane_offset, unsigned lds_base) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(lane_offset), "s"(src_base), "s"(lds_base) : "memory");
}
// Tells the compiler that a value every lane agrees on can live in scalar registers.
__device__ __forceinline__ unsigned long long uniform64(unsigned long long x) {
    return ((unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((unsigned)(x >> 32)) << 32) |
           (unsigned)__builtin_amdgcn_readfirstlane((unsigned)x);
}
__device__ __forceinline__ void dma_wait() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ unsigned lds_address(const void* p) {
    return (unsigned)(size_t)(const __attribute__((address_space(3))) void*)p;
}

constexpr float kLn2 = 0.6931471805599453f;

template <class T> struct Mfma;
template <> struct Mfma<F16> {
    static __device__ __forceinline__ float16_t run(uint4 a, uint4 b, float16_t c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ float4_t run16(uint4 a, uint4 b, float4_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
    }
};
template <> struct Mfma<BF16> {
    static __device__ __forceinline__ float16_t run(uint4 a, uint4 b, float16_t c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf168_t, a), __builtin_bit_cast(bf168_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ float4_t run16(uint4 a, uint4 b, float4_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf168_t, a), __builtin_bit_cast(bf168_t, b), c, 0, 0, 0);
    }
};

template <class T>
__device__ __forceinline__ uint4 pack8(const float* p) {
    return make_uint4(Elem<T>::pack(p[0], p[1]), Elem<T>::pack(p[2], p[3]), Elem<T>::pack(p[4], p[5]),
                      Elem<T>::pack(p[6], p[7]));
}

// Combine a value with the one held by the same lane of the other 32-lane half of the wave.
// (one swap of the upper half of a register with the lower half of its copy, in the vector ALU)
template <class Op> __device__ __forceinline__ float halves_combine(float x, Op op) {
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const swap_pair_t p = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const unsigned p0 = p[0], p1 = p[1];
    return op(__builtin_bit_cast(float, p0), __builtin_bit_cast(float, p1));
}
__device__ __forceinline__ float halves_max(float x) {
    return halves_combine(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float halves_sum(float x) {
    return halves_combine(x, [](float a, float b) { return a + b; });
}

typedef short short4_t __attribute__((ext_vector_type(4)));
// Transposing LDS read (ds_read_b64_tr_b16).  The sixteen lanes of a row each name four consecutive 16-bit
// elements; lane i receives element i % 4 of the lanes i / 4, i / 4 + 4, i / 4 + 8 and i / 4 + 12.  With lane s
// pointing at channels 4 (s % 4) .. + 3 of key s / 4, lane i ends up with channel i of four consecutive keys.
__device__ __forceinline__ uint2 lds_read_transposed(const unsigned char* p) {
    const short4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) short4_t*)(const __attribute__((address_space(3))) void*)p);
    return __builtin_bit_cast(uint2, v);
}

// Eight codes of a quantised row -> code * scale + zero -> eight values of the layer's 16-bit type.
template <class T, int BITS> __device__ __forceinline__ uint4 dequantise8(uint2 codes, uint32_t scale_zero) {
    const half2_t sz = __builtin_bit_cast(half2_t, scale_zero);
    const float scale = (float)sz[0], zero = (float)sz[1];
    uint32_t lo = codes.x, hi = codes.y;  // channels 0..3 and 4..7, one byte each
    if constexpr (BITS == 4) {
        hi = (codes.x >> 4) & 0x0f0f0f0fu;
        lo = codes.x & 0x0f0f0f0fu;
    }
    if constexpr (std::is_same<T, F16>::value) {
        // A code under the exponent byte 0x64 is the fp16 number 1024 + code, from which 1024 is taken off exactly; the
        // packed fma then rounds code * scale + zero once, to fp16, at three instructions per two values.
        const half2_t scale2 = {sz[0], sz[0]}, zero2 = {sz[1], sz[1]}, offset = {(_Float16)-1024.f, (_Float16)-1024.f};
        auto pair = [&](uint32_t word, uint32_t select) {
            const half2_t c = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, word, select)) + offset;
            return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(c, scale2, zero2));
        };
        return make_uint4(pair(lo, 0x04010400u), pair(lo, 0x04030402u), pair(hi, 0x04010400u), pair(hi, 0x04030402u));
    }
    float x[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[j] = __builtin_fmaf((float)((lo >> (8 * j)) & 0xffu), scale, zero);
        x[4 + j] = __builtin_fmaf((float)((hi >> (8 * j)) & 0xffu), scale, zero);
    }
    return pack8<T>(x);
}

}  // namespace lserve
