// Ranges of 16-bit rows and the quantiser of the paged cache, for the kernels that write pages.
#pragma once

#include "kernels.h"

namespace lserve {

// Smaller and larger of two pairs of fp16, and a pair with its signalling not-a-numbers quieted.  The first two return the other
// operand for a quiet not-a-number, but the quieted one itself for a signalling one, which would drop what the range held before:
// what comes from memory goes through quiet() first.  (Written out: ahead of the compiler's own forms goes such an instruction per
// operand, results of the forms themselves among them, where one per loaded pair will do.)
__device__ __forceinline__ half2_t pk_min(half2_t a, half2_t b) {
    half2_t r;
    asm("v_pk_min_f16 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ half2_t pk_max(half2_t a, half2_t b) {
    half2_t r;
    asm("v_pk_max_f16 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ half2_t quiet(uint32_t w) {
    const half2_t x = __builtin_bit_cast(half2_t, w);
    return pk_max(x, x);
}

// Smallest and largest of eight values (f: the same as numbers); what is not a number gives way.
template <class T> __device__ __forceinline__ void range8(const uint32_t (&)[4], const float (&f)[8], float& lo, float& hi) {
    lo = hi = quieted<T>(f[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) {
        const float x = quieted<T>(f[i]);
        lo = fminf(lo, x);
        hi = fmaxf(hi, x);
    }
}
template <> __device__ __forceinline__ void range8<F16>(const uint32_t (&w)[4], const float (&)[8], float& lo, float& hi) {
    half2_t l = quiet(w[0]), h = l;
#pragma unroll
    for (int i = 1; i < 4; ++i) {
        const half2_t x = quiet(w[i]);
        l = pk_min(l, x);
        h = pk_max(h, x);
    }
    lo = fminf((float)l[0], (float)l[1]);
    hi = fmaxf((float)h[0], (float)h[1]);
}

// Running channel-wise maximum and minimum of rows, eight channels to a lane.
template <class T> struct RowRange {
    float hi[8], lo[8];
    __device__ __forceinline__ RowRange() {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            hi[i] = -INFINITY;
            lo[i] = INFINITY;
        }
    }
    __device__ __forceinline__ void add(const uint4& x) {
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a = quieted<T>(Elem<T>::lo(w[i])), b = quieted<T>(Elem<T>::hi(w[i]));
            hi[2 * i] = fmaxf(hi[2 * i], a);
            lo[2 * i] = fminf(lo[2 * i], a);
            hi[2 * i + 1] = fmaxf(hi[2 * i + 1], b);
            lo[2 * i + 1] = fminf(lo[2 * i + 1], b);
        }
    }
    __device__ __forceinline__ float largest(int i) const { return hi[i]; }
    __device__ __forceinline__ float smallest(int i) const { return lo[i]; }
};
template <> struct RowRange<F16> {
    half2_t hi[4], lo[4];
    __device__ __forceinline__ RowRange() {
        const _Float16 inf = (_Float16)INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            hi[i] = half2_t{(_Float16)-inf, (_Float16)-inf};
            lo[i] = half2_t{inf, inf};
        }
    }
    __device__ __forceinline__ void add(const uint4& x) {
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const half2_t v = quiet(w[i]);
            hi[i] = pk_max(hi[i], v);
            lo[i] = pk_min(lo[i], v);
        }
    }
    __device__ __forceinline__ float largest(int i) const { return (float)hi[i / 2][i % 2]; }
    __device__ __forceinline__ float smallest(int i) const { return (float)lo[i / 2][i % 2]; }
};

// Asymmetric quantisation of one token row (Sec. 3.2: scale factor and zero point of a token are stored next to its features), to
// codes 0 .. levels = 2^BITS - 1:
//   zero = fp16(min), scale = fp16((max - zero) / levels), code = clamp(rint((x - zero) / scale), 0, levels),
// every step rounded as IEEE fp32 does, divisions too, so that the codes do not depend on the machine.
struct RowScale {
    float zero, scale;
    uint32_t pair;  // (scale, zero) as two fp16, as the pages keep them
};
template <int BITS> __device__ __forceinline__ RowScale row_scale(float lo, float hi) {
    constexpr float kLevels = (float)((1 << BITS) - 1);
    constexpr float kBig = 65504.f;  // largest finite fp16
    const _Float16 zero_h = (_Float16)fminf(fmaxf(lo, -kBig), kBig);
    const float zero = (float)zero_h;
    // (hi - zero) / levels: the product with the rounded reciprocal, corrected by its remainder, is the correctly rounded quotient
    // (for 15 and 255 with every one of the 2^23 significands); an infinite range, whose remainder is not a number, is its own
    // quotient (of either sign: rows of nothing but -inf have -inf - zero).
    constexpr float kInverse = 1.f / kLevels;
    const float range = hi - zero, q = range * kInverse;
    const float quotient = fabsf(range) == INFINITY ? range : __builtin_fmaf(__builtin_fmaf(-q, kLevels, range), kInverse, q);
    const _Float16 scale_h = (_Float16)fminf(quotient, kBig);
    const half2_t sz = {scale_h, zero_h};
    return {zero, (float)scale_h, __builtin_bit_cast(uint32_t, sz)};
}

// The codes of eight channels, packed as the pages keep them: 8 bits, one byte each, channels in order; 4 bits, byte j of the word holding
// channel j in its low and channel 4 + j in its high half, so that masking out either half leaves four codes in the byte lanes
// the 8-bit path uses.
template <int BITS> __device__ __forceinline__ uint2 codes8(const float (&f)[8], const RowScale& row) {
    constexpr float kLevels = (float)((1 << BITS) - 1);
    const float zero = row.zero, scale = row.scale;
    // code = rint of the fp32 quotient.  An IEEE division is some ten instructions, and eight of them per lane and row were
    // most of the write-back of quantised pages.  The product with the reciprocal is within 3 units in the last place of
    // the quotient, which for quotients up to 256 is less than 1e-4, so the two round to the same whole number unless the
    // product lies that close to a half.  That is two quotients in ten thousand, one lane in 600 (of eight quotients) and
    // one wavefront in ten (of 512), which then divides.  (Where the product is not a number or not finite, neither is the
    // quotient.)
    const float inv = __builtin_amdgcn_rcpf(scale);
    float t[8], off = 0.f;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const float a = (f[i] - zero) * inv, b = (f[i + 1] - zero) * inv;
        t[i] = __builtin_rintf(a);
        t[i + 1] = __builtin_rintf(b);
        off = fmaxf(fmaxf(off, fabsf(a - t[i])), fabsf(b - t[i + 1]));
    }
    if (off >= 0.4999f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = __builtin_rintf((f[i] - zero) / scale);
    }
    const float top = scale > 0.f ? kLevels : 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = __builtin_amdgcn_fmed3f(t[i], 0.f, top);  // 0 where there is no number
    auto bytes4 = [](float a, float b, float c, float d) {
        uint32_t u = __builtin_amdgcn_cvt_pk_u8_f32(a, 0, 0u);
        u = __builtin_amdgcn_cvt_pk_u8_f32(b, 1, u);
        u = __builtin_amdgcn_cvt_pk_u8_f32(c, 2, u);
        return (uint32_t)__builtin_amdgcn_cvt_pk_u8_f32(d, 3, u);
    };
    if constexpr (BITS == 8)
        return make_uint2(bytes4(t[0], t[1], t[2], t[3]), bytes4(t[4], t[5], t[6], t[7]));
    else
        return make_uint2(bytes4(__builtin_fmaf(t[4], 16.f, t[0]), __builtin_fmaf(t[5], 16.f, t[1]),
                                 __builtin_fmaf(t[6], 16.f, t[2]), __builtin_fmaf(t[7], 16.f, t[3])), 0u);
}

template <class T> __device__ __forceinline__ void unpack8(const uint32_t (&w)[4], float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = Elem<T>::lo(w[i]);
        f[2 * i + 1] = Elem<T>::hi(w[i]);
    }
}

// A row held by the 16 lanes of a DPP row, eight features per lane: the lane's eight codes and the token's (scale, zero).
template <class T, int BITS>
__device__ __forceinline__ void quantize_row(const uint4& x, uint2& packed, uint32_t& scale_zero) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    float f[8];
    unpack8<T>(w, f);
    float lo, hi;
    range8<T>(w, f, lo, hi);
    lo = fminf(lo, dpp_f<kDppXor1>(lo));
    hi = fmaxf(hi, dpp_f<kDppXor1>(hi));
    lo = fminf(lo, dpp_f<kDppXor2>(lo));
    hi = fmaxf(hi, dpp_f<kDppXor2>(hi));
    lo = fminf(lo, dpp_f<kDppHalfMirror>(lo));
    hi = fmaxf(hi, dpp_f<kDppHalfMirror>(hi));
    lo = fminf(lo, dpp_f<kDppMirror>(lo));
    hi = fmaxf(hi, dpp_f<kDppMirror>(hi));
    const RowScale row = row_scale<BITS>(lo, hi);
    packed = codes8<BITS>(f, row);
    scale_zero = row.pair;
}

// A row held by eight lanes, two pieces of eight features to a lane.
template <class T, int BITS>
__device__ __forceinline__ void quantize_pieces(const uint32_t (&x)[4], const uint32_t (&y)[4], uint2& x_codes, uint2& y_codes, uint32_t& scale_zero) {
    float f[8], g[8];
    unpack8<T>(x, f);
    unpack8<T>(y, g);
    float lo, hi, lo_y, hi_y;
    range8<T>(x, f, lo, hi);
    range8<T>(y, g, lo_y, hi_y);
    lo = fminf(lo, lo_y);
    hi = fmaxf(hi, hi_y);
    lo = fminf(lo, dpp_f<kDppXor1>(lo));
    hi = fmaxf(hi, dpp_f<kDppXor1>(hi));
    lo = fminf(lo, dpp_f<kDppXor2>(lo));
    hi = fmaxf(hi, dpp_f<kDppXor2>(hi));
    lo = fminf(lo, dpp_f<kDppHalfMirror>(lo));
    hi = fmaxf(hi, dpp_f<kDppHalfMirror>(hi));
    const RowScale row = row_scale<BITS>(lo, hi);
    x_codes = codes8<BITS>(f, row);
    y_codes = codes8<BITS>(g, row);
    scale_zero = row.pair;
}

}  // namespace lserve
