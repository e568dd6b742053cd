// Angles of rotary positions, and rows of heads normed and turned by them, for the kernels that turn rows.
#pragma once

#include "kernels.h"

namespace lserve {

// (scale cos, scale sin) of position times frequency: the angle in 64 bits, its whole turns dropped there, sine and cosine of the rest in 32.
__device__ __forceinline__ float2 turn_of(int position, double radians, float scale) {
    const double turns = (double)position * (radians * 0.15915494309189533577);
    float s, c;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
    return make_float2(c * scale, s * scale);
}

// Axis whose position turns a pair.
__device__ __forceinline__ int axis_of(const TurnArgs& t, int pair) { return (int)(t.axis_of[pair / 32] >> (2 * (pair % 32))) & 3; }

// Sum over groups of eight lanes; every lane of a group receives the total.
__device__ __forceinline__ float row8_sum(float x) {
    x += dpp_f<kDppXor1>(x);
    x += dpp_f<kDppXor2>(x);
    x += dpp_f<kDppHalfMirror>(x);
    return x;
}

// A row (a head of a token) is held by eight lanes, two pieces of eight channels to a lane.  With halves (channel i turns with i + R / 2) a lane has
// one piece of either half, or two neighbouring ones of what does not turn; interleaved (2 i with 2 i + 1) the two are eight apart.  Halves
// whose R is no multiple of 16 have partners in other lanes: they pass through LDS.
enum Layout { kHalves, kInterleaved, kOddHalves };
struct Pieces {
    int p0, p1;
    bool turns;  // kHalves: these pieces turn
};
template <int LAYOUT> __device__ __forceinline__ Pieces pieces_of(int l, int rotary_dim) {
    if (LAYOUT != kHalves) return {l, l + 8, true};
    const int half = rotary_dim / 16;
    return l < half ? Pieces{l, l + half, true} : Pieces{2 * l, 2 * l + 1, false};
}
// A lane's weights of a row's norm: of its two pieces.
struct Weights {
    float x[8], y[8];
};
__device__ __forceinline__ void load_weights(const float* weight, const Pieces& p, Weights& to) {
    if (weight) {
        const float4* w = reinterpret_cast<const float4*>(weight);
        const float4 a = w[2 * p.p0], b = w[2 * p.p0 + 1], c = w[2 * p.p1], d = w[2 * p.p1 + 1];
        to = {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}, {c.x, c.y, c.z, c.w, d.x, d.y, d.z, d.w}};
    }
}

// x - m over the root of mean((x - m)^2) + eps times the weight, in 32 bits throughout; m is 0 or the mean.
__device__ __forceinline__ void norm_row(float (&x)[8], float (&y)[8], const TurnArgs& t, bool weighted, const Weights& w) {
    if (t.norm == 2) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += x[i] + y[i];
        const float mean = row8_sum(sum) * (1.f / kHeadDim);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] -= mean;
            y[i] -= mean;
        }
    }
    float squares = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) squares = __builtin_fmaf(x[i], x[i], __builtin_fmaf(y[i], y[i], squares));
    const float inverse = rsqrtf(row8_sum(squares) * (1.f / kHeadDim) + t.eps);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] *= inverse;
        y[i] *= inverse;
    }
    if (weighted) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] *= w.x[i];
            y[i] *= w.y[i];
        }
    }
}

__device__ __forceinline__ float2 turned(float a, float b, float2 turn) {
    return make_float2(__builtin_fmaf(a, turn.x, -(b * turn.y)), __builtin_fmaf(b, turn.x, a * turn.y));
}

// A lane's two pieces of a row, normed and turned; turn: of its eight pairs (interleaved 0 .. 3 and 4 .. 7 are those of either piece).  Channels that do not turn keep their bits without a norm.
// kOddHalves: `room` is kHeadDim floats of LDS for the row, its own; turns: (cos, sin) of all pairs of the row's token.
template <class T, int LAYOUT, bool NORM>
__device__ __forceinline__ void turn_row(uint32_t (&x)[4], uint32_t (&y)[4], const float2 (&turn)[8], const TurnArgs& t, bool weighted,
                                         const Weights& w, const Pieces& p, float* room, const float2* turns) {
    float a[8], b[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        a[2 * i] = Elem<T>::lo(x[i]);
        a[2 * i + 1] = Elem<T>::hi(x[i]);
        b[2 * i] = Elem<T>::lo(y[i]);
        b[2 * i + 1] = Elem<T>::hi(y[i]);
    }
    if constexpr (NORM) {
        norm_row(a, b, t, weighted, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // what stands where nothing turns
            x[i] = Elem<T>::pack(a[2 * i], a[2 * i + 1]);
            y[i] = Elem<T>::pack(b[2 * i], b[2 * i + 1]);
        }
    }
    if constexpr (LAYOUT == kHalves) {
        uint32_t u[4], v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 first = turned(a[2 * i], b[2 * i], turn[2 * i]), second = turned(a[2 * i + 1], b[2 * i + 1], turn[2 * i + 1]);
            u[i] = Elem<T>::pack(first.x, second.x);
            v[i] = Elem<T>::pack(first.y, second.y);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = p.turns ? u[i] : x[i];
            y[i] = p.turns ? v[i] : y[i];
        }
    } else if constexpr (LAYOUT == kInterleaved) {
        const int pairs = t.rotary_dim / 2;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 first = turned(a[2 * i], a[2 * i + 1], turn[i]), second = turned(b[2 * i], b[2 * i + 1], turn[4 + i]);
            if (4 * p.p0 + i < pairs) x[i] = Elem<T>::pack(first.x, first.y);
            if (4 * p.p1 + i < pairs) y[i] = Elem<T>::pack(second.x, second.y);
        }
    } else {
        const int pairs = t.rotary_dim / 2;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            room[8 * p.p0 + i] = a[i];
            room[8 * p.p1 + i] = b[i];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (the row's lanes share a wavefront)
        auto at = [&](int channel, float own) {  // a channel of the row as it comes out
            if (channel >= 2 * pairs) return own;
            const bool upper = channel >= pairs;
            const int pair = upper ? channel - pairs : channel;
            const float2 both = upper ? turned(room[pair], own, turns[pair]) : turned(own, room[pair + pairs], turns[pair]);
            return upper ? both.y : both.x;
        };
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = 8 * p.p0 + 2 * i, d = 8 * p.p1 + 2 * i;
            const float a0 = at(c, a[2 * i]), a1 = at(c + 1, a[2 * i + 1]), b0 = at(d, b[2 * i]), b1 = at(d + 1, b[2 * i + 1]);
            const uint32_t u = Elem<T>::pack(a0, a1), v = Elem<T>::pack(b0, b1);
            // (channel by channel: what does not turn keeps its bits)
            x[i] = c + 1 < 2 * pairs ? u : c < 2 * pairs ? (u & 0xffffu) | (x[i] & 0xffff0000u) : x[i];
            y[i] = d + 1 < 2 * pairs ? v : d < 2 * pairs ? (v & 0xffffu) | (y[i] & 0xffff0000u) : y[i];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the next row takes the room over
    }
}

// Angles of a token in LDS: what a lane reads of its eight pairs is four pieces of sixteen bytes, each next to those of the other lanes of the row;
// the rows of neighbouring tokens start in other banks.  kOddHalves: pair by pair.
constexpr int kTurnRow = 80;  // float2 to a token
template <int LAYOUT> __device__ __forceinline__ int turn_place(int pair) {
    if (LAYOUT == kOddHalves) return pair;
    const int l = LAYOUT == kHalves ? pair / 8 : pair % 32 / 4, i = LAYOUT == kHalves ? pair % 8 : pair / 32 * 4 + pair % 4;
    return i / 2 * 16 + l * 2 + i % 2;
}
__device__ __forceinline__ void read_turns(const float2* row, int l, float2 (&turn)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 two = *reinterpret_cast<const float4*>(row + i * 16 + l * 2);
        turn[2 * i] = make_float2(two.x, two.y);
        turn[2 * i + 1] = make_float2(two.z, two.w);
    }
}

__device__ __forceinline__ void load_pieces(const void* base, size_t element, const Pieces& p, uint32_t (&x)[4], uint32_t (&y)[4]) {
    const uint4* row = reinterpret_cast<const uint4*>((const uint16_t*)base + element);
    const uint4 u = row[p.p0], v = row[p.p1];
    x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w;
    y[0] = v.x, y[1] = v.y, y[2] = v.z, y[3] = v.w;
}
__device__ __forceinline__ void store_pieces(void* base, size_t element, const Pieces& p, const uint32_t (&x)[4], const uint32_t (&y)[4]) {
    uint4* row = reinterpret_cast<uint4*>((uint16_t*)base + element);
    row[p.p0] = make_uint4(x[0], x[1], x[2], x[3]);
    row[p.p1] = make_uint4(y[0], y[1], y[2], y[3]);
}

// Waits for loads in flight into x and y: what follows, stores above all, is not asked for before they are there.  (A wait counts what was asked for
// since, and where some of that is conditional the compiler counts none of it: behind a row's stores it would wait for these too.)
__device__ __forceinline__ void arrived(uint32_t (&x)[4], uint32_t (&y)[4]) {
    asm volatile("" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]), "+v"(y[0]), "+v"(y[1]), "+v"(y[2]), "+v"(y[3])::"memory");
}

}  // namespace lserve
