// Rotary positions: pair i of a head's first `rotary` channels, (a, b), at
// position p becomes
//   (a cos - b sin, a sin + b cos) magnitude,  angle = p freq[i]
// (transposed: the angle's sign changed).  Pairs are (i, i + rotary / 2), "half",
// or (2 i, 2 i + 1), "interleaved"; the other channels stay.
//
// Angles are products in 64 bits, reduced to a part of a turn before they are
// rounded to fp32: far positions keep their fraction.  Rotations are computed
// in fp32 and rounded to bf16 once.
//
// Bound by memory: every value is read and written once, at 5.7 TB/s over 16384
// tokens of 40 heads of 128 (59 us).  A workgroup takes all heads of a token and
// computes their cosines and sines once, into LDS.
#include <math.h>

#include <algorithm>

#include "dq_chunk.h"
#include "dq_common.h"

namespace dq {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct RopeArgs {
    const uint16_t* in[2];       // queries, keys
    uint16_t* out[2];
    int64_t isb[2], ist[2], ish[2], osb[2], ost[2], osh[2];
    int heads[2];
    const double* freq;
    const int32_t* positions;
    int64_t psb, pst;
    const int32_t* starts;
    int T, t0, rotary, d;
    uint32_t tokens;             // of all sequences
    int split;                   // workgroups that share a token's heads
    int copies[2];               // the channels behind the rotated ones are copied
    float magnitude, sign;
};

constexpr int kMostPairs = 512;
constexpr uint32_t kAlongX = 1u << 23;           // tokens along x: a grid has under 2^32 work-items there

__device__ __forceinline__ float lo16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pair16(float x, float y) {
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x, (__bf16)y});
}

// One workgroup per token, or two that share its heads where tokens are few (fewer
// than 1024: 2.5 us in place of 3.1 for one token of 40 heads, 4.1 in place of 4.2
// for 512; 2048 tokens take 7.6 us with one, 8.6 with two).  Several tokens per
// workgroup gain nothing (16384 tokens: 62 us with one, 66 with four).  An item is a
// pair, or WIDE 16-byte pieces of 8 channels (half: one of each half), or as much
// behind the rotated channels.  A thread's first one is on its way while the angles
// are computed (48 x 33 tokens 11.0 to 7.2 us); more of them at a time only hold
// registers (two 7.3, three 7.7).
template <bool HALF, bool WIDE>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
    __shared__ float2 turn[kMostPairs];
    const int tid = threadIdx.x, pairs = a.rotary / 2;
    // (a workgroup behind the last token has no items; leaving here, before the other
    // arguments are there, would take 0.3 us more)
    const uint32_t at_z = blockIdx.z * kAlongX + blockIdx.x, token = min(at_z, a.tokens - 1);
    const int b = (int)(token / (uint32_t)a.T), t = (int)(token - (uint32_t)b * (uint32_t)a.T);
    const int step = WIDE ? (HALF ? 8 : 4) : 1;                          // pairs per item
    const int turned = pairs / step;
    const int rest = WIDE ? (a.d - a.rotary) / 8 : a.d - a.rotary;
    const uint32_t per = (uint32_t)(turned + rest);                      // items of a head
    const int items = at_z == token ? (a.heads[0] + a.heads[1]) * (int)per : 0, every = 256 * a.split;
    const uint16_t* in0 = a.in[0] + b * a.isb[0] + t * a.ist[0];
    const uint16_t* in1 = a.in[1] + b * a.isb[1] + t * a.ist[1];
    uint16_t* out0 = a.out[0] + b * a.osb[0] + t * a.ost[0];
    uint16_t* out1 = a.out[1] + b * a.osb[1] + t * a.ost[1];
    u32x4 x, y;
    uint16_t* to = nullptr;
    int e = -1;
    // first channel of an item
    auto channel = [&](int e) {
        if (e >= turned) return a.rotary + (e - turned) * (WIDE ? 8 : 1);
        return WIDE ? 8 * e : HALF ? e : 2 * e;
    };
    auto load = [&](int i) {
        e = -1;                                  // nothing, or nothing to do
        if (i >= items) return;
        int h = (int)((uint32_t)i / per);
        const int c = i - h * (int)per;
        const bool key = h >= a.heads[0];
        if (key) h -= a.heads[0];
        if (c >= turned && !(key ? a.copies[1] : a.copies[0])) return;
        e = c;
        const uint16_t* in = (key ? in1 : in0) + h * (key ? a.ish[1] : a.ish[0]) + channel(c);
        to = (key ? out1 : out0) + h * (key ? a.osh[1] : a.osh[0]) + channel(c);
        if constexpr (WIDE) {
            x = *reinterpret_cast<const u32x4*>(in);
            if (HALF && c < turned) y = *reinterpret_cast<const u32x4*>(in + pairs);
        } else {
            x[0] = in[0];
            if (c < turned) x[1] = in[HALF ? pairs : 1];
        }
    };
    int i = tid + 256 * (int)blockIdx.y;
    load(i);
    for (int p = tid; p < pairs; p += 256) {
        int64_t at = (int64_t)a.t0 + t;
        if (a.positions)
            at = a.positions[b * a.psb + t * a.pst];
        else if (a.starts)
            at += a.starts[b];
        double z = (double)at * a.freq[p] * 0.15915494309189533577;     // turns
        z -= rint(z);
        float s, c;
        sincospif(2.f * (float)z, &s, &c);
        turn[p] = float2{c * a.magnitude, s * a.sign};
    }
    __syncthreads();
    for (; i < items; i += every, load(i)) {
        if (e < 0) continue;
        if (e >= turned) {
            if constexpr (WIDE)
                *reinterpret_cast<u32x4*>(to) = x;
            else
                to[0] = (uint16_t)x[0];
            continue;
        }
        const float2* cs = &turn[e * step];
        if constexpr (!WIDE) {
            const float p = lo16(x[0]), q = lo16(x[1]);
            const uint32_t r = pair16(fmaf(p, cs->x, -(q * cs->y)), fmaf(p, cs->y, q * cs->x));
            to[0] = (uint16_t)r;
            to[HALF ? pairs : 1] = (uint16_t)(r >> 16);
        } else if constexpr (HALF) {
            u32x4 u, v;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 c0 = cs[2 * j], c1 = cs[2 * j + 1];
                const float x0 = lo16(x[j]), x1 = hi16(x[j]), y0 = lo16(y[j]), y1 = hi16(y[j]);
                u[j] = pair16(fmaf(x0, c0.x, -(y0 * c0.y)), fmaf(x1, c1.x, -(y1 * c1.y)));
                v[j] = pair16(fmaf(x0, c0.y, y0 * c0.x), fmaf(x1, c1.y, y1 * c1.x));
            }
            *reinterpret_cast<u32x4*>(to) = u;
            *reinterpret_cast<u32x4*>(to + pairs) = v;
        } else {
            u32x4 u;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float p = lo16(x[j]), q = hi16(x[j]);
                u[j] = pair16(fmaf(p, cs[j].x, -(q * cs[j].y)), fmaf(p, cs[j].y, q * cs[j].x));
            }
            *reinterpret_cast<u32x4*>(to) = u;
        }
    }
}

bool whole_pieces(const Q8Rows& r) {
    return ((reinterpret_cast<uintptr_t>(r.p) | (uintptr_t)(r.sb * 2) | (uintptr_t)(r.st * 2) | (uintptr_t)(r.sh * 2)) & 15) == 0;
}

}  // namespace

int launch_rope(int layout, int transposed, const double* freq, float magnitude, int32_t rotary, const RopeRows& q,
                const RopeRows& k, int32_t B, int32_t T, int32_t d, const int32_t* positions, int64_t pos_sb,
                int64_t pos_st, const int32_t* starts, int32_t t0, hipStream_t stream) {
    RopeArgs a;
    const RopeRows* rows[2] = {&q, &k};
    bool wide = layout == DQ_ROPE_HALF ? rotary % 16 == 0 : rotary % 8 == 0;
    wide = wide && d % 8 == 0;
    for (int i = 0; i < 2; ++i) {
        const RopeRows& r = *rows[i];
        a.in[i] = r.in.p;
        a.out[i] = const_cast<uint16_t*>(r.out.p);
        a.isb[i] = r.in.sb;
        a.ist[i] = r.in.st;
        a.ish[i] = r.in.sh;
        a.osb[i] = r.out.sb;
        a.ost[i] = r.out.st;
        a.osh[i] = r.out.sh;
        a.heads[i] = r.heads;
        a.copies[i] = r.in.p != r.out.p;
        if (r.heads) wide = wide && whole_pieces(r.in) && whole_pieces(r.out);
    }
    a.freq = freq;
    a.positions = positions;
    a.psb = pos_sb;
    a.pst = pos_st;
    a.starts = starts;
    a.T = T;
    a.t0 = t0;
    a.rotary = rotary;
    a.d = d;
    a.magnitude = magnitude;
    a.sign = transposed ? -magnitude : magnitude;
    a.tokens = (uint32_t)B * (uint32_t)T;        // at most 2^26
    a.split = a.tokens >= 1024 ? 1 : 2;
    const dim3 grid(std::min(a.tokens, kAlongX), a.split, (a.tokens + kAlongX - 1) / kAlongX);
    if (layout == DQ_ROPE_HALF)
        wide ? rope_kernel<true, true><<<grid, 256, 0, stream>>>(a) : rope_kernel<true, false><<<grid, 256, 0, stream>>>(a);
    else
        wide ? rope_kernel<false, true><<<grid, 256, 0, stream>>>(a)
             : rope_kernel<false, false><<<grid, 256, 0, stream>>>(a);
    return hip_check("rope launch", hipGetLastError());
}

}  // namespace dq
