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
// Bound by memory: every value is read and written once.  A workgroup takes
// the heads of a few tokens and computes their cosines and sines once.
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
    int64_t n;                   // B T
    int T, t0, rotary, d;
    int tokens, split;           // tokens of a workgroup, workgroups that share their heads
    int copies[2];               // the channels behind the rotated ones are copied
    float magnitude, sign;
};

constexpr int kTokens = 4;                   // tokens per workgroup, at most
constexpr int kMostPairs = 512;

__device__ __forceinline__ float lo16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pair16(float x, float y) {
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x, (__bf16)y});
}

// WIDE: whole 16-byte pieces of 8 channels (half: one of each half).
template <bool HALF, bool WIDE>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
    __shared__ float2 turn[kTokens][kMostPairs];
    __shared__ int where[kTokens][2];            // sequence, token
    const int tid = threadIdx.x, pairs = a.rotary / 2;
    const int64_t n0 = (int64_t)blockIdx.x * a.tokens;
    const int count = (int)min((int64_t)a.tokens, a.n - n0);
    for (int i = tid; i < count * pairs; i += 256) {
        const int k = i / pairs, p = i - k * pairs;
        const int b = (int)((n0 + k) / a.T), t = (int)((n0 + k) - (int64_t)b * a.T);
        int64_t at = (int64_t)a.t0 + t;
        if (a.positions)
            at = a.positions[b * a.psb + t * a.pst];
        else if (a.starts)
            at += a.starts[b];
        double x = (double)at * a.freq[p] * 0.15915494309189533577;     // turns
        x -= rint(x);
        float s, c;
        sincospif(2.f * (float)x, &s, &c);
        turn[k][p] = float2{c * a.magnitude, s * a.sign};
    }
    if (tid < count) {
        where[tid][0] = (int)((n0 + tid) / a.T);
        where[tid][1] = (int)((n0 + tid) % a.T);
    }
    __syncthreads();
    const int step = WIDE ? (HALF ? 8 : 4) : 1;                          // pairs per item
    const int turned = pairs / step;
    const int rest = WIDE ? (a.d - a.rotary) / 8 : a.d - a.rotary;
    const int per = turned + rest;                                       // items of a head
    const int heads = a.heads[0] + a.heads[1];
    const int items = count * heads * per;
    for (int i = tid + 256 * (int)blockIdx.y; i < items; i += 256 * a.split) {
        const int e = i % per, hk = i / per, k = hk / heads;
        int h = hk - k * heads;
        const int w = h >= a.heads[0];
        if (w) h -= a.heads[0];
        const int b = where[k][0], t = where[k][1];
        const uint16_t* in = a.in[w] + b * a.isb[w] + t * a.ist[w] + h * a.ish[w];
        uint16_t* out = a.out[w] + b * a.osb[w] + t * a.ost[w] + h * a.osh[w];
        if (e >= turned) {
            if (!a.copies[w]) continue;
            const int c = a.rotary + (e - turned) * (WIDE ? 8 : 1);
            if constexpr (WIDE)
                *reinterpret_cast<u32x4*>(out + c) = *reinterpret_cast<const u32x4*>(in + c);
            else
                out[c] = in[c];
            continue;
        }
        const float2* cs = &turn[k][e * step];
        if constexpr (!WIDE) {
            const int ca = HALF ? e : 2 * e, cb = HALF ? e + pairs : 2 * e + 1;
            const float x = bf16_to_f32(in[ca]), y = bf16_to_f32(in[cb]);
            const uint32_t r = pair16(fmaf(x, cs->x, -(y * cs->y)), fmaf(x, cs->y, y * cs->x));
            out[ca] = (uint16_t)r;
            out[cb] = (uint16_t)(r >> 16);
        } else if constexpr (HALF) {
            const u32x4 x = *reinterpret_cast<const u32x4*>(in + 8 * e);
            const u32x4 y = *reinterpret_cast<const u32x4*>(in + pairs + 8 * e);
            u32x4 u, v;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 c0 = cs[2 * j], c1 = cs[2 * j + 1];
                const float x0 = lo16(x[j]), x1 = hi16(x[j]), y0 = lo16(y[j]), y1 = hi16(y[j]);
                u[j] = pair16(fmaf(x0, c0.x, -(y0 * c0.y)), fmaf(x1, c1.x, -(y1 * c1.y)));
                v[j] = pair16(fmaf(x0, c0.y, y0 * c0.x), fmaf(x1, c1.y, y1 * c1.x));
            }
            *reinterpret_cast<u32x4*>(out + 8 * e) = u;
            *reinterpret_cast<u32x4*>(out + pairs + 8 * e) = v;
        } else {
            const u32x4 x = *reinterpret_cast<const u32x4*>(in + 8 * e);
            u32x4 u;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float p = lo16(x[j]), q = hi16(x[j]);
                u[j] = pair16(fmaf(p, cs[j].x, -(q * cs[j].y)), fmaf(p, cs[j].y, q * cs[j].x));
            }
            *reinterpret_cast<u32x4*>(out + 8 * e) = u;
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
    a.n = (int64_t)B * T;
    a.T = T;
    a.t0 = t0;
    a.rotary = rotary;
    a.d = d;
    a.magnitude = magnitude;
    a.sign = transposed ? -magnitude : magnitude;
    a.tokens = a.n >= 1024 * kTokens ? kTokens : 1;
    // few tokens: workgroups share a token's heads
    a.split = a.n >= 512 ? 1 : 2;
    const dim3 grid((unsigned)((a.n + a.tokens - 1) / a.tokens), a.split);
    if (layout == DQ_ROPE_HALF)
        wide ? rope_kernel<true, true><<<grid, 256, 0, stream>>>(a) : rope_kernel<true, false><<<grid, 256, 0, stream>>>(a);
    else
        wide ? rope_kernel<false, true><<<grid, 256, 0, stream>>>(a)
             : rope_kernel<false, false><<<grid, 256, 0, stream>>>(a);
    return hip_check("rope launch", hipGetLastError());
}

}  // namespace dq
