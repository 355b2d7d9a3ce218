// The 8-bit cache: keys and values as int8 or e4m3 codes with one fp32 scale
// for each block of 32 tokens of one (sequence, KV head) and tensor; its
// encoder, the read-back, decode attention over it (all tokens, or the first
// ones and the newest), the attention weight of every block, and the eviction
// of the blocks with the least of it.
//
// Numbers.  s = fl32(max |x| / Q) over the block's 32 x 128 values, Q = 127 or
// 448 (the type's largest); code = x / s rounded to the type's nearest value,
// ties to even; x^ = s code.
//
// Layout.  A block is 4096 bytes in the order in which the matrix cores take
// their operands, so that every read of the attention is 1024 contiguous bytes
// per wavefront and no byte moves between lanes.  With t = 0..31 the token and
// c = 0..127 the channel, lane = 16 grp + col:
//   keys:   byte c % 16 of piece ((t / 16) 2 + c / 64) 64 + ((c / 16) % 4) 16 + t % 16
//           (16-byte pieces; a lane's piece is 16 channels of one token: two
//           8-channel slices of the A operand of a 16x16x32 product)
//   values: byte ((c / 16) % 2) 8 + (t / 16) 4 + t % 4 of piece
//           ((c / 32) 4 + (t / 4) % 4) 16 + c % 16
//           (a lane's piece is two channels of the 8 tokens whose weights the
//           first product leaves in that lane)
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "dq_common.h"
#include "dq_q8.h"

namespace dq {
namespace {

constexpr int kD = 128;
constexpr int kBlk = DQ_Q8_BLOCK;            // tokens that share a scale
constexpr int kBlkBytes = kBlk * kD;
constexpr float kTiny = 0x1p-96f;            // a block below is stored as zeros

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// Index of block `blk` of (b, h) in a cache of nb_cap blocks per sequence, or
// in pool pages ([num_pages][H][page / 32]).
__device__ __forceinline__ int64_t block_index(const Pages& pg, int H, int nb_cap, int b, int h, int blk, bool& bad) {
    if (!pg.bt) return ((int64_t)b * H + h) * nb_cap + blk;
    const int64_t p = physical_page(pg, b, blk * kBlk, bad);
    const int bpp = 1 << (pg.page_shift - 5);
    return (p * H + h) * bpp + (blk & (bpp - 1));
}

__device__ __forceinline__ int wave_index(int waves) {
    return __builtin_amdgcn_readfirstlane((int)(blockIdx.x * waves + threadIdx.x / kWave));
}

// ------------------------------------------------------------------ encoder

struct EncArgs {
    const uint16_t* x[2];        // keys, values
    int64_t sb[2], st[2], sh[2];
    uint8_t* data[2];
    float* scale[2];
    uint32_t* status;
    Pages pg;
    int H, blk0, nblk, n_new, nb_cap;
    int aligned[2];              // rows are whole 16-byte pieces, a block spans under 2^31 bytes
};

// x / s with its last bit made odd where the quotient is not exact, so that a
// later rounding to fewer bits is the rounding of the exact quotient.  t is
// within an ulp of it; the sign of x - s t (exact: one rounding, of a nonzero
// number far from underflow) says on which side.
__device__ __forceinline__ float quotient_odd(float x, float s, float inv) {
    float t = x * inv;
    t = fmaf(fmaf(-s, t, x), inv, t);
    const float r = fmaf(-s, t, x);
    const uint32_t u = __float_as_uint(t);
    const uint32_t away = (__float_as_uint(r) ^ u) >> 31;      // 0: |x / s| > |t|
    const uint32_t v = (u & 1u) ? u : u + 1u - 2u * away;
    return __uint_as_float(r == 0.f ? u : v);
}

// Four quotients to four code bytes.
template <int FMT>
__device__ __forceinline__ uint32_t codes4(const float (&t)[4]) {
    if constexpr (FMT == DQ_Q8_E4M3) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(t[0], t[1], 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(t[2], t[3], w, true);
        return (uint32_t)w;
    } else {
        // t + 1.5 2^23 rounds t to an integer, ties to even, in the low bits
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(t[i] + 12582912.f);
        const uint32_t lo = __builtin_amdgcn_perm(w[1], w[0], 0x0C0C0400u);
        const uint32_t hi = __builtin_amdgcn_perm(w[3], w[2], 0x04000C0Cu);
        return lo | hi;
    }
}

// Whether a quotient within 2^-22 of t, relative, might lie on another side of
// a border between two codes than t does (or on it).
//   int8: the border is half an integer away from the nearest one.
//   e4m3: three bits behind the leading one stay, so borders have the 20 bits
//   below them at 0x80000; below 2^-6 the steps stay those of 2^-6, which
//   adding it shows.
template <int FMT>
__device__ __forceinline__ bool near_border(const float (&t)[8]) {
    if constexpr (FMT == DQ_Q8_E4M3) {
        uint32_t least = ~0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float m = fabsf(t[i]);
            const uint32_t u = __float_as_uint(m < 0x1p-6f ? m + 0x1p-6f : m);
            least = min(least, (u + 0x80008u) & 0xFFFFFu);
        }
        return least <= 16u;
    } else {
        float most = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(t[i] - ((t[i] + 12582912.f) - 12582912.f)));
        return most > 0.5f - 0x1p-14f;
    }
}

__device__ __forceinline__ uint32_t pk_max(uint32_t a, uint32_t b) {
    const u16x2 x = __builtin_bit_cast(u16x2, a), y = __builtin_bit_cast(u16x2, b);
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(x, y));
}

__device__ __forceinline__ uint32_t finite_pair(uint32_t w) {
    if ((w & 0x7F80u) == 0x7F80u) w &= 0xFFFF0000u;
    if ((w & 0x7F800000u) == 0x7F800000u) w &= 0x0000FFFFu;
    return w;
}

// A wavefront's LDS copy of a block of values, between the lanes' order of work
// (four neighbouring pieces each) and the order of memory (whole lines per
// access); pieces swap places so that neither order meets a bank twice.
__device__ __forceinline__ int staged(int piece) { return piece ^ ((piece >> 2) & 3); }

__device__ __forceinline__ uint32_t quad_xor2(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, false);   // quad_perm [2, 3, 0, 1]
}

// One wavefront per block, heads fastest, so that the wavefronts of a
// workgroup read neighbouring rows.  A lane holds 64 values: of keys, the
// 16 channels of its four pieces; of values, 8 channels 8 (lane % 16) of the
// tokens 16 h2 + 4 (lane / 16) + i, whose codes are byte-transposed in the
// lane and swapped with lane ^ 2, which holds the pieces' other halves.
// Sequences and tensors are grid axes and a block's rows 32-bit offsets from a
// uniform base (4 x 8171 tokens, 8 heads, to e4m3: 41 us; with one axis, its
// divisions, and 64-bit addresses 44.  The bytes alone take 40 at 5.0 TB/s).
template <int FMT, int WHICH>
__device__ __forceinline__ void encode_block(const EncArgs& a, int w, int lane, uint4* stage) {
    constexpr bool keys = WHICH == 0;
    const int h = w % a.H, blk = w / a.H, b = blockIdx.y;
    bool bad = false;
    const int64_t bi = block_index(a.pg, a.H, a.nb_cap, b, h, a.blk0 + blk, bad);
    if (bad) {
        if (lane == 0 && a.status) atomicOr(a.status, DQ_STATUS_PAGE);
        return;
    }
    const int rows = min(kBlk, a.n_new - blk * kBlk);
    const int64_t st = a.st[WHICH];
    const uint16_t* src = a.x[WHICH] + (int64_t)b * a.sb[WHICH] + (int64_t)h * a.sh[WHICH] + (int64_t)blk * kBlk * st;
    const int col = lane & 15, grp = lane >> 4;
    // load i: keys: token 16 (i / 4) + col, channels 64 ((i / 2) % 2) + 16 grp + 8 (i % 2);
    //         values: token 16 (i / 4) + 4 grp + i % 4, channels 8 col
    uint32_t x[8][4];
    const int row0 = keys ? col : 4 * grp;
    const int ch0 = keys ? 16 * grp : 8 * col;
    auto row = [](int i) { return 16 * (i >> 2) + (keys ? 0 : i & 3); };              // + row0
    auto channel = [](int i) { return keys ? 64 * ((i >> 1) & 1) + 8 * (i & 1) : 0; };   // + ch0
    if (rows >= kBlk && a.aligned[WHICH]) {
        const uint8_t* base = reinterpret_cast<const uint8_t*>(src);
        const uint32_t pitch = 2u * (uint32_t)st, mine = (uint32_t)row0 * pitch + 2u * (uint32_t)ch0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const u32x4 v = __builtin_nontemporal_load(
                reinterpret_cast<const u32x4*>(base + (mine + (uint32_t)row(i) * pitch + 2u * (uint32_t)channel(i))));
            x[i][0] = v[0];
            x[i][1] = v[1];
            x[i][2] = v[2];
            x[i][3] = v[3];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i][0] = x[i][1] = x[i][2] = x[i][3] = 0u;
            if (row0 + row(i) < rows) {
                const uint16_t* p = src + (row0 + row(i)) * st + ch0 + channel(i);
#pragma unroll
                for (int j = 0; j < 4; ++j) x[i][j] = (uint32_t)p[2 * j] | ((uint32_t)p[2 * j + 1] << 16);
            }
        }
    }
    // the largest magnitude: bf16 patterns without their signs order as integers
    auto largest = [&]() {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) m = pk_max(m, x[i][j] & 0x7FFF7FFFu);
        return wave_max((int)max(m & 0xFFFFu, m >> 16));
    };
    int top = largest();
    if (top >= 0x7F80) {         // infinities and NaN count as zeros
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) x[i][j] = finite_pair(x[i][j]);
        top = largest();
        if (lane == 0 && a.status) atomicOr(a.status, DQ_STATUS_RANGE);
    }
    const float amax = __uint_as_float((uint32_t)top << 16);
    const float s = amax < kTiny ? 0.f : amax / (FMT == DQ_Q8_E4M3 ? 448.f : 127.f);
    if (lane == 0) a.scale[WHICH][bi] = s;
    uint32_t code[8][2];
    if (s == 0.f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) code[i][0] = code[i][1] = 0u;
    } else {
        // x times the rounded reciprocal is within 2^-22 of the quotient: its code
        // is the quotient's unless a border is that near, which of the 512 values
        // at hand one is in 1 of 100 (e4m3) to 1 of 16 cases (int8).  Then
        // quotients of the block brought to magnitudes below 2 (exact powers of
        // 2; what underflows is 2^-149 of the largest value and rounds to 0)
        const float inv = 1.f / s;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float t[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                t[2 * j] = __uint_as_float(x[i][j] << 16) * inv;
                t[2 * j + 1] = __uint_as_float(x[i][j] & 0xFFFF0000u) * inv;
            }
            if (__builtin_amdgcn_ballot_w64(near_border<FMT>(t))) {
                const int e = max(-126, min(126, 127 - (top >> 7)));
                const float f = __uint_as_float((uint32_t)(e + 127) << 23);
                const float ss = s * f, exact_inv = 1.f / ss;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    t[2 * j] = quotient_odd(__uint_as_float(x[i][j] << 16) * f, ss, exact_inv);
                    t[2 * j + 1] = quotient_odd(__uint_as_float(x[i][j] & 0xFFFF0000u) * f, ss, exact_inv);
                }
            }
            const float lo[4] = {t[0], t[1], t[2], t[3]}, hi[4] = {t[4], t[5], t[6], t[7]};
            code[i][0] = codes4<FMT>(lo);
            code[i][1] = codes4<FMT>(hi);
        }
    }
    uint4* dst = reinterpret_cast<uint4*>(a.data[WHICH] + bi * kBlkBytes);
    if constexpr (keys) {
#pragma unroll
        for (int p = 0; p < 4; ++p)
            dst[64 * p + lane] = uint4{code[2 * p][0], code[2 * p][1], code[2 * p + 1][0], code[2 * p + 1][1]};
    } else {
        // o[x][h2]: channel 8 col + x of tokens 16 h2 + 4 grp + 0..3
        uint32_t o[8][2];
#pragma unroll
        for (int h2 = 0; h2 < 2; ++h2)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const uint32_t c0 = code[4 * h2][q], c1 = code[4 * h2 + 1][q], c2 = code[4 * h2 + 2][q],
                               c3 = code[4 * h2 + 3][q];
                // bytes k of c0..c3 -> one word, for k = 0..3
                const uint32_t a0 = __builtin_amdgcn_perm(c1, c0, 0x05010400u);   // c0.0 c1.0 c0.1 c1.1
                const uint32_t a1 = __builtin_amdgcn_perm(c3, c2, 0x05010400u);
                const uint32_t b0 = __builtin_amdgcn_perm(c1, c0, 0x07030602u);   // c0.2 c1.2 c0.3 c1.3
                const uint32_t b1 = __builtin_amdgcn_perm(c3, c2, 0x07030602u);
                o[4 * q + 0][h2] = __builtin_amdgcn_perm(a1, a0, 0x05040100u);
                o[4 * q + 1][h2] = __builtin_amdgcn_perm(a1, a0, 0x07060302u);
                o[4 * q + 2][h2] = __builtin_amdgcn_perm(b1, b0, 0x05040100u);
                o[4 * q + 3][h2] = __builtin_amdgcn_perm(b1, b0, 0x07060302u);
            }
        // col = 4 np + 2 n2 + half: pieces of channels 32 np + 8 half + x, this
        // lane's bytes 8 n2 ..; the lane with n2 = 0 writes x = 0..3, the other 4..7
        const int n2 = (col >> 1) & 1;
        const int p0 = ((col >> 2) * 4 + grp) * 16 + 8 * (col & 1) + 4 * n2;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t give0 = n2 ? o[k][0] : o[k + 4][0], give1 = n2 ? o[k][1] : o[k + 4][1];
            const uint32_t got0 = quad_xor2(give0), got1 = quad_xor2(give1);
            const uint32_t mine0 = n2 ? o[k + 4][0] : o[k][0], mine1 = n2 ? o[k + 4][1] : o[k][1];
            stage[staged(p0 + k)] = n2 ? uint4{got0, got1, mine0, mine1} : uint4{mine0, mine1, got0, got1};
        }
        wave_sync();
#pragma unroll
        for (int p = 0; p < 4; ++p) dst[64 * p + lane] = stage[staged(64 * p + lane)];
    }
}

template <int FMT>
__global__ __launch_bounds__(256) void q8_encode_kernel(EncArgs a) {
    __shared__ __align__(16) uint4 stage[4][256];
    const int lane = threadIdx.x & (kWave - 1), w = wave_index(4);
    if (w >= a.nblk * a.H) return;
    if (blockIdx.z == 0)
        encode_block<FMT, 0>(a, w, lane, stage[0]);
    else
        encode_block<FMT, 1>(a, w, lane, stage[threadIdx.x / kWave]);
}

// ---------------------------------------------------------------- read-back

struct ReadArgs {
    const uint8_t* data[2];
    const float* scale[2];
    uint16_t* out[2];
    int64_t sb[2], st[2], sh[2];
    uint32_t* status;
    Pages pg;
    int H, blk0, nblk, n, nb_cap;
    int aligned[2];
};

// Four code bytes to four floats.
template <int FMT>
__device__ __forceinline__ void floats4(uint32_t w, float (&f)[4]) {
    if constexpr (FMT == DQ_Q8_E4M3) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
        const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        f[0] = lo[0];
        f[1] = lo[1];
        f[2] = hi[0];
        f[3] = hi[1];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = (float)(int8_t)(w >> (8 * i));
    }
}

// fp32 to bf16, ties to even (finite values)
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
    uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
    x += 0x7FFFu + ((x >> 16) & 1u);
    y += 0x7FFFu + ((y >> 16) & 1u);
    return __builtin_amdgcn_perm(y, x, 0x07060302u);
}

template <int FMT, int WHICH>
__device__ __forceinline__ void read_block(const ReadArgs& a, int w, int lane, uint4* stage) {
    constexpr bool keys = WHICH == 0;
    const int h = w % a.H, blk = w / a.H, b = blockIdx.y;
    bool bad = false;
    const int64_t bi = block_index(a.pg, a.H, a.nb_cap, b, h, a.blk0 + blk, bad);
    if (bad && lane == 0 && a.status) atomicOr(a.status, DQ_STATUS_PAGE);
    const int rows = min(kBlk, a.n - blk * kBlk);
    const float s = a.scale[WHICH][bi];
    const u32x4* src = reinterpret_cast<const u32x4*>(a.data[WHICH] + bi * kBlkBytes);
    const int64_t st = a.st[WHICH];
    uint16_t* dst = a.out[WHICH] + (int64_t)b * a.sb[WHICH] + (int64_t)h * a.sh[WHICH] + (int64_t)blk * kBlk * st;
    const int col = lane & 15, grp = lane >> 4;
    uint32_t code[8][2];         // as in the encoder: 8 channels of one token per i
    u32x4 piece[4];
#pragma unroll
    for (int p = 0; p < 4; ++p)
        piece[p] = __builtin_nontemporal_load(src + 64 * p + lane);
    if constexpr (keys) {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            code[2 * p][0] = piece[p][0];
            code[2 * p][1] = piece[p][1];
            code[2 * p + 1][0] = piece[p][2];
            code[2 * p + 1][1] = piece[p][3];
        }
    } else {
        const int n2 = (col >> 1) & 1;
        const int p0 = ((col >> 2) * 4 + grp) * 16 + 8 * (col & 1) + 4 * n2;
#pragma unroll
        for (int p = 0; p < 4; ++p)
            stage[staged(64 * p + lane)] = uint4{piece[p][0], piece[p][1], piece[p][2], piece[p][3]};
        wave_sync();
        uint32_t o[8][2];
        uint4 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = stage[staged(p0 + k)];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t got0 = quad_xor2(n2 ? v[k].x : v[k].z), got1 = quad_xor2(n2 ? v[k].y : v[k].w);
            const uint32_t mine0 = n2 ? v[k].z : v[k].x, mine1 = n2 ? v[k].w : v[k].y;
            o[k][0] = n2 ? got0 : mine0;
            o[k][1] = n2 ? got1 : mine1;
            o[k + 4][0] = n2 ? mine0 : got0;
            o[k + 4][1] = n2 ? mine1 : got1;
        }
#pragma unroll
        for (int h2 = 0; h2 < 2; ++h2)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const uint32_t c0 = o[4 * q][h2], c1 = o[4 * q + 1][h2], c2 = o[4 * q + 2][h2], c3 = o[4 * q + 3][h2];
                const uint32_t a0 = __builtin_amdgcn_perm(c1, c0, 0x05010400u);
                const uint32_t a1 = __builtin_amdgcn_perm(c3, c2, 0x05010400u);
                const uint32_t b0 = __builtin_amdgcn_perm(c1, c0, 0x07030602u);
                const uint32_t b1 = __builtin_amdgcn_perm(c3, c2, 0x07030602u);
                code[4 * h2 + 0][q] = __builtin_amdgcn_perm(a1, a0, 0x05040100u);
                code[4 * h2 + 1][q] = __builtin_amdgcn_perm(a1, a0, 0x07060302u);
                code[4 * h2 + 2][q] = __builtin_amdgcn_perm(b1, b0, 0x05040100u);
                code[4 * h2 + 3][q] = __builtin_amdgcn_perm(b1, b0, 0x07060302u);
            }
    }
    const int row0 = keys ? col : 4 * grp;
    const int ch0 = keys ? 16 * grp : 8 * col;
    const uint32_t pitch = 2u * (uint32_t)st, mine = (uint32_t)row0 * pitch + 2u * (uint32_t)ch0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int row = 16 * (i >> 2) + (keys ? 0 : i & 3);                  // + row0
        const int channel = keys ? 64 * ((i >> 1) & 1) + 8 * (i & 1) : 0;    // + ch0
        float f[4], g[4];
        floats4<FMT>(code[i][0], f);
        floats4<FMT>(code[i][1], g);
        const uint4 v = {bf16_pair(f[0] * s, f[1] * s), bf16_pair(f[2] * s, f[3] * s),
                         bf16_pair(g[0] * s, g[1] * s), bf16_pair(g[2] * s, g[3] * s)};
        if (row0 + row < rows) {
            if (a.aligned[WHICH]) {
                uint8_t* p = reinterpret_cast<uint8_t*>(dst) + (mine + (uint32_t)row * pitch + 2u * (uint32_t)channel);
                *reinterpret_cast<uint4*>(p) = v;
            } else {
                uint16_t* p = dst + (row0 + row) * st + ch0 + channel;
                const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    p[2 * j] = (uint16_t)u[j];
                    p[2 * j + 1] = (uint16_t)(u[j] >> 16);
                }
            }
        }
    }
}

template <int FMT>
__global__ __launch_bounds__(256) void q8_read_kernel(ReadArgs a) {
    __shared__ __align__(16) uint4 stage[4][256];
    const int lane = threadIdx.x & (kWave - 1), w = wave_index(4);
    if (w >= a.nblk * a.H) return;
    if (blockIdx.z == 0)
        read_block<FMT, 0>(a, w, lane, stage[0]);
    else
        read_block<FMT, 1>(a, w, lane, stage[threadIdx.x / kWave]);
}

// ---------------------------------------------------------------- attention

// Visible blocks of a sequence: the first `head` ones, then those from `from`
// on; token t of them is visible if it is below the length and either below
// `sinks` or at least `start`.
struct Visible {
    int T, sinks, start, head, from, count;
};

__device__ __forceinline__ Visible visible(int T, int extra, int window, int sinks) {
    Visible v;
    v.T = T;
    const int nb = (T + kBlk - 1) / kBlk;
    if (window <= 0) {
        v.sinks = 0;
        v.start = 0;
        v.head = 0;
        v.from = 0;
    } else {
        v.sinks = min(sinks, T);
        const int64_t start = (int64_t)T + extra - window;
        v.start = (int)max((int64_t)0, min(start, (int64_t)T));
        v.head = (v.sinks + kBlk - 1) / kBlk;
        // a block that the first tokens and the window share is listed once
        v.from = max(v.head, v.start == T ? nb : v.start / kBlk);
    }
    v.count = v.head + max(0, nb - v.from);
    return v;
}

struct Q8Args {
    const uint16_t* q;
    const uint8_t* k;
    const float* ks;
    const uint8_t* v;
    const float* vs;
    const int32_t* seq_lens;
    const int32_t* extra_lens;   // tokens behind the cached ones, or NULL
    Pages pg;
    int Hq, Hkv, G, t_cap, window, sinks;
    int chunk, nchunks;          // blocks per chunk, chunk slots per sequence
    int B, target;               // target > 0: the chunk length follows the lengths
    int items;                   // most chunks per KV head
    float per_cu;                // just below 1 / CUs
    float scale_log2;
    float* lse;                  // [B][Hkv][t_cap / 32][G], or NULL
    float* lse_rest;             // with lse, of the same shape: what its rounding left
    float* out;                  // one chunk: the step's result goes here, or NULL
    float* scores;               // with out
    int early;                   // blocks are requested before the length is known
    uint32_t* status;
    int32_t* ws_hdr;
    float* ws_m;
    float* ws_l;
    float* ws_acc;
};

constexpr int kAWaves = 8;                   // wavefronts per workgroup (4 for short sequences)
constexpr int kGP = 8;                       // query-head slots
constexpr int kChunkCost = 8;                // what a chunk costs besides its blocks, in blocks
constexpr float kBig = 3e38f;

typedef const __attribute__((address_space(1))) uint8_t* GlobalBytes;

// Nontemporal: a step reads every block once, and lines that do not settle in
// L2 stream at 6.7 TB/s where they reached 5.8 (16 x 32768 tokens: 159 us
// against 189; one sequence of 32768 16.7 against 19.8, one of 4096, which
// would fit: no difference).
__device__ __forceinline__ uint4 load16(GlobalBytes p) {
    const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const __attribute__((address_space(1))) u32x4*>(p));
    return uint4{v[0], v[1], v[2], v[3]};
}

// Eight code bytes to eight fp16 values (exact for both types).
template <int FMT>
__device__ __forceinline__ f16x8 halves8(uint32_t lo, uint32_t hi) {
    f16x2 h[4];
    if constexpr (FMT == DQ_Q8_E4M3) {
        h[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, 1.f, false);
        h[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, 1.f, true);
        h[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, 1.f, false);
        h[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, 1.f, true);
    } else {
        // byte + 128 as the low bits of an fp16 in [1024, 2048), less 1152
        const uint32_t magic = 0x64646464u;
        const f16x2 off = {(_Float16)1152.f, (_Float16)1152.f};
        lo ^= 0x80808080u;
        hi ^= 0x80808080u;
        h[0] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(magic, lo, 0x04010400u)) - off;
        h[1] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(magic, lo, 0x04030402u)) - off;
        h[2] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(magic, hi, 0x04010400u)) - off;
        h[3] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(magic, hi, 0x04030402u)) - off;
    }
    f16x8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r[2 * i] = h[i][0];
        r[2 * i + 1] = h[i][1];
    }
    return r;
}

__device__ __forceinline__ f32x4 mfma_f16(const f16x8& a, const f16x8& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ float clamp_big(float x) { return __builtin_amdgcn_fmed3f(x, -kBig, kBig); }

// A uniform address of memory that this kernel does not write, through the
// scalar unit: what arrives there keeps out of the vector loads' order, so no
// wait for it waits for a prefetched block.
template <typename T>
__device__ __forceinline__ T scalar_load(const T* p) {
    return *reinterpret_cast<const __attribute__((address_space(4))) T*>(reinterpret_cast<uintptr_t>(p));
}

// What workgroup `id` works on, where the chunk length follows the sequences'
// lengths: all blocks there are, cut into about `target` equal chunks (at most
// `nchunks` in the longest sequence), sequence after sequence, head after head.
// A batch of unlike lengths then ends much as one of like lengths does, and a
// buffer's unused capacity costs nothing (chunks cut from the capacity alone:
// 4096 tokens in a buffer of 131072 28.7 us against 10.3; 16 sequences, one of
// 131072 and fifteen of 2000 tokens, 134 against 60).
struct Share {
    int b, h, c, chunk;          // c = -1: nothing
};

__device__ __forceinline__ int wave_scan(int v) {      // inclusive sums over the lanes
    v += dpp0<0x111, 0xF>(v);    // row_shr:1
    v += dpp0<0x112, 0xF>(v);    // row_shr:2
    v += dpp0<0x114, 0xF>(v);    // row_shr:4
    v += dpp0<0x118, 0xF>(v);    // row_shr:8
    v += dpp0<0x142, 0xA>(v);    // row_bcast:15 into rows 1 and 3
    v += dpp0<0x143, 0xC>(v);    // row_bcast:31 into rows 2 and 3
    return v;
}

__device__ __forceinline__ Share share_of(const Q8Args& a, int id, int lane) {
    auto blocks = [&](int T) { return (max(0, min(T, a.t_cap)) + kBlk - 1) / kBlk; };
    auto length = [&](int total, int longest) {
        if (total < longest * a.B / 4 * 3) {
            // unlike lengths leave many last chunks that are not full: six per CU,
            // but of two blocks per wavefront or more where one per CU has them
            const int c = (total + a.target - 1) / a.target;
            const int fine = max(max(min(c, 2 * kAWaves), (c + 5) / 6), (longest + a.nchunks - 1) / a.nchunks);
            return max((fine + 3) & ~3, 4);
        }
        // lane l tries (l + 1) step chunks per sequence: the blocks that the
        // busiest CU then takes
        const int step = (a.nchunks + 63) / 64, cuts = (lane + 1) * step;
        const int c = max(((uint32_t)(longest + cuts - 1) / (uint32_t)cuts + 3) & ~3u, 4u);
        const int n = (uint32_t)(longest + c - 1) / (uint32_t)c;
        // (items Hkv is at most 6 CUs + B Hkv)
        float cost = 3e8f;
        if (cuts <= a.nchunks && n * a.B <= a.items)
            cost = ceilf((float)(n * a.B * a.Hkv) * a.per_cu) * (float)(c + kChunkCost);
        const float least = wave_min(cost);
        const int best = __builtin_ctzll(__builtin_amdgcn_ballot_w64(cost == least));
        return __builtin_amdgcn_readlane(c, best);
    };
    if (a.B == 1) {
        const int n = blocks(scalar_load(a.seq_lens)), chunk = length(n, n), used = (n + chunk - 1) / chunk;
        if (id >= used * a.Hkv) return Share{0, 0, -1, chunk};
        return Share{0, id / used, id % used, chunk};
    }
    int total = 0, longest = 0;
    int mine = 0;                // blocks of sequence `lane` of the group at hand
    auto read = [&](int b0) { mine = b0 + lane < a.B ? blocks(a.seq_lens[b0 + lane]) : 0; };
    for (int b0 = 0; b0 < a.B; b0 += kWave) {
        read(b0);
        total += wave_sum(mine);
        longest = max(longest, wave_max(mine));
    }
    const int chunk = length(total, longest);
    // the full chunks, then the sequences' last ones that are not: short work
    // comes last and evens out the end
    for (int pass = 0; pass < 2; ++pass) {
        int before = 0;          // chunks of one head of the sequences before the group
        for (int b0 = 0; b0 < a.B; b0 += kWave) {
            if (a.B > kWave) read(b0);
            const int full = mine / chunk, own = pass == 0 ? full : (int)(mine > full * chunk);
            const int upto = before + wave_scan(own);
            const int all = __builtin_amdgcn_readlane(upto, 63);
            if (id < all * a.Hkv) {
                // the first sequence whose chunks, of all heads, reach past id
                const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto * a.Hkv > id));
                const int r = id - __builtin_amdgcn_readlane(upto - own, l) * a.Hkv;
                const int n = __builtin_amdgcn_readlane(own, l);
                return Share{b0 + l, r / n, pass == 0 ? r % n : __builtin_amdgcn_readlane(full, l), chunk};
            }
            before = all;
        }
        id -= before * a.Hkv;
    }
    return Share{0, 0, -1, chunk};
}

// One workgroup of eight (or four) wavefronts per (chunk of visible blocks, KV
// head, sequence); a wavefront takes every eighth block of the chunk and requests
// the next one's 8 KB before it works on the one at hand.
//   Scores: S^T (16 tokens x 16 columns) = K (16 x 128) Q^T on
//   v_mfma_f32_16x16x32_f16.  Codes are exact in fp16, and so are the query's
//   bf16 values once its largest is brought to 2^14 (its smaller ones down to
//   2^-28 of it, the rest to 2^-39 of it).  Columns g and g + 8 both hold query
//   head g.  Lane (grp, col) then has head col % 8 for tokens 16 h2 + 4 grp + i.
//   Softmax online, in fp32 and base 2; the maximum is exchanged between the
//   lanes of a head only when some lane exceeds it.
//   Values: weights p 2^15 are split into two fp16 terms (22 bits, down to
//   weights of 2^-18 of the largest), the first in the rows of heads 0..7, the
//   second in rows 8..15: one product of the 32 tokens gives both, its operand
//   the weights as they lie.  The block's scale is applied to the
//   product's fp32 result.
template <int FMT, bool TRACK, int WAVES>
__global__ __launch_bounds__(WAVES* kWave, 4) void q8_partial_kernel(Q8Args a) {
    __shared__ float wm[WAVES][kGP], wl[WAVES][kGP];
    __shared__ __align__(16) float wacc[WAVES][kGP][kD];
    int c = blockIdx.x, h = blockIdx.y, b = blockIdx.z, chunk = a.chunk;
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int G = a.G, NC = a.nchunks, nb_cap = a.t_cap / kBlk;
    const int col = lane & 15, grp = lane >> 4, head = col & 7;
    const bool first = (blockIdx.x | blockIdx.y | blockIdx.z) == 0 && tid == 0;
    if (a.target > 0) {
        const Share w = share_of(a, (int)blockIdx.x, lane);
        h = w.h;
        c = w.c;
        b = w.b;
        chunk = w.chunk;
        if (first) a.ws_hdr[0] = chunk * kBlk;
    } else if (first) {
        // a windowed step fills every chunk's slot, for whatever length: the
        // merge takes min(chunks, ceil(T / 1)) of them, and chunk c >= T is empty
        a.ws_hdr[0] = a.window > 0 ? 1 : chunk * kBlk;
    }
    if (first) {
        a.ws_hdr[1] = NC;
        a.ws_hdr[2] = 0;
        a.ws_hdr[3] = 0;          // values are in the caller's basis
    }
    // (uniform, which the compiler does not see)
    c = __builtin_amdgcn_readfirstlane(c);
    h = __builtin_amdgcn_readfirstlane(h);
    b = __builtin_amdgcn_readfirstlane(b);
    chunk = __builtin_amdgcn_readfirstlane(chunk);
    if (c < 0) return;            // more workgroups than chunks
    const int v0 = c * chunk;

    bool bad = false;
    uint4 kr[4], vr[4];
    float ks_next = 0.f, vs_next = 0.f;
    // where block `blk` lies: its pool page is looked up an iteration before it
    // is needed
    int page = 0;
    int64_t bi = 0;
    auto look_up = [&](int blk) {
        if (a.pg.bt) page = scalar_load(a.pg.bt + (int64_t)b * a.pg.max_pages + ((blk * kBlk) >> a.pg.page_shift));
    };
    auto locate = [&](int blk) {
        if (!a.pg.bt) {
            bi = ((int64_t)b * a.Hkv + h) * nb_cap + blk;
            return;
        }
        if (page < 0 || page >= a.pg.num_pages) {
            bad = true;
            page = 0;
        }
        const int bpp = 1 << (a.pg.page_shift - 5);
        bi = ((int64_t)page * a.Hkv + h) * bpp + (blk & (bpp - 1));
    };
    // (the empty statement keeps the block's address in scalar registers: one
    // vector register, the lane's offset, then serves every load)
    auto request_k = [&]() {
        GlobalBytes p = reinterpret_cast<GlobalBytes>(reinterpret_cast<uintptr_t>(a.k + bi * kBlkBytes));
        asm("" : "+s"(p));
#pragma unroll
        for (int i = 0; i < 4; ++i) kr[i] = load16(p + 16u * lane + 1024u * i);
        ks_next = scalar_load(a.ks + bi);
        vs_next = scalar_load(a.vs + bi);
    };
    auto request_v = [&]() {
        GlobalBytes p = reinterpret_cast<GlobalBytes>(reinterpret_cast<uintptr_t>(a.v + bi * kBlkBytes));
        asm("" : "+s"(p));
#pragma unroll
        for (int i = 0; i < 4; ++i) vr[i] = load16(p + 16u * lane + 1024u * i);
    };
    const int T_raw = scalar_load(a.seq_lens + b);
    const int extra = a.extra_lens ? max(0, scalar_load(a.extra_lens + b)) : 0;
    // the query: channels 64 (i / 2) + 16 grp + 8 (i % 2) .. of the lane's head
    uint4 raw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        raw[i] = uint4{0u, 0u, 0u, 0u};
        if (head < G)
            raw[i] = *reinterpret_cast<const uint4*>(a.q + ((int64_t)b * a.Hq + h * G + head) * kD + 64 * (i >> 1) +
                                                     16 * grp + 8 * (i & 1));
    }
    if (a.early) {
        locate(min(v0 + wave, nb_cap - 1));
        request_k();
        request_v();
    }
    const int T = max(0, min(T_raw, a.t_cap));
    const Visible vis = visible(T, extra, a.window, a.sinks);
    const int v1 = min(v0 + chunk, vis.count);
    const int64_t slot0 = ((int64_t)b * a.Hq + h * G) * (NC + kResSlots) + c;
    if (v0 >= v1) {
        if (a.out) {
            for (int i = tid; i < G * kD; i += WAVES * kWave) a.out[((int64_t)b * a.Hq + h * G) * kD + i] = 0.f;
        } else if (a.window > 0) {
            for (int i = tid; i < G * kD; i += WAVES * kWave) {
                const int64_t slot = slot0 + (int64_t)(i / kD) * (NC + kResSlots);
                a.ws_acc[slot * kD + i % kD] = 0.f;
                if (i % kD == 0) {
                    a.ws_m[slot] = -INFINITY;
                    a.ws_l[slot] = 0.f;
                }
            }
        }
        return;                   // without a window the merge ignores the chunk
    }

    // ---- the query, scaled to fp16, in the columns of its head
    f16x8 qb[4];
    float c_head;
    bool bad_q;
    {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            top = pk_max(top, pk_max(pk_max(raw[i].x & 0x7FFF7FFFu, raw[i].y & 0x7FFF7FFFu),
                                     pk_max(raw[i].z & 0x7FFF7FFFu, raw[i].w & 0x7FFF7FFFu)));
        // patterns without their signs order as integers, and as small floats
        float m = (float)max(top & 0xFFFFu, top >> 16);
        m = fmaxf(m, xor_lane<16>(m, lane));
        m = fmaxf(m, xor_lane<32>(m, lane));
        bad_q = m >= 32640.f;     // 0x7F80: an infinity or NaN
        const int up = bad_q ? 0 : 14 - (max((int)m >> 7, 1) - 127);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float lo = __uint_as_float(w[e] << 16), hi = __uint_as_float(w[e] & 0xFFFF0000u);
                qb[i][2 * e] = bad_q ? (_Float16)0.f : (_Float16)__builtin_ldexpf(lo, up);
                qb[i][2 * e + 1] = bad_q ? (_Float16)0.f : (_Float16)__builtin_ldexpf(hi, up);
            }
        }
        c_head = __builtin_ldexpf(a.scale_log2, -up);
    }

    float m_run = -3.4e38f, l_run = 0.f;
    f32x4 acc[8];
#pragma unroll
    for (int n = 0; n < 8; ++n) acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};

    auto block_of = [&](int v) { return v < vis.head ? v : vis.from + v - vis.head; };
    int v = v0 + wave;
    if (v < v1) {
        if (!a.early) {
            look_up(block_of(v));
            locate(block_of(v));
            request_k();
            request_v();
        }
        if (v + WAVES < v1) look_up(block_of(v + WAVES));
    }
    // One block; the next one is requested on the way (its keys once these have
    // become scores, its values once these are added) or there is none.  Two
    // copies: a request under a branch would make every wait one for all loads.
    auto step = [&](auto more) {
        const int blk = block_of(v), t0 = blk * kBlk;
        const int vn = v + WAVES;
        const float ks = ks_next, vs = vs_next;

        // ---- scores in base 2
        float x[8];
        const float cf = clamp_big(ks * c_head);
#pragma unroll
        for (int h2 = 0; h2 < 2; ++h2) {
            f32x4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint4 w = kr[2 * h2 + j];
                d = mfma_f16(halves8<FMT>(w.x, w.y), qb[2 * j], d);
                d = mfma_f16(halves8<FMT>(w.z, w.w), qb[2 * j + 1], d);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) x[4 * h2 + i] = clamp_big(d[i] * cf);
        }
        if constexpr (decltype(more)::value) {
            locate(block_of(vn));
            request_k();
            if (vn + WAVES < v1) look_up(block_of(vn + WAVES));
        }
        const bool whole = t0 + kBlk <= T && (t0 >= vis.start || t0 + kBlk <= vis.sinks);
        if (!whole) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int t = t0 + 16 * (e >> 2) + 4 * grp + (e & 3);
                if (!(t < T && (t >= vis.start || t < vis.sinks))) x[e] = -INFINITY;
            }
            // rows past the length may hold anything: no code stays
            uint32_t keep[2] = {0u, 0u};
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (t0 + 16 * (e >> 2) + 4 * grp + (e & 3) < T) keep[e >> 2] |= 0xFFu << (8 * (e & 3));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                vr[i].x &= keep[0];
                vr[i].y &= keep[1];
                vr[i].z &= keep[0];
                vr[i].w &= keep[1];
            }
        }

        // ---- online softmax of head col % 8
        float mt = x[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) mt = fmaxf(mt, x[e]);
        if (__builtin_amdgcn_ballot_w64(mt > m_run)) {
            mt = fmaxf(mt, xor_lane<16>(mt, lane));
            mt = fmaxf(mt, xor_lane<32>(mt, lane));
            const float mn = fmaxf(m_run, mt);
            const float corr = __builtin_amdgcn_exp2f(m_run - mn);
            m_run = mn;
            l_run *= corr;
            float cr[4];          // of the accumulators' rows: head (4 grp + i) % 8
#pragma unroll
            for (int i = 0; i < 4; ++i) cr[i] = __shfl(corr, (4 * grp + i) & 7);
#pragma unroll
            for (int n = 0; n < 8; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[n][i] *= cr[i];
        }
        // the second term of a weight below 2^-18 of the largest is a subnormal
        // fp16, 2^-40 of the largest off at most
        float ps = 0.f;
        uint32_t w2[4];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const f32x2 p = {__builtin_amdgcn_exp2f(x[e] - m_run), __builtin_amdgcn_exp2f(x[e + 1] - m_run)};
            ps += p[0];
            ps += p[1];
            const f32x2 f = {p[0] * 0x1p15f, p[1] * 0x1p15f};
            const f16x2 hi = __builtin_convertvector(f, f16x2);
            const f32x2 r = {f[0] - (float)hi[0], f[1] - (float)hi[1]};
            const f16x2 lo = __builtin_convertvector(r, f16x2);
            w2[e / 2] = __builtin_bit_cast(uint32_t, col < 8 ? hi : lo);
        }
        const f16x8 w = __builtin_bit_cast(f16x8, uint4{w2[0], w2[1], w2[2], w2[3]});
        l_run += ps;
        if constexpr (TRACK) {
            float bs = ps + xor_lane<16>(ps, lane);
            bs += xor_lane<32>(bs, lane);
            // the maximum and the logarithm as a rounded sum and what the rounding left,
            // which is the block's weight where the maximum is large (Knuth's two-sum)
            if (lane < G) {
                const int64_t i = (((int64_t)b * a.Hkv + h) * nb_cap + blk) * G + lane;
                const float lg = log2f(bs), sum = m_run + lg, of_lg = sum - m_run;
                a.lse[i] = sum;
                a.lse_rest[i] = bs == 0.f ? 0.f : (m_run - (sum - of_lg)) + (lg - of_lg);
            }
        }

        // ---- weighted values
        const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
        const float vsc = vs * 0x1p-15f;
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const f32x4 d0 = mfma_f16(w, halves8<FMT>(vr[n].x, vr[n].y), zero);
            const f32x4 d1 = mfma_f16(w, halves8<FMT>(vr[n].z, vr[n].w), zero);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                acc[2 * n][i] = fmaf(d0[i], vsc, acc[2 * n][i]);
                acc[2 * n + 1][i] = fmaf(d1[i], vsc, acc[2 * n + 1][i]);
            }
            // here, not behind the next request: few products' results at a time
            asm("" : "+v"(acc[2 * n]), "+v"(acc[2 * n + 1]));
        }
        if constexpr (decltype(more)::value) request_v();
    };
    if (v < v1) {
        for (; v + WAVES < v1; v += WAVES) step(std::true_type{});
        step(std::false_type{});
    }
    if (bad && lane == 0 && a.status) atomicOr(a.status, DQ_STATUS_PAGE);

    // ---- the two terms of a weight, then the wavefronts
    l_run += xor_lane<16>(l_run, lane);
    l_run += xor_lane<32>(l_run, lane);
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float lo = xor_lane<32>(acc[n][i], lane);
            if (grp < 2) wacc[wave][4 * grp + i][16 * n + col] = acc[n][i] + lo;
        }
    if (lane < kGP) {
        wm[wave][lane] = m_run;
        wl[wave][lane] = bad_q ? NAN : l_run;
    }
    __syncthreads();
    for (int i = tid; i < G * kD; i += WAVES * kWave) {
        const int g = i / kD, j = i % kD;
        float M = wm[0][g];
#pragma unroll
        for (int u = 1; u < WAVES; ++u) M = fmaxf(M, wm[u][g]);
        float s = 0.f, l = 0.f;
#pragma unroll
        for (int u = 0; u < WAVES; ++u) {
            const float e = exp2f(wm[u][g] - M);
            s = fmaf(wacc[u][g][j], e, s);
            l = fmaf(wl[u][g], e, l);
        }
        if (a.out) {
            a.out[((int64_t)b * a.Hq + h * G + g) * kD + j] = l == 0.f ? 0.f : s / l;
            continue;
        }
        const int64_t slot = slot0 + (int64_t)g * (NC + kResSlots);
        a.ws_acc[slot * kD + j] = s;
        if (j == 0) {
            a.ws_m[slot] = l == 0.f ? -INFINITY : M;
            a.ws_l[slot] = l;
        }
    }
    if constexpr (TRACK) {
        if (!a.scores) return;
        // the whole step is here: every block's weight (the barrier above orders
        // the wavefronts' writes of lse and lse_rest)
        float top[kGP], total[kGP];
#pragma unroll
        for (int g = 0; g < kGP; ++g) {
            float M = wm[0][g], l = 0.f;
#pragma unroll
            for (int u = 1; u < WAVES; ++u) M = fmaxf(M, wm[u][g]);
#pragma unroll
            for (int u = 0; u < WAVES; ++u) l = fmaf(wl[u][g], exp2f(wm[u][g] - M), l);
            top[g] = l == 0.f ? INFINITY : M;
            total[g] = log2f(l == 0.f ? 1.f : l);
        }
        for (int u = tid; u < vis.count; u += WAVES * kWave) {
            const int64_t i = ((int64_t)b * a.Hkv + h) * nb_cap + block_of(u);
            float w = 0.f;
#pragma unroll
            for (int g = 0; g < kGP; ++g)
                if (g < G) w += exp2f((a.lse[i * G + g] - top[g]) + (a.lse_rest[i * G + g] - total[g]));
            a.scores[i] += w;
        }
    }
}

// ----------------------------------------------------- merge and the scores

struct FinishArgs {
    const int32_t* seq_lens;
    const int32_t* extra_lens;
    const float* lse;
    const float* lse_rest;
    const int32_t* ws_hdr;
    const float* ws_m;
    const float* ws_l;
    const float* ws_acc;
    float* out;                  // [B][Hq][128], or NULL
    float* scores;               // [B][Hkv][t_cap / 32], or NULL
    int Hq, Hkv, G, t_cap, window, sinks, nc_max;
    int nc;                      // chunk slots per sequence, 0: as the workspace says
    int heads;                   // workgroups per KV head that merge: G or 0
};

constexpr int kScoreBlocks = 128;            // blocks per wavefront of the scores
constexpr int kFinishFirst = 8;              // partials per wavefront requested at once
constexpr int kFinishBatch = 16;             // partials per further memory round trip
// Up to so many merges have four wavefronts each, others one (four: 8 KV heads of
// one sequence of 4096 tokens 9.0 us the step against 10.7, one KV head of 120000
// tokens, whose partials are over two hundred, 16 against 39; one: 32 heads of 48
// sequences of up to 8192 tokens 94 against 99 us, most of whose requests find no
// partial).
constexpr int kFewMerges = 128;
constexpr int kMostChunks = 4 * kWave;       // (one wavefront has at most 32: many pairs)

// The first G workgroups of a (KV head, sequence) merge one query head each:
// wavefront w of W takes the partials w, w + W, ..., lane l the maximum and sum
// of the l-th of them and of all the channels 2 l and 2 l + 1; the wavefronts'
// results meet in LDS.  The others' wavefronts add block weights to the
// scores: sum_g 2^(lse of the block - lse of the step), the latter from the
// partials' maxima and sums (as many partials as lanes or fewer, in general).
// Both logarithms come in two parts, a large and a small one, and the large
// ones are subtracted first: exact where a weight counts, however large the scores.
template <int WAVES>
__global__ __launch_bounds__(WAVES* kWave) void q8_finish_kernel(FinishArgs a) {
    __shared__ float wm[WAVES], wl[WAVES];
    __shared__ float2 wacc[WAVES][kWave];
    const int h = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & (kWave - 1), G = a.G;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    // (the stores of this kernel are to other memory than these loads)
    const int NC = a.nc ? a.nc : min(max(scalar_load(a.ws_hdr + 1), 1), a.nc_max);
    const int64_t base = ((int64_t)b * a.Hq + h * G) * (NC + kResSlots);
    // a merging wavefront requests its first partials before it knows how many there are
    float2 x[kFinishBatch];
    float m_lane = 0.f, l_lane = 0.f;
    const bool merge = (int)blockIdx.x < a.heads;
    const int64_t s0 = base + (int64_t)blockIdx.x * (NC + kResSlots);
    auto partial = [&](int u, int last) {
        const int64_t slot = s0 + min(wave + WAVES * u, last);
        return *(reinterpret_cast<const float2*>(a.ws_acc + slot * kD) + lane);
    };
    // a residual window's partials, these many per wavefront
    constexpr int kRes = kResSlots / WAVES;
    float rm[kRes], rl[kRes];
    float2 rx[kRes];
    if (merge) {
        const int64_t s1 = s0 + min(wave + WAVES * lane, NC - 1);
        m_lane = a.ws_m[s1];
        l_lane = a.ws_l[s1];
#pragma unroll
        for (int u = 0; u < kFinishFirst; ++u) x[u] = partial(u, NC - 1);
        if (a.nc == 0) {
#pragma unroll
            for (int r = 0; r < kRes; ++r) {
                const int64_t slot = s0 + NC + wave * kRes + r;
                rm[r] = a.ws_m[slot];
                rl[r] = a.ws_l[slot];
                rx[r] = *(reinterpret_cast<const float2*>(a.ws_acc + slot * kD) + lane);
            }
        }
    }
    const int chunk = max(scalar_load(a.ws_hdr), 1);
    const int residual = a.nc ? 0 : min(max(scalar_load(a.ws_hdr + 2), 0), kResSlots);
    const int T = max(0, min(scalar_load(a.seq_lens + b), a.t_cap));
    const int nc = (int)min((int64_t)NC, ((int64_t)T + chunk - 1) / chunk), np = nc + residual;
    if (merge) {
        // partials 0 .. nc - 1, at most kMostChunks, and the residual window's
        const int n = max(0, nc - wave + WAVES - 1) / WAVES;
        if (lane >= n) m_lane = -INFINITY;
        float M = wave_max(m_lane);
#pragma unroll
        for (int r = 0; r < kRes; ++r) {
            if (wave * kRes + r >= residual) rm[r] = -INFINITY;
            M = fmaxf(M, rm[r]);
        }
        // (a partial without weight, or none: 0, whatever its slot holds)
        const float e_lane = m_lane == -INFINITY ? 0.f : exp2f(m_lane - M);
        float l = wave_sum(m_lane == -INFINITY ? 0.f : l_lane * e_lane);
        float2 acc = {0.f, 0.f};
#pragma unroll
        for (int r = 0; r < kRes; ++r) {
            if (rm[r] != -INFINITY) {
                const float e = exp2f(rm[r] - M);
                l = fmaf(rl[r], e, l);
                acc.x = fmaf(rx[r].x, e, acc.x);
                acc.y = fmaf(rx[r].y, e, acc.y);
            }
        }
        auto add = [&](int u0, int most) {
#pragma unroll
            for (int u = 0; u < kFinishBatch; ++u) {
                if (u < most && u0 + u < n) {
                    const float e = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(e_lane), u0 + u));
                    acc.x = fmaf(x[u].x, e, acc.x);
                    acc.y = fmaf(x[u].y, e, acc.y);
                }
            }
        };
        add(0, kFinishFirst);
        for (int u0 = kFinishFirst; u0 < n; u0 += kFinishBatch) {
#pragma unroll
            for (int u = 0; u < kFinishBatch; ++u) x[u] = partial(u0 + u, nc - 1);
            add(u0, kFinishBatch);
        }
        wacc[wave][lane] = acc;
        if (lane == 0) {
            wm[wave] = M;
            wl[wave] = l;
        }
        __syncthreads();
        if (wave > 0) return;
        float top = wm[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) top = fmaxf(top, wm[w]);
        float2 out = {0.f, 0.f};
        if (top != -INFINITY) {
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float e = exp2f(wm[w] - top);
                sum = fmaf(wl[w], e, sum);
                out.x = fmaf(wacc[w][lane].x, e, out.x);
                out.y = fmaf(wacc[w][lane].y, e, out.y);
            }
            out.x /= sum;
            out.y /= sum;
        }
        *(reinterpret_cast<float2*>(a.out + ((int64_t)b * a.Hq + h * G + (int)blockIdx.x) * kD) + lane) = out;
        return;
    }
    auto slot_of = [&](int g, int i) { return base + (int64_t)g * (NC + kResSlots) + (i < nc ? i : NC + i - nc); };
    const int extra = a.extra_lens ? max(0, scalar_load(a.extra_lens + b)) : 0;
    const Visible vis = visible(T, extra, a.window, a.sinks);
    const int first = (((int)blockIdx.x - a.heads) * WAVES + wave) * kScoreBlocks;
    if (first >= vis.count) return;
    // the blocks' terms are requested beside the partials' maxima and sums
    float term[kScoreBlocks / kWave][kGP], rest[kScoreBlocks / kWave][kGP], score[kScoreBlocks / kWave];
    int64_t at[kScoreBlocks / kWave];
#pragma unroll
    for (int r = 0; r < kScoreBlocks / kWave; ++r) {
        const int v = min(first + r * kWave + lane, vis.count - 1);
        at[r] = ((int64_t)b * a.Hkv + h) * (a.t_cap / kBlk) + (v < vis.head ? v : vis.from + v - vis.head);
        score[r] = a.scores[at[r]];
#pragma unroll
        for (int g = 0; g < kGP; ++g) {
            term[r][g] = a.lse[at[r] * G + min(g, G - 1)];
            rest[r][g] = a.lse_rest[at[r] * G + min(g, G - 1)];
        }
    }
    float m[kGP], l[kGP], top[kGP], total[kGP];
#pragma unroll
    for (int g = 0; g < kGP; ++g) {
        const bool in = g < G && lane < np;
        const int64_t s = slot_of(min(g, G - 1), min(lane, max(np - 1, 0)));
        m[g] = in ? a.ws_m[s] : -INFINITY;
        l[g] = in ? a.ws_l[s] : 0.f;
    }
#pragma unroll
    for (int g = 0; g < kGP; ++g) {
        top[g] = INFINITY;
        total[g] = 0.f;
        if (g < G) {
            float M = m[g];
            for (int i = lane + kWave; i < np; i += kWave) M = fmaxf(M, a.ws_m[slot_of(g, i)]);
            M = wave_max(M);
            if (M != -INFINITY) {
                float sum = l[g] * exp2f(m[g] - M);
                for (int i = lane + kWave; i < np; i += kWave)
                    sum += a.ws_l[slot_of(g, i)] * exp2f(a.ws_m[slot_of(g, i)] - M);
                top[g] = M;
                total[g] = log2f(wave_sum(sum));
            }
        }
    }
#pragma unroll
    for (int r = 0; r < kScoreBlocks / kWave; ++r) {
        float w = 0.f;
#pragma unroll
        for (int g = 0; g < kGP; ++g)
            if (g < G) w += exp2f((term[r][g] - top[g]) + (rest[r][g] - total[g]));
        if (first + r * kWave + lane < vis.count) a.scores[at[r]] = score[r] + w;
    }
}

// ----------------------------------------------------------------- eviction

struct EvictArgs {
    const int32_t* seq_lens;
    int32_t* new_lens;
    int32_t* kept;               // [B][H][keep]
    const float* scores;         // [B][H][nb_cap]
    float* to_scores;            // [B][H][to_cap]
    const uint8_t* data[2];
    const float* scale[2];
    uint8_t* to_data[2];
    float* to_scale[2];
    uint32_t* status;
    Pages pg;
    int H, t_cap, nb_cap, to_cap, keep, first, last;   // blocks, but t_cap
};

constexpr int kDigits = 2048;                // 11 bits of a key per pass

// Floats as unsigned integers of the same order (both zeros equal); NaN lowest.
__device__ __forceinline__ uint32_t order_key(float x) {
    if (x != x) return 0u;
    const uint32_t u = __float_as_uint(x + 0.f);
    return (u >> 31) ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ void new_length(const EvictArgs& a, int b) {
    const int T = max(0, min(a.seq_lens[b], a.t_cap));
    const int nb = (T + kBlk - 1) / kBlk;
    a.new_lens[b] = T - max(0, nb - a.keep) * kBlk;
}

// Where nothing overlaps: one wavefront, one block of a tensor.  The old blocks
// are read past the caches, the new ones stay in them for whoever reads them next
// (131072 tokens to half and read back: 143 us against 158 without, 150 with both
// past the caches).
__device__ __forceinline__ void copy_block(const EvictArgs& a, int64_t row, int which, int from, int i, int lane) {
    const u32x4* src = reinterpret_cast<const u32x4*>(a.data[which] + (row * a.nb_cap + from) * kBlkBytes) + lane;
    u32x4* dst = reinterpret_cast<u32x4*>(a.to_data[which] + (row * a.to_cap + i) * kBlkBytes) + lane;
    u32x4 x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = __builtin_nontemporal_load(src + 64 * k);
#pragma unroll
    for (int k = 0; k < 4; ++k) dst[64 * k] = x[k];
}

// One workgroup per (KV head, sequence) chooses the blocks, then one scan in
// block order writes the list and moves the scores and the two scales, each to
// a place at or before its own.  The choice, among the blocks that are neither
// the first nor the newest ones:
//   KEYS = 1 (up to one block per thread): a block's rank, the number of blocks
//   before it in the order of (score, lower index), counted against all others
//   (LDS broadcasts, two instructions per pair).  COPY: several workgroups choose the
//   same and then copy the kept blocks, one of them writes what else there is;
//   else a radix selection (11, 11 and 10 bits of a key) finds the smallest
//   kept key and how many of its ties are kept (the lowest indexes).  KEYS
//   THREADS blocks are read once and stay in registers; longer sequences are
//   read again in each pass and scanned in rounds of so many.
template <int THREADS, int KEYS, bool COPY = false>
__global__ __launch_bounds__(THREADS) void q8_select_kernel(EvictArgs a) {
    static_assert(KEYS == 1 || !COPY, "the list of kept blocks is in LDS");
    constexpr int kSelThreads = THREADS, kSelWaves = THREADS / kWave, kSelKeys = KEYS;
    __shared__ __align__(16) uint32_t hist[KEYS == 1 ? THREADS : kDigits];
    __shared__ uint32_t part[kSelWaves];
    __shared__ int list[COPY ? THREADS : 1];
    __shared__ uint32_t s_bin, s_rem;
    __shared__ int s_tie[kSelKeys][kSelWaves], s_kept[kSelKeys][kSelWaves];
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const int lane = tid & (kWave - 1), wave = tid / kWave;
    const int64_t row = (int64_t)b * a.H + h;
    const bool writes = !COPY || blockIdx.z == 0;         // the list, the scores and the scales
    const float* sc = a.scores + row * a.nb_cap;
    float* to = a.to_scores + row * a.to_cap;
    int32_t* kept = a.kept + row * a.keep;
    constexpr int kRound = kSelKeys * kSelThreads;
    float s[kSelKeys], x[kSelKeys][2];
    bool bad = false;
    auto read = [&](int i0, int n) {
#pragma unroll
        for (int r = 0; r < kSelKeys; ++r) {
            const int i = i0 + r * kSelThreads + tid;
            s[r] = x[r][0] = x[r][1] = 0.f;
            if (i < n) {
                s[r] = sc[i];
                if (writes) {
                    const int64_t bi = block_index(a.pg, a.H, a.nb_cap, b, h, i, bad);
                    x[r][0] = a.scale[0][bi];
                    x[r][1] = a.scale[1][bi];
                }
            }
        }
    };
    // the first round is requested before the length is known, but in pages,
    // whose table may name none behind it
    if (!a.pg.bt) read(0, a.nb_cap);
    const int T = max(0, min(a.seq_lens[b], a.t_cap));
    const int nb = (T + kBlk - 1) / kBlk;
    if (a.pg.bt) read(0, nb);
    const bool cut = nb > a.keep;
    const int lo = cut ? a.first : nb, hi = cut ? nb - a.last : nb;   // the blocks to choose from
    uint32_t prefix = 0, rem = cut ? (uint32_t)(a.keep - a.first - a.last) : 0u;
    const bool choose = rem > 0;
    bool among = false;                                   // KEYS = 1: this thread's block is kept
    if constexpr (KEYS == 1) {
        if (choose) {
            const uint32_t key = order_key(s[0]);
            const int m = hi - lo, me = tid - lo;
            if (me >= 0 && me < m) hist[me] = key;
            if (tid >= m && tid < ((m + 3) & ~3)) hist[tid] = 0u;   // (nothing is below 0)
            __syncthreads();
            // below the wavefront's own blocks ties count, above them they do not
            const int w0 = min(max(wave * kWave - lo, 0), m) & ~3;
            const int w1 = min((max((wave + 1) * kWave - lo, 0) + 3) & ~3, (m + 3) & ~3);
            const uint4* keys = reinterpret_cast<const uint4*>(hist);
            int rank = 0;
#pragma unroll 8
            for (int j = 0; j < w0; j += 4) {
                const uint4 k = keys[j / 4];
                rank += (k.x >= key) + (k.y >= key) + (k.z >= key) + (k.w >= key);
            }
#pragma unroll 4
            for (int j = w0; j < w1; j += 4) {
                const uint4 k = keys[j / 4];
                rank += (k.x > key || (k.x == key && j < me)) + (k.y > key || (k.y == key && j + 1 < me)) +
                        (k.z > key || (k.z == key && j + 2 < me)) + (k.w > key || (k.w == key && j + 3 < me));
            }
#pragma unroll 8
            for (int j = w1; j < m; j += 4) {
                const uint4 k = keys[j / 4];
                rank += (k.x > key) + (k.y > key) + (k.z > key) + (k.w > key);
            }
            among = rank < (int)rem;
        }
    } else if (choose) {
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
            const uint32_t digits = pass == 2 ? 1024u : 2048u;
            auto count = [&](float score, int i) {
                const uint32_t key = order_key(score);
                if (i >= lo && i < hi && (pass == 0 || (key >> (shift + (pass == 2 ? 10 : 11))) == prefix))
                    atomicAdd(&hist[(key >> shift) & (digits - 1)], 1u);
            };
            for (int d = tid; d < kDigits; d += kSelThreads) hist[d] = 0u;
            __syncthreads();
#pragma unroll
            for (int r = 0; r < kSelKeys; ++r) {
                const int i = r * kSelThreads + tid;
                if (i < nb) count(s[r], i);
            }
            for (int i = kRound + tid; i < nb; i += kSelThreads) count(sc[i], i);
            __syncthreads();
            // thread t: the digits 2047 - 2 t and 2046 - 2 t, counted from the top
            const int d = kDigits - 1 - 2 * tid;
            const uint32_t n0 = hist[d], n1 = hist[d - 1];
            uint32_t incl = n0 + n1;
#pragma unroll
            for (int k = 1; k < kWave; k <<= 1) {
                const uint32_t o = __shfl_up(incl, k);
                if (lane >= k) incl += o;
            }
            if (lane == kWave - 1) part[wave] = incl;
            __syncthreads();
            uint32_t above = incl - n0 - n1;
            for (int w = 0; w < wave; ++w) above += part[w];
            if (above < rem && rem <= above + n0) {
                s_bin = (uint32_t)d;
                s_rem = rem - above;
            } else if (above + n0 < rem && rem <= above + n0 + n1) {
                s_bin = (uint32_t)(d - 1);
                s_rem = rem - above - n0;
            }
            __syncthreads();
            prefix = (prefix << (pass == 2 ? 10 : 11)) | s_bin;
            rem = s_rem;
        }
    }
    // keys above `prefix` are kept, and the first `rem` equal to it
    int ties = 0, n = 0;                                  // of the blocks before this round
    const uint64_t below = (1ull << lane) - 1ull;
    for (int i0 = 0; i0 < nb; i0 += kRound) {
        if (i0) read(i0, nb);
        uint32_t keep = 0, tie = 0;                       // bit r: block i0 + 1024 r + tid
        int t[kSelKeys], pos[kSelKeys];
#pragma unroll
        for (int r = 0; r < kSelKeys; ++r) {
            const int i = i0 + r * kSelThreads + tid;
            if (i < nb) {
                bool k = i < lo || i >= hi;
                if (KEYS == 1) {
                    k = k || among;
                } else if (!k && choose) {
                    const uint32_t key = order_key(s[r]);
                    k = key > prefix;
                    tie |= (key == prefix ? 1u : 0u) << r;
                }
                keep |= (k ? 1u : 0u) << r;
            }
            const uint64_t tb = __builtin_amdgcn_ballot_w64((tie >> r) & 1u);
            t[r] = __popcll(tb & below);
            if (lane == 0) s_tie[r][wave] = __popcll(tb);
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kSelKeys; ++r) {
            int before = ties;
            for (int w = 0; w < kSelWaves; ++w) {
                if (w == wave) before = ties;
                ties += s_tie[r][w];
            }
            if (((tie >> r) & 1u) && before + t[r] < (int)rem) keep |= 1u << r;
            const uint64_t kb = __builtin_amdgcn_ballot_w64((keep >> r) & 1u);
            pos[r] = __popcll(kb & below);
            if (lane == 0) s_kept[r][wave] = __popcll(kb);
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kSelKeys; ++r) {
            int before = n;
            for (int w = 0; w < kSelWaves; ++w) {
                if (w == wave) before = n;
                n += s_kept[r][w];
            }
            if ((keep >> r) & 1u) {
                const int p = before + pos[r];
                if (COPY) list[p] = tid;
                if (writes) {
                    kept[p] = i0 + r * kSelThreads + tid;
                    to[p] = s[r];
                    bool tbad = false;
                    const int64_t ti = block_index(a.pg, a.H, a.to_cap, b, h, p, tbad);
                    if (!tbad) {
                        a.to_scale[0][ti] = x[r][0];
                        a.to_scale[1][ti] = x[r][1];
                    }
                    bad |= tbad;
                }
            }
        }
        __syncthreads();
    }
    if (bad && a.status) atomicOr(a.status, DQ_STATUS_PAGE);
    if (writes) {
        for (int i = n + tid; i < a.keep; i += kSelThreads) kept[i] = -1;
        const int end = a.scores == a.to_scores ? min(nb, a.to_cap) : a.to_cap;
        for (int i = n + tid; i < end; i += kSelThreads) to[i] = 0.f;
    }
    if constexpr (COPY) {
        if (writes && h == 0 && tid == 0) new_length(a, b);
        // (the round's last barrier is behind the list)
        for (int w = (int)blockIdx.z * kSelWaves + wave; w < 2 * n; w += (int)gridDim.z * kSelWaves)
            copy_block(a, row, w & 1, list[w >> 1], w >> 1, lane);
    }
}

// In place the kept blocks' codes move to places at or before their old ones,
// in order.  A workgroup owns 256 bytes of every block of one (KV head,
// sequence) and tensor and walks through the list, 32 blocks per wavefront and
// round: all of a round's pieces are read before any is written, and what a later
// round reads lies behind all that was written, so no workgroup waits for
// another.  The list is read a round ahead, the blocks past L2 (131072 tokens to
// half, selection included: 59 us; 102 with reads that settle in L2, 378 with one
// wavefront per workgroup; into another cache 53).  512 bytes or whole rows per
// workgroup leave CUs idle (one KV head 94 and 174 against 55 us).
constexpr int kMoveU = 8;                    // pieces of 16 bytes per lane and round
constexpr int kMoveBlocks = 4 * kMoveU;      // blocks per wavefront and round

__global__ __launch_bounds__(1024) void q8_move_kernel(EvictArgs a) {
    const int slice = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    if (slice == 0 && h == 0 && threadIdx.x == 0) new_length(a, b);
    const int which = slice >> 4, off = (slice & 15) * 256 + (lane & 15) * 16;
    const int32_t* kept = a.kept + ((int64_t)b * a.H + h) * a.keep;
    const int round = (int)blockDim.x / kWave * kMoveBlocks;
    const int mine = wave * kMoveBlocks + (lane >> 4);
    int from[kMoveU];
    auto list = [&](int i0) {
#pragma unroll
        for (int u = 0; u < kMoveU; ++u) from[u] = kept[min(i0 + mine + 4 * u, a.keep - 1)];
    };
    list(0);
    for (int i0 = 0; i0 < a.keep; i0 += round) {
        if (kept[i0] < 0) break;      // the list ends
        u32x4 x[kMoveU];
        int64_t to[kMoveU];           // the piece's block, -1: nothing moves
        int64_t at[kMoveU];
#pragma unroll
        for (int u = 0; u < kMoveU; ++u) {
            const int i = i0 + mine + 4 * u;
            to[u] = -1;
            if (i < a.keep && from[u] > i) {
                bool bad = false;
                at[u] = block_index(a.pg, a.H, a.nb_cap, b, h, from[u], bad);
                to[u] = block_index(a.pg, a.H, a.to_cap, b, h, i, bad);
                if (bad) to[u] = -1;
            }
        }
#pragma unroll
        for (int u = 0; u < kMoveU; ++u)
            if (to[u] >= 0)
                x[u] = __builtin_nontemporal_load(
                    reinterpret_cast<const u32x4*>(a.data[which] + at[u] * kBlkBytes + off));
        if (i0 + round < a.keep) list(i0 + round);
        // every read of the round is back before the first write
        __builtin_amdgcn_s_waitcnt(0);
        __builtin_amdgcn_sched_barrier(0);
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kMoveU; ++u)
            if (to[u] >= 0) *reinterpret_cast<u32x4*>(a.to_data[which] + to[u] * kBlkBytes + off) = x[u];
    }
}

// Into another cache: a wavefront per kept block and tensor.
__global__ __launch_bounds__(256) void q8_copy_kernel(EvictArgs a) {
    const int h = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & (kWave - 1);
    if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) new_length(a, b);
    const int w = wave_index(4), i = w >> 1;
    if (i >= a.keep) return;
    const int64_t row = (int64_t)b * a.H + h;
    const int from = a.kept[row * a.keep + i];
    if (from >= 0) copy_block(a, row, w & 1, from, i, lane);
}

}  // namespace

// ---------------------------------------------------------------- launchers

static bool rows_aligned(const void* p, int64_t sb, int64_t st, int64_t sh) {
    return ((reinterpret_cast<uintptr_t>(p) & 15) | ((sb | st | sh) & 7)) == 0 && st >= 0 && st < (1 << 24);
}

int launch_q8_encode(int format, const Pages& pg, const Q8Rows& k, const Q8Rows& v, int32_t B, int32_t H, int32_t t0,
                     int32_t n_new, int32_t t_cap, const Q8Cache& to, uint32_t* status, hipStream_t stream) {
    EncArgs a;
    const Q8Rows* rows[2] = {&k, &v};
    for (int i = 0; i < 2; ++i) {
        a.x[i] = rows[i]->p;
        a.sb[i] = rows[i]->sb;
        a.st[i] = rows[i]->st;
        a.sh[i] = rows[i]->sh;
        a.aligned[i] = rows_aligned(a.x[i], a.sb[i], a.st[i], a.sh[i]);
        a.data[i] = to.data[i];
        a.scale[i] = to.scale[i];
    }
    a.status = status;
    a.pg = pg;
    a.H = H;
    a.blk0 = t0 / kBlk;
    a.nblk = (int)(((int64_t)n_new + kBlk - 1) / kBlk);
    a.n_new = n_new;
    a.nb_cap = t_cap / kBlk;
    const int64_t waves = (int64_t)H * a.nblk;
    if (waves >= (1 << 26)) return DQ_ERR_INVALID_ARG;   // a grid has under 2^32 work-items along x
    const dim3 grid((unsigned)((waves + 3) / 4), B, 2);
    if (format == DQ_Q8_E4M3)
        q8_encode_kernel<DQ_Q8_E4M3><<<grid, 256, 0, stream>>>(a);
    else
        q8_encode_kernel<DQ_Q8_INT8><<<grid, 256, 0, stream>>>(a);
    return hip_check("q8_encode launch", hipGetLastError());
}

int launch_q8_read(int format, const Pages& pg, const Q8Cache& from, int32_t B, int32_t H, int32_t t0, int32_t n,
                   int32_t t_cap, const Q8Rows& k, const Q8Rows& v, uint32_t* status, hipStream_t stream) {
    ReadArgs a;
    const Q8Rows* rows[2] = {&k, &v};
    for (int i = 0; i < 2; ++i) {
        a.out[i] = const_cast<uint16_t*>(rows[i]->p);
        a.sb[i] = rows[i]->sb;
        a.st[i] = rows[i]->st;
        a.sh[i] = rows[i]->sh;
        a.aligned[i] = rows_aligned(a.out[i], a.sb[i], a.st[i], a.sh[i]);
        a.data[i] = from.data[i];
        a.scale[i] = from.scale[i];
    }
    a.status = status;
    a.pg = pg;
    a.H = H;
    a.blk0 = t0 / kBlk;
    a.nblk = (int)(((int64_t)n + kBlk - 1) / kBlk);
    a.n = n;
    a.nb_cap = t_cap / kBlk;
    const int64_t waves = (int64_t)H * a.nblk;
    if (waves >= (1 << 26)) return DQ_ERR_INVALID_ARG;   // a grid has under 2^32 work-items along x
    const dim3 grid((unsigned)((waves + 3) / 4), B, 2);
    if (format == DQ_Q8_E4M3)
        q8_read_kernel<DQ_Q8_E4M3><<<grid, 256, 0, stream>>>(a);
    else
        q8_read_kernel<DQ_Q8_INT8><<<grid, 256, 0, stream>>>(a);
    return hip_check("q8_read launch", hipGetLastError());
}

namespace {

// Blocks of one sequence that a step can see.
int64_t seen_blocks(int t_cap, int window, int sinks) {
    const int64_t nb = t_cap / kBlk;
    // a window of w tokens meets at most w / 32 + 2 blocks
    return window > 0 ? std::min(nb, ((int64_t)sinks + kBlk - 1) / kBlk + (int64_t)window / kBlk + 2) : nb;
}

// How a step is cut.
struct Q8Plan {
    int chunk, nchunks;          // blocks per chunk, chunk slots per sequence
    int target, items;           // > 0: chunks over all sequences, workgroups per KV head
    bool whole;                  // one chunk per sequence, nothing to merge
};

// One chunk per sequence where it is short (up to 16 blocks: 8 KV heads of one
// sequence of 512 tokens take 7.6 us in one launch, 7.9 in two) or where the
// (sequence, KV head) pairs fill the CUs by themselves (half of them: up to 64
// blocks, 32 sequences of 2048 tokens 22 against 27 us; twice: up to 128, 128
// of 4096 159 against 170 us; beyond, unlike lengths would leave CUs idle).
// Else the kernel or, behind a window, the loop below picks the chunk length
// for which the busiest CU has the least to do (3 sequences of 32768 tokens:
// 35 us; two workgroups per CU at any length 40, one 46).  At most 32 chunks
// per sequence (64 make no difference to one of 32768 tokens, 16.7 us, and cost
// a long one among fifteen short ones 2 of 60) unless that leaves CUs without
// work; at most 64 for the merges outside this file, which take as many in one
// pass (one KV head of 120000 tokens, partials and merge: 21 us against 42 with
// 235 chunks).
Q8Plan q8_plan(int64_t cus, int B, int Hkv, int t_cap, int window, int sinks, bool one_call) {
    const int64_t nb = seen_blocks(t_cap, window, sinks);
    const int64_t pairs = (int64_t)B * Hkv;
    Q8Plan p{};
    if (one_call && (nb <= 16 || (2 * pairs >= cus && nb <= 64) || (pairs >= 2 * cus && nb <= 128))) {
        p.chunk = (int)nb;
        p.nchunks = 1;
        p.whole = true;
        return p;
    }
    const int64_t most = std::min({(nb + 3) / 4, std::max<int64_t>(32, (cus + pairs - 1) / pairs),
                                   (int64_t)(one_call ? kMostChunks : kWave)});
    const int64_t target = std::max<int64_t>(1, cus / Hkv), items = std::min(6 * target + B, B * most);
    // (a workgroup reads all lengths; a grid has under 2^32 work-items along x)
    if (window == 0 && B <= 256 && B * nb < (1 << 30) && items * Hkv < (1 << 23)) {
        p.nchunks = (int)most;
        p.target = (int)target;
        p.items = (int)items;
        return p;
    }
    // (every call of a windowed step comes here: no 64-bit divisions)
    const uint32_t blocks = (uint32_t)nb;
    uint32_t chunk = blocks;
    double best = INFINITY;
    for (uint32_t n = 1; n <= (uint32_t)std::min<int64_t>(most, 64); ++n) {
        const uint32_t c = ((blocks + n - 1) / n + 3) & ~3u, used = (blocks + c - 1) / c;
        const double cost = std::ceil((double)(used * pairs) / (double)cus) * (double)(c + kChunkCost);
        if (cost < best) {
            best = cost;
            chunk = c;
        }
    }
    p.chunk = (int)chunk;
    p.nchunks = (int)((nb + chunk - 1) / chunk);
    return p;
}

template <int FMT, int WAVES>
void launch_q8_format(const Q8Args& a, dim3 grid, hipStream_t stream) {
    if (a.lse)
        q8_partial_kernel<FMT, true, WAVES><<<grid, WAVES * kWave, 0, stream>>>(a);
    else
        q8_partial_kernel<FMT, false, WAVES><<<grid, WAVES * kWave, 0, stream>>>(a);
}

}  // namespace

int launch_q8_partial(int format, const Pages& pg, const uint16_t* q, int32_t B, int32_t Hq, int32_t Hkv,
                      const Q8Cache& c, const int32_t* seq_lens, const int32_t* extra_lens, int32_t t_cap,
                      int32_t window, int32_t sinks, float scale, float* lse, float* out, float* scores, void* ws,
                      uint32_t* status, hipStream_t stream, int* slots) {
    const int cus = cu_count();
    const Q8Plan plan = q8_plan(cus, B, Hkv, t_cap, window, sinks, out != nullptr);
    const bool whole = plan.whole;
    if (slots) *slots = whole ? 0 : plan.nchunks;
    Q8Args a;
    a.q = q;
    a.k = c.data[0];
    a.ks = c.scale[0];
    a.v = c.data[1];
    a.vs = c.scale[1];
    a.seq_lens = seq_lens;
    a.extra_lens = extra_lens;
    a.pg = pg;
    a.Hq = Hq;
    a.Hkv = Hkv;
    a.G = Hq / Hkv;
    a.t_cap = t_cap;
    a.chunk = plan.chunk;
    a.nchunks = plan.nchunks;
    a.window = window;
    a.sinks = sinks;
    a.scale_log2 = scale * 1.4426950408889634f;
    a.lse = lse;
    a.out = whole ? out : nullptr;
    a.scores = whole ? scores : nullptr;
    a.B = B;
    a.target = plan.target;
    a.items = plan.items;
    a.per_cu = 0.99999f / (float)cus;
    a.early = whole && window == 0 && !pg.bt && (int64_t)Hkv * B <= cus;
    a.status = status;
    const int64_t held = ws_slots(B, Hq, t_cap);
    a.ws_hdr = static_cast<int32_t*>(ws);
    a.ws_acc = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + kWsHeader);
    a.ws_m = a.ws_acc + held * kD;
    a.ws_l = a.ws_m + held;
    a.lse_rest = a.ws_l + held;
    const dim3 grid = plan.target ? dim3((unsigned)plan.items * Hkv) : dim3(plan.nchunks, Hkv, B);
    // Four wavefronts where a sequence has few blocks (up to 8: 8 KV heads of one of
    // 37 tokens 5.4 us against 5.7) or the pairs fill the CUs twice and more (up to
    // 32: more workgroups start at a time; 300 sequences of 200 tokens 26 against 34
    // us, of 400 46 against 51, of 1000 104 both; beyond, unlike lengths lose: 128 of
    // up to 2000 51 against 47).
    const bool small = whole && (plan.chunk <= 8 || (plan.chunk <= 32 && (int64_t)B * Hkv >= 2 * cus));
    if (format == DQ_Q8_E4M3)
        small ? launch_q8_format<DQ_Q8_E4M3, 4>(a, grid, stream) : launch_q8_format<DQ_Q8_E4M3, 8>(a, grid, stream);
    else
        small ? launch_q8_format<DQ_Q8_INT8, 4>(a, grid, stream) : launch_q8_format<DQ_Q8_INT8, 8>(a, grid, stream);
    return hip_check("q8_partial launch", hipGetLastError());
}

int launch_q8_finish(int32_t B, int32_t Hq, int32_t Hkv, const int32_t* seq_lens, const int32_t* extra_lens,
                     int32_t t_cap, int32_t window, int32_t sinks, const float* lse, const void* ws, float* out,
                     float* scores, int slots, hipStream_t stream) {
    const int64_t held = ws_slots(B, Hq, t_cap);
    FinishArgs a;
    a.seq_lens = seq_lens;
    a.extra_lens = extra_lens;
    a.lse = lse;
    a.ws_hdr = static_cast<const int32_t*>(ws);
    a.ws_acc = reinterpret_cast<const float*>(static_cast<const uint8_t*>(ws) + kWsHeader);
    a.ws_m = a.ws_acc + held * kD;
    a.ws_l = a.ws_m + held;
    a.lse_rest = a.ws_l + held;
    a.out = out;
    a.scores = scores;
    a.Hq = Hq;
    a.Hkv = Hkv;
    a.G = Hq / Hkv;
    a.t_cap = t_cap;
    a.window = window;
    a.sinks = sinks;
    a.nc_max = (int)max_chunks(t_cap);
    a.nc = slots;
    a.heads = out ? a.G : 0;
    const bool four = (int64_t)B * Hq <= kFewMerges;
    const int each = kScoreBlocks * (four ? 4 : 1);
    const int64_t parts = scores ? (seen_blocks(t_cap, window, sinks) + each - 1) / each : 0;
    const dim3 grid((unsigned)(a.heads + parts), Hkv, B);
    if (four)
        q8_finish_kernel<4><<<grid, 4 * kWave, 0, stream>>>(a);
    else
        q8_finish_kernel<1><<<grid, kWave, 0, stream>>>(a);
    return hip_check("q8_finish launch", hipGetLastError());
}

int launch_q8_evict(const Pages& pg, int32_t B, int32_t H, const int32_t* seq_lens, int32_t* new_lens, int32_t t_cap,
                    int32_t to_cap, int32_t keep, int32_t first, int32_t last, const float* scores,
                    float* to_scores, const Q8Cache& from, const Q8Cache& to, int32_t* kept, uint32_t* status,
                    hipStream_t stream) {
    EvictArgs a;
    a.seq_lens = seq_lens;
    a.new_lens = new_lens;
    a.kept = kept;
    a.scores = scores;
    a.to_scores = to_scores;
    for (int i = 0; i < 2; ++i) {
        a.data[i] = from.data[i];
        a.scale[i] = from.scale[i];
        a.to_data[i] = to.data[i];
        a.to_scale[i] = to.scale[i];
    }
    a.status = status;
    a.pg = pg;
    a.H = H;
    a.t_cap = t_cap;
    a.nb_cap = t_cap / kBlk;
    a.to_cap = to_cap / kBlk;
    a.keep = keep / kBlk;
    a.first = first / kBlk;
    a.last = last / kBlk;
    // Into another cache a short sequence's choice is quick enough for every
    // workgroup that copies to make it again: one launch, two workgroups per CU (8 KV
    // heads of one sequence of 2048 tokens 5.2 us against 6.9 in two, 16 of 4096 tokens
    // 27 against 30; over 256 blocks no gain, one of 16384 17.8 against 17.5).  Not
    // where the new lengths replace the old ones, which all of them read.
    const bool apart = a.data[0] != a.to_data[0] && (new_lens + B <= seq_lens || seq_lens + B <= new_lens);
    if (apart && a.nb_cap <= 256) {
        const int64_t some = std::max<int64_t>(2 * cu_count() / ((int64_t)B * H), 1);
        const dim3 grid(H, B, (unsigned)std::min<int64_t>(some, (2 * a.keep + 3) / 4));
        q8_select_kernel<256, 1, true><<<grid, 256, 0, stream>>>(a);
        return hip_check("q8_select launch", hipGetLastError());
    }
    if (a.nb_cap <= 256)
        q8_select_kernel<256, 1><<<dim3(H, B), 256, 0, stream>>>(a);
    else if (a.nb_cap <= 512)
        q8_select_kernel<512, 1><<<dim3(H, B), 512, 0, stream>>>(a);
    else if (a.nb_cap <= 4096)
        q8_select_kernel<1024, 4><<<dim3(H, B), 1024, 0, stream>>>(a);
    else
        q8_select_kernel<1024, 8><<<dim3(H, B), 1024, 0, stream>>>(a);
    if (int rc = hip_check("q8_select launch", hipGetLastError())) return rc;
    const int waves = std::min((a.keep + kMoveBlocks - 1) / kMoveBlocks, 16);
    if (a.data[0] == a.to_data[0])
        q8_move_kernel<<<dim3(32, H, B), waves * kWave, 0, stream>>>(a);
    else
        q8_copy_kernel<<<dim3((unsigned)((2 * (int64_t)a.keep + 3) / 4), H, B), 256, 0, stream>>>(a);
    return hip_check("q8_move launch", hipGetLastError());
}

}  // namespace dq
