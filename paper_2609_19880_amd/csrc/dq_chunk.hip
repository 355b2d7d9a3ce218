// Attention of many queries of a sequence at once: the new tokens of a chunk
// over the 8-bit cache (causal, all of it or behind a window), or queries of
// another sequence over an encoder's states (the 8-bit cache again, or BF16).
//
//   o_r = sum_t a_rt v_t,  a_r = softmax over the visible t of scale q_r . k_t
//
// A row r is a (token, query head) pair: the G query heads that share a KV head
// are rows of one tile, token by token, so a few tokens fill a tile too and
// keys and values are read once for all of them.
//
// Products.  S^T (32 tokens x 32 rows) = K Q^T and O^T (128 channels x 32
// rows) += V^T P^T on v_mfma_f32_32x32x16: a lane holds one row's scores of 16
// tokens, softmax statistics stay in the lane (and its partner lane ^ 32), and
// the weights are the second product's operand where they lie.
//
// 8-bit codes are exact in fp16.  A key block's scale multiplies the scores; a
// value block's scale goes into the exponent of the weights, relative to the
// largest scale so far.  Queries are brought to a largest magnitude of 2^13 by
// a power of 2 of each row, exactly but for values 2^-37 of the largest.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "dq_chunk.h"
#include "dq_common.h"

namespace dq {
namespace {

constexpr int kD = 128;
constexpr int kBlk = DQ_Q8_BLOCK;
constexpr int kBlkBytes = kBlk * kD;
constexpr int kTile = 2;                     // blocks of 32 tokens per step
constexpr float kBig = 3e38f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kRowsOf = 32;                  // rows per wavefront
constexpr float kNoScale = -1e30f;           // log2 of the scale of a block of zeros

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

struct ChunkArgs {
    const uint16_t* q;
    int64_t q_sb, q_st, q_sh;
    uint16_t* out;
    int64_t o_sb, o_st, o_sh;
    const uint8_t* k;            // codes, or BF16 rows
    const uint8_t* v;
    const float* ks;
    const float* vs;
    int64_t k_sb, k_st, k_sh, v_sb, v_st, v_sh;
    const uint8_t* mask;
    int64_t mask_sb;
    const int32_t* q_lens;
    const int32_t* seq_lens;
    Pages pg;
    int B, Hq, H, G, n_q, t_cap, causal, window, sinks;
    int q_aligned, kv_aligned, out_aligned;
    float scale_log2;            // |softmax scale| log2 e
    int negative;                // the softmax scale is
    int target, least;           // work items wanted, fewest blocks of one
    uint32_t* status;
    float* ws_acc;               // [slot][rows][128]
    float* ws_ml;                // [slot][2][rows]
};

// ------------------------------------------------------------------- shares
//
// A segment is a tile of rows of one (sequence, KV head).  Where there are
// fewer segments than the GPU takes at a time, their tokens are cut into
// pieces of `chunk` blocks, so that there are about `target` work items; the
// pieces of a row are joined by the merge kernel.  Lengths are known on the
// device only, so every workgroup derives the same plan from them.

struct Seq {
    int T, n, tiles, units;      // tokens, new tokens, row tiles, most blocks that a row tile sees
};

template <int R>
__device__ __forceinline__ Seq seq_of(const ChunkArgs& a, int b) {
    Seq s;
    s.T = a.seq_lens ? max(0, min(a.seq_lens[b], a.t_cap)) : a.t_cap;
    s.n = a.q_lens ? max(0, min(a.q_lens[b], a.n_q)) : a.n_q;
    s.tiles = (s.n * a.G + R - 1) / R;
    const int all = (int)(((int64_t)s.T + kBlk - 1) / kBlk);
    s.units = all;
    if (a.window > 0) {
        const int64_t span = (int64_t)a.window + (R - 1) / a.G + 1;
        const int64_t most = (min((int64_t)a.sinks, (int64_t)s.T) + kBlk - 1) / kBlk + (span + 2 * kBlk - 1) / kBlk;
        s.units = (int)min((int64_t)all, most);
    }
    return s;
}

struct Item {
    int b, h, tile, c;           // tile = -1: nothing
    int chunk, slot;
};

// The blocks of one piece, and where item `id` lies.  All lanes agree.
template <int R>
__device__ __forceinline__ int plan_chunk(const ChunkArgs& a, int lane) {
    double total = 0, segs = 0;
    for (int b0 = 0; b0 < a.B; b0 += kWave) {
        double t = 0, s = 0;
        if (b0 + lane < a.B) {
            const Seq q = seq_of<R>(a, b0 + lane);
            s = q.tiles;
            t = (double)q.tiles * q.units;
        }
        total += wave_reduce(t, [](double x, double y) { return x + y; });
        segs += wave_reduce(s, [](double x, double y) { return x + y; });
    }
    total *= a.H;
    segs *= a.H;
    if (segs >= a.target) return 0x7FFFFFFE;
    const int c = (int)ceil(total / a.target);
    return max((c + 1) & ~1, a.least);
}

__device__ __forceinline__ int pieces(int units, int chunk) { return max(1, (units - 1) / chunk + 1); }

template <int R>
__device__ __forceinline__ int items_of(const ChunkArgs& a, const Seq& s, int chunk) {
    return s.tiles * pieces(s.units, chunk) * a.H;
}

__device__ __forceinline__ int scan64(int v) {         // inclusive sums over the lanes
    v += dpp0<0x111, 0xF>(v);
    v += dpp0<0x112, 0xF>(v);
    v += dpp0<0x114, 0xF>(v);
    v += dpp0<0x118, 0xF>(v);
    v += dpp0<0x142, 0xA>(v);
    v += dpp0<0x143, 0xC>(v);
    return v;
}

// Item number `id` of the plan: sequence after sequence, KV head after KV head,
// the last row tiles (which see most) first, their pieces in order.
template <int R>
__device__ __forceinline__ Item find_item(const ChunkArgs& a, int id, int lane) {
    Item it{0, 0, -1, 0, plan_chunk<R>(a, lane), 0};
    int all = 0;
    for (int b0 = 0; b0 < a.B; b0 += kWave)
        all += wave_sum(b0 + lane < a.B ? items_of<R>(a, seq_of<R>(a, b0 + lane), it.chunk) : 0);
    // workgroups go to the 8 XCDs in turn: an XCD takes items that follow each
    // other, which share keys and values in its L2
    const int per = (all + 7) / 8;
    const int x = (id & 7) * per + (id >> 3);
    if ((id >> 3) >= per || x >= all) return it;
    int before = 0;
    for (int b0 = 0; b0 < a.B; b0 += kWave) {
        Seq s{0, 0, 0, 0};
        int own = 0;
        if (b0 + lane < a.B) {
            s = seq_of<R>(a, b0 + lane);
            own = items_of<R>(a, s, it.chunk);
        }
        const int upto = before + scan64(own);
        const int last = __builtin_amdgcn_readlane(upto, 63);
        if (x < last) {
            const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > x));
            const int r = x - __builtin_amdgcn_readlane(upto - own, l);
            const int nc = pieces(__builtin_amdgcn_readlane(s.units, l), it.chunk);
            const int tiles = __builtin_amdgcn_readlane(s.tiles, l);
            it.b = b0 + l;
            it.h = r / (tiles * nc);
            it.tile = tiles - 1 - (r / nc) % tiles;
            it.c = r % nc;
            it.slot = x;
            return it;
        }
        before = last;
    }
    return it;
}

// The slot of piece 0 of (b, h, tile).
template <int R>
__device__ __forceinline__ int first_slot(const ChunkArgs& a, int b, int h, int tile, int chunk, int lane) {
    int before = 0;
    for (int b0 = 0; b0 < b; b0 += kWave)
        before += wave_sum(b0 + lane < b ? items_of<R>(a, seq_of<R>(a, b0 + lane), chunk) : 0);
    const Seq s = seq_of<R>(a, b);
    return before + (h * s.tiles + (s.tiles - 1 - tile)) * pieces(s.units, chunk);
}

// Blocks that rows [r0, r1) of a sequence see: the first `head`, then those
// from `from` on, `count` in all.
struct Sees {
    int T, off, head, from, count;
};

__device__ __forceinline__ Sees sees(const ChunkArgs& a, const Seq& s, int r0, int r1) {
    Sees v;
    v.T = s.T;
    v.off = a.causal ? s.T - s.n : 0;
    int end = s.T;
    if (a.causal) end = max(0, min(s.T, v.off + (r1 - 1) / a.G + 1));
    const int blocks = (int)(((int64_t)end + kBlk - 1) / kBlk);
    v.head = 0;
    v.from = 0;
    if (a.window > 0) {
        const int64_t start = (int64_t)v.off + r0 / a.G + 1 - a.window;
        v.head = (int)(((int64_t)min(a.sinks, end) + kBlk - 1) / kBlk);
        v.from = max(v.head, (int)(max((int64_t)0, min(start, (int64_t)end)) / kBlk));
    }
    v.count = v.head + max(0, blocks - v.from);
    return v;
}

// ------------------------------------------------------------------ numbers

template <int SRC>
__device__ __forceinline__ f32x16 mma(const u32x4& x, const u32x4& y, const f32x16& c) {
    if constexpr (SRC == kChunkBf16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c,
                                                       0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0,
                                                      0, 0);
}

// Four code bytes to four fp16 values (exact for both types).
template <int SRC>
__device__ __forceinline__ u32x2 halves4(uint32_t w) {
    f16x2 lo, hi;
    if constexpr (SRC == DQ_Q8_E4M3) {
        lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.f, false);
        hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.f, true);
    } else {
        // byte + 128 as the low bits of an fp16 in [1024, 2048), less 1152
        const uint32_t magic = 0x64646464u;
        const f16x2 off = {(_Float16)1152.f, (_Float16)1152.f};
        w ^= 0x80808080u;
        lo = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(magic, w, 0x04010400u)) - off;
        hi = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(magic, w, 0x04030402u)) - off;
    }
    return u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}

// Two weights as the second product's operand takes them, ties to even.
template <int SRC>
__device__ __forceinline__ uint32_t weights2(float x, float y) {
    if constexpr (SRC == kChunkBf16)
        return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x, (__bf16)y});
    else
        return __builtin_bit_cast(uint32_t, f16x2{(_Float16)x, (_Float16)y});
}

__device__ __forceinline__ uint32_t bf16_two(float x, float y) {
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x, (__bf16)y});
}

__device__ __forceinline__ float clamped(float x) {    // NaN stays
    x = x > kBig ? kBig : x;
    return x < -kBig ? -kBig : x;
}

// -------------------------------------------------------------- the kernel

// One workgroup of NW wavefronts per item: 32 NW rows, 32 per wavefront.
// Steps of 64 tokens: codes are read, converted to fp16 once for the workgroup
// and laid into LDS as the products take them (values transposed by the order
// of the codes, or, in BF16, by the LDS read).  The next step's codes are on
// their way meanwhile.
template <int SRC, int NW>
__global__ __launch_bounds__(NW* kWave, 2) void chunk_kernel(ChunkArgs a) {
    constexpr int R = NW * kRowsOf, NT = NW * kWave;
    constexpr bool q8 = SRC != kChunkBf16;
    constexpr int kPieces = q8 ? 1024 / NT : 2048 / NT;   // 16-byte pieces per thread and step
    __shared__ u32x4 lk[2][kTile][8][64];
    __shared__ u32x4 lv[2][kTile][8][64];
    __shared__ float2 lscale[2][kTile][2];       // keys: scale; values: log2 of it

    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int col = lane & 31, half = lane >> 5;
    const Item it = find_item<R>(a, (int)blockIdx.x, lane);
    if (it.tile < 0) return;
    const int b = __builtin_amdgcn_readfirstlane(it.b), h = __builtin_amdgcn_readfirstlane(it.h);
    const int tile = __builtin_amdgcn_readfirstlane(it.tile), piece = __builtin_amdgcn_readfirstlane(it.c);
    const int chunk = __builtin_amdgcn_readfirstlane(it.chunk);
    const Seq seq = seq_of<R>(a, b);
    const int rows = seq.n * a.G;                // of the whole sequence
    const int r0 = tile * R, r1 = min(r0 + R, rows);
    const Sees see = sees(a, seq, r0, r1);
    const int u0 = min((int64_t)piece * chunk, (int64_t)0x7FFFFFFF);
    const bool whole = pieces(see.count, chunk) == 1;
    if (u0 >= see.count && piece > 0) return;    // the merge does not ask for it
    const int u1 = (int)min((int64_t)u0 + chunk, (int64_t)see.count);

    // ------------------------------------------------ this lane's row
    const int wr0 = r0 + wave * kRowsOf, r = wr0 + col;
    const bool live = wr0 < rows, valid = r < rows;
    const int row = min(r, rows - 1);
    const int token = row / a.G, head = h * a.G + row % a.G;
    // what the row sees: t < limit and (t < sinks or t >= start)
    const int limit = a.causal ? max(0, min(see.T, see.off + token + 1)) : see.T;
    const int start = a.window > 0 ? (int)max((int64_t)0, (int64_t)see.off + token + 1 - a.window) : 0;
    const int sinks = a.sinks;
    const int lim_lo = __builtin_amdgcn_readfirstlane(limit);                    // rows are in order
    const int lim_hi = __builtin_amdgcn_readlane(limit, 31);
    const int start_hi = __builtin_amdgcn_readlane(start, 31);

    u32x4 qf[8];
    float qc = a.scale_log2, l = 0.f;
    {
        const uint16_t* p = a.q + (int64_t)b * a.q_sb + (int64_t)token * a.q_st + (int64_t)head * a.q_sh;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            // channels of operand j: as the keys' pieces hold them, or in order
            const int ch = q8 ? 16 * (2 * (j >> 1) + half) + 8 * (j & 1) : 16 * j + 8 * half;
            qf[j] = u32x4{0u, 0u, 0u, 0u};
            if (valid) {
                if (a.q_aligned) {
                    qf[j] = *reinterpret_cast<const u32x4*>(p + ch);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        qf[j][i] = (uint32_t)p[ch + 2 * i] | ((uint32_t)p[ch + 2 * i + 1] << 16);
                }
            }
            if (a.negative) qf[j] ^= 0x80008000u;
        }
        if constexpr (q8) {
            int top = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    top = max(top, max((int)(qf[j][i] & 0x7FFFu), (int)((qf[j][i] >> 16) & 0x7FFFu)));
            top = max(top, __float_as_int(xor_lane<32>(__int_as_float(top), lane)));
            const bool nan = top >= 0x7F80;      // infinities and NaN make the row NaN
            if (nan && limit > 0) l = NAN;
            const int e = top >= 0x80 ? (top >> 7) - 127 : -126;
            const int up = 13 - e;
            qc = ldexpf(qc, -up);
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x = ldexpf(__uint_as_float(qf[j][i] << 16), up);
                    const float y = ldexpf(__uint_as_float(qf[j][i] & 0xFFFF0000u), up);
                    qf[j][i] = nan ? 0u : weights2<SRC>(x, y);
                }
        }
    }

    // ------------------------------------------------ loads
    bool bad = false;
    auto block_of = [&](int u) { return u < see.head ? u : see.from + (u - see.head); };
    u32x4 reg[kPieces];
    float sreg[kPieces];
    // requests the step of blocks u, u + 1
    auto request = [&](int u) {
        if constexpr (q8) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int p = tid + i * NT;      // block, keys or values, piece
                const int blk = __builtin_amdgcn_readfirstlane(p >> 9), kind = __builtin_amdgcn_readfirstlane((p >> 8) & 1);
                reg[i] = u32x4{0u, 0u, 0u, 0u};
                sreg[i] = 0.f;
                if (u + blk < u1) {
                    const int at = block_of(u + blk);
                    int64_t bi;
                    if (a.pg.bt) {
                        const int64_t pp = physical_page(a.pg, b, at * kBlk, bad);
                        const int bpp = 1 << (a.pg.page_shift - 5);
                        bi = (pp * a.H + h) * bpp + (at & (bpp - 1));
                    } else {
                        bi = ((int64_t)b * a.H + h) * (a.t_cap / kBlk) + at;
                    }
                    reg[i] = reinterpret_cast<const u32x4*>((kind ? a.v : a.k) + bi * kBlkBytes)[p & 255];
                    if ((p & 255) == 0) sreg[i] = (kind ? a.vs : a.ks)[bi];
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int p = tid + i * NT;      // keys or values, token, piece
                const int kind = __builtin_amdgcn_readfirstlane(p >> 10), t = block_of(u) * kBlk + ((p >> 4) & 63), ch = 8 * (p & 15);
                reg[i] = u32x4{0u, 0u, 0u, 0u};
                bool in = t < see.T;
                // a hidden token's value must not reach the sum, whatever it is
                if (kind && a.mask && in) in = a.mask[(int64_t)b * a.mask_sb + t] != 0;
                if (in) {
                    const uint16_t* x = reinterpret_cast<const uint16_t*>(kind ? a.v : a.k) +
                                        (int64_t)b * (kind ? a.v_sb : a.k_sb) + (int64_t)h * (kind ? a.v_sh : a.k_sh) +
                                        (int64_t)t * (kind ? a.v_st : a.k_st) + ch;
                    if (a.kv_aligned) {
                        reg[i] = *reinterpret_cast<const u32x4*>(x);
                    } else {
#pragma unroll
                        for (int w = 0; w < 4; ++w)
                            reg[i][w] = (uint32_t)x[2 * w] | ((uint32_t)x[2 * w + 1] << 16);
                    }
                }
            }
        }
    };
    auto lay = [&](int buf) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int p = tid + i * NT;
            if constexpr (q8) {
                const int blk = p >> 9, kind = (p >> 8) & 1, at = p & 255;
                const u32x2 w0 = halves4<SRC>(reg[i][0]), w1 = halves4<SRC>(reg[i][1]);
                const u32x2 w2 = halves4<SRC>(reg[i][2]), w3 = halves4<SRC>(reg[i][3]);
                const u32x4 lo = {w0[0], w0[1], w1[0], w1[1]}, hi = {w2[0], w2[1], w3[0], w3[1]};
                if (kind == 0) {
                    // piece ((t / 16) 2 + c / 64) 64 + ((c / 16) % 4) 16 + t % 16
                    const int t = ((at >> 7) << 4) | (at & 15), slice = ((at >> 6) & 1) * 4 + ((at >> 4) & 3);
                    u32x4* to = &lk[buf][blk][(slice >> 1) * 2][(slice & 1) * 32 + t];
                    to[0] = lo;
                    to[64] = hi;
                } else {
                    // piece ((c / 32) 4 + (t / 4) % 4) 16 + c % 16
                    const int np = at >> 6, grp = (at >> 4) & 3;
                    u32x4* to = &lv[buf][blk][np * 2 + (grp >> 1)][(grp & 1) * 32 + (at & 15)];
                    to[0] = lo;
                    to[16] = hi;
                }
                if (at == 0) {
                    if (kind == 0)
                        lscale[buf][blk][0].x = sreg[i];
                    else
                        lscale[buf][blk][0].y = sreg[i] > 0.f ? __builtin_amdgcn_logf(sreg[i]) : kNoScale;
                }
            } else {
                const int kind = p >> 10, t = (p >> 4) & 63, g = p & 15;
                if (kind == 0)
                    lk[buf][t >> 5][g >> 1][(g & 1) * 32 + ((t & 31) ^ g)] = reg[i];
                else
                    (&lv[buf][0][0][0])[t * 16 + (g ^ ((t & 3) << 2))] = reg[i];
            }
        }
    };

    f32x16 o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
    float m = -INFINITY, vref = kNoScale;
    constexpr float kUp = q8 ? 7.f : 0.f;        // weights of the maximum are 2^7

    if (u0 < u1) {
        request(u0);
        lay(0);
    }
    __syncthreads();
    int buf = 0;
    for (int u = u0; u < u1; u += kTile, buf ^= 1) {
        if (u + kTile < u1) request(u + kTile);
        int t0[kTile];
#pragma unroll
        for (int i = 0; i < kTile; ++i) t0[i] = u + i < u1 ? block_of(u + i) * kBlk : 0x7FFFFF00;
        uint64_t shown = ~0ull;
        if (!q8 && a.mask) {
            const int t = t0[0] + lane;
            const bool on = t < see.T && a.mask[(int64_t)b * a.mask_sb + t] != 0;
            shown = __builtin_amdgcn_ballot_w64(on);
        }
        // (a wavefront whose rows see none of the step's tokens has nothing to do)
        if (live && t0[0] < lim_hi && shown != 0) {
            f32x16 s[kTile];
            float c[kTile], d[kTile], vl[kTile];
#pragma unroll
            for (int i = 0; i < kTile; ++i) {
#pragma unroll
                for (int e = 0; e < 16; ++e) s[i][e] = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const u32x4 kf = lk[buf][i][j][q8 ? lane : half * 32 + (col ^ (2 * j + half))];
                    s[i] = mma<SRC>(kf, qf[j], s[i]);
                }
                c[i] = qc;
                d[i] = 0.f;
                vl[i] = kNoScale;
                if constexpr (q8) {
                    c[i] = qc * lscale[buf][i][0].x;
                    vl[i] = lscale[buf][i][0].y;
                }
            }
            bool plain = shown == ~0ull;
#pragma unroll
            for (int i = 0; i < kTile; ++i) {
                plain = plain && t0[i] + kBlk <= lim_lo;
                if (a.window > 0) plain = plain && (t0[i] >= start_hi || t0[i] + kBlk <= sinks);
            }
            float top = NAN;                     // (stays where every score is NaN)
#pragma unroll
            for (int i = 0; i < kTile; ++i) {
                float x = s[i][0];
#pragma unroll
                for (int e = 1; e < 16; ++e) x = fmaxf(x, s[i][e]);
                top = fmaxf(top, x * c[i]);
            }
            if (!plain || __builtin_amdgcn_ballot_w64(fabsf(top) >= 0x1p11f) != 0) {
                // masks, and scores so large that a fused product would differ
                // from the maximum by more than a rounding of it
                plain = false;
                top = -INFINITY;
#pragma unroll
                for (int i = 0; i < kTile; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int in = 8 * (e >> 2) + 4 * half + (e & 3), t = t0[i] + in;
                        bool on = t < limit;
                        if (a.window > 0) on = on && (t < sinks || t >= start);
                        if (!q8) on = on && ((shown >> (i * kBlk + in)) & 1);
                        const float x = on ? clamped(s[i][e] * c[i]) : -INFINITY;
                        s[i][e] = x;
                        top = fmaxf(top, x);
                    }
            }
            top = fmaxf(top, xor_lane<32>(top, lane));
            // The sums keep the maximum they began with until a score exceeds it
            // by 8 (weights up to 2^15 then): most steps scale nothing.
            const float vtop = fmaxf(vl[0], vl[1]);
            const bool wide = q8 && vtop > vref;
            if (wide || __builtin_amdgcn_ballot_w64(top > m + 8.f) != 0) {
                // (row by row: a row's bits do not depend on its neighbours)
                const float mn = top > m + 8.f ? top : m;
                float f = m == mn ? 1.f : __builtin_amdgcn_exp2f(m - mn);
                m = mn;
                l *= f;
                if (wide) {
                    f *= __builtin_amdgcn_exp2f(vref - (vtop + 1.f));
                    vref = vtop + 1.f;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[i][e] *= f;
            }
            const float mu = m == -INFINITY ? 0.f : m;
            float e0[kTile];
#pragma unroll
            for (int i = 0; i < kTile; ++i) {
                // a block of zeros: any weight will do; below 2^-60 of the largest
                // scale fp16 weights are 0 in any case
                if constexpr (q8) d[i] = vl[i] <= kNoScale ? 0.f : fmaxf(vl[i] - vref, -60.f);
                e0[i] = kUp + d[i] - mu;
            }
            if (!plain) {
#pragma unroll
                for (int i = 0; i < kTile; ++i) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[i][e] -= mu;
                    c[i] = 1.f;
                    e0[i] = kUp + d[i];
                }
            }
#pragma unroll
            for (int i = 0; i < kTile; ++i) {
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    s[i][e] = __builtin_amdgcn_exp2f(fmaf(s[i][e], c[i], e0[i]));
                    sum += s[i][e];
                }
                l += q8 ? sum * __builtin_amdgcn_exp2f(-d[i]) : sum;
            }
#pragma unroll
            for (int i = 0; i < kTile; ++i)
#pragma unroll
                for (int st = 0; st < 2; ++st) {
                    const u32x4 pf = {weights2<SRC>(s[i][4 * st], s[i][4 * st + 1]),
                                      weights2<SRC>(s[i][4 * st + 2], s[i][4 * st + 3]),
                                      weights2<SRC>(s[i][8 + 4 * st], s[i][9 + 4 * st]),
                                      weights2<SRC>(s[i][10 + 4 * st], s[i][11 + 4 * st])};
#pragma unroll
                    for (int np = 0; np < 4; ++np) {
                        u32x4 vf;
                        if constexpr (q8) {
                            vf = lv[buf][i][np * 2 + st][lane];
                        } else {
                            // four rows of 16 channels, transposed: tokens .. + 0..3, then 16 further on
                            const int rr = (lane >> 2) & 3, x = (lane >> 4) & 1, q4 = lane & 3;
                            const int t = i * kBlk + 8 * st + 4 * half + rr;
                            const char* at = reinterpret_cast<const char*>(&lv[buf][0][0][0]) + t * 256 +
                                             ((4 * np + 2 * x + (q4 >> 1)) ^ (rr << 2)) * 16 + 8 * (q4 & 1);
                            typedef __attribute__((address_space(3))) i16x4* LdsRows;
                            const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsRows)(at));
                            const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsRows)(at + 16 * 256));
                            const u32x2 l2 = __builtin_bit_cast(u32x2, lo), h2 = __builtin_bit_cast(u32x2, hi);
                            vf = u32x4{l2[0], l2[1], h2[0], h2[1]};
                        }
                        o[np] = mma<SRC>(vf, pf, o[np]);
                    }
                }
        }
        if (u + kTile < u1) lay(buf ^ 1);
        __syncthreads();
    }
    if (bad && a.status) atomicOr(a.status, DQ_STATUS_PAGE);

    // ------------------------------------------------ results
    l += xor_lane<32>(l, lane);
    const float up = q8 ? __builtin_amdgcn_exp2f(vref) : 1.f;
    if (whole) {
        if (!valid) return;
        // rows that see nothing: zeros
        const float f = l == 0.f ? 0.f : up / l;
        uint16_t* p = a.out + (int64_t)b * a.o_sb + (int64_t)token * a.o_st + (int64_t)head * a.o_sh + 4 * half;
#pragma unroll
        for (int np = 0; np < 4; ++np)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t w0 = bf16_two(o[np][4 * i] * f, o[np][4 * i + 1] * f);
                const uint32_t w1 = bf16_two(o[np][4 * i + 2] * f, o[np][4 * i + 3] * f);
                uint16_t* x = p + 32 * np + 8 * i;
                if (a.out_aligned) {
                    *reinterpret_cast<u32x2*>(x) = u32x2{w0, w1};
                } else {
                    x[0] = (uint16_t)w0;
                    x[1] = (uint16_t)(w0 >> 16);
                    x[2] = (uint16_t)w1;
                    x[3] = (uint16_t)(w1 >> 16);
                }
            }
        return;
    }
    const int64_t slot = it.slot;
    float* acc = a.ws_acc + (slot * R + wave * kRowsOf + col) * kD + 4 * half;
#pragma unroll
    for (int np = 0; np < 4; ++np)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<f32x4*>(acc + 32 * np + 8 * i) =
                f32x4{o[np][4 * i] * up, o[np][4 * i + 1] * up, o[np][4 * i + 2] * up, o[np][4 * i + 3] * up};
    if (half == 0) {
        float* ml = a.ws_ml + slot * 2 * R + wave * kRowsOf + col;
        ml[0] = m;
        ml[R] = l;
    }
}

// The pieces of a row joined: one wavefront per row, two channels a lane.
template <int R>
__global__ __launch_bounds__(256) void chunk_merge_kernel(ChunkArgs a) {
    const int lane = threadIdx.x & (kWave - 1);
    const int b = blockIdx.y;
    const int64_t id = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
    const Seq seq = seq_of<R>(a, b);
    const int rows = seq.n * a.G;
    if (id >= (int64_t)rows * a.H) return;
    const int h = (int)(id / rows), r = (int)(id % rows), tile = r / R;
    const int chunk = plan_chunk<R>(a, lane);
    const Sees see = sees(a, seq, tile * R, min(tile * R + R, rows));
    const int nc = pieces(see.count, chunk);
    if (nc == 1) return;
    const int64_t slot = first_slot<R>(a, b, h, tile, chunk, lane);
    const float* ml = a.ws_ml + slot * 2 * R + r % R;
    float top = -INFINITY;
    for (int c = lane; c < nc; c += kWave) top = fmaxf(top, ml[(int64_t)c * 2 * R]);
    top = wave_max(top);
    float l = 0.f, x = 0.f, y = 0.f;
    const float* acc = a.ws_acc + (slot * R + r % R) * kD + 2 * lane;
    for (int c = 0; c < nc; ++c) {
        const float mc = ml[(int64_t)c * 2 * R];
        const float w = mc == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mc - top);
        const float2 v = *reinterpret_cast<const float2*>(acc + (int64_t)c * R * kD);
        l = fmaf(ml[(int64_t)c * 2 * R + R], w, l);
        x = fmaf(v.x, w, x);
        y = fmaf(v.y, w, y);
    }
    const float f = l == 0.f ? 0.f : 1.f / l;
    const int token = r / a.G, head = h * a.G + r % a.G;
    uint16_t* p = a.out + (int64_t)b * a.o_sb + (int64_t)token * a.o_st + (int64_t)head * a.o_sh + 2 * lane;
    const uint32_t w = bf16_two(x * f, y * f);
    if (a.out_aligned) {
        *reinterpret_cast<uint32_t*>(p) = w;
    } else {
        p[0] = (uint16_t)w;
        p[1] = (uint16_t)(w >> 16);
    }
}

// ------------------------------------------------------------------- host

constexpr int kTarget = 512;                 // work items wanted: two per CU
constexpr int kLeast = 8;                    // blocks of one piece, at least

struct HostPlan {
    int rows;                    // per tile
    int64_t segs, pieces, slots, grid;
};

HostPlan host_plan(int32_t B, int32_t n_q, int32_t Hq, int32_t Hkv, int32_t t_cap) {
    HostPlan p;
    const int64_t rows = (int64_t)n_q * (Hq / Hkv);
    p.rows = rows > 128 ? 256 : 128;
    p.segs = (int64_t)B * Hkv * ((rows + p.rows - 1) / p.rows);
    p.pieces = std::max<int64_t>(1, ((int64_t)t_cap / kBlk + kLeast) / kLeast);
    // (a plan that cuts has fewer than kTarget segments, each cut has at most one
    // piece more than an even share of the items wanted)
    p.slots = p.pieces == 1 ? 0 : std::min<int64_t>(2 * kTarget, p.segs * p.pieces);
    p.grid = (std::max(p.segs, p.slots) + 7) / 8 * 8;
    return p;
}

template <int SRC>
void launch_source(const ChunkArgs& a, const HostPlan& p, hipStream_t stream) {
    if (p.rows == 256)
        chunk_kernel<SRC, 8><<<dim3((unsigned)p.grid), 512, 0, stream>>>(a);
    else
        chunk_kernel<SRC, 4><<<dim3((unsigned)p.grid), 256, 0, stream>>>(a);
}

bool aligned16(const Q8Rows& r) {
    return ((reinterpret_cast<uintptr_t>(r.p) | (uintptr_t)(r.sb * 2) | (uintptr_t)(r.st * 2) | (uintptr_t)(r.sh * 2)) & 15) == 0;
}

}  // namespace

size_t chunk_workspace_bytes(int32_t B, int32_t n_q, int32_t Hq, int32_t Hkv, int32_t t_cap) {
    const HostPlan p = host_plan(B, n_q, Hq, Hkv, t_cap);
    return (size_t)p.slots * p.rows * (kD + 2) * sizeof(float);
}

int launch_chunk(const ChunkSource& src, const ChunkCall& c, void* ws, uint32_t* status, hipStream_t stream) {
    const HostPlan p = host_plan(c.B, c.n_q, c.Hq, c.Hkv, c.t_cap);
    ChunkArgs a;
    a.q = c.q.p;
    a.q_sb = c.q.sb;
    a.q_st = c.q.st;
    a.q_sh = c.q.sh;
    a.out = const_cast<uint16_t*>(c.out.p);
    a.o_sb = c.out.sb;
    a.o_st = c.out.st;
    a.o_sh = c.out.sh;
    const bool q8 = src.format != kChunkBf16;
    a.k = q8 ? src.cache.data[0] : reinterpret_cast<const uint8_t*>(src.k.p);
    a.v = q8 ? src.cache.data[1] : reinterpret_cast<const uint8_t*>(src.v.p);
    a.ks = src.cache.scale[0];
    a.vs = src.cache.scale[1];
    a.k_sb = src.k.sb;
    a.k_st = src.k.st;
    a.k_sh = src.k.sh;
    a.v_sb = src.v.sb;
    a.v_st = src.v.st;
    a.v_sh = src.v.sh;
    a.mask = src.mask;
    a.mask_sb = src.mask_sb;
    a.q_lens = c.q_lens;
    a.seq_lens = c.seq_lens;
    a.pg = src.pg;
    a.B = c.B;
    a.Hq = c.Hq;
    a.H = c.Hkv;
    a.G = c.Hq / c.Hkv;
    a.n_q = c.n_q;
    a.t_cap = c.t_cap;
    a.causal = c.causal;
    a.window = c.window;
    a.sinks = c.sinks;
    a.q_aligned = aligned16(c.q);
    a.kv_aligned = !q8 && aligned16(src.k) && aligned16(src.v);
    a.out_aligned = ((reinterpret_cast<uintptr_t>(c.out.p) | (uintptr_t)(c.out.sb * 2) | (uintptr_t)(c.out.st * 2) |
                      (uintptr_t)(c.out.sh * 2)) & 7) == 0;
    a.scale_log2 = fabsf(c.scale) * kLog2e;
    a.negative = c.scale < 0.f;
    a.target = kTarget;
    a.least = kLeast;
    a.status = status;
    a.ws_acc = static_cast<float*>(ws);
    a.ws_ml = a.ws_acc + p.slots * p.rows * kD;
    if (src.format == DQ_Q8_E4M3)
        launch_source<DQ_Q8_E4M3>(a, p, stream);
    else if (src.format == DQ_Q8_INT8)
        launch_source<DQ_Q8_INT8>(a, p, stream);
    else
        launch_source<kChunkBf16>(a, p, stream);
    if (int rc = hip_check("chunk launch", hipGetLastError())) return rc;
    if (p.slots == 0) return DQ_OK;
    // (segments are as many as the host counts where all chunks are full: then
    // it knows whether the plan cuts)
    if (!c.q_lens && p.segs >= kTarget) return DQ_OK;
    const dim3 grid((unsigned)(((int64_t)c.n_q * c.Hq + 3) / 4), c.B);
    if (p.rows == 256)
        chunk_merge_kernel<256><<<grid, 256, 0, stream>>>(a);
    else
        chunk_merge_kernel<128><<<grid, 256, 0, stream>>>(a);
    return hip_check("chunk_merge launch", hipGetLastError());
}

}  // namespace dq
