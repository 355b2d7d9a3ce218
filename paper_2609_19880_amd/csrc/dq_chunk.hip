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
// value block's scale goes into the exponent of the weights, relative to a power
// of 2 that follows what the row's blocks weigh.  Queries are brought to a largest
// magnitude of 2^13 to 2^14 by a power of 2 of each row: exactly down to 2^-30 of
// the largest (bf16's 8 bits above fp16's last, 2^-24), to 2^-38 of it below.
//
// Weights take the values' type, which the matrix instructions ask for: fp16 (11
// bits) over codes, bf16 (8 bits) over BF16 states, whose range fp16 does not hold.
// Where memory is what a call waits for (few rows) weights over BF16 states are two
// terms, 16 bits, and a product each; with many rows that would be half as much matrix
// work again, for an error beside the output's own rounding to bf16 of 0.0021 in place
// of 0.0017 in all.  The denominator is the sum of the rounded weights, so a common
// error of theirs cancels.
#include <float.h>
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
constexpr float kBig = 3e38f;
constexpr float kMostBf16 = 0x1.FEp127f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kRowsOf = 32;                  // rows per wavefront
constexpr float kNoScale = -1e30f;           // log2 of the scale of a block of zeros
constexpr float kNoRef = -1e29f;             // of what no sums are relative to (zeros are low beside it)

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
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
    int cuts;                    // pieces may be cut (0: every segment is one item)
    int planned;                 // the plan was made by a kernel of its own
    int groups;                  // of 64 sequences
    uint32_t* status;
    float* ws_acc;               // [slot][rows][128]: outputs of pieces
    float* ws_ml;                // [slot][2][rows]: their maxima and sums of weights
    int32_t* plan;               // the blocks of one piece, for the merge; planned: and what
                                 // find_item reads of 64 sequences at a time
};

// ------------------------------------------------------------------- shares
//
// A segment is a tile of rows of one (sequence, KV head).  Where there are
// fewer segments than would fill the GPU twice, or some have more blocks than a
// workgroup's share of all, their tokens are cut into pieces of `chunk` blocks;
// the pieces of a row are joined by the merge kernel.  Lengths are known on the
// device only, so every workgroup derives the same plan from them (of more than
// 64 sequences, or where the GPU is full anyway, a kernel of its own).

struct Seq {
    int T, n, tiles, units;      // tokens, new tokens, row tiles, most blocks that a row tile sees
};

// Sequences of few rows and of many have a kernel each (tiles: 0 for the other's).
// The border, measured on both sides: 64 x 10 queries over 1024 tokens (40 rows a
// head) take 54 us as few rows, 87 as many; 16 x 20 queries over 16384 tokens (80
// rows) 201 us as many, 288 as few with tiles of 128.
struct Few {
    static constexpr int kRows = 64;             // of a tile
    static constexpr bool kFew = true;
    static constexpr int kAtOnce = 256;          // workgroups that the GPU takes at a time: one per CU
    static constexpr int kCost = 16;             // what an item costs besides its blocks, in blocks
    static constexpr int kMergeRows = 8;         // of a merging workgroup
};
struct Many {
    static constexpr int kRows = 128;
    static constexpr bool kFew = false;
    static constexpr int kAtOnce = 768;          // three per CU
    static constexpr int kCost = 8;
    static constexpr int kMergeRows = 16;
};
constexpr int kLeast = 8;                        // blocks of one piece, at least (4: no faster)

template <typename K>
__device__ __forceinline__ Seq seq_of(const ChunkArgs& a, int b) {
    constexpr int R = K::kRows;
    Seq s;
    s.T = a.seq_lens ? max(0, min(a.seq_lens[b], a.t_cap)) : a.t_cap;
    s.n = a.q_lens ? max(0, min(a.q_lens[b], a.n_q)) : a.n_q;
    s.tiles = (s.n * a.G <= Few::kRows) == K::kFew ? (s.n * a.G + R - 1) / R : 0;
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

constexpr int kWhole = 0x7FFFFFFE;               // no piece is cut

// What pieces of c blocks take, `segs` segments' of `longest` blocks at most:
// rounds of as many as the GPU takes at a time, each its blocks and a piece's own cost.
template <typename K>
__host__ __device__ inline float plan_cost(float segs, int longest, int c) {
    const float items = segs * (float)((uint32_t)(longest + c - 1) / (uint32_t)c);
    if (items > 2 * K::kAtOnce && c < longest) return 3e38f;
    return ceilf(items / K::kAtOnce) * (float)(c + K::kCost);
}
// Blocks of a piece where a segment has n + 1 of them.
__host__ __device__ inline int plan_try(int longest, int n) {
    const int c = (int)((uint32_t)(longest + n) / (uint32_t)(n + 1));
    return c > kLeast ? c : kLeast;
}

// Sequence b0 + lane.
template <typename K>
__device__ __forceinline__ Seq seq_at(const ChunkArgs& a, int b0, int lane) {
    return b0 + lane < a.B ? seq_of<K>(a, b0 + lane) : Seq{0, 0, 0, 0};
}

// The blocks of one piece, of `segs` segments that have `total` blocks, the longest
// `longest`.  All lanes agree.
template <typename K>
__device__ __forceinline__ int plan_of(float total, float segs, int longest, int lane) {
    const bool full = segs >= 2 * K::kAtOnce;
    if (full || total < 0.75f * segs * (float)longest) {
        // Many segments: those longer than what each place has to do anyway are cut
        // (one sequence of 65536 tokens among 63 of 1024: 421 to 77 us).  Few:
        // unlike lengths leave pieces that are not full: small ones even out the end
        // (48 ragged chunks 600 us with pieces of what a place has, 616 to 630 with
        // 1.3 of it, or 1/1.5, 1/2 and 1/4)
        const int c = max((int)ceilf((full ? total + segs * K::kCost : total) / K::kAtOnce), kLeast);
        return c >= longest ? kWhole : c;
    }
    // lane l tries l + 1 pieces per segment
    const int c = plan_try(longest, lane);
    const float cost = plan_cost<K>(segs, longest, c), least = wave_min(cost);
    const int best = __builtin_amdgcn_readlane(c, __builtin_ctzll(__builtin_amdgcn_ballot_w64(cost == least)));
    return best >= longest ? kWhole : best;
}

// The same of all sequences, at most 64.  first: seq_at(a, 0, lane).
template <typename K>
__device__ __forceinline__ int plan_chunk(const ChunkArgs& a, const Seq& first, int lane) {
    // (sums in fp32: the same bits wherever they are taken; a chunk a millionth too
    // short adds an item, which the workspace has room for)
    float total, segs;
    int longest;
    if (a.B == 1) {
        const Seq q = seq_of<K>(a, 0);
        segs = (float)q.tiles;
        total = segs * (float)q.units;
        longest = q.units;
    } else {
        total = wave_sum((float)first.tiles * (float)first.units);
        segs = wave_sum((float)first.tiles);
        longest = wave_max(first.tiles ? first.units : 0);
    }
    return plan_of<K>(total * (float)a.H, segs * (float)a.H, longest, lane);
}

__device__ __forceinline__ int pieces(int units, int chunk) { return max(1, (units - 1) / chunk + 1); }

__device__ __forceinline__ int scan64(int v) {         // inclusive sums over the lanes
    v += dpp0<0x111, 0xF>(v);
    v += dpp0<0x112, 0xF>(v);
    v += dpp0<0x114, 0xF>(v);
    v += dpp0<0x118, 0xF>(v);
    v += dpp0<0x142, 0xA>(v);
    v += dpp0<0x143, 0xC>(v);
    return v;
}

// Work item `id`, or cut segment `id` (SEGMENT), with the slot of its (first) piece.
// Slots are those of cut segments, sequence after sequence, KV head after KV head,
// the last row tiles (which see most) first, their pieces in order.
//
// Workgroups go to the 8 XCDs in turn; what shares keys and values should meet in
// one L2, and all XCDs should have sequences of every length: each takes its
// heads of all sequences where there are a multiple of 8 (4 x 4096 queries over
// states of unlike lengths 2.57 to 2.11 ms), else an eighth of the items.  Items
// come in three passes, the whole pieces, the last ones of more than half a piece
// and the rest: short work evens out the end (48 ragged chunks 0.67 to 0.60 ms).
template <typename K, bool SEGMENT>
__device__ __forceinline__ Item find_item(const ChunkArgs& a, int id, int lane) {
    Item it{0, 0, -1, 0, kWhole, 0};
    if (a.cuts && (SEGMENT || a.planned)) it.chunk = *a.plan;
    if (SEGMENT && it.chunk == kWhole) return it;    // nothing to merge
    if (!a.cuts || (a.planned && it.chunk == kWhole)) {
        // every segment whole, as many as full chunks have: no lengths needed to find it
        const uint32_t tiles = K::kFew ? 1u : ((uint32_t)a.n_q * (uint32_t)a.G + K::kRows - 1) / K::kRows;
        const bool heads8 = a.H % 8 == 0;
        const uint32_t heads = heads8 ? (uint32_t)a.H / 8 : (uint32_t)a.H, all = (uint32_t)a.B * heads * tiles;
        uint32_t x = (uint32_t)id >> 3;
        if (!heads8) {
            const uint32_t per = (all + 7) / 8;
            if (x >= per) return it;
            x += (uint32_t)(id & 7) * per;
        }
        if (x >= all) return it;
        const uint32_t r = x / tiles;
        it.b = (int)(r / heads);
        it.h = (int)(r % heads);
        if (heads8) it.h = 8 * it.h + (id & 7);
        it.tile = (int)(tiles - 1 - x % tiles);
        if (it.tile >= seq_of<K>(a, it.b).tiles) it.tile = -1;
        return it;
    }
    const bool by_head = !SEGMENT && a.H % 8 == 0;
    Seq first{0, 0, 0, 0};
    if (a.B > 1 || !(SEGMENT || by_head)) first = seq_at<K>(a, 0, lane);
    if (!SEGMENT && !a.planned) {
        it.chunk = plan_chunk<K>(a, first, lane);
        if (id == 0 && threadIdx.x == 0) *a.plan = it.chunk;
    }
    const int heads = by_head ? a.H / 8 : a.H;   // of those that x counts
    int x = by_head ? id >> 3 : id;
    // pieces of a sequence's segment in a pass
    auto full = [&](int units) { return (int)((uint32_t)units / (uint32_t)it.chunk); };
    auto in_pass = [&](int units, int pass) {
        if (SEGMENT) return (int)(units > it.chunk);
        const int n = full(units);
        if (pass == 0) return n;
        const int rest = units - n * it.chunk;
        return (int)(rest > it.chunk / 2 ? pass == 1 : (rest > 0 || n == 0) && pass == 2);
    };
    if (!SEGMENT && !by_head) {
        const int all = a.planned ? a.plan[1] * heads : wave_sum(first.tiles * heads * pieces(first.units, it.chunk));
        const int per = (all + 7) / 8;
        if ((id >> 3) >= per) return it;
        x = (id & 7) * per + (id >> 3);
    }
    // of sequence b, whose first slot is `slot`: entry r of a pass
    auto entry = [&](int b, int tiles, int units, int slot, int pass, int r) {
        const uint32_t each = (uint32_t)in_pass(units, pass), t = (uint32_t)r / each, h = t / (uint32_t)tiles;
        const int late = (int)(t - h * (uint32_t)tiles);
        it.b = b;
        it.h = by_head ? 8 * (int)h + (id & 7) : (int)h;
        it.tile = tiles - 1 - late;
        it.c = SEGMENT ? 0 : pass == 0 ? r - (int)(t * each) : full(units);
        it.slot = slot + (it.h * tiles + late) * pieces(units, it.chunk) + it.c;
    };
    for (int pass = SEGMENT || it.chunk != kWhole ? 0 : 2; pass < (SEGMENT ? 1 : 3); ++pass) {
        if (a.B == 1) {
            // (uniform arithmetic, no sums over the lanes)
            const Seq s = seq_of<K>(a, 0);
            const int own = s.tiles * heads * in_pass(s.units, pass);
            if (x < own) {
                entry(0, s.tiles, s.units, 0, pass, x);
                return it;
            }
            x -= own;
            continue;
        }
        int before = 0, slots = 0, b0 = 0;
        if (a.planned) {
            // the 64 sequences that have the item, from the plan
            const int32_t* counts = a.plan + 4 + (SEGMENT ? 3 : pass) * a.groups;
            const int32_t* held_of = a.plan + 4 + 4 * a.groups;
            bool found = false;
            for (int g0 = 0; g0 < a.groups && !found; g0 += kWave) {
                const bool in = g0 + lane < a.groups;
                const int own = in ? counts[g0 + lane] * heads : 0, held = in ? held_of[g0 + lane] * a.H : 0;
                const int upto = before + scan64(own), held_upto = slots + scan64(held);
                const int last = __builtin_amdgcn_readlane(upto, 63);
                found = x < last;
                const int l = found ? __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > x)) : 63;
                before = found ? __builtin_amdgcn_readlane(upto - own, l) : last;
                slots = __builtin_amdgcn_readlane(found ? held_upto - held : held_upto, l);
                b0 = (g0 + l) * kWave;
            }
            if (!found) {
                x -= before;
                continue;
            }
        }
        // (not planned: all sequences)
        const Seq s = b0 == 0 ? first : seq_at<K>(a, b0, lane);
        const int own = s.tiles * heads * in_pass(s.units, pass), n = pieces(s.units, it.chunk);
        const int held = n > 1 ? s.tiles * a.H * n : 0;
        const int upto = before + scan64(own);
        const int last = __builtin_amdgcn_readlane(upto, 63);
        const int held_upto = slots + scan64(held);
        if (x < last) {
            const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > x));
            entry(b0 + l, __builtin_amdgcn_readlane(s.tiles, l), __builtin_amdgcn_readlane(s.units, l),
                  __builtin_amdgcn_readlane(held_upto - held, l), pass, x - __builtin_amdgcn_readlane(upto - own, l));
            return it;
        }
        x -= last;
    }
    return it;
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

// A uniform address of memory that this kernel does not write, through the
// scalar unit, beside the vector loads' order.
template <typename T>
__device__ __forceinline__ T scalar_load(const T* p) {
    return *reinterpret_cast<const __attribute__((address_space(4))) T*>(reinterpret_cast<uintptr_t>(p));
}

__device__ __forceinline__ float clamped(float x) {    // NaN stays
    x = x > kBig ? kBig : x;
    return x < -kBig ? -kBig : x;
}

// (infinities and NaN: NaN)
__device__ __forceinline__ float log_scale(float x) {
    return x == 0.f ? kNoScale : __builtin_amdgcn_logf(x) + (x - x);
}

// Two rounded weights' sum added to x, in fp32.
template <int SRC>
__device__ __forceinline__ float plus_weights(uint32_t w, float x) {
    if constexpr (SRC == kChunkBf16)
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), bf16x2{(__bf16)1.f, (__bf16)1.f}, x, false);
    else
        return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, w), f16x2{(_Float16)1.f, (_Float16)1.f}, x, false);
}

// ------------------------------------------------------- rows of a wavefront

// What 32 rows (one wavefront's) hold: queries as the first product's operand,
// sums, and the softmax state.  The lanes l and l ^ 32 share row l % 32; each
// has the scores of 16 of a block's 32 tokens, 8 (i / 4) + 4 (l / 32) + i % 4.
//
// The state's maximum m, a whole number, is not the running maximum but one that the
// sums keep until a block's weights, relative to it, add up to more than 2^15: weights
// of m itself are 2^2, so fp16 holds what lies 2^13 above and, to its 11 bits, 2^16
// below (to 2^-25 beyond; over codes times the 2^-2 or more of the block's scale that
// they hold).  Most blocks so need no maximum and scale nothing: their weights are
// computed with the m at hand and only checked (a running maximum adds 16 maxima, an
// exchange between two lanes and 64 products to the 126 vector instructions that a
// block takes).  A row's bits do not depend on the rows beside it, but where their
// scores pass 2^11.  (BF16: m itself weighs 1.  Any limit would do for bf16's range;
// 2^60 in place of 2^15 is no faster, 2^8 loses 4 %, and larger weights bring the sums
// of large values nearer to their end.)
//
// FINE: weights are two terms, p[2 + st] what rounding p[st] has left.
template <int SRC, bool FINE>
struct Rows {
    static constexpr bool q8 = SRC != kChunkBf16;
    static constexpr int kTerms = FINE ? 2 : 1;
    static constexpr float kUp = q8 ? 2.f : 0.f;
    static constexpr float kMost = 0x1p15f;

    u32x4 q[8];
    f32x16 o[4];
    float m, l, vref, qc;        // vref: log2 of the scale that the row's sums are relative to, an integer
    float off;                   // weights are exp2(score + off + log2 of the values' scale)
    int end;                     // the row sees t < end, of those t < sinks or t >= end - window
    int T, window, sinks;
    int lim_lo, lim_hi, start_hi;
    bool live, careful;   // careful: a row has no maximum yet, or one of 2^11 or more

    __device__ __forceinline__ void load(const ChunkArgs& a, const Sees& see, int b, int h, int r0, int rows, int lane) {
        const int half = lane >> 5, r = r0 + (lane & 31);
        const bool valid = r < rows;
        const int row = min(r, rows - 1), token = row / a.G, head = h * a.G + (row - token * a.G);
        live = r0 < rows;
        T = see.T;
        window = a.window > 0 ? a.window : 0x7FFFFFFF;
        sinks = a.sinks;
        end = a.causal ? see.off + token + 1 : T;                                // (may be negative)
        auto start = [&](int e) { return e <= window ? 0 : e - window; };
        lim_lo = max(0, min(T, __builtin_amdgcn_readfirstlane(end)));            // rows are in order
        lim_hi = max(0, min(T, __builtin_amdgcn_readlane(end, 31)));
        start_hi = start(__builtin_amdgcn_readlane(end, 31));
        m = -INFINITY;
        l = 0.f;
        vref = kNoRef;
        off = offset();
        qc = a.scale_log2;
        careful = true;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = f32x16{};
        const uint16_t* p = a.q + (int64_t)b * a.q_sb + (int64_t)token * a.q_st + (int64_t)head * a.q_sh;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            // channels of operand j: as the keys' pieces hold them, or in order
            const int ch = q8 ? 16 * (2 * (j >> 1) + half) + 8 * (j & 1) : 16 * j + 8 * half;
            q[j] = u32x4{0u, 0u, 0u, 0u};
            if (valid) {
                if (a.q_aligned) {
                    q[j] = *reinterpret_cast<const u32x4*>(p + ch);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        q[j][i] = (uint32_t)p[ch + 2 * i] | ((uint32_t)p[ch + 2 * i + 1] << 16);
                }
            }
            if (a.negative) q[j] ^= 0x80008000u;
        }
        int top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                top = max(top, max((int)(q[j][i] & 0x7FFFu), (int)((q[j][i] >> 16) & 0x7FFFu)));
        top = max(top, __float_as_int(xor_lane<32>(__int_as_float(top), lane)));
        const bool nan = top >= 0x7F80;          // infinities and NaN make the row NaN, if it sees a token
        if constexpr (q8) {
            if (nan && end > 0 && T > 0) l = NAN;
            const int up = 13 - (top >= 0x80 ? (top >> 7) - 127 : -126);
            qc = ldexpf(qc, -up);
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x = ldexpf(__uint_as_float(q[j][i] << 16), up);
                    const float y = ldexpf(__uint_as_float(q[j][i] & 0xFFFF0000u), up);
                    q[j][i] = nan ? 0u : weights2<SRC>(x, y);
                }
        } else if (nan) {                        // (one NaN channel: NaN with every key)
            q[0][0] = 0x7FC07FC0u;
        }
    }

    // Operands 4 part .. of the keys.
    __device__ __forceinline__ void scores(f32x16& s, int part, const u32x4 (&kf)[4]) const {
        if (part == 0) s = f32x16{};
#pragma unroll
        for (int j = 0; j < 4; ++j) s = mma<SRC>(kf[j], q[4 * part + j], s);
    }

    // The weights exp2(s c + e) and their sum, of the rounded ones.
    __device__ __forceinline__ float weigh(const f32x16& s, float c, float e, u32x4 (&p)[2 * kTerms]) const {
        float sum = 0.f;
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = 4 * st + 8 * (i >> 1) + 2 * (i & 1);
                float x = __builtin_amdgcn_exp2f(fmaf(s[at], c, e));
                float y = __builtin_amdgcn_exp2f(fmaf(s[at + 1], c, e));
                if constexpr (FINE) {            // (infinity would leave NaN)
                    x = x > kMostBf16 ? kMostBf16 : x;
                    y = y > kMostBf16 ? kMostBf16 : y;
                }
                p[st][i] = weights2<SRC>(x, y);
                sum = plus_weights<SRC>(p[st][i], sum);
                if constexpr (FINE) {
                    p[2 + st][i] = weights2<SRC>(x - __uint_as_float(p[st][i] << 16),
                                                 y - __uint_as_float(p[st][i] & 0xFFFF0000u));
                    sum = plus_weights<SRC>(p[2 + st][i], sum);
                }
            }
        return sum;
    }

    __device__ __forceinline__ float mu() const { return m == -INFINITY ? 0.f : m; }
    __device__ __forceinline__ int relative_to() const { return q8 ? (int)fmaxf(vref, -400.f) : 0; }
    __device__ __forceinline__ float offset() const { return q8 ? kUp - mu() - vref : kUp - mu(); }

    // The softmax of a block whose scores are s, times c: p are its weights.
    // t0: the block's first token; shown: bit t of it is clear where token t is
    // hidden; vl: log2 of the values' scale, kNoScale for a block of zeros (any
    // weight will do), NaN for one that is no number (rows that see it become NaN).
    __device__ __forceinline__ void block(f32x16& s, float c, float vl, int t0, uint32_t shown, int lane,
                                          u32x4 (&p)[2 * kTerms]) {
        c = fmaxf(c, 0x1p-120f);                 // (a factor of 0, which hidden scores could not bear)
        if (shown != ~0u || t0 + kBlk > lim_lo || (start_hi > 0 && t0 < start_hi && t0 + kBlk > sinks)) {
            auto below = [&](int t) { return t <= t0 ? 0u : t - t0 >= kBlk ? ~0u : (1u << (t - t0)) - 1u; };
            const uint32_t past = end <= window ? 0u : below(end - window);
            const uint32_t vis = (shown & below(min(end, T)) & (~past | below(sinks))) >> (4 * (lane >> 5));
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = (vis >> (8 * (e >> 2) + (e & 3))) & 1 ? s[e] : -INFINITY;
        }
        // Of the scale the weights hold 2^-2 and more (as long as they fit): less would
        // cost them bits of fp16, however much the block weighs.
        float d = 0.f;
        bool low = false;
        if constexpr (q8) {
            d = vl - vref;
            low = !(d >= -2.f);                  // (a block of zeros too, and one that is no number)
        }
        float sum = weigh(s, c, q8 ? off + vl : off, p);
        if (careful || (__builtin_amdgcn_ballot_w64(low) | __builtin_amdgcn_ballot_w64(sum > kMost)) != 0)
            sum = anew(s, c, sum, vl, low, d, lane, p);
        l += q8 ? sum * __builtin_amdgcn_exp2f(-d) : sum;
    }

    // The same with a new maximum or a new scale; d becomes the block's.  sum: of
    // the weights without them.  (Selections rather than branches, and one place
    // that scales the sums: with branches the compiler keeps both results.)
    //
    // What a row's sums are relative to, 2^(m + vref), goes by what its blocks weigh, a
    // scale times a weight: a block that is not seen, or weighs next to nothing, changes
    // nothing however large it is, one that makes up the output by its size alone keeps its
    // bits, and so do values beside zeros that have nearly all weight.  vref is
    // - the block's scale, rounded up to a power of 2 or twice that (room for others),
    //   times its largest weight, where the weights would not fit;
    // - its scale, where the weights would lose bits of it (low);
    // - or else as much lower as the maximum is higher.
    // Sums are scaled by a power of 2, exactly: down to 2^-126, up as far as they
    // stay below 2^124 (from sums of usual weights, 2^2 or less, by over 2^100).  Where
    // that is not enough the block's values are nothing beside the row's sums, and are
    // left out.
    __device__ __forceinline__ float anew(f32x16& s, float c, float sum, float vl, bool low, float& d, int lane,
                                          u32x4 (&p)[2 * kTerms]) {
        float top = s[0];                        // (NaN where every score is)
#pragma unroll
        for (int e = 1; e < 16; ++e) top = fmaxf(top, s[e]);
        if constexpr (!q8) l = top == INFINITY ? NAN : l;    // as the formula has it
        top *= c;
        // scores so large that a fused product would differ from the maximum by
        // more than a rounding of it
        const float high = top == -INFINITY ? 0.f : fabsf(top);
        const bool exact = __builtin_amdgcn_ballot_w64(fmaxf(fabsf(mu()), high) >= 0x1p11f) != 0;
        top = top == -INFINITY ? top : clamped(top);
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = exact && s[e] != -INFINITY ? clamped(s[e] * c) : s[e];
        top = ceilf(fmaxf(top, xor_lane<32>(top, lane)));            // (so that all scaling is by powers of 2)
        sum = fmaxf(sum, xor_lane<32>(sum, lane));
        const bool higher = (m == -INFINITY || (exact || low ? top > m + 4.f : sum > kMost)) && top > m;
        const float rise = higher && m != -INFINITY ? top - m : 0.f;
        float by = higher ? m - top : 0.f;
        l *= __builtin_amdgcn_exp2f(by);
        m = higher ? top : m;
        bool whole = true;                       // the weights hold the block's scale
        if constexpr (q8) {
            const bool seen = top != -INFINITY;
            l = seen && vl != vl ? NAN : l;
            // (no further down than a weight of 2^-200, which is nothing)
            const float weighs = vl + fmaxf(fminf(top - m, 0.f), -200.f), base = vref - rise;
            const bool over = weighs > base && (higher || sum > kMost || (exact && weighs > base + 4.f));
            float to = floorf(low ? vl : weighs) + 1.f;      // (room for scales of up to twice the size)
            to = seen && vl > kNoScale && (low || over) ? to : base;
            // (by any step: they add up)
            if (__builtin_amdgcn_ballot_w64(base > to) != 0) to = fmaxf(to, base - most_up(lane));
            by += vref - to;
            vref = to;
            whole = vl > kNoScale && vl - vref >= -2.f;
            d = whole ? vl - vref : 0.f;
        }
        off = offset();
        const int shift = (int)fmaxf(fminf(by, 400.f), -400.f);      // (zeros may have any: they stay)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[i][e] = ldexpf(o[i][e], shift);
        careful = __builtin_amdgcn_ballot_w64(!(fabsf(m) < 0x1p11f)) != 0;
        // (large scores: the difference first, which is exact where it counts)
        const float less = exact ? mu() : 0.f, e0 = exact ? kUp + d : !whole ? kUp - mu() : q8 ? off + vl : off;
        c = exact ? 1.f : c;
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] -= less;
        const float rounded = weigh(s, c, e0, p);
        if constexpr (q8)
#pragma unroll
            for (int st = 0; st < 2; ++st)
#pragma unroll
                for (int i = 0; i < 4; ++i) p[st][i] = whole ? p[st][i] : 0u;
        return rounded;
    }

    // By how many powers of 2 the row's sums may grow: zeros by any.
    __device__ __forceinline__ float most_up(int lane) const {
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, fabsf(o[i][e]));
        top = fmaxf(top, xor_lane<32>(top, lane));
        return top == 0.f ? 1e4f : 124.f - fmaxf(ceilf(__builtin_amdgcn_logf(top)), 0.f);
    }

    // The values of half of a block's tokens.
    __device__ __forceinline__ void values(const u32x4 (&vf)[4], const u32x4& p) {
#pragma unroll
        for (int np = 0; np < 4; ++np) o[np] = mma<SRC>(vf[np], p, o[np]);
    }
};

// -------------------------------------------------------------- the kernel


// A step's keys and values (64 tokens) in LDS.  Keys: operand j of a block at
// kKeyOp j, a lane's 16 bytes at half (kKeyOp / 2) + 16 (token % 32).  Codes
// become fp16; values of codes lie as their operands do (2 np + st, 1 KB each),
// BF16 values as rows that the LDS reads transposed.  Where rows of BF16 are
// written a piece of 8 channels at a time, 16 (keys) and 64 bytes (values) of
// padding keep the 16 pieces of a row in different banks.
template <int SRC>
struct Lds {
    static constexpr bool q8 = SRC != kChunkBf16;
    static constexpr int kKeyOp = q8 ? 1024 : 1056;
    static constexpr int kKeys = 8 * kKeyOp;
    static constexpr int kValRow = 320;
    static constexpr int kStage = kKeys + (q8 ? 8192 : kBlk * kValRow);
};

typedef const __attribute__((address_space(1))) uint8_t* GlobalBytes;
typedef const __attribute__((address_space(1))) float* GlobalFloats;
typedef const __attribute__((address_space(1))) int32_t* GlobalInts;
typedef const __attribute__((address_space(1))) u32x4* GlobalPieces;

// Eight channels of a BF16 row.
__device__ __forceinline__ u32x4 row_piece(const uint16_t* x, bool aligned) {
    if (aligned) return *reinterpret_cast<GlobalPieces>(reinterpret_cast<uintptr_t>(x));
    u32x4 r;
#pragma unroll
    for (int w = 0; w < 4; ++w) r[w] = (uint32_t)x[2 * w] | ((uint32_t)x[2 * w + 1] << 16);
    return r;
}

// Of a block's tokens, bit by bit, the first n (rows behind the last token are
// read as the last one's and hidden).
__device__ __forceinline__ uint32_t shown_to(int n) { return n >= kBlk ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }

template <int SRC>
__device__ __forceinline__ void read_keys(const char* at, int part, int lane, u32x4 (&kf)[4]) {
    const char* p = at + (lane >> 5) * (Lds<SRC>::kKeyOp / 2) + (lane & 31) * 16;
#pragma unroll
    for (int j = 0; j < 4; ++j) kf[j] = *reinterpret_cast<const u32x4*>(p + (4 * part + j) * Lds<SRC>::kKeyOp);
}

template <int SRC>
__device__ __forceinline__ void read_values(const char* at, int st, int lane, u32x4 (&vf)[4]) {
    if constexpr (Lds<SRC>::q8) {
#pragma unroll
        for (int np = 0; np < 4; ++np) vf[np] = *reinterpret_cast<const u32x4*>(at + (2 * np + st) * 1024 + lane * 16);
    } else {
        // four rows of 16 channels, transposed: tokens 8 st + 4 half + 0..3, then 16 further on
        const char* p = at + (4 * (lane >> 5) + ((lane >> 2) & 3)) * Lds<SRC>::kValRow + ((lane >> 4) & 1) * 32 +
                        (lane & 3) * 8 + 8 * st * Lds<SRC>::kValRow;
        typedef __attribute__((address_space(3))) i16x4* LdsRows;
#pragma unroll
        for (int np = 0; np < 4; ++np) {
            const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsRows)(p + 64 * np));
            const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsRows)(p + 64 * np + 16 * Lds<SRC>::kValRow));
            const u32x2 l2 = __builtin_bit_cast(u32x2, lo), h2 = __builtin_bit_cast(u32x2, hi);
            vf[np] = u32x4{l2[0], l2[1], h2[0], h2[1]};
        }
    }
}

// Infinities (and NaN) of BF16 values made zeros: what the weights' first terms have
// made of them stays as it is, whatever the second ones' signs are.
__device__ __forceinline__ void zeros_for_infinities(u32x4 (&vf)[4]) {
    u16x2 top = {0, 0};
#pragma unroll
    for (int np = 0; np < 4; ++np)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, vf[np][i] & 0x7FFF7FFFu));
    if (__builtin_amdgcn_ballot_w64(top[0] >= 0x7F80 || top[1] >= 0x7F80) == 0) return;
#pragma unroll
    for (int np = 0; np < 4; ++np)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w = vf[np][i];
            vf[np][i] = ((w & 0x7F80u) == 0x7F80u ? 0u : w & 0xFFFFu) |
                        ((w & 0x7F800000u) == 0x7F800000u ? 0u : w & 0xFFFF0000u);
        }
}

__device__ __forceinline__ void store_row(const ChunkArgs& a, int b, int token, int head, int ch, uint32_t w0,
                                          uint32_t w1) {
    uint16_t* x = a.out + (int64_t)b * a.o_sb + (int64_t)token * a.o_st + (int64_t)head * a.o_sh + ch;
    if (a.out_aligned) {
        *reinterpret_cast<u32x2*>(x) = u32x2{w0, w1};
    } else {
        x[0] = (uint16_t)w0;
        x[1] = (uint16_t)(w0 >> 16);
        x[2] = (uint16_t)w1;
        x[3] = (uint16_t)(w1 >> 16);
    }
}

constexpr int kThreads = 4 * kWave;

// A part's share in a row whose largest maximum is `top`, before division by the
// sum of all shares.  (Parts are joined as outputs, the sums divided by their
// weights: as sums the largest values, times weights of up to 2^15, would not fit.)
__device__ __forceinline__ float share(float m, float l, float top) {
    return l * (m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top));
}
__device__ __forceinline__ float inverse(float l) { return l == 0.f ? 0.f : 1.f / l; }   // rows that see nothing: zeros

// A sum, divided by its weights' and times the 2^up that it is relative to.
__device__ __forceinline__ float output(float sum, float f, int up) { return ldexpf(sum * f, up); }

// The outputs of a workgroup's wavefronts joined in LDS and written: wavefront
// w has rows 32 (w % parts) .. of the tokens that it has seen.  PAIRED: operand 2 m + e
// has channels 64 m + 32 (row / 16) + 16 e + row % 16, else 32 (2 m + e) + row.
constexpr int kJoinRow = 68;                     // floats: 64 channels, and 4 to keep rows in different banks

template <typename K, int WAVES, bool PAIRED>
__device__ __forceinline__ void join_rows(const ChunkArgs& a, const f32x16 (&o)[4], float m, float l, int up,
                                          float* join, float (&wm)[WAVES][kRowsOf], float (&wl)[WAVES][kRowsOf],
                                          float (&each)[WAVES][kRowsOf], int parts, int rows, int r0, int b, int h,
                                          bool whole, int64_t slot) {
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave, half = lane >> 5, col = lane & 31;
    const float f = inverse(l);
    if (half == 0) {
        wm[wave][col] = m;
        wl[wave][col] = l;
    }
#pragma unroll
    for (int m2 = 0; m2 < 2; ++m2) {             // channels 64 m2 ..
        __syncthreads();                         // (the area may still be read)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int ch = PAIRED ? 32 * (i >> 1) + 16 * e + 8 * (i & 1) + 4 * half : 32 * e + 8 * i + 4 * half;
                const f32x16& x = o[2 * m2 + e];
                *reinterpret_cast<f32x4*>(join + (wave * kRowsOf + col) * kJoinRow + ch) =
                    f32x4{output(x[4 * i], f, up), output(x[4 * i + 1], f, up), output(x[4 * i + 2], f, up),
                          output(x[4 * i + 3], f, up)};
            }
        if (m2 == 0 && tid < WAVES * kRowsOf) {  // (the shares, once; by every thread for itself: 1.5 us more)
            const int w = tid / kRowsOf, row = tid % kRowsOf;
            float top = -INFINITY, sum = 0.f;
            for (int x = w & (parts - 1); x < WAVES; x += parts) top = fmaxf(top, wm[x][row]);
            for (int x = w & (parts - 1); x < WAVES; x += parts) sum += share(wm[x][row], wl[x][row], top);
            each[w][row] = share(wm[w][row], wl[w][row], top) * inverse(sum);
            const int in = w * kRowsOf + row;
            if (!whole && w < parts && r0 + in < rows) {
                a.ws_ml[slot * 2 * K::kRows + in] = top;
                a.ws_ml[slot * 2 * K::kRows + K::kRows + in] = sum;
            }
        }
        __syncthreads();
        for (int i = tid; i < parts * kRowsOf * 16; i += WAVES * kWave) {
            const int in = i >> 4, ch = (i & 15) * 4, r = r0 + in;
            if (r >= rows) break;
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
            for (int w = in >> 5; w < WAVES; w += parts)
                acc += *reinterpret_cast<const f32x4*>(join + (w * kRowsOf + (in & 31)) * kJoinRow + ch) * each[w][in & 31];
            if (whole) {
                const int token = r / a.G, head = h * a.G + r - token * a.G;
                store_row(a, b, token, head, 64 * m2 + ch, bf16_two(acc[0], acc[1]), bf16_two(acc[2], acc[3]));
            } else {
                *reinterpret_cast<f32x4*>(a.ws_acc + (slot * K::kRows + in) * kD + 64 * m2 + ch) = acc;
            }
        }
    }
}

// One workgroup of four wavefronts per item: 128 rows, 32 per wavefront.  A
// block's codes are read, converted to fp16 once for the workgroup and laid into
// LDS as the products take them while the block before is worked on: one barrier
// per block.  Three wavefronts per SIMD, of three workgroups, hide one another's
// waits; more would leave too few registers for the sums (64), the queries (32)
// and a block's scores.
//
// Bound by no single unit: 4 x 8171 queries over themselves (32 heads, int8) run at
// 910 to 965 TFLOP/s, where the matrix units are busy 44 % of the time, other vector
// instructions (126 per wavefront and block, 16 of them exponentials) issue about
// as long, LDS is active 34 %, and the clock falls to 1.8 or 1.9 GHz.  Left out one at a
// time, the softmax's arithmetic gives back 16 %, the second product 9 %, loads 8 %,
// exponentials 5 %, the weights' sums or the conversions 2 to 3 %.  Twelve wavefronts
// per workgroup take 2 to 5 % less on the largest cases and more on the others: left
// as it is, one form for all.  Not faster: two wavefronts per SIMD with the blocks'
// steps interleaved, two or three blocks requested ahead, wavefront priorities.
template <int SRC>
__global__ __launch_bounds__(kThreads, 3) void chunk_kernel(ChunkArgs a) {
    typedef Lds<SRC> L;
    constexpr bool q8 = L::q8;
    constexpr int kPieces = q8 ? 2 : 4;          // 16-byte pieces per thread and block: keys, then values
    __shared__ __attribute__((aligned(16))) char lds[2 * L::kStage];
    __shared__ float2 lscale[2];                 // the keys' scale, log2 of the values'

    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const Item it = find_item<Many, false>(a, (int)blockIdx.x, lane);
    if (it.tile < 0) return;
    const int b = __builtin_amdgcn_readfirstlane(it.b), h = __builtin_amdgcn_readfirstlane(it.h);
    const int tile = __builtin_amdgcn_readfirstlane(it.tile), piece = __builtin_amdgcn_readfirstlane(it.c);
    const int chunk = __builtin_amdgcn_readfirstlane(it.chunk);
    const Seq seq = seq_of<Many>(a, b);
    const int rows = seq.n * a.G;                // of the whole sequence
    const int r0 = tile * Many::kRows;
    const Sees see = sees(a, seq, r0, min(r0 + Many::kRows, rows));
    const bool whole = pieces(see.count, chunk) == 1;
    const int u0 = (int)min((int64_t)piece * chunk, (int64_t)0x7FFFFF00);
    if (u0 >= see.count && piece > 0) return;    // the merge does not ask for it
    const int u1 = (int)min((int64_t)u0 + chunk, (int64_t)see.count);

    Rows<SRC, false> me;
    me.load(a, see, b, h, r0 + wave * kRowsOf, rows, lane);

    // ------------------------------------------------ loads
    bool bad = false;
    auto block_of = [&](int u) { return u < see.head ? u : see.from + (u - see.head); };
    u32x4 reg[kPieces];
    // Codes: pages are looked up a block before they are needed, in the vector
    // loads' order, and the scales come with the codes: nothing here waits for
    // memory, as a scalar load would make every wait for LDS do.  Block `at` lies
    // at page (H per_page) + h per_page + at % per_page; without a table the
    // sequence is the page.
    float sreg = 0.f;
    int page = b;
    const int per_page = a.pg.bt ? 1 << (a.pg.page_shift - 5) : a.t_cap / kBlk;
    const int in_page = a.pg.bt ? per_page - 1 : 0x7FFFFFFF, pages = a.pg.bt ? a.pg.num_pages : a.B;
    const uint32_t page_blocks = (uint32_t)(a.H * per_page);
    const int64_t head_blocks = (int64_t)h * per_page;
    GlobalInts table = (GlobalInts)(uintptr_t)(a.pg.bt + (a.pg.bt ? (int64_t)b * a.pg.max_pages : 0));
    GlobalBytes k_codes = (GlobalBytes)(uintptr_t)a.k, v_codes = (GlobalBytes)(uintptr_t)a.v;
    GlobalFloats scales = (GlobalFloats)(uintptr_t)(wave ? a.vs : a.ks);         // (wavefronts 0 and 1)
    uint32_t none = 0;                           // an offset that the compiler takes for a lane's
    asm("" : "+v"(none));
    // BF16: this thread's piece of rows 16 i + tid / 16
    const uint16_t* k_row = nullptr;
    const uint16_t* v_row = nullptr;
    int64_t k_st = 0, v_st = 0;
    if constexpr (!q8) {
        k_st = a.k_st;
        v_st = a.v_st;
        k_row = reinterpret_cast<const uint16_t*>(a.k) + b * a.k_sb + h * a.k_sh + 8 * (tid & 15);
        v_row = reinterpret_cast<const uint16_t*>(a.v) + b * a.v_sb + h * a.v_sh + 8 * (tid & 15);
    }
    auto look_up = [&](int u) {
        if (q8 && a.pg.bt && u < u1) page = table[((block_of(u) * kBlk) >> a.pg.page_shift) + none];
    };
    // requests block u
    auto request = [&](int u) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) reg[i] = u32x4{0u, 0u, 0u, 0u};
        if (u >= u1) return;
        if constexpr (q8) {
            const int at = __builtin_amdgcn_readfirstlane(page);
            const bool in = (uint32_t)at < (uint32_t)pages;
            bad = bad || !in;
            const int64_t bi = (int64_t)((uint64_t)(uint32_t)(in ? at : 0) * page_blocks) + head_blocks +
                               (block_of(u) & in_page);
            // (the empty statement keeps the block's address in scalar registers)
            GlobalBytes kp = k_codes + bi * kBlkBytes, vp = v_codes + bi * kBlkBytes;
            asm("" : "+s"(kp), "+s"(vp));
            reg[0] = *reinterpret_cast<GlobalPieces>(kp + 16u * (uint32_t)tid);
            reg[1] = *reinterpret_cast<GlobalPieces>(vp + 16u * (uint32_t)tid);
            if (wave < 2) sreg = (scales + bi)[none];
        } else {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int t = min(u * kBlk + 16 * (i & 1) + (tid >> 4), see.T - 1);
                reg[i] = row_piece(i >> 1 ? v_row + t * v_st : k_row + t * k_st, a.kv_aligned);
            }
        }
    };
    // BF16: the mask's byte of token lane % 32 of a block, and the tokens it shows
    uint32_t mreg = 0;
    const uint8_t* mask = !q8 && a.mask ? a.mask + b * a.mask_sb : nullptr;
    auto request_mask = [&](int u) {
        if (mask) {
            const int t = u * kBlk + (lane & 31);
            mreg = u < u1 && t < see.T ? mask[t] : 0;
        }
    };
    // of block u, whose mask was requested last
    auto shown_now = [&](int u) -> uint32_t {
        const uint32_t all = mask ? (uint32_t)__builtin_amdgcn_ballot_w64(mreg != 0) : ~0u;
        return q8 ? all : all & shown_to(see.T - u * kBlk);
    };
    auto keys_at = [&](int step) { return lds + (step & 1) * L::kStage; };
    auto values_at = [&](int step) { return lds + (step & 1) * L::kStage + L::kKeys; };
    // where this thread's pieces of stage 0 go
    int k_to, v_to;
    if constexpr (q8) {
        // piece ((t / 16) 2 + c / 64) 64 + ((c / 16) % 4) 16 + t % 16
        const int t = ((tid >> 7) << 4) | (tid & 15), slice = ((tid >> 6) & 1) * 4 + ((tid >> 4) & 3);
        k_to = (slice >> 1) * 2048 + (slice & 1) * 512 + t * 16;
        // piece ((c / 32) 4 + (t / 4) % 4) 16 + c % 16
        const int np = tid >> 6, grp = (tid >> 4) & 3;
        v_to = L::kKeys + (np * 2 + (grp >> 1)) * 1024 + (grp & 1) * 512 + (tid & 15) * 16;
    } else {
        k_to = (tid & 15) * (L::kKeyOp / 2) + (tid >> 4) * 16;
        v_to = L::kKeys + (tid >> 4) * L::kValRow + (tid & 15) * 16;
    }
    // lays what was requested into step `step`; of the values, those that `shown` shows
    auto lay = [&](int step, uint32_t shown) {
        char* to = lds + (step & 1) * L::kStage;
        if constexpr (q8) {
            if (tid == 0) lscale[step & 1].x = sreg;
            if (tid == kWave) lscale[step & 1].y = log_scale(sreg);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const u32x2 w0 = halves4<SRC>(reg[i][0]), w1 = halves4<SRC>(reg[i][1]);
                const u32x2 w2 = halves4<SRC>(reg[i][2]), w3 = halves4<SRC>(reg[i][3]);
                *reinterpret_cast<u32x4*>(to + (i ? v_to : k_to)) = u32x4{w0[0], w0[1], w1[0], w1[1]};
                *reinterpret_cast<u32x4*>(to + (i ? v_to + 256 : k_to + 1024)) = u32x4{w2[0], w2[1], w3[0], w3[1]};
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                *reinterpret_cast<u32x4*>(to + k_to + 256 * i) = reg[i];
                // (a hidden token's value must not reach the sum, whatever it is)
                if (!((shown >> (16 * i + (tid >> 4))) & 1)) reg[2 + i] = u32x4{0u, 0u, 0u, 0u};
                *reinterpret_cast<u32x4*>(to + v_to + 16 * i * L::kValRow) = reg[2 + i];
            }
        }
    };

    if (u0 < u1) {
        look_up(u0);
        request_mask(u0);
        request(u0);
        look_up(u0 + 1);
        uint32_t shown = shown_now(u0);
        lay(0, shown);
        request_mask(u0 + 1);
        request(u0 + 1);
        look_up(u0 + 2);
        __syncthreads();
        int step = 0;
        for (int u = u0; u < u1; ++u, ++step) {
            const uint32_t shown_next = shown_now(u + 1);
            lay(step + 1, shown_next);
            request_mask(u + 2);
            request(u + 2);
            look_up(u + 3);
            __builtin_amdgcn_sched_barrier(0);
            const int t0 = block_of(u) * kBlk;
            // (a wavefront whose rows see none of the block has nothing to do)
            if (me.live && t0 < me.lim_hi && shown != 0) {
                f32x16 s;
                u32x4 p[2];
                float c = me.qc, vl = kNoScale;
                if constexpr (q8) {
                    const float2 both = lscale[step & 1];
                    c *= both.x;
                    vl = both.y;
                }
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    u32x4 kf[4];
                    read_keys<SRC>(keys_at(step), part, lane, kf);
                    me.scores(s, part, kf);
                    __builtin_amdgcn_sched_barrier(0);
                }
                me.block(s, c, vl, t0, shown, lane, p);
#pragma unroll
                for (int st = 0; st < 2; ++st) {
                    u32x4 vf[4];
                    __builtin_amdgcn_sched_barrier(0);
                    read_values<SRC>(values_at(step), st, lane, vf);
                    me.values(vf, p[st]);
                }
            }
            shown = shown_next;
            __syncthreads();
        }
    }
    if (bad && a.status) atomicOr(a.status, DQ_STATUS_PAGE);
    // (whole vectors up to here: or the loop copies the sums' elements at every turn)
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(me.o[i]));

    // ------------------------------------------------ results
    const float l = me.l + xor_lane<32>(me.l, lane);
    const float f = inverse(l);
    const int up = me.relative_to();
    const int half = lane >> 5;
    const int64_t slot = it.slot;
    if (whole) {
        const int r = r0 + wave * kRowsOf + (lane & 31), token = r / a.G, head = h * a.G + r - token * a.G;
        if (r >= rows) return;
#pragma unroll
        for (int np = 0; np < 4; ++np)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                store_row(a, b, token, head, 32 * np + 8 * i + 4 * half,
                          bf16_two(output(me.o[np][4 * i], f, up), output(me.o[np][4 * i + 1], f, up)),
                          bf16_two(output(me.o[np][4 * i + 2], f, up), output(me.o[np][4 * i + 3], f, up)));
        return;
    }
    float* acc = a.ws_acc + (slot * Many::kRows + wave * kRowsOf + (lane & 31)) * kD + 4 * half;
#pragma unroll
    for (int np = 0; np < 4; ++np)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<f32x4*>(acc + 32 * np + 8 * i) =
                f32x4{output(me.o[np][4 * i], f, up), output(me.o[np][4 * i + 1], f, up),
                      output(me.o[np][4 * i + 2], f, up), output(me.o[np][4 * i + 3], f, up)};
    if (half == 0) {
        float* ml = a.ws_ml + slot * 2 * Many::kRows + wave * kRowsOf + (lane & 31);
        ml[0] = me.m;
        ml[Many::kRows] = l;
    }
}

// ------------------------------------------------------ few rows, one sequence
//
// Up to 64 rows of a (sequence, KV head): a wavefront takes every eighth block
// (or every fourth, of one half of the rows) straight from memory and converts
// it for itself; the wavefronts' sums are joined in LDS at the end.  Bound by
// memory: a block's codes are requested as soon as the registers of the last
// one's are free, keys while the weights are computed, values while the next
// scores are.  16 x 8 queries over 32768 e4m3 tokens (32 heads) take 174 to 177 us, 6.1
// TB/s (262 with the codes converted through LDS for all wavefronts).
//
// Values of codes: a lane reads whole 16-byte pieces (two channels 16 apart of 8
// tokens), so that operand 2 m + e has channels 64 m + 32 (row / 16) + 16 e +
// row % 16 in its rows.  BF16 rows go through an LDS area of the wavefront's own.

constexpr int kFewWaves = 8;
constexpr int kFewThreads = kFewWaves * kWave;
template <int SRC>
__global__ __launch_bounds__(kFewThreads, 2) void few_kernel(ChunkArgs a) {
    typedef Lds<SRC> L;
    constexpr bool q8 = L::q8;
    constexpr int kJoin = kFewWaves * kRowsOf * kJoinRow * 4, kOwn = q8 ? 0 : L::kStage;
    __shared__ __attribute__((aligned(16))) char lds[kJoin > kFewWaves * kOwn ? kJoin : kFewWaves * kOwn];
    __shared__ float wm[kFewWaves][kRowsOf], wl[kFewWaves][kRowsOf], each[kFewWaves][kRowsOf];

    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const Item it = find_item<Few, false>(a, (int)blockIdx.x, lane);
    if (it.tile < 0) return;
    const int b = __builtin_amdgcn_readfirstlane(it.b), h = __builtin_amdgcn_readfirstlane(it.h);
    const int piece = __builtin_amdgcn_readfirstlane(it.c), chunk = __builtin_amdgcn_readfirstlane(it.chunk);
    const Seq seq = seq_of<Few>(a, b);
    const int rows = seq.n * a.G;
    const Sees see = sees(a, seq, 0, rows);
    const bool whole = pieces(see.count, chunk) == 1;
    const int u0 = (int)min((int64_t)piece * chunk, (int64_t)0x7FFFFF00);
    if (u0 >= see.count && piece > 0) return;
    const int u1 = (int)min((int64_t)u0 + chunk, (int64_t)see.count);
    const int parts = rows > kRowsOf ? 2 : 1;    // of the rows
    const int part = wave & (parts - 1), first = wave >> (parts - 1), every = kFewWaves / parts;

    bool bad = false;
    auto block_of = [&](int u) { return u < see.head ? u : see.from + (u - see.head); };
    constexpr int kRaw = q8 ? 4 : 8;
    u32x4 kraw[kRaw], vraw[kRaw];
    float ks = 0.f, vs = 0.f, ks_next = 0.f, vs_next = 0.f;
    uint32_t mreg = 0;
    // codes: as in chunk_kernel; pages a block ahead
    int page = b;
    const int per_page = a.pg.bt ? 1 << (a.pg.page_shift - 5) : a.t_cap / kBlk;
    const int in_page = a.pg.bt ? per_page - 1 : 0x7FFFFFFF, pages = a.pg.bt ? a.pg.num_pages : a.B;
    const uint32_t page_blocks = (uint32_t)(a.H * per_page);
    const int64_t head_blocks = (int64_t)h * per_page;
    const int32_t* table = a.pg.bt ? a.pg.bt + (int64_t)b * a.pg.max_pages : nullptr;
    const int k_lane = ((lane >> 4) & 1) * 2048 + (lane & 15) * 16 + (lane >> 5) * 256;
    const int v_lane = ((lane >> 4) & 1) * 1024 + (lane & 15) * 16 + (lane >> 5) * 256;
    int64_t bi = 0;
    auto look_up = [&](int u) {
        if (q8 && table && u < u1) page = scalar_load(table + ((block_of(u) * kBlk) >> a.pg.page_shift));
    };
    auto locate = [&](int u) {
        if constexpr (q8) {
            if (u >= u1) return;
            const bool in = (uint32_t)page < (uint32_t)pages;
            bad = bad || !in;
            bi = (int64_t)((uint64_t)(uint32_t)(in ? page : 0) * page_blocks) + head_blocks + (block_of(u) & in_page);
            ks_next = scalar_load(a.ks + bi);
            vs_next = scalar_load(a.vs + bi);
        }
    };
    auto request = [&](u32x4 (&raw)[kRaw], int u, bool values) {
        if (u >= u1) return;
        if constexpr (q8) {
            GlobalBytes p = (GlobalBytes)(uintptr_t)((values ? a.v : a.k) + bi * kBlkBytes) + (values ? v_lane : k_lane);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                raw[i] = __builtin_nontemporal_load(
                    reinterpret_cast<GlobalPieces>(p + (values ? (i >> 1) * 2048 + (i & 1) * 512 : i * 512)));
        } else {
            const int64_t st = values ? a.v_st : a.k_st;
            const uint16_t* base = reinterpret_cast<const uint16_t*>(values ? a.v : a.k) +
                                   b * (values ? a.v_sb : a.k_sb) + h * (values ? a.v_sh : a.k_sh) + 8 * (lane & 15);
            const int t = u * kBlk + (lane >> 4);
            if (a.kv_aligned && u * kBlk + kBlk <= see.T) {
                const uint16_t* x = base + t * st;
#pragma unroll
                for (int i = 0; i < 8; ++i, x += 4 * st)
                    raw[i] = *reinterpret_cast<GlobalPieces>(reinterpret_cast<uintptr_t>(x));
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) raw[i] = row_piece(base + min(t + 4 * i, see.T - 1) * st, a.kv_aligned);
            }
        }
    };
    const uint8_t* mask = !q8 && a.mask ? a.mask + b * a.mask_sb : nullptr;
    auto request_mask = [&](int u) {
        if (mask) {
            const int t = u * kBlk + (lane & 31);
            mreg = u < u1 && t < see.T ? mask[t] : 0;
        }
    };
    char* own = lds + wave * kOwn;

    int u = u0 + first;
    look_up(u);
    locate(u);
    request_mask(u);
    request(kraw, u, false);
    request(vraw, u, true);
    look_up(u + every);
    constexpr bool fine = !q8;
    Rows<SRC, fine> me;
    me.load(a, see, b, h, part * kRowsOf, rows, lane);
    for (; u < u1; u += every) {
        const int t0 = block_of(u) * kBlk;
        uint32_t shown = mask ? (uint32_t)__builtin_amdgcn_ballot_w64(mreg != 0) : ~0u;
        if (!q8) shown &= shown_to(see.T - t0);
        const bool on = t0 < me.lim_hi && shown != 0;
        f32x16 s = f32x16{};
        u32x4 p[fine ? 4 : 2];
        float c = me.qc, vl = kNoScale;
        if constexpr (q8) {
            ks = ks_next;
            vs = vs_next;
            c *= ks;
            vl = log_scale(vs);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const u32x2 w0 = halves4<SRC>(kraw[i][0]), w1 = halves4<SRC>(kraw[i][1]);
                const u32x2 w2 = halves4<SRC>(kraw[i][2]), w3 = halves4<SRC>(kraw[i][3]);
                s = mma<SRC>(u32x4{w0[0], w0[1], w1[0], w1[1]}, me.q[2 * i], s);
                s = mma<SRC>(u32x4{w2[0], w2[1], w3[0], w3[1]}, me.q[2 * i + 1], s);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                *reinterpret_cast<u32x4*>(own + (lane & 15) * (L::kKeyOp / 2) + (4 * i + (lane >> 4)) * 16) = kraw[i];
            wave_sync();
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                u32x4 kf[4];
                read_keys<SRC>(own, j, lane, kf);
                me.scores(s, j, kf);
            }
        }
        request_mask(u + every);
        locate(u + every);
        request(kraw, u + every, false);
        look_up(u + 2 * every);
        if (on) {
            me.block(s, c, vl, t0, shown, lane, p);
            if constexpr (q8) {
#pragma unroll
                for (int st = 0; st < 2; ++st)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const u32x4& w = vraw[2 * i + st];
                        const u32x2 w0 = halves4<SRC>(w[0]), w1 = halves4<SRC>(w[1]);
                        const u32x2 w2 = halves4<SRC>(w[2]), w3 = halves4<SRC>(w[3]);
                        me.o[2 * i] = mma<SRC>(u32x4{w0[0], w0[1], w1[0], w1[1]}, p[st], me.o[2 * i]);
                        me.o[2 * i + 1] = mma<SRC>(u32x4{w2[0], w2[1], w3[0], w3[1]}, p[st], me.o[2 * i + 1]);
                    }
            } else {
                // (a hidden token's value must not reach the sum, whatever it is)
                if (shown != ~0u) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (!((shown >> (4 * i + (lane >> 4))) & 1)) vraw[i] = u32x4{0u, 0u, 0u, 0u};
                }
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    *reinterpret_cast<u32x4*>(own + L::kKeys + (4 * i + (lane >> 4)) * L::kValRow + (lane & 15) * 16) =
                        vraw[i];
                wave_sync();
#pragma unroll
                for (int st = 0; st < 2; ++st) {
                    u32x4 vf[4];
                    read_values<SRC>(own + L::kKeys, st, lane, vf);
                    me.values(vf, p[st]);
                    if constexpr (fine) {
                        zeros_for_infinities(vf);
                        me.values(vf, p[2 + st]);
                    }
                }
            }
        }
        wave_sync();
        request(vraw, u + every, true);
    }
    if (bad && a.status) atomicOr(a.status, DQ_STATUS_PAGE);
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(me.o[i]));

    join_rows<Few, kFewWaves, q8>(a, me.o, me.m, me.l + xor_lane<32>(me.l, lane), me.relative_to(),
                                  reinterpret_cast<float*>(lds), wm, wl, each, parts, rows, 0, b, h, whole, it.slot);
}

// The pieces of a segment's rows joined: half a wavefront has a row at a time, four
// channels a lane.  Bound by latency (plan, lengths, maxima, sums) where pieces are
// few: one row for each half of a workgroup's wavefronts, 4.5 us for 16 pieces (7.1
// with two rows); by memory where they are many (50 MB of them 13 us), and there
// fewer workgroups, each of which looks its segment up, take less (48 ragged chunks
// 473 us with two rows, 486 with one).
// Over the 32 lanes of half a wavefront; every lane gets the result.
template <typename Op>
__device__ __forceinline__ float half_reduce(float v, int lane, Op op) {
    v = op(v, xor_lane<1>(v, lane));
    v = op(v, xor_lane<2>(v, lane));
    v = op(v, xor_lane<4>(v, lane));
    v = op(v, xor_lane<8>(v, lane));
    return op(v, xor_lane<16>(v, lane));
}

template <typename K>
__device__ __forceinline__ void merge_rows(const ChunkArgs& a, int id, int lane) {
    constexpr int R = K::kRows, kMergeRows = K::kMergeRows, kParts = R / kMergeRows;
    const Item it = find_item<K, true>(a, id / kParts, lane);
    if (it.tile < 0 || it.chunk == kWhole) return;
    const int b = __builtin_amdgcn_readfirstlane(it.b), h = __builtin_amdgcn_readfirstlane(it.h);
    const int tile = __builtin_amdgcn_readfirstlane(it.tile);
    const Seq seq = seq_of<K>(a, b);
    const int rows = seq.n * a.G, r0 = tile * R;
    const Sees see = sees(a, seq, r0, min(r0 + R, rows));
    const int nc = __builtin_amdgcn_readfirstlane(pieces(see.count, it.chunk));
    if (nc == 1) return;
    const int64_t slot = __builtin_amdgcn_readfirstlane(it.slot);
    const int ch = 4 * (lane & 31);
    for (int i = (int)threadIdx.x >> 5; i < kMergeRows; i += 8) {
        const int in = (id % kParts) * kMergeRows + i, r = r0 + in;
        if (r >= rows) break;
        const float* ml = a.ws_ml + slot * 2 * R + in;
        const float* acc = a.ws_acc + (slot * R + in) * kD + ch;
        // 32 pieces at a time: lane c % 32 has piece c's maximum and sum; outputs come
        // eight loads at a time, the first ones on their way beside those
        const int mine = lane & 31;
        auto max_of = [&](int c) { return ml[(int64_t)c * 2 * R]; };
        auto sum_of = [&](int c) { return ml[(int64_t)c * 2 * R + R]; };
        f32x4 v[8];
        auto outputs = [&](int c0) {
#pragma unroll
            for (int c = 0; c < 8; ++c)
                v[c] = *reinterpret_cast<const f32x4*>(acc + (int64_t)min(c0 + c, nc - 1) * R * kD);
        };
        outputs(0);
        const float m0 = mine < nc ? max_of(mine) : -INFINITY, l0 = mine < nc ? sum_of(mine) : 0.f;
        float top = m0;
        for (int c = mine + 32; c < nc; c += 32) top = fmaxf(top, max_of(c));
        top = half_reduce(top, lane, [](float p, float q) { return fmaxf(p, q); });
        float l = share(m0, l0, top);
        for (int c = mine + 32; c < nc; c += 32) l += share(max_of(c), sum_of(c), top);
        const float each = inverse(half_reduce(l, lane, [](float p, float q) { return p + q; }));
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        for (int c0 = 0; c0 < nc; c0 += 32) {
            float w = share(m0, l0, top) * each;
            if (c0 > 0) w = c0 + mine < nc ? share(max_of(c0 + mine), sum_of(c0 + mine), top) * each : 0.f;
            const int n = min(32, nc - c0);
            for (int c1 = 0; c1 < n; c1 += 8) {
                if (c0 + c1 > 0) outputs(c0 + c1);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const float wc = __shfl(w, min(c1 + c, 31), 32);
                    if (c1 + c < n) x += v[c] * wc;
                }
            }
        }
        const int token = r / a.G, head = h * a.G + r - token * a.G;
        store_row(a, b, token, head, ch, bf16_two(x[0], x[1]), bf16_two(x[2], x[3]));
    }
}

__global__ __launch_bounds__(256) void chunk_merge_kernel(ChunkArgs few, ChunkArgs many, int few_groups) {
    const int lane = threadIdx.x & (kWave - 1);
    if ((int)blockIdx.x < few_groups)
        merge_rows<Few>(few, blockIdx.x, lane);
    else
        merge_rows<Many>(many, (int)blockIdx.x - few_groups, lane);
}

// The plan of many sequences: the blocks of one piece, and for each 64 sequences
// their items of each pass, cut segments and slots (of one KV head).
constexpr int kPlanWaves = 16;

template <typename K>
__device__ __forceinline__ void plan_all(const ChunkArgs& a, int wave, int lane, float (&sums)[2][kPlanWaves],
                                         int (&most)[kPlanWaves], int (&items)[kPlanWaves]) {
    float total = 0, segs = 0;
    int longest = 0;
    for (int g = wave; g < a.groups; g += kPlanWaves) {
        const Seq s = seq_at<K>(a, g * kWave, lane);
        total += wave_sum((float)s.tiles * (float)s.units);
        segs += wave_sum((float)s.tiles);
        longest = max(longest, wave_max(s.tiles ? s.units : 0));
    }
    if (lane == 0) {
        sums[0][wave] = total;
        sums[1][wave] = segs;
        most[wave] = longest;
    }
    __syncthreads();
    total = segs = 0;
    for (int w = 0; w < kPlanWaves; ++w) {
        total += sums[0][w];
        segs += sums[1][w];
        longest = max(longest, most[w]);
    }
    const int chunk = plan_of<K>(total * (float)a.H, segs * (float)a.H, longest, lane);
    int all = 0;
    if (chunk != kWhole) {
        for (int g = wave; g < a.groups; g += kPlanWaves) {
            const Seq s = seq_at<K>(a, g * kWave, lane);
            const int n = pieces(s.units, chunk), full = s.units / chunk, rest = s.units - full * chunk;
            const int long_end = rest > chunk / 2, short_end = !long_end && (rest > 0 || full == 0);
            const int first = wave_sum(s.tiles * full), second = wave_sum(s.tiles * long_end);
            const int third = wave_sum(s.tiles * short_end), cut = wave_sum(n > 1 ? s.tiles : 0);
            const int slots = wave_sum(n > 1 ? s.tiles * n : 0);
            if (lane == 0) {
                int32_t* t = a.plan + 4 + g;
                t[0] = first;
                t[a.groups] = second;
                t[2 * a.groups] = third;
                t[3 * a.groups] = cut;
                t[4 * a.groups] = slots;
            }
            all += first + second + third;
        }
    }
    if (lane == 0) items[wave] = all;
    __syncthreads();
    if (wave == 0 && lane == 0) {
        all = 0;
        for (int w = 0; w < kPlanWaves; ++w) all += items[w];
        a.plan[0] = chunk;
        a.plan[1] = all;
    }
}

__global__ __launch_bounds__(kPlanWaves * kWave) void chunk_plan_kernel(ChunkArgs few, ChunkArgs many) {
    __shared__ float sums[2][kPlanWaves];
    __shared__ int most[kPlanWaves], items[kPlanWaves];
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    if (blockIdx.x == 0 && few.planned) plan_all<Few>(few, wave, lane, sums, most, items);
    if (blockIdx.x == 1 && many.planned) plan_all<Many>(many, wave, lane, sums, most, items);
}

// ------------------------------------------------------------------- host

// A kernel's part of the work, as far as the host knows it.
struct HostPlan {
    bool runs, planned;
    int rows;                    // per tile
    int64_t segs, slots, grid;
    int64_t merges;              // workgroups of the merge
    int64_t plan;                // numbers of the plan

    // sums, maxima and weights of the slots, and the plan
    int64_t floats() const { return slots ? slots * rows * (kD + 2) + plan : 0; }
};

template <typename K>
HostPlan host_plan(int32_t B, int32_t n_q, int32_t Hq, int32_t Hkv, int32_t t_cap, bool lens, int units = 0) {
    HostPlan p;
    const int64_t rows = (int64_t)n_q * (Hq / Hkv);
    // chunks of unlike lengths may be of either kind
    p.runs = K::kFew ? rows <= Few::kRows || lens : rows > Few::kRows;
    p.rows = K::kRows;
    p.segs = (int64_t)B * Hkv * (K::kFew ? 1 : (rows + p.rows - 1) / p.rows);
    const int64_t pieces = std::max<int64_t>(1, ((int64_t)t_cap / kBlk + kLeast) / kLeast);
    // Where one sequence's segments take every place nothing is longer than a
    // place's share; else what fills the GPU twice may still have a longest one.
    const int64_t own = p.segs / B;
    bool cuts = p.runs && pieces > 1 && (lens || p.segs < 2 * K::kAtOnce || own < K::kAtOnce);
    if (cuts && units > 0) {
        // every segment has these blocks, so the plan is known here: none is cut
        // where no plan costs less, and nothing is merged
        float least = plan_cost<K>((float)p.segs, units, std::max(units, kLeast));
        bool better = false;
        for (int n = 1; n < kWave; ++n) better |= plan_cost<K>((float)p.segs, units, plan_try(units, n)) < least;
        cuts = better;
    }
    // Pieces are of a place's share, or of like segments twice as many as places:
    // there are as many cut segments as places at most, of twice as many pieces, and
    // a last piece of every segment beside the whole ones.
    p.planned = cuts && (B > kWave || (!lens && p.segs >= 2 * K::kAtOnce));
    p.plan = 4 + (5 * (((int64_t)B + kWave - 1) / kWave) + 3) / 4 * 4;
    p.slots = cuts ? std::min<int64_t>(2 * K::kAtOnce + 8, p.segs * pieces) : 0;
    const int64_t items = cuts ? std::min<int64_t>(std::max<int64_t>(p.segs, K::kAtOnce) + K::kAtOnce + 8, p.segs * pieces)
                               : p.segs;
    p.grid = (items + 7) / 8 * 8;
    p.merges = cuts ? std::min<int64_t>(K::kAtOnce + 8, p.segs) * (K::kRows / K::kMergeRows) : 0;
    return p;
}

template <int SRC>
int launch_source(const ChunkArgs& few, const HostPlan& pf, const ChunkArgs& many, const HostPlan& pm,
                  hipStream_t stream) {
    if (pf.runs) few_kernel<SRC><<<dim3((unsigned)pf.grid), kFewThreads, 0, stream>>>(few);
    if (pm.runs) chunk_kernel<SRC><<<dim3((unsigned)pm.grid), kThreads, 0, stream>>>(many);
    return hip_check("chunk launch", hipGetLastError());
}

bool aligned16(const Q8Rows& r) {
    return ((reinterpret_cast<uintptr_t>(r.p) | (uintptr_t)(r.sb * 2) | (uintptr_t)(r.st * 2) | (uintptr_t)(r.sh * 2)) & 15) == 0;
}

}  // namespace

size_t chunk_workspace_bytes(int32_t B, int32_t n_q, int32_t Hq, int32_t Hkv, int32_t t_cap) {
    // (with or without lengths of the chunks: the larger)
    return (size_t)(host_plan<Few>(B, n_q, Hq, Hkv, t_cap, true).floats() +
                    host_plan<Many>(B, n_q, Hq, Hkv, t_cap, true).floats()) * sizeof(float);
}

int launch_chunk(const ChunkSource& src, const ChunkCall& c, void* ws, uint32_t* status, hipStream_t stream) {
    // blocks of every segment, where no lengths on the device say otherwise
    const int units = c.q_lens || c.seq_lens || c.window > 0 ? 0 : (int)(((int64_t)c.t_cap + kBlk - 1) / kBlk);
    const HostPlan pf = host_plan<Few>(c.B, c.n_q, c.Hq, c.Hkv, c.t_cap, c.q_lens != nullptr, units);
    const HostPlan pm = host_plan<Many>(c.B, c.n_q, c.Hq, c.Hkv, c.t_cap, c.q_lens != nullptr, units);
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
    a.groups = (c.B + kWave - 1) / kWave;
    a.causal = c.causal;
    a.window = c.window;
    a.sinks = c.sinks;
    a.q_aligned = aligned16(c.q);
    a.kv_aligned = !q8 && aligned16(src.k) && aligned16(src.v);
    a.out_aligned = ((reinterpret_cast<uintptr_t>(c.out.p) | (uintptr_t)(c.out.sb * 2) | (uintptr_t)(c.out.st * 2) |
                      (uintptr_t)(c.out.sh * 2)) & 7) == 0;
    a.scale_log2 = std::min(fabsf(c.scale) * kLog2e, FLT_MAX);           // (infinity times a score of 0: NaN)
    a.negative = c.scale < 0.f;
    a.status = status;
    ChunkArgs few = a, many = a;
    few.cuts = pf.slots > 0;
    many.cuts = pm.slots > 0;
    few.planned = pf.planned;
    many.planned = pm.planned;
    few.ws_acc = static_cast<float*>(ws);
    few.ws_ml = few.ws_acc + pf.slots * pf.rows * kD;
    few.plan = reinterpret_cast<int32_t*>(few.ws_ml + pf.slots * pf.rows * 2);
    many.ws_acc = few.ws_acc + pf.floats();
    many.ws_ml = many.ws_acc + pm.slots * pm.rows * kD;
    many.plan = reinterpret_cast<int32_t*>(many.ws_ml + pm.slots * pm.rows * 2);
    if (pf.planned || pm.planned) {
        chunk_plan_kernel<<<2, kPlanWaves * kWave, 0, stream>>>(few, many);
        if (int rc = hip_check("chunk_plan launch", hipGetLastError())) return rc;
    }
    int rc;
    if (src.format == DQ_Q8_E4M3)
        rc = launch_source<DQ_Q8_E4M3>(few, pf, many, pm, stream);
    else if (src.format == DQ_Q8_INT8)
        rc = launch_source<DQ_Q8_INT8>(few, pf, many, pm, stream);
    else
        rc = launch_source<kChunkBf16>(few, pf, many, pm, stream);
    if (rc != DQ_OK) return rc;
    if (pf.merges + pm.merges == 0) return DQ_OK;
    chunk_merge_kernel<<<dim3((unsigned)(pf.merges + pm.merges)), 256, 0, stream>>>(few, many, (int)pf.merges);
    return hip_check("chunk_merge launch", hipGetLastError());
}

}  // namespace dq
