// Launchers of the attention of many queries (dq_chunk.hip) and of the rotary
// positions (dq_rope.hip).  Return DQ_OK or an error code.
#pragma once

#include "dq_q8.h"

namespace dq {

// What a call of the chunk attention attends over: 8-bit codes, contiguous or
// in pool pages, or BF16 rows at element strides.
struct ChunkSource {
    int format;                  // DQ_Q8_INT8, DQ_Q8_E4M3 or kChunkBf16
    Pages pg;
    Q8Cache cache;
    Q8Rows k, v;
    const uint8_t* mask;         // BF16: [B][t_cap] at stride mask_sb, zero = hidden, or NULL
    int64_t mask_sb;
};
constexpr int kChunkBf16 = 2;

struct ChunkCall {
    Q8Rows q, out;               // (out is written)
    int32_t B, n_q, Hq, Hkv, t_cap;
    const int32_t* q_lens;       // or NULL: n_q each
    const int32_t* seq_lens;     // or NULL: t_cap each
    int causal;
    int32_t window, sinks;
    float scale;
};

size_t chunk_workspace_bytes(int32_t B, int32_t n_q, int32_t Hq, int32_t Hkv, int32_t t_cap);
int launch_chunk(const ChunkSource& src, const ChunkCall& c, void* ws, uint32_t* status, hipStream_t stream);

struct RopeRows {
    Q8Rows in, out;
    int32_t heads;
};
int launch_rope(int layout, int transposed, const double* freq, float magnitude, int32_t rotary, const RopeRows& q,
                const RopeRows& k, int32_t B, int32_t T, int32_t d, const int32_t* positions, int64_t pos_sb,
                int64_t pos_st, const int32_t* starts, int32_t t0, hipStream_t stream);

}  // namespace dq
