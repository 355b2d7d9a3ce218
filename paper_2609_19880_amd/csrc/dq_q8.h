// Launchers of the 8-bit cache (dq_q8.hip).  Return DQ_OK or an error code.
#pragma once

#include "dq_internal.h"

namespace dq {

// The 8-bit cache: keys [0] and values [1].
struct Q8Cache {
    uint8_t* data[2];
    float* scale[2];
};
// bf16 rows [B][T][H][128] at element strides.
struct Q8Rows {
    const uint16_t* p;
    int64_t sb, st, sh;
};
int launch_q8_encode(int format, const Pages& pg, const Q8Rows& k, const Q8Rows& v, int32_t B, int32_t H, int32_t t0,
                     int32_t n_new, int32_t t_cap, const Q8Cache& to, uint32_t* status, hipStream_t stream);
int launch_q8_read(int format, const Pages& pg, const Q8Cache& from, int32_t B, int32_t H, int32_t t0, int32_t n,
                   int32_t t_cap, const Q8Rows& k, const Q8Rows& v, uint32_t* status, hipStream_t stream);
// out: the step's result where one chunk holds the whole of every sequence
// (*slots is 0 then, scores included); else the partials alone are written, at
// *slots per (sequence, query head).  slots may be NULL without out.
int launch_q8_partial(int format, const Pages& pg, const uint16_t* q, int32_t B, int32_t Hq, int32_t Hkv,
                      const Q8Cache& c, const int32_t* seq_lens, const int32_t* extra_lens, int32_t t_cap,
                      int32_t window, int32_t sinks, float scale, float* lse, float* out, float* scores, void* ws,
                      uint32_t* status, hipStream_t stream, int* slots);
// The merge (out, may be NULL) and the blocks' weights (scores, may be NULL) of
// `slots` partials, 0: as many as the workspace says.
int launch_q8_finish(int32_t B, int32_t Hq, int32_t Hkv, const int32_t* seq_lens, const int32_t* extra_lens,
                     int32_t t_cap, int32_t window, int32_t sinks, const float* lse, const void* ws, float* out,
                     float* scores, int slots, hipStream_t stream);
// keep, first and last in tokens, multiples of 32
int launch_q8_evict(const Pages& pg, int32_t B, int32_t H, const int32_t* seq_lens, int32_t* new_lens, int32_t t_cap,
                    int32_t to_cap, int32_t keep, int32_t first, int32_t last, const float* scores,
                    float* to_scores, const Q8Cache& from, const Q8Cache& to, int32_t* kept, uint32_t* status,
                    hipStream_t stream);

}  // namespace dq
