// Declarations shared by the kernels of linear layers on 8-bit codes (linear8.hip) and their C entry points (linear8_api.hip).
// gfx950 only.
#pragma once

#include "lpq_internal.h"

namespace lpq {

enum { LINEAR8_MAX_D = 1 << 17,        // sums of this many products of two codes stay below 2^31
       LINEAR8_MAX_ROWS = 1 << 25 };   // of a launch: 64 threads for a row of codes, 32 for a channel, fewer than 2^32 in all

// Blocks of 64 features that a row takes, an even number.
static inline int row_blocks(int d) { return (int)round_up(d, 128) / 64; }

// Rows of codes in blocks (linear8.hip) and their scales.  The features from d to the end of the last block are 0 in one of two operands.
struct RowCodes {
    const int8_t *codes;
    const float *scales;
    int64_t n;
};

struct Linear8Out {
    void *p;
    int64_t ld;
    int type;
    const float *bias;       // null or one per channel
};

// rows: tokens of a workgroup's tile, channels: of its tile; parts: shares of the features, whose sums are joined by a second kernel (0: one
// workgroup has all tokens and reads the weights past LDS).
struct Linear8Plan {
    int rows, channels, parts;
    size_t bytes;            // of workspace, for the parts
};
Linear8Plan linear8_plan(int64_t m, int64_t n, int d);
hipError_t launch_encode_rows(const void *x, int64_t ldx, int type, int64_t n, int d, int8_t *codes, float *scales, hipStream_t st);
// Few rows, whose codes the product's own kernel makes.
bool linear8_fused(int64_t m, int d);
hipError_t launch_linear8_fused(const void *x, int64_t ldx, int64_t m, const RowCodes &w, int d, const Linear8Out &out, hipStream_t st);
hipError_t launch_linear8(const RowCodes &x, const RowCodes &w, int d, const Linear8Out &out, const Linear8Plan &plan, void *workspace, hipStream_t st);

}  // namespace lpq
