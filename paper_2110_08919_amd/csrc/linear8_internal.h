// Declarations shared by the kernels of linear layers on 8-bit codes (linear8.hip) and their C entry points (linear8_api.hip).
// gfx950 only.
#pragma once

#include "lpq_internal.h"

namespace lpq {

enum { ROW_CODES_ALIGN = 128,          // rows of codes are read in runs of this many bytes
       LINEAR8_MAX_D = 1 << 17,        // sums of this many products of two codes stay below 2^31
       LINEAR8_MAX_STRIDE = 1 << 20 }; // between rows of codes: 256 of them lie within 32-bit offsets

// Rows of codes [n][d], `ld` bytes apart (a multiple of 16, at least d rounded up to ROW_CODES_ALIGN; the bytes between are 0 in
// one of two operands), and their scales.
struct RowCodes {
    const int8_t *codes;
    const float *scales;
    int64_t ld, n;
};

struct Linear8Out {
    void *p;
    int64_t ld;
    int type;
    const float *bias;       // null or one per channel
};

// rows: tokens of a workgroup's tile, channels: of its tile; parts: shares of the features, whose sums are joined by a second kernel.
struct Linear8Plan {
    int rows, channels, parts;
    size_t bytes;            // of workspace, for the parts
};
Linear8Plan linear8_plan(int64_t m, int64_t n, int d);
hipError_t launch_encode_rows(const void *x, int64_t ldx, int type, int64_t n, int d, int8_t *codes, int64_t ld, float *scales, hipStream_t st);
hipError_t launch_linear8(const RowCodes &x, const RowCodes &w, int d, const Linear8Out &out, const Linear8Plan &plan, void *workspace, hipStream_t st);

}  // namespace lpq
