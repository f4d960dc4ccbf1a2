// Which pages of a key-value cache a query can find large inner products in.
//
// Scores.  For a row of query codes z and any token of a page, sum_i z_i c_i <= sum_i max(z_i lo_i, z_i hi_i) with lo and
// hi the page's bounds.  The sum over the rows of a key-value head separates: sum_i w+_i hi_i + w-_i lo_i with
// w+ = sum of the rows' positive codes, w- of the negative ones, so a page costs one integer product of 2 dpad bytes
// however many query heads share it.  |w| <= 127 * 128 rows = two digits of 7 bits; a 16x16x64 matrix instruction takes
// 16 pages as rows and the two digits as two of its columns, which also sums over the lanes.  Exact in int32:
// 128 * 16256 * 256 = 5.3e8.  Bound by reading the bounds (2 dpad bytes per page and head).
//
// Picking.  The n_select largest (score, then lower page): one workgroup per (sequence, head) holds the scores in
// registers, finds the n_select-th largest by bisection over the bits that differ between them (each step counts with
// one ballot per register, no atomics, so the result does not depend on any order), and writes the pages out in
// ascending order.
//
// Tables of up to 512 pages: one launch, whose workgroup scores all pages of a (sequence, head) and picks; the second launch and
// the scores' way through memory would cost more than the larger part of the chip gains.  Bound by round trips to memory.
//
// Measured, 8 heads of 128, 4 query heads each: 16 sequences of 71 000 to 129 000 tokens (25 000 pages of 64, 51.5 MB of bounds) scores
// 14.7 us, 3.5 TB/s: 8.4 at the rate of a streaming read, the rest is the chain of length, page number and bounds before the first
// product; picking 128 of some 1570 pages of each head 7.8; one sequence of 250 pages 8.6 in one launch.
#include "kv_internal.h"
#include "wave_ops.h"

namespace lpq {

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));

constexpr int THREADS = 256;
constexpr int UNROLL = 4;                              // groups of 16 pages a wave has in flight
constexpr int block_pages(int threads) { return threads / 64 * 16 * UNROLL; }
constexpr int FUSED_PAGES = block_pages(512);

__device__ __forceinline__ int pages_of(int len, int page_shift, int table_pages)
{
    if (len <= 0) return 0;
    const int np = (int)(((int64_t)len + (1 << page_shift) - 1) >> page_shift);
    return np < table_pages ? np : table_pages;
}

// Sortable image of a page's score: 0 = not there, all ones = kept in any case.
__device__ __forceinline__ uint32_t key_of(int32_t score, int page, int np, int keep_first, int keep_last)
{
    if (score == INT32_MIN) return 0;
    if (page < keep_first || page >= np - keep_last) return 0xFFFFFFFFu;
    return (uint32_t)score ^ 0x80000000u;
}

// By a workgroup of NT threads with KEYS scores each.  More pages than that (beyond NT * KEYS) are read again from memory at
// every step.
template <int NT, int KEYS, bool AGAIN>
__device__ __forceinline__ void pick(const int32_t *score, int np, const KvSelect &s, int32_t *out)
{
    constexpr int W = NT / 64;
    __shared__ uint32_t red[2][W];
    __shared__ int count[2][W];
    __shared__ int before[2][KEYS * W];
    constexpr int CUTS = KEYS == 1 ? 7 : 3;
    __shared__ int cut[2][W][CUTS];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int rounds = AGAIN ? (np + NT * KEYS - 1) / (NT * KEYS) : 1;
    uint32_t key[KEYS];
    auto fetch = [&](int round) {
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            const int page = (round * KEYS + i) * NT + tid;
            key[i] = page < np ? key_of(score[page], page, np, s.keep_first, s.keep_last) : 0;
        }
    };
    // number of pages that are there, smallest and largest score among those not kept in any case
    uint32_t lo = 0xFFFFFFFFu, hi = 0;
    int there = 0;
    for (int r = 0; r < rounds; ++r) {
        fetch(r);
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            there += __popcll(__ballot(key[i] != 0));
            if (key[i] != 0 && key[i] != 0xFFFFFFFFu) {
                lo = key[i] < lo ? key[i] : lo;
                hi = key[i] > hi ? key[i] : hi;
            }
        }
    }
    lo = wave_all(lo, [](uint32_t x, uint32_t y) { return x < y ? x : y; });
    hi = wave_all(hi, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
    if (lane == 0) { red[0][wave] = lo; red[1][wave] = hi; count[0][wave] = there; }
    __syncthreads();
    there = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        lo = red[0][w] < lo ? red[0][w] : lo;
        hi = red[1][w] > hi ? red[1][w] : hi;
        there += count[0][w];
    }
    const int want = there < s.n_select ? there : s.n_select;
    // Largest bound T with at least `want` keys >= T: T in [lo, hi], or all ones where the pages kept in any case are enough.
    // Each step counts for CUTS bounds at once (ballots of a wave, summed over the waves through LDS) and leaves one of
    // CUTS + 1 parts of the interval.
    auto enough = [&](uint32_t from, uint32_t by, uint32_t span, int buf) {      // how many of from + by, from + 2 by .. are low enough
        int c[CUTS] = {};
        for (int r = 0; r < rounds; ++r) {
            if (AGAIN) fetch(r);
#pragma unroll
            for (int j = 0; j < CUTS; ++j) {
                const uint32_t at = from + ((j + 1) * by < span ? (j + 1) * by : span);
#pragma unroll
                for (int i = 0; i < KEYS; ++i) c[j] += __popcll(__ballot(key[i] >= at));
            }
        }
        int mine = 0;
#pragma unroll
        for (int j = 0; j < CUTS; ++j) mine = lane == j ? c[j] : mine;
        if (lane < CUTS) cut[buf][wave][lane] = mine;
        __syncthreads();
        mine = 0;
        if (lane < CUTS) {
#pragma unroll
            for (int w = 0; w < W; ++w) mine += cut[buf][w][lane];
        }
        return __popcll(__ballot(lane < CUTS && mine >= want));
    };
    uint32_t T = 0xFFFFFFFFu;
    int buf = 0;
    if (want > 0 && enough(0xFFFFFFFFu, 0, 0, buf) == 0) {
        // here some scored page is wanted: lo <= hi, and at least `want` keys are >= lo
        uint32_t a = lo, span = hi - lo;
        while (span) {
            buf ^= 1;
            const uint32_t by = span / (CUTS + 1) + 1;       // CUTS by < 2^32
            const int k = enough(a, by, span, buf);
            const uint32_t under = k * by < span ? k * by : span;
            if (k < CUTS) span = (k + 1) * by < span ? (k + 1) * by - 1 : span - 1;      // that one is too high
            span -= under;
            a += under;
        }
        T = a;
    }
    // Pages above T all, of those at T the first ones.
    int above_all = 0, equal_all = 0;                        // keys > T, == T of the rounds before
    int total_above = 0;
    if (AGAIN) {
        int c = 0;
        for (int r = 0; r < rounds; ++r) {
            fetch(r);
#pragma unroll
            for (int i = 0; i < KEYS; ++i) c += __popcll(__ballot(key[i] > T));
        }
        __syncthreads();
        if (lane == 0) count[0][wave] = c;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w) total_above += count[0][w];
    }
    for (int r = 0; r < rounds; ++r) {
        if (AGAIN) fetch(r);
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            const int up = __popcll(__ballot(key[i] > T)), eq = __popcll(__ballot(key[i] == T && T != 0));
            if (lane == 0) { before[0][i * W + wave] = up; before[1][i * W + wave] = eq; }
        }
        __syncthreads();
        if (wave < 2) {      // wave 0 sums what lies before each entry of the first list, wave 1 of the second
            int run = wave == 0 ? above_all : equal_all;
            for (int e0 = 0; e0 < KEYS * W; e0 += 64) {
                const int v = e0 + lane < KEYS * W ? before[wave][e0 + lane] : 0;
                const int sum = (int)wave_scan((uint32_t)v);
                if (e0 + lane < KEYS * W) before[wave][e0 + lane] = run + sum - v;
                run += __builtin_amdgcn_readlane(sum, 63);
            }
            if (lane == 0) count[wave][0] = run;
        }
        __syncthreads();
        if (!AGAIN) total_above = count[0][0];
        const int ties = want - total_above;                 // keys equal to T to take
        const uint64_t below = lane == 0 ? 0 : ~0ull >> (64 - lane);
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            const uint64_t up = __ballot(key[i] > T), eq = __ballot(key[i] == T && T != 0);
            const int rank_up = before[0][i * W + wave] + __popcll(up & below);
            const int rank_eq = before[1][i * W + wave] + __popcll(eq & below);
            const bool take = key[i] > T || (key[i] == T && T != 0 && rank_eq < ties);
            if (take) out[rank_up + (rank_eq < ties ? rank_eq : ties)] = (r * KEYS + i) * NT + tid;
        }
        above_all = count[0][0];
        equal_all = count[1][0];
        __syncthreads();
    }
    for (int i = want + tid; i < s.n_select; i += NT) out[i] = -1;
}

template <int NT, int KEYS, bool AGAIN>
__global__ __launch_bounds__(NT) void kv_pick_kernel(KvView kv, KvSelect s)
{
    const int pair = blockIdx.x, np = pages_of(kv_uniform(s.lengths)[pair / kv.heads], kv.page_shift, s.table_pages);
    pick<NT, KEYS, AGAIN>(s.scores + (int64_t)pair * s.table_pages, np, s, s.pages + (int64_t)pair * s.n_select);
}

template <int DP, int NT, bool FUSED>
__global__ __launch_bounds__(NT) void kv_score_kernel(KvView kv, KvQueries q, KvSelect s, int blocks_per)
{
    constexpr int STEPS = 2 * DP / 64, WAVES = NT / 64, BLOCK_PAGES = block_pages(NT);
    __shared__ float red[WAVES];
    __shared__ __align__(16) int8_t digit[2][2 * DP];
    __shared__ int wsum[2 * DP];
    const int pair = blockIdx.x / blocks_per, part = blockIdx.x % blocks_per;
    const int h = pair % kv.heads, b = pair / kv.heads;
    const int np = pages_of(kv_uniform(s.lengths)[b], kv.page_shift, s.table_pages);
    if (!FUSED && part * BLOCK_PAGES >= np) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 15, g = lane >> 4;

    // Query codes: z = rint(q s * (127 / A)), A the largest |q s| of the head's rows; what is not finite counts as 0.
    const int rows = q.new_tokens * q.group, chunks = DP / 8, items = rows * chunks;
    const int64_t base = (int64_t)b * q.ld_seq + (int64_t)h * q.group * q.ld_head;
    auto row_at = [&](int r) { return base + (int64_t)(r / q.group) * q.ld_token + (int64_t)(r % q.group) * q.ld_head; };
    auto fetch = [&](int t, float *st) {
        const int r = t / chunks, c0 = (t % chunks) * 8;
        kv_load_floats8(kv.key.s + h * DP + c0, st);
        return kv_load8(q.p, q.type, row_at(r) + c0, t < items ? kv.dim - c0 : 0);
    };
    auto scaled = [&](int t, Raw8 raw, const float *st, float *v) {
        kv_floats8(raw, q.type, t < items ? kv.dim - (t % chunks) * 8 : 0, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = __fmul_rn(v[e], st[e]);
            v[e] = fabsf(x) <= 3.402823466e38f ? x : 0.0f;
        }
    };
    float step[8], mine[8];
    const Raw8 raw = fetch(tid, step);

    // The pages' bounds, behind the first queries: loads are waited for in order, so these arrive while the queries are made ready.
    const int32_t *table = s.table + (int64_t)b * s.ld_table;
    const int page0 = part * BLOCK_PAGES + wave * 16 * UNROLL;
    int32_t id[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        const int page = page0 + 16 * u + n;
        id[u] = page < np ? table[page] : -1;
        if (id[u] >= kv.pages) id[u] = -1;
    }
    v4i x[UNROLL][STEPS];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        const int8_t *row = kv.bounds + ((int64_t)(id[u] < 0 ? 0 : id[u]) * kv.heads + h) * 2 * DP + g * 16;
#pragma unroll
        for (int st = 0; st < STEPS; ++st) x[u][st] = *reinterpret_cast<const v4i *>(row + 64 * st);
    }

    for (int i = tid; i < 2 * DP; i += NT) wsum[i] = 0;
    float most = 0.0f;
    scaled(tid, raw, step, mine);
#pragma unroll
    for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(mine[e]));
    for (int t = tid + NT; t < items; t += NT) {
        float st[8], v[8];
        const Raw8 x = fetch(t, st);
        scaled(t, x, st, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(v[e]));
    }
    most = __uint_as_float(wave_all(__float_as_uint(most), [](uint32_t x, uint32_t y) { return x > y ? x : y; }));      // 0 or more: ordered as integers too
    if (lane == 0) red[wave] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) most = fmaxf(most, red[w]);
    // below that, 127 / A would leave the range of binary32
    const float f = most > 1e-30f ? __fdiv_rn(127.0f, most) : 0.0f;
    auto add = [&](int t, const float *v) {
        const int c0 = (t % chunks) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int z = (int)rintf(__fmul_rn(v[e], f));
            if (z) atomicAdd(&wsum[(z > 0 ? DP : 0) + c0 + e], z);      // integers: the order does not matter
        }
    };
    add(tid, mine);
    for (int t = tid + NT; t < items; t += NT) {
        float st[8], v[8];
        const Raw8 x = fetch(t, st);
        scaled(t, x, st, v);
        add(t, v);
    }
    __syncthreads();
    for (int i = tid; i < 2 * DP; i += NT) {
        const int w = wsum[i], a = w < 0 ? -w : w, hi = a >> 7, lo = a & 127;
        digit[0][i] = (int8_t)(w < 0 ? -hi : hi);
        digit[1][i] = (int8_t)(w < 0 ? -lo : lo);
    }
    __syncthreads();

    v4i wd[STEPS];
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
        const v4i zero = {0, 0, 0, 0};
        wd[st] = n < 2 ? *reinterpret_cast<const v4i *>(&digit[n & 1][st * 64 + g * 16]) : zero;
    }
    __shared__ int32_t local[FUSED ? BLOCK_PAGES : 1];
    int32_t *out = FUSED ? local : s.scores + (int64_t)pair * s.table_pages;
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        v4i acc = {0, 0, 0, 0};
#pragma unroll
        for (int st = 0; st < STEPS; ++st) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[u][st], wd[st], acc, 0, 0, 0);
        // column 0: the high digits, column 1: the low ones; register j of lane (n, g): page 4 g + j
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int low = __shfl_xor(acc[j], 1, 64);
            const int there = __shfl(id[u], 4 * g + j, 64);
            const int page = page0 + 16 * u + 4 * g + j;
            if (n == 0 && page < np) out[page] = there < 0 ? INT32_MIN : 128 * acc[j] + low;
        }
    }
    if (FUSED) {
        __syncthreads();
        pick<NT, BLOCK_PAGES / NT, false>(local, np, s, s.pages + (int64_t)pair * s.n_select);
    }
}

template <int DP>
void launch_scores(const KvView &kv, const KvQueries &q, const KvSelect &s, hipStream_t st)
{
    const int pairs = s.nseq * kv.heads;
    if (s.table_pages <= block_pages(256)) kv_score_kernel<DP, 256, true><<<pairs, 256, 0, st>>>(kv, q, s, 1);
    else if (s.table_pages <= FUSED_PAGES) kv_score_kernel<DP, 512, true><<<pairs, 512, 0, st>>>(kv, q, s, 1);
    else {
        const int per = (int)ceil_div(s.table_pages, block_pages(THREADS));
        kv_score_kernel<DP, THREADS, false><<<pairs * per, THREADS, 0, st>>>(kv, q, s, per);
    }
}

}  // namespace

bool kv_select_needs_scores(int64_t table_pages) { return table_pages > FUSED_PAGES; }

hipError_t launch_kv_select(const KvView &kv, const KvQueries &q, const KvSelect &s, hipStream_t st)
{
    if (s.nseq <= 0) return hipSuccess;
    const int pairs = s.nseq * kv.heads;
    switch (kv.dpad) {
    case 64: launch_scores<64>(kv, q, s, st); break;
    case 128: launch_scores<128>(kv, q, s, st); break;
    case 192: launch_scores<192>(kv, q, s, st); break;
    default: launch_scores<256>(kv, q, s, st); break;
    }
    // as few keys to a thread as there are pages for: each step of the bisection looks at all of them
    if (s.table_pages <= FUSED_PAGES) return hipGetLastError();
    if (s.table_pages <= 256 * 4) kv_pick_kernel<256, 4, false><<<pairs, 256, 0, st>>>(kv, s);
    else if (s.table_pages <= 512 * 4) kv_pick_kernel<512, 4, false><<<pairs, 512, 0, st>>>(kv, s);
    else if (s.table_pages <= 1024 * 4) kv_pick_kernel<1024, 4, false><<<pairs, 1024, 0, st>>>(kv, s);
    else if (s.table_pages <= 1024 * 16) kv_pick_kernel<1024, 16, false><<<pairs, 1024, 0, st>>>(kv, s);
    else kv_pick_kernel<1024, 16, true><<<pairs, 1024, 0, st>>>(kv, s);
    return hipGetLastError();
}

}  // namespace lpq
