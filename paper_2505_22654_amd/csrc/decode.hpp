// Launch interface of the operators around the pruned prefill: rotary positions, the paged 8-bit
// cache and the attention over it.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace vscan {

// One launch of an entry point, timed and logged like the others (api.cpp).
int enqueue(const char *name, hipStream_t s, hipError_t (*launch)(const void *args, hipStream_t s),
            const void *args);

constexpr int kRopeMaxPairs = 128;
struct RopeArgs {
    const void *in[2];             // q, k
    void *out[2];
    int64_t in_stride[2][3];       // elements: sequence, head, token
    int64_t out_stride[2][3];
    int heads[2];
    const int32_t *positions;      // [axes, B, S]
    const double *inv_freq;        // [rot/2]
    int B, S, dh, rot, adjacent, inverse, copy_rest, is_bf16;
    uint8_t axis[kRopeMaxPairs];   // of every pair
};
hipError_t launch_rope(const void *args, hipStream_t s);

// head_dim rounded up to what a 16-byte load per lane of four 16-lane rows covers
inline int cache_dp(int head_dim) { return (head_dim + 63) / 64 * 64; }
constexpr int kCacheGroup = 16;    // tokens of a group: the rows of one matrix operand
constexpr int kScaleExpMin = -120, kScaleExpMax = 120;

struct PlanArgs {
    const int32_t *cached_len, *new_len, *free_blocks, *free_head;
    int32_t *block_table, *slot_map, *kv_len, *free_head_out, *missing;
    int32_t *requests;             // scratch [B, 4]: c, n, first free entry, unused
    int B, n_new, block_shift, n_blocks, max_blocks, n_free;
};
// Workgroups of the launch that reads the lengths, if it writes the tables too, and 0 if a second launch
// has to.  One workgroup may write up to kPlanAlone rows by itself; several, a row a thread, each read all
// lengths, so the requests must fit a workgroup and no input may be overwritten while another reads it.
// GPU time, us: 32 requests, 32 x 3427 rows: two launches 5.9, workgroups of 16384 rows 10.6, 4096 5.6,
// 1024 4.2; 256 x 16 rows: one workgroup 5.4, four 4.1.  (A launch more is 2.5 us of the host's time.)
constexpr int kPlanThreads = 1024, kPlanAlone = 4096;
inline int plan_workgroups(const PlanArgs &a) {
    const int64_t rows = (int64_t)a.B * a.n_new, parts = (rows + kPlanThreads - 1) / kPlanThreads;
    if (a.B <= kPlanThreads && a.kv_len != a.cached_len && a.free_head_out != a.free_head)
        return parts < 1 ? 1 : parts < 256 ? (int)parts : 256;
    return rows <= kPlanAlone ? 1 : 0;
}
// Whether `requests` may be written: not where one launch holds them in LDS whatever overlaps.
inline bool plan_needs_scratch(int64_t B, int64_t n_new) { return B > kPlanThreads || B * n_new > kPlanAlone; }
// Workgroups of a request where a second launch writes the tables.  (n_new may be anything below 2^31.)
constexpr int kTableThreads = 256;
inline int plan_table_parts(int n_new) { return (int)(((int64_t)n_new + kTableThreads * 4 - 1) / (kTableThreads * 4)); }
hipError_t launch_cache_plan(const void *args, hipStream_t s);
hipError_t launch_cache_tables(const void *args, hipStream_t s);

struct StoreArgs {
    const void *x[2];              // k, v
    uint8_t *cache[2];
    float *scale[2];
    const int32_t *slot_map;
    int B, Hkv, n_new, seq_len, dh, block_shift, n_blocks, is_bf16;
};
// Pages (a block's part of one kv head, of k or of v) of a workgroup: a wave or all of it each.  32 sequences
// of 1267 tokens, 8 kv heads x 128 in bf16, GPU time in us of a wave and of a workgroup to a page: blocks of
// 32 32.7 and 44.8, of 64 36.0 and 33.1, of 128 45.3 and 34.1; one token 4.1 and 4.7 in any, but a wave takes
// long to fill or rescale a large page.
constexpr int store_pages(int block_size) { return block_size <= 32 ? 4 : 1; }
// Blocks that n_new rows of a sequence can touch.
constexpr int64_t store_runs(int64_t n_new, int block_size) { return (n_new + block_size - 2) / block_size + 1; }
hipError_t launch_cache_store(const void *args, hipStream_t s);

struct AttendArgs {
    const void *q;
    const uint8_t *k_cache, *v_cache;
    const float *k_scale, *v_scale;
    const int32_t *block_table, *kv_len, *new_len;  // new_len may be NULL
    void *out;
    float *part_acc;               // [B*Hkv, rows, chunks, dp], chunks > 1 only
    float *part_stat;              // [B*Hkv, rows, chunks, 2]: maximum, sum
    int B, Hq, Hkv, T, dh, block_shift, n_blocks, max_blocks, max_len, is_bf16;
    float scale, far_scale;        // times log2(e), and that times kFarScale
    int row_tiles, row_waves, row_blocks, chunk, chunks;  // attend_form
};
constexpr int kAttendWaves = 4;
constexpr float kFarScale = 0x1p24f;
// Keys that a wave takes at a time, by the tiles of 16 rows that it holds.
constexpr int attend_tile(int row_tiles) { return row_tiles > 1 ? 32 : 64; }
constexpr bool attend_many_fits(bool is_bf16, int head_dim) { return is_bf16 || head_dim <= 192; }
// How a call is cut into workgroups: fills the last five fields from the others.
// A workgroup of the few-row kernel holds one tile of 16 rows, of the many-row kernel 32 rows a wave.  16
// sequences of 8 kv heads, 3000 keys, GPU time in us, few and many: 8 rows 19.9 and 21.6, 16 rows 20.4 and
// 22.3, 20 rows (two tiles of 16) 24.5 and 22.3, 32 rows 26.7 and 23.1.  In fp32 with heads above 192 the many-row
// kernel would not fit the registers (4 x 4 kv heads, 1024 rows, 2000 keys 208 us, few rows at a time 100; at
// 192 66 and 82).
// Two of the many-row kernel's waves share their keys, each with rows of its own, where that leaves a
// workgroup a CU: keys are read half as often, but walked by half the waves; not for three tiles of 32 rows, which
// two waves would take as four.  One and two row waves, by the workgroups that two make:
//   1 x 4 kv heads, 63 rows, 2304 keys (4): 14.2, 18.8     4 x 4, 63 rows, 30000 keys (16): 36.2, 39.0
//   16 x 8, 36 rows, 3000 keys (128): 27.7, 31.8           16 x 8, 64 rows (128): 29.3, 33.0
//   64 x 4, 49 rows, 3000 keys (256): 48.1, 44.9           16 x 8, 192 rows (384): 75.6, 68.0
//   64 x 8, 64 rows, 3000 keys (512): 92, 80               64 x 8, 128 rows (1024): 155, 133
//   three tiles: 64 x 8, 80 rows (1024): 118, 137; 96 rows 124, 133; 64 x 4, 96 rows, 2000 keys, heads of 256 99, 111
// (Of an odd number of tiles above that it is either: 64 x 8, 160 rows 188, 173, 224 rows 241, 257, 288 rows 300, 276.)
// Keys are cut into chunks until every CU has one workgroup, as long as each wave has a tile of keys; more
// chunks cost more in the joining launch than they bring:
//   1 x 4 kv heads, 2304 keys: 1 chunk 15.4, 2 13.2, 3 11.4, 9 (a tile a wave) 10.3
//   5 x 8 kv heads, 1391 keys in fp32: 1 chunk 14.5, 3 12.8, 6 11.5
//   4 x 4 kv heads, up to 65536 keys: 8 chunks 52.9, 16 45.1, 32 46.6, 64 52.1, 128 65.2
//   32 x 32 kv heads, up to 3427 keys: 1 chunk 129, 2 136, 4 146
inline void attend_form(AttendArgs &a) {
    constexpr int64_t kCus = 256;
    const int64_t rows = (int64_t)(a.Hq / a.Hkv) * a.T, heads = (int64_t)a.B * a.Hkv;
    a.row_tiles = rows <= kCacheGroup || !attend_many_fits(a.is_bf16, a.dh) ? 1 : 2;
    const int64_t tiles = (rows + 2 * kCacheGroup - 1) / (2 * kCacheGroup);  // of a row wave
    const bool three = tiles == 3 && heads * tiles < (int64_t)1 << 24;  // (as one grid takes them)
    a.row_waves = a.row_tiles == 2 && tiles > 1 && !three && heads * ((tiles + 1) / 2) >= kCus ? 2 : 1;
    const int block = kCacheGroup * a.row_tiles * a.row_waves;
    a.row_blocks = (int)((rows + block - 1) / block);
    const int64_t units = heads * a.row_blocks;
    const int step = attend_tile(a.row_tiles) * kAttendWaves / a.row_waves;
    const int64_t most = a.max_len > step ? (a.max_len + step - 1) / step : 1;
    const int64_t wanted = (kCus + units - 1) / units, chunks = wanted < most ? wanted : most;
    a.chunk = (int)(((a.max_len + chunks - 1) / chunks + step - 1) / step * step);
    if (a.chunk < step) a.chunk = step;
    a.chunks = a.max_len > a.chunk ? (a.max_len + a.chunk - 1) / a.chunk : 1;
}
hipError_t launch_cache_attend(const void *args, hipStream_t s);
hipError_t launch_cache_combine(const void *args, hipStream_t s);

}  // namespace vscan
