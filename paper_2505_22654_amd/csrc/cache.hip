// The paged 8-bit cache: blocks handed to the requests of a batch, and new tokens written.
#include <hip/hip_runtime.h>

#include "common.hpp"
#include "decode.hpp"

namespace {

using namespace vscan;

// ---- block tables, slots and lengths -----------------------------------------------------------
// need_b = ceil((c+n)/size) - ceil(c/size); request b's blocks start at head + sum of the needs
// before it.  One workgroup scans the needs (the bound is its latency: a few dependent rounds of
// loads, shuffles and one barrier pair per 1024 requests); it knows whether there are blocks enough
// only at the end, so the tables are written afterwards, from what it leaves in `requests`.
constexpr int kPlanThreads = 1024;

struct Request {
    int c, n, first;  // tokens held, tokens to come, entry of free_blocks (n < 0: nothing handed out)
};

__device__ __forceinline__ int ceil_shift(int v, int shift) {
    return (int)(((int64_t)v + (1 << shift) - 1) >> shift);
}

// Slots of rows r, r + step, .. of request b, and its table entries.
__device__ void write_request(const PlanArgs &a, int b, const Request &q, int r, int step) {
    const int size_mask = (1 << a.block_shift) - 1;
    const int f = ceil_shift(q.c, a.block_shift);
    int32_t *row = a.block_table + (int64_t)b * a.max_blocks;
    for (; r < a.n_new; r += step) {
        int slot = -1;
        if (r < q.n) {
            const int p = q.c + r, j = p >> a.block_shift;
            const int block = j < f ? row[j] : a.free_blocks[q.first + j - f];
            if (j >= f && ((p & size_mask) == 0)) row[j] = block;
            if ((unsigned)block < (unsigned)a.n_blocks) slot = (block << a.block_shift) + (p & size_mask);
        }
        a.slot_map[(int64_t)b * a.n_new + r] = slot;
    }
}

__global__ __launch_bounds__(kPlanThreads) void cache_plan_kernel(PlanArgs a, int tables) {
    __shared__ int64_t wave_total[kPlanThreads / kWave];
    __shared__ Request held[kPlanThreads];
    const int t = threadIdx.x;
    const int cap = a.max_blocks << a.block_shift;
    const int head = min(max(*a.free_head, 0), a.n_free);
    int64_t before = 0;  // blocks of the requests of earlier rounds
    for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
        const int b = b0 + t;
        int c = 0, n = 0;
        if (b < a.B) {
            c = min(max(a.cached_len[b], 0), cap);
            n = min(max(a.new_len[b], 0), min(a.n_new, cap - c));
        }
        const int need = ceil_shift(c + n, a.block_shift) - ceil_shift(c, a.block_shift);
        int64_t sum = need;  // inclusive over the wave
        for (int d = 1; d < kWave; d *= 2) {
            const int64_t other = __shfl_up(sum, d, kWave);
            if (lane_id() >= d) sum += other;
        }
        __syncthreads();
        if (lane_id() == kWave - 1) wave_total[wave_id()] = sum;
        __syncthreads();
        int64_t mine = before + sum - need;
        for (int w = 0; w < kPlanThreads / kWave; ++w) {
            if (w < wave_id()) mine += wave_total[w];
            before += wave_total[w];
        }
        // an entry past the list is never used: the total is past it too then
        const int first = (int)min((int64_t)head + mine, (int64_t)a.n_free);
        if (b < a.B) {
            a.requests[4 * b] = c;
            a.requests[4 * b + 1] = n;
            a.requests[4 * b + 2] = first;
        }
    }
    const int64_t short_by = head + before - a.n_free;
    if (t == 0) {
        *a.free_head_out = short_by > 0 ? head : head + (int)before;
        *a.missing = short_by > 0 ? (int)min(short_by, (int64_t)0x7fffffff) : 0;
    }
    // every thread takes back what it wrote itself
    for (int b = t; b < a.B; b += kPlanThreads) {
        const int c = a.requests[4 * b], n = a.requests[4 * b + 1];
        a.kv_len[b] = short_by > 0 ? c : c + n;
        if (short_by > 0) a.requests[4 * b + 1] = -1;
    }
    if (!tables) return;
    // threads of a request: as many as it has rows, up to what a round over all requests leaves
    int each = 1;
    while (each < a.n_new && each * 2 * min(a.B, kPlanThreads) <= kPlanThreads) each *= 2;
    const int at_once = kPlanThreads / each;
    for (int b0 = 0; b0 < a.B; b0 += at_once) {
        __syncthreads();
        // request b was written by thread b % kPlanThreads
        const int own = (t - b0) & (kPlanThreads - 1), mine = b0 + own;
        if (own < at_once && mine < a.B)
            held[own] = {a.requests[4 * mine], a.requests[4 * mine + 1], a.requests[4 * mine + 2]};
        __syncthreads();
        const int i = t / each, b = b0 + i;
        if (b < a.B) write_request(a, b, held[i], t % each, each);
    }
}

constexpr int kTableThreads = 256;
__global__ __launch_bounds__(kTableThreads) void cache_tables_kernel(PlanArgs a, int row_parts) {
    const int b = blockIdx.x / row_parts, part = blockIdx.x % row_parts;
    const Request q = {a.requests[4 * b], a.requests[4 * b + 1], a.requests[4 * b + 2]};
    write_request(a, b, q, part * kTableThreads + threadIdx.x, row_parts * kTableThreads);
}

// ---- new keys and values -----------------------------------------------------------------------
// One workgroup per (k or v, sequence, kv head, block that the new rows touch): the largest absolute
// value of the block's new rows gives the scale, then every 16-byte piece of the block that changes
// is made anew.  Bound: HBM (2 or 4 bytes in and one out per value); the rows are read twice, the
// second time from the cache.
constexpr int kStoreThreads = 256;

// least e with amax <= 448 * 2^e (448 = 1.75 * 2^8), held inside what a scale may be
__device__ __forceinline__ int scale_exp(float amax) {
    const uint32_t u = __float_as_uint(amax);
    const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return min(max(e, kScaleExpMin), kScaleExpMax);
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// four floats -> four e4m3 bytes, nearest even
__device__ __forceinline__ uint32_t to_fp8(float a, float b, float c, float d) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}
__device__ __forceinline__ uint32_t rescale_fp8(uint32_t w, float f) {
    return to_fp8(__builtin_amdgcn_cvt_f32_fp8(w, 0) * f, __builtin_amdgcn_cvt_f32_fp8(w, 1) * f,
                  __builtin_amdgcn_cvt_f32_fp8(w, 2) * f, __builtin_amdgcn_cvt_f32_fp8(w, 3) * f);
}

template <typename T>
__global__ __launch_bounds__(kStoreThreads) void cache_store_kernel(StoreArgs a, int dp, int runs) {
    __shared__ float red[kStoreThreads / kWave];
    __shared__ int first_bad;
    const int kind = blockIdx.y;
    const int run = blockIdx.x % runs, hk = blockIdx.x / runs % a.Hkv, b = blockIdx.x / runs / a.Hkv;
    const int size = 1 << a.block_shift;
    const int32_t *slots = a.slot_map + (int64_t)b * a.n_new;
    const int s0 = slots[0];
    const int off0 = s0 >= 0 ? s0 & (size - 1) : 0;
    const int r0 = max(0, run * size - off0), r1 = min(a.n_new, (run + 1) * size - off0);
    if (r0 >= r1) return;
    const int slot = slots[r0];
    if (slot < 0 || (slot >> a.block_shift) >= a.n_blocks) return;
    const int64_t page = (int64_t)(slot >> a.block_shift) * a.Hkv + hk;
    const int off = slot & (size - 1);
    // rows that continue the first one inside its block
    if (threadIdx.x == 0) first_bad = min(r1 - r0, size - off);
    __syncthreads();
    for (int i = threadIdx.x; i < r1 - r0; i += kStoreThreads)
        if (slots[r0 + i] != slot + i) atomicMin(&first_bad, i);
    __syncthreads();
    const int n = first_bad;

    const T *src = static_cast<const T *>(a.x[kind]) + ((int64_t)(b * a.Hkv + hk) * a.seq_len + r0) * a.dh;
    constexpr int kPer = ElemTraits<T>::kPer16B;
    float amax = 0.f;
    for (int i = threadIdx.x; i < n * a.dh / kPer; i += kStoreThreads) {
        float f[kPer];
        unpack16<T>(load16(src, (int64_t)i * 16), f);
#pragma unroll
        for (int e = 0; e < kPer; ++e) amax = fmaxf(amax, fabsf(f[e]));
    }
    amax = block_max(amax, red);
    const bool begun = off == 0;
    float *scale = a.scale[kind] + page;
    int e = scale_exp(amax), e_old = e;
    if (!begun) {
        e_old = (int)(__float_as_uint(*scale) >> 23 & 255u) - 127;
        e_old = min(max(e_old, kScaleExpMin), kScaleExpMax);
        e = max(e, e_old);
    }
    __syncthreads();
    if (threadIdx.x == 0) *scale = pow2(e);
    const bool grown = e > e_old;
    const float inv = pow2(-e), shrink = pow2(max(e_old - e, -126));

    // pieces: dp of 16 bytes per group of 16 tokens
    uint8_t *block = a.cache[kind] + page * size * dp;
    const int g0 = begun || grown ? 0 : off / kCacheGroup;
    const int g1 = begun ? size / kCacheGroup : (off + n + kCacheGroup - 1) / kCacheGroup;
    for (int i = threadIdx.x; i < (g1 - g0) * dp; i += kStoreThreads) {
        const int group = g0 + i / dp, piece = i % dp;
        uint4 *dst = reinterpret_cast<uint4 *>(block + (int64_t)(group * dp + piece) * kCacheGroup);
        uint4 out = begun ? zero16() : *dst;
        uint32_t *w = &out.x;
        if (kind == 0) {  // 16 dims of one token
            const int row = group * kCacheGroup + piece % kCacheGroup - off, d0 = piece / kCacheGroup * 16;
            if (row >= n || (row < 0 && !grown)) {
                if (!begun) continue;
            } else if (row < 0) {
                for (int j = 0; j < 4; ++j) w[j] = rescale_fp8(w[j], shrink);
            } else {
                float f[16];
                for (int j = 0; j < 16; ++j)
                    f[j] = d0 + j < a.dh ? load_elem(src + (int64_t)row * a.dh + d0 + j) * inv : 0.f;
                for (int j = 0; j < 4; ++j) w[j] = to_fp8(f[4 * j], f[4 * j + 1], f[4 * j + 2], f[4 * j + 3]);
            }
        } else {  // four tokens of dims d0, d0 + 16, d0 + 32, d0 + 48
            const int row = group * kCacheGroup + piece / 16 % 4 * 4 - off, d0 = piece / 64 * 64 + piece % 16;
            if (!begun && (row >= n || (row + 3 < 0 && !grown))) continue;
            for (int j = 0; j < 4; ++j) {
                const int d = d0 + 16 * j;
                float f[4];
                uint32_t fresh = 0;  // bytes of new tokens
                for (int r = 0; r < 4; ++r) {
                    const bool is_new = row + r >= 0 && row + r < n;
                    fresh |= is_new ? 0xffu << (8 * r) : 0u;
                    f[r] = is_new && d < a.dh ? load_elem(src + (int64_t)(row + r) * a.dh + d) * inv : 0.f;
                }
                const uint32_t now = to_fp8(f[0], f[1], f[2], f[3]);
                uint32_t old = w[j];
                if (grown) {  // bytes of the tokens before the new ones
                    const uint32_t before = row >= 0 ? 0u : row <= -4 ? ~0u : (1u << (8 * -row)) - 1u;
                    old = (rescale_fp8(old, shrink) & before) | (old & ~before);
                }
                w[j] = (now & fresh) | (old & ~fresh);
            }
        }
        *dst = out;
    }
}

}  // namespace

namespace vscan {

hipError_t launch_cache_plan(const void *args, hipStream_t s) {
    const PlanArgs &a = *static_cast<const PlanArgs *>(args);
    hipLaunchKernelGGL(cache_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, a, plan_in_one(a) ? 1 : 0);
    return hipGetLastError();
}

hipError_t launch_cache_tables(const void *args, hipStream_t s) {
    const PlanArgs &a = *static_cast<const PlanArgs *>(args);
    const int parts = (a.n_new + kTableThreads * 4 - 1) / (kTableThreads * 4);
    hipLaunchKernelGGL(cache_tables_kernel, dim3(a.B * parts), dim3(kTableThreads), 0, s, a, parts);
    return hipGetLastError();
}

hipError_t launch_cache_store(const void *args, hipStream_t s) {
    const StoreArgs &a = *static_cast<const StoreArgs *>(args);
    const int runs = (a.n_new + (1 << a.block_shift) - 2) / (1 << a.block_shift) + 1;
    const dim3 grid(a.B * a.Hkv * runs, 2);
    if (a.is_bf16)
        hipLaunchKernelGGL(cache_store_kernel<bf16_t>, grid, dim3(kStoreThreads), 0, s, a, cache_dp(a.dh), runs);
    else
        hipLaunchKernelGGL(cache_store_kernel<float>, grid, dim3(kStoreThreads), 0, s, a, cache_dp(a.dh), runs);
    return hipGetLastError();
}

}  // namespace vscan
