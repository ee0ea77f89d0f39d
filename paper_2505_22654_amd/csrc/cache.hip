// The paged 8-bit cache: blocks handed to the requests of a batch, and new tokens written.
#include <hip/hip_runtime.h>

#include "common.hpp"
#include "decode.hpp"

namespace {

using namespace vscan;

// ---- block tables, slots and lengths -----------------------------------------------------------
// need_b = ceil((c+n)/size) - ceil(c/size); request b's blocks start at head + sum of the needs
// before it.  A workgroup scans the needs (the bound is its latency: a few dependent rounds of
// loads, shuffles and one barrier pair per 1024 requests); it knows whether there are blocks enough
// only at the end, so the tables are written afterwards.  Where a launch writes them too, each of its
// workgroups scans for itself and keeps the requests in LDS; only the first writes lengths and head.
struct Request {
    int c, n, first;  // tokens held, tokens to come, entry of free_blocks (n < 0: nothing handed out)
};

__device__ __forceinline__ int ceil_shift(int v, int shift) {
    return (int)(((int64_t)v + (1 << shift) - 1) >> shift);
}

// The slot of row r of request b, and the table entry of a block that it begins.
__device__ __forceinline__ void write_row(const PlanArgs &a, int b, const Request &q, int r) {
    const int size_mask = (1 << a.block_shift) - 1;
    const int f = ceil_shift(q.c, a.block_shift);
    int slot = -1;
    if (r < q.n) {
        int32_t *row = a.block_table + (int64_t)b * a.max_blocks;
        const int p = q.c + r, j = p >> a.block_shift;
        const int block = j < f ? row[j] : a.free_blocks[q.first + j - f];
        if (j >= f && ((p & size_mask) == 0)) row[j] = block;
        if ((unsigned)block < (unsigned)a.n_blocks) slot = (block << a.block_shift) + (p & size_mask);
    }
    a.slot_map[(int64_t)b * a.n_new + r] = slot;
}

__global__ __launch_bounds__(kPlanThreads) void cache_plan_kernel(PlanArgs a, int tables) {
    __shared__ int64_t wave_total[kPlanThreads / kWave];
    __shared__ Request held[kPlanThreads];
    const int t = threadIdx.x;
    const bool in_lds = tables && a.B <= kPlanThreads;
    const int cap = a.max_blocks << a.block_shift;
    const int head = min(max(*a.free_head, 0), a.n_free);
    int64_t before = 0;  // blocks of the requests of earlier rounds
    Request own = {};
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
        own = {c, n, (int)min((int64_t)head + mine, (int64_t)a.n_free)};
        if (!in_lds && b < a.B) {
            a.requests[4 * b] = own.c;
            a.requests[4 * b + 1] = own.n;
            a.requests[4 * b + 2] = own.first;
        }
    }
    const int64_t short_by = head + before - a.n_free;
    if (blockIdx.x == 0) {
        if (t == 0) {
            *a.free_head_out = short_by > 0 ? head : head + (int)before;
            *a.missing = short_by > 0 ? (int)min(short_by, (int64_t)0x7fffffff) : 0;
        }
        // every thread takes back what it wrote itself
        for (int b = t; b < a.B; b += kPlanThreads) {
            const int c = in_lds ? own.c : a.requests[4 * b], n = in_lds ? own.n : a.requests[4 * b + 1];
            a.kv_len[b] = short_by > 0 ? c : c + n;
            if (!in_lds && short_by > 0) a.requests[4 * b + 1] = -1;
        }
    }
    if (!tables) return;
    held[t] = {own.c, short_by > 0 ? -1 : own.n, own.first};
    __syncthreads();
    const uint32_t rows = (uint32_t)a.B * a.n_new;
    for (uint32_t i = blockIdx.x * kPlanThreads + t; i < rows; i += gridDim.x * kPlanThreads) {
        const int b = i / (uint32_t)a.n_new;
        const Request q = in_lds ? held[b] : Request{a.requests[4 * b], a.requests[4 * b + 1], a.requests[4 * b + 2]};
        write_row(a, b, q, i - (uint32_t)b * a.n_new);
    }
}

__global__ __launch_bounds__(kTableThreads) void cache_tables_kernel(PlanArgs a, int row_parts) {
    const int b = blockIdx.x / row_parts, part = blockIdx.x % row_parts;
    const Request q = {a.requests[4 * b], a.requests[4 * b + 1], a.requests[4 * b + 2]};
    // (unsigned: the last step goes past n_new by a quarter of it)
    for (uint32_t r = part * kTableThreads + threadIdx.x; r < (uint32_t)a.n_new; r += row_parts * kTableThreads)
        write_row(a, b, q, (int)r);
}

// ---- new keys and values -----------------------------------------------------------------------
// A page (a block's part of one kv head, of k or of v) is the work of one wave up to 32 tokens, of a
// workgroup above.  A lane owns units of 4 tokens x 8 dims: it loads them with whole rows side by side,
// and keeps them while the largest absolute value of the page's new rows gives the scale.  After
// rounding it holds 32 bytes that belong to pieces of its neighbours: one exchange (k) or a 4x4
// transposition (v) between lanes of a quad leaves two whole 16-byte pieces of the page per unit.
// Bound: HBM (2 or 4 bytes in and one out per value).  32 sequences of up to 1267 tokens, 32 heads x 128 in
// bf16 (803 MB): 154 us cold (5.2 TB/s, as a copy), in fp32 (1.34 GB) 259; one token of each 4.7 us, in fp32 4.5, a
// launch's latency.  With every
// page's rows requested before its slot is known, which hides a load but reads the rows of ragged batches
// that go nowhere, 190 us; loads with the non-temporal hint 160 (8 heads, 35 MB, from the caches: 31 us
// without, 36 with); stores with it 258, as no store fills a line by itself.
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

// the value of the lane whose number differs in bit 0 (or bit 1)
__device__ __forceinline__ uint32_t from_xor1(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, true);
}
__device__ __forceinline__ uint32_t from_xor2(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, true);
}
// w[e] of lane q of a quad -> w[q] of lane e, as w[e]
__device__ __forceinline__ void transpose4(uint32_t *w, int q) {
    const bool o1 = q & 1, o2 = q & 2;
#pragma unroll
    for (int e = 0; e < 4; e += 2) {
        const uint32_t r = from_xor1(o1 ? w[e] : w[e + 1]);
        if (o1) w[e] = r;
        else w[e + 1] = r;
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const uint32_t r = from_xor2(o2 ? w[e] : w[e + 2]);
        if (o2) w[e] = r;
        else w[e + 2] = r;
    }
}

// A unit of a page: 4 tokens from `token` on, 8 dims from `dim` on, and where its two pieces lie.
struct Unit {
    int token, dim, piece[2], piece_token[2];  // bytes from the start of the page
};
template <int DP>
__device__ __forceinline__ Unit unit_at(int u, int kind) {
    const int p = u % (DP / 8), quad = u / (DP / 8), group = (quad >> 2) * kCacheGroup * DP;
    Unit r;
    r.token = quad * 4;
    if (kind == 0) {  // [dp/16][16 tokens][16 dims]: lanes 2c and 2c + 1 hold the halves of column c
        r.dim = p * 8;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            r.piece_token[i] = quad * 4 + 2 * i + (p & 1);
            r.piece[i] = group + (p >> 1) * 256 + ((quad & 3) * 4 + 2 * i + (p & 1)) * 16;
        }
    } else {  // [dp/64][4 quads][16 dims][4][4 tokens]: the lanes of a quad hold dims 16 apart
        r.dim = (p >> 3) * 64 + (p & 3) * 16 + (p >> 2 & 1) * 8;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            r.piece_token[i] = quad * 4;
            r.piece[i] = group + (p >> 3) * 1024 + (quad & 3) * 256 + ((p >> 2 & 1) * 8 + 4 * i + (p & 3)) * 16;
        }
    }
    return r;
}

// What a unit's rows look like in memory: 8 entries of each of 4 tokens.
template <typename T>
struct Rows {
    static constexpr int kLoads = 8 / ElemTraits<T>::kPer16B;
    uint4 raw[4][kLoads];
    __device__ __forceinline__ void load(const T *src, int row, int n, int dim, int dh) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                raw[j][i] = load16_guard(src, ((int64_t)(row + j) * dh + dim) * (int)sizeof(T) + 16 * i,
                                         row + j >= 0 && row + j < n && dim < dh);
    }
    __device__ __forceinline__ void get(int j, float *f) const {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) unpack16<T>(raw[j][i], f + i * ElemTraits<T>::kPer16B);
    }
    // rows from n on were read before it was known that they go elsewhere
    __device__ __forceinline__ float largest(int row, int n, bool finite) const {
        float m = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float f[8], r = 0.f;
            get(j, f);
#pragma unroll
            for (int e = 0; e < 8; ++e) r = fmaxf(r, finite && fabsf(f[e]) == INFINITY ? 0.f : fabsf(f[e]));
            m = row + j < n ? fmaxf(m, r) : m;
        }
        return m;
    }
    // the unit's two pieces
    __device__ __forceinline__ void pieces(int kind, float inv, uint4 *out) const {
        if (kind == 0) {
            uint32_t w[4][2];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float f[8];
                get(j, f);
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] *= inv;
                w[j][0] = to_fp8(f[0], f[1], f[2], f[3]);
                w[j][1] = to_fp8(f[4], f[5], f[6], f[7]);
            }
            const bool odd = lane_id() & 1;
#pragma unroll
            for (int i = 0; i < 2; ++i) {  // even lanes keep tokens 0 and 2, odd ones 1 and 3
                const uint32_t *mine = odd ? w[2 * i + 1] : w[2 * i], *theirs = odd ? w[2 * i] : w[2 * i + 1];
                const uint32_t a = mine[0], b = mine[1];
                const uint32_t c = from_xor1(theirs[0]), d = from_xor1(theirs[1]);
                out[i] = odd ? make_uint4(c, d, a, b) : make_uint4(a, b, c, d);
            }
        } else {
            float f[4][8];
#pragma unroll
            for (int j = 0; j < 4; ++j) get(j, f[j]);
            uint32_t w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = to_fp8(f[0][e] * inv, f[1][e] * inv, f[2][e] * inv, f[3][e] * inv);
            transpose4(w, lane_id() & 3);
            transpose4(w + 4, lane_id() & 3);
            out[0] = make_uint4(w[0], w[1], w[2], w[3]);
            out[1] = make_uint4(w[4], w[5], w[6], w[7]);
        }
    }
};

// kHold: units that a lane keeps between the two passes; further ones are read again.
template <typename T, int DP, int LANES, int kHold>
__global__ __launch_bounds__(kStoreThreads) void cache_store_kernel(StoreArgs a, int runs, int pages) {
    __shared__ float red[kStoreThreads / kWave];
    __shared__ int first_bad;
    const int lane = threadIdx.x % LANES;
    int id = blockIdx.x * (kStoreThreads / LANES) + (LANES == kWave ? __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) : 0);
    if (id >= pages) return;
    const int kind = id % 2;
    id /= 2;
    const int run = id % runs, hk = id / runs % a.Hkv, b = id / runs / a.Hkv;
    const int size = 1 << a.block_shift;
    const int32_t *slots = a.slot_map + (int64_t)b * a.n_new;
    const int s0 = slots[0];
    const int off0 = s0 >= 0 ? s0 & (size - 1) : 0;
    const int r0 = max(0, run * size - off0), r1 = min(a.n_new, (run + 1) * size - off0);
    if (r0 >= r1) return;
    // the run's rows start at this offset wherever they go (off below, for slots as they are made)
    const int at0 = run ? 0 : off0;
    const T *src = static_cast<const T *>(a.x[kind]) + ((int64_t)(b * a.Hkv + hk) * a.seq_len + r0) * a.dh;
    const int q0 = at0 / 4, q1 = (at0 + r1 - r0 + 3) / 4;  // quads of tokens that the rows lie in
    const int units = (q1 - q0) * (DP / 8);
    Rows<T> held[kHold];
    auto load = [&](int rows) {
#pragma unroll
        for (int i = 0; i < kHold; ++i) {
            const int u = lane + i * LANES;
            if (u < units) {
                const Unit un = unit_at<DP>(q0 * (DP / 8) + u, kind);
                held[i].load(src, un.token - at0, rows, un.dim, a.dh);
            }
        }
    };

    int n = r1 - r0;
    const int mine = slots[r0 + min(lane, n - 1)], slot = run ? slots[r0] : s0;
    if (slot < 0 || (slot >> a.block_shift) >= a.n_blocks || (slot & (size - 1)) != at0) return;
    if (run == 0) load(n);  // ahead of knowing how many of them follow each other: a token's latency
    const int64_t page = (int64_t)(slot >> a.block_shift) * a.Hkv + hk;
    // rows that continue the first one
    if constexpr (LANES == kWave) {
        const uint64_t bad = __ballot(lane < n && mine != slot + lane);
        if (bad) n = __ffsll((unsigned long long)bad) - 1;
    } else {
        if (lane == 0) first_bad = n;
        __syncthreads();
        if (lane < n && mine != slot + lane) atomicMin(&first_bad, lane);
        __syncthreads();
        n = first_bad;
    }
    if (run) load(n);
    // (fmaxf passes NaN over)
    auto largest = [&](bool finite) {
        float m = 0.f;
#pragma unroll
        for (int i = 0; i < kHold; ++i) {
            const int u = lane + i * LANES;
            if (u < units) m = fmaxf(m, held[i].largest(unit_at<DP>(q0 * (DP / 8) + u, kind).token - at0, n, finite));
        }
        for (int u = lane + kHold * LANES; u < units; u += LANES) {
            const Unit un = unit_at<DP>(q0 * (DP / 8) + u, kind);
            Rows<T> rows;
            rows.load(src, un.token - at0, n, un.dim, a.dh);
            m = fmaxf(m, rows.largest(un.token - at0, n, finite));
        }
        if constexpr (LANES > kWave) return block_max(m, red);
        else return wave_max(m);
    };
    float amax = largest(false);
    if (amax == INFINITY) amax = largest(true);

    const bool begun = at0 == 0;
    float *scale = a.scale[kind] + page;
    int e = scale_exp(amax), e_old = e;
    if (!begun) {
        e_old = (int)(__float_as_uint(*scale) >> 23 & 255u) - 127;
        e_old = min(max(e_old, kScaleExpMin), kScaleExpMax);
        e = max(e, e_old);
    }
    if constexpr (LANES > kWave) __syncthreads();
    if (lane == 0) *scale = pow2(e);
    const bool grown = e > e_old;
    const float inv = pow2(-e), shrink = pow2(max(e_old - e, -126));
    uint8_t *block = a.cache[kind] + page * size * DP;

    // Bytes of a piece's tokens: new ones from `now`, earlier ones as they are or under the larger
    // scale, later ones zero in a block that is begun and as they are in another.
    auto write = [&](const Unit &un, const uint4 *now) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = un.piece_token[i] - at0;
            const uint32_t one = row >= 0 && row < n ? ~0u : 0u;  // k: the token of the piece
            uint32_t fresh = one, earlier = row < 0 ? ~0u : 0u;
            if (kind == 1) {
                fresh = 0;
#pragma unroll
                for (int r = 0; r < 4; ++r) fresh |= row + r >= 0 && row + r < n ? 0xffu << (8 * r) : 0u;
                earlier = row >= 0 ? 0u : row <= -4 ? ~0u : (1u << (8 * -row)) - 1u;
            }
            if (!begun && fresh == 0 && !(grown && earlier)) continue;
            uint4 *dst = reinterpret_cast<uint4 *>(block + un.piece[i]);
            uint4 out = zero16();
            if (!begun && fresh != ~0u) {
                out = *dst;
                if (grown && earlier) {
                    out.x = (rescale_fp8(out.x, shrink) & earlier) | (out.x & ~earlier);
                    out.y = (rescale_fp8(out.y, shrink) & earlier) | (out.y & ~earlier);
                    out.z = (rescale_fp8(out.z, shrink) & earlier) | (out.z & ~earlier);
                    out.w = (rescale_fp8(out.w, shrink) & earlier) | (out.w & ~earlier);
                }
            }
            out.x = (now[i].x & fresh) | (out.x & ~fresh);
            out.y = (now[i].y & fresh) | (out.y & ~fresh);
            out.z = (now[i].z & fresh) | (out.z & ~fresh);
            out.w = (now[i].w & fresh) | (out.w & ~fresh);
            *dst = out;
        }
    };
    // (the exchanges between lanes: units of a quad of lanes end together, a page has a multiple of 8)
    uint4 now[2];
#pragma unroll
    for (int i = 0; i < kHold; ++i) {
        const int u = lane + i * LANES;
        if (u < units) {
            held[i].pieces(kind, inv, now);
            write(unit_at<DP>(q0 * (DP / 8) + u, kind), now);
        }
    }
    for (int u = lane + kHold * LANES; u < units; u += LANES) {
        const Unit un = unit_at<DP>(q0 * (DP / 8) + u, kind);
        Rows<T> rows;
        rows.load(src, un.token - at0, n, un.dim, a.dh);
        rows.pieces(kind, inv, now);
        write(un, now);
    }
    now[0] = now[1] = zero16();
    if (begun)
        for (int u = q1 * (DP / 8) + lane; u < size / 4 * (DP / 8); u += LANES) write(unit_at<DP>(u, kind), now);
    else if (grown)
        for (int u = lane; u < q0 * (DP / 8); u += LANES) write(unit_at<DP>(u, kind), now);
}

template <typename T, int DP, int LANES, int kHold>
hipError_t launch_store_as(const StoreArgs &a, hipStream_t s) {
    const int runs = (int)store_runs(a.n_new, 1 << a.block_shift);
    const int pages = 2 * a.B * a.Hkv * runs, per = kStoreThreads / LANES;
    hipLaunchKernelGGL((cache_store_kernel<T, DP, LANES, kHold>), dim3((pages + per - 1) / per), dim3(kStoreThreads), 0,
                       s, a, runs, pages);
    return hipGetLastError();
}

// A lane holds no more units than it can meet: 32 sequences of 1267 tokens, 8 kv heads x 128 in bf16, GPU
// time in us with just enough units and with four: blocks of 16 31.2 and 41.4, of 32 (two units) 32.7 and
// 34.5, of 64 33.1 and 47.3, of 128 (two) 34.1 and 38.0.
template <typename T, int DP, int LANES>
hipError_t launch_store_lanes(const StoreArgs &a, int units, hipStream_t s) {
    constexpr int kMost = sizeof(T) == 2 ? 4 : 2;  // 64 registers
    constexpr int kPage = (LANES == kWave ? 32 : 256) / 4 * (DP / 8);  // units of the largest page
    if constexpr (kPage > 2 * LANES && kMost > 2)
        if (units > 2 * LANES) return launch_store_as<T, DP, LANES, kMost>(a, s);
    if constexpr (kPage > LANES)
        if (units > LANES) return launch_store_as<T, DP, LANES, 2>(a, s);
    return launch_store_as<T, DP, LANES, 1>(a, s);
}

template <typename T, int DP>
hipError_t launch_store_dp(const StoreArgs &a, hipStream_t s) {
    const int size = 1 << a.block_shift;
    // quads that one call's rows can lie in
    const int units = min(size / 4, (a.n_new + 6) / 4) * (DP / 8);
    return store_pages(size) > 1 ? launch_store_lanes<T, DP, kWave>(a, units, s)
                                 : launch_store_lanes<T, DP, kStoreThreads>(a, units, s);
}

template <typename T>
hipError_t launch_store_t(const StoreArgs &a, hipStream_t s) {
    switch (cache_dp(a.dh)) {
        case 64: return launch_store_dp<T, 64>(a, s);
        case 128: return launch_store_dp<T, 128>(a, s);
        case 192: return launch_store_dp<T, 192>(a, s);
        default: return launch_store_dp<T, 256>(a, s);
    }
}

}  // namespace

namespace vscan {

hipError_t launch_cache_plan(const void *args, hipStream_t s) {
    const PlanArgs &a = *static_cast<const PlanArgs *>(args);
    const int workgroups = plan_workgroups(a);
    hipLaunchKernelGGL(cache_plan_kernel, dim3(workgroups ? workgroups : 1), dim3(kPlanThreads), 0, s, a, workgroups > 0);
    return hipGetLastError();
}

hipError_t launch_cache_tables(const void *args, hipStream_t s) {
    const PlanArgs &a = *static_cast<const PlanArgs *>(args);
    const int parts = plan_table_parts(a.n_new);
    hipLaunchKernelGGL(cache_tables_kernel, dim3(a.B * parts), dim3(kTableThreads), 0, s, a, parts);
    return hipGetLastError();
}

hipError_t launch_cache_store(const void *args, hipStream_t s) {
    const StoreArgs &a = *static_cast<const StoreArgs *>(args);
    return a.is_bf16 ? launch_store_t<bf16_t>(a, s) : launch_store_t<float>(a, s);
}

}  // namespace vscan
