// Attention of a few or many queries over the paged 8-bit cache.
//
// Rows are the (query, query head) pairs of one kv head, 16 to a matrix tile.  Keys are taken 64 at
// a time: S^T = K Q^T with 16x16x32 bf16 instructions, whose accumulators hold, for lane (j, g), the
// logits of row j and tokens 4g .. 4g+3 of each group of 16 - which is the operand layout of
// O^T = V^T P^T, so the weights never leave the lane's registers.  The cache is stored in operand
// order: a lane's 16 bytes are one load, a wave's load is 1 KiB in a row, and nothing is staged in
// LDS.  e4m3 values are exact in bf16 (V with its power-of-two scale applied on the way, K's scale
// goes into the logits); fp32 queries go as three bf16 planes, weights as two (bf16 results) or three
// (fp32).  Softmax in one pass against a reference that is raised only when a logit passes it by
// more than 2^8, so that most tiles need no exchange between lanes.
//
// Few rows: the four waves of a workgroup take the tiles of a chunk of keys in turn and add their
// results in LDS; with few sequences the keys are cut into chunks over workgroups and joined by a
// second launch.  Bound: HBM (2 dh bytes per token and kv head).  Many rows: a wave has rows of its
// own and walks over all keys; bound by the exponentials and conversions beside the matrix pipe.
#include <hip/hip_runtime.h>
#include <math.h>

#include "common.hpp"
#include "decode.hpp"
#include "launch.hpp"

namespace {

using namespace vscan;

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

constexpr int kTile = kAttendTile, kWaves = kAttendWaves, kGroups = kTile / kCacheGroup;
constexpr float kLazy = 8.f;

// eight e4m3 values (two dwords) times a power of two each -> bf16, exactly
__device__ __forceinline__ bf16x8_t from_fp8(uint32_t lo, uint32_t hi, float s_lo, float s_hi) {
    const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s_lo, false);
    const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s_lo, true);
    const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s_hi, false);
    const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s_hi, true);
    bf16x8_t r = {a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    return r;
}

__device__ __forceinline__ uint32_t word(const uint4 &v, int i) {
    return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
}

// x as `P` bf16 planes whose sum it is (to 8 bits per plane)
template <int P>
__device__ __forceinline__ void split(float x, __bf16 *out) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
        out[p] = (__bf16)x;
        x -= (float)out[p];
    }
}

// Lengths of one sequence as the kernels use them.
struct Span {
    int len, n, first;  // tokens held, queries, position of query 0
};
__device__ __forceinline__ Span span_of(const AttendArgs &a, int b) {
    Span s;
    s.len = min(max(a.kv_len[b], 0), a.max_len);
    s.n = a.new_len ? min(max(a.new_len[b], 0), a.T) : a.T;
    s.first = s.len - s.n;
    return s;
}

// Stores four adjacent dims of an output row.
template <typename T>
__device__ __forceinline__ void store4(T *p, float a, float b, float c, float d);
template <>
__device__ __forceinline__ void store4<float>(float *p, float a, float b, float c, float d) {
    *reinterpret_cast<float4 *>(p) = make_float4(a, b, c, d);
}
template <>
__device__ __forceinline__ void store4<bf16_t>(bf16_t *p, float a, float b, float c, float d) {
    union {
        __bf16 h[4];
        uint2 u;
    } o;
    o.h[0] = (__bf16)a;
    o.h[1] = (__bf16)b;
    o.h[2] = (__bf16)c;
    o.h[3] = (__bf16)d;
    *reinterpret_cast<uint2 *>(p) = o.u;
}

// The 64 keys of a tile: where their groups lie and whether they are there.
struct TileAt {
    int64_t base[kGroups];  // bytes from the start of k_cache / v_cache
    float ks[kGroups], vs[kGroups];
    bool there[kGroups];
};

template <typename T, int DP, int NR, bool ROWS>
__global__ __launch_bounds__(kWaves *kWave) void attend_kernel(AttendArgs a) {
    constexpr int kH = DP / 64;            // 16-byte loads per lane and group
    constexpr int kD = DP / 16;            // tiles of 16 dims
    constexpr bool kF32 = sizeof(T) == 4;
    constexpr int kQ = kF32 ? 3 : 1, kP = kF32 ? 3 : 2;
    constexpr int kRows = 16 * NR;
    extern __shared__ float4 lds4[];

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = lane_id(), j = lane & 15, g = lane >> 4;
    int id = blockIdx.x;
    const int chunk = id % a.chunks;
    id /= a.chunks;
    const int rb = id % a.row_blocks;
    id /= a.row_blocks;
    const int hk = id % a.Hkv, b = id / a.Hkv;
    const int G = a.Hq / a.Hkv, rows = G * a.T;
    const Span sp = span_of(a, b);

    // rows of this wave: row r is query r / G, head hk * G + r % G
    const int row0 = (ROWS ? rb * kWaves + wave : rb) * kRows;
    const int t0 = row0 / G, t1 = min((min(row0 + kRows, rows) - 1) / G, sp.n - 1);
    const bool any = row0 < rows && t0 <= t1;
    const int reach = any ? max(sp.first + t1 + 1, 0) : 0;    // keys the last row sees
    const int all_see = any ? max(sp.first + t0 + 1, 0) : 0;  // keys every row sees
    const int k0 = chunk * a.chunk, k1 = min(k0 + a.chunk, reach);
    // the joining launch reads the chunks that a row reaches into; the first one always
    if (a.chunks > 1 && chunk > 0 && k0 >= reach && !ROWS) return;

    bf16x8_t qf[NR][2 * kH][kQ];
    int lim[NR];
    int64_t row_at[NR];  // element offset of the row in q and out; < 0: no such row
    bool zero[NR];       // a padding row: written as zero
#pragma unroll
    for (int nr = 0; nr < NR; ++nr) {
        const int r = row0 + nr * 16 + j;
        const int t = r / G, head = hk * G + (r - t * G);
        const bool here = r < rows;
        row_at[nr] = here ? (((int64_t)b * a.Hq + head) * a.T + t) * a.dh : -1;
        zero[nr] = t >= sp.n;
        lim[nr] = here && !zero[nr] ? max(sp.first + t + 1, 0) : reach;
        const T *src = static_cast<const T *>(a.q) + (here ? row_at[nr] : 0);
#pragma unroll
        for (int c = 0; c < 2 * kH; ++c) {
            const int d = (c >> 1) * 64 + g * 16 + (c & 1) * 8;
            const bool ok = here && d < a.dh;
            float f[8];
            if constexpr (kF32) {
                unpack16<float>(load16_guard(src, (int64_t)d * 4, ok), f);
                unpack16<float>(load16_guard(src, (int64_t)d * 4 + 16, ok), f + 4);
            } else {
                unpack16<bf16_t>(load16_guard(src, (int64_t)d * 2, ok), f);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                __bf16 p[kQ];
                split<kQ>(f[e], p);
#pragma unroll
                for (int q = 0; q < kQ; ++q) qf[nr][c][q][e] = p[q];
            }
        }
    }

    f32x4_t acc[NR][kD];
    float m[NR], l[NR];
#pragma unroll
    for (int nr = 0; nr < NR; ++nr) {
        m[nr] = -INFINITY;
        l[nr] = 0.f;
#pragma unroll
        for (int d = 0; d < kD; ++d) acc[nr][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }

    const int32_t *table = a.block_table + (int64_t)b * a.max_blocks;
    const int size = 1 << a.block_shift;
    auto locate = [&](int kt, TileAt &at) {
#pragma unroll
        for (int u = 0; u < kGroups; ++u) {
            const int key = kt + u * kCacheGroup;
            at.there[u] = key < k1;
            int block = at.there[u] ? table[key >> a.block_shift] : -1;
            at.there[u] = (unsigned)block < (unsigned)a.n_blocks;
            const int64_t page = at.there[u] ? (int64_t)block * a.Hkv + hk : 0;
            at.base[u] = (page * size + (key & (size - 1))) * DP;
            at.ks[u] = at.there[u] ? a.k_scale[page] * a.scale : 0.f;
            at.vs[u] = at.there[u] ? a.v_scale[page] : 1.f;
        }
    };
    auto fetch = [&](const uint8_t *cache, const TileAt &at, uint4 (*to)[kH]) {
#pragma unroll
        for (int u = 0; u < kGroups; ++u)
#pragma unroll
            for (int h = 0; h < kH; ++h) {
                to[u][h] = zero16();
                if (at.there[u]) to[u][h] = load16(cache + at.base[u], h * 1024 + lane * 16);
            }
    };

    const int step = ROWS ? kTile : kTile * kWaves;
    int kt = k0 + (ROWS ? 0 : wave * kTile);
    TileAt at;
    uint4 kb[kGroups][kH], vb[kGroups][kH];
    if (kt < k1) {
        locate(kt, at);
        fetch(a.k_cache, at, kb);
        fetch(a.v_cache, at, vb);
    }
    for (; kt < k1; kt += step) {
        TileAt next;
        const bool more = kt + step < k1;
        if (more) locate(kt + step, next);

        // logits
        f32x4_t s[NR][kGroups];
#pragma unroll
        for (int u = 0; u < kGroups; ++u) {
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) s[nr][u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < 2 * kH; ++c) {
                const bf16x8_t ka = from_fp8(word(kb[u][c >> 1], 2 * (c & 1)), word(kb[u][c >> 1], 2 * (c & 1) + 1), 1.f, 1.f);
#pragma unroll
                for (int q = kQ - 1; q >= 0; --q)
#pragma unroll
                    for (int nr = 0; nr < NR; ++nr)
                        s[nr][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qf[nr][c][q], s[nr][u], 0, 0, 0);
            }
        }
        if (more) fetch(a.k_cache, next, kb);

        // a tile that every row sees whole needs no masks
        const bool whole = kt + kTile <= all_see && at.there[0] && at.there[1] && at.there[2] && at.there[3];
        if (!whole) {
            // what lies behind the last token is not read as a value
#pragma unroll
            for (int u = 0; u < kGroups; ++u) {
                const int left = sp.len - (kt + u * kCacheGroup + 4 * g);
                const uint32_t keep = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
#pragma unroll
                for (int h = 0; h < kH; ++h) {
                    vb[u][h].x &= keep;
                    vb[u][h].y &= keep;
                    vb[u][h].z &= keep;
                    vb[u][h].w &= keep;
                }
            }
        }
#pragma unroll
        for (int nr = 0; nr < NR; ++nr) {
            float top = -INFINITY;
#pragma unroll
            for (int u = 0; u < kGroups; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float x = s[nr][u][r] * at.ks[u];
                    if (!whole) {
                        const int key = kt + u * kCacheGroup + 4 * g + r;
                        x = at.there[u] && key < lim[nr] ? x : -INFINITY;
                    }
                    s[nr][u][r] = x;
                    top = fmaxf(top, x);
                }
            if (__any(top > m[nr] + kLazy)) {
                top = fmaxf(top, __shfl_xor(top, 16, kWave));
                top = fmaxf(top, __shfl_xor(top, 32, kWave));
                const float now = fmaxf(m[nr], top);
                const float f = now == m[nr] ? 1.f : __builtin_amdgcn_exp2f(m[nr] - now);
                m[nr] = now;
                l[nr] *= f;
#pragma unroll
                for (int d = 0; d < kD; ++d)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[nr][d][r] *= f;
            }
            const float ref = m[nr] == -INFINITY ? 0.f : m[nr];
            float sum = 0.f;
#pragma unroll
            for (int u = 0; u < kGroups; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    s[nr][u][r] = __builtin_amdgcn_exp2f(s[nr][u][r] - ref);
                    sum += s[nr][u][r];
                }
            l[nr] += sum;
        }

        // values
#pragma unroll
        for (int v = 0; v < kGroups / 2; ++v) {
            bf16x8_t pb[NR][kP];
#pragma unroll
            for (int nr = 0; nr < NR; ++nr)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    __bf16 p[kP];
                    split<kP>(s[nr][2 * v + (e >> 2)][e & 3], p);
#pragma unroll
                    for (int q = 0; q < kP; ++q) pb[nr][q][e] = p[q];
                }
#pragma unroll
            for (int d = 0; d < kD; ++d) {
                const bf16x8_t va = from_fp8(word(vb[2 * v][d >> 2], d & 3), word(vb[2 * v + 1][d >> 2], d & 3),
                                             at.vs[2 * v], at.vs[2 * v + 1]);
#pragma unroll
                for (int q = kP - 1; q >= 0; --q)
#pragma unroll
                    for (int nr = 0; nr < NR; ++nr)
                        acc[nr][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pb[nr][q], acc[nr][d], 0, 0, 0);
            }
        }
        if (more) {
            fetch(a.v_cache, next, vb);
            at = next;
        }
    }

#pragma unroll
    for (int nr = 0; nr < NR; ++nr) {
        l[nr] += __shfl_xor(l[nr], 16, kWave);
        l[nr] += __shfl_xor(l[nr], 32, kWave);
    }

    T *out = static_cast<T *>(a.out);
    // Four dims of a finished row: to `out`, or with its maximum and sum to the scratch of the chunk.
    auto finish = [&](int nr, int d, float mx, float sum, f32x4_t o) {
        if (row_at[nr] < 0) return;
        const int dim = 16 * d + 4 * g;
        if (a.chunks == 1) {
            if (dim >= a.dh) return;
            const float f = zero[nr] || !(sum > 0.f) ? 0.f : 1.f / sum;
            if (f == 0.f) o = f32x4_t{0.f, 0.f, 0.f, 0.f};
            store4<T>(out + row_at[nr] + dim, o[0] * f, o[1] * f, o[2] * f, o[3] * f);
            return;
        }
        const int64_t part = (((int64_t)b * a.Hkv + hk) * rows + row0 + nr * 16 + j) * a.chunks + chunk;
        *reinterpret_cast<float4 *>(a.part_acc + part * DP + dim) = make_float4(o[0], o[1], o[2], o[3]);
        if (d == 0 && g == 0) {
            a.part_stat[2 * part] = mx;
            a.part_stat[2 * part + 1] = sum;
        }
    };

    if constexpr (ROWS) {
#pragma unroll
        for (int nr = 0; nr < NR; ++nr)
#pragma unroll
            for (int d = 0; d < kD; ++d) finish(nr, d, m[nr], l[nr], acc[nr][d]);
    } else {
        // the waves' results, 16 rows at a time: [wave][d][lane] and per wave and row (maximum, sum)
        float *stat = reinterpret_cast<float *>(lds4 + kWaves * kD * kWave);
#pragma unroll
        for (int nr = 0; nr < NR; ++nr) {
            __syncthreads();
#pragma unroll
            for (int d = 0; d < kD; ++d)
                lds4[(wave * kD + d) * kWave + lane] = make_float4(acc[nr][d][0], acc[nr][d][1], acc[nr][d][2], acc[nr][d][3]);
            if (g == 0) {
                stat[(wave * 16 + j) * 2] = m[nr];
                stat[(wave * 16 + j) * 2 + 1] = l[nr];
            }
            __syncthreads();
            float mx = -INFINITY, sum = 0.f, f[kWaves];
#pragma unroll
            for (int w = 0; w < kWaves; ++w) mx = fmaxf(mx, stat[(w * 16 + j) * 2]);
            const float ref = mx == -INFINITY ? 0.f : mx;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                f[w] = __builtin_amdgcn_exp2f(stat[(w * 16 + j) * 2] - ref);
                sum += f[w] * stat[(w * 16 + j) * 2 + 1];
            }
#pragma unroll
            for (int i = 0; i < kD / kWaves; ++i) {
                const int d = i * kWaves + wave;
                f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    const float4 x = lds4[(w * kD + d) * kWave + lane];
                    o[0] += f[w] * x.x;
                    o[1] += f[w] * x.y;
                    o[2] += f[w] * x.z;
                    o[3] += f[w] * x.w;
                }
                finish(nr, d, mx, sum, o);
            }
        }
    }
}

// Joins the chunks of a row: one thread per four dims.
constexpr int kCombineThreads = 256;
template <typename T>
__global__ __launch_bounds__(kCombineThreads) void combine_kernel(AttendArgs a, int dp) {
    const int per_row = dp / 4;
    const int64_t id = (int64_t)blockIdx.x * kCombineThreads + threadIdx.x;
    const int G = a.Hq / a.Hkv, rows = G * a.T;
    const int64_t row = id / per_row;
    const int dim = (int)(id % per_row) * 4;
    if (row >= (int64_t)a.B * a.Hkv * rows || dim >= a.dh) return;
    const int r = (int)(row % rows), t = r / G;
    const int64_t bh = row / rows;
    const int hk = (int)(bh % a.Hkv), b = (int)(bh / a.Hkv);
    const Span sp = span_of(a, b);
    const int lim = t < sp.n ? max(sp.first + t + 1, 0) : 0;
    const int n = (int)(((int64_t)lim + a.chunk - 1) / a.chunk);
    float mx = -INFINITY, sum = 0.f;
    const float *stat = a.part_stat + row * a.chunks * 2;
    for (int c = 0; c < n; ++c) mx = fmaxf(mx, stat[2 * c]);
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
    if (mx > -INFINITY) {
        for (int c = 0; c < n; ++c) {
            const float f = __builtin_amdgcn_exp2f(stat[2 * c] - mx);
            const float4 x = *reinterpret_cast<const float4 *>(a.part_acc + (row * a.chunks + c) * dp + dim);
            sum += f * stat[2 * c + 1];
            o[0] += f * x.x;
            o[1] += f * x.y;
            o[2] += f * x.z;
            o[3] += f * x.w;
        }
        const float inv = 1.f / sum;
        for (int e = 0; e < 4; ++e) o[e] *= inv;
    }
    const int64_t at = (((int64_t)b * a.Hq + hk * G + (r - t * G)) * a.T + t) * a.dh + dim;
    store4<T>(static_cast<T *>(a.out) + at, o[0], o[1], o[2], o[3]);
}

template <typename T, int DP, int NR>
hipError_t launch_nr(const AttendArgs &a, hipStream_t s) {
    const dim3 grid((unsigned)((int64_t)a.B * a.Hkv * a.row_blocks * a.chunks));
    if (a.split_rows) {
        hipLaunchKernelGGL((attend_kernel<T, DP, NR, true>), grid, dim3(kWaves * kWave), 0, s, a);
    } else {
        constexpr size_t lds = kWaves * (DP / 16) * kWave * 16 + kWaves * 16 * 2 * sizeof(float);
        if constexpr (lds > 65536) {
            static std::atomic<uint64_t> done{0};
            const hipError_t e = allow_large_lds(attend_kernel<T, DP, NR, false>, done);
            if (e != hipSuccess) return e;
        }
        hipLaunchKernelGGL((attend_kernel<T, DP, NR, false>), grid, dim3(kWaves * kWave), lds, s, a);
    }
    return hipGetLastError();
}

template <typename T, int DP>
hipError_t launch_dp(const AttendArgs &a, hipStream_t s) {
    constexpr int kMost = sizeof(T) == 2 ? (DP > 128 ? 2 : 4) : (DP > 128 ? 1 : 2);
    if (a.row_tiles == 1) return launch_nr<T, DP, 1>(a, s);
    if constexpr (kMost >= 2)
        if (a.row_tiles == 2) return launch_nr<T, DP, 2>(a, s);
    if constexpr (kMost >= 4)
        if (a.row_tiles == 4) return launch_nr<T, DP, 4>(a, s);
    return hipErrorInvalidValue;
}

template <typename T>
hipError_t launch_t(const AttendArgs &a, hipStream_t s) {
    switch (cache_dp(a.dh)) {
        case 64: return launch_dp<T, 64>(a, s);
        case 128: return launch_dp<T, 128>(a, s);
        case 192: return launch_dp<T, 192>(a, s);
        default: return launch_dp<T, 256>(a, s);
    }
}

}  // namespace

namespace vscan {

hipError_t launch_cache_attend(const void *args, hipStream_t s) {
    const AttendArgs &a = *static_cast<const AttendArgs *>(args);
    return a.is_bf16 ? launch_t<bf16_t>(a, s) : launch_t<float>(a, s);
}

hipError_t launch_cache_combine(const void *args, hipStream_t s) {
    const AttendArgs &a = *static_cast<const AttendArgs *>(args);
    const int dp = cache_dp(a.dh);
    const int64_t items = (int64_t)a.B * a.Hq * a.T * (dp / 4);
    const dim3 grid((unsigned)((items + kCombineThreads - 1) / kCombineThreads));
    if (a.is_bf16)
        hipLaunchKernelGGL(combine_kernel<bf16_t>, grid, dim3(kCombineThreads), 0, s, a, dp);
    else
        hipLaunchKernelGGL(combine_kernel<float>, grid, dim3(kCombineThreads), 0, s, a, dp);
    return hipGetLastError();
}

}  // namespace vscan
