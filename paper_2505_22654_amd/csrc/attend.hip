// Attention of a few or many queries over the paged 8-bit cache.
//
// Rows are the (query, query head) pairs of one kv head, 16 to a matrix tile.  S^T = K Q^T with
// 16x16x32 instructions, whose accumulators hold, for lane (j, g), the logits of row j and tokens
// 4g .. 4g+3 of each group of 16 - which is the operand layout of O^T = V^T P^T, so the weights never
// leave the lane's registers.  The cache is stored in operand order: a lane's 16 bytes are one load, a
// wave's load is 1 KiB in a row, and nothing is staged in LDS.
//
// bf16 calls: K as bf16 (exact) times q; V as fp16 (exact) times the weights in fp16 (2^-11 of each;
// bf16's 2^-8 would add as much to the error as the result's own rounding).  fp32 calls: q and the
// weights as three bf16 planes each, V as bf16.  K's scale goes into the logits; V's, a power of two,
// is taken relative to the largest that the wave has met: down to 2^-15 with the values, beyond that
// with the weights, whose reference it then enters, so that the largest contributions keep their bits.
// Softmax in one pass against a reference that is raised only where a logit passes it by more than
// 2^8, so that most tiles need no exchange between lanes.
//
// The four waves of a workgroup take the tiles of its keys in turn and add their results in LDS; where
// sequences and rows leave compute units idle the keys are cut into chunks over workgroups, which a
// second launch joins.  Few rows: bound by HBM (2 dh bytes per token and kv head).  Many rows: by the
// vector instructions beside the matrix pipe (per logit a multiply-add, a maximum, an exponential and
// a sum, and the conversions).
#include <hip/hip_runtime.h>
#include <math.h>

#include <type_traits>

#include "common.hpp"
#include "decode.hpp"
#include "launch.hpp"

namespace {

using namespace vscan;

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

constexpr int kWaves = kAttendWaves;
constexpr float kNothing = -1e30f;  // reference of a row that has seen no key
constexpr float kBias = 4.f;        // the largest weight is 2^4 when the reference is set ..
constexpr float kRaise = 12.f;      // .. and at most 2^12 until it is raised (fp16 holds 2^16)
constexpr int kValueExp = -15;      // e4m3's 2^-9 times 2^-15 is fp16's smallest number
constexpr int kWeightExp = -100;    // sums of weights without this factor stay inside fp32

template <typename T>
struct Operand;  // what V and the weights are multiplied as
template <>
struct Operand<bf16_t> {
    typedef f16x8_t vec;
    typedef f16x2_t pair;
    static constexpr int kPlanes = 1, kQueryPlanes = 1;
    static __device__ __forceinline__ pair from_fp8(uint32_t w, float s, bool hi) {
        return hi ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, s, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, s, false);
    }
    static __device__ __forceinline__ f32x4_t mfma(vec a, vec b, f32x4_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
};
template <>
struct Operand<float> {
    typedef bf16x8_t vec;
    typedef bf16x2_t pair;
    static constexpr int kPlanes = 3, kQueryPlanes = 3;
    static __device__ __forceinline__ pair from_fp8(uint32_t w, float s, bool hi) {
        return hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false);
    }
    static __device__ __forceinline__ f32x4_t mfma(vec a, vec b, f32x4_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};

// eight e4m3 values (two dwords), times a power of two each dword
template <typename O>
__device__ __forceinline__ typename O::vec from_fp8(uint32_t lo, uint32_t hi, float s_lo, float s_hi) {
    const typename O::pair a = O::from_fp8(lo, s_lo, false), b = O::from_fp8(lo, s_lo, true);
    const typename O::pair c = O::from_fp8(hi, s_hi, false), d = O::from_fp8(hi, s_hi, true);
    typename O::vec r = {a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    return r;
}

__device__ __forceinline__ uint32_t word(const uint4 &v, int i) {
    return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
}

// Two numbers as P planes of the operand's type, whose sum they are (to its bits per plane).
template <typename O, int P>
__device__ __forceinline__ void split(f32x2_t x, typename O::pair *out) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
        out[p] = __builtin_convertvector(x, typename O::pair);
        if (p + 1 < P) {
            x[0] -= (float)out[p][0];
            x[1] -= (float)out[p][1];
        }
    }
}

// Exponent of a power of two.
__device__ __forceinline__ int exp_of(float s) {
    const int e = (int)(__float_as_uint(s) >> 23 & 255u) - 127;
    return min(max(e, kScaleExpMin), kScaleExpMax);
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(min(max(e, -126), 127) + 127) << 23); }

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
__device__ __forceinline__ void store4(T *p, f32x4_t v);
template <>
__device__ __forceinline__ void store4<float>(float *p, f32x4_t v) {
    *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
}
template <>
__device__ __forceinline__ void store4<bf16_t>(bf16_t *p, f32x4_t v) {
    union {
        __bf16 h[4];
        uint2 u;
    } o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o.h[i] = (__bf16)v[i];
    *reinterpret_cast<uint2 *>(p) = o.u;
}

// The keys of a tile: where its groups of 16 lie, and their scales.
template <int kGroups>
struct TileAt {
    int64_t base[kGroups];  // bytes from the start of k_cache / v_cache
    float ks[kGroups], vs[kGroups];
    bool there[kGroups];
};

template <typename T, int DP, int NR, int kTile>
__global__ __launch_bounds__(kWaves *kWave, DP <= 128 && sizeof(T) == 2 ? 2 : 1) void attend_kernel(AttendArgs a) {
    typedef Operand<T> O;
    constexpr int kGroups = kTile / kCacheGroup;
    constexpr int kStages = NR > 1 && DP <= 128 ? 2 : 1;  // tiles in flight
    constexpr int kH = DP / 64;  // 16-byte loads per lane and group
    constexpr int kD = DP / 16;  // tiles of 16 dims
    constexpr int kQ = O::kQueryPlanes, kP = O::kPlanes;
    extern __shared__ float4 lds4[];

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = lane_id(), j = lane & 15, g = lane >> 4;
    int id = blockIdx.x;
    const int chunk = id % a.chunks;
    id /= a.chunks;
    const int rb = id % a.row_blocks;
    id /= a.row_blocks;
    const int hk = id % a.Hkv, b = id / a.Hkv;
    const int G = a.Hq / a.Hkv, rows = G * a.T, size = 1 << a.block_shift;
    const int32_t *table = a.block_table + (int64_t)b * a.max_blocks;

    const int k0 = chunk * a.chunk, step = kTile * kWaves;
    int kt = k0 + wave * kTile;
    // Block numbers of the wave's next kBatch tiles, a group of 16 tokens to a lane; the first are read
    // ahead of knowing whether the tokens are there.
    constexpr int kBatch = kWave / kGroups;
    auto blocks_from = [&](int kt) {
        const int64_t key = kt + (int64_t)(lane / kGroups) * step + lane % kGroups * kCacheGroup;
        return table[min(key >> a.block_shift, (int64_t)a.max_blocks - 1)];
    };
    int block_ahead = blocks_from(kt);
    const Span sp = span_of(a, b);

    // row r is query r / G, head hk * G + r % G
    const int row0 = rb * 16 * NR;
    const int t0 = row0 / G, t1 = min((min(row0 + 16 * NR, rows) - 1) / G, sp.n - 1);
    const int reach = t0 <= t1 ? max(sp.first + t1 + 1, 0) : 0;    // keys the last row sees
    const int all_see = t0 <= t1 ? max(sp.first + t0 + 1, 0) : 0;  // keys every row sees
    const int k1 = min(k0 + a.chunk, reach);
    // the joining launch reads the chunks that a row reaches into
    if (a.chunks > 1 && k0 >= reach) return;

    // A batch: the lane's block (-1: no such tokens) and its scales, and the next batch's blocks.  Waited
    // for here, so that no later load of the loop is.
    int lane_block, located = 0, batch_kt = kt;
    float lane_ks, lane_vs;
    auto next_batch = [&]() {
        const int64_t key = batch_kt + (int64_t)(lane / kGroups) * step + lane % kGroups * kCacheGroup;
        lane_block = key < k1 && (unsigned)block_ahead < (unsigned)a.n_blocks ? block_ahead : -1;
        const int64_t page = (int64_t)max(lane_block, 0) * a.Hkv + hk;
        lane_ks = a.k_scale[page];
        lane_vs = a.v_scale[page];
        const int64_t next = batch_kt + (int64_t)kBatch * step;
        batch_kt = next < k1 ? (int)next : k1;
        block_ahead = blocks_from(batch_kt);
        asm volatile("" ::"v"(lane_ks), "v"(lane_vs), "v"(block_ahead));
    };
    // Where a tile lies (what is not there is read from the first page: no load depends on a branch).
    auto locate = [&](int kt, TileAt<kGroups> &at) {
        if (located == kBatch) {
            next_batch();
            located = 0;
        }
#pragma unroll
        for (int u = 0; u < kGroups; ++u) {
            const int from = located * kGroups + u, block = __builtin_amdgcn_readlane(lane_block, from);
            at.there[u] = block >= 0;
            at.base[u] = (((int64_t)max(block, 0) * a.Hkv + hk) * size + ((kt + u * kCacheGroup) & (size - 1))) * DP;
            at.ks[u] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(lane_ks), from));
            at.vs[u] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(lane_vs), from));
        }
        ++located;
    };
    auto fetch = [&](const uint8_t *cache, const TileAt<kGroups> &at, uint4 (*to)[kH]) {
#pragma unroll
        for (int u = 0; u < kGroups; ++u)
#pragma unroll
            for (int h = 0; h < kH; ++h) to[u][h] = load16(cache + at.base[u], h * 1024 + lane * 16);
    };
    bf16x8_t qf[NR][2 * kH][kQ];
    int lim[NR];
    int64_t row_at[NR];  // element offset of the row in q and out; < 0: no such row
    bool padding[NR];    // a row past new_len: written as zero
#pragma unroll
    for (int nr = 0; nr < NR; ++nr) {
        const int r = row0 + nr * 16 + j;
        const int t = r / G, head = hk * G + (r - t * G);
        const bool here = r < rows;
        row_at[nr] = here ? (((int64_t)b * a.Hq + head) * a.T + t) * a.dh : -1;
        padding[nr] = t >= sp.n;
        lim[nr] = here && !padding[nr] ? max(sp.first + t + 1, 0) : reach;
        const T *src = static_cast<const T *>(a.q) + (here ? row_at[nr] : 0);
#pragma unroll
        for (int c = 0; c < 2 * kH; ++c) {
            const int d = (c >> 1) * 64 + g * 16 + (c & 1) * 8;
            const bool ok = here && d < a.dh;
            if constexpr (kQ == 1) {
                union {
                    uint4 u;
                    bf16x8_t v;
                } raw;
                raw.u = load16_guard(src, (int64_t)d * 2, ok);
                qf[nr][c][0] = raw.v;
            } else {
                float f[8];
                unpack16<float>(load16_guard(src, (int64_t)d * 4, ok), f);
                unpack16<float>(load16_guard(src, (int64_t)d * 4 + 16, ok), f + 4);
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    bf16x2_t p[kQ];
                    split<Operand<float>, kQ>(f32x2_t{f[e], f[e + 1]}, p);
#pragma unroll
                    for (int q = 0; q < kQ; ++q) {
                        qf[nr][c][q][e] = p[q][0];
                        qf[nr][c][q][e + 1] = p[q][1];
                    }
                }
            }
        }
    }

    TileAt<kGroups> ats[kStages];
    uint4 kbs[kStages][kGroups][kH], vbs[kStages][kGroups][kH];
    if (kt < k1) {
        next_batch();
#pragma unroll
        for (int i = 0; i < kStages; ++i) {
            locate(kt + i * step, ats[i]);
            fetch(a.k_cache, ats[i], kbs[i]);
            fetch(a.v_cache, ats[i], vbs[i]);
        }
    }
    // (the queries are waited for here, not in the loop)
#pragma unroll
    for (int nr = 0; nr < NR; ++nr)
#pragma unroll
        for (int c = 0; c < 2 * kH; ++c)
#pragma unroll
            for (int q = 0; q < kQ; ++q) asm volatile("" ::"v"(qf[nr][c][q]));

    f32x4_t acc[NR][kD];
    float m[NR], l[NR];
    int eref = kScaleExpMin;  // acc holds sums in units of 2^eref
#pragma unroll
    for (int nr = 0; nr < NR; ++nr) {
        m[nr] = kNothing;
        l[nr] = 0.f;
#pragma unroll
        for (int d = 0; d < kD; ++d) acc[nr][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }

    // A tile; kMask: some of its tokens are not there or not seen by every row.
    auto tile = [&](auto masked, const TileAt<kGroups> &at, uint4 (*kb)[kH], uint4 (*vb)[kH], const TileAt<kGroups> &next) {
        constexpr bool kMask = decltype(masked)::value;
        f32x4_t s[NR][kGroups];
#pragma unroll
        for (int u = 0; u < kGroups; ++u) {
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) s[nr][u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < 2 * kH; ++c) {
                const bf16x8_t ka = from_fp8<Operand<float>>(word(kb[u][c >> 1], 2 * (c & 1)), word(kb[u][c >> 1], 2 * (c & 1) + 1), 1.f, 1.f);
#pragma unroll
                for (int q = kQ - 1; q >= 0; --q)
#pragma unroll
                    for (int nr = 0; nr < NR; ++nr)
                        s[nr][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qf[nr][c][q], s[nr][u], 0, 0, 0);
            }
        }
        fetch(a.k_cache, next, kb);

        // V's scale relative to 2^eref: as a factor of the values, and of the weights as an exponent in
        // their logits, which the sums are freed of again
        float c[kGroups], va[kGroups], we[kGroups], wi[kGroups];
        int top_e = kScaleExpMin;
#pragma unroll
        for (int u = 0; u < kGroups; ++u) {
            c[u] = at.ks[u] * a.scale;
            if (!kMask || at.there[u]) top_e = max(top_e, exp_of(at.vs[u]));
        }
        const int now_e = max(eref, top_e);
#pragma unroll
        for (int u = 0; u < kGroups; ++u) {
            const int e = exp_of(at.vs[u]) - now_e, w = kP == 1 ? max(min(e - kValueExp, 0), kWeightExp) : 0;
            va[u] = pow2(e - w);
            we[u] = (float)w;
            wi[u] = pow2(-w);
        }

        float x[NR][kGroups * 4];
        auto logits = [&](int nr, float ref) {
            float top = -INFINITY;
#pragma unroll
            for (int u = 0; u < kGroups; ++u) {
                const float add = we[u] - ref;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float v = fmaf(s[nr][u][r], c[u], add);
                    if constexpr (kMask) v = at.there[u] && kt + u * kCacheGroup + 4 * g + r < lim[nr] ? v : -INFINITY;
                    x[nr][4 * u + r] = v;
                    top = fmaxf(top, v);
                }
            }
            return top;
        };
        float highest = -INFINITY;
#pragma unroll
        for (int nr = 0; nr < NR; ++nr) highest = fmaxf(highest, logits(nr, m[nr]));
        if (top_e > eref || __any(highest > kRaise)) {
            const float unit = pow2(eref - now_e);
            eref = now_e;
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) {
                float top = logits(nr, 0.f);
                top = fmaxf(top, __shfl_xor(top, 16, kWave));
                top = fmaxf(top, __shfl_xor(top, 32, kWave));
                const float now = fmaxf(m[nr], top - kBias);
                const float f = __builtin_amdgcn_exp2f(m[nr] - now);
                m[nr] = now;
                l[nr] *= f;
#pragma unroll
                for (int d = 0; d < kD; ++d) acc[nr][d] *= f * unit;
                logits(nr, now);
            }
        }
        if constexpr (kMask) {
            // what lies behind the last token is not read as a value
#pragma unroll
            for (int u = 0; u < kGroups; ++u) {
                const int left = sp.len - (kt + u * kCacheGroup + 4 * g);
                const uint32_t keep = left <= 0 || !at.there[u] ? 0u : left >= 4 ? ~0u : (1u << (8 * left)) - 1u;
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
        for (int v = 0; v < kGroups / 2; ++v) {
            typename O::vec pb[NR][kP];
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float *w = x[nr] + 4 * (2 * v + i);
                    float sum = 0.f;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        w[r] = __builtin_amdgcn_exp2f(w[r]);
                        sum += w[r];
                    }
                    l[nr] = fmaf(sum, wi[2 * v + i], l[nr]);
#pragma unroll
                    for (int r = 0; r < 4; r += 2) {
                        typename O::pair p[kP];
                        split<O, kP>(f32x2_t{w[r], w[r + 1]}, p);
#pragma unroll
                        for (int q = 0; q < kP; ++q) {
                            pb[nr][q][4 * i + r] = p[q][0];
                            pb[nr][q][4 * i + r + 1] = p[q][1];
                        }
                    }
                }
            }
#pragma unroll
            for (int d = 0; d < kD; ++d) {
                const typename O::vec vv = from_fp8<O>(word(vb[2 * v][d >> 2], d & 3), word(vb[2 * v + 1][d >> 2], d & 3),
                                                       va[2 * v], va[2 * v + 1]);
#pragma unroll
                for (int q = kP - 1; q >= 0; --q)
#pragma unroll
                    for (int nr = 0; nr < NR; ++nr) acc[nr][d] = O::mfma(vv, pb[nr][q], acc[nr][d]);
            }
        }
        fetch(a.v_cache, next, vb);
    };

    // The tile of a stage, after which the stage takes the tile kStages steps on.
    auto advance = [&](auto masked, int stage) {
        TileAt<kGroups> next;
        locate(kt + kStages * step, next);
        tile(masked, ats[stage], kbs[stage], vbs[stage], next);
        ats[stage] = next;
        kt += step;
    };
    // tiles that every row sees whole, as far as all their blocks are there; then the others
    while (kt + (kStages - 1) * step + kTile <= min(k1, all_see)) {
        bool whole = true;
#pragma unroll
        for (int i = 0; i < kStages; ++i)
#pragma unroll
            for (int u = 0; u < kGroups; ++u) whole = whole && ats[i].there[u];
        if (!whole) break;
#pragma unroll
        for (int i = 0; i < kStages; ++i) advance(std::false_type(), i);
    }
    while (kt < k1) {
#pragma unroll
        for (int i = 0; i < kStages; ++i)
            if (kt < k1) advance(std::true_type(), i);
    }

#pragma unroll
    for (int nr = 0; nr < NR; ++nr) {
        l[nr] += __shfl_xor(l[nr], 16, kWave);
        l[nr] += __shfl_xor(l[nr], 32, kWave);
    }

    // the waves' results, 16 rows at a time: [wave][d][lane], per wave and row (reference, sum), per wave eref
    float *stat = reinterpret_cast<float *>(lds4 + kWaves * kD * kWave);
    int *refs = reinterpret_cast<int *>(stat + kWaves * 16 * 2);
    if (lane == 0) refs[wave] = eref;
    T *out = static_cast<T *>(a.out);
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
        float mx = kNothing, sum = 0.f, f[kWaves];
        int e = kScaleExpMin;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            mx = fmaxf(mx, stat[(w * 16 + j) * 2]);
            e = max(e, refs[w]);
        }
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            f[w] = __builtin_amdgcn_exp2f(stat[(w * 16 + j) * 2] - mx);
            sum += f[w] * stat[(w * 16 + j) * 2 + 1];
        }
        // a row without keys, or past new_len, is zero
        const float inv = sum > 0.f && !padding[nr] ? 1.f / sum : 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) f[w] *= inv * pow2(refs[w] - e);
        const float unit = pow2(e);
#pragma unroll
        for (int d = wave; d < kD; d += kWaves) {
            const int dim = 16 * d + 4 * g;
            f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float4 y = lds4[(w * kD + d) * kWave + lane];
                o[0] += f[w] * y.x;
                o[1] += f[w] * y.y;
                o[2] += f[w] * y.z;
                o[3] += f[w] * y.w;
            }
            o *= unit;
            if (row_at[nr] < 0) continue;
            if (a.chunks == 1) {
                if (dim < a.dh) store4<T>(out + row_at[nr] + dim, o);
                continue;
            }
            // the chunk's result, with its reference and sum, for the joining launch
            const int64_t part = (((int64_t)b * a.Hkv + hk) * rows + row0 + nr * 16 + j) * a.chunks + chunk;
            store4<float>(a.part_acc + part * DP + dim, o);
            if (d == 0 && g == 0) {
                a.part_stat[2 * part] = mx;
                a.part_stat[2 * part + 1] = sum;
            }
        }
    }
}

// Joins the chunks of a row, each of which is an average with its sum of weights.  A wave per row, so
// many lanes per chunk that they hold its dims four at a time; bound by latency, so the averages are
// requested before it is known what they weigh.
constexpr int kCombineThreads = 256, kAhead = 4;
template <typename T, int DP>
__global__ __launch_bounds__(kCombineThreads) void combine_kernel(AttendArgs a) {
    constexpr int kLanes = DP / 4, kSets = kWave / kLanes;  // lanes of a chunk, chunks at a time
    const int G = a.Hq / a.Hkv, rows = G * a.T, lane = lane_id();
    const int64_t row = (int64_t)blockIdx.x * (kCombineThreads / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (row >= (int64_t)a.B * a.Hkv * rows) return;
    const int set = min(lane / kLanes, kSets - 1), dim = lane % kLanes * 4;
    const float *stat = a.part_stat + row * a.chunks * 2, *part = a.part_acc + row * a.chunks * DP + dim;
    const int r = (int)(row % rows), t = r / G;
    const int64_t bh = row / rows;
    const int hk = (int)(bh % a.Hkv), b = (int)(bh / a.Hkv);
    const Span sp = span_of(a, b);
    const int lim = t < sp.n ? max(sp.first + t + 1, 0) : 0;
    const int n = (int)(((int64_t)lim + a.chunk - 1) / a.chunk);
    float mx = kNothing, sum = 0.f;
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
    for (int c0 = 0; c0 < n; c0 += kAhead * kSets) {
        float4 x[kAhead];
        float m[kAhead], l[kAhead], top = kNothing;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int c = c0 + i * kSets + set, at = min(c, n - 1);
            x[i] = *reinterpret_cast<const float4 *>(part + (int64_t)at * DP);
            m[i] = c < n ? stat[2 * at] : kNothing;
            l[i] = c < n ? stat[2 * at + 1] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) top = fmaxf(top, m[i]);
        const float now = fmaxf(mx, top), keep = __builtin_amdgcn_exp2f(mx - now);
        mx = now;
        sum *= keep;
        o *= keep;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const float f = __builtin_amdgcn_exp2f(m[i] - now) * l[i];
            sum += f;
            o[0] += f * x[i].x;
            o[1] += f * x[i].y;
            o[2] += f * x[i].z;
            o[3] += f * x[i].w;
        }
    }
#pragma unroll
    for (int d = kLanes; d < kLanes * kSets; d *= 2) {
        const float other = __shfl_xor(mx, d, kWave), now = fmaxf(mx, other);
        const float f = __builtin_amdgcn_exp2f(mx - now), fo = __builtin_amdgcn_exp2f(other - now);
        mx = now;
        sum = sum * f + __shfl_xor(sum, d, kWave) * fo;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = o[e] * f + __shfl_xor(o[e], d, kWave) * fo;
    }
    if (lane >= kLanes || dim >= a.dh) return;
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    const int64_t at = (((int64_t)b * a.Hq + hk * G + (r - t * G)) * a.T + t) * a.dh + dim;
    store4<T>(static_cast<T *>(a.out) + at, o * inv);
}

template <typename T, int DP, int NR>
hipError_t launch_as(const AttendArgs &a, hipStream_t s) {
    constexpr int kTile = attend_tile(NR);
    const dim3 grid((unsigned)((int64_t)a.B * a.Hkv * a.row_blocks * a.chunks));
    constexpr size_t lds = kWaves * (DP / 16) * kWave * 16 + kWaves * 16 * 2 * sizeof(float) + kWaves * sizeof(int);
    if constexpr (lds > 65536) {
        static std::atomic<uint64_t> done{0};
        const hipError_t e = allow_large_lds(attend_kernel<T, DP, NR, kTile>, done);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((attend_kernel<T, DP, NR, kTile>), grid, dim3(kWaves * kWave), lds, s, a);
    return hipGetLastError();
}

template <typename T, int DP>
hipError_t launch_dp(const AttendArgs &a, hipStream_t s) {
    if constexpr (sizeof(T) == 2 || DP <= 128)
        if (a.row_tiles == 2) return launch_as<T, DP, 2>(a, s);
    return launch_as<T, DP, 1>(a, s);
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

template <typename T>
hipError_t launch_combine(const AttendArgs &a, hipStream_t s) {
    constexpr int kRows = kCombineThreads / kWave;
    const dim3 grid((unsigned)(((int64_t)a.B * a.Hq * a.T + kRows - 1) / kRows));
    switch (cache_dp(a.dh)) {
        case 64: hipLaunchKernelGGL((combine_kernel<T, 64>), grid, dim3(kCombineThreads), 0, s, a); break;
        case 128: hipLaunchKernelGGL((combine_kernel<T, 128>), grid, dim3(kCombineThreads), 0, s, a); break;
        case 192: hipLaunchKernelGGL((combine_kernel<T, 192>), grid, dim3(kCombineThreads), 0, s, a); break;
        default: hipLaunchKernelGGL((combine_kernel<T, 256>), grid, dim3(kCombineThreads), 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace

namespace vscan {

hipError_t launch_cache_attend(const void *args, hipStream_t s) {
    const AttendArgs &a = *static_cast<const AttendArgs *>(args);
    return a.is_bf16 ? launch_t<bf16_t>(a, s) : launch_t<float>(a, s);
}

hipError_t launch_cache_combine(const void *args, hipStream_t s) {
    const AttendArgs &a = *static_cast<const AttendArgs *>(args);
    return a.is_bf16 ? launch_combine<bf16_t>(a, s) : launch_combine<float>(a, s);
}

}  // namespace vscan
