// Attention of a few or many queries over the paged 8-bit cache.
//
// Rows are the (query, query head) pairs of one kv head.  S^T = K Q^T and O^T = V^T P^T: the
// accumulators of the first product hold a row's weights in the lanes and order in which the second
// takes them, so they never leave the registers.  The cache is stored in operand order: a lane's 16
// bytes are one load, and nothing is staged in LDS.
//
// bf16 calls: K (as bf16, exact) times q; V as fp16 (exact) times the weights as two fp16 planes, whose sum is a
// weight to 2^-22.  (With one, 2^-11 of each weight, a sum of many keys is off by a tenth of the result's own
// rounding, and 7 % of the results are another bf16 number.  That takes 180 us where two planes take 232, 512 rows of 8
// sequences over 4096 keys; 46 and 56, 3 x 300 over 2604; 126 and 128, one of 32 sequences, bound by memory.)  fp32
// calls: q and the weights as three bf16 planes each, V as bf16.  (The 8-bit instructions would take K as it is
// stored, with q in two planes, 6 % faster.  But they drop what lies 2^-11 to 2^-14 below the largest product of a
// sum, where those of bf16 keep 2^-21: logits with one large product were off by 1e-2.)  K's scale goes into the
// logits; V's, a power of two, is taken relative to the largest that the wave has met: down to 2^-15 with the values,
// beyond that with the weights, whose reference it then enters, so that the largest contributions keep their bits.
// Softmax in one pass against a reference that is raised only where a lane's weights of a tile add up to more
// than 2^12, so that most tiles need no exchange between lanes and no maximum.
//
// Two forms, by rows (`attend_form`): up to 16, with 16x16x32 instructions and 64 keys at a time (bound by HBM: 2 dh
// bytes per token and kv head); more, 32 to a wave, with 32x32x16 instructions and 32 keys at a time, two tiles in
// flight (bound by the vector unit beside the matrix pipe: per logit a multiply-add, an exponential and a sum, and
// K's, V's and the weights' conversions; a matrix instruction keeps the vector unit from issuing for some cycles
// whatever its size, so the large ones overlap better: 96 multiply-adds and 16 exponentials with 514 cycles of them
// 667, with 16x16x32 861).
// The four waves of a workgroup take the tiles of its keys in turn and add their results in LDS; where
// sequences and rows leave compute units idle the keys are cut into chunks over workgroups, which a
// second launch joins.
//
// Measured, bf16, dh = 128, GPU time of calls on one set of inputs: one token of 32 sequences with 32 heads, up to
// 3427 keys, 127 us (5.4 TB/s from memory); of 4 sequences with 28 heads of 4, up to 65536 keys, 45 us (53 on five sets
// in turn); of one with 2304 keys 10.4 us, two launches' latency.  512 tokens of 8 sequences, 28 heads of 4, over 4096
// keys 230 us (589 TFLOP/s of the two products), over 8192 440 us (624), over 16384 854 us (648); 4 x 700 over 3000, 32
// heads, 145 us (505); 3 x 300 over 2604, 28 of 4, 56 us (343: 396 workgroups on 256 CUs).  With one plane of the
// weights a maximum of every tile took 4 us more in the first of these prompts, and more rows a wave (64: 280 us where
// 32 took 179), eight waves (245) and rows over all four waves (203) lost to this split.
#include <hip/hip_runtime.h>
#include <float.h>
#include <limits.h>
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
constexpr float kNothing = -FLT_MAX;  // reference of a row that has seen no key: below every finite logit
constexpr float kBias = 4.f;        // the largest weight is 2^4 when the reference is set ..
constexpr float kRaise = 4096.f;    // .. and a lane's sum of a tile at most this until it is raised (fp16 holds 2^16)
constexpr float kMostExp = 12.f;    // log2(kRaise)
constexpr int kValueExp = -15;      // e4m3's 2^-9 times 2^-15 is fp16's smallest number
constexpr int kWeightExp = -100;    // sums of weights without this factor stay inside fp32

template <typename T>
struct Operand;  // what V and the weights are multiplied as
template <>
struct Operand<bf16_t> {
    typedef f16x8_t vec;
    typedef f16x2_t pair;
    static constexpr int kPlanes = 2, kQueryPlanes = 1;
    static __device__ __forceinline__ pair from_fp8(uint32_t w, float s, bool hi) {
        return hi ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, s, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, s, false);
    }
    static __device__ __forceinline__ f32x4_t mfma(vec a, vec b, f32x4_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16_t mfma32(vec a, vec b, f32x16_t c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
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
    static __device__ __forceinline__ f32x16_t mfma32(vec a, vec b, f32x16_t c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
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
            x[0] = fmaf((float)out[p][0], -1.f, x[0]);  // (one instruction, from a half)
            x[1] = fmaf((float)out[p][1], -1.f, x[1]);
        }
    }
}

// Exponent of a power of two.
__device__ __forceinline__ int exp_of(float s) {
    const int e = (int)(__float_as_uint(s) >> 23 & 255u) - 127;
    return min(max(e, kScaleExpMin), kScaleExpMax);
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(min(max(e, -126), 127) + 127) << 23); }

// References of large logits.  A reference is a rounded number, exponents are taken from exact products: from 2^25 on,
// where numbers are 4 apart, the largest exponent may be other than kBias by as much, and by more than fp16 holds from
// 2^28 on.  So a reference above its row's largest logit (`rest`: the largest exponent) goes down a step, and exponents
// against a reference that has just been set are cut to kMostExp: keys within a step of the largest logit, which fp32
// does not tell apart, then weigh the same.  (NaN stays NaN.)
constexpr float kCoarse = 0x1p25f;
__device__ __forceinline__ bool is_coarse(float now) { return fabsf(now) >= kCoarse && fabsf(now) < FLT_MAX; }  // (kNothing is not)
__device__ __forceinline__ float lower_reference(float m, float now, float rest) {
    if (!is_coarse(now) || !(rest < 0.f)) return now;
    const int bits = __float_as_int(now);
    return fmaxf(m, __int_as_float(now > 0.f ? bits - 1 : bits + 1));
}
template <bool kMost>
__device__ __forceinline__ float at_most(float x) { return kMost && x > kMostExp ? kMostExp : x; }

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

// What a workgroup works on: rows of a kv head, and a chunk of its sequence's keys.
struct Work {
    int chunk, hk, b, G, rows, row0;
    int k0, k1;          // keys of the chunk that the last row sees
    int all_see, reach;  // keys that every row sees, and the last one
    int block_reach;     // .. and the last row of the workgroup
    Span sp;
};
template <int kRows, int kRowWaves>
__device__ __forceinline__ Work work_of(const AttendArgs &a, int row_wave) {
    Work w;
    int id = blockIdx.x;
    w.chunk = id % a.chunks;
    id /= a.chunks;
    const int block0 = id % a.row_blocks * (kRows * kRowWaves);
    id /= a.row_blocks;
    w.hk = id % a.Hkv;
    w.b = id / a.Hkv;
    w.G = a.Hq / a.Hkv;
    w.rows = w.G * a.T;
    w.sp = span_of(a, w.b);
    // row r is query r / G, head hk * G + r % G
    w.row0 = block0 + row_wave * kRows;
    auto sees = [&](int r) {
        const int t = min((min(r, w.rows) - 1) / w.G, w.sp.n - 1);  // the last query before row r
        return max(w.sp.first + t + 1, 0);
    };
    const int t0 = w.row0 / w.G;
    const bool any = w.row0 < w.rows && t0 < w.sp.n;
    w.reach = any ? sees(w.row0 + kRows) : 0;
    w.all_see = any ? max(w.sp.first + t0 + 1, 0) : 0;
    w.block_reach = kRowWaves == 1 ? w.reach : block0 / w.G < w.sp.n ? sees(block0 + kRows * kRowWaves) : 0;
    w.k0 = w.chunk * a.chunk;
    w.k1 = min(w.k0 + a.chunk, w.reach);
    return w;
}

// A row of a lane.
struct Row {
    int64_t at;    // element offset in q and out; < 0: no such row
    int lim;       // keys it sees
    bool padding;  // past new_len: written as zero
};
__device__ __forceinline__ Row row_of(const AttendArgs &a, const Work &w, int r) {
    Row x;
    const int t = r / w.G, head = w.hk * w.G + (r - t * w.G);
    const bool here = r < w.rows;
    x.at = here ? (((int64_t)w.b * a.Hq + head) * a.T + t) * a.dh : -1;
    x.padding = t >= w.sp.n;
    x.lim = here && !x.padding ? max(w.sp.first + t + 1, 0) : w.reach;
    return x;
}

// Queries at the top of the range.  K goes into the products without its scale, so up to 256 products of 448 and an
// entry of kFar stay inside fp32; where an entry of a wave's rows is larger, they are all taken by 2^-24, which
// the factor of the logits makes up for (c above 2^127 then: infinite logits, and NaN).
constexpr float kFar = 0x1p104f, kNear = 1.f / kFarScale;
// Eight entries of a query.
template <typename T>
struct QueryPiece {
    uint4 raw[sizeof(T) / 2];
    __device__ __forceinline__ void load(const AttendArgs &a, const Row &row, int d) {
        const bool ok = row.at >= 0 && !row.padding && d < a.dh;
        const T *src = static_cast<const T *>(a.q) + max(row.at, (int64_t)0);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) raw[i] = load16_guard(src, (int64_t)d * (int)sizeof(T) + 16 * i, ok);
    }
    __device__ __forceinline__ void get(float *f) const {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) unpack16<T>(raw[i], f + i * ElemTraits<T>::kPer16B);
    }
    __device__ __forceinline__ float largest() const {
        float f[8], top = 0.f;
        get(f);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(f[e]));
        return top;
    }
    __device__ __forceinline__ void come_near() {
        float f[8];
        get(f);
        if constexpr (sizeof(T) == 2) {
            union {
                __bf16 h[8];
                uint4 u;
            } o;
#pragma unroll
            for (int e = 0; e < 8; ++e) o.h[e] = (__bf16)(f[e] * kNear);
            raw[0] = o.u;
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                raw[i] = make_uint4(__float_as_uint(f[4 * i] * kNear), __float_as_uint(f[4 * i + 1] * kNear),
                                    __float_as_uint(f[4 * i + 2] * kNear), __float_as_uint(f[4 * i + 3] * kNear));
        }
    }
    // as planes of bf16
    __device__ __forceinline__ void planes(bf16x8_t *out) const;
};
template <typename T>
__device__ __forceinline__ void QueryPiece<T>::planes(bf16x8_t *out) const {
    if constexpr (sizeof(T) == 2) {
        out[0] = __builtin_bit_cast(bf16x8_t, raw[0]);
    } else {
        float f[8];
        get(f);
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            bf16x2_t p[3];
            split<Operand<float>, 3>(f32x2_t{f[e], f[e + 1]}, p);
#pragma unroll
            for (int q = 0; q < 3; ++q) {
                out[q][e] = p[q][0];
                out[q][e + 1] = p[q][1];
            }
        }
    }
}
// Whether one of the wave's rows is too large as it is; if so they are all scaled.
template <typename T, int kN>
__device__ __forceinline__ bool come_near(QueryPiece<T> (&q)[kN]) {
    float top = 0.f;
#pragma unroll
    for (int c = 0; c < kN; ++c) top = fmaxf(top, q[c].largest());
    const bool far = __builtin_amdgcn_readfirstlane(__any(top >= kFar && top < INFINITY));
    if (__builtin_expect(far, 0)) {
#pragma unroll
        for (int c = 0; c < kN; ++c) q[c].come_near();
    }
    return far;
}

// The keys of a tile: where its groups of 16 lie, and their scales.
template <int kGroups>
struct TileAt {
    int64_t base[kGroups];  // bytes from the start of k_cache / v_cache
    float c[kGroups];       // factor of its logits
    int e[kGroups];         // exponent of V's scale
    bool there[kGroups];
};

// The tiles of a wave: `step` keys apart.  Block numbers and scales of its next 64 groups of 16 tokens
// are kept a group to a lane, so that a tile's come without a load.
template <int kGroups, int DP>
struct Walk {
    static constexpr int kBatch = kWave / kGroups;  // tiles
    const AttendArgs &a;
    const int32_t *table;
    int hk, step, k1, batch_kt, located = 0, block_ahead, lane_block, lane_e;
    float lane_c;
    bool far = false;  // queries are scaled by kNear

    __device__ __forceinline__ Walk(const AttendArgs &args, int b, int hk_, int step_, int kt)
        : a(args), table(args.block_table + (int64_t)b * args.max_blocks), hk(hk_), step(step_), batch_kt(kt) {
        block_ahead = blocks_from();  // ahead of knowing whether the tokens are there
    }
    __device__ __forceinline__ int64_t lane_key() const {
        return batch_kt + (int64_t)(lane_id() / kGroups) * step + lane_id() % kGroups * kCacheGroup;
    }
    __device__ __forceinline__ int blocks_from() const {
        return table[min(lane_key() >> a.block_shift, (int64_t)a.max_blocks - 1)];
    }
    // A batch: the lane's block (-1: no such tokens) and its scales, and the next batch's blocks.
    __device__ __forceinline__ void next_batch() {
        lane_block = lane_key() < k1 && (unsigned)block_ahead < (unsigned)a.n_blocks ? block_ahead : -1;
        const int64_t page = (int64_t)max(lane_block, 0) * a.Hkv + hk;
        lane_c = a.k_scale[page];
        lane_e = __float_as_int(a.v_scale[page]);
        const int64_t next = batch_kt + (int64_t)kBatch * step;
        batch_kt = next < k1 ? (int)next : k1;
        block_ahead = blocks_from();
        located = 0;
    }
    // (waited for at once, so that no later load of the loop is)
    __device__ __forceinline__ void settle() {
        lane_c *= far ? a.far_scale : a.scale;
        lane_e = lane_block >= 0 ? exp_of(__int_as_float(lane_e)) : kScaleExpMin;
        asm volatile("" ::"v"(block_ahead));
    }
    // Where the tile at key kt lies, from the table.
    __device__ __forceinline__ void look_up(int kt, TileAt<kGroups> &at) const {
        const int size = 1 << a.block_shift;
#pragma unroll
        for (int u = 0; u < kGroups; ++u) {
            const int key = kt + u * kCacheGroup, block = key < k1 ? table[key >> a.block_shift] : -1;
            at.there[u] = (unsigned)block < (unsigned)a.n_blocks;
            at.base[u] = (((int64_t)(at.there[u] ? block : 0) * a.Hkv + hk) * size + (key & (size - 1))) * DP;
        }
    }
    // Where the next tile lies, at key kt (what is not there is read from the first page: no load depends
    // on a branch).
    __device__ __forceinline__ void locate(int kt, TileAt<kGroups> &at) {
        if (located == kBatch) {
            next_batch();
            settle();
        }
        const int size = 1 << a.block_shift;
#pragma unroll
        for (int u = 0; u < kGroups; ++u) {
            const int block = __builtin_amdgcn_readlane(lane_block, located * kGroups + u);
            at.there[u] = block >= 0;
            at.base[u] = (((int64_t)max(block, 0) * a.Hkv + hk) * size + ((kt + u * kCacheGroup) & (size - 1))) * DP;
        }
        scales_of(located, at);
        ++located;
    }
    __device__ __forceinline__ void scales_of(int tile, TileAt<kGroups> &at) const {
#pragma unroll
        for (int u = 0; u < kGroups; ++u) {
            at.c[u] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(lane_c), tile * kGroups + u));
            at.e[u] = __builtin_amdgcn_readlane(lane_e, tile * kGroups + u);
        }
    }
    // The first kStages tiles: their keys and values are requested before their scales, and what `far` looks
    // at, the queries, have come.
    template <int kStages, typename Fetch, typename Far>
    __device__ __forceinline__ void begin(int kt, int end, TileAt<kGroups> *ats, Fetch fetch, Far is_far) {
        k1 = end;
        next_batch();
#pragma unroll
        for (int i = 0; i < kStages; ++i) {
            locate(kt + i * step, ats[i]);
            fetch(i);
        }
        far = is_far();
        settle();
#pragma unroll
        for (int i = 0; i < kStages; ++i) scales_of(i, ats[i]);
    }
};

// V's scales relative to 2^eref: as a factor of the values, and of the weights as an exponent in their
// logits, which the sums are freed of again.
template <int kGroups, bool kSplitScale>
struct Scales {
    float values[kGroups], weights[kGroups], sums[kGroups];
    int now;  // eref with this tile's scales
    __device__ __forceinline__ void of(const TileAt<kGroups> &at, int eref) {
        now = eref;
#pragma unroll
        for (int u = 0; u < kGroups; ++u) now = max(now, at.e[u]);
#pragma unroll
        for (int u = 0; u < kGroups; ++u) {
            const int e = at.e[u] - now, w = kSplitScale ? max(min(e - kValueExp, 0), kWeightExp) : 0;
            values[u] = pow2(e - w);
            weights[u] = (float)w;
            sums[u] = pow2(-w);
        }
    }
};

// Walks over the wave's tiles: whole ones, which every row sees and whose blocks are all there, without
// masks, as far as they come first; then the others.
template <int kTile, int kStages, typename At, typename Tile>
__device__ __forceinline__ void walk_tiles(int kt, int step, const Work &w, const At *ats, Tile tile) {
    constexpr int kGroups = kTile / kCacheGroup;
    while (kt + (kStages - 1) * step + kTile <= min(w.k1, w.all_see)) {
        bool whole = true;
#pragma unroll
        for (int i = 0; i < kStages; ++i)
#pragma unroll
            for (int u = 0; u < kGroups; ++u) whole = whole && ats[i].there[u];
        if (!whole) break;
#pragma unroll
        for (int i = 0; i < kStages; ++i, kt += step) tile(std::false_type(), i, kt);
    }
    while (kt < w.k1) {
#pragma unroll
        for (int i = 0; i < kStages; ++i)
            if (kt < w.k1) {
                tile(std::true_type(), i, kt);
                kt += step;
            }
    }
}

// Bytes of four tokens of V that are there: those from `left` on lie behind the last one, or not there.
__device__ __forceinline__ uint32_t value_mask(int left, bool there) {
    return left <= 0 || !there ? 0u : left >= 4 ? ~0u : (1u << (8 * left)) - 1u;
}

// NaN bytes of four e4m3 values: as 0xff.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
    const uint32_t top = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
    return (top >> 7) * 255u;
}
__device__ __forceinline__ uint32_t take_nan(uint32_t &w) {
    const uint32_t n = nan_bytes(w);
    w &= ~n;
    return n;
}
// A weight of 0 does not keep a NaN out of a sum.  So the masked tiles, where some rows do not see a key,
// leave NaN out, and a wave that has met any goes over those tiles once more at its end: ones where a value is
// NaN times ones where a row sees its key count what makes a sum NaN.
template <typename O>
__device__ __forceinline__ typename O::vec ones_at(uint32_t lo, uint32_t hi) {
    return from_fp8<O>(nan_bytes(lo) & 0x38383838u, nan_bytes(hi) & 0x38383838u, 1.f, 1.f);  // 0x38: 1.0
}
// .. of the eight keys lo .. lo + 3 and hi .. hi + 3
template <typename O>
__device__ __forceinline__ typename O::vec seen_keys(int lo, int hi, int lim) {
    typename O::vec r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (e < 4 ? lo + e : hi + e - 4) < lim ? 1.f : 0.f;
    return r;
}

// A sum of 0 is that of a row without keys, unless the row sees some and each logit is minus infinity (an
// infinite query whose products have one sign): softmax has no value there, and the row is NaN.  Such a chunk's
// reference is the number above kNothing; other chunks may still have keys with weight, so the last to join decides.
constexpr float kHollow = -0x1.fffffcp127f;
static_assert(kHollow > kNothing, "");
// Whether a row that sees `lim` keys sees one of the workgroup's chunk.  (Its place is worked out again: kept
// through the loop over the keys it cost heads of 256 2.5 % of their time.)
__device__ __forceinline__ bool sees_any(const AttendArgs &a, int lim) {
    int id = blockIdx.x;
    asm volatile("" : "+s"(id));
    const int32_t *table = a.block_table + (int64_t)(id / a.chunks / a.row_blocks / a.Hkv) * a.max_blocks;
    const int k0 = id % a.chunks * a.chunk, k1 = min(k0 + a.chunk, lim);
    bool any = false;
    for (int key = k0; key < k1 && !any; key += 1 << a.block_shift)
        any = (unsigned)table[key >> a.block_shift] < (unsigned)a.n_blocks;
    return any;
}

// The results of the waves of a workgroup for a lane's row, from (reference, sum) pairs and scale
// references in LDS: factors of their accumulators, and what the row has in all.
template <int kN>
struct Joined {
    float f[kN], mx, sum, unit;
};
template <int kN>
__device__ __forceinline__ Joined<kN> join_waves(const AttendArgs &a, const Row &row, const float *stat, const int *refs,
                                                 int rows, int j) {
    Joined<kN> r;
    int e = kScaleExpMin;
    r.mx = kNothing;
    r.sum = 0.f;
#pragma unroll
    for (int v = 0; v < kN; ++v) {
        r.mx = fmaxf(r.mx, stat[(v * rows + j) * 2]);
        e = max(e, refs[v]);
    }
#pragma unroll
    for (int v = 0; v < kN; ++v) {
        r.f[v] = __builtin_amdgcn_exp2f(stat[(v * rows + j) * 2] - r.mx);
        r.sum += r.f[v] * stat[(v * rows + j) * 2 + 1];
    }
    // a row without keys, or past new_len, is zero
    const float inv = r.sum > 0.f && !row.padding ? 1.f / r.sum : 0.f;
#pragma unroll
    for (int v = 0; v < kN; ++v) r.f[v] *= inv * pow2(refs[v] - e);
    r.unit = pow2(e);
    if (__builtin_expect(__any(r.sum == 0.f), 0) && r.sum == 0.f && sees_any(a, row.lim)) {
        if (a.chunks == 1) r.unit = NAN;
        r.mx = kHollow;
    }
    return r;
}
// Four dims of a row: `at` are the waves' accumulators, `stride` apart.
template <typename T, int DP, int kN>
__device__ __forceinline__ void write_row(const AttendArgs &a, const Work &w, const Row &row, int r, int dim,
                                          const Joined<kN> &jn, const float4 *at, int stride, bool first) {
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < kN; ++v) {
        const float4 y = at[v * stride];
        o[0] += jn.f[v] * y.x;
        o[1] += jn.f[v] * y.y;
        o[2] += jn.f[v] * y.z;
        o[3] += jn.f[v] * y.w;
    }
    o *= jn.unit;
    if (row.padding) o = f32x4_t{0.f, 0.f, 0.f, 0.f};  // (a NaN of a value would stay one under a factor of 0)
    if (row.at < 0) return;
    if (a.chunks == 1) {
        if (dim < a.dh) store4<T>(static_cast<T *>(a.out) + row.at + dim, o);
        return;
    }
    // the chunk's result, with its reference and sum, for the joining launch
    const int64_t part = (((int64_t)w.b * a.Hkv + w.hk) * w.rows + r) * a.chunks + w.chunk;
    store4<float>(a.part_acc + part * DP + dim, o);
    if (first) {
        a.part_stat[2 * part] = jn.mx;
        a.part_stat[2 * part + 1] = jn.sum;
    }
}

// Up to 16 rows.  Lane (j, g) = (lane % 16, lane / 16): row j; of each group of 16 tokens logits of tokens
// 4g .. 4g+3; of O^T dims 16d + 4g .. +3 of its tiles d.
template <typename T, int DP>
__global__ __launch_bounds__(kWaves *kWave, DP <= 128 && sizeof(T) == 2 ? 2 : 1) void attend_few_kernel(AttendArgs a) {
    typedef Operand<T> O;
    constexpr int kTile = attend_tile(1), kGroups = kTile / kCacheGroup;
    constexpr int kH = DP / 64;  // 16-byte loads per lane and group
    constexpr int kD = DP / 16;  // tiles of 16 dims
    constexpr int kQ = O::kQueryPlanes, kP = O::kPlanes, step = kTile * kWaves;
    extern __shared__ float4 lds4[];

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = lane_id(), j = lane & 15, g = lane >> 4;
    const int chunk = blockIdx.x % a.chunks, hk = blockIdx.x / a.chunks / a.row_blocks % a.Hkv;
    const int kt0 = chunk * a.chunk + wave * kTile;
    Walk<kGroups, DP> walk(a, blockIdx.x / a.chunks / a.row_blocks / a.Hkv, hk, step, kt0);
    const Work w = work_of<16, 1>(a, 0);
    // the joining launch reads the chunks that a row reaches into
    if (a.chunks > 1 && w.k0 >= w.reach) return;

    const Row row = row_of(a, w, w.row0 + j);
    QueryPiece<T> queries[2 * kH];
#pragma unroll
    for (int c = 0; c < 2 * kH; ++c) queries[c].load(a, row, (c >> 1) * 64 + g * 16 + (c & 1) * 8);

    auto fetch = [&](const uint8_t *cache, const TileAt<kGroups> &at, uint4 (*to)[kH]) {
#pragma unroll
        for (int u = 0; u < kGroups; ++u)
#pragma unroll
            for (int h = 0; h < kH; ++h) to[u][h] = load16(cache + at.base[u], h * 1024 + lane * 16);
    };
    TileAt<kGroups> at[1];
    uint4 kb[kGroups][kH], vb[kGroups][kH];
    if (kt0 < w.k1) {
        walk.template begin<1>(kt0, w.k1, at, [&](int) {
            fetch(a.k_cache, at[0], kb);
            fetch(a.v_cache, at[0], vb);
        }, [&] { return come_near(queries); });
    }
    bf16x8_t qf[2 * kH][kQ];
#pragma unroll
    for (int c = 0; c < 2 * kH; ++c) queries[c].planes(qf[c]);
    // (the queries are waited for here, not in the loop)
#pragma unroll
    for (int c = 0; c < 2 * kH; ++c)
#pragma unroll
        for (int q = 0; q < kQ; ++q) asm volatile("" ::"v"(qf[c][q]));

    f32x4_t acc[kD];
    float m = kNothing, l = 0.f;
    int eref = kScaleExpMin;  // acc holds sums in units of 2^eref
    int nan_from = INT_MAX;   // the first masked tile with a NaN
#pragma unroll
    for (int d = 0; d < kD; ++d) acc[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    walk_tiles<kTile, 1>(kt0, step, w, at, [&](auto masked, int, int kt) {
        constexpr bool kMask = decltype(masked)::value;
        TileAt<kGroups> next;
        walk.locate(kt + step, next);
        f32x4_t s[kGroups];
#pragma unroll
        for (int u = 0; u < kGroups; ++u) {
            s[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < 2 * kH; ++c) {
                const bf16x8_t ka = from_fp8<Operand<float>>(word(kb[u][c >> 1], 2 * (c & 1)), word(kb[u][c >> 1], 2 * (c & 1) + 1), 1.f, 1.f);
#pragma unroll
                for (int q = kQ - 1; q >= 0; --q) s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qf[c][q], s[u], 0, 0, 0);
            }
        }
        fetch(a.k_cache, next, kb);

        Scales<kGroups, sizeof(T) == 2> sc;
        sc.of(at[0], eref);
        __builtin_amdgcn_sched_barrier(0);  // (the products and the next keys' requests first)
        typename O::vec pb[kGroups / 2][kP];
        float sums[kGroups];
        auto logit = [&](int u, int r, float add) {
            float v = fmaf(s[u][r], at[0].c[u], add);
            if constexpr (kMask) v = at[0].there[u] && kt + u * kCacheGroup + 4 * g + r < row.lim ? v : -INFINITY;
            return v;
        };
        auto weigh = [&](float ref, auto most) {
            constexpr bool kMost = decltype(most)::value;
            float all = 0.f;
#pragma unroll
            for (int u = 0; u < kGroups; ++u) {
                const float add = sc.weights[u] - ref;
                sums[u] = 0.f;
#pragma unroll
                for (int r = 0; r < 4; r += 2) {
                    const float p0 = __builtin_amdgcn_exp2f(at_most<kMost>(logit(u, r, add)));
                    const float p1 = __builtin_amdgcn_exp2f(at_most<kMost>(logit(u, r + 1, add)));
                    typename O::pair pp[kP];
                    split<O, kP>(f32x2_t{p0, p1}, pp);
                    sums[u] += p0;
                    sums[u] += p1;
#pragma unroll
                    for (int q = 0; q < kP; ++q) {
                        pb[u / 2][q][4 * (u & 1) + r] = pp[q][0];
                        pb[u / 2][q][4 * (u & 1) + r + 1] = pp[q][1];
                    }
                }
                all += sums[u];
            }
            return all;
        };
        if (__any(weigh(m, std::false_type()) > kRaise) || sc.now > eref) {
            float top = -INFINITY;
#pragma unroll
            for (int u = 0; u < kGroups; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) top = fmaxf(top, logit(u, r, sc.weights[u]));
            top = fmaxf(top, __shfl_xor(top, 16, kWave));
            top = fmaxf(top, __shfl_xor(top, 32, kWave));
            float now = fmaxf(m, top - kBias);
            if (__builtin_expect(__any(is_coarse(now)), 0)) {
                float rest = -INFINITY;
#pragma unroll
                for (int u = 0; u < kGroups; ++u)
#pragma unroll
                    for (int r = 0; r < 4; ++r) rest = fmaxf(rest, logit(u, r, sc.weights[u] - now));
                rest = fmaxf(rest, __shfl_xor(rest, 16, kWave));
                rest = fmaxf(rest, __shfl_xor(rest, 32, kWave));
                now = lower_reference(m, now, rest);
            }
            const float f = __builtin_amdgcn_exp2f(m - now), fu = f * pow2(eref - sc.now);
            m = now;
            eref = __builtin_amdgcn_readfirstlane(sc.now);
            l *= f;
#pragma unroll
            for (int d = 0; d < kD; ++d) acc[d] *= fu;
            weigh(now, std::true_type());
        }
        if constexpr (kMask) {
#pragma unroll
            for (int u = 0; u < kGroups; ++u) {
                const uint32_t keep = value_mask(w.sp.len - (kt + u * kCacheGroup + 4 * g), at[0].there[u]);
#pragma unroll
                for (int h = 0; h < kH; ++h) {
                    vb[u][h].x &= keep;
                    vb[u][h].y &= keep;
                    vb[u][h].z &= keep;
                    vb[u][h].w &= keep;
                }
            }
            uint32_t nan = 0;
#pragma unroll
            for (int u = 0; u < kGroups; ++u)
#pragma unroll
                for (int h = 0; h < kH; ++h) nan |= take_nan(vb[u][h].x) | take_nan(vb[u][h].y) | take_nan(vb[u][h].z) | take_nan(vb[u][h].w);
            if (__any(nan)) nan_from = min(nan_from, kt);
        }
#pragma unroll
        for (int v = 0; v < kGroups / 2; ++v) {
            l = fmaf(sums[2 * v], sc.sums[2 * v], l);
            l = fmaf(sums[2 * v + 1], sc.sums[2 * v + 1], l);
#pragma unroll
            for (int d = 0; d < kD; ++d) {
                const typename O::vec vv = from_fp8<O>(word(vb[2 * v][d >> 2], d & 3), word(vb[2 * v + 1][d >> 2], d & 3),
                                                       sc.values[2 * v], sc.values[2 * v + 1]);
#pragma unroll
                for (int q = kP - 1; q >= 0; --q) acc[d] = O::mfma(vv, pb[v][q], acc[d]);
            }
        }
        fetch(a.v_cache, next, vb);
        at[0] = next;
        if constexpr (sizeof(T) == 4 || DP > 128) settle_products<4>();  // (accumulators that are copied for the next tile)
    });

    settle_products<4>();
    if (nan_from < w.k1) {
        for (int kt = nan_from; kt < w.k1; kt += step) {
            TileAt<kGroups> t;
            walk.look_up(kt, t);
            fetch(a.v_cache, t, vb);
#pragma unroll
            for (int v = 0; v < kGroups / 2; ++v) {
                const int lo = kt + 2 * v * kCacheGroup + 4 * g, up = lo + kCacheGroup;
                const typename O::vec seen = seen_keys<O>(t.there[2 * v] ? lo : INT_MAX - 4, t.there[2 * v + 1] ? up : INT_MAX - 4, row.lim);
#pragma unroll
                for (int d = 0; d < kD; ++d) {
                    const uint32_t w0 = word(vb[2 * v][d >> 2], d & 3), w1 = word(vb[2 * v + 1][d >> 2], d & 3);
                    const f32x4_t count = O::mfma(ones_at<O>(w0, w1), seen, f32x4_t{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[d][r] = count[r] > 0.f ? NAN : acc[d][r];
                }
            }
        }
    }
    l += __shfl_xor(l, 16, kWave);
    l += __shfl_xor(l, 32, kWave);
    float *stat = reinterpret_cast<float *>(lds4 + kWaves * kD * kWave);
    int *refs = reinterpret_cast<int *>(stat + kWaves * 16 * 2);
#pragma unroll
    for (int d = 0; d < kD; ++d) lds4[(wave * kD + d) * kWave + lane] = make_float4(acc[d][0], acc[d][1], acc[d][2], acc[d][3]);
    if (g == 0) {
        stat[(wave * 16 + j) * 2] = m;
        stat[(wave * 16 + j) * 2 + 1] = l;
    }
    if (lane == 0) refs[wave] = eref;
    __syncthreads();
    const Joined<kWaves> jn = join_waves<kWaves>(a, row, stat, refs, 16, j);
#pragma unroll
    for (int i = 0; i < kD / kWaves; ++i) {
        const int d = i * kWaves + wave;
        write_row<T, DP, kWaves>(a, w, row, w.row0 + j, 16 * d + 4 * g, jn, lds4 + d * kWave + lane, kD * kWave, d == 0 && g == 0);
    }
}

// 32 rows.  Lane (j, g) = (lane % 32, lane / 32): row j; accumulator register r of a product holds its row
// 8 (r / 4) + 4 g + r % 4, so of a tile's 32 tokens a lane has those of the first group of 16 in registers
// 0 .. 7 and those of the second in 8 .. 15.  As the row of V^T, lane j % 16 of half hi = j / 16 takes, of a
// pair of 64 dims, dim 16 s + j % 16 of the hi-th for tile s (s = 0 .. 3: all of its 16-byte pieces); of a
// last 64 dims without a pair, dim 16 (2 hi + s) + j % 16 for tile s (s = 0, 1: half of them).
template <typename T, int DP, int kRowWaves>
__global__ __launch_bounds__(kWaves *kWave, DP <= 128 && sizeof(T) == 2 ? 2 : 1) void attend_many_kernel(AttendArgs a) {
    typedef Operand<T> O;
    constexpr int kTile = attend_tile(2), kGroups = 2;
    constexpr int kStages = DP <= 128 && sizeof(T) == 2 ? 2 : 1;  // tiles in flight
    constexpr int kC = DP / 32;                 // 16-byte loads of K per lane
    constexpr int kPairs = DP / 128;            // pairs of 64 dims of V: a 16-byte piece per lane and four tokens
    constexpr bool kOdd = DP % 128 != 0;        // and a last 64 dims: half a piece
    constexpr int kD = DP / 32;                 // tiles of 32 dims
    constexpr int kKeyWaves = kWaves / kRowWaves;  // waves that share rows
    constexpr int kQ = O::kQueryPlanes, kP = O::kPlanes, step = kTile * kKeyWaves;
    extern __shared__ float4 lds4[];

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), key_wave = wave % kKeyWaves, row_wave = wave / kKeyWaves;
    const int lane = lane_id(), j = lane & 31, g = lane >> 5, i16 = lane & 15, hi = lane >> 4 & 1;
    const int chunk = blockIdx.x % a.chunks, hk = blockIdx.x / a.chunks / a.row_blocks % a.Hkv;
    const int kt0 = chunk * a.chunk + key_wave * kTile;
    Walk<kGroups, DP> walk(a, blockIdx.x / a.chunks / a.row_blocks / a.Hkv, hk, step, kt0);
    const Work w = work_of<32, kRowWaves>(a, row_wave);
    if (a.chunks > 1 && w.k0 >= w.block_reach) return;

    const Row row = row_of(a, w, w.row0 + j);
    QueryPiece<T> queries[2 * kC];
#pragma unroll
    for (int c = 0; c < 2 * kC; ++c) queries[c].load(a, row, (c >> 1) * 32 + g * 16 + (c & 1) * 8);

    struct Values {
        uint4 pair[4][kPairs > 0 ? kPairs : 1];  // [tokens 8a + 4g ..][pair of 64 dims]
        uint2 odd[4];
    };
    auto fetch_keys = [&](const TileAt<kGroups> &at, uint4 *to) {
        const uint8_t *from = a.k_cache + (hi ? at.base[1] : at.base[0]) + g * 256 + i16 * 16;
#pragma unroll
        for (int c = 0; c < kC; ++c) to[c] = load16(from, c * 512);
    };
    auto fetch_values = [&](const TileAt<kGroups> &at, Values &to) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint8_t *from = a.v_cache + at.base[q >> 1];
#pragma unroll
            for (int p = 0; p < kPairs; ++p)
                to.pair[q][p] = load16(from, p * 2048 + (q & 1) * 512 + (hi * 1024 + g * 256 + i16 * 16));
            if constexpr (kOdd)
                to.odd[q] = *reinterpret_cast<const uint2 *>(from + kPairs * 2048 + (q & 1) * 512 + (g * 256 + i16 * 16 + hi * 8));
        }
    };
    // a lane's part of the u-th 16 tokens as rows of V^T tile d
    auto value_words = [](const Values &vb, int u, int d, uint32_t &lo, uint32_t &up) {
        const int p = d >> 2, t = d & 3;
        const bool odd = p >= kPairs;
        lo = odd ? (t ? vb.odd[2 * u].y : vb.odd[2 * u].x) : word(vb.pair[2 * u][p < kPairs ? p : 0], t);
        up = odd ? (t ? vb.odd[2 * u + 1].y : vb.odd[2 * u + 1].x) : word(vb.pair[2 * u + 1][p < kPairs ? p : 0], t);
    };
    TileAt<kGroups> ats[kStages];
    uint4 kbs[kStages][kC];
    Values vbs[kStages];
    if (kt0 < w.k1) {
        walk.template begin<kStages>(kt0, w.k1, ats, [&](int i) {
            fetch_keys(ats[i], kbs[i]);
            fetch_values(ats[i], vbs[i]);
        }, [&] { return come_near(queries); });
    }
    bf16x8_t qf[2 * kC][kQ];
#pragma unroll
    for (int c = 0; c < 2 * kC; ++c) queries[c].planes(qf[c]);
    // (the queries are waited for here, not in the loop)
#pragma unroll
    for (int c = 0; c < 2 * kC; ++c)
#pragma unroll
        for (int q = 0; q < kQ; ++q) asm volatile("" ::"v"(qf[c][q]));

    f32x16_t acc[kD];
    float m = kNothing, l = 0.f;
    int eref = kScaleExpMin, nan_from = INT_MAX;
#pragma unroll
    for (int d = 0; d < kD; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[d][r] = 0.f;

    walk_tiles<kTile, kStages>(kt0, step, w, ats, [&](auto masked, int stage, int kt) {
        constexpr bool kMask = decltype(masked)::value;
        TileAt<kGroups> &at = ats[stage], next;
        uint4 *kb = kbs[stage];
        Values &vb = vbs[stage];
        walk.locate(kt + kStages * step, next);
        f32x16_t s;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
        for (int c = 0; c < 2 * kC; ++c) {
            const bf16x8_t ka = from_fp8<Operand<float>>(word(kb[c >> 1], 2 * (c & 1)), word(kb[c >> 1], 2 * (c & 1) + 1), 1.f, 1.f);
#pragma unroll
            for (int q = kQ - 1; q >= 0; --q) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka, qf[c][q], s, 0, 0, 0);
        }
        fetch_keys(next, kb);

        Scales<kGroups, sizeof(T) == 2> sc;
        sc.of(at, eref);
        __builtin_amdgcn_sched_barrier(0);  // (the products and the next keys' requests first)
        typename O::vec pb[kGroups][kP];
        float sums[kGroups];
        auto logit = [&](int r, float add) {
            float v = fmaf(s[r], at.c[r >> 3], add);
            if constexpr (kMask) v = at.there[r >> 3] && kt + 8 * (r >> 2) + 4 * g + (r & 3) < row.lim ? v : -INFINITY;
            return v;
        };
        auto weigh = [&](float ref, auto most) {
            constexpr bool kMost = decltype(most)::value;
#pragma unroll
            for (int u = 0; u < kGroups; ++u) {
                const float add = sc.weights[u] - ref;
                sums[u] = 0.f;
#pragma unroll
                for (int r = 0; r < 8; r += 2) {
                    const float p0 = __builtin_amdgcn_exp2f(at_most<kMost>(logit(8 * u + r, add)));
                    const float p1 = __builtin_amdgcn_exp2f(at_most<kMost>(logit(8 * u + r + 1, add)));
                    typename O::pair pp[kP];
                    split<O, kP>(f32x2_t{p0, p1}, pp);
                    sums[u] += p0;
                    sums[u] += p1;
#pragma unroll
                    for (int q = 0; q < kP; ++q) {
                        pb[u][q][r] = pp[q][0];
                        pb[u][q][r + 1] = pp[q][1];
                    }
                }
            }
            return sums[0] + sums[1];
        };
        if (__any(weigh(m, std::false_type()) > kRaise) || sc.now > eref) {
            float top = -INFINITY;
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, logit(r, sc.weights[r >> 3]));
            top = fmaxf(top, __shfl_xor(top, 32, kWave));
            float now = fmaxf(m, top - kBias);
            if (__builtin_expect(__any(is_coarse(now)), 0)) {
                float rest = -INFINITY;
#pragma unroll
                for (int r = 0; r < 16; ++r) rest = fmaxf(rest, logit(r, sc.weights[r >> 3] - now));
                rest = fmaxf(rest, __shfl_xor(rest, 32, kWave));
                now = lower_reference(m, now, rest);
            }
            const float f = __builtin_amdgcn_exp2f(m - now), fu = f * pow2(eref - sc.now);
            m = now;
            eref = __builtin_amdgcn_readfirstlane(sc.now);
            l *= f;
#pragma unroll
            for (int d = 0; d < kD; ++d) acc[d] *= fu;
            weigh(now, std::true_type());
        }
        if constexpr (kMask) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t keep = value_mask(w.sp.len - (kt + 8 * q + 4 * g), at.there[q >> 1]);
#pragma unroll
                for (int p = 0; p < kPairs; ++p) {
                    vb.pair[q][p].x &= keep;
                    vb.pair[q][p].y &= keep;
                    vb.pair[q][p].z &= keep;
                    vb.pair[q][p].w &= keep;
                }
                if constexpr (kOdd) {
                    vb.odd[q].x &= keep;
                    vb.odd[q].y &= keep;
                }
            }
            uint32_t nan = 0;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
#pragma unroll
                for (int p = 0; p < kPairs; ++p)
                    nan |= take_nan(vb.pair[q][p].x) | take_nan(vb.pair[q][p].y) | take_nan(vb.pair[q][p].z) | take_nan(vb.pair[q][p].w);
                if constexpr (kOdd) nan |= take_nan(vb.odd[q].x) | take_nan(vb.odd[q].y);
            }
            if (__any(nan)) nan_from = min(nan_from, kt);
        }
#pragma unroll
        for (int u = 0; u < kGroups; ++u) {
            l = fmaf(sums[u], sc.sums[u], l);
#pragma unroll
            for (int d = 0; d < kD; ++d) {
                uint32_t lo, up;
                value_words(vb, u, d, lo, up);
                const typename O::vec vv = from_fp8<O>(lo, up, sc.values[u], sc.values[u]);
#pragma unroll
                for (int q = kP - 1; q >= 0; --q) acc[d] = O::mfma32(vv, pb[u][q], acc[d]);
            }
        }
        fetch_values(next, vb);
        at = next;
        if constexpr (sizeof(T) == 4 || DP > 128) settle_products<4>();
    });

    settle_products<4>();
    if (nan_from < w.k1) {
        for (int kt = nan_from; kt < w.k1; kt += step) {
            TileAt<kGroups> at;
            Values vb;
            walk.look_up(kt, at);
            fetch_values(at, vb);
#pragma unroll
            for (int u = 0; u < kGroups; ++u) {
                const int lo = at.there[u] ? kt + u * kCacheGroup + 4 * g : INT_MAX - 12;
                const typename O::vec seen = seen_keys<O>(lo, lo + 8, row.lim);
#pragma unroll
                for (int d = 0; d < kD; ++d) {
                    uint32_t w0, w1;
                    value_words(vb, u, d, w0, w1);
                    f32x16_t count;
#pragma unroll
                    for (int r = 0; r < 16; ++r) count[r] = 0.f;
                    count = O::mfma32(ones_at<O>(w0, w1), seen, count);
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[d][r] = count[r] > 0.f ? NAN : acc[d][r];
                }
            }
        }
    }
    l += __shfl_xor(l, 32, kWave);
    // half of the tiles at a time: [wave][tile][register quad][lane]
    constexpr int kHalf = kD / 2;
    float *stat = reinterpret_cast<float *>(lds4 + kWaves * kHalf * 4 * kWave);
    int *refs = reinterpret_cast<int *>(stat + kWaves * 32 * 2);
    if (g == 0) {
        stat[(wave * 32 + j) * 2] = m;
        stat[(wave * 32 + j) * 2 + 1] = l;
    }
    if (lane == 0) refs[wave] = eref;
    Joined<kKeyWaves> jn;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        if (half) __syncthreads();
#pragma unroll
        for (int i = 0; i < kHalf; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x16_t &c = acc[half * kHalf + i];
                lds4[((wave * kHalf + i) * 4 + q) * kWave + lane] = make_float4(c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]);
            }
        __syncthreads();
        if (half == 0) jn = join_waves<kKeyWaves>(a, row, stat + row_wave * kKeyWaves * 64, refs + row_wave * kKeyWaves, 32, j);
#pragma unroll
        for (int i = 0; i < kHalf; ++i)
#pragma unroll
            for (int q = key_wave; q < 4; q += kKeyWaves) {
                // register quad q of a tile: dims 8 (q % 2) + 4 g .. +3 of 16, of the half q / 2
                const int d = half * kHalf + i, p = d >> 2, t = d & 3, inner = 8 * (q & 1) + 4 * g;
                const int dim = p < kPairs ? 64 * (2 * p + (q >> 1)) + 16 * t + inner
                                           : 128 * kPairs + 16 * (2 * (q >> 1) + t) + inner;
                write_row<T, DP, kKeyWaves>(a, w, row, w.row0 + j, dim, jn,
                                            lds4 + ((row_wave * kKeyWaves * kHalf + i) * 4 + q) * kWave + lane,
                                            kHalf * 4 * kWave, d == 0 && q == 0 && g == 0);
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
    const float inv = sum > 0.f ? 1.f / sum : mx == kHollow ? NAN : 0.f;
    const int64_t at = (((int64_t)b * a.Hq + hk * G + (r - t * G)) * a.T + t) * a.dh + dim;
    store4<T>(static_cast<T *>(a.out) + at, o * inv);
}

template <typename Kernel>
hipError_t launch_attend(Kernel kernel, const AttendArgs &a, size_t lds, std::atomic<uint64_t> &done, hipStream_t s) {
    if (lds > 65536) {
        const hipError_t e = allow_large_lds(kernel, done);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)((int64_t)a.B * a.Hkv * a.row_blocks * a.chunks)), dim3(kWaves * kWave), lds, s, a);
    return hipGetLastError();
}

template <typename T, int DP>
hipError_t launch_dp(const AttendArgs &a, hipStream_t s) {
    static std::atomic<uint64_t> few{0}, one{0}, two{0};
    const size_t acc = kWaves * DP * 16 * sizeof(float), refs = kWaves * sizeof(int);
    if constexpr (attend_many_fits(sizeof(T) == 2, DP)) {
        const size_t lds = acc + kWaves * 32 * 2 * sizeof(float) + refs;
        if (a.row_tiles == 2 && a.row_waves == 2) return launch_attend(attend_many_kernel<T, DP, 2>, a, lds, two, s);
        if (a.row_tiles == 2) return launch_attend(attend_many_kernel<T, DP, 1>, a, lds, one, s);
    }
    return launch_attend(attend_few_kernel<T, DP>, a, acc + kWaves * 16 * 2 * sizeof(float) + refs, few, s);
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
