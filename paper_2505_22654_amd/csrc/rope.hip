// Rotary positions of q and k over several axes.
//
// A row's pair (x, y) is turned by w = position * frequency.  The exact product, as two 64-bit numbers, is
// reduced to a quadrant and a rest of at most pi/4, with pi/2 in two parts (rounded, the product alone would be
// off by 2^-23 at the ends of 32 bits); sine and cosine of the rest are their Taylor sums to x^9 and x^10 in
// 32 bits (remainders 1.8e-9 and 1.2e-10 at pi/4).  Angles depend on the token and the pair only, so
// a thread keeps its pairs' values and walks over heads with them.  Bound: HBM, a read and a write of
// every entry.  Angles handed around through LDS, with neighbouring heads in one workgroup, took 17.2 to
// 20.5 us where this takes 16.9 (4352 tokens x 32 heads x 128, from the caches).
#include <hip/hip_runtime.h>

#include "common.hpp"
#include "decode.hpp"

namespace {

using namespace vscan;

__device__ __forceinline__ void turn(int position, double freq, bool inverse, float &c, float &s) {
    const double w = (double)position * freq, rest = fma((double)position, freq, -w);
    const double n = rint(w * 0.63661977236758134308);  // 2 / pi
    // w - n pi/2: the first part of pi/2 leaves an exact difference, to 2^-53
    const float a = (float)(fma(-n, 1.57079632679489655800, w) + fma(-n, 6.12323399573676603587e-17, rest));
    const int quadrant = (int)(n - 4.0 * floor(n * 0.25));
    const float z = a * a;
    const float sn = fmaf(a * z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), a);
    const float cs = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
    const bool swap = quadrant & 1;
    c = swap ? sn : cs;
    s = swap ? cs : sn;
    if (quadrant == 1 || quadrant == 2) c = -c;
    if (quadrant >= 2) s = -s;
    if (inverse) s = -s;
}

// As vectors: the compiler takes a struct apart and stores its bytes in pieces of 2, 4 and 8.  Ten sets of inputs in
// turn, more than the caches hold, us in pieces, whole, and whole with the non-temporal hint:
//   4352 tokens x 32 heads x 128 in bf16: 23.6, 18.6 (3.8 TB/s; 15.5 on one set, from the caches), 19.5
//   2 x 4096 tokens x 40 heads x 128 in bf16: 39.5, 31.4 (5.3 TB/s), 35.6; x 72, in pieces of 8 bytes: 33.6, 25.8
//   2 x 2745 tokens x 32 heads x 80 in fp32: 28.7, 25.4 (4.4 TB/s), 28.7
__device__ __forceinline__ void put16(char *p, const uint4 &v) {
    *reinterpret_cast<u32x4_t *>(p) = u32x4_t{v.x, v.y, v.z, v.w};
}
__device__ __forceinline__ void put8(char *p, const uint2 &v) {
    typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
    *reinterpret_cast<u32x2_t *>(p) = u32x2_t{v.x, v.y};
}
// N consecutive entries of a row: 8 or 16 bytes
template <typename T, int N>
struct Piece;
template <>
struct Piece<bf16_t, 8> {
    uint4 raw;
    __device__ __forceinline__ void load(const char *p) { raw = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void get(float *f) const { unpack16<bf16_t>(raw, f); }
    __device__ __forceinline__ void store(char *p, const float *f) const {
        union {
            __bf16 h[8];
            uint4 u;
        } o;
        for (int i = 0; i < 8; ++i) o.h[i] = (__bf16)f[i];
        put16(p, o.u);
    }
};
template <>
struct Piece<bf16_t, 4> {
    uint2 raw;
    __device__ __forceinline__ void load(const char *p) { raw = *reinterpret_cast<const uint2 *>(p); }
    __device__ __forceinline__ void get(float *f) const {
        f[0] = bf16_lo(raw.x);
        f[1] = bf16_hi(raw.x);
        f[2] = bf16_lo(raw.y);
        f[3] = bf16_hi(raw.y);
    }
    __device__ __forceinline__ void store(char *p, const float *f) const {
        union {
            __bf16 h[4];
            uint2 u;
        } o;
        for (int i = 0; i < 4; ++i) o.h[i] = (__bf16)f[i];
        put8(p, o.u);
    }
};
template <>
struct Piece<float, 4> {
    uint4 raw;
    __device__ __forceinline__ void load(const char *p) { raw = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void get(float *f) const { unpack16<float>(raw, f); }
    __device__ __forceinline__ void store(char *p, const float *f) const {
        put16(p, make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])));
    }
};

constexpr int kThreads = 256;

// N: entries of a piece.  In halves a thread owns a piece of either half (N pairs); with adjacent
// pairs one piece (N/2 pairs).  Pieces of the entries past rot_dim are copied where a tensor is not
// turned in place.
template <typename T, int N, bool ADJ>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a, int pieces, int rest, int per_slice) {
    const int id = blockIdx.x * kThreads + threadIdx.x;
    const int all = pieces + rest;
    if (id >= a.B * a.S * all) return;
    const int piece = id % all, token = id / all;
    const int b = token / a.S, s = token - b * a.S;
    constexpr int kPairs = ADJ ? N / 2 : N;
    constexpr int kBytes = N * (int)sizeof(T);
    const bool turned = piece < pieces;
    float c[kPairs], sn[kPairs];
    if (turned) {
#pragma unroll
        for (int e = 0; e < kPairs; ++e) {
            const int i = piece * kPairs + e;
            const int p = a.positions[((int64_t)a.axis[i] * a.B + b) * a.S + s];
            turn(p, a.inv_freq[i], a.inverse, c[e], sn[e]);
        }
    }
    const int off = turned ? piece * kBytes : a.rot * (int)sizeof(T) + (piece - pieces) * kBytes;
    const int second = a.rot / 2 * (int)sizeof(T);
    const int total = a.heads[0] + a.heads[1];
    const int h1 = min(total, (int)(blockIdx.y + 1) * per_slice);
    for (int h = blockIdx.y * per_slice; h < h1; ++h) {
        const int which = h >= a.heads[0], head = which ? h - a.heads[0] : h;
        const int64_t *is = a.in_stride[which], *os = a.out_stride[which];
        const char *src = static_cast<const char *>(a.in[which]) +
                          (b * is[0] + head * is[1] + s * is[2]) * (int64_t)sizeof(T) + off;
        char *dst = static_cast<char *>(a.out[which]) +
                    (b * os[0] + head * os[1] + s * os[2]) * (int64_t)sizeof(T) + off;
        Piece<T, N> p, p2;
        float x[N], y[N];
        p.load(src);
        if (!turned) {
            p.get(x);
            p.store(dst, x);
            continue;
        }
        if constexpr (ADJ) {
            p.get(x);
#pragma unroll
            for (int e = 0; e < kPairs; ++e) {
                y[2 * e] = x[2 * e] * c[e] - x[2 * e + 1] * sn[e];
                y[2 * e + 1] = x[2 * e] * sn[e] + x[2 * e + 1] * c[e];
            }
            p.store(dst, y);
        } else {
            p2.load(src + second);
            p.get(x);
            p2.get(y);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float u = x[e] * c[e] - y[e] * sn[e], v = x[e] * sn[e] + y[e] * c[e];
                x[e] = u;
                y[e] = v;
            }
            p.store(dst, x);
            p2.store(dst + second, y);
        }
    }
}

// Heads are cut into slices until there are 1024 workgroups: fewer leave loads missing, more work out
// angles again.  4352 tokens x 32 heads x 128 in bf16, ten sets in turn, with 256, 512, 1024, 2048 and 4096
// workgroups: 31.2, 21.0, 18.8, 18.9, 22.4 us.
template <typename T, int N, bool ADJ>
hipError_t launch(const RopeArgs &a, hipStream_t s) {
    const int pieces = ADJ ? a.rot / N : a.rot / 2 / N;
    const int rest = a.copy_rest ? (a.dh - a.rot) / N : 0;
    const int64_t items = (int64_t)a.B * a.S * (pieces + rest);
    const int blocks = (int)((items + kThreads - 1) / kThreads);
    const int heads = a.heads[0] + a.heads[1];
    int slices = 1;
    while (slices < heads && (int64_t)blocks * slices < 1024) slices *= 2;
    const int per = (heads + slices - 1) / slices;
    const dim3 grid(blocks, (heads + per - 1) / per);
    hipLaunchKernelGGL((rope_kernel<T, N, ADJ>), grid, dim3(kThreads), 0, s, a, pieces, rest, per);
    return hipGetLastError();
}

}  // namespace

namespace vscan {

hipError_t launch_rope(const void *args, hipStream_t s) {
    const RopeArgs &a = *static_cast<const RopeArgs *>(args);
    if (!a.is_bf16) return a.adjacent ? launch<float, 4, true>(a, s) : launch<float, 4, false>(a, s);
    if (a.adjacent) return launch<bf16_t, 8, true>(a, s);
    // halves of a multiple of 8 entries start on 16 bytes
    return a.rot % 16 == 0 ? launch<bf16_t, 8, false>(a, s) : launch<bf16_t, 4, false>(a, s);
}

}  // namespace vscan
