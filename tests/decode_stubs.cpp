// CPU stand-ins for the kernel launchers behind vscan_rope and the vscan_cache_* calls: they check
// that the scratch the host layer hands out lies inside the window the test has announced, and that
// the grid a call asks for covers its rows and keys.
#include <stdlib.h>

#include "../paper_2505_22654_amd/csrc/decode.hpp"

namespace {
uintptr_t g_lo, g_hi;
int g_launches;

void need(bool ok) {
    if (!ok) abort();
}
void inside(const void *p, size_t bytes) {
    const uintptr_t u = reinterpret_cast<uintptr_t>(p);
    need(u >= g_lo && u + bytes <= g_hi);
}
}  // namespace

extern "C" {
void vscan_test_decode_window(void *base, size_t bytes) {
    g_lo = reinterpret_cast<uintptr_t>(base);
    g_hi = g_lo + bytes;
    g_launches = 0;
}
int vscan_test_decode_launches() { return g_launches; }
}

namespace vscan {

hipError_t launch_rope(const void *args, hipStream_t) {
    const RopeArgs &a = *static_cast<const RopeArgs *>(args);
    for (int i = 0; i < 2; ++i) need(!a.heads[i] || (a.in[i] && a.out[i]));
    for (int i = 0; i < a.rot / 2; ++i) need(a.axis[i] < 4);
    ++g_launches;
    return hipSuccess;
}

hipError_t launch_cache_plan(const void *args, hipStream_t) {
    const PlanArgs &a = *static_cast<const PlanArgs *>(args);
    if (plan_needs_scratch(a.B, a.n_new)) inside(a.requests, (size_t)a.B * 16);
    else need(plan_workgroups(a) > 0 && a.B <= kPlanThreads);
    ++g_launches;
    return hipSuccess;
}
hipError_t launch_cache_tables(const void *args, hipStream_t s) { return launch_cache_plan(args, s); }

hipError_t launch_cache_store(const void *args, hipStream_t) {
    const StoreArgs &a = *static_cast<const StoreArgs *>(args);
    need(a.seq_len >= a.n_new);
    ++g_launches;
    return hipSuccess;
}

hipError_t launch_cache_attend(const void *args, hipStream_t) {
    const AttendArgs &a = *static_cast<const AttendArgs *>(args);
    const int64_t rows = (int64_t)(a.Hq / a.Hkv) * a.T;
    const int block = kCacheGroup * a.row_tiles * a.row_waves;
    need((int64_t)a.row_blocks * block >= rows && (int64_t)(a.row_blocks - 1) * block < rows);
    need(a.chunks >= 1 && (int64_t)a.chunk * a.chunks >= a.max_len && a.chunk % (kAttendWaves / a.row_waves * attend_tile(a.row_tiles)) == 0);
    if (a.chunks > 1) {
        const size_t parts = (size_t)a.B * a.Hkv * rows * a.chunks;
        inside(a.part_acc, parts * cache_dp(a.dh) * 4);
        inside(a.part_stat, parts * 8);
        need(reinterpret_cast<uintptr_t>(a.part_acc + parts * cache_dp(a.dh)) <= reinterpret_cast<uintptr_t>(a.part_stat));
    }
    ++g_launches;
    return hipSuccess;
}
hipError_t launch_cache_combine(const void *args, hipStream_t) {
    need(static_cast<const AttendArgs *>(args)->chunks > 1);
    ++g_launches;
    return hipSuccess;
}

}  // namespace vscan
