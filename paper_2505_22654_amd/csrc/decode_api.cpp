// Entry points around the pruned prefill: argument validation, workspace planning and kernel
// sequencing of vscan_rope and the vscan_cache_* calls.  As in api.cpp everything before the first
// launch is host code that never touches the HIP runtime.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "../../include/vscan.h"
#include "decode.hpp"
#include "log.hpp"

namespace {

using namespace vscan;

constexpr size_t kAlign = 256;
constexpr int64_t kMaxWorkgroups = (int64_t)1 << 24;  // of 256 threads: a grid has less than 2^32 threads
inline size_t align_up(size_t v) { return (v + kAlign - 1) & ~(kAlign - 1); }
inline bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline int elem_bytes(int dtype) { return dtype == VSCAN_BF16 ? 2 : 4; }

inline int finish(const char *entry, int rc) {
    if (rc != VSCAN_OK) logf("%s -> %d (%s)", entry, rc, vscan_status_string(rc));
    return rc;
}

// ---- rotary positions --------------------------------------------------------------------------
int check_rope(const vscan_rope_desc *d) {
    if (!d) return VSCAN_ERR_NULL;
    if (d->struct_size != sizeof(vscan_rope_desc)) return VSCAN_ERR_VERSION;
    if (d->dtype != VSCAN_F32 && d->dtype != VSCAN_BF16) return VSCAN_ERR_DTYPE;
    if (d->order != VSCAN_ROPE_SECTIONS && d->order != VSCAN_ROPE_CYCLED) return VSCAN_ERR_DTYPE;
    if (d->pairing != VSCAN_ROPE_HALVES && d->pairing != VSCAN_ROPE_ADJACENT) return VSCAN_ERR_DTYPE;
    if (d->batch < 0 || d->seq_len < 0 || d->q_heads < 0 || d->kv_heads < 0) return VSCAN_ERR_SHAPE;
    if (d->q_heads > 1024 || d->kv_heads > 1024) return VSCAN_ERR_SHAPE;
    if (d->head_dim < 8 || d->head_dim % 8 || d->head_dim > 256) return VSCAN_ERR_SHAPE;
    if (d->rot_dim < 8 || d->rot_dim % 8 || d->rot_dim > d->head_dim) return VSCAN_ERR_SHAPE;
    if (d->n_axes < 1 || d->n_axes > VSCAN_ROPE_MAX_AXES) return VSCAN_ERR_SHAPE;
    if (d->inverse != 0 && d->inverse != 1) return VSCAN_ERR_SHAPE;
    int64_t pairs = 0;
    for (int a = 0; a < d->n_axes; ++a) {
        if (d->sections[a] < 0) return VSCAN_ERR_SHAPE;
        pairs += d->sections[a];
    }
    if (pairs != d->rot_dim / 2) return VSCAN_ERR_SHAPE;
    // (sequence, token, piece) triples are counted in 32 bits
    if ((int64_t)d->batch * d->seq_len * 64 >= ((int64_t)1 << 31)) return VSCAN_ERR_UNSUPPORTED;
    return VSCAN_OK;
}

// Axis of every pair.
void rope_axes(const vscan_rope_desc *d, uint8_t *axis) {
    int left[VSCAN_ROPE_MAX_AXES], n = 0;
    memcpy(left, d->sections, sizeof(left));
    for (int i = d->n_axes; i < VSCAN_ROPE_MAX_AXES; ++i) left[i] = 0;
    if (d->order == VSCAN_ROPE_SECTIONS) {
        for (int a = 0; a < d->n_axes; ++a)
            for (int i = 0; i < left[a]; ++i) axis[n++] = (uint8_t)a;
        return;
    }
    while (n < d->rot_dim / 2)
        for (int a = 0; a < d->n_axes; ++a)
            if (left[a] > 0) {
                --left[a];
                axis[n++] = (uint8_t)a;
            }
}

// Strides of a tensor [B, heads, S, dh] as the kernel takes them; false where they cannot be used.
bool rope_strides(const int64_t given[3], int64_t heads, int64_t S, int64_t dh, int es, int64_t out[3]) {
    if (given[0] == 0 && given[1] == 0 && given[2] == 0) {
        out[0] = heads * S * dh;
        out[1] = S * dh;
        out[2] = dh;
        return true;
    }
    for (int i = 0; i < 3; ++i) {
        // the largest offset in bytes stays inside 64 bits
        if (given[i] < 0 || given[i] > ((int64_t)1 << 34) || given[i] * es % 16) return false;
        out[i] = given[i];
    }
    return true;
}

// Whether no two rows of dh entries share memory: sorted by stride, each axis steps over all that
// the smaller ones reach.
bool rows_apart(const int64_t stride[3], int64_t B, int64_t heads, int64_t S, int64_t dh) {
    struct Axis {
        int64_t stride, size;
    } a[3] = {{stride[0], B}, {stride[1], heads}, {stride[2], S}};
    std::sort(a, a + 3, [](const Axis &x, const Axis &y) { return x.stride < y.stride; });
    if (B == 0 || heads == 0 || S == 0) return true;
    int64_t reach = dh;
    for (const Axis &x : a) {
        if (x.size <= 1) continue;
        if (x.stride < reach) return false;
        reach += x.stride * (x.size - 1);
    }
    return true;
}

int rope(const vscan_rope_desc *d, void *q, void *k, const int32_t *positions, const double *inv_freq,
         void *q_out, void *k_out, void *stream) {
    const int rc = check_rope(d);
    if (rc != VSCAN_OK) return rc;
    const int es = elem_bytes(d->dtype);
    RopeArgs a;
    memset(&a, 0, sizeof(a));
    void *const in[2] = {q, k}, *const out[2] = {q_out, k_out};
    const int heads[2] = {d->q_heads, d->kv_heads};
    const int64_t *const given[2] = {d->q_stride, d->k_stride};
    for (int i = 0; i < 2; ++i) {
        if (!heads[i]) continue;
        if (!rope_strides(given[i], heads[i], d->seq_len, d->head_dim, es, a.in_stride[i]))
            return VSCAN_ERR_SHAPE;
        if (!out[i] && !rows_apart(a.in_stride[i], d->batch, heads[i], d->seq_len, d->head_dim))
            return VSCAN_ERR_SHAPE;
    }
    if (d->batch == 0 || d->seq_len == 0 || (!heads[0] && !heads[1])) return VSCAN_OK;
    if (!positions || !inv_freq) return VSCAN_ERR_NULL;
    for (int i = 0; i < 2; ++i) {
        if (heads[i] && !in[i]) return VSCAN_ERR_NULL;
        if (!aligned(in[i], 16) || !aligned(out[i], 16)) return VSCAN_ERR_ALIGN;
    }
    if (!aligned(positions, 4) || !aligned(inv_freq, 8)) return VSCAN_ERR_ALIGN;
    for (int i = 0; i < 2; ++i) {
        if (!heads[i]) continue;
        a.heads[i] = heads[i];
        a.in[i] = in[i];
        a.out[i] = out[i] ? out[i] : in[i];
        const int64_t dense[3] = {(int64_t)heads[i] * d->seq_len * d->head_dim,
                                  (int64_t)d->seq_len * d->head_dim, d->head_dim};
        memcpy(a.out_stride[i], out[i] ? dense : a.in_stride[i], sizeof(dense));
        a.copy_rest |= out[i] != nullptr;
    }
    a.positions = positions;
    a.inv_freq = inv_freq;
    a.B = d->batch;
    a.S = d->seq_len;
    a.dh = d->head_dim;
    a.rot = d->rot_dim;
    a.adjacent = d->pairing == VSCAN_ROPE_ADJACENT;
    a.inverse = d->inverse;
    a.is_bf16 = d->dtype == VSCAN_BF16;
    rope_axes(d, a.axis);
    return enqueue("rope", static_cast<hipStream_t>(stream), launch_rope, &a);
}

// ---- the cache ---------------------------------------------------------------------------------
int check_cache(const vscan_cache_desc *d) {
    if (!d) return VSCAN_ERR_NULL;
    if (d->struct_size != sizeof(vscan_cache_desc)) return VSCAN_ERR_VERSION;
    if (d->dtype != VSCAN_F32 && d->dtype != VSCAN_BF16) return VSCAN_ERR_DTYPE;
    if (d->batch < 0 || d->batch > 65535 || d->n_blocks < 1 || d->max_blocks < 1 || d->n_new < 0)
        return VSCAN_ERR_SHAPE;
    if (d->q_heads < 1 || d->kv_heads < 1 || d->q_heads % d->kv_heads || d->q_heads > 1024)
        return VSCAN_ERR_SHAPE;
    if (d->head_dim < 8 || d->head_dim % 8 || d->head_dim > 256) return VSCAN_ERR_SHAPE;
    if (d->block_size < 16 || d->block_size > 256 || (d->block_size & (d->block_size - 1)))
        return VSCAN_ERR_SHAPE;
    if (d->seq_len < 0 || (d->seq_len && d->seq_len < d->n_new) || d->max_len < 0) return VSCAN_ERR_SHAPE;
    const int64_t lim = (int64_t)1 << 31;
    if ((int64_t)d->n_blocks * d->block_size >= lim || (int64_t)d->max_blocks * d->block_size >= lim)
        return VSCAN_ERR_SHAPE;
    if ((int64_t)d->max_len > (int64_t)d->max_blocks * d->block_size) return VSCAN_ERR_SHAPE;
    // table entries, slots and (block, head) pairs are counted in 32 bits
    if ((int64_t)d->batch * d->max_blocks >= lim || (int64_t)d->batch * d->n_new >= lim ||
        (int64_t)d->n_blocks * d->kv_heads >= lim)
        return VSCAN_ERR_UNSUPPORTED;
    return VSCAN_OK;
}

inline int shift_of(int block_size) {
    int s = 0;
    while ((1 << s) < block_size) ++s;
    return s;
}

int cache_plan(const vscan_cache_desc *d, const int32_t *cached_len, const int32_t *new_len,
               const int32_t *free_blocks, int32_t n_free, const int32_t *free_head,
               int32_t *block_table, int32_t *slot_map, int32_t *kv_len, int32_t *free_head_out,
               int32_t *missing, void *workspace, size_t workspace_bytes, void *stream) {
    size_t need = 0;
    const int rc = vscan_cache_plan_workspace_size(d, &need);
    if (rc != VSCAN_OK) return rc;
    if (n_free < 0) return VSCAN_ERR_SHAPE;
    if (!free_head || !free_head_out || !missing || (n_free && !free_blocks)) return VSCAN_ERR_NULL;
    if (d->batch && (!cached_len || !new_len || !block_table || !kv_len || (d->n_new && !slot_map)))
        return VSCAN_ERR_NULL;
    const void *const all[] = {cached_len, new_len, free_blocks, free_head, block_table,
                               slot_map, kv_len, free_head_out, missing};
    for (const void *p : all)
        if (!aligned(p, 4)) return VSCAN_ERR_ALIGN;
    if (need && (!workspace || workspace_bytes < need)) return VSCAN_ERR_WORKSPACE;
    if (need && !aligned(workspace, 16)) return VSCAN_ERR_ALIGN;
    PlanArgs a;
    a.cached_len = cached_len;
    a.new_len = new_len;
    a.free_blocks = free_blocks;
    a.free_head = free_head;
    a.block_table = block_table;
    a.slot_map = slot_map;
    a.kv_len = kv_len;
    a.free_head_out = free_head_out;
    a.missing = missing;
    a.requests = static_cast<int32_t *>(workspace);
    a.B = d->batch;
    a.n_new = d->n_new;
    a.block_shift = shift_of(d->block_size);
    a.n_blocks = d->n_blocks;
    a.max_blocks = d->max_blocks;
    a.n_free = n_free;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const int rc2 = enqueue("cache_plan", s, launch_cache_plan, &a);
    if (rc2 != VSCAN_OK || plan_workgroups(a)) return rc2;
    return enqueue("cache_tables", s, launch_cache_tables, &a);
}

int cache_store(const vscan_cache_desc *d, const void *k, const void *v, const int32_t *slot_map,
                void *k_cache, void *v_cache, float *k_scale, float *v_scale, void *stream) {
    const int rc = check_cache(d);
    if (rc != VSCAN_OK) return rc;
    // one wave or workgroup per (k or v, sequence, kv head, block that the new rows touch)
    const int64_t runs = store_runs(d->n_new, d->block_size);
    if ((int64_t)d->batch * d->kv_heads * runs * 2 >= kMaxWorkgroups * store_pages(d->block_size)) return VSCAN_ERR_UNSUPPORTED;
    if (d->batch == 0 || d->n_new == 0) return VSCAN_OK;
    if (!k || !v || !slot_map || !k_cache || !v_cache || !k_scale || !v_scale) return VSCAN_ERR_NULL;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) ||
        !aligned(slot_map, 4) || !aligned(k_scale, 4) || !aligned(v_scale, 4))
        return VSCAN_ERR_ALIGN;
    StoreArgs a;
    a.x[0] = k;
    a.x[1] = v;
    a.cache[0] = static_cast<uint8_t *>(k_cache);
    a.cache[1] = static_cast<uint8_t *>(v_cache);
    a.scale[0] = k_scale;
    a.scale[1] = v_scale;
    a.slot_map = slot_map;
    a.B = d->batch;
    a.Hkv = d->kv_heads;
    a.n_new = d->n_new;
    a.seq_len = d->seq_len ? d->seq_len : d->n_new;
    a.dh = d->head_dim;
    a.block_shift = shift_of(d->block_size);
    a.n_blocks = d->n_blocks;
    a.is_bf16 = d->dtype == VSCAN_BF16;
    return enqueue("cache_store", static_cast<hipStream_t>(stream), launch_cache_store, &a);
}

struct AttendPlan {
    AttendArgs a;
    size_t off_stat, bytes;
};
int plan_attend(const vscan_cache_desc *d, AttendPlan *p) {
    const int rc = check_cache(d);
    if (rc != VSCAN_OK) return rc;
    AttendArgs &a = p->a;
    memset(&a, 0, sizeof(a));
    a.B = d->batch;
    a.Hq = d->q_heads;
    a.Hkv = d->kv_heads;
    a.T = d->n_new;
    a.dh = d->head_dim;
    a.block_shift = shift_of(d->block_size);
    a.n_blocks = d->n_blocks;
    a.max_blocks = d->max_blocks;
    a.max_len = d->max_len ? d->max_len : d->max_blocks * d->block_size;
    a.is_bf16 = d->dtype == VSCAN_BF16;
    a.scale = (d->scale > 0.f ? d->scale : 1.0f / sqrtf((float)d->head_dim)) * 1.44269504088896341f;
    a.far_scale = a.scale * kFarScale;
    p->off_stat = p->bytes = 0;
    const int64_t rows = (int64_t)(a.Hq / a.Hkv) * a.T;
    // rows, and keys a few tiles past the last one, are counted in 32 bits
    if (rows >= ((int64_t)1 << 30) || (int64_t)a.B * a.Hkv * rows >= ((int64_t)1 << 31) || a.max_len > (1 << 30))
        return VSCAN_ERR_UNSUPPORTED;
    if (a.B == 0 || rows == 0) return VSCAN_OK;
    attend_form(a);
    if ((int64_t)a.B * a.Hkv * a.row_blocks * a.chunks >= kMaxWorkgroups) return VSCAN_ERR_UNSUPPORTED;
    if (a.chunks > 1) {
        const size_t parts = (size_t)a.B * a.Hkv * rows * a.chunks;
        p->off_stat = align_up(parts * cache_dp(a.dh) * sizeof(float));
        p->bytes = p->off_stat + align_up(parts * 2 * sizeof(float));
    }
    return VSCAN_OK;
}

int cache_attend(const vscan_cache_desc *d, const void *q, const void *k_cache, const void *v_cache,
                 const float *k_scale, const float *v_scale, const int32_t *block_table,
                 const int32_t *kv_len, const int32_t *new_len, void *out, void *workspace,
                 size_t workspace_bytes, void *stream) {
    AttendPlan p;
    const int rc = plan_attend(d, &p);
    if (rc != VSCAN_OK) return rc;
    AttendArgs &a = p.a;
    if (a.B == 0 || a.T == 0) return VSCAN_OK;
    if (!q || !k_cache || !v_cache || !k_scale || !v_scale || !block_table || !kv_len || !out)
        return VSCAN_ERR_NULL;
    if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(out, 16) ||
        !aligned(k_scale, 4) || !aligned(v_scale, 4) || !aligned(block_table, 4) ||
        !aligned(kv_len, 4) || !aligned(new_len, 4))
        return VSCAN_ERR_ALIGN;
    if (p.bytes && (!workspace || workspace_bytes < p.bytes)) return VSCAN_ERR_WORKSPACE;
    if (p.bytes && !aligned(workspace, 16)) return VSCAN_ERR_ALIGN;
    a.q = q;
    a.k_cache = static_cast<const uint8_t *>(k_cache);
    a.v_cache = static_cast<const uint8_t *>(v_cache);
    a.k_scale = k_scale;
    a.v_scale = v_scale;
    a.block_table = block_table;
    a.kv_len = kv_len;
    a.new_len = new_len;
    a.out = out;
    a.part_acc = static_cast<float *>(workspace);
    a.part_stat = a.chunks > 1 ? reinterpret_cast<float *>(static_cast<unsigned char *>(workspace) + p.off_stat)
                               : nullptr;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const int rc2 = enqueue("cache_attend", s, launch_cache_attend, &a);
    if (rc2 != VSCAN_OK || a.chunks == 1) return rc2;
    return enqueue("cache_combine", s, launch_cache_combine, &a);
}

}  // namespace

extern "C" {

int vscan_rope(const vscan_rope_desc *desc, void *q, void *k, const int32_t *positions,
               const double *inv_freq, void *q_out, void *k_out, void *stream) {
    return finish("vscan_rope", rope(desc, q, k, positions, inv_freq, q_out, k_out, stream));
}

int vscan_cache_size(const vscan_cache_desc *desc, size_t *cache_bytes, size_t *scale_bytes) {
    if (!cache_bytes || !scale_bytes) return VSCAN_ERR_NULL;
    const int rc = check_cache(desc);
    if (rc != VSCAN_OK) return rc;
    *cache_bytes = (size_t)desc->n_blocks * desc->kv_heads * desc->block_size * cache_dp(desc->head_dim);
    *scale_bytes = (size_t)desc->n_blocks * desc->kv_heads * sizeof(float);
    return VSCAN_OK;
}

int vscan_cache_plan_workspace_size(const vscan_cache_desc *desc, size_t *bytes) {
    if (!bytes) return VSCAN_ERR_NULL;
    const int rc = check_cache(desc);
    if (rc != VSCAN_OK) return rc;
    *bytes = plan_needs_scratch(desc->batch, desc->n_new) ? align_up((size_t)desc->batch * 4 * sizeof(int32_t)) : 0;
    return VSCAN_OK;
}

int vscan_cache_plan(const vscan_cache_desc *desc, const int32_t *cached_len, const int32_t *new_len,
                     const int32_t *free_blocks, int32_t n_free, const int32_t *free_head,
                     int32_t *block_table, int32_t *slot_map, int32_t *kv_len,
                     int32_t *free_head_out, int32_t *missing, void *workspace,
                     size_t workspace_bytes, void *stream) {
    return finish("vscan_cache_plan",
                  cache_plan(desc, cached_len, new_len, free_blocks, n_free, free_head, block_table,
                             slot_map, kv_len, free_head_out, missing, workspace, workspace_bytes,
                             stream));
}

int vscan_cache_store(const vscan_cache_desc *desc, const void *k, const void *v,
                      const int32_t *slot_map, void *k_cache, void *v_cache, float *k_scale,
                      float *v_scale, void *stream) {
    return finish("vscan_cache_store", cache_store(desc, k, v, slot_map, k_cache, v_cache, k_scale,
                                                   v_scale, stream));
}

int vscan_cache_attend_workspace_size(const vscan_cache_desc *desc, size_t *bytes) {
    if (!bytes) return VSCAN_ERR_NULL;
    AttendPlan p;
    const int rc = plan_attend(desc, &p);
    if (rc == VSCAN_OK) *bytes = p.bytes;
    return rc;
}

int vscan_cache_attend(const vscan_cache_desc *desc, const void *q, const void *k_cache,
                       const void *v_cache, const float *k_scale, const float *v_scale,
                       const int32_t *block_table, const int32_t *kv_len, const int32_t *new_len,
                       void *out, void *workspace, size_t workspace_bytes, void *stream) {
    return finish("vscan_cache_attend",
                  cache_attend(desc, q, k_cache, v_cache, k_scale, v_scale, block_table, kv_len,
                               new_len, out, workspace, workspace_bytes, stream));
}

}  // extern "C"
