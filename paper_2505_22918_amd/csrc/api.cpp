// C ABI of librettention: host-side argument checks, then launches on the
// caller's stream.  Nothing here allocates device memory or synchronises.

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <algorithm>
#include <initializer_list>
#include <numeric>
#include <utility>

#include "../../include/rettention.h"
#include "heads.h"
#include "kernels.h"
#include "train.h"

namespace {

thread_local char g_err[512] = "";

rt_status fail(rt_status s, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof(g_err), fmt, ap);
    va_end(ap);
    return s;
}

rt_status ok() {
    g_err[0] = '\0';
    return RT_OK;
}

rt_status hip_status(hipError_t e, const char* what) {
    if (e != hipSuccess) return fail(RT_EHIP, "%s: %s", what, hipGetErrorString(e));
    return ok();
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Shape checks shared by every tensor call; sets *empty when there is no work.
rt_status check_dims(const rt_dims& d, bool* empty) {
    if (d.B < 0 || d.H < 0 || d.T < 0) return fail(RT_EINVAL, "negative dims B=%d H=%d T=%d", d.B, d.H, d.T);
    if (d.D != 64 && d.D != 72) return fail(RT_EUNSUPPORTED, "head width D=%d (supported: 64, 72)", d.D);
    const int64_t rows = (int64_t)d.B * d.H * d.T;
    if (rows * d.D >= (int64_t)1 << 40) return fail(RT_EINVAL, "tensor too large");
    if ((int64_t)d.B * d.H >= (int64_t)1 << 24) return fail(RT_EINVAL, "B*H too large");
    // buffer record counts and offsets within one head are 32-bit, with 2^30
    // kept free as the out-of-range offset that reads zeros
    if ((int64_t)d.T * d.D * 2 > (int64_t)1 << 30) return fail(RT_EINVAL, "T=%d too long for one head", d.T);
    *empty = rows == 0;
    return RT_OK;
}

rt_status check_tensor(const void* p, const char* name) {
    if (!p) return fail(RT_EINVAL, "%s is NULL", name);
    if (!aligned16(p)) return fail(RT_EINVAL, "%s is not 16-byte aligned", name);
    return RT_OK;
}

rt_status check_stat(const void* p, const char* name) {
    if (!p) return fail(RT_EINVAL, "%s is NULL", name);
    if ((reinterpret_cast<uintptr_t>(p) & 3u) != 0) return fail(RT_EINVAL, "%s is not 4-byte aligned", name);
    return RT_OK;
}

rt_status check_block(int32_t block) {
    if (block != 32 && block != 64) return fail(RT_EUNSUPPORTED, "block=%d (supported: 32, 64)", block);
    return RT_OK;
}

#define RT_TRY(expr)                  \
    do {                              \
        rt_status _s = (expr);        \
        if (_s != RT_OK) return _s;   \
    } while (0)

rt_status check_qkv(const void* q, const void* k, const void* v, void* o) {
    RT_TRY(check_tensor(q, "q"));
    RT_TRY(check_tensor(k, "k"));
    RT_TRY(check_tensor(v, "v"));
    RT_TRY(check_tensor(o, "o"));
    return RT_OK;
}

int64_t tensor_bytes(const rt_dims& d, int64_t elem) { return (int64_t)d.B * d.H * d.T * d.D * elem; }

// The byte ranges [a, a + na) and [b, b + nb) share a byte.
bool overlaps(const void* a, int64_t na, const void* b, int64_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}

// Attention outputs are written by one work item per query block while every
// work item reads K and V (and its own Q rows), so an output that overlaps an
// input would be read back by other work items; no overlap is accepted.
rt_status check_no_overlap(const void* out, int64_t out_bytes, const char* out_name,
                           std::initializer_list<std::pair<const void*, int64_t>> ins, const char* in_names) {
    for (const auto& in : ins)
        if (in.first && overlaps(out, out_bytes, in.first, in.second))
            return fail(RT_EINVAL, "%s overlaps %s (outputs must not alias the inputs)", out_name, in_names);
    return RT_OK;
}

// Optional row statistics: they must not overlap each other, o or the other
// listed buffers.
rt_status check_stats_overlap(const rt_dims& d, const float* row_max, const float* row_sum, const void* o,
                              std::initializer_list<std::pair<const void*, int64_t>> others) {
    const int64_t ns = tensor_bytes(d, 4) / d.D, nt = tensor_bytes(d, 2);
    for (const float* st : {row_max, row_sum}) {
        if (!st) continue;
        RT_TRY(check_no_overlap(st, ns, "row_max / row_sum", {{o, nt}}, "o"));
        RT_TRY(check_no_overlap(st, ns, "row_max / row_sum", others, "another output or input"));
    }
    if (row_max && row_sum && overlaps(row_max, ns, row_sum, ns))
        return fail(RT_EINVAL, "row_max overlaps row_sum");
    return RT_OK;
}

rt::AttnArgs base_args(const void* q, const void* k, const void* v, const rt_dims& d, int32_t block,
                       void* o, float* row_max, float* row_sum) {
    rt::AttnArgs a{};
    a.q = static_cast<const uint16_t*>(q);
    a.k = static_cast<const uint16_t*>(k);
    a.v = static_cast<const uint16_t*>(v);
    a.o = static_cast<uint16_t*>(o);
    a.row_max = row_max;
    a.row_sum = row_sum;
    a.stat_stride = 1;
    a.T = d.T;
    a.n_blk = (int32_t)ceil_div(d.T, block);
    const int64_t items = (int64_t)d.B * d.H * a.n_blk;
    a.n_items = (int32_t)items;
    a.per_xcd = (int32_t)ceil_div(items, 8);
    a.scale_nat = (float)(1.0 / std::sqrt((double)d.D));
    a.scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)d.D));
    return a;
}

rt_status check_items(const rt_dims& d, int32_t block) {
    const int64_t items = (int64_t)d.B * d.H * ceil_div(d.T, block);
    if (8 * ceil_div(items, 8) > INT32_MAX) return fail(RT_EINVAL, "too many query blocks");
    return RT_OK;
}

rt_status check_bsr(const rt_bsr* m, const rt_dims& d) {
    if (!m) return fail(RT_EINVAL, "mask is NULL");
    RT_TRY(check_block(m->block));
    const int64_t nb = ceil_div(d.T, m->block);
    if (m->n_qblk != nb) return fail(RT_EINVAL, "n_qblk=%d but ceil(T/block)=%lld", m->n_qblk, (long long)nb);
    if (m->nnz < 0) return fail(RT_EINVAL, "nnz=%d", m->nnz);
    if (nb > 0 && m->nnz == 0) return fail(RT_EINVAL, "empty mask: every query block needs a kept key block (Eq.5)");
    if (nb > 0 && (!m->row_ptr || !m->col_idx)) return fail(RT_EINVAL, "row_ptr / col_idx is NULL");
    const int64_t bh = (int64_t)d.B * d.H;
    if (m->n_masks != 0 && m->n_masks != 1 && m->n_masks != d.H && m->n_masks != bh)
        return fail(RT_EINVAL, "n_masks=%d (need 1, H=%d or B*H=%lld)", m->n_masks, d.H, (long long)bh);
    return RT_OK;
}

void set_mask(rt::AttnArgs& a, const rt_bsr* m, const rt_dims& d) {
    a.row_ptr = m->row_ptr;
    a.col_idx = m->col_idx;
    a.nnz = m->nnz;
    a.n_masks = m->n_masks > 1 ? m->n_masks : 1;
    a.heads = d.H;
}

int64_t lcm64(int64_t a, int64_t b) { return a / std::gcd(a, b) * b; }

// Validates a pattern and fills the launch arguments (mask and outputs aside).
rt_status pattern_args(const rt_pattern* p, int32_t T, int32_t block, rt::IndexArgs* out, int64_t* nnz) {
    if (!p) return fail(RT_EINVAL, "pattern is NULL");
    RT_TRY(check_block(block));
    if (T < 1) return fail(RT_EINVAL, "T=%d (need T >= 1)", T);
    const int64_t nb = ceil_div(T, block);
    if (nb > 4096) return fail(RT_EUNSUPPORTED, "ceil(T/block)=%lld exceeds 4096 blocks", (long long)nb);
    rt::IndexArgs a{};
    a.kind = p->kind;
    a.T = T;
    a.block = block;
    a.n_blk = (int32_t)nb;
    a.keep = p->keep;
    a.lcm = 1;
    if (p->n_masks < 0) return fail(RT_EINVAL, "n_masks=%d", p->n_masks);
    a.n_masks = p->n_masks > 1 ? p->n_masks : 1;
    if (a.n_masks > 1 && p->kind != RT_PAT_EXPLICIT)
        return fail(RT_EINVAL, "n_masks=%d: the window patterns are the same for every head", p->n_masks);
    if (a.n_masks > 1 && (int64_t)a.n_masks * nb > 32768)
        return fail(RT_EUNSUPPORTED, "n_masks * ceil(T/block) = %lld exceeds 32768",
                    (long long)a.n_masks * nb);
    switch (p->kind) {
        case RT_PAT_EXPLICIT:
            *nnz = -1;
            break;
        case RT_PAT_LOCAL2D: {
            if (p->grid_h < 1 || p->grid_w < 1 || p->grid_h > 65535 || p->grid_w > 65535)
                return fail(RT_EINVAL, "grid %dx%d out of range", p->grid_h, p->grid_w);
            if ((int64_t)p->grid_h * p->grid_w != T)
                return fail(RT_EINVAL, "grid_h*grid_w=%lld != T=%d", (long long)p->grid_h * p->grid_w, T);
            if (p->keep < 1) return fail(RT_EINVAL, "keep=%d (need >= 1)", p->keep);
            a.grid_h = p->grid_h;
            a.grid_w = p->grid_w;
            const int64_t last = T - (nb - 1) * block;
            a.lcm = nb > 1 ? lcm64(block, last) : last;
            *nnz = nb * std::min<int64_t>(p->keep, nb);
            break;
        }
        case RT_PAT_VIDEO3D: {
            if (p->grid_h < 1 || p->grid_w < 1 || p->frames < 1 || p->grid_h > 65535 || p->grid_w > 65535 ||
                p->frames > 65535 || p->n_text < 0)
                return fail(RT_EINVAL, "video grid %dx%dx%d / n_text=%d out of range", p->frames, p->grid_h,
                            p->grid_w, p->n_text);
            if ((int64_t)p->n_text + (int64_t)p->frames * p->grid_h * p->grid_w != T)
                return fail(RT_EINVAL, "n_text + frames*grid_h*grid_w != T=%d", T);
            if (p->keep < 1) return fail(RT_EINVAL, "keep=%d (need >= 1)", p->keep);
            a.grid_h = p->grid_h;
            a.grid_w = p->grid_w;
            a.frames = p->frames;
            a.n_text = p->n_text;
            const int64_t ntb = ceil_div(p->n_text, block);
            a.n_tblk = (int32_t)ntb;
            const int64_t nv = nb - ntb;
            if (nv >= 1) {
                const int64_t last = T - (nb - 1) * block;
                a.lcm = nv > 1 ? lcm64(block, last) : last;
            }
            *nnz = ntb * ntb + (nb - ntb) * (ntb + std::min<int64_t>(p->keep, nv));
            break;
        }
        default:
            return fail(RT_EINVAL, "unknown pattern kind %d", p->kind);
    }
    *out = a;
    return RT_OK;
}

}  // namespace

extern "C" {

const char* rt_status_str(rt_status s) {
    switch (s) {
        case RT_OK: return "ok";
        case RT_EINVAL: return "invalid argument";
        case RT_EUNSUPPORTED: return "unsupported configuration";
        case RT_ECAPACITY: return "output capacity too small";
        case RT_EHIP: return "HIP runtime error";
    }
    return "unknown status";
}

const char* rt_last_error(void) { return g_err; }

int32_t rt_version(void) { return 100; }

rt_status rt_index_size(const rt_pattern* pattern, int32_t T, int32_t block, int32_t* nnz_out) {
    if (!nnz_out) return fail(RT_EINVAL, "nnz_out is NULL");
    rt::IndexArgs a{};
    int64_t nnz = 0;
    RT_TRY(pattern_args(pattern, T, block, &a, &nnz));
    if (pattern->kind == RT_PAT_EXPLICIT) {
        if (!pattern->host_mask) return fail(RT_EINVAL, "EXPLICIT pattern needs host_mask for sizing");
        nnz = 0;
        const int64_t rows = (int64_t)a.n_masks * a.n_blk;
        for (int64_t r = 0; r < rows; ++r) {
            const uint8_t* row = pattern->host_mask + r * a.n_blk;
            int64_t kept = 0;
            for (int64_t j = 0; j < a.n_blk; ++j) kept += row[j] != 0;
            // Eq.5 normalises over the kept keys: an empty kept set has no softmax
            if (kept == 0)
                return fail(RT_EINVAL, "mask %lld, query block %lld keeps no key block (Eq.5 needs one)",
                            (long long)(r / a.n_blk), (long long)(r % a.n_blk));
            nnz += kept;
        }
    }
    if (nnz > INT32_MAX) return fail(RT_EINVAL, "nnz exceeds int32");
    *nnz_out = (int32_t)nnz;
    return ok();
}

rt_status rt_index_build(const rt_pattern* pattern, int32_t T, int32_t block, int32_t* row_ptr,
                         int32_t* col_idx, int32_t capacity, void* stream) {
    rt::IndexArgs a{};
    int64_t nnz = 0;
    RT_TRY(pattern_args(pattern, T, block, &a, &nnz));
    if (!row_ptr || !col_idx) return fail(RT_EINVAL, "row_ptr / col_idx is NULL");
    if (capacity < 0) return fail(RT_EINVAL, "capacity=%d", capacity);
    if (pattern->kind == RT_PAT_EXPLICIT) {
        if (!pattern->mask) return fail(RT_EINVAL, "EXPLICIT pattern needs a device mask");
        if (pattern->host_mask) {
            int32_t need = 0;
            RT_TRY(rt_index_size(pattern, T, block, &need));
            nnz = need;
        }
    }
    if (nnz >= 0 && capacity < nnz)
        return fail(RT_ECAPACITY, "capacity=%d but the mask has %lld entries", capacity, (long long)nnz);
    a.mask = pattern->mask;
    a.row_ptr = row_ptr;
    a.col_idx = col_idx;
    a.capacity = capacity;
    return hip_status(rt::launch_index_build(a, static_cast<hipStream_t>(stream)), "index build launch");
}

rt_status rt_bsr_check(const rt_bsr* mask, const int32_t* host_row_ptr, const int32_t* host_col_idx) {
    if (!mask) return fail(RT_EINVAL, "mask is NULL");
    RT_TRY(check_block(mask->block));
    if (mask->n_qblk < 0 || mask->nnz < 0 || mask->n_masks < 0)
        return fail(RT_EINVAL, "n_qblk=%d nnz=%d n_masks=%d", mask->n_qblk, mask->nnz, mask->n_masks);
    const int64_t nb = mask->n_qblk, nm = mask->n_masks > 1 ? mask->n_masks : 1;
    if (nb == 0) return mask->nnz == 0 ? ok() : fail(RT_EINVAL, "nnz=%d for a mask without rows", mask->nnz);
    if (!host_row_ptr || !host_col_idx) return fail(RT_EINVAL, "host_row_ptr / host_col_idx is NULL");
    int64_t last = 0;
    for (int64_t m = 0; m < nm; ++m) {
        const int32_t* rp = host_row_ptr + m * (nb + 1);
        for (int64_t i = 0; i < nb; ++i) {
            if (rp[i] < 0 || rp[i + 1] > mask->nnz)
                return fail(RT_EINVAL, "mask %lld row %lld: offsets [%d, %d) outside [0, nnz=%d]", (long long)m,
                            (long long)i, rp[i], rp[i + 1], mask->nnz);
            // Eq.5 normalises over the kept keys: an empty kept set has no softmax
            if (rp[i + 1] <= rp[i])
                return fail(RT_EINVAL, "mask %lld, query block %lld keeps no key block (Eq.5 needs one)",
                            (long long)m, (long long)i);
            for (int32_t e = rp[i]; e < rp[i + 1]; ++e) {
                const int32_t c = host_col_idx[e];
                if (c < 0 || c >= nb)
                    return fail(RT_EINVAL, "mask %lld row %lld: key block %d outside [0, %lld)", (long long)m,
                                (long long)i, c, (long long)nb);
                if (e > rp[i] && c <= host_col_idx[e - 1])
                    return fail(RT_EINVAL, "mask %lld row %lld: key blocks not strictly ascending", (long long)m,
                                (long long)i);
            }
        }
        last = std::max<int64_t>(last, rp[nb]);
    }
    if (last != mask->nnz)
        return fail(RT_EINVAL, "nnz=%d but the row offsets end at %lld", mask->nnz, (long long)last);
    return ok();
}

namespace {

// Shape checks of the dynamic index build; fills the counts it needs.
rt_status dynamic_shape(const rt_dims& dims, int32_t block, int32_t keep, int64_t* n_blk, int64_t* kk,
                        int64_t* nnz, int64_t* ws_bytes) {
    bool empty = false;
    RT_TRY(check_dims(dims, &empty));
    RT_TRY(check_block(block));
    if (keep < 1) return fail(RT_EINVAL, "keep=%d (need >= 1)", keep);
    const int64_t nb = ceil_div(dims.T, block);
    if (nb > 4096) return fail(RT_EUNSUPPORTED, "ceil(T/block)=%lld exceeds 4096 blocks", (long long)nb);
    const int64_t bh = (int64_t)dims.B * dims.H;
    *n_blk = nb;
    *kk = std::min<int64_t>(keep, nb);
    *nnz = bh * nb * *kk;
    if (*nnz > INT32_MAX || bh * (nb + 1) > INT32_MAX) return fail(RT_EINVAL, "mask too large for int32 offsets");
    *ws_bytes = 2 * bh * nb * dims.D * (int64_t)sizeof(float);
    return RT_OK;
}

}  // namespace

rt_status rt_dynamic_index_workspace(rt_dims dims, int32_t block, int32_t keep, int64_t* bytes) {
    if (!bytes) return fail(RT_EINVAL, "bytes is NULL");
    int64_t nb, kk, nnz, ws;
    RT_TRY(dynamic_shape(dims, block, keep, &nb, &kk, &nnz, &ws));
    *bytes = ws;
    return ok();
}

rt_status rt_dynamic_index_noalloc(const void* q, const void* k, rt_dims dims, int32_t block, int32_t keep,
                                   int32_t* row_ptr, int32_t* col_idx, int32_t capacity, void* stream) {
    int64_t nb, kk, nnz, ws;
    RT_TRY(dynamic_shape(dims, block, keep, &nb, &kk, &nnz, &ws));
    if (ws > rt::kDynScratchFloats * (int64_t)sizeof(float))
        return fail(RT_ECAPACITY, "the shape needs %lld workspace bytes, the allocation-free build holds %lld",
                    (long long)ws, (long long)(rt::kDynScratchFloats * (int64_t)sizeof(float)));
    if ((int64_t)dims.B * dims.H * dims.T == 0) return ok();
    float* scratch = nullptr;
    RT_TRY(hip_status(rt::dynamic_scratch(&scratch), "workspace address"));
    return rt_dynamic_index(q, k, dims, block, keep, row_ptr, col_idx, capacity, scratch, ws, stream);
}

rt_status rt_dynamic_index(const void* q, const void* k, rt_dims dims, int32_t block, int32_t keep,
                           int32_t* row_ptr, int32_t* col_idx, int32_t capacity, void* workspace,
                           int64_t workspace_bytes, void* stream) {
    int64_t nb, kk, nnz, ws;
    RT_TRY(dynamic_shape(dims, block, keep, &nb, &kk, &nnz, &ws));
    if ((int64_t)dims.B * dims.H * dims.T == 0) return ok();
    RT_TRY(check_tensor(q, "q"));
    RT_TRY(check_tensor(k, "k"));
    RT_TRY(check_stat(row_ptr, "row_ptr"));
    RT_TRY(check_stat(col_idx, "col_idx"));
    RT_TRY(check_tensor(workspace, "workspace"));
    if (capacity < nnz)
        return fail(RT_ECAPACITY, "capacity=%d but the mask has %lld entries", capacity, (long long)nnz);
    if (workspace_bytes < ws)
        return fail(RT_ECAPACITY, "workspace of %lld bytes, %lld needed", (long long)workspace_bytes, (long long)ws);
    const int64_t nt = tensor_bytes(dims, 2);
    const int64_t nrp = (int64_t)dims.B * dims.H * (nb + 1) * 4, nci = nnz * 4;
    RT_TRY(check_no_overlap(row_ptr, nrp, "row_ptr", {{q, nt}, {k, nt}, {col_idx, nci}, {workspace, ws}},
                            "q, k, col_idx or the workspace"));
    RT_TRY(check_no_overlap(col_idx, nci, "col_idx", {{q, nt}, {k, nt}, {workspace, ws}}, "q, k or the workspace"));
    RT_TRY(check_no_overlap(workspace, ws, "workspace", {{q, nt}, {k, nt}}, "q or k"));
    rt::DynIndexArgs a{};
    a.q = static_cast<const uint16_t*>(q);
    a.k = static_cast<const uint16_t*>(k);
    a.B = dims.B;
    a.H = dims.H;
    a.T = dims.T;
    a.D = dims.D;
    a.block = block;
    a.n_blk = (int32_t)nb;
    a.keep = keep;
    a.qsum = static_cast<float*>(workspace);
    a.kmean = a.qsum + (size_t)dims.B * dims.H * nb * dims.D;
    a.row_ptr = row_ptr;
    a.col_idx = col_idx;
    return hip_status(rt::launch_dynamic_index(a, static_cast<hipStream_t>(stream)), "dynamic index launch");
}

rt_status rt_attn_full(const void* q, const void* k, const void* v, rt_dims dims, int32_t block, void* o,
                       float* row_max, float* row_sum, void* stream) {
    bool empty = false;
    RT_TRY(check_dims(dims, &empty));
    RT_TRY(check_block(block));
    if (empty) return ok();
    RT_TRY(check_qkv(q, k, v, o));
    if (row_max) RT_TRY(check_stat(row_max, "row_max"));
    if (row_sum) RT_TRY(check_stat(row_sum, "row_sum"));
    const int64_t nt = tensor_bytes(dims, 2);
    RT_TRY(check_no_overlap(o, nt, "o", {{q, nt}, {k, nt}, {v, nt}}, "q, k or v"));
    RT_TRY(check_stats_overlap(dims, row_max, row_sum, o, {}));
    RT_TRY(check_items(dims, block));
    rt::AttnArgs a = base_args(q, k, v, dims, block, o, row_max, row_sum);
    a.dense = 1;
    return hip_status(rt::launch_attention(a, dims.D, block, rt::kAttn, static_cast<hipStream_t>(stream)),
                      "full attention launch");
}

rt_status rt_attn_sparse(const void* q, const void* k, const void* v, rt_dims dims, const rt_bsr* mask,
                         void* o, float* row_max, float* row_sum, void* stream) {
    bool empty = false;
    RT_TRY(check_dims(dims, &empty));
    RT_TRY(check_bsr(mask, dims));
    if (empty) return ok();
    RT_TRY(check_qkv(q, k, v, o));
    if (row_max) RT_TRY(check_stat(row_max, "row_max"));
    if (row_sum) RT_TRY(check_stat(row_sum, "row_sum"));
    const int64_t nt = tensor_bytes(dims, 2);
    RT_TRY(check_no_overlap(o, nt, "o", {{q, nt}, {k, nt}, {v, nt}}, "q, k or v"));
    RT_TRY(check_stats_overlap(dims, row_max, row_sum, o, {}));
    RT_TRY(check_items(dims, mask->block));
    rt::AttnArgs a = base_args(q, k, v, dims, mask->block, o, row_max, row_sum);
    set_mask(a, mask, dims);
    return hip_status(rt::launch_attention(a, dims.D, mask->block, rt::kAttn, static_cast<hipStream_t>(stream)),
                      "sparse attention launch");
}

rt_status rt_attn_cache(const void* q, const void* k, const void* v, rt_dims dims, const rt_bsr* mask, void* o,
                        float* row_max, float* row_sum, float* rho, void* resid, void* stream) {
    bool empty = false;
    RT_TRY(check_dims(dims, &empty));
    RT_TRY(check_bsr(mask, dims));
    if (empty) return ok();
    RT_TRY(check_qkv(q, k, v, o));
    if (rho) RT_TRY(check_stat(rho, "rho"));
    RT_TRY(check_tensor(resid, "resid"));
    if (row_max) RT_TRY(check_stat(row_max, "row_max"));
    if (row_sum) RT_TRY(check_stat(row_sum, "row_sum"));
    const int64_t nt = tensor_bytes(dims, 2), ns = tensor_bytes(dims, 4) / dims.D;
    RT_TRY(check_no_overlap(o, nt, "o", {{q, nt}, {k, nt}, {v, nt}, {resid, nt}}, "q, k, v or resid"));
    RT_TRY(check_no_overlap(resid, nt, "resid", {{q, nt}, {k, nt}, {v, nt}}, "q, k or v"));
    if (rho)
        RT_TRY(check_no_overlap(rho, ns, "rho", {{q, nt}, {k, nt}, {v, nt}, {o, nt}, {resid, nt}},
                                "q, k, v, o or resid"));
    RT_TRY(check_stats_overlap(dims, row_max, row_sum, o, {{resid, nt}, {rho, ns}}));
    RT_TRY(check_items(dims, mask->block));
    rt::AttnArgs a = base_args(q, k, v, dims, mask->block, o, row_max, row_sum);
    set_mask(a, mask, dims);
    a.rho_out = rho;
    a.resid_out = static_cast<uint16_t*>(resid);
    return hip_status(rt::launch_attention(a, dims.D, mask->block, rt::kAttnCache, static_cast<hipStream_t>(stream)),
                      "caching-step launch");
}

rt_status rt_attn_postmask(const void* q, const void* k, const void* v, rt_dims dims, const rt_bsr* mask, void* o,
                           void* stream) {
    bool empty = false;
    RT_TRY(check_dims(dims, &empty));
    RT_TRY(check_bsr(mask, dims));
    if (empty) return ok();
    RT_TRY(check_qkv(q, k, v, o));
    const int64_t nt = tensor_bytes(dims, 2);
    RT_TRY(check_no_overlap(o, nt, "o", {{q, nt}, {k, nt}, {v, nt}}, "q, k or v"));
    RT_TRY(check_items(dims, mask->block));
    rt::AttnArgs a = base_args(q, k, v, dims, mask->block, o, nullptr, nullptr);
    set_mask(a, mask, dims);
    a.postmask = 1;
    return hip_status(rt::launch_attention(a, dims.D, mask->block, rt::kAttnCache, static_cast<hipStream_t>(stream)),
                      "post-softmax masking launch");
}

rt_status rt_cache_build(const void* o_full, const float* m_full, const float* l_full, const void* o_sparse,
                         const float* m_sparse, const float* l_sparse, rt_dims dims, float* rho, void* resid,
                         void* stream) {
    bool empty = false;
    RT_TRY(check_dims(dims, &empty));
    if (empty) return ok();
    RT_TRY(check_tensor(o_full, "o_full"));
    RT_TRY(check_tensor(o_sparse, "o_sparse"));
    RT_TRY(check_tensor(resid, "resid"));
    if (rho) {  // without a ratio the statistics are not read
        RT_TRY(check_stat(m_full, "m_full"));
        RT_TRY(check_stat(l_full, "l_full"));
        RT_TRY(check_stat(m_sparse, "m_sparse"));
        RT_TRY(check_stat(l_sparse, "l_sparse"));
        RT_TRY(check_stat(rho, "rho"));
    }
    {
        const int64_t nt = tensor_bytes(dims, 2), ns = tensor_bytes(dims, 4) / dims.D;
        const std::initializer_list<std::pair<const void*, int64_t>> ins = {
            {o_full, nt}, {o_sparse, nt}, {m_full, ns}, {l_full, ns}, {m_sparse, ns}, {l_sparse, ns}};
        RT_TRY(check_no_overlap(resid, nt, "resid", ins, "an input"));
        if (rho) {
            RT_TRY(check_no_overlap(rho, ns, "rho", ins, "an input"));
            RT_TRY(check_no_overlap(rho, ns, "rho", {{resid, nt}}, "resid"));
        }
    }
    const int64_t rows = (int64_t)dims.B * dims.H * dims.T;
    if (!rho) m_full = l_full = m_sparse = l_sparse = nullptr;
    return hip_status(rt::launch_cache_build(static_cast<const uint16_t*>(o_full), m_full, l_full,
                                             static_cast<const uint16_t*>(o_sparse), m_sparse, l_sparse, rows,
                                             dims.D, rho, static_cast<uint16_t*>(resid),
                                             static_cast<hipStream_t>(stream)),
                      "cache build launch");
}

rt_status rt_attn_sparse_reshape(const void* q, const void* k, const void* v, rt_dims dims, const rt_bsr* mask,
                                 const float* rho, const void* resid, float rho_delta, void* o, float* row_max,
                                 float* row_sum, void* stream) {
    bool empty = false;
    RT_TRY(check_dims(dims, &empty));
    RT_TRY(check_bsr(mask, dims));
    if (!std::isfinite(rho_delta)) return fail(RT_EINVAL, "rho_delta is not finite");
    if (empty) return ok();
    RT_TRY(check_qkv(q, k, v, o));
    if (rho) RT_TRY(check_stat(rho, "rho"));
    RT_TRY(check_tensor(resid, "resid"));
    if (row_max) RT_TRY(check_stat(row_max, "row_max"));
    if (row_sum) RT_TRY(check_stat(row_sum, "row_sum"));
    const int64_t nt = tensor_bytes(dims, 2), ns = tensor_bytes(dims, 4) / dims.D;
    RT_TRY(check_no_overlap(o, nt, "o", {{q, nt}, {k, nt}, {v, nt}, {resid, nt}, {rho, ns}},
                            "q, k, v, resid or rho"));
    RT_TRY(check_stats_overlap(dims, row_max, row_sum, o, {{resid, nt}, {rho, ns}}));
    RT_TRY(check_items(dims, mask->block));
    rt::AttnArgs a = base_args(q, k, v, dims, mask->block, o, row_max, row_sum);
    set_mask(a, mask, dims);
    a.rho = rho;
    a.resid = static_cast<const uint16_t*>(resid);
    a.rho_delta = rho_delta;
    return hip_status(rt::launch_attention(a, dims.D, mask->block, rt::kAttnReshape, static_cast<hipStream_t>(stream)),
                      "sparse+reshape launch");
}

rt_status rt_reshape_apply(const void* o_sparse, const float* rho, const void* resid, float rho_delta,
                           rt_dims dims, void* o, void* stream) {
    bool empty = false;
    RT_TRY(check_dims(dims, &empty));
    if (!std::isfinite(rho_delta)) return fail(RT_EINVAL, "rho_delta is not finite");
    if (empty) return ok();
    RT_TRY(check_tensor(o_sparse, "o_sparse"));
    RT_TRY(check_tensor(resid, "resid"));
    RT_TRY(check_tensor(o, "o"));
    if (rho) RT_TRY(check_stat(rho, "rho"));
    {
        const int64_t nt = tensor_bytes(dims, 2), ns = tensor_bytes(dims, 4) / dims.D;
        RT_TRY(check_no_overlap(o, nt, "o", {{o_sparse, nt}, {resid, nt}, {rho, ns}}, "o_sparse, resid or rho"));
    }
    const int64_t rows = (int64_t)dims.B * dims.H * dims.T;
    return hip_status(rt::launch_reshape_apply(static_cast<const uint16_t*>(o_sparse), rho,
                                               static_cast<const uint16_t*>(resid), rho_delta, rows, dims.D,
                                               static_cast<uint16_t*>(o), static_cast<hipStream_t>(stream)),
                      "reshape launch");
}

// ---- training ----------------------------------------------------------------------------

namespace {

// A transposed mask against the mask it belongs to.
rt_status check_transposed(const rt_bsr* t, const rt_bsr* m) {
    if (!t) return fail(RT_EINVAL, "the transposed mask is NULL");
    const int32_t nm = m->n_masks > 1 ? m->n_masks : 1, nt = t->n_masks > 1 ? t->n_masks : 1;
    if (t->block != m->block || t->n_qblk != m->n_qblk || nt != nm)
        return fail(RT_EINVAL, "the transposed mask (block=%d n_qblk=%d n_masks=%d) is not of this mask (%d, %d, %d)",
                    t->block, t->n_qblk, nt, m->block, m->n_qblk, nm);
    if (t->nnz < m->nnz)
        return fail(RT_ECAPACITY, "the transposed mask has room for %d entries, the mask has %d", t->nnz, m->nnz);
    RT_TRY(check_stat(t->row_ptr, "the transposed mask's row_ptr"));
    RT_TRY(check_tensor(t->col_idx, "the transposed mask's col_idx"));
    return RT_OK;
}

// How the lists of a transposed mask with room for `entries` are split over workgroups, so that no long one (a text
// block's, which all query blocks keep, or one that all score well) holds a call up: after `seg` entries, twice the mean
// list and 16 at least, in masks of more than 40 blocks; and what the plan and the parts of split lists take at most.
// Where nothing turns out to be split, that the plan could be costs a launch for the sums.  Gradients of 12 heads, each
// with a mask of its own, new in each call, unsplit and by this rule: 83 blocks with random lists 58.1 and 63.2 us, with
// one block that all queries keep 142 and 72, dynamic masks 159 and 77; 55 blocks 39.9 and 42.5, 94 and 51.  Up to 40
// blocks splitting would cost 2 us without such a block (32 blocks 21.1 and 23.0) and gain up to 20 with one (59 and
// 38; 24 blocks 38 and 32); the masks of images of that size hold none.
struct Plan {
    int32_t seg, max_more, max_base;  // entries of a part; parts beyond the first ones, and numbers of parts, at most
    int64_t first, values;  // the plan's place behind the entries, and the size of it all
    int32_t fold = 1, max_slots = 0;  // of a gradient call
};

rt_status plan_of(const rt_bsr* m, int32_t entries, Plan* out) {
    const int64_t rows = (int64_t)(m->n_masks > 1 ? m->n_masks : 1) * m->n_qblk;
    const int64_t seg = m->n_qblk <= 40 ? std::max(m->n_qblk, 1)
                                        : std::max<int64_t>(16, 2 * ceil_div(entries, std::max<int64_t>(rows, 1)));
    const int64_t splits = m->n_qblk > seg ? entries / seg : 0;
    // the plan's int32 places, and a wave for each row in a launch of less than 2^32 threads
    if (rows + 2 * splits > INT32_MAX / 8 || rows >= (int64_t)1 << 26) return fail(RT_EINVAL, "too many mask rows");
    out->seg = (int32_t)seg;
    out->max_more = (int32_t)splits;
    out->max_base = (int32_t)(2 * splits);
    out->first = ceil_div(entries, 4) * 4;
    out->values = out->first + 4 * (rows + 2 * splits);
    return RT_OK;
}

// How many parts a workgroup of the gradient call takes together: as many as keep a list's share below what each of
// the workgroups that run at once (six to a CU) walks in the call.  Fewer cost more sums than they gain, more hold the
// call up: CogVideoX-2B with two samples (four text blocks kept by all 278) 630 us and 22 for the sums with parts of 36
// entries, 595 and 9.5 with 96; one head of it, all in all, 66 us in parts of 36, 53 in parts of 16 and 139 of 96.
void fold_parts(const rt_dims& d, const rt_bsr* m, Plan* p) {
    const int64_t kept = (int64_t)d.B * d.H / (m->n_masks > 1 ? m->n_masks : 1) * m->nnz;
    p->fold = (int32_t)std::max<int64_t>(1, std::min(kept / 1536 / p->seg, ceil_div(m->n_qblk, p->seg)));
    if ((int64_t)p->fold * p->seg >= m->n_qblk)  // no list is longer
        p->max_more = p->max_slots = 0;
    else
        p->max_slots = p->fold > 1 ? 2 * p->max_base / p->fold : p->max_base;
}

int64_t mask_ptr_bytes(const rt_bsr* m) {
    return (int64_t)(m->n_masks > 1 ? m->n_masks : 1) * ((int64_t)m->n_qblk + 1) * 4;
}

typedef std::pair<const void*, int64_t> range;

// No output overlaps an input or another output.
rt_status check_ranges(std::initializer_list<std::pair<range, const char*>> outs, std::initializer_list<range> ins) {
    for (auto o = outs.begin(); o != outs.end(); ++o) {
        if (!o->first.first) continue;
        RT_TRY(check_no_overlap(o->first.first, o->first.second, o->second, ins, "an input"));
        for (auto p = outs.begin(); p != o; ++p)
            if (p->first.first && overlaps(o->first.first, o->first.second, p->first.first, p->first.second))
                return fail(RT_EINVAL, "%s overlaps %s", o->second, p->second);
    }
    return RT_OK;
}

int32_t whole64(int32_t T) { return (int32_t)ceil_div(T, 64) * 64; }

// Workgroups that share the walk of a tile of dense gradients.  Where there are few tiles, as many as fill the CUs once
// (a tile has two walks; twice where they are 64 stages of 64 rows and more), each with 4 stages at least, if that takes
// the time of 8 stages, about a microsecond each, off a walk: the sums are a launch of their own.  One head of 1175
// tokens 26 -> 19 us, of 2734 50 -> 27 (30 with two workgroups to a CU), two of 8192 141 -> 127.
int32_t dense_split(const rt_dims& d) {
    const int64_t n = (int64_t)d.B * d.H * ceil_div(d.T, rt::kDenseRows), stages = ceil_div(d.T, 64);
    const int64_t s = std::min((stages >= 64 ? 256 : 128) / std::max<int64_t>(n, 1), stages / 4);
    return s > 1 && stages - ceil_div(stages, s) >= 8 ? (int32_t)s : 1;
}

// Row values, and the parts of split lists or walks.
int64_t backward_workspace(const rt_dims& d, const rt_bsr* m, const Plan& p) {
    const int64_t bh = (int64_t)d.B * d.H, values = bh * whole64(d.T) * 8;
    if (m) return values + bh / (m->n_masks > 1 ? m->n_masks : 1) * p.max_slots * 2 * m->block * d.D * 4;
    const int64_t split = dense_split(d);
    return values + (split > 1 ? split * bh * ceil_div(d.T, rt::kDenseRows) * 3 * rt::kDenseRows * d.D * 4 : 0);
}

// What the dense and the sparse gradient call check and set alike (rho and the mask aside).
rt_status grad_args(const void* q, const void* k, const void* v, const void* o, const float* row_max,
                    const float* row_sum, const void* d_o, const rt_dims& d, void* dq, void* dk, void* dv,
                    void* workspace, int64_t workspace_bytes, int64_t need, rt::GradArgs* out) {
    RT_TRY(check_qkv(q, k, v, const_cast<void*>(o)));
    RT_TRY(check_tensor(d_o, "d_o"));
    RT_TRY(check_stat(row_max, "row_max"));
    RT_TRY(check_stat(row_sum, "row_sum"));
    RT_TRY(check_tensor(dq, "dq"));
    RT_TRY(check_tensor(dk, "dk"));
    RT_TRY(check_tensor(dv, "dv"));
    RT_TRY(check_tensor(workspace, "workspace"));
    if (workspace_bytes < need)
        return fail(RT_ECAPACITY, "workspace of %lld bytes, %lld needed", (long long)workspace_bytes, (long long)need);
    if ((int64_t)d.B * d.H * whole64(d.T) >= (int64_t)1 << 29)  // 8 threads a row, in one launch
        return fail(RT_EINVAL, "too many rows: B=%d H=%d T=%d", d.B, d.H, d.T);
    rt::GradArgs a{};
    a.q = static_cast<const uint16_t*>(q);
    a.k = static_cast<const uint16_t*>(k);
    a.v = static_cast<const uint16_t*>(v);
    a.o = static_cast<const uint16_t*>(o);
    a.d_o = static_cast<const uint16_t*>(d_o);
    a.row_max = row_max;
    a.row_sum = row_sum;
    a.dq = static_cast<uint16_t*>(dq);
    a.dk = static_cast<uint16_t*>(dk);
    a.dv = static_cast<uint16_t*>(dv);
    a.row_vals = static_cast<float*>(workspace);
    a.T64 = whole64(d.T);
    a.T = d.T;
    a.heads = d.H;
    a.n_bh = d.B * d.H;
    a.scale_nat = (float)(1.0 / std::sqrt((double)d.D));
    a.scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)d.D));
    *out = a;
    return RT_OK;
}

int64_t type_bytes(int32_t type) { return type == RT_F32 ? 4 : 2; }

// Shape checks of the norm calls; *rows may come out 0.
rt_status check_norm(const rt_norm_dims& d, int64_t* rows) {
    if (d.n0 < 0 || d.n1 < 0 || d.n2 < 0) return fail(RT_EINVAL, "negative dims n0=%d n1=%d n2=%d", d.n0, d.n1, d.n2);
    if (d.type != RT_BF16 && d.type != RT_F16 && d.type != RT_F32) return fail(RT_EUNSUPPORTED, "type=%d", d.type);
    if (d.weight_type != d.type && d.weight_type != RT_F32)
        return fail(RT_EUNSUPPORTED, "weight_type=%d (supported: fp32, or the rows' type)", d.weight_type);
    if (d.width < 1) return fail(RT_EINVAL, "width=%d (need >= 1)", d.width);
    if (d.width > 16384) return fail(RT_EUNSUPPORTED, "width=%d (supported: up to 16384)", d.width);
    if (d.weight_sets != 1 && d.weight_sets != d.n0)
        return fail(RT_EINVAL, "weight_sets=%d (need 1 or n0=%d)", d.weight_sets, d.n0);
    if (d.weight_sets > 65535) return fail(RT_EUNSUPPORTED, "weight_sets=%d (supported: up to 65535)", d.weight_sets);
    const int64_t n01 = (int64_t)d.n0 * d.n1;
    if (n01 > INT32_MAX || n01 * d.n2 > INT32_MAX) return fail(RT_EINVAL, "n0 * n1 * n2 must be below 2^31");
    *rows = n01 * d.n2;
    return RT_OK;
}

// Checks the rows of one tensor: alignment to its elements, strides that stay within 2^48 elements.  Writes the byte
// span from its first to its last element; distinct: no two rows may share memory (outputs).
rt_status check_rows(const void* p, const int64_t stride[3], const rt_norm_dims& d, bool distinct, const char* name,
                     int64_t* span) {
    if (!p) return fail(RT_EINVAL, "%s is NULL", name);
    if (!stride) return fail(RT_EINVAL, "%s's strides are NULL", name);
    const int64_t size = type_bytes(d.type);
    if (reinterpret_cast<uintptr_t>(p) % (uintptr_t)size != 0)
        return fail(RT_EINVAL, "%s is not aligned to its elements", name);
    const int64_t n[3] = {d.n0, d.n1, d.n2};
    int64_t last = 0;
    for (int i = 0; i < 3; ++i) {
        if (n[i] < 2) continue;
        if (stride[i] < 0) return fail(RT_EINVAL, "%s has a negative stride", name);
        if (stride[i] > ((int64_t)1 << 48) / n[i]) return fail(RT_EINVAL, "%s is too large", name);
        last += stride[i] * (n[i] - 1);
    }
    if (distinct) {  // from the closest rows on, each index's step has to pass over what the ones before it cover
        int order[3] = {0, 1, 2};
        std::sort(order, order + 3, [&](int x, int y) { return stride[x] < stride[y]; });
        int64_t covered = d.width;
        for (int i : order) {
            if (n[i] < 2) continue;
            if (stride[i] < covered) return fail(RT_EINVAL, "rows of %s share memory", name);
            covered += stride[i] * (n[i] - 1);
        }
    }
    *span = (last + d.width) * size;
    return RT_OK;
}

// Strides as the kernels take them, and whether rows can be counted flat and read in 16-byte pieces.
void set_rows(rt::NormArgs& a, const rt_norm_dims& d, std::initializer_list<std::pair<const void*, const int64_t*>> ts) {
    const int64_t size = type_bytes(d.type);
    a.flat = 1;
    a.vec = d.width % 8 == 0;
    for (const auto& t : ts) {
        const int64_t* s = t.second;
        // rows of each index below 2 have no step to fit
        const int64_t step = d.n2 > 1 ? s[2] : (d.n1 > 1 ? s[1] : (d.n0 > 1 ? s[0] : 0));
        const bool one = (d.n2 < 2 || s[2] == step) && (d.n1 < 2 || s[1] == step * d.n2) &&
                         (d.n0 < 2 || s[0] == step * d.n2 * d.n1);
        if (!one) a.flat = 0;
        if ((reinterpret_cast<uintptr_t>(t.first) & 15u) != 0) a.vec = 0;
        const int64_t n[3] = {d.n0, d.n1, d.n2};
        for (int i = 0; i < 3; ++i)
            if (n[i] > 1 && s[i] * size % 16 != 0) a.vec = 0;
    }
}

void set_strides(int64_t (&to)[3], const int64_t* s, const rt_norm_dims& d, int32_t flat) {
    to[0] = d.n0 > 1 ? s[0] : 0;
    to[1] = d.n1 > 1 ? s[1] : 0;
    to[2] = d.n2 > 1 ? s[2] : 0;
    if (flat) to[2] = d.n2 > 1 ? s[2] : (d.n1 > 1 ? s[1] : (d.n0 > 1 ? s[0] : 0));
}

void set_norm(rt::NormArgs& a, const rt_norm_dims& d, int64_t rows, const void* x, const int64_t* xs,
              const void* weight) {
    a.x = x;
    a.weight = weight;
    a.n1 = d.n1;
    a.n2 = d.n2;
    a.sets = (uint32_t)d.weight_sets;
    a.rows_per_set = (uint32_t)(rows / d.weight_sets);
    a.width = d.width;
    a.type = d.type;
    a.weight_f32 = d.weight_type == RT_F32;
    set_strides(a.xs, xs, d, a.flat);
}

rt_status check_weight(const void* p, const rt_norm_dims& d, const char* name) {
    const uintptr_t size = (uintptr_t)type_bytes(d.weight_type);
    if (p && reinterpret_cast<uintptr_t>(p) % size != 0) return fail(RT_EINVAL, "%s is not aligned to its elements", name);
    return RT_OK;
}

// Workgroups (partial sums of the columns) of a weight set, at most: over all sets those that the chip holds at once,
// two to a CU (one where a row takes 1024 lanes).  More of them walk fewer rows each behind the same start and join:
// 8192 rows of 1152 in 1024 workgroups 24.5 us, in 512 19.2; 384 19.5.
int32_t norm_parts(const rt_norm_dims& d) {
    const int64_t all = d.width <= 2048 || (d.width <= 8192 && d.width % 8 == 0) ? 512 : 256;
    return (int32_t)std::max<int64_t>(1, all / std::max(1, d.weight_sets));
}

int64_t norm_workspace(const rt_norm_dims& d) {
    return std::max<int64_t>(16, (int64_t)d.weight_sets * norm_parts(d) * 2 * d.width * 4);
}

}  // namespace

rt_status rt_index_transpose_size(const rt_bsr* mask, int32_t entries, int64_t* values) {
    if (!values) return fail(RT_EINVAL, "values is NULL");
    if (!mask) return fail(RT_EINVAL, "mask is NULL");
    RT_TRY(check_block(mask->block));
    if (mask->n_qblk < 0 || mask->n_masks < 0 || entries < 0)
        return fail(RT_EINVAL, "n_qblk=%d n_masks=%d entries=%d", mask->n_qblk, mask->n_masks, entries);
    Plan p{};
    RT_TRY(plan_of(mask, entries, &p));
    *values = p.values;
    return ok();
}

rt_status rt_index_transpose(const rt_bsr* mask, int32_t T, const rt_bsr* t, void* stream) {
    if (!mask) return fail(RT_EINVAL, "mask is NULL");
    if (T < 0) return fail(RT_EINVAL, "T=%d", T);
    const int64_t nm = mask->n_masks > 1 ? mask->n_masks : 1;
    // (any count of masks: the heads are not known here)
    RT_TRY(check_bsr(mask, rt_dims{1, (int32_t)nm, T, 64}));
    if (mask->n_qblk == 0) return ok();
    RT_TRY(check_transposed(t, mask));
    Plan p{};
    RT_TRY(plan_of(mask, t->nnz, &p));
    const int64_t np = mask_ptr_bytes(mask), nc = (int64_t)mask->nnz * 4;
    RT_TRY(check_ranges({{{t->row_ptr, np}, "the transposed row_ptr"}, {{t->col_idx, p.values * 4}, "the transposed col_idx"}},
                        {{mask->row_ptr, np}, {mask->col_idx, nc}}));
    rt::TransposeArgs a{};
    a.row_ptr = mask->row_ptr;
    a.col_idx = mask->col_idx;
    a.nnz = mask->nnz;
    a.n_blk = mask->n_qblk;
    a.n_masks = (int32_t)nm;
    a.t_row_ptr = const_cast<int32_t*>(t->row_ptr);
    a.t_col_idx = const_cast<int32_t*>(t->col_idx);
    a.t_nnz = t->nnz;
    a.plan = a.t_col_idx + p.first;
    a.seg = p.seg;
    a.max_more = p.max_more;
    return hip_status(rt::launch_index_transpose(a, static_cast<hipStream_t>(stream)), "index transpose launch");
}

rt_status rt_attn_full_backward_workspace(rt_dims dims, int64_t* bytes) {
    if (!bytes) return fail(RT_EINVAL, "bytes is NULL");
    bool empty = false;
    RT_TRY(check_dims(dims, &empty));
    *bytes = backward_workspace(dims, nullptr, Plan{});
    return ok();
}

rt_status rt_attn_full_backward(const void* q, const void* k, const void* v, const void* o, const float* row_max,
                                const float* row_sum, const void* d_o, rt_dims dims, void* dq, void* dk, void* dv,
                                void* workspace, int64_t workspace_bytes, void* stream) {
    bool empty = false;
    RT_TRY(check_dims(dims, &empty));
    if (empty) return ok();
    RT_TRY(check_items(dims, 32));
    // two workgroups of 256 threads for each tile, in whole eights, in one launch
    if (16 * ceil_div((int64_t)dims.B * dims.H * ceil_div(dims.T, rt::kDenseRows), 8) * 256 >= (int64_t)1 << 32)
        return fail(RT_EINVAL, "too many rows: B=%d H=%d T=%d", dims.B, dims.H, dims.T);
    const int64_t nt = tensor_bytes(dims, 2), ns = tensor_bytes(dims, 4) / dims.D;
    const int64_t need = backward_workspace(dims, nullptr, Plan{});
    rt::GradArgs a{};
    RT_TRY(grad_args(q, k, v, o, row_max, row_sum, d_o, dims, dq, dk, dv, workspace, workspace_bytes, need, &a));
    a.split = dense_split(dims);
    a.part = a.row_vals + (int64_t)dims.B * dims.H * 2 * a.T64;
    RT_TRY(check_ranges({{{dq, nt}, "dq"}, {{dk, nt}, "dk"}, {{dv, nt}, "dv"}, {{workspace, need}, "workspace"}},
                        {{q, nt}, {k, nt}, {v, nt}, {o, nt}, {d_o, nt}, {row_max, ns}, {row_sum, ns}}));
    return hip_status(rt::launch_attention_backward(a, dims.D, static_cast<hipStream_t>(stream)),
                      "full attention gradient launch");
}

rt_status rt_attn_sparse_backward_workspace(rt_dims dims, const rt_bsr* mask, int32_t room, int64_t* bytes) {
    if (!bytes) return fail(RT_EINVAL, "bytes is NULL");
    bool empty = false;
    RT_TRY(check_dims(dims, &empty));
    RT_TRY(check_bsr(mask, dims));
    const int32_t entries = room > 0 ? room : mask->nnz;
    if (entries < mask->nnz) return fail(RT_ECAPACITY, "room for %d entries, the mask has %d", entries, mask->nnz);
    Plan p{};
    RT_TRY(plan_of(mask, entries, &p));
    fold_parts(dims, mask, &p);
    *bytes = backward_workspace(dims, mask, p);
    return ok();
}

rt_status rt_attn_sparse_backward(const void* q, const void* k, const void* v, const void* o, const float* row_max,
                                  const float* row_sum, const void* d_o, rt_dims dims, const rt_bsr* mask,
                                  const rt_bsr* t, const float* rho, float rho_delta, void* dq, void* dk, void* dv,
                                  float* d_rho, void* workspace, int64_t workspace_bytes, void* stream) {
    bool empty = false;
    RT_TRY(check_dims(dims, &empty));
    RT_TRY(check_bsr(mask, dims));
    if (!std::isfinite(rho_delta)) return fail(RT_EINVAL, "rho_delta is not finite");
    if (d_rho && !rho) return fail(RT_EINVAL, "d_rho needs rho");
    if (empty) return ok();
    RT_TRY(check_transposed(t, mask));
    RT_TRY(check_items(dims, 32));
    if (rho) RT_TRY(check_stat(rho, "rho"));
    if (d_rho) RT_TRY(check_stat(d_rho, "d_rho"));
    const int64_t nt = tensor_bytes(dims, 2), ns = tensor_bytes(dims, 4) / dims.D;
    Plan p{};
    RT_TRY(plan_of(mask, t->nnz, &p));
    fold_parts(dims, mask, &p);
    const int64_t need = backward_workspace(dims, mask, p), bh = (int64_t)dims.B * dims.H;
    const int64_t uses = bh / (mask->n_masks > 1 ? mask->n_masks : 1);
    if ((uses * p.max_more + 2 * bh * mask->n_qblk + 32) * 2 * mask->block >= (int64_t)1 << 32)
        return fail(RT_EINVAL, "too many key blocks");  // 2 * block threads each, in one launch
    rt::GradArgs a{};
    RT_TRY(grad_args(q, k, v, o, row_max, row_sum, d_o, dims, dq, dk, dv, workspace, workspace_bytes, need, &a));
    const int64_t np = mask_ptr_bytes(mask), nc = (int64_t)mask->nnz * 4;
    RT_TRY(check_ranges({{{dq, nt}, "dq"}, {{dk, nt}, "dk"}, {{dv, nt}, "dv"}, {{d_rho, ns}, "d_rho"},
                         {{workspace, need}, "workspace"}},
                        {{q, nt}, {k, nt}, {v, nt}, {o, nt}, {d_o, nt}, {row_max, ns}, {row_sum, ns}, {rho, ns},
                         {mask->row_ptr, np}, {mask->col_idx, nc}, {t->row_ptr, np}, {t->col_idx, p.values * 4}}));
    a.rho = rho;
    a.rho_delta = rho_delta;
    a.d_rho = d_rho;
    a.row_ptr = mask->row_ptr;
    a.col_idx = mask->col_idx;
    a.nnz = mask->nnz;
    a.t_col_idx = t->col_idx;
    a.t_nnz = t->nnz;
    a.plan = t->col_idx + p.first;
    a.t_row_ptr = t->row_ptr;
    a.seg = p.seg;
    a.max_more = p.max_more;
    a.fold = p.fold;
    a.max_base = p.max_base;
    a.max_slots = p.max_slots;
    a.part = a.row_vals + bh * 2 * a.T64;
    a.n_masks = mask->n_masks > 1 ? mask->n_masks : 1;
    a.n_blk = mask->n_qblk;
    a.block = mask->block;
    return hip_status(rt::launch_attention_backward(a, dims.D, static_cast<hipStream_t>(stream)),
                      "sparse attention gradient launch");
}

rt_status rt_layer_norm(const void* x, const int64_t x_stride[3], const void* weight, const void* bias,
                        rt_norm_dims dims, float eps, void* y, const int64_t y_stride[3], float* mean, float* rstd,
                        void* stream) {
    int64_t rows = 0, x_span = 0, y_span = 0;
    RT_TRY(check_norm(dims, &rows));
    if (!std::isfinite(eps) || eps < 0) return fail(RT_EINVAL, "eps is negative or not finite");
    if (rows == 0) return ok();
    RT_TRY(check_rows(x, x_stride, dims, false, "x", &x_span));
    RT_TRY(check_rows(y, y_stride, dims, true, "y", &y_span));
    RT_TRY(check_weight(weight, dims, "weight"));
    RT_TRY(check_weight(bias, dims, "bias"));
    if (mean) RT_TRY(check_stat(mean, "mean"));
    if (rstd) RT_TRY(check_stat(rstd, "rstd"));
    const int64_t nw = (int64_t)dims.weight_sets * dims.width * type_bytes(dims.weight_type);
    RT_TRY(check_ranges({{{y, y_span}, "y"}, {{mean, rows * 4}, "mean"}, {{rstd, rows * 4}, "rstd"}},
                        {{x, x_span}, {weight, nw}, {bias, nw}}));
    rt::NormArgs a{};
    set_rows(a, dims, {{x, x_stride}, {y, y_stride}});
    if (weight && !aligned16(weight)) a.vec = 0;
    if (bias && !aligned16(bias)) a.vec = 0;
    set_norm(a, dims, rows, x, x_stride, weight);
    a.bias = bias;
    a.eps = eps;
    a.y = y;
    set_strides(a.ys, y_stride, dims, a.flat);
    a.mean_out = mean;
    a.rstd_out = rstd;
    return hip_status(rt::launch_norm(a, static_cast<hipStream_t>(stream)), "layer norm launch");
}

rt_status rt_layer_norm_backward_workspace(rt_norm_dims dims, int64_t* bytes) {
    if (!bytes) return fail(RT_EINVAL, "bytes is NULL");
    int64_t rows = 0;
    RT_TRY(check_norm(dims, &rows));
    *bytes = norm_workspace(dims);
    return ok();
}

rt_status rt_layer_norm_backward(const void* dy, const int64_t dy_stride[3], const void* x, const int64_t x_stride[3],
                                 const float* mean, const float* rstd, const void* weight, rt_norm_dims dims, void* dx,
                                 const int64_t dx_stride[3], float* d_weight, float* d_bias, void* workspace,
                                 int64_t workspace_bytes, void* stream) {
    int64_t rows = 0, x_span = 0, y_span = 0, dx_span = 0;
    RT_TRY(check_norm(dims, &rows));
    if (d_weight) RT_TRY(check_stat(d_weight, "d_weight"));
    if (d_bias) RT_TRY(check_stat(d_bias, "d_bias"));
    const int64_t ns = (int64_t)dims.weight_sets * dims.width * 4, need = norm_workspace(dims);
    rt::NormArgs a{};
    a.dweight = d_weight;
    a.dbias = d_bias;
    a.sets = (uint32_t)dims.weight_sets;
    a.width = dims.width;
    if (rows == 0) {  // sums over no rows
        RT_TRY(check_ranges({{{d_weight, ns}, "d_weight"}, {{d_bias, ns}, "d_bias"}}, {}));
        if ((!d_weight && !d_bias) || dims.weight_sets == 0) return ok();
        return hip_status(rt::launch_norm_backward(a, 0, static_cast<hipStream_t>(stream)), "layer norm gradient launch");
    }
    RT_TRY(check_rows(dy, dy_stride, dims, false, "dy", &y_span));
    RT_TRY(check_rows(x, x_stride, dims, false, "x", &x_span));
    RT_TRY(check_rows(dx, dx_stride, dims, true, "dx", &dx_span));
    RT_TRY(check_weight(weight, dims, "weight"));
    RT_TRY(check_stat(mean, "mean"));
    RT_TRY(check_stat(rstd, "rstd"));
    RT_TRY(check_tensor(workspace, "workspace"));
    if (workspace_bytes < need)
        return fail(RT_ECAPACITY, "workspace of %lld bytes, %lld needed", (long long)workspace_bytes, (long long)need);
    const int64_t nw = (int64_t)dims.weight_sets * dims.width * type_bytes(dims.weight_type);
    RT_TRY(check_ranges({{{dx, dx_span}, "dx"}, {{d_weight, ns}, "d_weight"}, {{d_bias, ns}, "d_bias"},
                         {{workspace, need}, "workspace"}},
                        {{dy, y_span}, {x, x_span}, {mean, rows * 4}, {rstd, rows * 4}, {weight, nw}}));
    set_rows(a, dims, {{dy, dy_stride}, {x, x_stride}, {dx, dx_stride}});
    if (weight && !aligned16(weight)) a.vec = 0;
    set_norm(a, dims, rows, x, x_stride, weight);
    a.dy = dy;
    a.dx = dx;
    set_strides(a.ys, dy_stride, dims, a.flat);
    set_strides(a.dxs, dx_stride, dims, a.flat);
    a.mean = mean;
    a.rstd = rstd;
    a.partial = static_cast<float*>(workspace);
    return hip_status(rt::launch_norm_backward(a, norm_parts(dims), static_cast<hipStream_t>(stream)),
                      "layer norm gradient launch");
}

// ---- rotary positions ----------------------------------------------------------------------

namespace {

// How a thread's pieces and heads are chosen: the widest piece that all rows start on and hold whole numbers of, and as
// many heads as leave 32 waves to a CU (a token's angles are formed once for them all).
void set_rope(rt::RopeArgs& a, std::initializer_list<std::pair<const void*, const int64_t*>> ts) {
    const int64_t size = type_bytes(a.type), n[3] = {a.B, a.H, a.T};
    a.vec = 1;
    for (int v : {8, 4}) {
        if (v * size > 16 || a.D % v || (a.half && a.pairs % v)) continue;
        bool fits = true;
        for (const auto& t : ts) {
            fits = fits && reinterpret_cast<uintptr_t>(t.first) % (uintptr_t)(v * size) == 0;
            for (int i = 0; i < 3; ++i) fits = fits && (n[i] < 2 || t.second[i] % v == 0);
        }
        if (fits) {
            a.vec = v;
            break;
        }
    }
    const int64_t one = std::max<int64_t>(1, (int64_t)a.B * a.T * rt::rope_places(a)), want = 256 * 32 * 64;
    const int64_t groups = std::min(ceil_div(want, one), ceil_div(a.H, rt::kRopeAhead));
    a.each = (int32_t)(ceil_div(ceil_div(a.H, groups), rt::kRopeAhead) * rt::kRopeAhead);
    a.groups = (int32_t)ceil_div(a.H, a.each);
}

rt_status rope(const void* x, const int64_t* x_stride, const void* positions, const double* freq, const int32_t* axis,
               float amplitude, const rt_rope_dims& d, bool inverse, void* y, const int64_t* y_stride, void* stream) {
    if (d.B < 0 || d.H < 0 || d.T < 0) return fail(RT_EINVAL, "negative dims B=%d H=%d T=%d", d.B, d.H, d.T);
    if (d.type != RT_BF16 && d.type != RT_F16 && d.type != RT_F32) return fail(RT_EUNSUPPORTED, "type=%d", d.type);
    if (d.position_type != RT_POS_I32 && d.position_type != RT_POS_I64 && d.position_type != RT_POS_F32)
        return fail(RT_EUNSUPPORTED, "position_type=%d", d.position_type);
    if (d.layout != RT_ROPE_INTERLEAVED && d.layout != RT_ROPE_HALF) return fail(RT_EUNSUPPORTED, "layout=%d", d.layout);
    if (d.D < 2) return fail(RT_EINVAL, "width D=%d (need >= 2)", d.D);
    if (d.D > 16384) return fail(RT_EUNSUPPORTED, "width D=%d (supported: up to 16384)", d.D);
    if (d.rotated < 2 || d.rotated > d.D || d.rotated % 2)
        return fail(RT_EINVAL, "rotated=%d (need an even number of 2 to D=%d elements)", d.rotated, d.D);
    if (d.axes < 1) return fail(RT_EINVAL, "axes=%d (need >= 1)", d.axes);
    if (d.axes > 16) return fail(RT_EUNSUPPORTED, "axes=%d (supported: up to 16)", d.axes);
    if (!std::isfinite(amplitude)) return fail(RT_EINVAL, "amplitude is not finite");
    if (d.B == 0 || d.H == 0 || d.T == 0) return ok();
    if ((int64_t)d.T * d.D >= (int64_t)1 << 32 || (int64_t)d.B * d.H > INT32_MAX ||
        (int64_t)d.B * d.H >= ((int64_t)1 << 48) / d.T)
        return fail(RT_EINVAL, "tensor too large");
    const rt_norm_dims rows{d.B, d.H, d.T, d.D, d.type, d.type, 1};
    int64_t x_span = 0, y_span = 0;
    RT_TRY(check_rows(x, x_stride, rows, false, "x", &x_span));
    RT_TRY(check_rows(y, y_stride, rows, true, "y", &y_span));
    const int64_t pos_size = d.position_type == RT_POS_I64 ? 8 : 4, sets = d.per_sample ? d.B : 1;
    if (!positions) return fail(RT_EINVAL, "positions is NULL");
    if (reinterpret_cast<uintptr_t>(positions) % (uintptr_t)pos_size) return fail(RT_EINVAL, "positions is not aligned to its elements");
    if (!freq) return fail(RT_EINVAL, "freq is NULL");
    if (reinterpret_cast<uintptr_t>(freq) % 8) return fail(RT_EINVAL, "freq is not 8-byte aligned");
    if (d.axes > 1) RT_TRY(check_stat(axis, "axis"));
    bool same = x == y;  // in place: every thread reads its elements before it writes them
    const int64_t n[3] = {d.B, d.H, d.T};
    for (int i = 0; i < 3; ++i) same = same && (n[i] < 2 || x_stride[i] == y_stride[i]);
    const int64_t np = sets * d.T * d.axes * pos_size, nf = (int64_t)d.rotated / 2 * 8;
    RT_TRY(check_no_overlap(y, y_span, "y", {{positions, np}, {freq, nf}, {d.axes > 1 ? axis : nullptr, nf / 2}}, "an input"));
    if (!same) RT_TRY(check_no_overlap(y, y_span, "y", {{x, x_span}}, "x"));
    rt::RopeArgs a{};
    a.x = x;
    a.y = y;
    a.positions = positions;
    a.freq = freq;
    a.axis = axis;
    for (int i = 0; i < 3; ++i) {
        a.xs[i] = n[i] > 1 ? x_stride[i] : 0;
        a.ys[i] = n[i] > 1 ? y_stride[i] : 0;
    }
    a.B = d.B;
    a.H = d.H;
    a.T = d.T;
    a.D = d.D;
    a.pairs = d.rotated / 2;
    a.axes = d.axes;
    a.type = d.type;
    a.pos_type = d.position_type;
    a.half = d.layout == RT_ROPE_HALF;
    a.per_sample = d.per_sample != 0;
    a.inverse = inverse;
    a.amplitude = amplitude;
    set_rope(a, {{x, x_stride}, {y, y_stride}});
    if (rt::rope_blocks(a) >= (int64_t)1 << 24) return fail(RT_EINVAL, "tensor too large");  // 256 threads each, in one launch
    return hip_status(rt::launch_rope(a, static_cast<hipStream_t>(stream)), "rotary position launch");
}

}  // namespace

rt_status rt_rope(const void* x, const int64_t x_stride[3], const void* positions, const double* freq, const int32_t* axis,
                  float amplitude, rt_rope_dims dims, void* y, const int64_t y_stride[3], void* stream) {
    return rope(x, x_stride, positions, freq, axis, amplitude, dims, false, y, y_stride, stream);
}

rt_status rt_rope_backward(const void* dy, const int64_t dy_stride[3], const void* positions, const double* freq,
                           const int32_t* axis, float amplitude, rt_rope_dims dims, void* dx, const int64_t dx_stride[3],
                           void* stream) {
    return rope(dy, dy_stride, positions, freq, axis, amplitude, dims, true, dx, dx_stride, stream);
}

// ---- differential attention ----------------------------------------------------------------

namespace {

rt_status check_diff(const rt_diff_dims& d) {
    if (d.B < 0 || d.H < 0 || d.Tq < 0 || d.Tk < 0)
        return fail(RT_EINVAL, "negative dims B=%d H=%d Tq=%d Tk=%d", d.B, d.H, d.Tq, d.Tk);
    if (d.D != 64 && d.D != 72) return fail(RT_EUNSUPPORTED, "head width D=%d (supported: 64, 72)", d.D);
    const int64_t bh = (int64_t)d.B * d.H, t = std::max(d.Tq, d.Tk);
    if (bh >= (int64_t)1 << 23) return fail(RT_EINVAL, "B*H too large");
    // buffer record counts and offsets within one head are 32-bit, as in the other attention calls; values are 2 D wide
    if (t * d.D * 4 > (int64_t)1 << 30) return fail(RT_EINVAL, "Tq=%d Tk=%d too long for one head", d.Tq, d.Tk);
    if (bh * t * d.D * 2 >= (int64_t)1 << 40) return fail(RT_EINVAL, "tensor too large");
    // threads of a launch: 256 for every tile of 128 rows, and 16 for each row in whole 64
    if (bh * whole64((int32_t)t) >= (int64_t)1 << 28) return fail(RT_EINVAL, "too many rows: B=%d H=%d Tq=%d Tk=%d", d.B, d.H, d.Tq, d.Tk);
    return RT_OK;
}

// Bytes of the calls' tensors
struct DiffBytes {
    int64_t q, k, v, o, stat, lam, lens;
};
DiffBytes diff_bytes(const rt_diff_dims& d, int32_t n_lam) {
    const int64_t bh = (int64_t)d.B * d.H;
    return {bh * d.Tq * d.D * 4, bh * d.Tk * d.D * 4, bh * d.Tk * d.D * 4, bh * d.Tq * d.D * 4, bh * d.Tq * 8, (int64_t)n_lam * 4,
            (int64_t)d.B * 4};
}

// Forward: whether a workgroup's waves share the keys of 32 queries, and workgroups that share a tile's keys, by an
// estimate of the times.  Sharing keys starts four times as many workgroups, one to a CU, and reads the keys four times
// as often: 8 heads of 2048 tokens 43 us against 60 of tiles of 128, 4 heads of 3000, 72 wide, 65 against 81 of tiles in
// parts; but 35 heads of 700, 72 wide, 50 against 32, 18 heads of 4055 queries over 2391 keys 244 against 205.  Parts cost
// their sums' way through memory: 8 heads of 2500 tokens 96 us in three, 74 whole, 6 heads of 7460 and fewer keys 348 and
// 258; but 4 heads of 200 queries over 6000 keys 21 in eight, 34 in two.  The estimate's rates are fitted to 108 drawn calls
// in up to 13 plans each, for which its choice is 0.3 % above the best in the mean, 8 at most.
struct DiffPlan {
    int32_t by_keys, split;
};
DiffPlan diff_plan(const rt_diff_dims& d, bool lens) {
    // where samples have numbers of keys of their own, as if five eighths of the heads had work (60 heads of 177 queries over
    // 6590 keys and fewer 98 us as if all had, 88 six eighths, 55 five; 9 heads of 7238 tokens and fewer keys 322, 263, 263)
    const int64_t bh = ceil_div((int64_t)d.B * d.H * (lens && d.Tq > 32 ? 5 : 8), 8), chunks = ceil_div(d.Tk, 32);
    DiffPlan p{0, 1};
    int64_t best = INT64_MAX;
    // (of 32 queries, a tile of four waves would keep one busy)
    for (int by_keys = d.Tq <= 32 && chunks > 4; by_keys < 2; ++by_keys) {
        const int64_t n = bh * ceil_div(d.Tq, by_keys ? 32 : rt::kDiffRows), slots = by_keys ? 256 : 512;
        for (int64_t s = 1; s <= rt::kDiffParts; ++s) {
            if (s > 1 && (n * s > 2 * slots || chunks < (by_keys ? 8 : 4) * s)) break;
            // tenths of microseconds: of a chunk in a wave alone on its SIMD, or one of two (a quarter more 72 wide); of a
            // workgroup's start and end
            const int64_t m = n * s, late = m % slots, own = ceil_div(chunks, by_keys ? 4 * s : s);
            auto each = [&](int64_t chunk, int64_t ends) { return own * chunk * (d.D == 72 ? 5 : 4) / 4 + ends; };
            int64_t t = by_keys ? ceil_div(m, slots) * each(13, 50)
                                : m / slots * each(16, 35) + (late ? each(late <= 256 ? 11 : 16, 35) : 0);
            if (s > 1) t += 65 + bh * s * d.Tq * d.D * 32 / 180000;  // the parts, written and read
            if (t < best) {
                best = t;
                p = DiffPlan{by_keys, (int32_t)s};
            }
        }
    }
    return p;
}
// The larger need of calls with and without numbers of keys, which is what every call is given.
int64_t diff_workspace(const rt_diff_dims& d, const DiffPlan& one, const DiffPlan& other) {
    const int64_t s = std::max(one.split, other.split);
    return std::max<int64_t>(16, s > 1 ? (int64_t)d.B * d.H * s * 2 * d.Tq * (2 * d.D + 3) * 4 : 0);
}

// When `slots` workgroups at once are through n1 of length l1 and then n2 of length l2.
int64_t finish(int64_t n1, int64_t l1, int64_t n2, int64_t l2, int64_t slots) {
    const int64_t rounds = n1 / slots, late = n1 % slots, early = slots - late;
    int64_t t = rounds * l1;
    if (late) {
        const int64_t fit = ceil_div(l1, l2) * early;  // taken while the last of the first are under way
        if (n2 <= fit) return std::max(t + l1, t + ceil_div(n2, early) * l2);
        n2 -= fit;
        t += l1;
    }
    return t + ceil_div(n2, slots) * l2;
}

// Backward: whether eight waves take a tile, and workgroups that share the walk of a tile of keys, of queries, by an
// estimate of when the last workgroup ends.  Eight waves to a tile, two to a SIMD where there is a tile to a CU: 16 heads
// of 1024 tokens, 72 wide, 56 us against 67, 15 heads of 2734 queries over 1175 keys and fewer 92 against 122; but 15 heads
// of 1500 tokens 95 against 79.  Parts, of either side's walks: one head of 4096 tokens 55 us, by eight waves in four of dK
// and dV and three of dQ, 122 whole; 32 heads of 4096 queries over 226 keys and fewer, 72 wide, 95 in six, 246 whole (their
// dK and dV are 64 tiles of 128 chunks each); the other way round (4 heads of 200 queries over 6000 keys) 35 and 163; 8
// heads of 961 queries over 3723 keys, 72 wide, 98 in two of dQ, 153 whole; but 8 heads of 2500 tokens 145 in two, 119
// whole.  The estimate's rates are fitted to 273 drawn calls in up to 24 plans each, for which its choice is 1.4 % above
// the best in the mean, 43 at most.
struct DiffBackPlan {
    int32_t two, q_first, split_k, split_q;
};
DiffBackPlan diff_back_plan(const rt_diff_dims& d, bool lens) {
    const int64_t bh = (int64_t)d.B * d.H, nk = bh * ceil_div(d.Tk, rt::kDiffRows), nq = bh * ceil_div(d.Tq, rt::kDiffRows);
    DiffBackPlan p{0, 0, 1, 1};
    if (nk == 0 || nq == 0) return p;
    // half microseconds: of a walk's chunks of 32 rows, two waves to a SIMD
    const int64_t wk = 4 * ceil_div(d.Tq, 32), wq = 3 * ceil_div(d.Tk, 32);
    const int64_t longest = std::max(wk, wq);
    // where samples have numbers of keys of their own, tiles are counted as if seven eighths had work, parts as if five did
    const int64_t share = lens && d.B > 1 ? 7 : 8, rk = ceil_div(nk * share, 8), rq = ceil_div(nq * share, 8);
    int64_t best = INT64_MAX;
    for (int two = 0; two < (nk + nq > 4096 ? 1 : 2); ++two) {
        for (int i = 1; i <= 32; ++i) {
            const int64_t part = std::max<int64_t>(1, ceil_div(longest, i));
            const int64_t sk = std::max<int64_t>(1, ceil_div(wk, part)), sq = std::max<int64_t>(1, ceil_div(wq, part));
            // the parts in whole tiles of 128 x D; a gigabyte and a half of them at most
            const int64_t parts = (sk > 1 ? nk * sk * 4 : 0) + (sq > 1 ? nq * sq * 2 : 0);
            if (i > 1 && (part < 16 || parts > 40000)) break;
            const int64_t slots = two ? 256 : 512;
            // of four waves' time for a walk, eight take two thirds, four alone on their CU seven eighths, a quarter more 72
            // wide; its start and end, with the row values of short heads
            const int64_t rate = (two ? 26 : (rk * sk + rq * sq <= 256 ? 34 : 40)) * (d.D == 72 ? 5 : 4);
            const int64_t ends = (two ? 34 : 28) + (d.Tq <= rt::kDiffShort ? ceil_div(d.Tq, two ? 32 : 16) : 0);
            const int64_t lk = ceil_div(wk, sk) * rate / 160 + ends, lq = ceil_div(wq, sq) * rate / 160 + ends;
            const bool q_first = lq > lk;  // what takes longer begins first
            int64_t t = q_first ? finish(rq * sq, lq, rk * sk, lk, slots) : finish(rk * sk, lk, rq * sq, lq, slots);
            if (parts) t += t / 8 + 16 + parts * (lens ? 5 : 8) * rt::kDiffRows * d.D / 1300000;  // written and read
            if (t < best) {
                best = t;
                p = DiffBackPlan{two, q_first, (int32_t)sk, (int32_t)sq};
            }
        }
    }
    return p;
}
// Floats of the row values, and of the sums of 16 rows for dlam, in 64 bits
int64_t diff_vals(const rt_diff_dims& d) { return (int64_t)d.B * d.H * 4 * whole64(d.Tq); }
int64_t diff_lam_part(const rt_diff_dims& d) { return (int64_t)d.B * d.H * (whole64(d.Tq) / 16) * 2; }
int64_t diff_part_k(const rt_diff_dims& d, int64_t split) {
    return (int64_t)d.B * d.H * ceil_div(d.Tk, rt::kDiffRows) * split * 4 * rt::kDiffRows * d.D;
}
int64_t diff_part_q(const rt_diff_dims& d, int64_t split) {
    return (int64_t)d.B * d.H * ceil_div(d.Tq, rt::kDiffRows) * split * 2 * rt::kDiffRows * d.D;
}
// The plans of calls with and without numbers of keys, made once a call (up to 4 us of the host's time), and the larger need.
struct DiffBackPlans {
    DiffBackPlan of[2];  // [whether there are numbers of keys]
    int64_t workspace;
};
DiffBackPlans diff_back_plans(const rt_diff_dims& d) {
    DiffBackPlans r{{diff_back_plan(d, false), diff_back_plan(d, true)}, 16};
    for (const DiffBackPlan& p : r.of) {
        const int64_t parts = (p.split_k > 1 ? diff_part_k(d, p.split_k) : 0) + (p.split_q > 1 ? diff_part_q(d, p.split_q) : 0);
        r.workspace = std::max(r.workspace, (diff_vals(d) + diff_lam_part(d) + parts) * 4);
    }
    return r;
}

// What both calls check and set alike.
rt_status diff_args(const void* q, const void* k, const void* v, const float* lam, int32_t n_lam, const int32_t* k_lens,
                    const rt_diff_dims& d, rt::DiffArgs* out) {
    if (n_lam != 1 && n_lam != d.H) return fail(RT_EINVAL, "n_lam=%d (need 1 or H=%d)", n_lam, d.H);
    if (d.Tq > 0 && d.B > 0 && d.H > 0) RT_TRY(check_tensor(q, "q"));
    if (d.Tk > 0 && d.B > 0 && d.H > 0) {
        RT_TRY(check_tensor(k, "k"));
        RT_TRY(check_tensor(v, "v"));
    }
    if (n_lam > 0) RT_TRY(check_stat(lam, "lam"));
    if (k_lens) RT_TRY(check_stat(k_lens, "k_lens"));
    rt::DiffArgs a{};
    a.q = static_cast<const uint16_t*>(q);
    a.k = static_cast<const uint16_t*>(k);
    a.v = static_cast<const uint16_t*>(v);
    a.lam = lam;
    a.lam_step = n_lam == d.H && d.H > 1 ? 1 : 0;
    a.k_lens = k_lens;
    a.by_len = k_lens && d.Tq > 32 && d.B > 1 && d.B <= 64;
    a.B = d.B;
    a.H = d.H;
    a.Tq = d.Tq;
    a.Tk = d.Tk;
    a.n_bh = d.B * d.H;
    a.scale_nat = (float)(1.0 / std::sqrt((double)d.D));
    a.scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)d.D));
    a.move = rt::kDiffMove / a.scale_log2;
    *out = a;
    return RT_OK;
}

}  // namespace

rt_status rt_attn_diff_workspace(rt_diff_dims dims, int64_t* bytes) {
    if (!bytes) return fail(RT_EINVAL, "bytes is NULL");
    RT_TRY(check_diff(dims));
    *bytes = diff_workspace(dims, diff_plan(dims, false), diff_plan(dims, true));
    return ok();
}

rt_status rt_attn_diff(const void* q, const void* k, const void* v, const float* lam, int32_t n_lam, const int32_t* k_lens,
                       rt_diff_dims dims, void* o, void* o2, float* row_max, float* row_sum, void* workspace,
                       int64_t workspace_bytes, void* stream) {
    RT_TRY(check_diff(dims));
    rt::DiffArgs a{};
    if (dims.B == 0 || dims.H == 0 || dims.Tq == 0) return ok();
    RT_TRY(diff_args(q, k, v, lam, n_lam, k_lens, dims, &a));
    RT_TRY(check_tensor(o, "o"));
    const int given = (o2 != nullptr) + (row_max != nullptr) + (row_sum != nullptr);
    if (given % 3) return fail(RT_EINVAL, "o2, row_max and row_sum are written together or not at all");
    if (given) {
        RT_TRY(check_tensor(o2, "o2"));
        RT_TRY(check_stat(row_max, "row_max"));
        RT_TRY(check_stat(row_sum, "row_sum"));
    }
    const DiffPlan plan = diff_plan(dims, k_lens != nullptr);
    const int64_t need = plan.split > 1 ? diff_workspace(dims, plan, diff_plan(dims, k_lens == nullptr)) : 0;
    a.split = plan.split;
    const void* ws = a.split > 1 ? workspace : nullptr;
    if (a.split > 1) {
        RT_TRY(check_tensor(workspace, "workspace"));
        if (workspace_bytes < need)
            return fail(RT_ECAPACITY, "workspace of %lld bytes, %lld needed", (long long)workspace_bytes, (long long)need);
    }
    const DiffBytes n = diff_bytes(dims, n_lam);
    RT_TRY(check_ranges({{{o, n.o}, "o"}, {{o2, n.o}, "o2"}, {{row_max, n.stat}, "row_max"}, {{row_sum, n.stat}, "row_sum"},
                         {{ws, need}, "workspace"}},
                        {{q, n.q}, {k, n.k}, {v, n.v}, {lam, n.lam}, {k_lens, n.lens}}));
    a.o = static_cast<uint16_t*>(o);
    a.o2 = static_cast<uint16_t*>(o2);
    a.row_max = row_max;
    a.row_sum = row_sum;
    a.by_keys = plan.by_keys;
    a.part = static_cast<float*>(workspace);
    return hip_status(rt::launch_diff(a, dims.D, static_cast<hipStream_t>(stream)), "differential attention launch");
}

rt_status rt_attn_diff_backward_workspace(rt_diff_dims dims, int64_t* bytes) {
    if (!bytes) return fail(RT_EINVAL, "bytes is NULL");
    RT_TRY(check_diff(dims));
    *bytes = diff_back_plans(dims).workspace;
    return ok();
}

rt_status rt_attn_diff_backward(const void* q, const void* k, const void* v, const float* lam, int32_t n_lam,
                                const int32_t* k_lens, const void* o, const void* o2, const float* row_max,
                                const float* row_sum, const void* d_o, rt_diff_dims dims, void* dq, void* dk, void* dv,
                                float* d_lam, void* workspace, int64_t workspace_bytes, void* stream) {
    RT_TRY(check_diff(dims));
    rt::DiffArgs a{};
    RT_TRY(diff_args(q, k, v, lam, n_lam, k_lens, dims, &a));
    if (n_lam > 0) RT_TRY(check_stat(d_lam, "d_lam"));
    const bool rows = a.n_bh > 0 && dims.Tq > 0, cols = a.n_bh > 0 && dims.Tk > 0;
    if (rows) {
        RT_TRY(check_tensor(o, "o"));
        RT_TRY(check_tensor(o2, "o2"));
        RT_TRY(check_stat(row_max, "row_max"));
        RT_TRY(check_stat(row_sum, "row_sum"));
        RT_TRY(check_tensor(d_o, "d_o"));
        RT_TRY(check_tensor(dq, "dq"));
        RT_TRY(check_tensor(workspace, "workspace"));
    }
    if (cols) {
        RT_TRY(check_tensor(dk, "dk"));
        RT_TRY(check_tensor(dv, "dv"));
    }
    const DiffBackPlans plans = diff_back_plans(dims);
    const DiffBackPlan& plan = plans.of[k_lens != nullptr];
    const int64_t need = plans.workspace;
    if (rows && workspace_bytes < need)
        return fail(RT_ECAPACITY, "workspace of %lld bytes, %lld needed", (long long)workspace_bytes, (long long)need);
    const DiffBytes n = diff_bytes(dims, n_lam);
    RT_TRY(check_ranges({{{rows ? dq : nullptr, n.q}, "dq"}, {{cols ? dk : nullptr, n.k}, "dk"}, {{cols ? dv : nullptr, n.v}, "dv"},
                         {{n_lam ? d_lam : nullptr, n.lam}, "d_lam"}, {{rows ? workspace : nullptr, need}, "workspace"}},
                        {{q, n.q}, {k, n.k}, {v, n.v}, {lam, n.lam}, {k_lens, n.lens}, {o, n.o}, {o2, n.o}, {row_max, n.stat},
                         {row_sum, n.stat}, {d_o, n.o}}));
    a.o = static_cast<uint16_t*>(const_cast<void*>(o));
    a.o2 = static_cast<uint16_t*>(const_cast<void*>(o2));
    a.row_max = const_cast<float*>(row_max);
    a.row_sum = const_cast<float*>(row_sum);
    a.d_o = static_cast<const uint16_t*>(d_o);
    a.dq = static_cast<uint16_t*>(dq);
    a.dk = static_cast<uint16_t*>(dk);
    a.dv = static_cast<uint16_t*>(dv);
    a.d_lam = d_lam;
    a.T64 = whole64(dims.Tq);
    a.row_vals = static_cast<float*>(workspace);
    a.two = plan.two;
    a.q_first = plan.q_first;
    // one launch where all run at once on the chip, and the workgroup that sums a weight's gradient has few rows (16 heads of 60 that share one: 16.9 against 24 us)
    const int64_t tiles = (int64_t)a.n_bh * (ceil_div(dims.Tk, rt::kDiffRows) + ceil_div(dims.Tq, rt::kDiffRows));
    a.short_rows = dims.Tq <= rt::kDiffShort && tiles <= 256 && plan.split_k == 1 && plan.split_q == 1 &&
                   (int64_t)(a.lam_step ? dims.B : a.n_bh) * dims.Tq <= 256;
    a.split_k = plan.split_k;
    a.split_q = plan.split_q;
    a.lam_part = reinterpret_cast<double*>(a.row_vals + diff_vals(dims));
    a.part_k = a.row_vals + diff_vals(dims) + diff_lam_part(dims);
    a.part_q = a.part_k + (a.split_k > 1 ? diff_part_k(dims, a.split_k) : 0);
    if (n_lam == 0) return ok();  // no heads
    return hip_status(rt::launch_diff_backward(a, dims.D, static_cast<hipStream_t>(stream)),
                      "differential attention gradient launch");
}

}  // extern "C"
