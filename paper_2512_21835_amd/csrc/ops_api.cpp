// C entry points of include/stage_ops.h: every argument checked, then the launch.
#include "stage_ops.h"

#include <cmath>

#include "device_guard.h"
#include "ops_kernels.h"
#include "stage.h"

using namespace stg;

namespace {

bool on16(const void *p) { return ((uintptr_t)p & 15) == 0; }
bool is_type(int t) { return t == STAGE_F32 || t == STAGE_BF16; }
// Rows of `width` elements, `ld` apart, starting on 16-byte boundaries (strides that no index of ours overflows).
bool rows_ok(const void *p, int64_t ld, int64_t width, int type) {
    return p && on16(p) && ld >= width && ld < (int64_t(1) << 40) && ld % (type == STAGE_F32 ? 4 : 8) == 0;
}

bool heads_ok(int hq, int hkv) {
    if (hkv < 1 || hq < 1 || hkv > 65536 || hq > 65536 || hq % hkv != 0) return false;
    const int g = hq / hkv;
    return g == 1 || g == 2 || g == 4 || g == 8;
}

bool sizes_ok(const stage_batch &b, const stage_cache &c, int rows, int n_q_heads) {
    return b.n_seqs >= 1 && b.n_seqs <= STAGE_OPS_MAX_SEQS && b.max_rows >= 1 && b.max_len >= 1 && b.max_blocks >= 1 &&
           b.max_blocks <= STAGE_OPS_MAX_BLOCKS && b.max_len <= kBlockTokens * b.max_blocks && rows >= 0 &&
           rows <= STAGE_OPS_MAX_ROWS && c.n_blocks >= 1 && (c.head_dim == 64 || c.head_dim == 128) && is_type(c.type) &&
           heads_ok(n_q_heads, c.n_kv_heads);
}

bool pointers_ok(const stage_batch &b, const stage_cache &c) {
    return b.row_start && b.length && b.block_table && c.pool && on16(c.pool);
}

bool device_ok(int device) {
    static const int count = [] {   // (devices do not come and go while a process runs)
        int n = 0;
        if (hipGetDeviceCount(&n) == hipSuccess) return n;
        (void)hipGetLastError();
        return 0;
    }();
    return device >= 0 && device < count;
}

OpRows op_rows(const stage_batch &b, const stage_cache &c, int rows) {
    OpRows r{};
    r.row_start = b.row_start;
    r.length = b.length;
    r.table = b.block_table;
    r.n_seqs = b.n_seqs;
    r.max_rows = b.max_rows < rows ? b.max_rows : rows;
    r.max_len = b.max_len;
    r.max_blocks = b.max_blocks;
    r.rows = rows;
    r.n_blocks = c.n_blocks;
    return r;
}

int status(hipError_t e) {
    if (e == hipSuccess) return STAGE_OK;
    return e == hipErrorInvalidValue ? STAGE_EINVAL : STAGE_EHIP;
}

bool window_sizes(const stage_window_args &a) {
    return sizes_ok(a.batch, a.cache, a.rows, a.n_q_heads) && a.window >= 0 && a.sinks >= 0 && is_type(a.type) &&
           (a.scale == 0.f || (std::fabs(a.scale) >= 1e-30f && std::fabs(a.scale) <= 1e30f));
}

WindowArgs window_args(const stage_window_args &a, void *workspace) {
    WindowArgs w{};
    w.q = a.q;
    w.out = a.out;
    w.type = a.type;
    w.q_ld = a.q_ld;
    w.out_ld = a.out_ld;
    w.pool = a.cache.pool;
    w.n_q_heads = a.n_q_heads;
    w.n_kv_heads = a.cache.n_kv_heads;
    w.head_dim = a.cache.head_dim;
    w.kv_type = a.cache.type;
    // (no window: one beyond every position, which sequences of more than max_len tokens have as well)
    w.window = a.window == 0 || a.window > kMaxLength ? kMaxLength : a.window;
    w.sinks = a.sinks > a.batch.max_len ? a.batch.max_len : a.sinks;
    w.scale = a.scale == 0.f ? 1.f / std::sqrt((float)a.cache.head_dim) : a.scale;
    w.part = static_cast<float *>(workspace);
    w.rows = op_rows(a.batch, a.cache, a.rows);
    return w;
}

bool adapter_sizes(const stage_adapter_args &a) {
    return a.rows >= 0 && a.rows <= STAGE_OPS_MAX_ROWS && a.k >= 8 && a.k % 8 == 0 && a.n >= 8 && a.n % 8 == 0 &&
           a.k <= (1 << 24) && a.n <= (1 << 24) && a.n_adapters >= 1 && a.max_rank >= 4 && a.max_rank % 4 == 0 &&
           a.max_rank <= STAGE_OPS_MAX_RANK && is_type(a.type);
}

AdapterArgs adapter_args(const stage_adapter_args &a, void *workspace) {
    AdapterArgs p{};
    p.x = a.x;
    p.base = a.base;
    p.out = a.out;
    p.type = a.type;
    p.x_ld = a.x_ld;
    p.base_ld = a.base_ld;
    p.out_ld = a.out_ld;
    p.rows = a.rows;
    p.k = a.k;
    p.n = a.n;
    p.n_adapters = a.n_adapters;
    p.max_rank = a.max_rank;
    p.a = static_cast<const uint16_t *>(a.a);
    p.b = static_cast<const uint16_t *>(a.b);
    p.ids = a.ids;
    p.ranks = a.ranks;
    p.scales = a.scales;
    p.part = static_cast<float *>(workspace);
    return p;
}

// The workspace of a call: STAGE_OK, or why not.
int workspace_ok(const void *workspace, int64_t have, size_t need) {
    if (need == 0) return STAGE_OK;
    if (have < 0 || (size_t)have < need) return STAGE_ENOMEM;
    return workspace && on16(workspace) ? STAGE_OK : STAGE_EINVAL;
}

}  // namespace

extern "C" {

int stage_norm_rope_append(const stage_append_args *p, void *stream) {
    if (!p) return STAGE_EINVAL;
    const stage_append_args &a = *p;
    if (!sizes_ok(a.batch, a.cache, a.rows, a.n_q_heads) || !is_type(a.qkv_type) || !is_type(a.q_type) ||
        !(a.eps >= 0.f) || a.n_angles < 1 || !pointers_ok(a.batch, a.cache) || !a.cos || !a.sin || !on16(a.cos) || !on16(a.sin))
        return STAGE_EINVAL;
    const int d = a.cache.head_dim, half = d / 2;
    const int64_t q_width = (int64_t)a.n_q_heads * d, width = q_width + 2 * (int64_t)a.cache.n_kv_heads * d;
    if (!rows_ok(a.qkv, a.qkv_ld, width, a.qkv_type) || !rows_ok(a.q_out, a.q_ld, q_width, a.q_type) ||
        (a.q_gain && !on16(a.q_gain)) || (a.k_gain && !on16(a.k_gain)))
        return STAGE_EINVAL;
    if (a.q_out == a.qkv && (a.q_type != a.qkv_type || a.q_ld != a.qkv_ld)) return STAGE_EINVAL;
    AppendArgs r{};
    r.axis1 = r.axis2 = half;
    if (a.positions) {
        const int32_t *s = a.section;
        if (a.n_axes == 1) {
            if (s[0] != half) return STAGE_EINVAL;
        } else if (a.n_axes == 3) {
            if (s[0] < 0 || s[1] < 0 || s[2] < 0 || s[0] > half || s[1] > half || s[2] > half || s[0] + s[1] + s[2] != half)
                return STAGE_EINVAL;
            r.axis1 = s[0];
            r.axis2 = s[0] + s[1];
        } else {
            return STAGE_EINVAL;
        }
    }
    if (!device_ok(a.device)) return STAGE_EINVAL;
    if (a.rows == 0) return STAGE_OK;
    r.qkv = a.qkv;
    r.qkv_type = a.qkv_type;
    r.n_part = 1;
    r.qkv_ld = a.qkv_ld;
    r.q_out = a.q_out;
    r.q_type = a.q_type;
    r.q_ld = a.q_ld;
    r.q_gain = static_cast<const uint16_t *>(a.q_gain);
    r.k_gain = static_cast<const uint16_t *>(a.k_gain);
    r.eps = a.eps;
    r.cos_t = a.cos;
    r.sin_t = a.sin;
    r.n_angles = a.n_angles;
    r.positions = a.positions;
    r.pool = a.cache.pool;
    r.n_q_heads = a.n_q_heads;
    r.n_kv_heads = a.cache.n_kv_heads;
    r.head_dim = d;
    r.kv_type = a.cache.type;
    r.rows = op_rows(a.batch, a.cache, a.rows);
    DeviceGuard dg(a.device);
    return status(launch_norm_rope_append(r, static_cast<hipStream_t>(stream)));
}

int stage_window_workspace(const stage_window_args *a, int64_t *bytes) {
    if (!a || !bytes || !window_sizes(*a) || !device_ok(a->device)) return STAGE_EINVAL;
    DeviceGuard dg(a->device);
    *bytes = (int64_t)window_workspace(window_args(*a, nullptr));
    return STAGE_OK;
}

int stage_window_attention(const stage_window_args *p, void *workspace, int64_t workspace_bytes, void *stream) {
    if (!p) return STAGE_EINVAL;
    const stage_window_args &a = *p;
    if (!window_sizes(a) || !pointers_ok(a.batch, a.cache)) return STAGE_EINVAL;
    const int64_t width = (int64_t)a.n_q_heads * a.cache.head_dim;
    if (!rows_ok(a.q, a.q_ld, width, a.type) || !rows_ok(a.out, a.out_ld, width, a.type)) return STAGE_EINVAL;
    if (a.out == a.q && a.out_ld != a.q_ld) return STAGE_EINVAL;
    if (!device_ok(a.device)) return STAGE_EINVAL;
    DeviceGuard dg(a.device);
    const WindowArgs w = window_args(a, workspace);
    const int rc = workspace_ok(workspace, workspace_bytes, window_workspace(w));
    if (rc != STAGE_OK || a.rows == 0) return rc;
    return status(launch_window_attention(w, static_cast<hipStream_t>(stream)));
}

int stage_adapter_workspace(const stage_adapter_args *a, int64_t *bytes) {
    if (!a || !bytes || !adapter_sizes(*a) || !device_ok(a->device)) return STAGE_EINVAL;
    DeviceGuard dg(a->device);
    *bytes = (int64_t)adapter_workspace(adapter_args(*a, nullptr));
    return STAGE_OK;
}

int stage_adapter_add(const stage_adapter_args *p, void *workspace, int64_t workspace_bytes, void *stream) {
    if (!p) return STAGE_EINVAL;
    const stage_adapter_args &a = *p;
    if (!adapter_sizes(a) || !rows_ok(a.x, a.x_ld, a.k, a.type) || !rows_ok(a.base, a.base_ld, a.n, a.type) ||
        !rows_ok(a.out, a.out_ld, a.n, a.type) || !a.a || !a.b || !on16(a.a) || !on16(a.b) || !a.ids)
        return STAGE_EINVAL;
    if ((a.out == a.base && a.out_ld != a.base_ld) || a.base_ld > (int64_t(1) << 25)) return STAGE_EINVAL;   // (16 rows within 32 bits)
    if (!device_ok(a.device)) return STAGE_EINVAL;
    DeviceGuard dg(a.device);
    const AdapterArgs w = adapter_args(a, workspace);
    const int rc = workspace_ok(workspace, workspace_bytes, adapter_workspace(w));
    if (rc != STAGE_OK || a.rows == 0) return rc;
    return status(launch_adapter_add(w, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
