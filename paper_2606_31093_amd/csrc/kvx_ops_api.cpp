// kvx_ops_api.cpp -- the C-ABI of the calls that compute with a paged cache
// (include/kvx.h, "A decode step"): host-side validation, the device's view
// of every pointer, and the launch on the caller's stream.

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>

#include "kvx.h"
#include "kvx_host.h"
#include "kvx_ops.h"

using namespace kvx;

namespace {

// The pool as the computing calls take it: elements of 16 bits, or 8 (e4m3).
int check_values(const kvx_pool *pool, int32_t layer, const float *scales, Shape &s) {
    int st;
    if ((st = check_pool(pool, "pool", s))) return st;
    if (s.e != 1 && s.e != 2)
        return fail(KVX_ERR_SHAPE, "pool: elem_bytes must be 2 (the rows' type) or 1 (e4m3), got %d", s.e);
    if (layer < 0 || layer >= s.L) return fail(KVX_ERR_RANGE, "layer %d outside [0, %d)", layer, s.L);
    if (scales && s.e != 1) return fail(KVX_ERR_SHAPE, "scales are for e4m3 pools (elem_bytes 1)");
    if ((reinterpret_cast<uintptr_t>(scales) & 3u) != 0) return fail(KVX_ERR_ALIGN, "scales is not 4-byte aligned");
    return KVX_OK;
}

int check_records(const void *reqs, int32_t n_reqs, int32_t max_tokens, uint32_t *dev_err) {
    const int st = check_common(static_cast<const kvx_req *>(reqs), n_reqs, dev_err);
    if (st) return st;
    if (max_tokens < 0 || max_tokens > KVX_MAX_TOKENS)
        return fail(KVX_ERR_RANGE, "max_tokens %d outside [0, %d]", max_tokens, KVX_MAX_TOKENS);
    return KVX_OK;
}

// Bytes from base to the end of the last row; -1 if they overflow.
int64_t rows_bytes(const kvx_rows *x) {
    if (x->num_rows == 0 || x->num_heads == 0) return 0;
    const int64_t a = mul_checked(x->num_rows - 1, x->row_stride), b = mul_checked(x->num_heads - 1, x->head_stride);
    if (a < 0 || b < 0 || a > (int64_t(1) << 60) || b > (int64_t(1) << 60)) return -1;
    return (a + b + x->head_dim) * 2;
}

int check_rows(const kvx_rows *x, const char *name) {
    if (!x) return fail(KVX_ERR_NULL, "%s: rows are NULL", name);
    if (x->reserved != 0) return fail(KVX_ERR_RANGE, "%s: reserved field must be 0", name);
    if (x->dtype != KVX_BF16 && x->dtype != KVX_F16)
        return fail(KVX_ERR_SHAPE, "%s: dtype must be KVX_BF16 or KVX_F16 (got %d)", name, x->dtype);
    if (x->num_rows < 0 || x->num_heads < 1 || x->head_dim < 1)
        return fail(KVX_ERR_SHAPE, "%s: num_heads and head_dim must be >= 1, num_rows >= 0", name);
    if (x->row_stride < 0 || x->head_stride < 0) return fail(KVX_ERR_RANGE, "%s: strides must be >= 0", name);
    if (x->row_stride % 8 || x->head_stride % 8 || x->head_dim % 8)
        return fail(KVX_ERR_ALIGN, "%s: strides and head_dim must be multiples of 8 elements", name);
    if (!aligned16(x->base)) return fail(KVX_ERR_ALIGN, "%s: base %p is not 16-byte aligned", name, x->base);
    const int64_t bytes = rows_bytes(x);
    if (bytes < 0) return fail(KVX_ERR_RANGE, "%s: rows exceed 2^61 bytes", name);
    if (bytes > 0 && !x->base) return fail(KVX_ERR_NULL, "%s: base is NULL", name);
    return KVX_OK;
}

// The first n rows of an output, which wavefronts write in any order, share no element:
// |i * row_stride - j * head_stride| >= head_dim for all i < n and j < num_heads but 0, 0.
int check_apart(const kvx_rows *x, int64_t n, const char *name) {
    const int64_t a = x->row_stride, b = x->head_stride, D = x->head_dim, m = x->num_heads;
    bool apart = (n <= 1 || a >= D) && (m <= 1 || b >= D);
    if (apart && n > 1 && m > 1 && a < (m - 1) * b + D && b < (n - 1) * a + D) {
        // neither do rows hold all heads nor heads all rows: the rows next to each head
        for (int64_t j = 1; j < m && apart; ++j) {
            const int64_t i = j * b / a;
            apart = (i >= n || j * b - i * a >= D) && (i + 1 >= n || (i + 1) * a - j * b >= D);
        }
    }
    return apart ? KVX_OK
                 : fail(KVX_ERR_RANGE, "%s: rows of %lld elements share elements (row_stride %lld, head_stride %lld)", name,
                        (long long)D, (long long)a, (long long)b);
}

int view_rows(const kvx_rows *x, const char *name, bool device_only, Known &known, Rows &out) {
    const int64_t bytes = rows_bytes(x);
    void *d = nullptr;
    int st;
    if (bytes > 0 && (st = device_view(x->base, bytes, name, &d, known, nullptr, device_only))) return st;
    out = Rows{static_cast<char *>(d), x->row_stride * 2, x->head_stride * 2, x->num_heads};
    return KVX_OK;
}

// A required or optional array: its device address (nullptr if there is none).
template <typename T>
int view(T *ptr, int64_t bytes, const char *name, bool device_only, Known &known, T **out) {
    *out = nullptr;
    if (!ptr || bytes == 0) return KVX_OK;
    void *d = nullptr;
    const int st = device_view(ptr, bytes, name, &d, known, nullptr, device_only);
    *out = static_cast<T *>(d);
    return st;
}

// The layer of a pool whose memory, table and scales are viewed; an output
// pool must be device memory.
int view_layer(const kvx_pool *pool, int32_t layer, const int32_t *pt, int64_t pt_len, bool output, Known &known,
               Layer &out) {
    char *base;
    const int32_t *table;
    int st;
    if ((st = view(static_cast<char *>(pool->base), pool_bytes(pool), "pool base", output, known, &base))) return st;
    if ((st = view(pt, pt_len * 4, "pt", false, known, &table))) return st;
    const Side s = pool_side(pool, base, table, pt_len, layer, 0, 0, pool->num_heads);
    out = Layer{s.base, s.s_p, s.s_c, s.s_t, s.s_h, table, pt_len, pool->num_pages, pool->num_kv, pool->num_heads,
                pool->head_dim, make_fastdiv((uint32_t)pool->page_tokens)};
    return KVX_OK;
}

bool token_major(const kvx_pool *pool) { return pool->layout == KVX_LPCTHD || pool->layout == KVX_PLCTHD; }

int launched(int e) {
    return e == hipSuccess ? KVX_OK
                           : fail(KVX_ERR_HIP, "kernel launch failed: %s", hipGetErrorString((hipError_t)e));
}

// Lengths and strides of accumulators and lists.
int check_array(const void *ptr, int64_t len, int64_t stride, const char *name) {
    if (len < 0 || len > INT64_MAX / 4 || stride < 0)
        return fail(KVX_ERR_RANGE, "%s: length %lld or stride %lld out of range", name, (long long)len,
                    (long long)stride);
    if (len > 0 && !ptr) return fail(KVX_ERR_NULL, "%s is NULL but has %lld elements", name, (long long)len);
    if ((reinterpret_cast<uintptr_t>(ptr) & 3u) != 0) return fail(KVX_ERR_ALIGN, "%s is not 4-byte aligned", name);
    return KVX_OK;
}

// The shapes that kvx_attend serves.
int check_attend(const Shape &s, int32_t n_reqs, int32_t q_heads, int32_t v_dim) {
    if (n_reqs < 0 || n_reqs > KVX_MAX_REQS)
        return fail(KVX_ERR_RANGE, "n_reqs %d outside [0, %d]", n_reqs, KVX_MAX_REQS);
    if (s.e != 1 && s.e != 2) return fail(KVX_ERR_SHAPE, "pool: elem_bytes must be 2 or 1 (got %d)", s.e);
    if (q_heads < 1 || q_heads > 1024 || q_heads % s.H)
        return fail(KVX_ERR_SHAPE, "%d query heads: a multiple of the pool's %d up to 1024 is needed", q_heads, s.H);
    if (s.D > 576 || v_dim < 1 || v_dim > 512 || v_dim > s.D || v_dim % 8 || (s.C == 2 && v_dim != s.D))
        return fail(KVX_ERR_SHAPE, "head_dim %d (at most 576) with v_dim %d (a multiple of 8 up to 512 and head_dim, "
                    "equal to it when num_kv is 2)", s.D, v_dim);
    return KVX_OK;
}

}  // namespace

extern "C" {

int kvx_append(const kvx_pool *pool, int32_t layer, const float *scales, const kvx_rows *q, const kvx_rows *q_out,
               const kvx_rows *k, const kvx_rows *v, const kvx_rope *rope, const int32_t *pt, int64_t pt_len,
               const kvx_append_req *reqs, int32_t n_reqs, int32_t max_tokens, uint32_t *dev_err, void *stream) {
    g_last_error.clear();
    Shape s;
    int st;
    if ((st = check_values(pool, layer, scales, s))) return st;
    if ((st = check_rows(k, "k"))) return st;
    if (k->num_heads != s.H || k->head_dim != s.D)
        return fail(KVX_ERR_SHAPE, "k has %d heads of %d, the pool %d of %d", k->num_heads, k->head_dim, s.H, s.D);
    if (s.C == 2) {
        if ((st = check_rows(v, "v"))) return st;
        if (v->num_heads != s.H || v->head_dim != s.D || v->dtype != k->dtype || v->num_rows != k->num_rows)
            return fail(KVX_ERR_SHAPE, "v differs from k in heads, head_dim, dtype or rows");
    } else if (v) {
        return fail(KVX_ERR_SHAPE, "v must be NULL for a pool of num_kv 1");
    }
    if (!q != !q_out) return fail(KVX_ERR_NULL, "q and q_out: both or neither");
    if (q) {
        if ((st = check_rows(q, "q"))) return st;
        if ((st = check_rows(q_out, "q_out"))) return st;
        if (q->head_dim != s.D || q->dtype != k->dtype || q->num_rows != k->num_rows)
            return fail(KVX_ERR_SHAPE, "q differs from k in head_dim, dtype or rows");
        if (q_out->num_heads != q->num_heads || q_out->head_dim != q->head_dim || q_out->dtype != q->dtype ||
            q_out->num_rows != q->num_rows)
            return fail(KVX_ERR_SHAPE, "q_out differs from q in heads, head_dim, dtype or rows");
        if ((st = check_apart(q_out, q_out->num_rows, "q_out"))) return st;
    }
    if (((int64_t)(q ? q->num_heads : 0) + 2 * s.H) * s.D > (1 << 26))
        return fail(KVX_ERR_SHAPE, "a token's rows hold more than 2^26 elements");
    const int32_t rot = rope ? rope->rot_dim : 0;
    if (rope) {
        if (rot < 0 || rot % 2 || rope->rot_off < 0 || (int64_t)rope->rot_off + rot > s.D || rot > 16384)
            return fail(KVX_ERR_SHAPE, "rope: rot_dim %d (even, at most 16384) from rot_off %d in a head_dim of %d", rot,
                        rope->rot_off, s.D);
        if (rope->interleaved != 0 && rope->interleaved != 1)
            return fail(KVX_ERR_RANGE, "rope: interleaved must be 0 or 1 (got %d)", rope->interleaved);
        if (rot > 0 && !rope->freq) return fail(KVX_ERR_NULL, "rope: freq is NULL");
        if ((reinterpret_cast<uintptr_t>(rope->freq) & 3u) != 0)
            return fail(KVX_ERR_ALIGN, "rope: freq is not 4-byte aligned");
    }
    if ((st = check_records(reqs, n_reqs, max_tokens, dev_err))) return st;
    if ((st = check_table(pt, pt_len, "pt"))) return st;
    if (n_reqs == 0) return KVX_OK;
    AppendParams P{};
    Known known;
    if ((st = view_layer(pool, layer, pt, pt_len, true, known, P.pool))) return st;
    if ((st = view(scales, (int64_t)s.C * s.H * 4, "scales", false, known, &P.scales))) return st;
    if (q && (st = view_rows(q, "q", false, known, P.q))) return st;
    if (q && (st = view_rows(q_out, "q_out", true, known, P.q_out))) return st;
    if ((st = view_rows(k, "k", false, known, P.k))) return st;
    if (v && (st = view_rows(v, "v", false, known, P.v))) return st;
    if (rot && (st = view(rope->freq, (int64_t)rot / 2 * 4, "rope freq", false, known, &P.freq))) return st;
    if ((st = view(reqs, (int64_t)n_reqs * (int64_t)sizeof *reqs, "reqs", false, known, &P.reqs))) return st;
    if ((st = view(dev_err, 4, "dev_err", true, known, &P.err))) return st;
    P.num_rows = k->num_rows;
    P.half = rot / 2;
    P.rot_off = rope ? rope->rot_off : 0;
    P.interleaved = rope ? rope->interleaved : 0;
    P.amplitude = rope ? rope->amplitude : 1.f;
    P.n_reqs = n_reqs;
    P.max_tokens = max_tokens;
    P.f16 = k->dtype == KVX_F16;
    P.e4m3 = s.e == 1;
    return launched(launch_append(P, static_cast<hipStream_t>(stream)));
}

int64_t kvx_attend_workspace(const kvx_pool *pool, int32_t n_reqs, int32_t q_heads, int32_t v_dim,
                             int32_t max_tokens, int32_t accumulate) {
    g_last_error.clear();
    Shape s;
    if (pool_shape(pool, "pool", s) || check_attend(s, n_reqs, q_heads, v_dim)) return -1;
    if (max_tokens < 0 || max_tokens > KVX_MAX_TOKENS) {
        fail(KVX_ERR_RANGE, "max_tokens %d outside [0, %d]", max_tokens, KVX_MAX_TOKENS);
        return -1;
    }
    AttendParams P{};
    P.pool.C = s.C;
    P.pool.H = s.H;
    P.pool.D = s.D;
    P.G = q_heads / s.H;
    P.token_major = token_major(pool);
    P.e4m3 = s.e == 1;
    P.Dv = v_dim;
    P.n_reqs = n_reqs;
    P.max_tokens = max_tokens;
    float any = 0.f;
    P.acc = accumulate ? &any : nullptr;
    plan_attend(P);
    return attend_workspace(P, nullptr);
}

int kvx_attend(const kvx_pool *pool, int32_t layer, const float *scales, const kvx_rows *q, const kvx_rows *out,
               float *lse, float scale, const int32_t *pt, int64_t pt_len, const kvx_attend_req *reqs, int32_t n_reqs,
               int32_t max_tokens, float *acc, int64_t acc_len, int64_t acc_stride, void *workspace,
               int64_t workspace_bytes, uint32_t *dev_err, void *stream) {
    g_last_error.clear();
    Shape s;
    int st;
    if ((st = check_values(pool, layer, scales, s))) return st;
    if ((st = check_rows(q, "q"))) return st;
    if ((st = check_rows(out, "out"))) return st;
    if ((st = check_attend(s, n_reqs, q->num_heads, out->head_dim))) return st;
    if (q->head_dim != s.D) return fail(KVX_ERR_SHAPE, "q has head_dim %d, the pool %d", q->head_dim, s.D);
    if (out->num_heads != q->num_heads || out->dtype != q->dtype)
        return fail(KVX_ERR_SHAPE, "out differs from q in heads or dtype");
    if (q->num_rows < n_reqs || out->num_rows < n_reqs)
        return fail(KVX_ERR_RANGE, "q and out hold %lld and %lld rows for %d records", (long long)q->num_rows,
                    (long long)out->num_rows, n_reqs);
    if ((st = check_apart(out, n_reqs, "out"))) return st;
    if ((st = check_records(reqs, n_reqs, max_tokens, dev_err))) return st;
    if ((st = check_table(pt, pt_len, "pt"))) return st;
    if ((reinterpret_cast<uintptr_t>(lse) & 3u) != 0) return fail(KVX_ERR_ALIGN, "lse is not 4-byte aligned");
    if (acc && (st = check_array(acc, acc_len, acc_stride, "acc"))) return st;
    if (n_reqs == 0) return KVX_OK;
    AttendParams P{};
    P.pool.C = s.C;
    P.pool.H = s.H;
    P.pool.D = s.D;
    P.G = q->num_heads / s.H;
    P.token_major = token_major(pool);
    P.e4m3 = s.e == 1;
    P.Dv = out->head_dim;
    P.n_reqs = n_reqs;
    P.max_tokens = max_tokens;
    P.acc = acc;
    plan_attend(P);
    const int64_t need = attend_workspace(P, nullptr);
    if (!workspace) return fail(KVX_ERR_NULL, "workspace is NULL");
    if (!aligned16(workspace)) return fail(KVX_ERR_ALIGN, "workspace %p is not 16-byte aligned", workspace);
    if (workspace_bytes < need)
        return fail(KVX_ERR_RANGE, "workspace holds %lld bytes, this call needs %lld", (long long)workspace_bytes,
                    (long long)need);
    Known known;
    char *ws;
    if ((st = view_layer(pool, layer, pt, pt_len, false, known, P.pool))) return st;
    if ((st = view(scales, (int64_t)s.C * s.H * 4, "scales", false, known, &P.scales))) return st;
    if ((st = view_rows(q, "q", false, known, P.q))) return st;
    if ((st = view_rows(out, "out", true, known, P.out))) return st;
    if ((st = view(lse, (int64_t)n_reqs * q->num_heads * 4, "lse", true, known, &P.lse))) return st;
    if ((st = view(acc, acc_len * 4, "acc", true, known, &P.acc))) return st;
    if ((st = view(static_cast<char *>(workspace), need, "workspace", true, known, &ws))) return st;
    if ((st = view(reqs, (int64_t)n_reqs * (int64_t)sizeof *reqs, "reqs", false, known, &P.reqs))) return st;
    if ((st = view(dev_err, 4, "dev_err", true, known, &P.err))) return st;
    // the kernel reads an entry for every position, also where none is in range
    if (!P.pool.pt) P.pool.pt = reinterpret_cast<const int32_t *>(P.reqs);
    P.acc_len = acc_len;
    P.acc_stride = acc_stride;
    if (acc && !P.acc) P.acc = acc;      // no elements: every record with positions is malformed
    (void)attend_workspace(P, ws);
    P.scale_log2 = scale * 1.4426950408889634f;
    P.f16 = q->dtype == KVX_F16;
    return launched(launch_attend(P, static_cast<hipStream_t>(stream)));
}

int kvx_select_kept(const float *acc, int64_t acc_len, int64_t acc_stride, int32_t rows, const kvx_select_req *reqs,
                    int32_t n_reqs, int32_t max_tokens, int32_t *kept, int64_t kept_len, int64_t kept_stride,
                    float *acc_out, int64_t acc_out_len, int64_t acc_out_stride, uint32_t *dev_err, void *stream) {
    g_last_error.clear();
    int st;
    if (rows < 1 || rows > (1 << 20)) return fail(KVX_ERR_RANGE, "rows %d outside [1, %d]", rows, 1 << 20);
    if ((st = check_array(acc, acc_len, acc_stride, "acc"))) return st;
    if ((st = check_array(kept, kept_len, kept_stride, "kept"))) return st;
    if (acc_out && (st = check_array(acc_out, acc_out_len, acc_out_stride, "acc_out"))) return st;
    if ((st = check_records(reqs, n_reqs, max_tokens, dev_err))) return st;
    if (n_reqs == 0) return KVX_OK;
    SelectParams P{};
    Known known;
    if ((st = view(acc, acc_len * 4, "acc", false, known, &P.acc))) return st;
    if ((st = view(kept, kept_len * 4, "kept", true, known, &P.kept))) return st;
    if ((st = view(acc_out, acc_out_len * 4, "acc_out", true, known, &P.out))) return st;
    if ((st = view(reqs, (int64_t)n_reqs * (int64_t)sizeof *reqs, "reqs", false, known, &P.reqs))) return st;
    if ((st = view(dev_err, 4, "dev_err", true, known, &P.err))) return st;
    if (acc_out && !P.out) P.out = acc_out;      // no elements: only empty records are well formed
    P.acc_len = acc_len;
    P.acc_stride = acc_stride;
    P.rows = rows;
    P.n_reqs = n_reqs;
    P.max_tokens = max_tokens;
    P.kept_len = kept_len;
    P.kept_stride = kept_stride;
    P.out_len = acc_out_len;
    P.out_stride = acc_out_stride;
    return launched(launch_select(P, static_cast<hipStream_t>(stream)));
}

int kvx_transfer_kept(const kvx_pool *src, const kvx_pool *dst, const kvx_slice *slice, const int32_t *src_pt,
                      int64_t src_pt_len, const int32_t *dst_pt, int64_t dst_pt_len, const kvx_req *reqs,
                      int32_t n_reqs, int32_t max_tokens, const int32_t *kept, int64_t kept_len, int64_t kept_stride,
                      uint32_t *dev_err, void *stream) {
    g_last_error.clear();
    Shape ss, ds;
    int st;
    if ((st = check_pool(src, "src", ss))) return st;
    if ((st = check_pool(dst, "dst", ds))) return st;
    kvx_slice sl;
    if (slice) {
        sl = *slice;
        if ((st = check_slice(sl, ss, ds))) return st;
    } else {
        if ((st = same_shape(ss, ds))) return st;
        sl = kvx_slice{0, 0, ss.L, 0, 0, ss.C, 0, 0, ss.H, 0};
    }
    if ((st = check_records(reqs, n_reqs, max_tokens, dev_err))) return st;
    if ((st = check_table(src_pt, src_pt_len, "src_pt"))) return st;
    if ((st = check_table(dst_pt, dst_pt_len, "dst_pt"))) return st;
    if ((st = check_array(kept, kept_len, kept_stride, "kept"))) return st;
    if ((int64_t)sl.num_layers * sl.num_heads > (1 << 20))
        return fail(KVX_ERR_RANGE, "%lld lists a record: at most %d",
                    (long long)sl.num_layers * sl.num_heads, 1 << 20);
    if (n_reqs == 0 || sl.num_layers == 0 || sl.num_kv == 0 || sl.num_heads == 0) return KVX_OK;
    Views v;
    if ((st = view_all(src->base, pool_bytes(src), dst->base, pool_bytes(dst), src_pt, src_pt_len, dst_pt, dst_pt_len,
                       reqs, n_reqs, dev_err, v)))
        return st;
    KeptParams P{};
    if ((st = view(kept, kept_len * 4, "kept", false, v.known, &P.kept))) return st;
    P.src = pool_side(src, v.src, v.src_pt, src_pt_len, sl.src_layer0, sl.src_kv0, sl.src_head0, sl.num_heads);
    P.dst = pool_side(dst, v.dst, v.dst_pt, dst_pt_len, sl.dst_layer0, sl.dst_kv0, sl.dst_head0, sl.num_heads);
    P.reqs = v.reqs;
    P.n_reqs = n_reqs;
    P.max_tokens = max_tokens;
    P.L = sl.num_layers;
    P.C = sl.num_kv;
    P.H = sl.num_heads;
    P.vpr = (int32_t)((int64_t)ss.D * ss.e / 16);      // rows of up to 2 GiB
    P.kept_len = kept_len;
    P.kept_stride = kept_stride;
    P.err = v.err;
    P.fd_Ts = make_fastdiv((uint32_t)P.src.T);
    P.fd_Td = make_fastdiv((uint32_t)P.dst.T);
    P.fd_vpr = make_fastdiv((uint32_t)P.vpr);
    return launched(launch_kept(P, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
