// kvx_host.h -- host-side checks shared by the entry points of libkvx: the
// thread's error message, descriptor and table checks, device views of the
// caller's pointers and the byte strides of a pool layout.
#pragma once

#include <hip/hip_runtime.h>
#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>

#include <string>

#include "kvx.h"
#include "kvx_internal.h"

namespace kvx {

inline thread_local std::string g_last_error;

inline int fail(int status, const char *fmt, ...) {
    char msg[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(msg, sizeof msg, fmt, ap);
    va_end(ap);
    g_last_error = msg;
    return status;
}

// a * b for non-negative operands, or -1 if the product exceeds int64.
inline int64_t mul_checked(int64_t a, int64_t b) {
    if (a < 0 || b < 0) return -1;
    if (a != 0 && b > INT64_MAX / a) return -1;
    return a * b;
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Element shape shared by both sides of a call.
struct Shape {
    int32_t L, C, H, D, e;
};

inline int check_shape(const char *name, const Shape &s) {
    if (s.L < 1 || s.H < 1 || s.D < 1)
        return fail(KVX_ERR_SHAPE, "%s: num_layers, num_heads and head_dim must be >= 1", name);
    if (s.C != 1 && s.C != 2) return fail(KVX_ERR_LAYOUT, "%s: num_kv must be 1 or 2 (got %d)", name, s.C);
    if (s.e != 1 && s.e != 2 && s.e != 4 && s.e != 8)
        return fail(KVX_ERR_SHAPE, "%s: elem_bytes must be 1, 2, 4 or 8 (got %d)", name, s.e);
    const int64_t row = (int64_t)s.D * s.e;
    if (row % 16 != 0)
        return fail(KVX_ERR_ALIGN, "%s: head_dim * elem_bytes = %lld is not a multiple of 16", name,
                    (long long)row);
    const int64_t token = mul_checked(mul_checked(mul_checked(s.L, s.C), s.H), row);
    if (token < 0 || token > (int64_t(1) << 31))
        return fail(KVX_ERR_SHAPE, "%s: one token spans more than 2 GiB across all layers", name);
    return KVX_OK;
}

inline int pool_shape(const kvx_pool *p, const char *name, Shape &s) {
    if (!p) return fail(KVX_ERR_NULL, "%s: pool descriptor is NULL", name);
    s = Shape{p->num_layers, p->num_kv, p->num_heads, p->head_dim, p->elem_bytes};
    int st = check_shape(name, s);
    if (st) return st;
    if (p->layout < KVX_LPCTHD || p->layout > KVX_PLCHTD)
        return fail(KVX_ERR_LAYOUT, "%s: unknown layout %d", name, p->layout);
    if (p->page_tokens < 1 || p->page_tokens > KVX_MAX_PAGE_TOKENS)
        return fail(KVX_ERR_SHAPE, "%s: page_tokens %d outside [1, %d]", name, p->page_tokens,
                    KVX_MAX_PAGE_TOKENS);
    if (p->num_pages < 1) return fail(KVX_ERR_SHAPE, "%s: num_pages must be >= 1", name);
    // A tile (one page of one layer) must stay below 2^31 16-byte vectors.
    const int64_t tile_vecs = (int64_t)s.C * p->page_tokens * s.H * (s.D * s.e / 16);
    if (tile_vecs >= (int64_t(1) << 31))
        return fail(KVX_ERR_SHAPE, "%s: one page of one layer exceeds 32 GiB", name);
    return KVX_OK;
}

inline int64_t pool_bytes(const kvx_pool *p) {
    int64_t b = mul_checked(mul_checked(mul_checked(p->num_layers, p->num_kv), p->num_heads),
                            (int64_t)p->head_dim * p->elem_bytes);
    b = mul_checked(mul_checked(b, p->page_tokens), p->num_pages);
    return b;
}

inline int same_shape(const Shape &a, const Shape &b) {
    if (a.L != b.L || a.C != b.C || a.H != b.H || a.D != b.D || a.e != b.e)
        return fail(KVX_ERR_SHAPE,
                    "source and destination differ in element shape: (L,C,H,D,e) = "
                    "(%d,%d,%d,%d,%d) vs (%d,%d,%d,%d,%d)",
                    a.L, a.C, a.H, a.D, a.e, b.L, b.C, b.H, b.D, b.e);
    return KVX_OK;
}

// Device allocations that pointers of this call were found in.  Small inputs
// (tables, records, the error word) often share one, and each look-up of a
// pointer costs the call 0.2-0.4 us.
struct Known {
    struct {
        uintptr_t lo, hi;
    } a[4];
    int n = 0;
};

// `need` bytes from p on lie before the end of the allocation.
inline int check_extent(const char *name, const void *ptr, int64_t need, uintptr_t lo, uintptr_t hi) {
    const uintptr_t p = reinterpret_cast<uintptr_t>(ptr);
    if (need <= 0 || (p >= lo && p < hi && (uint64_t)(hi - p) >= (uint64_t)need)) return KVX_OK;
    return fail(KVX_ERR_RANGE,
                "%s (%p) needs %lld bytes, but its allocation [%p, +%zu) ends %lld "
                "bytes after it",
                name, ptr, (long long)need, reinterpret_cast<void *>(lo), (size_t)(hi - lo),
                (long long)(p < hi && p >= lo ? (int64_t)(hi - p) : 0));
}

// The device must be able to address `ptr` (device memory or mapped pinned
// host memory), and the allocation it points into must hold the `need`
// bytes from `ptr` on that the call may touch.  On success *dev_ptr is the
// address kernels use and *is_host (if given) tells whether it is host
// memory.  With `device_only` pinned host memory is refused too.
inline int device_view(const void *ptr, int64_t need, const char *name, void **dev_ptr, Known &known,
                bool *is_host = nullptr, bool device_only = false) {
    const uintptr_t p = reinterpret_cast<uintptr_t>(ptr);
    for (int k = 0; k < known.n; ++k)
        if (p >= known.a[k].lo && p < known.a[k].hi) {        // memory of the current device
            *dev_ptr = const_cast<void *>(ptr);
            if (is_host) *is_host = false;
            return check_extent(name, ptr, need, known.a[k].lo, known.a[k].hi);
        }
    hipPointerAttribute_t attr;
    hipError_t e = hipPointerGetAttributes(&attr, ptr);
    if (e != hipSuccess) {
        (void)hipGetLastError();  // clear the sticky error the query leaves
        return fail(KVX_ERR_RANGE, "%s (%p) is not memory the GPU can address (%s)", name, ptr,
                    hipGetErrorString(e));
    }
    const bool dev_mem = attr.type == hipMemoryTypeDevice || attr.type == hipMemoryTypeManaged ||
                         attr.type == hipMemoryTypeUnified;
    const bool host_mem = attr.type == hipMemoryTypeHost && attr.devicePointer;
    if (!dev_mem && !host_mem)
        return fail(KVX_ERR_RANGE, "%s (%p) is not device memory or mapped pinned host memory",
                    name, ptr);
    if (device_only && !dev_mem)
        return fail(KVX_ERR_RANGE, "%s (%p) must be device memory (pinned host memory is refused)",
                    name, ptr);
    if (attr.type == hipMemoryTypeDevice) {
        // Device memory of another GPU would fault the kernel unless peer
        // access happened to be enabled; this library runs on one GPU.
        int cur = 0;
        const hipError_t ge = hipGetDevice(&cur);
        if (ge != hipSuccess)
            return fail(KVX_ERR_HIP, "hipGetDevice failed: %s", hipGetErrorString(ge));
        if (attr.device != cur)
            return fail(KVX_ERR_RANGE, "%s (%p) is memory of device %d, but the current device is %d",
                        name, ptr, attr.device, cur);
    }
    if (need > 0) {
        // The allocation around `ptr` must reach `need` bytes past it: a
        // descriptor larger than its memory would make the kernel read or
        // write outside the allocation.  Where the runtime reports no
        // allocation range for the pointer, the extent cannot be checked.
        hipDeviceptr_t lo = nullptr;
        size_t size = 0;
        const hipError_t re = hipMemGetAddressRange(&lo, &size, const_cast<void *>(ptr));
        if (re != hipSuccess) {
            (void)hipGetLastError();
        } else {
            const uintptr_t a = reinterpret_cast<uintptr_t>(lo);
            const int st = check_extent(name, ptr, need, a, a + size);
            if (st) return st;
            if (attr.type == hipMemoryTypeDevice && known.n < 4) {
                known.a[known.n].lo = a;
                known.a[known.n++].hi = a + size;
            }
        }
    }
    *dev_ptr = dev_mem ? const_cast<void *>(ptr) : attr.devicePointer;
    if (is_host) *is_host = !dev_mem;
    return KVX_OK;
}

// Byte strides of (layer, page, kv, slot, head) for a pool layout, with the
// base moved to (layer0, kv0, head0) of the range the call copies; `heads`
// is how many heads it copies.
inline Side pool_side(const kvx_pool *p, void *base, const int32_t *pt, int64_t pt_len,
                    int32_t layer0, int32_t kv0, int32_t head0, int32_t heads) {
    const int64_t row = (int64_t)p->head_dim * p->elem_bytes;
    const int64_t L = p->num_layers, N = p->num_pages, C = p->num_kv, T = p->page_tokens,
                  H = p->num_heads;
    Side s{};
    const bool token_major = p->layout == KVX_LPCTHD || p->layout == KVX_PLCTHD;
    if (token_major) {
        s.s_h = row;
        s.s_t = H * row;
    } else {
        s.s_t = row;
        s.s_h = T * row;
    }
    s.s_c = T * H * row;
    if (p->layout == KVX_LPCTHD || p->layout == KVX_LPCHTD) {
        s.s_p = C * s.s_c;
        s.s_l = N * s.s_p;
    } else {
        s.s_l = C * s.s_c;
        s.s_p = L * s.s_l;
    }
    s.base = static_cast<char *>(base) + layer0 * s.s_l + kv0 * s.s_c + head0 * s.s_h;
    s.pt = pt;
    s.pt_len = pt_len;
    s.T = p->page_tokens;
    s.N = p->num_pages;
    // The copied heads of consecutive slots form one run when each slot's
    // copied rows are adjacent and slots follow each other without a gap.
    s.tok_contig = s.s_t == heads * row && (heads == 1 || s.s_h == row);
    s.cap_bytes = 0;
    return s;
}

inline Side buf_side(const kvx_buf *b, void *base) {
    Side s{};
    s.base = static_cast<char *>(base);
    s.tok_contig = 1;
    s.T = 1;
    s.N = 0;
    s.cap_bytes = b->capacity_elems * b->elem_bytes;
    return s;
}

// Host-only checks of a pool descriptor (no HIP call).
inline int check_pool(const kvx_pool *p, const char *name, Shape &s) {
    int st = pool_shape(p, name, s);
    if (st) return st;
    if (!p->base) return fail(KVX_ERR_NULL, "%s: base is NULL", name);
    if (!aligned16(p->base)) return fail(KVX_ERR_ALIGN, "%s: base %p is not 16-byte aligned", name, p->base);
    if (pool_bytes(p) < 0) return fail(KVX_ERR_RANGE, "%s: pool size exceeds 2^63 bytes", name);
    return KVX_OK;
}

// Host-only checks of a buffer descriptor.
inline int check_buf(const kvx_buf *b, const char *name, Shape &s) {
    if (!b) return fail(KVX_ERR_NULL, "%s: buffer descriptor is NULL", name);
    s = Shape{b->num_layers, b->num_kv, b->num_heads, b->head_dim, b->elem_bytes};
    int st = check_shape(name, s);
    if (st) return st;
    if (b->reserved != 0) return fail(KVX_ERR_RANGE, "%s: reserved field must be 0", name);
    // An empty buffer may have no memory at all: no record can then address it.
    if (!b->base && b->capacity_elems != 0) return fail(KVX_ERR_NULL, "%s: base is NULL", name);
    if (!aligned16(b->base)) return fail(KVX_ERR_ALIGN, "%s: base %p is not 16-byte aligned", name, b->base);
    if (b->capacity_elems < 0 || mul_checked(b->capacity_elems, b->elem_bytes) < 0)
        return fail(KVX_ERR_RANGE, "%s: capacity_elems out of range", name);
    return KVX_OK;
}

// Host-only checks of a page table.
inline int check_table(const int32_t *pt, int64_t len, const char *name) {
    if (len < 0 || len > INT64_MAX / 4) return fail(KVX_ERR_RANGE, "%s: length %lld out of range", name,
                                                    (long long)len);
    if (len > 0 && !pt) return fail(KVX_ERR_NULL, "%s is NULL but has %lld entries", name, (long long)len);
    if ((reinterpret_cast<uintptr_t>(pt) & 3u) != 0) return fail(KVX_ERR_ALIGN, "%s is not 4-byte aligned", name);
    return KVX_OK;
}

// Host-only checks of the record array and the error word.
inline int check_common(const kvx_req *reqs, int32_t n_reqs, uint32_t *dev_err) {
    if (n_reqs < 0 || n_reqs > KVX_MAX_REQS)
        return fail(KVX_ERR_RANGE, "n_reqs %d outside [0, %d]", n_reqs, KVX_MAX_REQS);
    if (n_reqs > 0 && !reqs) return fail(KVX_ERR_NULL, "reqs is NULL");
    if ((reinterpret_cast<uintptr_t>(reqs) & 7u) != 0) return fail(KVX_ERR_ALIGN, "reqs is not 8-byte aligned");
    if ((reinterpret_cast<uintptr_t>(dev_err) & 3u) != 0)
        return fail(KVX_ERR_ALIGN, "dev_err is not 4-byte aligned");
    return KVX_OK;
}

// Device views of every pointer a launch uses.
struct Views {
    void *src = nullptr, *dst = nullptr;
    bool src_host = false, dst_host = false;
    const int32_t *src_pt = nullptr, *dst_pt = nullptr;
    const kvx_req *reqs = nullptr;
    uint32_t *err = nullptr;
    Known known;
};

inline int view_all(const void *src, int64_t src_bytes, const void *dst, int64_t dst_bytes,
             const int32_t *src_pt, int64_t src_pt_len, const int32_t *dst_pt, int64_t dst_pt_len,
             const kvx_req *reqs, int32_t n_reqs, uint32_t *dev_err, Views &v) {
    int st;
    void *d = nullptr;
    // A NULL base here is an empty buffer (pools are never NULL): nothing to view.
    if (src && (st = device_view(src, src_bytes, "src base", &v.src, v.known, &v.src_host))) return st;
    if (dst && (st = device_view(dst, dst_bytes, "dst base", &v.dst, v.known, &v.dst_host))) return st;
    if (src_pt_len > 0) {
        if ((st = device_view(src_pt, src_pt_len * 4, "src_pt", &d, v.known))) return st;
        v.src_pt = static_cast<const int32_t *>(d);
    }
    if (dst_pt_len > 0) {
        if ((st = device_view(dst_pt, dst_pt_len * 4, "dst_pt", &d, v.known))) return st;
        v.dst_pt = static_cast<const int32_t *>(d);
    }
    if ((st = device_view(reqs, (int64_t)n_reqs * (int64_t)sizeof(kvx_req), "reqs", &d, v.known))) return st;
    v.reqs = static_cast<const kvx_req *>(d);
    if (dev_err) {
        // Bits are OR-ed in with device atomics, which pinned host memory
        // does not support on every platform: the word lives in device memory.
        if ((st = device_view(dev_err, 4, "dev_err", &d, v.known, nullptr, /*device_only=*/true))) return st;
        v.err = static_cast<uint32_t *>(d);
    }
    return KVX_OK;
}

// A slice's ranges must lie inside both pools; rows must have the same
// width on both sides.
inline int check_slice(const kvx_slice &sl, const Shape &s, const Shape &d) {
    if (s.D != d.D || s.e != d.e)
        return fail(KVX_ERR_SHAPE, "head_dim/elem_bytes differ: (%d, %d) vs (%d, %d)", s.D, s.e,
                    d.D, d.e);
    if (sl.reserved != 0) return fail(KVX_ERR_RANGE, "slice: reserved field must be 0");
    const struct {
        const char *what;
        int32_t s0, d0, n, smax, dmax;
    } r[3] = {{"layer", sl.src_layer0, sl.dst_layer0, sl.num_layers, s.L, d.L},
              {"kv", sl.src_kv0, sl.dst_kv0, sl.num_kv, s.C, d.C},
              {"head", sl.src_head0, sl.dst_head0, sl.num_heads, s.H, d.H}};
    for (const auto &x : r) {
        if (x.n < 0 || x.s0 < 0 || x.d0 < 0 || (int64_t)x.s0 + x.n > x.smax ||
            (int64_t)x.d0 + x.n > x.dmax)
            return fail(KVX_ERR_RANGE,
                        "slice %s range: src [%d, %lld) of %d, dst [%d, %lld) of %d", x.what, x.s0,
                        (long long)x.s0 + x.n, x.smax, x.d0, (long long)x.d0 + x.n, x.dmax);
    }
    return KVX_OK;
}

}  // namespace kvx
