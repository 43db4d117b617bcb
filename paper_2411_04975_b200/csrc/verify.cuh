// What the kernels of the verifier's side of a step share: the rows of a request, the types of a cache, checks of arguments.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

struct Request {
    long long begin;          // first row in the row arrays
    int count;                // rows; 0: idle, or its numbers make no sense
    int cached;               // places before them
    int status;
};

// Rows of request i.  `need_table`: its places have to lie inside its table.
__device__ __forceinline__ Request sd_request(const sd_rows& b, int i, long long page_size, int shared = 0) {
    Request r;
    const long long lo = b.d_offsets[i], hi = b.d_offsets[i + 1];
    r.begin = lo; r.cached = b.d_cached[i]; r.status = 0; r.count = (int)(hi - lo);
    if (hi == lo && lo >= 0 && lo <= b.rows) { r.count = 0; r.cached = 0; return r; }
    if (lo < 0 || hi < lo || hi > b.rows || hi - lo > b.max_draft + 1 || r.cached < shared || r.cached < 0 ||
        (long long)r.cached + (hi - lo) > page_size * b.table_stride) {
        r.count = 0; r.cached = 0; r.status = SD_STATUS_BAD_ROWS;
    }
    return r;
}

// Bit j: row sees draft node j of its request (row 0: none; without a mask all before it and itself).
__device__ __forceinline__ unsigned long long sd_tree_bits(const sd_rows& b, int i, int row) {
    if (row == 0) return 0ull;
    if (!b.d_mask) return row >= 64 ? ~0ull : (1ull << row) - 1;
    const int words = (b.max_draft + 31) >> 5;
    const uint32_t* m = b.d_mask + ((long long)i * b.max_draft + row - 1) * words;
    unsigned long long bits = m[0];
    if (words > 1) bits |= (unsigned long long)m[1] << 32;
    return b.max_draft >= 64 ? bits : bits & ((1ull << b.max_draft) - 1);
}

// Page of `place`, -1 if it is none of the cache's.
__device__ __forceinline__ int sd_page(const sd_rows& b, int n_pages, int i, int entry) {
    const int p = b.d_table[(long long)i * b.table_stride + entry];
    return (unsigned)p < (unsigned)n_pages ? p : -1;
}

template <class T> struct Elem;
template <> struct Elem<__nv_bfloat16> {
    static __device__ __forceinline__ float2 up(uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u)); }
    static __device__ __forceinline__ uint32_t down(float a, float b) { uint32_t r; asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a)); return r; }
};
template <> struct Elem<__half> {
    static __device__ __forceinline__ float2 up(uint32_t v) { __half2 h; memcpy(&h, &v, 4); return __half22float2(h); }
    static __device__ __forceinline__ uint32_t down(float a, float b) { uint32_t r; asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a)); return r; }
};

// Two products, or products and sums, at once.
__device__ __forceinline__ float2 sd_mul2(float2 a, float2 b) {
    float2 r;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmul.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}" : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float2 sd_fma2(float2 a, float2 b, float2 c) {
    float2 r;
    asm("{\n\t.reg .b64 x, y, z, u;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\tfma.rn.f32x2 u, x, y, z;\n\tmov.b64 {%0, %1}, u;\n\t}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return r;
}

__device__ __forceinline__ float2 sd_add2(float2 a, float2 b) {
    float2 r;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}" : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}

template <class T>
__device__ __forceinline__ void sd_unpack(const uint4& v, float* x) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) { const float2 f = Elem<T>::up(w[k]); x[2 * k] = f.x; x[2 * k + 1] = f.y; }
}

template <class T>
__device__ __forceinline__ uint4 sd_pack(const float* x) {
    return make_uint4(Elem<T>::down(x[0], x[1]), Elem<T>::down(x[2], x[3]), Elem<T>::down(x[4], x[5]), Elem<T>::down(x[6], x[7]));
}

// ---- host: arguments -----------------------------------------------------------------------
inline bool sd_aligned(const void* p) { return ((uintptr_t)p & 15) == 0; }
// Rows and heads that are written: each has a place of its own.
inline bool sd_out_strides_ok(const int64_t* s, int rows, int heads) { return (rows <= 1 || s[0] > 0) && (heads <= 1 || s[1] > 0); }
inline bool sd_stride_ok(long long s) { return s >= 0 && s % 8 == 0; }

// Whether the current device can be given these pointers: the memory `p` lies on is its own (or the host's).
inline int sd_check_pointer(const void* p) {
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return SD_ERR_CUDA;
    cudaPointerAttributes a;
    if (cudaPointerGetAttributes(&a, p) != cudaSuccess) return SD_ERR_CUDA;
    if (a.type == cudaMemoryTypeDevice && a.device != dev) return SD_ERR_INVALID_ARG;
    return a.type == cudaMemoryTypeUnregistered ? SD_ERR_INVALID_ARG : SD_OK;
}

inline int sd_check_cache(const sd_cache* c, const sd_rows* b) {
    if (!c || !b || !c->d_k || !c->d_v || !sd_aligned(c->d_k) || !sd_aligned(c->d_v)) return SD_ERR_INVALID_ARG;
    if (c->dtype != SD_BF16 && c->dtype != SD_FP16) return SD_ERR_INVALID_ARG;
    if (c->head_dim != 64 && c->head_dim != 128) return SD_ERR_INVALID_ARG;
    if (c->kv_heads < 1 || c->kv_heads > 1024 || c->n_layers < 1 || c->n_pages < 1 || c->page_size < 1) return SD_ERR_INVALID_ARG;
    const int p = c->page_size;
    if (!(p == 8 || p == 16 || p == 32 || p == 64 || p % 128 == 0 || b->table_stride == 1)) return SD_ERR_INVALID_ARG;
    for (int k = 0; k < 4; ++k) {                                // (a stride is not looked at where there is one of a kind)
        const bool used = k == 0 ? c->n_layers > 1 : k == 1 ? c->n_pages > 1 : k == 2 ? c->page_size > 1 : c->kv_heads > 1;
        if (used && (c->k_stride[k] <= 0 || c->v_stride[k] <= 0 || c->k_stride[k] % 8 || c->v_stride[k] % 8)) return SD_ERR_INVALID_ARG;
    }
    if (b->n < 0 || b->rows < 0 || b->max_draft < 0 || b->max_draft > SD_MAX_SPEC || b->table_stride < 1) return SD_ERR_INVALID_ARG;
    if ((long long)b->table_stride * c->page_size > (1ll << 31) - 1024) return SD_ERR_INVALID_ARG;
    if (b->n > 0 && (!b->d_cached || !b->d_table)) return SD_ERR_INVALID_ARG;
    return SD_OK;
}
