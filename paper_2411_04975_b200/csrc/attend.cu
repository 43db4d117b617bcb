// sd_attend: attention of the rows of draft trees over their requests' paged caches.
#include "verify.cuh"

namespace {

struct AttendArgs {
    sd_cache c;
    sd_rows b;
    sd_attend_params p;
    const void* q;
    void* out;
    float* lse;
};

constexpr int WARPS = 4;

// A block per row and head; a warp takes every fourth place, its lanes the elements of the head.  Running maximum, sum and weighted values
// per warp, joined at the end.
template <class T, int D>
__global__ void __launch_bounds__(32 * WARPS) attend_kernel(const __grid_constant__ AttendArgs a) {
    sd_chain_begin();
    constexpr int E = D / 32;
    const sd_rows& b = a.b;
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5, h = blockIdx.y;
    const long long row = blockIdx.x;
    __shared__ unsigned long long s_bits[SD_MAX_SPEC + 1];
    __shared__ float s_m[WARPS], s_l[WARPS], s_o[WARPS][D];
    if (b.d_status && h == 0 && t == 0)
        for (int i = blockIdx.x; i < b.n; i += gridDim.x) {
            const Request r = sd_request(b, i, a.c.page_size, a.p.shared);
            int st = r.status;
            if (r.count)
                for (int e = 0; e <= (r.cached + r.count - 1) / a.c.page_size; ++e)
                    if (sd_page(b, a.c.n_pages, i, e) < 0) st |= SD_STATUS_BAD_PAGE;
            b.d_status[i] = st;
        }
    if (row >= b.rows) return;
    int i = 0;
    for (int base = 0; base < b.n; base += 32 * WARPS)
        i += __syncthreads_count(base + t < b.n && b.d_offsets[base + t + 1] <= row);
    if (i >= b.n) return;
    const Request r = sd_request(b, i, a.c.page_size, a.p.shared);
    if (row < r.begin || row >= r.begin + r.count) return;
    for (int k = t; k < r.count; k += 32 * WARPS) s_bits[k] = sd_tree_bits(b, i, k);
    __syncthreads();
    const int local = (int)(row - r.begin), W = a.p.window, hk = h / (a.p.q_heads / a.c.kv_heads);
    const unsigned long long mine = s_bits[local];
    const int position = r.cached + __popcll(mine);
    const T* q = (const T*)a.q + row * a.p.q_stride[0] + h * a.p.q_stride[1];
    float qf[E], o[E] = {}, m = -INFINITY, l = 0.f;
    for (int e = 0; e < E; ++e) qf[e] = (float)q[lane + 32 * e] * a.p.scale;
    for (int p = warp; p < r.cached + r.count; p += WARPS) {
        int at = p;
        if (p >= r.cached) {
            const int tree = p - r.cached;
            if (tree && !(mine >> (tree - 1) & 1)) continue;
            at = r.cached + __popcll(s_bits[tree]);
        }
        if (W && position - at >= W && at >= a.p.sinks) continue;
        const int page = sd_page(b, a.c.n_pages, i, p / a.c.page_size);
        if (page < 0) continue;
        const long long line = p % a.c.page_size;
        const T* k = (const T*)a.c.d_k + page * a.c.k_stride[1] + line * a.c.k_stride[2] + hk * a.c.k_stride[3];
        const T* v = (const T*)a.c.d_v + page * a.c.v_stride[1] + line * a.c.v_stride[2] + hk * a.c.v_stride[3];
        float s = 0.f;
        for (int e = 0; e < E; ++e) s += qf[e] * (float)k[lane + 32 * e];
        for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
        const float top = fmaxf(m, s), base = top == -INFINITY ? 0.f : top, keep = expf(m - base), w = expf(s - base);
        m = top;
        l = l * keep + w;
        for (int e = 0; e < E; ++e) o[e] = o[e] * keep + w * (float)v[lane + 32 * e];
    }
    if (lane == 0) { s_m[warp] = m; s_l[warp] = l; }
    for (int e = 0; e < E; ++e) s_o[warp][lane + 32 * e] = o[e];
    __syncthreads();
    if (t < D) {
        float top = -INFINITY, sum = 0.f, x = 0.f;
        for (int w = 0; w < WARPS; ++w) top = fmaxf(top, s_m[w]);
        const float base = top == -INFINITY ? 0.f : top;
        for (int w = 0; w < WARPS; ++w) {
            const float f = expf(s_m[w] - base);
            sum += s_l[w] * f;
            x += s_o[w][t] * f;
        }
        ((T*)a.out)[row * a.p.out_stride[0] + h * a.p.out_stride[1] + t] = (T)(sum == 0.f ? 0.f : x / sum);
        if (a.lse && t == 0) a.lse[row * a.p.q_heads + h] = sum == 0.f ? -INFINITY : base + logf(sum);
    }
}

int check(const sd_cache* cache, const sd_rows* rows, const sd_attend_params* prm) {
    const int rc = sd_check_cache(cache, rows);
    if (rc != SD_OK) return rc;
    if (!prm || prm->q_heads < 1 || prm->q_heads > 65535 || prm->q_heads % cache->kv_heads) return SD_ERR_INVALID_ARG;
    if (prm->window < 0 || prm->sinks < 0 || prm->shared < 0 || !(prm->scale == prm->scale)) return SD_ERR_INVALID_ARG;
    for (int k = 0; k < 2; ++k)
        if (!sd_stride_ok(prm->q_stride[k]) || !sd_stride_ok(prm->out_stride[k])) return SD_ERR_INVALID_ARG;
    return SD_OK;
}

}  // namespace

extern "C" int64_t sd_attend_workspace(const sd_cache* cache, const sd_rows* rows, const sd_attend_params* prm) {
    const int rc = check(cache, rows, prm);
    return rc != SD_OK ? rc : 256;
}

extern "C" int sd_attend(const sd_cache* cache, const sd_rows* rows, const sd_attend_params* prm, const void* d_q, void* d_out,
                         float* d_lse, void* d_workspace, int64_t workspace_bytes, void* stream) {
    int rc = check(cache, rows, prm);
    if (rc != SD_OK) return rc;
    if (rows->n == 0 || (rows->rows == 0 && !rows->d_status)) return SD_OK;
    if (!rows->d_offsets || (rows->rows > 0 && (!d_q || !d_out)) || !sd_aligned(d_q) || !sd_aligned(d_out)) return SD_ERR_INVALID_ARG;
    if (!d_workspace || (uintptr_t)d_workspace % 256) return SD_ERR_INVALID_ARG;
    if (workspace_bytes < sd_attend_workspace(cache, rows, prm)) return SD_ERR_CAPACITY;
    rc = sd_check_pointer(cache->d_k);
    if (rc != SD_OK) return rc;
    const AttendArgs a = {*cache, *rows, *prm, d_q, d_out, d_lse};
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(rows->rows > 0 ? rows->rows : 1, prm->q_heads); cfg.blockDim = dim3(32 * WARPS); cfg.stream = (cudaStream_t)stream;
    cfg.attrs = &attr; cfg.numAttrs = 1;
    cudaError_t e;
    if (cache->dtype == SD_BF16) e = cache->head_dim == 128 ? cudaLaunchKernelEx(&cfg, attend_kernel<__nv_bfloat16, 128>, a) : cudaLaunchKernelEx(&cfg, attend_kernel<__nv_bfloat16, 64>, a);
    else e = cache->head_dim == 128 ? cudaLaunchKernelEx(&cfg, attend_kernel<__half, 128>, a) : cudaLaunchKernelEx(&cfg, attend_kernel<__half, 64>, a);
    return e == cudaSuccess ? SD_OK : SD_ERR_CUDA;
}
