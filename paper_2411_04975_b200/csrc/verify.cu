// The verifier's side of a step beside attention: sd_rotate, sd_accept, sd_commit.
#include "verify.cuh"

namespace {

// ---- sd_rotate -----------------------------------------------------------------------------
// A block per row; the row's heads go to groups of head_dim / 8 lanes, eight elements a lane.  Bound by the bytes of
// the row: every element is read once and written once.
constexpr int ROT_THREADS = 256;
constexpr int ROT_BATCH = 4;                                      // heads of a group that are loaded before any is worked on

struct RotateArgs {
    sd_cache c;
    sd_rows b;
    sd_rotate_params p;
    const void *q, *k, *v, *qw, *kw;
    const double* freq;
    const int32_t* positions;
    void* out;
};

template <class T, int D, bool INTERLEAVED>
__global__ void __launch_bounds__(ROT_THREADS) rotate_kernel(const __grid_constant__ RotateArgs a) {
    sd_chain_begin();
    constexpr int LANES = D / 8, GROUPS = ROT_THREADS / LANES;
    __shared__ float s_cos[D / 2], s_sin[D / 2];
    __shared__ int s_line;                                        // of the page; -1: rows and page make no sense
    __shared__ int s_page;
    const int t = threadIdx.x, lane = t % LANES, group = t / LANES;
    const sd_rows& b = a.b;

    if (b.d_status && t == ROT_THREADS - 1)
        for (int i = blockIdx.x; i < b.n; i += gridDim.x) {
            const Request r = sd_request(b, i, a.c.page_size);
            int st = r.status;
            if (r.count)
                for (int e = r.cached / a.c.page_size; e <= (r.cached + r.count - 1) / a.c.page_size; ++e)
                    if (sd_page(b, a.c.n_pages, i, e) < 0) st |= SD_STATUS_BAD_PAGE;
            b.d_status[i] = st;
        }
    const long long row = blockIdx.x;
    if (row >= b.rows) return;
    const int heads = a.p.q_heads + 2 * a.c.kv_heads;

    auto source = [&](int h) -> const T* {
        if (h < a.p.q_heads) return (const T*)a.q + row * a.p.q_stride[0] + h * a.p.q_stride[1];
        h -= a.p.q_heads;
        if (h < a.c.kv_heads) return (const T*)a.k + row * a.p.k_stride[0] + h * a.p.k_stride[1];
        return (const T*)a.v + row * a.p.v_stride[0] + (h - a.c.kv_heads) * a.p.v_stride[1];
    };
    uint4 raw[ROT_BATCH];
#pragma unroll
    for (int e = 0; e < ROT_BATCH; ++e)
        if (group + e * GROUPS < heads) raw[e] = *(const uint4*)(source(group + e * GROUPS) + lane * 8);

    int i = 0;                                                    // the request: offsets that are not above the row
    for (int base = 0; base < b.n; base += ROT_THREADS)
        i += __syncthreads_count(base + t < b.n && b.d_offsets[base + t + 1] <= row);
    if (i >= b.n) return;                                         // behind the last request
    const Request r = sd_request(b, i, a.c.page_size);
    if (row < r.begin || row >= r.begin + r.count) return;
    const int local = (int)(row - r.begin);
    if (t == 0) {
        const int place = r.cached + local;
        s_page = sd_page(b, a.c.n_pages, i, place / a.c.page_size);
        s_line = place % a.c.page_size;
    }
    if (t < a.p.rot_dim / 2) {
        const int pos = a.positions ? a.positions[row] : r.cached + __popcll(sd_tree_bits(b, i, local));
        double turns = (double)pos * a.freq[t] * 0.15915494309189533577;      // 1 / 2 pi
        turns -= rint(turns);
        float sn, cs;
        sincospif(2.0f * (float)turns, &sn, &cs);
        s_cos[t] = cs * a.p.scale;
        s_sin[t] = sn * a.p.scale;
    }
    __syncthreads();
    const int half = a.p.rot_dim / 2;
    const long long in_k = s_page * a.c.k_stride[1] + s_line * a.c.k_stride[2], in_v = s_page * a.c.v_stride[1] + s_line * a.c.v_stride[2];

    for (int base = 0; base < heads; base += GROUPS * ROT_BATCH) {
        const int first = base + group;
        if (base) {
#pragma unroll
            for (int e = 0; e < ROT_BATCH; ++e)
                if (first + e * GROUPS < heads) raw[e] = *(const uint4*)(source(first + e * GROUPS) + lane * 8);
        }
#pragma unroll
        for (int e = 0; e < ROT_BATCH; ++e) {
            const int h = first + e * GROUPS;
            const bool live = h < heads;                          // (all lanes stay for the shuffles)
            if (live && h >= a.p.q_heads + a.c.kv_heads) {
                if (s_page >= 0)
                    *(uint4*)((T*)a.c.d_v + in_v + (h - a.p.q_heads - a.c.kv_heads) * a.c.v_stride[3] + lane * 8) = raw[e];
            }
            float x[8], y[8];
            sd_unpack<T>(raw[e], x);
            const bool is_q = h < a.p.q_heads;
            const T* w = (const T*)(is_q ? a.qw : a.kw);
            if (a.qw || a.kw) {
                float sum = 0.f;
#pragma unroll
                for (int k = 0; k < 8; ++k) sum += x[k] * x[k];
#pragma unroll
                for (int d = LANES / 2; d > 0; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
                if (w) {
                    const float inv = 1.0f / sqrtf(sum / D + a.p.eps);
                    float wf[8];
                    sd_unpack<T>(*(const uint4*)(w + lane * 8), wf);
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = x[k] * inv * wf[k];
                }
            }
            const int at = lane * 8;
            if (INTERLEAVED) {
#pragma unroll
                for (int k = 0; k < 8; k += 2) {
                    y[k] = x[k]; y[k + 1] = x[k + 1];
                    if (at < a.p.rot_dim) {
                        const float c = s_cos[(at + k) / 2], s = s_sin[(at + k) / 2];
                        y[k] = x[k] * c - x[k + 1] * s;
                        y[k + 1] = x[k + 1] * c + x[k] * s;
                    }
                }
            } else {
                const bool low = at < half;
                const int other = (threadIdx.x & 31 & ~(LANES - 1)) + (at < a.p.rot_dim ? (low ? lane + half / 8 : lane - half / 8) : lane);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float z = __shfl_sync(~0u, x[k], other);
                    y[k] = x[k];
                    if (at < a.p.rot_dim) {
                        const int j = low ? at + k : at + k - half;
                        y[k] = low ? x[k] * s_cos[j] - z * s_sin[j] : x[k] * s_cos[j] + z * s_sin[j];
                    }
                }
            }
            if (!live || h >= a.p.q_heads + a.c.kv_heads) continue;
            if (is_q) *(uint4*)((T*)a.out + row * a.p.out_stride[0] + h * a.p.out_stride[1] + at) = sd_pack<T>(y);
            else if (s_page >= 0) *(uint4*)((T*)a.c.d_k + in_k + (h - a.p.q_heads) * a.c.k_stride[3] + at) = sd_pack<T>(y);
        }
    }
}

// ---- sd_accept -----------------------------------------------------------------------------
// The largest logit of a row, by a block.  The row is cut into chunks of 16 bytes (the first and the last may be shorter: a
// row starts anywhere); a thread keeps the largest value it has seen and the chunk it was in, and only the winner's chunk is read
// again for the place.  Bound by reading the logits.
constexpr int MAX_THREADS = 512;

template <class T> __device__ __forceinline__ float as_float(T v);
template <> __device__ __forceinline__ float as_float(float v) { return v; }
template <> __device__ __forceinline__ float as_float(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float as_float(__nv_bfloat16 v) { return __bfloat162float(v); }

// Order of floats as that of unsigned numbers; both zeros alike, NaN above all.  Never 0.
__device__ __forceinline__ uint32_t order_key(float f) {
    if (f != f) return 0xFFFFFFFFu;
    const uint32_t u = __float_as_uint(f + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

template <class T>
__global__ void __launch_bounds__(MAX_THREADS) row_max_kernel(const T* logits, long long stride, int vocab, int32_t* targets) {
    sd_chain_begin();
    constexpr int PER = 16 / sizeof(T);
    const T* row = logits + blockIdx.x * stride;
    const int t = threadIdx.x;
    const int head = min(vocab, (int)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(T));   // elements before the first 16-byte boundary
    const int chunks = 1 + (vocab - head + PER - 1) / PER;
    auto bounds = [&](int c, int& lo, int& hi) {
        lo = c == 0 ? 0 : head + (c - 1) * PER;
        hi = c == 0 ? head : min(lo + PER, vocab);
    };
    uint32_t best = 0;
    int where = 0;
    for (int c = t; c < chunks; c += MAX_THREADS) {
        int lo, hi;
        bounds(c, lo, hi);
        uint32_t m = 0;
        if (hi - lo == PER && c > 0) {
            T v[PER];
            *(uint4*)v = *(const uint4*)(row + lo);
#pragma unroll
            for (int k = 0; k < PER; ++k) m = max(m, order_key(as_float(v[k])));
        } else {
            for (int k = lo; k < hi; ++k) m = max(m, order_key(as_float(row[k])));
        }
        if (m > best) { best = m; where = c; }
    }
    unsigned long long all = (unsigned long long)best << 32 | (0xFFFFFFFFu - (uint32_t)where);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) all = max(all, __shfl_xor_sync(~0u, all, d));
    __shared__ unsigned long long s_all[MAX_THREADS / 32];
    if ((t & 31) == 0) s_all[t / 32] = all;
    __syncthreads();
    if (t == 0) {
        for (int w = 1; w < MAX_THREADS / 32; ++w) all = max(all, s_all[w]);
        int lo, hi;
        bounds((int)(0xFFFFFFFFu - (uint32_t)all), lo, hi);
        for (int k = lo; k < hi; ++k)
            if (order_key(as_float(row[k])) == (uint32_t)(all >> 32)) { targets[blockIdx.x] = k; break; }
    }
}

struct WalkArgs {
    int n, rows, M;
    const int64_t* offsets;
    const int32_t *tokens, *parents, *targets;
    int32_t* path;
    int64_t* new_offsets;
    int32_t *new_tokens, *status;
};

// The accepted paths, a warp each, then their begins and tokens, by one block.
__global__ void __launch_bounds__(1024) walk_kernel(const WalkArgs a) {
    sd_chain_begin();
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    __shared__ long long s_sum[32];
    __shared__ long long s_base;
    for (int i = warp; i < a.n; i += 32) {
        const long long lo = a.offsets[i], hi = a.offsets[i + 1];
        const bool bad = lo < 0 || hi < lo || hi > a.rows || hi - lo > a.M + 1;
        const int count = bad ? 0 : (int)(hi - lo);
        int tok[2], par[2], tgt[3];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int j = lane + 32 * e;
            const bool node = j < count - 1;
            tok[e] = node ? a.tokens[(long long)i * a.M + j] : -1;
            par[e] = node ? a.parents[(long long)i * a.M + j] : -2;
        }
#pragma unroll
        for (int e = 0; e < 3; ++e) tgt[e] = lane + 32 * e < count ? a.targets[lo + lane + 32 * e] : -1;
        int32_t* path = a.path + (long long)i * (a.M + 1);
        int kept = 0, cur = 0;                                    // row
        if (count) {
            for (;;) {
                if (lane == 0) path[kept] = cur;
                ++kept;
                const int want = __shfl_sync(~0u, cur >= 64 ? tgt[2] : cur >= 32 ? tgt[1] : tgt[0], cur & 31);
                const unsigned f0 = __ballot_sync(~0u, par[0] == cur - 1 && tok[0] == want && lane + 1 > cur);
                const unsigned f1 = __ballot_sync(~0u, par[1] == cur - 1 && tok[1] == want && lane + 33 > cur);
                if (f0) cur = __ffs(f0);
                else if (f1) cur = 32 + __ffs(f1);
                else break;
            }
        }
        for (int j = kept + lane; j <= a.M; j += 32) path[j] = -1;
        if (lane == 0) {
            a.new_offsets[i + 1] = kept;
            if (a.status) a.status[i] = bad ? SD_STATUS_BAD_ROWS : SD_STATUS_OK;
        }
    }
    if (t == 0) { a.new_offsets[0] = 0; s_base = 0; }
    __syncthreads();
    for (int first = 0; first < a.n; first += 1024) {             // begins: running sums of the lengths
        long long x = first + t < a.n ? a.new_offsets[first + t + 1] : 0;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long y = __shfl_up_sync(~0u, x, d);
            if (lane >= d) x += y;
        }
        if (lane == 31) s_sum[warp] = x;
        __syncthreads();
        if (warp == 0) {
            long long y = s_sum[lane];
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const long long z = __shfl_up_sync(~0u, y, d);
                if (lane >= d) y += z;
            }
            s_sum[lane] = y;
        }
        __syncthreads();
        x += s_base + (warp ? s_sum[warp - 1] : 0);
        if (first + t < a.n) a.new_offsets[first + t + 1] = x;
        __syncthreads();
        if (t == 1023) s_base = x;
        __syncthreads();
    }
    for (int i = warp; i < a.n; i += 32) {
        const long long lo = a.offsets[i], at = a.new_offsets[i];
        const int kept = (int)(a.new_offsets[i + 1] - at);
        for (int j = lane; j < kept; j += 32) a.new_tokens[at + j] = a.targets[lo + a.path[(long long)i * (a.M + 1) + j]];
    }
    for (long long k = s_base + t; k < a.rows; k += 1024) a.new_tokens[k] = -1;
}

// ---- sd_commit -----------------------------------------------------------------------------
// A block per request, layer and one of keys and values; a thread per 16 bytes of a line.  Lines only move to smaller places, and a
// path ascends: what a batch of lines overwrites, no later batch reads.  Bound by the lines moved (and by the latency of path, table, line).
constexpr int COMMIT_BATCH = 8;

struct CommitArgs {
    sd_cache c;
    sd_rows b;
    const int32_t* path;
    int32_t* cached_out;
};

__global__ void __launch_bounds__(128) commit_kernel(const __grid_constant__ CommitArgs a) {
    sd_chain_begin();
    const sd_rows& b = a.b;
    const int i = blockIdx.x, side = blockIdx.y & 1, layer = blockIdx.y >> 1, t = threadIdx.x;
    __shared__ int s_path[SD_MAX_SPEC + 1], s_src[SD_MAX_SPEC + 1], s_dst[SD_MAX_SPEC + 1];     // pages
    __shared__ int s_bad;
    const int M1 = b.max_draft + 1;
    if (t == 0) s_bad = 0;
    __syncthreads();
    const int cached = b.d_cached[i];
    int p = -1, kept;
    const int P = a.c.page_size;
    if (t < M1) p = a.path[(long long)i * M1 + t];
    kept = __syncthreads_count(p >= 0);
    if (t < M1) {
        s_path[t] = p;
        const int before = t ? a.path[(long long)i * M1 + t - 1] : -1;
        bool bad = t < kept ? p <= before || p > b.max_draft || (t == 0 && p != 0) : p != -1;
        if (t < kept && !bad) {
            if (cached < 0 || (long long)cached + p >= (long long)P * b.table_stride) bad = true;
            else {
                s_src[t] = sd_page(b, a.c.n_pages, i, (cached + p) / P);
                s_dst[t] = sd_page(b, a.c.n_pages, i, (cached + t) / P);
                if (p != t && (s_src[t] < 0 || s_dst[t] < 0)) atomicOr(&s_bad, SD_STATUS_BAD_PAGE);
            }
        }
        if (bad) atomicOr(&s_bad, SD_STATUS_BAD_ROWS);
    }
    __syncthreads();
    const int bad = s_bad;
    if (blockIdx.y == 0 && t == 0) {
        if (b.d_status) b.d_status[i] = bad;
    }
    (void)layer; (void)side;
    if (!(bad & SD_STATUS_BAD_ROWS)) {
        const int64_t* st = side ? a.c.v_stride : a.c.k_stride;
        char* base = (char*)(side ? a.c.d_v : a.c.d_k) + 2 * (layer * st[0]);
        const int per = a.c.head_dim / 8, columns = a.c.kv_heads * per;
        for (int col = t; col < columns; col += blockDim.x) {
            char* at = base + 2 * ((col / per) * st[3] + (col % per) * 8);
            for (int first = 0; first < kept; first += COMMIT_BATCH) {
                uint4 v[COMMIT_BATCH];
#pragma unroll
                for (int e = 0; e < COMMIT_BATCH; ++e) {
                    const int j = first + e;
                    if (j < kept && s_path[j] != j && s_src[j] >= 0 && s_dst[j] >= 0)
                        v[e] = *(const uint4*)(at + 2 * (s_src[j] * st[1] + (cached + s_path[j]) % P * st[2]));
                }
#pragma unroll
                for (int e = 0; e < COMMIT_BATCH; ++e) {
                    const int j = first + e;
                    if (j < kept && s_path[j] != j && s_src[j] >= 0 && s_dst[j] >= 0)
                        *(uint4*)(at + 2 * (s_dst[j] * st[1] + (cached + j) % P * st[2])) = v[e];
                }
            }
        }
    }
}

// After the lines: the new lengths (the other kernel's blocks read the old ones, which may be the same memory).
__global__ void __launch_bounds__(128) lengths_kernel(const __grid_constant__ CommitArgs a) {
    sd_chain_begin();
    const int i = blockIdx.x * 128 + threadIdx.x;
    if (i >= a.b.n) return;
    const int M1 = a.b.max_draft + 1, cached = a.b.d_cached[i];
    int kept = 0, before = -1;
    bool bad = false;
    for (int j = 0; j < M1; ++j) {
        const int p = a.path[(long long)i * M1 + j];
        if (p >= 0) bad |= kept != j || p <= before || p > a.b.max_draft || (j == 0 && p != 0) || (long long)cached + p >= (long long)a.c.page_size * a.b.table_stride;
        else bad |= p != -1;
        if (p >= 0) { ++kept; before = p; }
    }
    a.cached_out[i] = bad || (kept && cached < 0) ? cached : cached + kept;
}

}  // namespace

extern "C" int sd_rotate(const sd_cache* cache, const sd_rows* rows, const sd_rotate_params* prm, const void* d_q, const void* d_k,
                         const void* d_v, const double* d_freq, const int32_t* d_positions, const void* d_q_weight,
                         const void* d_k_weight, void* d_q_out, void* stream) {
    int rc = sd_check_cache(cache, rows);
    if (rc != SD_OK) return rc;
    if (!prm || prm->q_heads < 1 || prm->q_heads > 65536 || prm->q_heads % cache->kv_heads) return SD_ERR_INVALID_ARG;
    if (prm->rot_dim < 0 || prm->rot_dim > cache->head_dim || prm->rot_dim % 16 || (prm->rot_dim && !d_freq)) return SD_ERR_INVALID_ARG;
    if (!(prm->eps >= 0)) return SD_ERR_INVALID_ARG;
    if (rows->n == 0 || (rows->rows == 0 && !rows->d_status)) return SD_OK;
    if (!rows->d_offsets) return SD_ERR_INVALID_ARG;
    if (rows->rows > 0) {
        if (!d_q || !d_k || !d_v || !d_q_out) return SD_ERR_INVALID_ARG;
        for (const void* p : {d_q, d_k, d_v, (const void*)d_q_out, d_q_weight, d_k_weight})
            if (!sd_aligned(p)) return SD_ERR_INVALID_ARG;
        for (int k = 0; k < 2; ++k)
            if (!sd_stride_ok(prm->q_stride[k]) || !sd_stride_ok(prm->k_stride[k]) || !sd_stride_ok(prm->v_stride[k]) || !sd_stride_ok(prm->out_stride[k]))
                return SD_ERR_INVALID_ARG;
    }
    rc = sd_check_pointer(cache->d_k);
    if (rc != SD_OK) return rc;
    const RotateArgs a = {*cache, *rows, *prm, d_q, d_k, d_v, d_q_weight, d_k_weight, d_freq, d_positions, d_q_out};
    const unsigned grid = rows->rows > 0 ? rows->rows : 1;
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e;
#define SD_ROTATE(T, D) (prm->interleaved ? sd_launch(rotate_kernel<T, D, true>, grid, ROT_THREADS, 0, st, a) : sd_launch(rotate_kernel<T, D, false>, grid, ROT_THREADS, 0, st, a))
    if (cache->dtype == SD_BF16) e = cache->head_dim == 128 ? SD_ROTATE(__nv_bfloat16, 128) : SD_ROTATE(__nv_bfloat16, 64);
    else e = cache->head_dim == 128 ? SD_ROTATE(__half, 128) : SD_ROTATE(__half, 64);
#undef SD_ROTATE
    return e == cudaSuccess ? SD_OK : SD_ERR_CUDA;
}

extern "C" int sd_accept(int32_t n, int32_t rows, int32_t max_draft, int32_t vocab, int32_t dtype, int64_t row_stride, const void* d_logits,
                         const int64_t* d_offsets, const int32_t* d_tokens, const int32_t* d_parents, int32_t* d_targets, int32_t* d_path,
                         int64_t* d_new_offsets, int32_t* d_new_tokens, int32_t* d_status, void* stream) {
    if (n < 0 || rows < 0 || max_draft < 0 || max_draft > SD_MAX_SPEC || vocab < 1 || vocab > (1 << 30)) return SD_ERR_INVALID_ARG;
    if (dtype != SD_BF16 && dtype != SD_FP16 && dtype != SD_FP32) return SD_ERR_INVALID_ARG;
    if (!d_new_offsets || (n > 0 && (!d_offsets || !d_path)) || (n > 0 && max_draft > 0 && (!d_tokens || !d_parents))) return SD_ERR_INVALID_ARG;
    if (rows > 0 && (!d_logits || !d_targets || !d_new_tokens || row_stride < vocab)) return SD_ERR_INVALID_ARG;
    if ((uintptr_t)d_logits % (dtype == SD_FP32 ? 4 : 2)) return SD_ERR_INVALID_ARG;
    const int rc = sd_check_pointer(d_new_offsets);
    if (rc != SD_OK) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    if (rows > 0) {
        cudaError_t e;
        if (dtype == SD_BF16) e = sd_launch(row_max_kernel<__nv_bfloat16>, rows, MAX_THREADS, 0, st, (const __nv_bfloat16*)d_logits, (long long)row_stride, vocab, d_targets);
        else if (dtype == SD_FP16) e = sd_launch(row_max_kernel<__half>, rows, MAX_THREADS, 0, st, (const __half*)d_logits, (long long)row_stride, vocab, d_targets);
        else e = sd_launch(row_max_kernel<float>, rows, MAX_THREADS, 0, st, (const float*)d_logits, (long long)row_stride, vocab, d_targets);
        if (e != cudaSuccess) return SD_ERR_CUDA;
    }
    const WalkArgs a = {n, rows, max_draft, d_offsets, d_tokens, d_parents, d_targets, d_path, d_new_offsets, d_new_tokens, d_status};
    return sd_launch(walk_kernel, 1, 1024, 0, st, a) == cudaSuccess ? SD_OK : SD_ERR_CUDA;
}

extern "C" int sd_commit(const sd_cache* cache, const sd_rows* rows, const int32_t* d_path, int32_t* d_new_cached, void* stream) {
    int rc = sd_check_cache(cache, rows);
    if (rc != SD_OK) return rc;
    if (cache->n_layers > 32767) return SD_ERR_INVALID_ARG;
    if (rows->n == 0) return SD_OK;
    if (!d_path || !d_new_cached) return SD_ERR_INVALID_ARG;
    rc = sd_check_pointer(cache->d_k);
    if (rc != SD_OK) return rc;
    const CommitArgs a = {*cache, *rows, d_path, d_new_cached};
    cudaStream_t st = (cudaStream_t)stream;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(rows->n, 2 * cache->n_layers); cfg.blockDim = dim3(128); cfg.stream = st;
    cfg.attrs = &attr; cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, commit_kernel, a) != cudaSuccess) return SD_ERR_CUDA;
    return sd_launch(lengths_kernel, (rows->n + 127) / 128, 128, 0, st, a) == cudaSuccess ? SD_OK : SD_ERR_CUDA;
}
