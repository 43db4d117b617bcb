// The verifier's side of a step beside attention: sd_rotate, sd_accept, sd_commit.
#include "verify.cuh"

#include <cooperative_groups.h>

#include <algorithm>

namespace {

// ---- sd_rotate -----------------------------------------------------------------------------
// A block takes a few rows of one request (one, where there are few; ROT_ROWS in a large batch), so that what it looks up - where the rows are, how deep,
// in which page - is two reads behind one another for all of them.  A row's heads go to the lanes of one or more warps, head_dim / 8 lanes a head and eight
// elements a lane, always the same eight: what they are multiplied by (cosine, sine and weight in one factor for the element and one for the other of its
// pair) is kept for all heads: in registers, but for some 22 words of a thread, which six blocks a multiprocessor (80 registers) leave no room for.  (Factors read from shared memory for every head, and pairs exchanged in 32 bits, took 400
// instructions for 256 elements and 69 us for 256 requests of up to 65 rows, now 33, 4.3 of the 6.55 TB/s that a
// copy reaches.)  x' = x w / sqrt(mean(x^2) + eps) has its factor at the end, behind the turn, which is linear: y = (x_a m + x_b o) / sqrt(...).  Bound by the bytes of the
// rows, every element is read once and written once; one request (5.2 - 5.6 us): by the host, whose call takes as
// long (3.5 in a graph: the launch and three reads behind one another).
constexpr int ROT_THREADS = 128, ROT_WARPS = ROT_THREADS / 32;
constexpr int ROT_ROWS = 4;
constexpr int ROT_BATCH = 4;                                      // pieces that a lane has under way

struct RotateArgs {
    sd_cache c;
    sd_rows b;
    sd_rotate_params p;
    const void *q, *k, *v, *qw, *kw;
    const double* freq;
    const int32_t* positions;
    void* out;
    int chunks, per;              // of a request: blocks, rows a block
};

// Pieces of ROT_BATCH heads from `first` on, a step from one to the next.
template <class T>
__device__ __forceinline__ void load_heads(uint4* raw, const T* from, long long stride, int count, int first, int step, int lane) {
#pragma unroll
    for (int e = 0; e < ROT_BATCH; ++e) {
        const int h = first + e * step;
        if (h < count) raw[e] = ((const uint4*)(from + h * stride))[lane];
    }
}

// One kind of a row's heads, `count` of them, the first batch of which is in `next`: normed where there is a weight, turned, written to `to` (nowhere: null).
template <class T, int D, bool INTERLEAVED>
__device__ __forceinline__ void turn_heads(uint4* next, const T* from, long long from_stride, T* to, long long to_stride, int count, int first, int step, int lane, const T* weight, float eps,
                                           const float2* turn, int rot_dim) {
    constexpr int LANES = D / 8;
    const int at = lane * 8, half = rot_dim / 2;
    const bool turned = at < rot_dim, low = at < half;
    const int other = INTERLEAVED || !turned ? lane : low ? lane + half / 8 : lane - half / 8;   // the lane that has the pairs' other elements
    const int source = (threadIdx.x & 31 & ~(LANES - 1)) + other;
    float2 mine[4], others[4];                                    // y = mine * x + others * (the pair's other element)
    {
        float w[8], v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = v[k] = 1.f;
        if (weight) {
            sd_unpack<T>(((const uint4*)weight)[lane], w);
            sd_unpack<T>(((const uint4*)weight)[other], v);
        }
        float m[8], o[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float2 c = turned ? turn[INTERLEAVED ? (at + k) / 2 : low ? at + k : at + k - half] : make_float2(1.f, 0.f);
            const bool begins = INTERLEAVED ? k % 2 == 0 : low;   // the first of its pair
            m[k] = c.x * w[k];
            o[k] = (begins ? -c.y : c.y) * v[INTERLEAVED ? k ^ 1 : k];
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) { mine[k] = make_float2(m[2 * k], m[2 * k + 1]); others[k] = make_float2(o[2 * k], o[2 * k + 1]); }
    }
    uint4 raw[ROT_BATCH];
    for (int base = 0; base < count; base += step * ROT_BATCH) {  // (the same for all lanes)
#pragma unroll
        for (int e = 0; e < ROT_BATCH; ++e) raw[e] = next[e];
        load_heads<T>(next, from, from_stride, count, base + first + step * ROT_BATCH, step, lane);
#pragma unroll
        for (int e = 0; e < ROT_BATCH; ++e) {
            if (base + e * step >= count) break;
            const int h = base + first + e * step;
            const uint32_t words[4] = {raw[e].x, raw[e].y, raw[e].z, raw[e].w};
            float2 x[4], y[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                x[k] = Elem<T>::up(words[k]);
                y[k] = sd_mul2(x[k], mine[k]);
            }
            if (INTERLEAVED) {
                if (turned)
#pragma unroll
                    for (int k = 0; k < 4; ++k) y[k] = sd_fma2(make_float2(x[k].y, x[k].x), others[k], y[k]);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint32_t z = __shfl_sync(~0u, words[k], source);
                    if (turned) y[k] = sd_fma2(Elem<T>::up(z), others[k], y[k]);
                }
            }
            if (weight) {
                float2 two = sd_mul2(x[0], x[0]);
#pragma unroll
                for (int k = 1; k < 4; ++k) two = sd_fma2(x[k], x[k], two);
                float sum = two.x + two.y;
#pragma unroll
                for (int d = LANES / 2; d > 0; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
                const float inv = rsqrtf(sum * (1.0f / D) + eps);
#pragma unroll
                for (int k = 0; k < 4; ++k) y[k] = sd_mul2(y[k], make_float2(inv, inv));
            }
            if (to && h < count)
                ((uint4*)(to + h * to_stride))[lane] = make_uint4(Elem<T>::down(y[0].x, y[0].y), Elem<T>::down(y[1].x, y[1].y), Elem<T>::down(y[2].x, y[2].y), Elem<T>::down(y[3].x, y[3].y));
        }
    }
}

template <class T, int D, bool INTERLEAVED>
__global__ void __launch_bounds__(ROT_THREADS, 6) rotate_kernel(const __grid_constant__ RotateArgs a) {
    sd_chain_begin();
    constexpr int LANES = D / 8, GROUPS = 32 / LANES;             // of a warp
    __shared__ float2 s_turn[ROT_ROWS][D / 2];                    // cosine and sine
    __shared__ int s_page[ROT_ROWS];
    const int t = threadIdx.x, warp = t >> 5, lane = t % LANES;
    const sd_rows& b = a.b;
    const int i = blockIdx.x / a.chunks, first_row = blockIdx.x % a.chunks * a.per;
    const Request r = sd_request(b, i, a.c.page_size);
    if (b.d_status && first_row == 0 && t == ROT_THREADS - 1) {
        int st = r.status;
        if (r.count)
            for (int e = r.cached / a.c.page_size; e <= (r.cached + r.count - 1) / a.c.page_size; ++e)
                if (sd_page(b, a.c.n_pages, i, e) < 0) st |= SD_STATUS_BAD_PAGE;
        b.d_status[i] = st;
    }
    const int rows = min(a.per, r.count - first_row);
    if (rows <= 0) return;
    const long long begin = r.begin + first_row;
    // a row's warps
    const int parts = ROT_WARPS / a.per, e = warp / parts, first = (warp % parts) * GROUPS + (t & 31) / LANES, step = parts * GROUPS;
    const bool works = e < rows;
    const T *q_from = (const T*)a.q + (begin + e) * a.p.q_stride[0], *k_from = (const T*)a.k + (begin + e) * a.p.k_stride[0], *v_from = (const T*)a.v + (begin + e) * a.p.v_stride[0];
    uint4 next[ROT_BATCH];
    if (works) load_heads<T>(next, q_from, a.p.q_stride[1], a.p.q_heads, first, step, lane);

    const int half = a.p.rot_dim / 2;
    if (t < rows) s_page[t] = sd_page(b, a.c.n_pages, i, (r.cached + first_row + t) / a.c.page_size);
    for (int k = t; k < rows * (D / 2); k += ROT_THREADS) {
        const int row = k / (D / 2), j = k % (D / 2);
        if (j >= half) continue;
        const int pos = a.positions ? a.positions[begin + row] : r.cached + __popcll(sd_tree_bits(b, i, first_row + row));
        double turns = (double)pos * a.freq[j] * 0.15915494309189533577;      // 1 / 2 pi
        turns -= rint(turns);
        float sn, cs;
        sincospif(2.0f * (float)turns, &sn, &cs);
        s_turn[row][j] = make_float2(cs * a.p.scale, sn * a.p.scale);
    }
    __syncthreads();
    if (!works) return;
    turn_heads<T, D, INTERLEAVED>(next, q_from, a.p.q_stride[1], (T*)a.out + (begin + e) * a.p.out_stride[0], a.p.out_stride[1], a.p.q_heads, first, step, lane,
                                  (const T*)a.qw, a.p.eps, s_turn[e], a.p.rot_dim);
    const int page = s_page[e], line = (r.cached + first_row + e) % a.c.page_size;
    load_heads<T>(next, k_from, a.p.k_stride[1], a.c.kv_heads, first, step, lane);
    uint4 value[ROT_BATCH];
    load_heads<T>(value, v_from, a.p.v_stride[1], a.c.kv_heads, first, step, lane);
    turn_heads<T, D, INTERLEAVED>(next, k_from, a.p.k_stride[1], page < 0 ? nullptr : (T*)a.c.d_k + page * a.c.k_stride[1] + line * a.c.k_stride[2], a.c.k_stride[3], a.c.kv_heads, first,
                                  step, lane, (const T*)a.kw, a.p.eps, s_turn[e], a.p.rot_dim);
    if (page < 0) return;
    T* to = (T*)a.c.d_v + page * a.c.v_stride[1] + line * a.c.v_stride[2];
    for (int base = 0; base < a.c.kv_heads; base += step * ROT_BATCH) {
        if (base) load_heads<T>(value, v_from, a.p.v_stride[1], a.c.kv_heads, base + first, step, lane);
#pragma unroll
        for (int k = 0; k < ROT_BATCH; ++k) {
            const int h = base + first + k * step;
            if (h < a.c.kv_heads) ((uint4*)(to + h * a.c.v_stride[3]))[lane] = value[k];
        }
    }
}

// ---- sd_accept -----------------------------------------------------------------------------
// The largest logit of a row, by a block.  The row is cut into chunks of 16 bytes (the first and the last may be shorter: a
// row starts anywhere); a thread keeps the largest value it has seen and the chunk it was in, and only the winner's chunk is read
// again for the place.  Bound by reading the logits: 256 requests' rows of 128,256 bf16 numbers 219 us, 6.7 TB/s (reads alone are faster than a copy); one request 9.6 - 10.6 us, the host's
// time for two launches (6.0 in a graph).
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

// The largest of a chunk of 16 bytes.
__device__ __forceinline__ uint32_t largest(const uint4& v, float) {
    return max(max(order_key(__uint_as_float(v.x)), order_key(__uint_as_float(v.y))), max(order_key(__uint_as_float(v.z)), order_key(__uint_as_float(v.w))));
}
__device__ __forceinline__ uint32_t largest(const uint4& v, __nv_bfloat16) {
    __nv_bfloat162 h[4];
    memcpy(h, &v, 16);
    const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
    return max(order_key(__low2float(m)), order_key(__high2float(m)));
}
__device__ __forceinline__ uint32_t largest(const uint4& v, __half) {
    __half2 h[4];
    memcpy(h, &v, 16);
    const __half2 m = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
    return max(order_key(__low2float(m)), order_key(__high2float(m)));
}

// A cluster of `blocks` blocks a row; the first gets the others' results and says what it is.
template <class T>
__global__ void __launch_bounds__(MAX_THREADS) row_max_kernel(const T* logits, long long stride, int vocab, int32_t* targets, int blocks) {
    sd_chain_begin();
    auto cluster = cooperative_groups::this_cluster();
    if (blocks > 1) cluster.barrier_arrive();                     // (waited for before the first's memory is written to: it is there by then)
    constexpr int PER = 16 / sizeof(T), AHEAD = 4;
    const int rank = blockIdx.x % blocks, first = rank * MAX_THREADS, step = blocks * MAX_THREADS;
    const long long r = blockIdx.x / blocks;
    const T* row = logits + r * stride;
    const int t = threadIdx.x;
    const int head = min(vocab, (int)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(T));   // elements before the first 16-byte boundary
    const int whole = (vocab - head) / PER, tail = head + whole * PER;
    const uint4* chunk = (const uint4*)(row + head);
    uint32_t best = 0;
    int where = 0;                                                // chunk; -1: what is before them, `whole`: what is behind
    if (rank == 0 && t < head) { best = order_key(as_float(row[t])); where = -1; }
    int c = first + t;
    for (; c + (AHEAD - 1) * step < whole; c += AHEAD * step) {
        uint4 v[AHEAD];
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) v[e] = __ldcs(chunk + c + e * step);
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) {
            const uint32_t m = largest(v[e], T());
            if (m > best) { best = m; where = c + e * step; }
        }
    }
    for (; c < whole; c += step) {
        const uint32_t m = largest(__ldcs(chunk + c), T());
        if (m > best) { best = m; where = c; }
    }
    if (rank == 0 && t < vocab - tail) {
        const uint32_t m = order_key(as_float(row[tail + t]));
        if (m > best) { best = m; where = whole; }
    }
    unsigned long long all = (unsigned long long)best << 32 | (0xFFFFFFFEu - (uint32_t)where);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) all = max(all, __shfl_xor_sync(~0u, all, d));
    __shared__ unsigned long long s_all[MAX_THREADS / 32], s_block[8];
    if ((t & 31) == 0) s_all[t / 32] = all;
    __syncthreads();
    if (t < 32) {
        all = t < MAX_THREADS / 32 ? s_all[t] : 0;
#pragma unroll
        for (int d = MAX_THREADS / 64; d > 0; d >>= 1) all = max(all, __shfl_xor_sync(~0u, all, d));
    }
    if (blocks > 1) {
        cluster.barrier_wait();
        if (t == 0) *cluster.map_shared_rank(&s_block[rank], 0) = all;
        cluster.sync();
        if (rank) return;
        all = 0;
        for (int e = 0; e < blocks; ++e) all = max(all, s_block[e]);
    }
    if (t < 32) {
        const int won = (int)(0xFFFFFFFEu - (uint32_t)all), lo = won < 0 ? 0 : head + won * PER, n = won < 0 ? head : min(PER, vocab - lo);
        const bool it = t < n && order_key(as_float(row[lo + t])) == (uint32_t)(all >> 32);
        const unsigned found = __ballot_sync(~0u, it);
        if (t == 0) targets[r] = lo + __ffs(found) - 1;
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

// The accepted paths, a warp each, then their begins and tokens.  One block, or a cluster of them that take a part of the requests each and tell the others how
// many tokens it has.
constexpr int WALK_THREADS = 512, WALK_BLOCKS = 8;

__global__ void __launch_bounds__(WALK_THREADS) walk_kernel(const WalkArgs a) {
    sd_chain_begin();
    constexpr int WARPS = WALK_THREADS / 32;
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5, blocks = gridDim.x, rank = blockIdx.x;
    auto cluster = cooperative_groups::this_cluster();
    if (blocks > 1) cluster.barrier_arrive();                     // (waited for before the others' memory is written to: they are there by then)
    __shared__ long long s_sum[WARPS], s_base, s_first, s_block[WALK_BLOCKS];
    const int part = (a.n + blocks - 1) / blocks, lo_i = min(rank * part, a.n), hi_i = min(lo_i + part, a.n);
    for (int i = lo_i + warp; i < hi_i; i += WARPS) {
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
    __syncthreads();
    long long mine = 0;                                           // tokens of the block's requests
    if (blocks > 1) {
        for (int i = lo_i + t; i < hi_i; i += WALK_THREADS) mine += a.new_offsets[i + 1];
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) mine += __shfl_xor_sync(~0u, mine, d);
        if (lane == 0) s_sum[warp] = mine;
        __syncthreads();
        cluster.barrier_wait();
        if (t < blocks) {
            mine = 0;
            for (int w = 0; w < WARPS; ++w) mine += s_sum[w];
            *cluster.map_shared_rank(&s_block[rank], t) = mine;
        }
        cluster.sync();
    }
    if (t == 0) {
        long long before = 0;
        for (int e = 0; e < rank; ++e) before += s_block[e];
        s_base = before;
        s_first = min(before, (long long)a.rows);
        if (rank == 0) a.new_offsets[0] = 0;
    }
    __syncthreads();
    for (int first = lo_i; first < hi_i; first += WALK_THREADS) {  // begins: running sums of the lengths
        long long x = first + t < hi_i ? a.new_offsets[first + t + 1] : 0;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long y = __shfl_up_sync(~0u, x, d);
            if (lane >= d) x += y;
        }
        if (lane == 31) s_sum[warp] = x;
        __syncthreads();
        x += s_base;
        for (int w = 0; w < warp; ++w) x += s_sum[w];
        if (first + t < hi_i) a.new_offsets[first + t + 1] = min(x, (long long)a.rows);   // (more where offsets that descend give rows to two requests)
        __syncthreads();
        if (t == WALK_THREADS - 1) s_base = x;
        __syncthreads();
    }
    for (int i = lo_i + warp; i < hi_i; i += WARPS) {
        const long long lo = a.offsets[i], begin = i == lo_i ? s_first : a.new_offsets[i];   // (what is before the block's first is another block's)
        const int kept = (int)(a.new_offsets[i + 1] - begin);     // (less than the path where there is no room for it)
        int32_t* path = a.path + (long long)i * (a.M + 1);
#pragma unroll
        for (int e = 0; e < 3; ++e) {
            const int j = lane + 32 * e, p = j <= a.M ? path[j] : -1;
            if (p < 0) continue;
            if (j < kept) a.new_tokens[begin + j] = a.targets[lo + p];
            else path[j] = -1;
        }
    }
    if (rank == blocks - 1)
        for (long long k = s_base + t; k < a.rows; k += WALK_THREADS) a.new_tokens[k] = -1;
}

// ---- sd_commit -----------------------------------------------------------------------------
// A cluster per request, whose blocks take the planes (keys or values of a layer) in turns; a thread per 16 bytes of a line.  Lines only move to smaller
// places, and a path ascends: what a batch of lines overwrites, no later batch reads.  The new length is written when all blocks have read the old one, which
// may be the same memory.  256 requests, 32 layers, 8 heads of 128: 25 - 27 us; the 225 - 271 lines of them that move
// (100 requests move any) are 59 - 71 MB, 9 - 11 us of the memory's time: a thread has the two or three lines of one request and plane under way, one plane after another.  One request
// 4.6 - 5.1 us, the host's time (1.4 in a graph: path, table and line behind one another).
constexpr int COMMIT_BATCH = 4, COMMIT_THREADS = 256;

struct CommitArgs {
    sd_cache c;
    sd_rows b;
    const int32_t* path;
    int32_t* cached_out;
    int blocks;
};

__global__ void __launch_bounds__(COMMIT_THREADS) commit_kernel(const __grid_constant__ CommitArgs a) {
    sd_chain_begin();
    const sd_rows& b = a.b;
    const int i = blockIdx.x / a.blocks, rank = blockIdx.x % a.blocks, t = threadIdx.x;
    __shared__ long long s_src[2][SD_MAX_SPEC + 1], s_dst[2][SD_MAX_SPEC + 1];      // of keys, of values: elements from the plane's begin
    __shared__ int s_moves, s_bad;
    const int M1 = b.max_draft + 1, P = a.c.page_size;
    if (t == 0) { s_bad = 0; s_moves = 0; }
    const int cached = b.d_cached[i];
    const int32_t* path = a.path + (long long)i * M1;
    const int p = t < M1 ? path[t] : -1, before = t > 0 && t < M1 ? path[t - 1] : -1;
    const int kept = __syncthreads_count(p >= 0);
    if (t < M1 && (t < kept ? p <= before || p > b.max_draft || (t == 0 && p != 0) || cached < 0 || (long long)cached + p >= (long long)P * b.table_stride : p != -1))
        atomicOr(&s_bad, SD_STATUS_BAD_ROWS);
    const int bad_rows = __syncthreads_or(s_bad);
    if (!bad_rows) {                                              // (behind the first row that moves all do)
        const bool moves = t < kept && p != t;
        int src = -1, dst = -1;
        if (moves) {
            src = sd_page(b, a.c.n_pages, i, (cached + p) / P);
            dst = sd_page(b, a.c.n_pages, i, (cached + t) / P);
            if (src < 0 || dst < 0) atomicOr(&s_bad, SD_STATUS_BAD_PAGE);
        }
        if (moves) {
            const bool lines = src >= 0 && dst >= 0;
            const int sl = (cached + p) % P, dl = (cached + t) % P;
            s_src[0][t] = lines ? src * a.c.k_stride[1] + sl * a.c.k_stride[2] : -1;
            s_dst[0][t] = dst * a.c.k_stride[1] + dl * a.c.k_stride[2];
            s_src[1][t] = src * a.c.v_stride[1] + sl * a.c.v_stride[2];
            s_dst[1][t] = dst * a.c.v_stride[1] + dl * a.c.v_stride[2];
            atomicAdd(&s_moves, 1);
        }
    }
    __syncthreads();
    if (!bad_rows && s_moves) {
        const int begin = kept - s_moves, per = a.c.head_dim / 8, columns = a.c.kv_heads * per;
        for (int e = rank * COMMIT_THREADS + t; e < 2 * a.c.n_layers * columns; e += a.blocks * COMMIT_THREADS) {
            const int plane = e / columns, col = e - plane * columns, side = plane & 1, head = col / per;
            const int64_t* st = side ? a.c.v_stride : a.c.k_stride;
            uint16_t* at = (uint16_t*)(side ? a.c.d_v : a.c.d_k) + (plane >> 1) * st[0] + head * st[3] + (col - head * per) * 8;
            for (int first = begin; first < kept; first += COMMIT_BATCH) {
                uint4 v[COMMIT_BATCH];
#pragma unroll
                for (int j = 0; j < COMMIT_BATCH; ++j)
                    if (first + j < kept && s_src[0][first + j] >= 0) v[j] = *(const uint4*)(at + s_src[side][first + j]);
#pragma unroll
                for (int j = 0; j < COMMIT_BATCH; ++j)
                    if (first + j < kept && s_src[0][first + j] >= 0) *(uint4*)(at + s_dst[side][first + j]) = v[j];
            }
        }
    }
    if (a.blocks > 1) cooperative_groups::this_cluster().sync();
    if (rank == 0 && t == 0) {
        a.cached_out[i] = bad_rows ? cached : cached + kept;
        if (b.d_status) b.d_status[i] = s_bad;
    }
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
        if (!sd_out_strides_ok(prm->out_stride, rows->rows, prm->q_heads)) return SD_ERR_INVALID_ARG;
        for (int k = 0; k < 2; ++k)
            if (!sd_stride_ok(prm->q_stride[k]) || !sd_stride_ok(prm->k_stride[k]) || !sd_stride_ok(prm->v_stride[k]) || !sd_stride_ok(prm->out_stride[k]))
                return SD_ERR_INVALID_ARG;
    }
    rc = sd_check_pointer(cache->d_k);
    if (rc != SD_OK) return rc;
    // A row a block while that makes no more blocks than are at work at once; else four, which look up together.
    const int most = rows->max_draft + 1, per = (long long)rows->n * most <= 1024 ? 1 : ROT_ROWS, chunks = (std::min(most, std::max(rows->rows, 1)) + per - 1) / per;
    if ((long long)rows->n * chunks > 0x7FFFFFFF) return SD_ERR_INVALID_ARG;
    const RotateArgs a = {*cache, *rows, *prm, d_q, d_k, d_v, d_q_weight, d_k_weight, d_freq, d_positions, d_q_out, chunks, per};
    const unsigned grid = rows->n * chunks;
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
        // Up to eight blocks a row where the rows are too few to fill the device.
        int blocks = 1;
        while (blocks < 8 && rows * blocks < 128 && vocab / blocks >= 16 * MAX_THREADS) blocks *= 2;
        cudaError_t e;
#define SD_ROW_MAX(T) sd_launch_clusters(row_max_kernel<T>, (unsigned)rows * blocks, blocks, MAX_THREADS, 0, st, (const T*)d_logits, (long long)row_stride, vocab, d_targets, blocks)
        e = dtype == SD_BF16 ? SD_ROW_MAX(__nv_bfloat16) : dtype == SD_FP16 ? SD_ROW_MAX(__half) : SD_ROW_MAX(float);
#undef SD_ROW_MAX
        if (e != cudaSuccess) return SD_ERR_CUDA;
    }
    const WalkArgs a = {n, rows, max_draft, d_offsets, d_tokens, d_parents, d_targets, d_path, d_new_offsets, d_new_tokens, d_status};
    const int blocks = n > WALK_THREADS / 32 ? WALK_BLOCKS : 1;   // (a warp a request)
    return sd_launch_clusters(walk_kernel, blocks, blocks, WALK_THREADS, 0, st, a) == cudaSuccess ? SD_OK : SD_ERR_CUDA;
}

extern "C" int sd_commit(const sd_cache* cache, const sd_rows* rows, const int32_t* d_path, int32_t* d_new_cached, void* stream) {
    int rc = sd_check_cache(cache, rows);
    if (rc != SD_OK) return rc;
    if (cache->n_layers > 32767) return SD_ERR_INVALID_ARG;
    if (rows->n == 0) return SD_OK;
    if (!d_path || !d_new_cached) return SD_ERR_INVALID_ARG;
    rc = sd_check_pointer(cache->d_k);
    if (rc != SD_OK) return rc;
    // Eight blocks a request, fewer where there is not so much to move.
    const long long pieces = 2ll * cache->n_layers * cache->kv_heads * (cache->head_dim / 8);
    if (pieces > 0x7FFFFFFF / 2) return SD_ERR_INVALID_ARG;
    int blocks = 1;
    while (blocks < 8 && pieces > blocks * COMMIT_THREADS) blocks *= 2;
    if ((long long)rows->n * blocks > 0x7FFFFFFF) return SD_ERR_INVALID_ARG;
    const CommitArgs a = {*cache, *rows, d_path, d_new_cached, blocks};
    return sd_launch_clusters(commit_kernel, (unsigned)rows->n * blocks, blocks, COMMIT_THREADS, 0, (cudaStream_t)stream, a) == cudaSuccess ? SD_OK : SD_ERR_CUDA;
}
