// sd_attend: attention of the rows of draft trees over their requests' paged caches.
//
// The work is a list of UNITS: up to 256 rows of one request and one head of the cache (row and query head packed: row r, head g of the group is packed row
// r * group + g) times the 128-line TILES of the cache that any of them sees; with a shared prefix also units of 256 packed rows of the
// whole batch times the prefix's tiles.  The list is cut into as many equal pieces as there are blocks, in the middle of units where that
// falls so, so that every multiprocessor reads as much of the cache as any other, whatever the lengths; each block finds its piece from the lengths by itself.
// Rows of a unit that was cut are left as partial results (normalised, with the logarithm of their sum) and joined by a second kernel.
//
// A block is one producer warp (tiled copies of keys and values into a ring in shared memory), one warp that issues the products, one that walks the
// list, and two groups of four warps that compute the softmax, a thread per row.  Two chains of (scores, softmax, product with the values)
// are in flight, one per group: for a unit of up to 128 rows the groups take tiles in turns and join their results at the end, for a larger one each has 128 rows of every tile.
// While one group is at its softmax the tensor cores work for the other.  Scores and results are in tensor memory; the weights go back over the scores
// and are read from there.
#include "blackwell.cuh"
#include "verify.cuh"

#include <algorithm>

namespace {

constexpr int TILE = 128;                                         // lines of the cache a step
constexpr int THREADS = 384;                                      // four warps that feed, eight that compute
constexpr int UNITS = 2;                                          // units that the list's walker is ahead
constexpr float RESCALE = 8.0f;                                   // results are rescaled when a row's maximum has grown by 2^8 (weights stay below that)

struct AttendArgs {
    sd_cache c;
    sd_rows b;
    sd_attend_params p;
    const void* q;
    void* out;
    float* lse;
    struct Cut* cuts;             // [grid]: the unit that begins in block c and is cut
    float* part;                  // [2 * grid][256][D]: rows of a cut unit; slot 2c: it came from the block before, 2c + 1: it goes on in the next
    float* part_lse;              // [2 * grid][256]
    float* plane[2];              // with a shared prefix: [rows * q_heads][D], what is behind it and it
    float* plane_lse[2];          // [rows * q_heads]
};

struct Cut {
    int first, last;              // blocks that have a part of it; none where last < first
    int rows, m0, head, prefix;
    long long begin;
};

enum { DONE = 0, TAIL = 1, PREFIX = 2 };
enum { FINAL = 0, PLANE = 1, SLOT = 2 };

struct Unit {
    long long begin;              // row of the row arrays that packed row 0 belongs to
    int kind;
    int request, head;
    int m0, rows;                 // packed rows
    int cached, count;            // of the request
    int k0, k1;                   // steps: of the unit's list of tiles
    int sink_tiles, next_tile;    // the list: tiles 0 .. sink_tiles - 1, then from next_tile on
    int to, slot;                 // FINAL, PLANE, SLOT
};

// Tiles that request r needs.
struct Tiles {
    int sinks, next, count;
};
__device__ __forceinline__ Tiles tiles_of(const sd_attend_params& p, int prefix_tiles, const Request& r) {
    Tiles t;
    const int all = (r.cached + r.count + TILE - 1) / TILE;
    t.sinks = 0;
    t.next = prefix_tiles;
    if (p.window) {
        t.next = max(0, r.cached - p.window + 1) / TILE;
        t.sinks = min(min(p.sinks, r.cached) + TILE - 1, r.cached + TILE - 1) / TILE;
        if (t.sinks >= t.next) { t.sinks = 0; t.next = 0; }
    }
    t.count = t.sinks + all - t.next;
    return t;
}

template <int D>
struct Shape {
    static constexpr int HALVES = D / 64;
    static constexpr int SLOT_BYTES = TILE * D * 2, HALF_BYTES = TILE * 128;
    static constexpr int SLOTS = D == 128 ? 5 : 8;
    static constexpr int Q_BYTES = 128 * D * 2;
    static constexpr int RING = 0, Q = SLOTS * SLOT_BYTES, REST = Q + 2 * Q_BYTES;
};

struct Rest {                     // of shared memory
    uint64_t full[8], empty[8], s_full[2], p_ready[2], o_done[2], q_full, unit_full[UNITS], unit_empty[UNITS], meet, group_meet[2], over;
    uint32_t tmem;
    int stop;
    int begun[2];                 // the group has begun its results itself: the first product adds to them
    uint32_t lines[2][4];         // lines of the group's tile with values that are no numbers
    Unit units[UNITS];
};
template <int D> constexpr int smem_bytes() { return Shape<D>::REST + (int)sizeof(Rest); }

__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float lg2(float x) { float y; asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// Bits of the places [a, b) among the 32 from `at` on.
__device__ __forceinline__ uint32_t range_bits(int a, int b, int at) {
    const int lo = min(max(a - at, 0), 32), hi = min(max(b - at, 0), 32);
    return hi <= lo ? 0u : (0xFFFFFFFFu >> (32 - hi)) & (0xFFFFFFFFu << lo);
}

// What a row sees: places [0, sinks) and [from, cached), and of the rows of its request row 0 (root) and those of `tree`.
struct Sight {
    int sinks, from, cached;
    bool root;
    unsigned long long tree;
    __device__ __forceinline__ uint32_t word(int at) const {
        uint32_t w = range_bits(from, cached, at) | range_bits(0, sinks, at);
        const int s = at - cached;                                // the word's first place, as a row
        const unsigned long long lo = tree << 1 | (unsigned long long)root, hi = tree >> 63;
        if (s > -32 && s <= 64) w |= s < 0 ? (uint32_t)(lo << -s) : s < 64 ? (uint32_t)(lo >> s | (s ? hi << (64 - s) : 0)) : (uint32_t)hi;
        return w;
    }
};

template <class T> struct IsBf16 { static constexpr bool v = false; };
template <> struct IsBf16<__nv_bfloat16> { static constexpr bool v = true; };

// ---- the list's walker ---------------------------------------------------------------------
template <int D>
__device__ void walk_units(const AttendArgs& a, Rest* s, int lane) {
    const sd_rows& b = a.b;
    const int G = a.p.q_heads / a.c.kv_heads, H = a.c.kv_heads;
    const int prefix_tiles = a.p.window ? 0 : a.p.shared / TILE;
    long long total_rows = b.d_offsets[b.n];
    total_rows = total_rows < 0 ? 0 : total_rows > b.rows ? b.rows : total_rows;
    // a unit costs its tiles and one more, for its begin and end
    auto cost_of = [&](int i, Request& r, Tiles& t) -> long long {
        r = sd_request(b, i, a.c.page_size, a.p.shared);
        if (!r.count) return 0;
        t = tiles_of(a.p, prefix_tiles, r);
        return (long long)H * ((r.count * G + 255) / 256) * (t.count + 1);
    };
    long long sum = 0;
    int some = 0x7FFFFFFF;                                        // a request with rows: the prefix is read through its pages
    for (int i = lane; i < b.n; i += 32) {
        Request r; Tiles t;
        sum += cost_of(i, r, t);
        if (r.count) some = min(some, i);
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        sum += __shfl_xor_sync(~0u, sum, d);
        some = min(some, __shfl_xor_sync(~0u, some, d));
    }
    const long long groups = (total_rows * G + 255) / 256, prefix_cost = prefix_tiles && sum ? H * groups * (prefix_tiles + 1) : 0;
    const long long all = sum + prefix_cost;
    const long long quota = max((all + gridDim.x - 1) / gridDim.x, 4ll);
    const long long lo = min(quota * blockIdx.x, all), hi = min(lo + quota, all);
    Cut cut;
    cut.first = 0; cut.last = -1;

    int at = 0;                                                   // units handed out
    bool ok = true;
    // unit u of a run of them, `tiles` each, that begins at `base` of the list; false: the piece ends before it
    auto hand_out = [&](Unit& u, long long begin, int tiles) -> bool {
        if (begin >= hi) return false;
        const long long first = begin + 1, end = first + tiles;   // of its tiles
        u.k0 = (int)(max(first, lo) - first); u.k1 = (int)(min(end, hi) - first);
        if (u.k1 <= u.k0) return true;
        const bool whole = u.k0 == 0 && u.k1 == tiles;
        u.to = !whole ? SLOT : prefix_tiles ? PLANE : FINAL;
        u.slot = whole ? (u.kind == PREFIX) : 2 * blockIdx.x + (u.k0 == 0);
        if (!whole && u.k0 == 0) {
            cut.first = blockIdx.x; cut.last = (int)((end - 1) / quota);
            cut.rows = u.rows; cut.m0 = u.m0; cut.head = u.head; cut.prefix = u.kind == PREFIX; cut.begin = u.begin;
        }
        const int e = at % UNITS;
        ok = at < UNITS || bw_wait_warp(bw_smem(&s->unit_empty[e]), (at / UNITS - 1) & 1, &s->stop);
        if (!ok) return false;
        if (lane == 0) {
            s->units[e] = u;
            bw_arrive(bw_smem(&s->unit_full[e]));
        }
        ++at;
        return true;
    };
    if (hi > lo) {
        Unit u;
        u.sink_tiles = 0;
        bool more = true;
        if (lo < prefix_cost) {
            const int per = prefix_tiles + 1;
            u.kind = PREFIX; u.request = some; u.begin = 0; u.cached = a.p.shared; u.count = 0; u.next_tile = 0;
            for (long long k = lo / per; more && k < H * groups; ++k) {
                u.head = (int)(k / groups); u.m0 = (int)(k % groups) * 256;
                u.rows = (int)min(256ll, total_rows * G - u.m0);
                more = hand_out(u, k * per, prefix_tiles);
            }
        }
        long long base = prefix_cost;
        u.kind = TAIL;
        for (int first = 0; more && first < b.n && base < hi; first += 32) {      // 32 requests at a time, then those of them that the piece touches
            Request r; Tiles t = {0, 0, 0};
            r.count = 0;
            long long cost = 0;
            if (first + lane < b.n) cost = cost_of(first + lane, r, t);
            long long end = cost;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const long long x = __shfl_up_sync(~0u, end, d);
                if (lane >= d) end += x;
            }
            end += base;
            unsigned touched = __ballot_sync(~0u, cost > 0 && end > lo && end - cost < hi);
            while (more && touched) {
                const int l = __ffs(touched) - 1;
                touched &= touched - 1;
                const long long begin = __shfl_sync(~0u, end - cost, l);
                u.request = first + l;
                u.begin = __shfl_sync(~0u, r.begin, l); u.cached = __shfl_sync(~0u, r.cached, l); u.count = __shfl_sync(~0u, r.count, l);
                u.sink_tiles = __shfl_sync(~0u, t.sinks, l); u.next_tile = __shfl_sync(~0u, t.next, l);
                const int tiles = __shfl_sync(~0u, t.count, l), per = tiles + 1, packed = u.count * G, parts = (packed + 255) / 256;
                for (long long k = max(0ll, lo - begin) / per; more && k < (long long)H * parts; ++k) {
                    u.head = (int)(k / parts); u.m0 = (int)(k % parts) * 256;
                    u.rows = min(256, packed - u.m0);
                    more = hand_out(u, begin + k * per, tiles);
                }
            }
            base = __shfl_sync(~0u, end, 31);
        }
    }
    if (lane == 0 && a.cuts) a.cuts[blockIdx.x] = cut;
    const int e = at % UNITS;
    if (ok && (at < UNITS || bw_wait_warp(bw_smem(&s->unit_empty[e]), (at / UNITS - 1) & 1, &s->stop)) && lane == 0) {
        s->units[e].kind = DONE;
        bw_arrive(bw_smem(&s->unit_full[e]));
    }
}

// Pages that a request's rows see: told where one is none of the cache's.
__device__ void write_status(const AttendArgs& a, int lane) {
    const sd_rows& b = a.b;
    for (int i = blockIdx.x; i < b.n; i += gridDim.x) {
        const Request r = sd_request(b, i, a.c.page_size, a.p.shared);
        int st = r.status;
        if (r.count) {
            const int P = a.c.page_size, from = a.p.window ? max(0, r.cached - a.p.window + 1) : 0;
            const int sinks = a.p.window ? min(min(a.p.sinks, r.cached), from) : 0;
            bool bad = false;
            for (int e = lane; e < (sinks + P - 1) / P; e += 32) bad |= sd_page(b, a.c.n_pages, i, e) < 0;
            for (int e = from / P + lane; e <= (r.cached + r.count - 1) / P; e += 32) bad |= sd_page(b, a.c.n_pages, i, e) < 0;
            if (__any_sync(~0u, bad)) st |= SD_STATUS_BAD_PAGE;
        }
        if (lane == 0) b.d_status[i] = st;
    }
}

// ---- copies --------------------------------------------------------------------------------
template <int D>
__device__ void produce(const AttendArgs& a, const CUtensorMap* mk, const CUtensorMap* mv, Rest* s, uint32_t ring, int box, int lane) {
    using S = Shape<D>;
    const int P = a.c.page_size;
    uint32_t it = 0;                                              // slots filled
    for (int n = 0;; ++n) {
        if (!bw_wait_warp(bw_smem(&s->unit_full[n % UNITS]), (n / UNITS) & 1, &s->stop)) break;
        const Unit u = s->units[n % UNITS];
        bw_arrive_warp(bw_smem(&s->unit_empty[n % UNITS]));
        if (u.kind == DONE) return;
        const int piece = lane / S::HALVES, half = lane % S::HALVES;
        auto place_of = [&](int k) { return TILE * (k < u.sink_tiles ? k : u.next_tile + k - u.sink_tiles) + piece * box; };
        const int length = u.kind == PREFIX ? u.cached : u.cached + u.count;
        auto page_of = [&](int k) {
            const int p = place_of(k);
            if (k >= u.k1 || piece * box >= TILE || p >= length) return -1;
            const int page = sd_page(a.b, a.c.n_pages, u.request, p / P);
            return page < 0 ? a.c.n_pages : page;                 // (a page that is none: beyond the last, where a copy fills in zeros)
        };
        int page = page_of(u.k0);
        bool ok = true;
        for (int k = u.k0; k < u.k1 && ok; ++k) {
            const int next = page_of(k + 1), line = place_of(k) % P;
            const int boxes = __popc(__ballot_sync(~0u, page >= 0));
            for (int v = 0; v < 2 && ok; ++v, ++it) {
                const uint32_t e = it % S::SLOTS, bar = bw_smem(&s->full[e]);
                ok = it < S::SLOTS || bw_wait_warp(bw_smem(&s->empty[e]), (it / S::SLOTS - 1) & 1, &s->stop);
                if (!ok) break;
                if (lane == 0) bw_arrive_expect(bar, boxes * box * 128);
                __syncwarp();
                if (page >= 0) bw_load_4d(ring + e * S::SLOT_BYTES + half * S::HALF_BYTES + piece * box * 128, v ? mv : mk, half * 64, line, u.head, page, bar);
            }
            page = next;
        }
        if (!ok) break;
    }
    for (uint32_t e = 0; e < S::SLOTS && e < it; ++e) {           // given up: the copies in flight come to their end
        const uint32_t last = (it - 1 - e) / S::SLOTS * S::SLOTS + e;
        int never = 0;
        bw_wait_slow(bw_smem(&s->full[e]), (last / S::SLOTS) & 1, &never, 200000000ll);
    }
}

// ---- products ------------------------------------------------------------------------------
// (One thread.)  False: given up.
template <class T, int D>
__device__ bool multiply(Rest* s, uint32_t ring, uint32_t q, uint32_t tmem) {
    using S = Shape<D>;
    constexpr uint32_t qk = bw_idesc(IsBf16<T>::v, 128, TILE, false), pv = bw_idesc(IsBf16<T>::v, 128, D, true);
    uint32_t it = 0, count[2] = {0, 0};
    for (int n = 0;; ++n) {
        if (!bw_wait(bw_smem(&s->unit_full[n % UNITS]), (n / UNITS) & 1, &s->stop)) return false;
        const int kind = s->units[n % UNITS].kind, tiles = s->units[n % UNITS].k1 - s->units[n % UNITS].k0, rows = s->units[n % UNITS].rows;
        bw_arrive(bw_smem(&s->unit_empty[n % UNITS]));
        if (kind == DONE) return true;
        const bool wide = rows > 128;
        const int jobs = wide ? 2 * tiles : tiles;
        if (!bw_wait(bw_smem(&s->q_full), n & 1, &s->stop)) return false;
        auto scores = [&](int j) -> bool {
            const int w = j & 1, tile = wide ? j >> 1 : j;
            const uint32_t e = (it + 2 * tile) % S::SLOTS;
            if (!bw_wait(bw_smem(&s->full[e]), ((it + 2 * tile) / S::SLOTS) & 1, &s->stop)) return false;
            bw_fence_after();
            const uint32_t qa = q + (wide ? w * S::Q_BYTES : 0), ka = ring + e * S::SLOT_BYTES;
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                const uint32_t off = k / 4 * S::HALF_BYTES + k % 4 * 32;
                bw_mma(tmem + w * TILE, bw_desc(qa + off), bw_desc(ka + off), qk, k > 0);
            }
            bw_commit(bw_smem(&s->s_full[w]));
            if (!wide || w) bw_commit(bw_smem(&s->empty[e]));
            return true;
        };
        for (int j = 0; j < min(jobs, 2); ++j)
            if (!scores(j)) return false;
        for (int j = 0; j < jobs; ++j) {
            const int w = j & 1, tile = wide ? j >> 1 : j;
            const uint32_t e = (it + 2 * tile + 1) % S::SLOTS;
            if (!bw_wait(bw_smem(&s->full[e]), ((it + 2 * tile + 1) / S::SLOTS) & 1, &s->stop)) return false;
            if (!bw_wait(bw_smem(&s->p_ready[w]), count[w]++ & 1, &s->stop)) return false;
            bw_fence_after();
            const bool add = j >= 2 || *(volatile int*)&s->begun[w];
            const uint32_t va = ring + e * S::SLOT_BYTES;
#pragma unroll
            for (int k = 0; k < TILE / 16; ++k)
                bw_mma_ts(tmem + 2 * TILE + w * TILE, tmem + w * TILE + k * 8, bw_desc_across(va + k * 2048, S::HALF_BYTES), pv, add || k > 0);
            if (!wide || w) bw_commit(bw_smem(&s->empty[e]));
            if (j + 2 >= jobs) bw_commit(bw_smem(&s->o_done[w]));
            else if (!scores(j + 2)) return false;
        }
        it += 2 * tiles;
    }
}

// ---- softmax -------------------------------------------------------------------------------
template <class T, int D>
struct Softmax {
    using S = Shape<D>;
    static constexpr float BIAS = IsBf16<T>::v ? 0.0f : 7.0f;     // fp16 weights are 2^7 as large: more of the small ones are above its least number
    const AttendArgs& a;
    Rest* s;
    uint8_t* base;                                                // of shared memory
    uint32_t tmem;                                                // with the warp's lanes
    const int w, t;                                               // group, thread in it: packed row of its tile
    uint32_t meets = 0, group_meets = 0, s_count = 0, o_count[2] = {0, 0}, it = 0;
    float scale;                                                  // of scores, for powers of two; its sign is in the queries

    __device__ bool meet() { bw_arrive_warp(bw_smem(&s->meet)); return bw_wait_warp(bw_smem(&s->meet), meets++ & 1, &s->stop); }

    __device__ bool meet_of(bool both) {
        if (both) return meet();
        bw_arrive_warp(bw_smem(&s->group_meet[w]));
        return bw_wait_warp(bw_smem(&s->group_meet[w]), group_meets++ & 1, &s->stop);
    }

    __device__ void load_q(const Unit& u, int G, bool wide) {
        const int m = u.m0 + (wide ? w * 128 : 0) + t;
        const bool row = (wide ? w * 128 : 0) + t < u.rows;
        const int r = m / G;
        const uint4* src = (const uint4*)((const T*)a.q + (u.begin + r) * a.p.q_stride[0] + (long long)(u.head * G + m - r * G) * a.p.q_stride[1]);
        uint8_t* to = base + S::Q + (wide ? w * S::Q_BYTES : 0) + t * 128;
        constexpr int PIECES = D / 8;
        const int first = wide ? 0 : w * (PIECES / 2), count = wide ? PIECES : PIECES / 2;
        const uint32_t flip = a.p.scale < 0.f ? 0x80008000u : 0u, keep = a.p.scale == 0.f ? 0u : ~0u;
#pragma unroll 8
        for (int k = 0; k < count; ++k) {
            const int c = first + k;
            uint4 x = make_uint4(0, 0, 0, 0);
            if (row) x = src[c];
            x.x = (x.x ^ flip) & keep; x.y = (x.y ^ flip) & keep; x.z = (x.z ^ flip) & keep; x.w = (x.w ^ flip) & keep;
            *(uint4*)(to + c / 8 * S::HALF_BYTES + ((c % 8) ^ (t & 7)) * 16) = x;
        }
        bw_fence_async();
        bw_arrive_warp(bw_smem(&s->q_full));
    }

    __device__ Sight sight(const Unit& u, int G, bool row, int r) {
        Sight g = {0, 0, u.cached, false, 0ull};
        if (!row || u.kind != TAIL) return g;
        const sd_rows& b = a.b;
        const unsigned long long bits = sd_tree_bits(b, u.request, r), here = u.count >= 65 ? ~0ull : (1ull << (u.count - 1)) - 1;
        g.root = true;
        g.tree = bits & here;
        const int W = a.p.window;
        if (W) {
            const int at = u.cached + __popcll(bits);             // the row's position
            g.from = max(0, at - W + 1);
            g.sinks = min(a.p.sinks, u.cached);
            if (W <= SD_MAX_SPEC) {                               // rows of the tree may be outside the window
                g.root = at - u.cached < W || u.cached < a.p.sinks;
                for (unsigned long long left = g.tree; left; left &= left - 1) {
                    const int j = __ffsll(left) - 1, p = u.cached + __popcll(sd_tree_bits(b, u.request, j + 1));
                    if (at - p >= W && p >= a.p.sinks) g.tree &= ~(1ull << j);
                }
            }
        }
        if (a.p.shared / TILE && !W) g.from = a.p.shared / TILE * TILE;
        return g;
    }

    // A weight of 0 does not take a value that is no number out of a product.  Lines of a masked tile that hold such are cleared, and what rows do see of them is added
    // to the results here, line by line.  (`values`: the tile.)  Called by a whole group, or by both where both use the tile.
    __device__ bool clear_lines(uint8_t* values, bool both, bool busy, bool first, const uint32_t* words, float power) {
        uint8_t* mine = values + t * 128;
        uint32_t found = 0;
#pragma unroll
        for (int c = 0; c < D / 8; ++c) {
            const uint4 x = *(const uint4*)(mine + c / 8 * S::HALF_BYTES + ((c % 8) ^ (t & 7)) * 16);
            found |= no_number(x.x) | no_number(x.y) | no_number(x.z) | no_number(x.w);
        }
        const uint32_t of_warp = __ballot_sync(~0u, found != 0);
        if ((t & 31) == 0) s->lines[w][t >> 5] = of_warp;
        if (!meet_of(both)) return false;
        uint32_t lines[4], any = 0;
#pragma unroll
        for (int c = 0; c < 4; ++c) any |= lines[c] = s->lines[w][c];
        if (!any) return true;
        const uint32_t S0 = tmem + w * TILE, O0 = tmem + 2 * TILE + w * TILE;
        if (busy) {
            if (first)                                            // the results begin here
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    uint32_t x[32] = {};
                    bw_st32(O0 + c, x);
                }
            bw_wait_st();
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
                const uint32_t word = words[c];
                for (uint32_t left = lines[c]; left; left &= left - 1) {
                    const int l = 32 * c + __ffs(left) - 1;
                    const bool seen = word >> (l & 31) & 1;
                    if (!__any_sync(~0u, seen)) continue;
                    const float p = ex2(fmaf(__uint_as_float(bw_ld1(S0 + l)), scale, -power));
#pragma unroll 1
                    for (int d = 0; d < D; d += 32) {
                        uint32_t x[32];
                        bw_ld32(O0 + d, x);
                        bw_wait_ld32(x);
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            const int at = d + e;
                            const float2 v = Elem<T>::up(*(const uint32_t*)(values + l * 128 + at / 64 * S::HALF_BYTES + ((at % 64 / 8) ^ (l & 7)) * 16 + at % 8 * 2));
                            if (seen) {
                                x[e] = __float_as_uint(__uint_as_float(x[e]) + p * v.x);
                                x[e + 1] = __float_as_uint(__uint_as_float(x[e + 1]) + p * v.y);
                            }
                        }
                        bw_st32(O0 + d, x);
                        bw_wait_st();
                    }
                }
            }
        }
        if (first && t == 0) s->begun[w] = 1;
        if (!meet_of(both)) return false;
        if (found && (w == 0 || !both)) {
#pragma unroll
            for (int c = 0; c < D / 8; ++c) *(uint4*)(mine + c / 8 * S::HALF_BYTES + c % 8 * 16) = make_uint4(0, 0, 0, 0);
            bw_fence_async();
        }
        __syncwarp();
        return both ? meet() : true;
    }

    // Whether any of the two 16-bit numbers of a word is none (all bits of the exponent set).
    static __device__ __forceinline__ uint32_t no_number(uint32_t x) {
        constexpr uint32_t E = IsBf16<T>::v ? 0x7F807F80u : 0x7C007C00u, ONE = IsBf16<T>::v ? 0x00800080u : 0x04000400u;
        return ((x & E) + ONE) & 0x80008000u;
    }

    __device__ bool run(const Unit& u, int n);
};

template <class T, int D>
__device__ bool Softmax<T, D>::run(const Unit& u, int n) {
    const int G = a.p.q_heads / a.c.kv_heads, warp = t >> 5;
    const bool wide = u.rows > 128;
    const int tiles = u.k1 - u.k0, jobs = wide ? 2 * tiles : tiles, mrow = (wide ? w * 128 : 0) + t;
    const bool row = mrow < u.rows;
    const bool busy = (wide ? w * 128 : 0) + warp * 32 < u.rows;  // any row of the warp
    const int r = (u.m0 + mrow) / G;
    if (!meet()) return false;                                    // both groups are through with the unit before: its queries, its results
    load_q(u, G, wide);
    const Sight see = sight(u, G, row, r);
    if (t == 0) s->begun[w] = 0;
    // tiles that every row sees whole
    const int W = a.p.window, plain_to = u.cached, plain_from = W ? u.cached + SD_MAX_SPEC - W + 1 : 0, plain_sinks = W ? min(a.p.sinks, u.cached) : 0;
    const uint32_t S0 = tmem + w * TILE, O0 = tmem + 2 * TILE + w * TILE;
    float top = -INFINITY, sum = 0.f;                             // the row's reference for powers, and its sum

    for (int j = w; j < jobs; j += 2) {
        const int k = u.k0 + (wide ? j >> 1 : j);
        const int p0 = TILE * (k < u.sink_tiles ? k : u.next_tile + k - u.sink_tiles);
        const bool masked = u.kind == TAIL && !(p0 + TILE <= plain_to && (p0 >= plain_from || p0 + TILE <= plain_sinks));
        if (!bw_wait_warp(bw_smem(&s->s_full[w]), s_count++ & 1, &s->stop)) return false;
        bw_fence_after();
        uint32_t words[4] = {~0u, ~0u, ~0u, ~0u};
        if (masked)
#pragma unroll
            for (int c = 0; c < 4; ++c) words[c] = see.word(p0 + 32 * c);
        float alpha = 1.0f;
        bool rescale = false;
        float power = 0.f;
        if (busy) {
            float mx = -INFINITY;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t x[32];
                bw_ld32(S0 + 32 * c, x);
                bw_wait_ld32(x);
                if (masked) {
#pragma unroll
                    for (int e = 0; e < 32; ++e) mx = fmaxf(mx, words[c] >> e & 1 ? __uint_as_float(x[e]) : -INFINITY);
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) mx = fmaxf(mx, __uint_as_float(x[e]));
                }
            }
            const bool up = mx != -INFINITY && !((mx - top) * scale <= RESCALE);
            if (up) {
                alpha = ex2((top - mx) * scale);
                sum *= alpha;
                top = mx;
            }
            rescale = __any_sync(~0u, up) && j >= 2;
            power = (top == -INFINITY ? 0.f : top * scale) - BIAS;
            if (rescale) {
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    uint32_t x[32];
                    bw_ld32(O0 + c, x);
                    bw_wait_ld32(x);
#pragma unroll
                    for (int e = 0; e < 32; ++e) x[e] = __float_as_uint(__uint_as_float(x[e]) * alpha);
                    bw_st32(O0 + c, x);
                }
            }
        }
        if (masked) {
            const uint32_t v = it + 2 * (wide ? j >> 1 : j) + 1;
            if (!bw_wait_warp(bw_smem(&s->full[v % S::SLOTS]), (v / S::SLOTS) & 1, &s->stop)) return false;
            if (!clear_lines(base + S::RING + v % S::SLOTS * S::SLOT_BYTES, wide, busy, j < 2, words, power)) return false;
        }
        if (busy) {
            float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < 4; c += 2) {
                uint32_t out[32];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t x[32];
                    bw_ld32(S0 + 32 * (c + h), x);
                    bw_wait_ld32(x);
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        float p = ex2(fmaf(__uint_as_float(x[e]), scale, -power)), q = ex2(fmaf(__uint_as_float(x[e + 1]), scale, -power));
                        if (masked) {
                            p = words[c + h] >> e & 1 ? p : 0.f;
                            q = words[c + h] >> (e + 1) & 1 ? q : 0.f;
                        }
                        part[e % 4] += p;
                        part[e % 4 + 1] += q;
                        out[16 * h + e / 2] = Elem<T>::down(p, q);
                    }
                }
                bw_st32(S0 + 16 * c, out);
            }
            sum += (part[0] + part[1]) + (part[2] + part[3]);
        }
        bw_wait_st();
        bw_fence_before();
        bw_arrive_warp(bw_smem(&s->p_ready[w]));
    }

    // ---- results
    const long long grow = u.begin + r;
    const int h = u.head * G + (u.m0 + mrow - r * G);
    auto place = [&](float*& to, float*& to_lse) {
        if (u.to == SLOT) { to = a.part + ((long long)u.slot * 256 + mrow) * D; to_lse = a.part_lse + (long long)u.slot * 256 + mrow; }
        else { const long long at = grow * a.p.q_heads + h; to = a.plane[u.slot] + at * D; to_lse = a.plane_lse[u.slot] + at; }
    };
    auto put = [&](const float* x, int c, int count) {            // columns c ..
        if (u.to == FINAL) {
            T* to = (T*)a.out + grow * a.p.out_stride[0] + h * a.p.out_stride[1] + c;
#pragma unroll
            for (int e = 0; e < 32; e += 8)
                if (e < count) *(uint4*)(to + e) = sd_pack<T>(x + e);
        } else {
            float *to, *to_lse;
            place(to, to_lse);
#pragma unroll
            for (int e = 0; e < 32; e += 4)
                if (e < count) *(float4*)(to + c + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
        }
    };
    auto put_lse = [&](float m, float l) {
        const float v = l == 0.f ? -INFINITY : m * scale + lg2(l) - BIAS;
        if (u.to == FINAL) { if (a.lse) a.lse[grow * a.p.q_heads + h] = v * 0.69314718055994531f; }
        else {
            float *to, *to_lse;
            place(to, to_lse);
            *to_lse = v;
        }
    };
    if (wide) {
        if (!bw_wait_warp(bw_smem(&s->o_done[w]), o_count[w]++ & 1, &s->stop)) return false;
        o_count[w ^ 1]++;
        bw_fence_after();
        if (busy) {
            const float inv = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
                uint32_t x[32];
                bw_ld32(O0 + c, x);
                bw_wait_ld32(x);
                float y[32];
#pragma unroll
                for (int e = 0; e < 32; ++e) y[e] = sum == 0.f ? 0.f : __uint_as_float(x[e]) * inv;
                if (row) put(y, c, 32);
                __syncwarp();
            }
            if (row) put_lse(top, sum);
        }
    } else {
        float2* ml = (float2*)(base + S::Q + S::Q_BYTES);         // (the second queries' place, which such a unit does not use)
        ml[w * 128 + t] = make_float2(top, sum);
        if (!meet()) return false;
        if (!bw_wait_warp(bw_smem(&s->o_done[0]), o_count[0]++ & 1, &s->stop)) return false;
        if (jobs > 1 && !bw_wait_warp(bw_smem(&s->o_done[1]), o_count[1]++ & 1, &s->stop)) return false;
        bw_fence_after();
        if (busy) {
            const float2 x0 = ml[t], x1 = ml[128 + t];
            const float m = fmaxf(x0.x, x1.x), ref = m == -INFINITY ? 0.f : m;
            const float f0 = ex2((x0.x - ref) * scale), f1 = jobs > 1 ? ex2((x1.x - ref) * scale) : 0.f;
            const float l = x0.y * f0 + (jobs > 1 ? x1.y * f1 : 0.f), inv = l == 0.f ? 0.f : 1.0f / l;
            const float g0 = f0 * inv, g1 = f1 * inv;
#pragma unroll 1
            for (int c = w * (D / 2); c < (w + 1) * (D / 2); c += 32) {
                uint32_t x[32], z[32];
                bw_ld32(tmem + 2 * TILE + c, x);
                bw_wait_ld32(x);
                if (jobs > 1) {
                    bw_ld32(tmem + 3 * TILE + c, z);
                    bw_wait_ld32(z);
                }
                float y[32];
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                    y[e] = g0 == 0.f ? 0.f : __uint_as_float(x[e]) * g0;
                    if (jobs > 1 && g1 != 0.f) y[e] += __uint_as_float(z[e]) * g1;
                    if (l == 0.f) y[e] = 0.f;
                }
                if (row) put(y, c, 32);
                __syncwarp();
            }
            if (row && w == 0) put_lse(m, l);
        }
    }
    bw_fence_before();
    it += 2 * tiles;
    return true;
}

template <class T, int D>
__global__ void __launch_bounds__(THREADS, 1) attend_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv, int box) {
    using S = Shape<D>;
    extern __shared__ __align__(1024) uint8_t smem[];
    Rest* s = (Rest*)(smem + S::REST);
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
    if (t == 0) {
        for (int e = 0; e < S::SLOTS; ++e) { bw_bar_init(bw_smem(&s->full[e]), 1); bw_bar_init(bw_smem(&s->empty[e]), 1); }
        for (int e = 0; e < 2; ++e) { bw_bar_init(bw_smem(&s->s_full[e]), 1); bw_bar_init(bw_smem(&s->p_ready[e]), 4); bw_bar_init(bw_smem(&s->o_done[e]), 1); }
        for (int e = 0; e < UNITS; ++e) { bw_bar_init(bw_smem(&s->unit_full[e]), 1); bw_bar_init(bw_smem(&s->unit_empty[e]), 10); }
        bw_bar_init(bw_smem(&s->q_full), 8);
        bw_bar_init(bw_smem(&s->meet), 8);
        bw_bar_init(bw_smem(&s->group_meet[0]), 4); bw_bar_init(bw_smem(&s->group_meet[1]), 4);
        bw_bar_init(bw_smem(&s->over), 1);
        s->stop = 0; s->begun[0] = s->begun[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        bw_prefetch_map(&mk); bw_prefetch_map(&mv);
    }
    if (warp == 1) bw_tmem_alloc(bw_smem(&s->tmem), 512);
    bw_fence_before();
    __syncthreads();
    bw_fence_after();
    sd_chain_begin();
    const uint32_t tmem = s->tmem, ring = bw_smem(smem + S::RING);
    if (warp == 0) produce<D>(a, &mk, &mv, s, ring, box, lane);
    else if (warp == 1) {
        if (lane == 0 && !multiply<T, D>(s, ring, bw_smem(smem + S::Q), tmem)) {
            int never = 0;                                        // the products in flight come to their end
            bw_commit(bw_smem(&s->over));
            bw_wait_slow(bw_smem(&s->over), 0, &never, 200000000ll);
        }
    } else if (warp == 2) walk_units<D>(a, s, lane);
    else if (warp == 3) {
        if (a.b.d_status) write_status(a, lane);
    } else {
        Softmax<T, D> f = {a, s, smem, tmem + ((uint32_t)(warp & 3) << 21), (warp - 4) >> 2, (t - 128) & 127};
        f.scale = a.p.scale == 0.f ? 1.4426950408889634f : fabsf(a.p.scale) * 1.4426950408889634f;
        for (int n = 0;; ++n) {
            if (!bw_wait_warp(bw_smem(&s->unit_full[n % UNITS]), (n / UNITS) & 1, &s->stop)) break;
            const Unit u = s->units[n % UNITS];
            bw_arrive_warp(bw_smem(&s->unit_empty[n % UNITS]));
            if (u.kind == DONE || !f.run(u, n)) break;
        }
    }
    __syncwarp();
    bw_fence_before();
    __syncthreads();
    if (warp == 1) {
        bw_fence_after();
        bw_tmem_free(tmem, 512);
    }
    if (s->stop && a.b.d_status)                                  // given up
        for (int i = t; i < a.b.n; i += THREADS) atomicOr(&a.b.d_status[i], SD_STATUS_FAILED);
}

// ---- joining -------------------------------------------------------------------------------
// A warp per row of a cut unit: its parts by their sums.
constexpr int JOIN_ROWS = 8;

template <class T, int D>
__device__ void join_row(const AttendArgs& a, const Cut& c, int m, int lane, bool planes) {
    constexpr int E = D / 32;
    const int G = a.p.q_heads / a.c.kv_heads, packed = c.m0 + m, r = packed / G, h = c.head * G + packed - r * G;
    auto slot = [&](int k) { return (long long)(2 * (c.first + k) + (k == 0)) * 256 + m; };
    const int parts = c.last - c.first + 1;
    float top = -INFINITY;
    bool nan = false;
    for (int k = lane; k < parts; k += 32) {
        const float v = a.part_lse[slot(k)];
        nan |= v != v;
        top = fmaxf(top, v);
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
    if (__any_sync(~0u, nan)) top = NAN;
    const float ref = top == -INFINITY ? 0.f : top;
    float sum = 0.f, x[E] = {};
    for (int k = 0; k < parts; ++k) {
        const float f = ex2(a.part_lse[slot(k)] - ref);
        const float* y = a.part + slot(k) * D + lane * E;
        sum += f;
        if (f == 0.f) continue;                                   // (a part in which the row sees nothing)
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] += f * y[e];
    }
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = sum == 0.f ? 0.f : x[e] * inv;
    const long long row = c.begin + r;
    const float lse = sum == 0.f ? -INFINITY : ref + lg2(sum);
    if (planes) {
        const long long at = row * a.p.q_heads + h;
        float* to = (c.prefix ? a.plane[1] : a.plane[0]) + at * D + lane * E;
#pragma unroll
        for (int e = 0; e < E; ++e) to[e] = x[e];
        if (lane == 0) (c.prefix ? a.plane_lse[1] : a.plane_lse[0])[at] = lse;
    } else {
        T* to = (T*)a.out + row * a.p.out_stride[0] + h * a.p.out_stride[1] + lane * E;
#pragma unroll
        for (int e = 0; e < E; e += 2) *(uint32_t*)(to + e) = Elem<T>::down(x[e], x[e + 1]);
        if (lane == 0 && a.lse) a.lse[row * a.p.q_heads + h] = lse * 0.69314718055994531f;
    }
}

template <class T, int D>
__global__ void __launch_bounds__(32 * JOIN_ROWS) join_cuts_kernel(const __grid_constant__ AttendArgs a, bool planes) {
    sd_chain_begin();
    const Cut c = a.cuts[blockIdx.x];
    if (c.last < c.first) return;
    const int lane = threadIdx.x & 31;
    for (int m = blockIdx.y * JOIN_ROWS + (threadIdx.x >> 5); m < c.rows; m += gridDim.y * JOIN_ROWS) join_row<T, D>(a, c, m, lane, planes);
}
// With a shared prefix: it and what is behind it, a warp per row and head.
template <class T, int D>
__global__ void __launch_bounds__(256) join_planes_kernel(const __grid_constant__ AttendArgs a) {
    sd_chain_begin();
    constexpr int E = D / 32;
    const sd_rows& b = a.b;
    const int lane = threadIdx.x & 31;
    const long long row = blockIdx.x;
    int i = 0;
    for (int base = 0; base < b.n; base += 256)
        i += __syncthreads_count(base + (int)threadIdx.x < b.n && b.d_offsets[base + threadIdx.x + 1] <= row);
    if (i >= b.n) return;
    const Request r = sd_request(b, i, a.c.page_size, a.p.shared);
    if (row < r.begin || row >= r.begin + r.count) return;
    for (int h = threadIdx.x >> 5; h < a.p.q_heads; h += 8) {
        const long long at = row * a.p.q_heads + h;
        const float l0 = a.plane_lse[0][at], l1 = a.plane_lse[1][at];
        float top = fmaxf(l0, l1);
        if (l0 != l0 || l1 != l1) top = NAN;
        const float ref = top == -INFINITY ? 0.f : top, f0 = ex2(l0 - ref), f1 = ex2(l1 - ref), sum = f0 + f1, inv = sum == 0.f ? 0.f : 1.0f / sum;
        float x[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            x[e] = 0.f;
            if (f0 != 0.f) x[e] += f0 * a.plane[0][at * D + lane * E + e];
            if (f1 != 0.f) x[e] += f1 * a.plane[1][at * D + lane * E + e];
            x[e] = sum == 0.f ? 0.f : x[e] * inv;
        }
        T* to = (T*)a.out + row * a.p.out_stride[0] + h * a.p.out_stride[1] + lane * E;
#pragma unroll
        for (int e = 0; e < E; e += 2) *(uint32_t*)(to + e) = Elem<T>::down(x[e], x[e + 1]);
        if (lane == 0 && a.lse) a.lse[row * a.p.q_heads + h] = sum == 0.f ? -INFINITY : (ref + lg2(sum)) * 0.69314718055994531f;
    }
}

// ---- host ----------------------------------------------------------------------------------
int check(const sd_cache* cache, const sd_rows* rows, const sd_attend_params* prm) {
    const int rc = sd_check_cache(cache, rows);
    if (rc != SD_OK) return rc;
    if (!prm || prm->q_heads < 1 || prm->q_heads > 65536 || prm->q_heads % cache->kv_heads) return SD_ERR_INVALID_ARG;
    if (prm->window < 0 || prm->sinks < 0 || prm->shared < 0 || !(prm->scale - prm->scale == 0.f)) return SD_ERR_INVALID_ARG;
    for (int k = 0; k < 2; ++k)
        if (!sd_stride_ok(prm->q_stride[k]) || !sd_stride_ok(prm->out_stride[k])) return SD_ERR_INVALID_ARG;
    if ((long long)rows->rows * (prm->q_heads / cache->kv_heads) > (1ll << 31) - 1024) return SD_ERR_INVALID_ARG;
    for (int k = 1; k < 4; ++k)                                   // (tiled copies count bytes in 40 bits)
        if (cache->k_stride[k] >= 1ll << 38 || cache->v_stride[k] >= 1ll << 38) return SD_ERR_INVALID_ARG;
    return SD_OK;
}

struct Room {
    int blocks;
    bool planes;
    int64_t cuts, part, part_lse, plane, plane_lse, all;          // bytes; begins of the parts
};

// Blocks and workspace of a call: as many blocks as multiprocessors, fewer where the longest lengths that the tables hold make less work than that.
int room_for(const sd_cache* c, const sd_rows* b, const sd_attend_params* p, Room* r) {
    int dev, sms;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return SD_ERR_CUDA;
    const long long G = p->q_heads / c->kv_heads, longest = ((long long)b->table_stride * c->page_size + TILE - 1) / TILE + 1;
    const long long units = (long long)c->kv_heads * (b->n + ((long long)b->rows * G + 255) / 256);   // (of both kinds: no more than that each)
    r->planes = p->shared >= TILE && !p->window;
    r->blocks = (int)std::max(1ll, std::min((long long)sms, (2 * units * longest + 3) / 4));
    int64_t at = 0;
    auto take = [&](int64_t bytes) { const int64_t was = at; at += (bytes + 255) / 256 * 256; return was; };
    r->cuts = take(r->blocks * (int64_t)sizeof(Cut));
    r->part = take(2ll * r->blocks * 256 * c->head_dim * 4);
    r->part_lse = take(2ll * r->blocks * 256 * 4);
    const int64_t lines = r->planes ? (int64_t)b->rows * p->q_heads : 0;
    r->plane = take(2 * lines * c->head_dim * 4);
    r->plane_lse = take(2 * lines * 4);
    r->all = at;
    return SD_OK;
}

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                 CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
    static const EncodeTiled f = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        return cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess ? (EncodeTiled)p : nullptr;
    }();
    return f;
}

// A page's lines of a head in pieces of 64 elements.
bool map_of(CUtensorMap* m, const sd_cache* c, void* base, const int64_t* stride, int box) {
    const EncodeTiled f = encode_tiled();
    if (!f) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)c->head_dim, (cuuint64_t)c->page_size, (cuuint64_t)c->kv_heads, (cuuint64_t)c->n_pages};
    cuuint64_t bytes[3];
    const int64_t from[3] = {stride[2], stride[3], stride[1]};
    for (int k = 0; k < 3; ++k) bytes[k] = dims[k + 1] > 1 ? (cuuint64_t)from[k] * 2 : (cuuint64_t)c->head_dim * 2;
    const cuuint32_t shape[4] = {64, (cuuint32_t)box, 1, 1}, step[4] = {1, 1, 1, 1};
    return f(m, c->dtype == SD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, base, dims, bytes, shape, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class T, int D>
int launch(const AttendArgs& a, const Room& r, int box, cudaStream_t st) {
    CUtensorMap mk, mv;
    if (!map_of(&mk, &a.c, a.c.d_k, a.c.k_stride, box) || !map_of(&mv, &a.c, a.c.d_v, a.c.v_stride, box)) return SD_ERR_CUDA;
    // (At every call: a cudaDeviceReset takes the limit away.)
    SD_CUDA_OK(cudaFuncSetAttribute(attend_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes<D>()));
    SD_CUDA_OK(sd_launch(attend_kernel<T, D>, r.blocks, THREADS, smem_bytes<D>(), st, a, mk, mv, box));
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(r.blocks, 4); cfg.blockDim = dim3(32 * JOIN_ROWS); cfg.stream = st;
    cfg.attrs = &attr; cfg.numAttrs = 1;
    SD_CUDA_OK(cudaLaunchKernelEx(&cfg, join_cuts_kernel<T, D>, a, r.planes));
    if (r.planes) SD_CUDA_OK(sd_launch(join_planes_kernel<T, D>, a.b.rows, 256, 0, st, a));
    return SD_OK;
}

}  // namespace

extern "C" int64_t sd_attend_workspace(const sd_cache* cache, const sd_rows* rows, const sd_attend_params* prm) {
    int rc = check(cache, rows, prm);
    Room r;
    if (rc == SD_OK) rc = room_for(cache, rows, prm, &r);
    return rc != SD_OK ? rc : r.all;
}

extern "C" int sd_attend(const sd_cache* cache, const sd_rows* rows, const sd_attend_params* prm, const void* d_q, void* d_out,
                         float* d_lse, void* d_workspace, int64_t workspace_bytes, void* stream) {
    int rc = check(cache, rows, prm);
    if (rc != SD_OK) return rc;
    if (rows->n == 0 || (rows->rows == 0 && !rows->d_status)) return SD_OK;
    if (!rows->d_offsets || (rows->rows > 0 && (!d_q || !d_out)) || !sd_aligned(d_q) || !sd_aligned(d_out)) return SD_ERR_INVALID_ARG;
    if (!d_workspace || (uintptr_t)d_workspace % 256) return SD_ERR_INVALID_ARG;
    Room r;
    rc = room_for(cache, rows, prm, &r);
    if (rc != SD_OK) return rc;
    if (workspace_bytes < r.all) return SD_ERR_CAPACITY;
    rc = sd_check_pointer(cache->d_k);
    if (rc != SD_OK) return rc;
    char* w = (char*)d_workspace;
    const int64_t lines = r.planes ? (int64_t)rows->rows * prm->q_heads : 0;
    const AttendArgs a = {*cache, *rows, *prm, d_q, d_out, d_lse, (Cut*)(w + r.cuts), (float*)(w + r.part), (float*)(w + r.part_lse),
                          {(float*)(w + r.plane), (float*)(w + r.plane) + lines * cache->head_dim}, {(float*)(w + r.plane_lse), (float*)(w + r.plane_lse) + lines}};
    const int box = std::min(cache->page_size, TILE);
    cudaStream_t st = (cudaStream_t)stream;
    if (cache->dtype == SD_BF16) return cache->head_dim == 128 ? launch<__nv_bfloat16, 128>(a, r, box, st) : launch<__nv_bfloat16, 64>(a, r, box, st);
    return cache->head_dim == 128 ? launch<__half, 128>(a, r, box, st) : launch<__half, 64>(a, r, box, st);
}
