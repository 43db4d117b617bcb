// sd_attend: attention of the rows of draft trees over their requests' paged caches.
//
// The work is a list of UNITS: some rows of one request with the query heads that share one head of the cache (row r, head g of the group: packed row
// r * group + g; as many whole rows as give up to 128 packed ones, or twice that) times the 128-line TILES of the cache that any of them sees; with a
// shared prefix also units of the whole batch's rows times the prefix's tiles.  The list is cut into as many equal pieces as there are blocks, in the middle of units where that
// falls so, so that every multiprocessor reads as much of the cache as any other, whatever the lengths; each block finds its piece from the lengths by itself.
// Rows of a unit that was cut are left as partial results (normalised, with the logarithm of their sum) and joined by a second kernel.
//
// A block is a warp that walks the list and copies queries and keys, one that copies values, both into a ring in shared memory, and two groups of four warps that
// compute the softmax, a thread per packed row, each with a warp that issues its products.  Two chains of (scores, softmax, product with the values)
// are in flight, one per group: for a unit of up to 128 rows the groups take tiles in turns and join their results at the end, for a larger one each has 128 rows of every tile.
// While one group is at its softmax the tensor cores work for the other.  Scores and results are in tensor memory; the weights go back over the scores
// and are read from there.
//
// The mathematics: out = sum_p exp(s_p - m) v_p / sum_p exp(s_p - m), s_p = scale * q k_p, in one pass over the places p.  m is a reference that follows the running maximum
// in steps (a row's sum and result are multiplied by 2^(old - new) only when the maximum has grown by 2^8, so that seldom anything is rescaled and no weight passes 2^8);
// parts with references of their own, of the two groups or of several blocks, are put together by the logarithms of their sums.  Scores, sums and results have 32 bits;
// weights are rounded to the type of the values, as the tensor cores want them, and a row's sum adds up the weights as they were before.
//
// What bounds it (bf16, 32 query heads on 8 heads of the cache of 128 elements where nothing else is said; microseconds of a call with its joins, and what the bytes or
// products that it cannot do without would take of that at the measured 6.55 TB/s or 1,625 TFLOP/s):
//   one token, 8,191 places               20     26 %: launches, code fetched for the first time, one chain copy - products - softmax - products, the join
//                                                (18.9 in a graph, so the host is not what bounds it)
//   16 requests, 32 .. 400 places         23     10 %: the same (fp16, 16 heads of 64, drafts of up to 32): 256 units on 148 multiprocessors, some 11 us of units' ends
//   a draft of 24, 131,072 places        135     61 %: copies in the middle, the same begin and end around it
//   64 requests, 1,000 .. 8,192 places   348     54 %: tiles of 256 rows take 3,800 cycles (products 2,050 of them; a group's chain of scores, maximum, weights, product
//                                                is longer than what the other group and the tensor cores need meanwhile), units' ends 12,000 cycles each
//   128 requests, window of 1,024     201 - 210  41 %: units' ends and the two tiles at the window's edges, which take five times as long as whole ones
//   256 requests, 4,096 places shared    405     26 % of the products: tiles as above, 32-bit planes of both parts and their join (18)
#include "blackwell.cuh"
#include "verify.cuh"

#include <algorithm>
#include <atomic>
#include <cmath>

namespace {

constexpr int TILE = 128;                                         // lines of the cache a step
constexpr int THREADS = 384;                                      // four warps that feed, eight that compute
constexpr int UNITS = 3;                                          // units that are known: the one at work and two more
constexpr int CHUNKS = 64;                                        // that the requests are added up in
// What the list's parts cost (measured: a tile of one group's rows 2,000 cycles where the cache's bandwidth is not what holds it up, of both 3,800 at most; a unit's
// begin and end 12,000).
constexpr int NARROW = 2, WIDE = 3, ENDS = 8;
constexpr int LEAST = 8;                                          // of a block's piece: a shorter one costs more to join than it saves
constexpr float BIAS_FP16 = 7.0f;                                 // fp16 weights are 2^7 as large: more of the small ones are above its least number
constexpr float RESCALE = 8.0f;                                   // results are rescaled when a row's maximum has grown by 2^8 (weights stay below that)

struct Cut {
    int first, last;              // blocks that have a part of it; none where last < first
    int rows, head, prefix;       // rows of the row arrays; head of the cache
    long long begin;
};

struct AttendArgs {
    sd_cache c;
    sd_rows b;
    sd_attend_params p;
    const void* q;
    void* out;
    float* lse;
    int group, tile_rows;         // query heads that share a head of the cache; rows whose heads make a tile's packed rows
    float scale;                  // of scores, for powers of two; not negative: the products turn the sign
    long long limit;              // cycles that a wait may take
    int box;                      // lines that one copy fetches
    int* gave_up;                 // [grid]: whether block c has given up a wait
    Cut* cuts;                    // [grid]: the unit that begins in block c and is cut
    float* part;                  // [2 * grid][256][D]: packed rows of a cut unit; slot 2c: it came from the block before, 2c + 1: it goes on in the next
    float* part_lse;              // [2 * grid][256]
    float* plane[2];              // with a shared prefix: [rows * q_heads][D], what is behind it and it
    float* plane_lse[2];          // [rows * q_heads]
};

enum { DONE = 0, TAIL = 1, PREFIX = 2 };
enum { FINAL = 0, PLANE = 1, SLOT = 2 };

struct Unit {
    long long begin;              // its first row in the row arrays
    int kind;
    int request, head;
    int row0, rows;               // of the request
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
        t.sinks = (min(p.sinks, r.cached) + TILE - 1) / TILE;
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
    // Barriers of the ring: for two rounds of it.  A wait tells a barrier's phase from the one before it and from no other.  With a barrier a slot, a group that leaves tiles
    // to the other one could take a slot that still waits for its last but one filling as filled (copies do not land in order), and the warp that copies values, slots that
    // have turns with the keys, one whose last but one reader is late as free.  What lies two rounds back, though, is always behind: keys are copied in order, those of a
    // tile when the readers of the ring's round before are through, and no group gets ahead of the other by more than that.
    static constexpr int BARS = 2 * SLOTS;
    static constexpr int Q_BYTES = 128 * D * 2;
    static constexpr int RING = 0, Q = SLOTS * SLOT_BYTES, REST = Q + 2 * Q_BYTES;
};

struct Rest {                     // of shared memory
    uint64_t full[16], empty[16], s_full[2], p_ready[2], o_done[2], q_full[2], q_empty[2], unit_full[UNITS], unit_empty[UNITS], meet, group_meet[2], over[2], lead;
    uint32_t tmem;
    Waits waits;
    int begun[2];                 // the group has begun its results itself: the first product adds to them
    uint32_t lines[2][4];         // lines of the group's tile with values that are no numbers
    int costs[CHUNKS], all, some; // of the list: chunks of requests, the whole; a request with rows (the prefix is read through its pages)
    int end;                      // of the requests' rows in the row arrays
    Unit units[UNITS];
    float2 sums[2][128];          // of the groups' rows: reference and sum
};
template <int D> constexpr int smem_bytes() { return Shape<D>::REST + (int)sizeof(Rest); }
static_assert(smem_bytes<128>() <= 232448 && smem_bytes<64>() <= 232448);

__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float rcp(float x) { float y; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }   // (of sums: some way from the least numbers)
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

// Row r of request u.request.
__device__ __noinline__ Sight sight_of(const sd_rows& b, int request, int cached, int count, int r, int W, int sinks) {
    Sight g = {0, 0, cached, true, 0ull};
    const unsigned long long bits = sd_tree_bits(b, request, r);
    g.tree = bits & (count >= 65 ? ~0ull : (1ull << (count - 1)) - 1);
    if (W) {
        const int at = cached + __popcll(bits);                   // the row's position
        g.from = max(0, at - W + 1);
        g.sinks = min(sinks, cached);
        if (W <= SD_MAX_SPEC) {                                   // rows of the tree may be outside the window
            g.root = at - cached < W || cached < sinks;
            for (unsigned long long left = g.tree; left; left &= left - 1) {
                const int j = __ffsll(left) - 1, p = cached + __popcll(sd_tree_bits(b, request, j + 1));
                if (at - p >= W && p >= sinks) g.tree &= ~(1ull << j);
            }
        }
    }
    return g;
}

template <class T> struct IsBf16 { static constexpr bool v = false; };
template <> struct IsBf16<__nv_bfloat16> { static constexpr bool v = true; };

// Each warp is through with its part: has any given up?  Then nobody asks for more now, and what was asked for comes to its end (of warps too that were through before).
__device__ __forceinline__ bool all_through(Rest* s) {
    __syncwarp();
    bw_fence_before();
    asm volatile("barrier.cta.sync 1, %0;" ::"n"(THREADS) : "memory");
    return s->waits.stop;
}

// Given up: the copies in flight come to their end: of queries, and those of lines that a warp has copied, up to slot `it`.
__device__ __noinline__ void drain(uint64_t* full, uint32_t slots, uint32_t filled) {
    for (uint32_t e = 0; e < slots && e < filled; ++e) {
        const uint32_t last = (filled - 1 - e) / slots * slots + e;
        bw_wait_end(bw_smem(&full[e]), (last / slots) & 1);
    }
}

template <int D>
__device__ __noinline__ void drain_lines(Rest* s, uint32_t it) {
    constexpr uint32_t BARS = Shape<D>::BARS;
    for (uint32_t k = it >= BARS ? it - BARS : it % 2; k < it; k += 2) bw_wait_end(bw_smem(&s->full[k % BARS]), (k / BARS) & 1);
}

// Pages that a request's rows see: told where one is none of the cache's.  (A shared prefix is read through the pages of one request: all rows see those.)
__device__ __noinline__ void write_status(const AttendArgs& a, const Rest* s, int lane) {
    const sd_rows& b = a.b;
    const int prefix_places = a.p.window ? 0 : a.p.shared / TILE * TILE;
    bool prefix = false;
    if (s->some < b.n) {
#pragma unroll 1
        for (int e = lane; e < (prefix_places + a.c.page_size - 1) / a.c.page_size; e += 32) prefix |= sd_page(b, a.c.n_pages, s->some, e) < 0;
    }
#pragma unroll 1
    for (int i = blockIdx.x; i < b.n; i += gridDim.x) {
        const Request r = sd_request(b, i, a.c.page_size, a.p.shared);
        int st = r.status;
        if (r.count) {
            const int P = a.c.page_size, from = a.p.window ? max(0, r.cached - a.p.window + 1) : 0;
            const int sinks = a.p.window ? min(min(a.p.sinks, r.cached), from) : 0;
            bool bad = prefix;
#pragma unroll 1
            for (int e = lane; e < (sinks + P - 1) / P; e += 32) bad |= sd_page(b, a.c.n_pages, i, e) < 0;
#pragma unroll 1
            for (int e = from / P + lane; e <= (r.cached + r.count - 1) / P; e += 32) bad |= sd_page(b, a.c.n_pages, i, e) < 0;
            if (__any_sync(~0u, bad)) st |= SD_STATUS_BAD_PAGE;
        }
        if (lane == 0) b.d_status[i] = st;
    }
}

// ---- copies --------------------------------------------------------------------------------
// A unit's keys (v = 0) or values (1): slots of the ring in turns.  (A warp for each: a copy takes 75 to 90 cycles to issue, and a tile of small pages is many.)
template <int D>
struct Lines {
    using S = Shape<D>;
    const AttendArgs& a;
    const CUtensorMap* map;
    Rest* s;
    const uint32_t ring, v;
    const int piece, half;                                        // of a tile and of a head, that this lane fetches
    uint32_t it;                                                  // the next slot
    // what is known of the tile to come
    bool here;
    int page, line;

    // Pages are looked up a tile ahead, and not looked at before they are needed.  Lines that no row sees are not fetched.
    __device__ __forceinline__ void look(const Unit& u, int k) {
        const int in_tile = piece * a.box, p = TILE * (k < u.sink_tiles ? k : u.next_tile + k - u.sink_tiles) + in_tile, entry = p / a.c.page_size;
        const int W = a.p.window, from = W && u.kind == TAIL ? max(0, u.cached - W + 1) : 0, length = u.kind == PREFIX ? u.cached : u.cached + u.count;
        here = k < u.k1 && in_tile < TILE && p < length && (p + a.box > from || (p < a.p.sinks && p < u.cached));
        page = 0;
        if (here) page = a.b.d_table[(long long)u.request * a.b.table_stride + entry];
        line = p - entry * a.c.page_size;
    }
    // Tile k of the unit, whose pages have been looked up, and a look at the next.  False: given up.
    __device__ __forceinline__ bool copy(const Unit& u, int k, bool wide) {
        const uint32_t e = it % S::SLOTS, bar = bw_smem(&s->full[it % S::BARS]), before = it - S::SLOTS;
        const int boxes = __popc(__ballot_sync(~0u, here));
        if (it >= S::SLOTS && !bw_wait_warp(bw_smem(&s->empty[before % S::BARS]), (before / S::BARS) & 1, &s->waits)) return false;
        if ((threadIdx.x & 31) == 0) {
            if (!wide) bw_arrive(bw_smem(&s->empty[it % S::BARS]));          // (for the group that does not use it)
            bw_arrive_expect(bar, boxes * a.box * 128);
        }
        if ((unsigned)page >= (unsigned)a.c.n_pages) page = a.c.n_pages;                  // (a page that is none: beyond the last, where a copy fills in zeros)
        const bool was = here;
        const int y = line, w = page;
        look(u, k + 1);
        __syncwarp();
        if (was) bw_load_4d(ring + e * S::SLOT_BYTES + half * S::HALF_BYTES + piece * a.box * 128, map, half * 64, y, u.head, w, bar);
        it += 2;
        return true;
    }
};

template <int D>
__device__ void copy_values(Lines<D> f) {
    for (int n = 0;; ++n) {
        if (!bw_wait_warp(bw_smem(&f.s->unit_full[n % UNITS]), (n / UNITS) & 1, &f.s->waits)) break;
        const Unit& u = f.s->units[n % UNITS];
        if (u.kind == DONE) break;
        const bool wide = u.rows > f.a.tile_rows;
        const int k1 = u.k1;
        bool ok = true;
        f.look(u, u.k0);
#pragma unroll 1
        for (int k = u.k0; k < k1 && ok; ++k) ok = f.copy(u, k, wide);
        if (!ok) break;
        bw_arrive_warp(bw_smem(&f.s->unit_empty[n % UNITS]));
    }
    if (f.a.b.d_status) write_status(f.a, f.s, threadIdx.x & 31);
    if (all_through(f.s)) drain_lines<D>(f.s, f.it);
}

// ---- the list's walker ---------------------------------------------------------------------
// What a request's units cost.  (31 bits are enough: the host has seen to that.)
struct Quote {
    long long begin;
    int count, cached;            // its rows, the places before them
    int sinks, next, tiles;       // of a unit
    int last;                     // cost of a head's last unit (which may have less rows than the others)
    int cost;                     // of all
};
__device__ __forceinline__ int unit_cost(bool wide, int tiles) { return ENDS + tiles * (wide ? WIDE : NARROW); }
__device__ __forceinline__ void price(Quote& e, int heads, int tile_rows) {
    const int before = (e.count - 1) / (2 * tile_rows);           // units of a head before the last
    e.last = unit_cost(e.count - before * 2 * tile_rows > tile_rows, e.tiles);
    e.cost = heads * (before * unit_cost(true, e.tiles) + e.last);
}
__device__ __noinline__ Quote quote_of(const AttendArgs& a, int prefix_tiles, int i) {
    const Request r = sd_request(a.b, i, a.c.page_size, a.p.shared);
    Quote e = {r.begin, r.count, r.cached, 0, 0, 0, 0, 0};
    if (r.count) {
        const Tiles t = tiles_of(a.p, prefix_tiles, r);
        e.sinks = t.sinks; e.next = t.next; e.tiles = t.count;
        price(e, a.c.kv_heads, a.tile_rows);
    }
    return e;
}

__device__ __forceinline__ int chunk_size(int n) { return (n + 32 * CHUNKS - 1) / (32 * CHUNKS) * 32; }

// By the whole block: what the requests cost, in chunks.
__device__ void add_up(const AttendArgs& a, Rest* s, int t) {
    const int prefix_tiles = a.p.window ? 0 : a.p.shared / TILE, size = chunk_size(a.b.n);
#pragma unroll 1
    for (int first = t & ~31; first < a.b.n; first += THREADS) {  // (a warp's requests are in one chunk)
        const int i = first + (t & 31);
        int cost = 0, has = 0x7FFFFFFF, end = 0;
        if (i < a.b.n) {
            const Quote e = quote_of(a, prefix_tiles, i);
            cost = e.cost;
            if (e.count) { has = i; end = (int)e.begin + e.count; }
        }
        __syncwarp();
        cost = __reduce_add_sync(~0u, cost);
        has = __reduce_min_sync(~0u, has);
        end = __reduce_max_sync(~0u, end);
        if ((t & 31) == 0 && cost) {
            atomicAdd(&s->costs[first / size], cost);
            atomicAdd(&s->all, cost);
            atomicMin(&s->some, has);
            atomicMax(&s->end, end);
        }
    }
}

// Hands out the units of the block's piece, and copies their queries and keys.
template <int D>
__device__ void walk_units(const AttendArgs& a, const CUtensorMap* mq, Rest* s, uint32_t q, Lines<D> keys, int lane) {
    using S = Shape<D>;
    const sd_rows& b = a.b;
    const int H = a.c.kv_heads, most = 2 * a.tile_rows;           // rows of a unit
    const int prefix_tiles = a.p.window ? 0 : a.p.shared / TILE, sum = s->all, some = s->some;
    // the prefix, as if it were a request before the others, with all rows up to the last of a request (not the last offset, which may make no sense)
    Quote prefix = {0, 0, a.p.shared, 0, 0, prefix_tiles, 0, 0};
    if (prefix_tiles && sum) {
        prefix.count = s->end;
        price(prefix, H, a.tile_rows);
    }
    const int all = sum + prefix.cost, quota = max((all + (int)gridDim.x - 1) / (int)gridDim.x, LEAST);
    const int lo = (int)min((long long)quota * blockIdx.x, (long long)all), hi = min(lo + quota, all);
    Cut cut;
    cut.first = 0; cut.last = -1;
    int at = 0, base = 0;                                         // units handed out; of the list, what is behind
    int start = prefix.cost ? -32 : 0;
    if (lo >= prefix.cost) {                                      // the chunk of requests that the piece begins in
        const int c0 = s->costs[2 * lane], c1 = s->costs[2 * lane + 1];
        int end = c0 + c1;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int x = __shfl_up_sync(~0u, end, d);
            if (lane >= d) end += x;
        }
        const int from = lo - prefix.cost, l = min(31, __popc(__ballot_sync(~0u, end <= from)));
        const int before = __shfl_sync(~0u, end - c0 - c1, l), c = __shfl_sync(~0u, c0, l), second = before + c <= from;
        start = (2 * l + second) * chunk_size(b.n);
        base = prefix.cost + before + (second ? c : 0);
    }
    uint32_t qi = 0;                                              // tiles of queries
    bool ok = true;
    // 32 requests at a time, then those of them that the piece touches, then their units
#pragma unroll 1
    for (int first = start; ok && first < b.n && base < hi; first += 32) {
        Quote e = {0, 0, 0, 0, 0, 0, 0, 0};
        if (first < 0) { if (lane == 0) e = prefix; }
        else if (first + lane < b.n) e = quote_of(a, prefix_tiles, first + lane);
        __syncwarp();
        int end = e.cost;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int x = __shfl_up_sync(~0u, end, d);
            if (lane >= d) end += x;
        }
        end += base;
        unsigned touched = __ballot_sync(~0u, e.cost > 0 && end > lo && end - e.cost < hi);
#pragma unroll 1
        while (ok && touched) {
            const int l = __ffs(touched) - 1;
            touched &= touched - 1;
            Unit u;
            u.kind = first < 0 ? PREFIX : TAIL;
            u.request = first < 0 ? some : first + l;
            u.cached = __shfl_sync(~0u, e.cached, l); u.count = __shfl_sync(~0u, e.count, l);
            u.sink_tiles = __shfl_sync(~0u, e.sinks, l); u.next_tile = __shfl_sync(~0u, first < 0 ? 0 : e.next, l);
            const int begin = __shfl_sync(~0u, end - e.cost, l), tiles = __shfl_sync(~0u, e.tiles, l), last = __shfl_sync(~0u, e.last, l);
            const int parts = (u.count + most - 1) / most, full = unit_cost(true, tiles), per_head = (parts - 1) * full + last;
            const long long rows_begin = __shfl_sync(~0u, e.begin, l);
            int off = max(0, lo - begin), head = off / per_head, part = min((off - head * per_head) / full, parts - 1);
            int from = begin + head * per_head + part * full;
#pragma unroll 1
            while (from < hi && head < H) {
                u.head = head; u.row0 = part * most; u.begin = rows_begin + u.row0;
                u.rows = min(most, u.count - u.row0);
                const bool wide = u.rows > a.tile_rows;
                // tile k begins at first + k * step of the list; the block that has this place has the tile
                const int first_place = from + ENDS, step = wide ? WIDE : NARROW;
                u.k0 = (max(lo - first_place, 0) + step - 1) / step;
                u.k1 = min((max(hi - first_place, 0) + step - 1) / step, tiles);
                from += part == parts - 1 ? last : full;
                if (++part == parts) { part = 0; ++head; }
                if (u.k1 <= u.k0) continue;
                const bool whole = u.k0 == 0 && u.k1 == tiles;
                u.to = !whole ? SLOT : prefix_tiles ? PLANE : FINAL;
                u.slot = whole ? first < 0 : 2 * blockIdx.x + (u.k0 == 0);
                if (!whole && u.k0 == 0) {
                    cut.first = blockIdx.x; cut.last = (first_place + (tiles - 1) * step) / quota;
                    cut.rows = u.rows; cut.head = u.head; cut.prefix = first < 0; cut.begin = u.begin;
                }
                const int place = at % UNITS;
                ok = at < UNITS || bw_wait_warp(bw_smem(&s->unit_empty[place]), (at / UNITS - 1) & 1, &s->waits);
                if (!ok) break;
                if (lane == 0) {
                    s->units[place] = u;
                    bw_arrive(bw_smem(&s->unit_full[place]));
                }
                ++at;
                keys.look(u, u.k0);
#pragma unroll 1
                for (int k = u.k0; k < u.k1 && ok; ++k) {
                    ok = keys.copy(u, k, wide);
                    if (k > u.k0) continue;
                    // its queries: a tile's rows and heads in one copy for each half of the head; rows behind the unit's come along and are left alone
#pragma unroll 1
                    for (int row = 0; row < u.rows; row += a.tile_rows) {
                        const uint32_t slot = qi % 2, bar = bw_smem(&s->q_full[slot]);
                        ok = qi < 2 || bw_wait_warp(bw_smem(&s->q_empty[slot]), (qi / 2 - 1) & 1, &s->waits);
                        if (!ok) break;
                        ++qi;                                     // (counted when it is asked for: drain() looks for the last of each slot)
                        if (lane) continue;
                        bw_arrive_expect(bar, S::HALVES * 128 * a.group * a.tile_rows);
#pragma unroll 1
                        for (int h = 0; h < S::HALVES; ++h) bw_load_3d(q + slot * S::Q_BYTES + h * S::HALF_BYTES, mq, h * 64, u.head * a.group, (int)u.begin + row, bar);
                    }
                }
                if (!ok) break;
            }
        }
        base = __shfl_sync(~0u, end, 31);
    }
    if (lane == 0) a.cuts[blockIdx.x] = cut;
    const int e = at % UNITS;
    if (ok && (at < UNITS || bw_wait_warp(bw_smem(&s->unit_empty[e]), (at / UNITS - 1) & 1, &s->waits)) && lane == 0) {
        s->units[e].kind = DONE;
        bw_arrive(bw_smem(&s->unit_full[e]));
    }
    if (all_through(s)) {
        drain(s->q_full, 2, qi);
        drain_lines<D>(s, keys.it);
    }
}

// ---- products ------------------------------------------------------------------------------
// (A warp for each group: to wait, to issue and to commit takes it as long as the products take.)  `leader`: the lane that issues.
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(~0u, x, 0); }   // (the same in all lanes, and known to be)

template <class T, int D>
__device__ void multiply(const AttendArgs& a, Rest* s, uint32_t ring, uint32_t q, uint32_t tmem_, int w, bool leader) {
    using S = Shape<D>;
    const uint32_t qk = bw_idesc(IsBf16<T>::v, 128, TILE, false, a.p.scale < 0.f);
    constexpr uint32_t pv = bw_idesc(IsBf16<T>::v, 128, D, true, false);
    const uint32_t tmem = uniform(tmem_), S0 = tmem + w * TILE, O0 = tmem + 2 * TILE + w * TILE;
    uint32_t it = 0, qi = 0, count = 0, wides = 0;                // slots, queries, jobs, wide units behind
    for (int n = 0;; ++n) {
        if (!bw_wait_warp(bw_smem(&s->unit_full[n % UNITS]), (n / UNITS) & 1, &s->waits)) return;
        const Unit& u = s->units[n % UNITS];
        const int kind = uniform(u.kind), tiles = uniform(u.k1 - u.k0);
        const bool wide = uniform(u.rows) > a.tile_rows;
        bw_arrive_warp(bw_smem(&s->unit_empty[n % UNITS]));
        if (kind == DONE) return;
        const int step = wide ? 1 : 2, first = wide ? 0 : w;      // the group's tiles
        const uint32_t mine = (qi + (wide ? w : 0)) % 2;          // its queries
        // Of a wide unit the second group begins when the first is halfway through its first tile: from then on the one computes while the other's products run.
        if (wide && w && !bw_wait_warp(bw_smem(&s->lead), wides++ & 1, &s->waits)) return;
        for (int k = 0; k < (wide ? 2 : 1); ++k) {
            const uint32_t e = (qi + k) % 2;
            if (!bw_wait_warp(bw_smem(&s->q_full[e]), ((qi + k) / 2) & 1, &s->waits)) return;
            if (e != mine || first >= tiles) bw_arrive_warp(bw_smem(&s->q_empty[e]));   // (not used by this group)
        }
#pragma unroll 1
        for (int j = first - step; j < tiles; j += step) {        // (scores are a tile ahead)
            const int next = j + step;
            const uint32_t v = it + 2 * j + 1, k = it + 2 * next;
            if (j >= 0) {
                if (!bw_wait_warp(bw_smem(&s->full[v % S::BARS]), (v / S::BARS) & 1, &s->waits)) return;
                if (!bw_wait_warp(bw_smem(&s->p_ready[w]), count++ & 1, &s->waits)) return;
                bw_fence_after();
                const bool add = j >= step || uniform(*(volatile int*)&s->begun[w]);
                const uint64_t vd = bw_desc_across(ring + v % S::SLOTS * S::SLOT_BYTES, S::HALF_BYTES);
#pragma unroll
                for (int i = 0; i < TILE / 16; ++i) bw_mma_ts(O0, S0 + i * 8, vd + (i * 2048 >> 4), pv, add || i > 0, leader);
            }
            if (next < tiles) {
                if (!bw_wait_warp(bw_smem(&s->full[k % S::BARS]), (k / S::BARS) & 1, &s->waits)) return;
                bw_fence_after();
                const uint64_t qd = bw_desc(q + mine * S::Q_BYTES), kd = bw_desc(ring + k % S::SLOTS * S::SLOT_BYTES);
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    const uint32_t off = (i / 4 * S::HALF_BYTES + i % 4 * 32) >> 4;
                    bw_mma(S0, qd + off, kd + off, qk, i > 0, leader);
                }
                bw_commit(bw_smem(&s->s_full[w]), leader);
                bw_commit(bw_smem(&s->empty[k % S::BARS]), leader);
                if (next + step >= tiles) bw_commit(bw_smem(&s->q_empty[mine]), leader);
            }
            if (j >= 0) {
                bw_commit(bw_smem(&s->empty[v % S::BARS]), leader);
                if (next >= tiles) bw_commit(bw_smem(&s->o_done[w]), leader);
            }
        }
        it += 2 * tiles;
        qi += wide ? 2 : 1;
    }
}

// ---- values that are no numbers ------------------------------------------------------------
// A weight of 0 does not take such a value out of a product.  So in a tile that not every row sees whole, lines that hold one are cleared, and what rows do see of
// them is added to the results line by line.

// Whether any of the two 16-bit numbers of a word is none (all bits of the exponent set).
template <class T> __device__ __forceinline__ uint32_t no_number(uint32_t x) {
    constexpr uint32_t E = IsBf16<T>::v ? 0x7F807F80u : 0x7C007C00u, ONE = IsBf16<T>::v ? 0x00800080u : 0x04000400u;
    return ((x & E) + ONE) & 0x80008000u;
}

// Lines of a warp's quarter of the tile.
template <class T, int D>
__device__ __forceinline__ uint32_t lines_without_numbers(const uint8_t* values, int t) {
    const uint8_t* mine = values + t * 128;
    uint32_t found = 0;
#pragma unroll 4
    for (int c = 0; c < D / 8; ++c) {
        const uint4 x = *(const uint4*)(mine + c / 8 * Shape<D>::HALF_BYTES + ((c % 8) ^ (t & 7)) * 16);
        found |= no_number<T>(x.x) | no_number<T>(x.y) | no_number<T>(x.z) | no_number<T>(x.w);
    }
    return __ballot_sync(~0u, found != 0);
}

// ---- softmax -------------------------------------------------------------------------------
__device__ __forceinline__ float max3(float a, float b, float c) { float r; asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }

// Two weights in the type of the values.  They are not negative, so that for bf16 half a step can be added to their bits (a tie goes up); the conversion
// instruction shares a pipe with the powers of two.
template <class T> __device__ __forceinline__ uint32_t weights(float2 p);
template <> __device__ __forceinline__ uint32_t weights<__nv_bfloat16>(float2 p) { return __byte_perm(__float_as_uint(p.x) + 0x8000u, __float_as_uint(p.y) + 0x8000u, 0x7632); }
template <> __device__ __forceinline__ uint32_t weights<__half>(float2 p) { return Elem<__half>::down(p.x, p.y); }

template <class T, int D>
struct Softmax {
    using S = Shape<D>;
    static constexpr float BIAS = IsBf16<T>::v ? 0.0f : BIAS_FP16;
    const AttendArgs& a;
    Rest* s;
    uint8_t* base;                                                // of shared memory
    uint32_t tmem;                                                // with the warp's lanes
    const int w, t;                                               // group, thread in it: packed row of its tile
    const int my_row, my_head;                                    // of the tile's rows, of the group's heads
    uint32_t meets = 0, group_meets = 0, s_count = 0, o_count0 = 0, o_count1 = 0, it = 0;

    __device__ __forceinline__ bool meet() { return meet_of(true); }
    __device__ __forceinline__ bool meet_of(bool both) {
        const uint32_t bar = bw_smem(both ? &s->meet : &s->group_meet[w]), parity = (both ? meets++ : group_meets++) & 1;
        bw_arrive_warp(bar);
        return bw_wait_warp(bar, parity, &s->waits);
    }
    __device__ bool run(int n);
    __device__ bool finish(const Unit& u, float top, float sum, bool row, bool busy, int r);
};

// The warp's results times alpha.  (Seldom: out of line.)
template <int D>
__device__ __noinline__ void scale_results(uint32_t O0, float alpha) {
    __syncwarp();
#pragma unroll 1
    for (int c = 0; c < D; c += 16) {
        uint32_t y[16];
        bw_ld16(O0 + c, y);
        bw_wait_ld16(y);
#pragma unroll
        for (int e = 0; e < 16; ++e) y[e] = __float_as_uint(__uint_as_float(y[e]) * alpha);
        bw_st16(O0 + c, y);
    }
    bw_wait_st();
}

// The largest of 32 scores and m.
__device__ __forceinline__ void most_of(const uint32_t* v, float* m) {
#pragma unroll
    for (int e = 0; e < 32; e += 8)
#pragma unroll
        for (int q = 0; q < 4; ++q) m[q] = max3(m[q], __uint_as_float(v[e + q]), __uint_as_float(v[e + 4 + q]));
}

// A tile that not every row sees whole: scores that a row does not see become -inf, in tensor memory, so that the rest is the same for all tiles.  Returns the largest.
// (Out of line, as all that follows for such tiles: in the loop over tiles its instructions and registers cost whole tiles a quarter of their time.)
__device__ __noinline__ float hide(const Sight& see, int place, uint32_t S0) {
    __syncwarp();
    float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    uint32_t x[32], y[32];
    auto hidden = [&](uint32_t* v, int c) {
        const uint32_t word = see.word(place + c);
        const bool whole = __all_sync(~0u, word == ~0u);
        __syncwarp();
        bw_wait_ld32(v);
        if (c + 32 < TILE) bw_ld32(S0 + c + 32, v == x ? y : x);
        if (!whole) {
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] = word >> e & 1 ? v[e] : 0xFF800000u;
            bw_st32(S0 + c, v);
        }
        most_of(v, m);
    };
    bw_ld32(S0, x);
#pragma unroll 1
    for (int c = 0; c < TILE; c += 64) {
        hidden(x, c);
        hidden(y, c + 32);
    }
    bw_wait_st();
    return fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
}

// Behind the weights of such a tile: if lines of its values hold no numbers, those that the warp's rows see are added to the results and all are cleared (see above).
struct Border {
    uint8_t* values;
    uint32_t S0, O0, v_full, v_parity, meets, group_meets;
    int w, t, place;
    bool busy, first, both;
};

// Their part in the results, which begin here if it is the first tile.
template <class T, int D>
__device__ __noinline__ void add_lines(const uint32_t* lines, const Sight& see, const Border& b) {
    __syncwarp();
    if (b.first)
#pragma unroll 1
        for (int c = 0; c < D; c += 8) {
            uint32_t x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = 0;
            bw_st8(b.O0 + c, x);
        }
    bw_wait_st();
#pragma unroll 1
    for (int l = 0; l < TILE; ++l) {
        if (!(lines[l / 32] >> l % 32 & 1)) continue;
        const bool seen = see.word(b.place + l) & 1;
        if (!__any_sync(~0u, seen)) continue;
        __syncwarp();
        const uint32_t two = bw_ld1(b.S0 + l / 2);
        const float2 weight = Elem<T>::up(two);
        const float p = l % 2 ? weight.y : weight.x;
#pragma unroll 1
        for (int d = 0; d < D; d += 8) {
            uint32_t x[8];
            bw_ld8(b.O0 + d, x);
            bw_wait_ld8(x);
            float v[8];
            sd_unpack<T>(*(const uint4*)(b.values + l * 128 + d / 64 * Shape<D>::HALF_BYTES + ((d % 64 / 8) ^ (l & 7)) * 16), v);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (seen) x[e] = __float_as_uint(__uint_as_float(x[e]) + p * v[e]);
            __syncwarp();
            bw_st8(b.O0 + d, x);
            bw_wait_st();
        }
    }
}

template <class T, int D>
__device__ __noinline__ bool clear_lines(Rest* s, const Sight& see, Border& b) {
    auto meet = [&](bool both) {
        const uint32_t bar = bw_smem(both ? &s->meet : &s->group_meet[b.w]), parity = (both ? b.meets++ : b.group_meets++) & 1;
        bw_arrive_warp(bar);
        return bw_wait_warp(bar, parity, &s->waits);
    };
    if (!bw_wait_warp(b.v_full, b.v_parity, &s->waits)) return false;
    const uint32_t of_warp = lines_without_numbers<T, D>(b.values, b.t);
    if ((b.t & 31) == 0) s->lines[b.w][b.t >> 5] = of_warp;
    if (!meet(b.both)) return false;
    uint32_t lines = 0;
#pragma unroll
    for (int c = 0; c < 4; ++c) lines |= s->lines[b.w][c];
    if (!lines) return true;
    if (b.busy) add_lines<T, D>(s->lines[b.w], see, b);
    if (b.first && b.t == 0) s->begun[b.w] = 1;
    if (!meet(b.both)) return false;
    if ((s->lines[b.w][b.t >> 5] >> (b.t & 31) & 1) && (b.w == 0 || !b.both)) {
#pragma unroll 1
        for (int c = 0; c < D / 8; ++c) *(uint4*)(b.values + b.t * 128 + c / 8 * Shape<D>::HALF_BYTES + c % 8 * 16) = make_uint4(0, 0, 0, 0);
        bw_fence_async();
    }
    __syncwarp();
    return b.both ? meet(true) : true;
}

template <class T, int D>
__device__ bool Softmax<T, D>::run(int n) {
    const Unit& u = s->units[n % UNITS];
    if (u.kind == DONE) return false;
    const bool wide = u.rows > a.tile_rows;
    const int tiles = u.k1 - u.k0, jobs = wide ? 2 * tiles : tiles;
    const int r = (wide ? w * a.tile_rows : 0) + my_row;          // of the unit's rows
    const bool row = my_row < a.tile_rows && r < u.rows;
    const bool busy = __any_sync(~0u, row);                       // any row of the warp
    // tiles that every row sees whole: up to plain_end, but of those not the ones from sinks_end to plain_from
    const int W = a.p.window;
    const int plain_end = u.kind == PREFIX ? 0x7FFFFFFF : u.cached / TILE, plain_from = W ? max(0, u.cached + SD_MAX_SPEC - W + TILE) / TILE : 0, sinks_end = W ? min(a.p.sinks, u.cached) / TILE : 0;
    const int k0 = u.k0, sink_tiles = u.sink_tiles, behind = u.next_tile - sink_tiles;
    Sight see = {0, 0, u.cached, false, 0ull};
    if (row && u.kind == TAIL) see = sight_of(a.b, u.request, u.cached, u.count, u.row0 + r, W, a.p.sinks);
    if (!meet()) return false;                                    // both groups are through with the results of the unit before
    if (t == 0) s->begun[w] = 0;
    const uint32_t S0 = tmem + w * TILE, O0 = tmem + 2 * TILE + w * TILE;
    const float scale = a.scale;
    float top = -INFINITY, sum = 0.f;                             // the row's reference for powers, and its sum

#pragma unroll 1
    for (int j = w; j < jobs; j += 2) {
        const int k = k0 + (wide ? j >> 1 : j), number = k < sink_tiles ? k : k + behind;
        const bool masked = number >= plain_end || (number < plain_from && number >= sinks_end);
        if (wide && j == 0 && (masked || !busy)) bw_arrive_warp(bw_smem(&s->lead));     // (a border takes both groups)
        if (!bw_wait_warp(bw_smem(&s->s_full[w]), s_count++ & 1, &s->waits)) return false;
        bw_fence_after();
        if (busy) {
            // 32 scores at a time, the next ones on their way; twice from tensor memory, for the maximum and for the weights (all in registers at once: spills, and
            // twice the instructions, which then do not stay in the instruction cache)
            uint32_t x[32], y[32];
            float mx;
            if (masked) {
                mx = hide(see, number * TILE, S0);
                bw_ld32(S0, x);
            } else {
                float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                bw_ld32(S0, x);
#pragma unroll 1
                for (int c = 0; c < TILE; c += 64) {
                    bw_wait_ld32(x);
                    bw_ld32(S0 + c + 32, y);
                    most_of(x, m);
                    bw_wait_ld32(y);
                    bw_ld32(S0 + (c + 64) % TILE, x);             // (at the end: the first ones again)
                    most_of(y, m);
                }
                mx = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
            }
            const bool up = row && mx != -INFINITY && !((mx - top) * scale <= RESCALE);
            if (__any_sync(~0u, up)) {
                const float alpha = up ? ex2((top - mx) * scale) : 1.f;
                if (up) top = mx;
                sum *= alpha;
                if (j >= 2) {
                    bw_wait_ld32(x);
                    scale_results<D>(O0, alpha);
                    bw_ld32(S0, x);
                }
            }
            if (wide && j == 0 && !masked) bw_arrive_warp(bw_smem(&s->lead));
            const float power = (top == -INFINITY ? 0.f : top * scale) - BIAS;
            __syncwarp();
            const float2 by = make_float2(scale, scale), less = make_float2(-power, -power);
            float2 part[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
            auto weigh = [&](uint32_t* v) {
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                    const float2 z = sd_fma2(make_float2(__uint_as_float(v[e]), __uint_as_float(v[e + 1])), by, less);
                    const float2 p = make_float2(ex2(z.x), ex2(z.y));
                    part[e / 2 % 2] = sd_add2(part[e / 2 % 2], p);
                    v[e / 2] = weights<T>(p);
                }
            };
#pragma unroll 1
            for (int c = 0; c < TILE; c += 64) {                  // (weights are half as wide: they come to lie over scores that have been read)
                bw_wait_ld32(x);
                bw_ld32(S0 + c + 32, y);
                weigh(x);
                bw_st16(S0 + c / 2, x);
                bw_wait_ld32(y);
                if (c == 0) bw_ld32(S0 + 64, x);
                weigh(y);
                bw_st16(S0 + c / 2 + 16, y);
            }
            sum += (part[0].x + part[0].y) + (part[1].x + part[1].y);
        }
        __syncwarp();
        if (masked) {
            bw_wait_st();
            const uint32_t vs = it + 2 * (wide ? j >> 1 : j) + 1;
            Border b = {base + S::RING + vs % S::SLOTS * S::SLOT_BYTES, S0, O0, bw_smem(&s->full[vs % S::BARS]), (vs / S::BARS) & 1, meets, group_meets, w, t, number * TILE, busy, j < 2, wide};
            if (!clear_lines<T, D>(s, see, b)) return false;
            meets = b.meets; group_meets = b.group_meets;
        }
        bw_wait_st();
        bw_fence_before();
        bw_arrive_warp(bw_smem(&s->p_ready[w]));
    }
    if (!finish(u, top, sum, row, busy, r)) return false;
    it += 2 * tiles;
    bw_arrive_warp(bw_smem(&s->unit_empty[n % UNITS]));
    return true;
}

// A unit's results: O[A] * g0, with the other group's part O[A + TILE] * g1 where both have one.
template <class T, int D>
__device__ __forceinline__ bool Softmax<T, D>::finish(const Unit& u, float top, float sum, bool row, bool busy, int r) {
    const bool wide = u.rows > a.tile_rows, two = !wide && u.k1 - u.k0 > 1;
    const float scale = a.scale;
    float g0 = 1.f, g1 = 0.f, m = top, l = sum;
    int c0 = 0, c1 = D;
    uint32_t A = tmem + 2 * TILE + w * TILE;
    if (!wide) {
        s->sums[w][t] = make_float2(top, sum);
        if (!meet()) return false;
    }
    if (!wide || w == 0) { if (!bw_wait_warp(bw_smem(&s->o_done[0]), o_count0 & 1, &s->waits)) return false; }
    if (two || (wide && w == 1)) { if (!bw_wait_warp(bw_smem(&s->o_done[1]), o_count1 & 1, &s->waits)) return false; }
    ++o_count0;
    o_count1 += wide || two;
    bw_fence_after();
    if (!busy) return true;
    if (!wide) {
        const float2 x0 = s->sums[0][t], x1 = s->sums[1][t];
        m = two ? fmaxf(x0.x, x1.x) : x0.x;
        const float ref = m == -INFINITY ? 0.f : m;
        g0 = ex2((x0.x - ref) * scale);
        g1 = two ? ex2((x1.x - ref) * scale) : 0.f;
        l = x0.y * g0 + (two ? x1.y * g1 : 0.f);
        A = tmem + 2 * TILE;
        c0 = w * (D / 2); c1 = c0 + D / 2;
    }
    const float inv = l == 0.f ? 0.f : rcp(l);
    g0 *= inv;
    g1 *= inv;
    const int h = u.head * a.group + my_head, to = u.to, mrow = (wide ? w * 128 : 0) + t;
    const long long at = (u.begin + r) * a.p.q_heads + h;         // row and query head
    T* out = (T*)a.out + (u.begin + r) * a.p.out_stride[0] + h * a.p.out_stride[1];
    float* part = to == SLOT ? a.part + ((long long)u.slot * 256 + mrow) * D : a.plane[u.slot & 1] + at * D;
    uint32_t x[16], z[16];
    __syncwarp();
    bw_ld16(A + c0, x);
    if (two) bw_ld16(A + TILE + c0, z);
#pragma unroll 1
    for (int c = c0; c < c1; c += 16) {
        bw_wait_ld16(x);
        if (two) bw_wait_ld16(z);
        float y[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {                            // (a part without a weight may hold anything)
            y[e] = g0 == 0.f ? 0.f : __uint_as_float(x[e]) * g0;
            if (g1 != 0.f) y[e] += __uint_as_float(z[e]) * g1;
        }
        __syncwarp();
        if (c + 16 < c1) {                                        // (the next ones come while these are written)
            bw_ld16(A + c + 16, x);
            if (two) bw_ld16(A + TILE + c + 16, z);
        }
        if (row) {
            if (to == FINAL) {
                *(uint4*)(out + c) = sd_pack<T>(y);
                *(uint4*)(out + c + 8) = sd_pack<T>(y + 8);
            } else {
#pragma unroll
                for (int e = 0; e < 16; e += 4) *(float4*)(part + c + e) = make_float4(y[e], y[e + 1], y[e + 2], y[e + 3]);
            }
        }
        __syncwarp();
    }
    if (row && (wide || w == 0)) {
        const float lse = l == 0.f ? -INFINITY : m * scale + lg2(l) - BIAS;
        if (to != FINAL) *(to == SLOT ? a.part_lse + (long long)u.slot * 256 + mrow : a.plane_lse[u.slot & 1] + at) = lse;
        else if (a.lse) a.lse[at] = lse * 0.69314718055994531f;
    }
    __syncwarp();
    bw_fence_before();
    return true;
}

template <class T, int D>
__global__ void __launch_bounds__(THREADS, 1) attend_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                                                            const __grid_constant__ CUtensorMap mq) {
    using S = Shape<D>;
    extern __shared__ __align__(1024) uint8_t smem[];
    Rest* s = (Rest*)(smem + S::REST);
    const int t = threadIdx.x, warp = uniform(t >> 5), lane = t & 31;
    if (t == 0) {
        for (int e = 0; e < S::BARS; ++e) { bw_bar_init(bw_smem(&s->full[e]), 1); bw_bar_init(bw_smem(&s->empty[e]), 2); }
        for (int e = 0; e < 2; ++e) {
            bw_bar_init(bw_smem(&s->s_full[e]), 1); bw_bar_init(bw_smem(&s->p_ready[e]), 4); bw_bar_init(bw_smem(&s->o_done[e]), 1);
            bw_bar_init(bw_smem(&s->q_full[e]), 1); bw_bar_init(bw_smem(&s->q_empty[e]), 2); bw_bar_init(bw_smem(&s->group_meet[e]), 4);
            bw_bar_init(bw_smem(&s->over[e]), 1);
        }
        for (int e = 0; e < UNITS; ++e) { bw_bar_init(bw_smem(&s->unit_full[e]), 1); bw_bar_init(bw_smem(&s->unit_empty[e]), 11); }
        bw_bar_init(bw_smem(&s->meet), 8);
        bw_bar_init(bw_smem(&s->lead), 4);
        s->waits.stop = 0; s->waits.limit = a.limit; s->begun[0] = s->begun[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (t < CHUNKS) s->costs[t] = 0;
    if (t == CHUNKS) { s->all = 0; s->some = 0x7FFFFFFF; s->end = 0; }
    if (t == 32 * 3) { bw_prefetch_map(&mk); bw_prefetch_map(&mv); bw_prefetch_map(&mq); }
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (warp == 1) bw_tmem_alloc(bw_smem(&s->tmem), 512);         // (not before the wait: a kernel there, of another library, may still ask for some, and would wait for this one)
    add_up(a, s, t);
    bw_fence_before();
    __syncthreads();
    bw_fence_after();
    const uint32_t tmem = s->tmem, ring = bw_smem(smem + S::RING), q = bw_smem(smem + S::Q);
    if (warp == 0 || warp == 2) {
        Lines<D> f = {a, warp ? &mv : &mk, s, ring, (uint32_t)warp >> 1, lane / S::HALVES, lane % S::HALVES, (uint32_t)warp >> 1};
        if (warp == 0) walk_units<D>(a, &mq, s, q, f, lane);
        else copy_values<D>(f);
    } else if (warp == 1 || warp == 3) {
        const bool leader = bw_elect();
        multiply<T, D>(a, s, ring, q, tmem, warp >> 1, leader);
        if (all_through(s)) {
            bw_commit(bw_smem(&s->over[warp >> 1]), leader);
            bw_wait_end(bw_smem(&s->over[warp >> 1]), 0);
        }
    } else {
        const int row = (t - 128) & 127;
        Softmax<T, D> f = {a, s, smem, tmem + ((uint32_t)(warp & 3) << 21), (warp - 4) >> 2, row, row / a.group, row % a.group};
        for (int n = 0;; ++n) {
            if (!bw_wait_warp(bw_smem(&s->unit_full[n % UNITS]), (n / UNITS) & 1, &s->waits)) break;
            if (!f.run(n)) break;
        }
        all_through(s);
    }
    __syncwarp();
    if (s->waits.stop) __syncthreads();                           // (what was asked for has come to its end)
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // (from the begin on, the next kernel's waiting blocks cost small calls a quarter)
    if (warp == 1) {
        bw_fence_after();
        bw_tmem_free(tmem, 512);
    }
    if (t == 0) a.gave_up[blockIdx.x] = s->waits.stop;
}

// ---- joining -------------------------------------------------------------------------------
// A warp per packed row of a cut unit: its parts by their sums.  Rows of few calls are many, so that what a row takes is the latency of its loads: the cut, then its
// sums and eight parts at once (one token over a long context 23.5 -> 19.5 us against a kernel that first looked up where a row belongs and loaded parts behind the sums; 20 since it asks
// first whether a block has given up).
constexpr int JOIN_ROWS = 8, JOIN_BLOCKS = 16, AHEAD = 8, MOST_BLOCKS = 1024;

// By a whole block: has any of attend_kernel's given up?  (Told here, behind all of them, so that no block's status comes after it.)
__device__ __forceinline__ bool any_gave_up(const AttendArgs& a, int blocks) {
    bool any = false;
    for (int e = threadIdx.x; e < blocks; e += blockDim.x) any |= a.gave_up[e] != 0;
    return __syncthreads_or(any);
}

// Then all requests are told, and their rows say so too: a call need not ask for statuses.
template <int D>
__device__ __noinline__ void tell_given_up(const AttendArgs& a) {
    const sd_rows& b = a.b;
    constexpr int PER = D / 8;                                    // pieces of 16 bytes of a head
    for (int i = blockIdx.x; i < b.n; i += gridDim.x) {
        if (b.d_status && threadIdx.x == 0) b.d_status[i] |= SD_STATUS_FAILED;
        const Request r = sd_request(b, i, a.c.page_size, a.p.shared);
        for (int e = threadIdx.x; e < r.count * a.p.q_heads; e += blockDim.x) {
            const long long row = r.begin + e / a.p.q_heads;
            const int h = e % a.p.q_heads;
            uint4* to = (uint4*)((uint16_t*)a.out + row * a.p.out_stride[0] + h * a.p.out_stride[1]);
            for (int c = 0; c < PER; ++c) to[c] = make_uint4(0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu);   // (no number in either type)
            if (a.lse) a.lse[row * a.p.q_heads + h] = NAN;
        }
    }
}

template <class T, int D>
__device__ void join_row(const AttendArgs& a, const Cut& c, int m, int lane, bool planes) {
    constexpr int E = D / 32;
    const int r = m / a.group, h = c.head * a.group + m - r * a.group;
    const int mrow = r < a.tile_rows ? m : 128 + m - a.tile_rows * a.group;             // (the second tile's rows begin at 128)
    auto slot = [&](int k) { return (long long)(2 * (c.first + k) + (k == 0)) * 256 + mrow; };
    const int parts = c.last - c.first + 1;
    float top = -INFINITY, sum = 0.f, x[E] = {};                  // running, 32 parts at a time
#pragma unroll 1
    for (int first = 0; first < parts; first += 32) {
        const int n = min(32, parts - first);
        const float v = lane < n ? a.part_lse[slot(first + lane)] : -INFINITY;
        float z[AHEAD][E];
        auto fetch = [&](int k0) {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (k0 + k < n) {
                    const float* y = a.part + slot(first + k0 + k) * D + lane * E;
                    if constexpr (E == 4) { const float4 x = *(const float4*)y; z[k][0] = x.x; z[k][1] = x.y; z[k][2] = x.z; z[k][3] = x.w; }
                    else { const float2 x = *(const float2*)y; z[k][0] = x.x; z[k][1] = x.y; }
                }
        };
        fetch(0);                                                 // (on their way together with the sums)
        float most = v;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor_sync(~0u, most, d));
        most = fmaxf(most, top);
        const float ref = most == -INFINITY ? 0.f : most, keep = ex2(top - ref), f = ex2(v - ref);
        float total = f;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) total += __shfl_xor_sync(~0u, total, d);
        sum = sum * keep + total;
        top = most;
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] *= keep;
#pragma unroll 1
        for (int k0 = 0;;) {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const float g = __shfl_sync(~0u, f, (k0 + k) & 31);
                if (k0 + k < n && g != 0.f)                       // (0: a part in which the row sees nothing)
#pragma unroll
                    for (int e = 0; e < E; ++e) x[e] += g * z[k][e];
            }
            k0 += AHEAD;
            if (k0 >= n) break;
            fetch(k0);
        }
    }
    const float inv = sum == 0.f ? 0.f : rcp(sum);
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = sum == 0.f ? 0.f : x[e] * inv;
    const long long row = c.begin + r;
    const float lse = sum == 0.f ? -INFINITY : top + lg2(sum);
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

// JOIN_BLOCKS blocks for each place that a cut may have: most find none.  (With 8 a long context whose rows are cut 18 times takes 3 us longer, with 32 small calls 1 us.)
template <class T, int D>
__global__ void __launch_bounds__(32 * JOIN_ROWS) join_cuts_kernel(const __grid_constant__ AttendArgs a, bool planes, int blocks) {
    sd_chain_begin();
    const Cut c = a.cuts[blockIdx.x % blocks];
    if (any_gave_up(a, blocks)) { tell_given_up<D>(a); return; }
    if (c.last < c.first) return;
#pragma unroll 1
    for (int m = blockIdx.x / blocks * JOIN_ROWS + (threadIdx.x >> 5); m < c.rows * a.group; m += gridDim.x / blocks * JOIN_ROWS) join_row<T, D>(a, c, m, threadIdx.x & 31, planes);
}

// With a shared prefix: it and what is behind it, a warp per row and head.
template <class T, int D>
__global__ void __launch_bounds__(256) join_planes_kernel(const __grid_constant__ AttendArgs a, int blocks) {
    sd_chain_begin();
    if (any_gave_up(a, blocks)) return;                           // (told already)
    constexpr int E = D / 32;
    const sd_rows& b = a.b;
    const int lane = threadIdx.x & 31;
    const long long row = blockIdx.x;
    int i = 0;
    for (int base = 0; base < b.n; base += 256)
        i += __syncthreads_count(base + (int)threadIdx.x < b.n && b.d_offsets[base + threadIdx.x + 1] <= row);
    auto holds = [&](int request) {
        if (request >= b.n) return false;
        const Request r = sd_request(b, request, a.c.page_size, a.p.shared);
        return row >= r.begin && row < r.begin + r.count;
    };
    if (!holds(i)) {                                              // a row of no request, or behind offsets that make no sense: among all
        bool found = false;
        for (int at = threadIdx.x; at < b.n; at += 256) found |= holds(at);
        if (!__syncthreads_or(found)) return;
    }
    for (int h = threadIdx.x >> 5; h < a.p.q_heads; h += 8) {
        const long long at = row * a.p.q_heads + h;
        const float l0 = a.plane_lse[0][at], l1 = a.plane_lse[1][at];
        float top = fmaxf(l0, l1);
        if (l0 != l0 || l1 != l1) top = NAN;
        const float ref = top == -INFINITY ? 0.f : top, f0 = ex2(l0 - ref), f1 = ex2(l1 - ref), sum = f0 + f1, inv = sum == 0.f ? 0.f : rcp(sum);
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
constexpr long long WAIT_LIMIT = 4000000000;                      // two seconds
std::atomic<long long> g_limit{0};                                // of sd_debug_attend_limit

int check(const sd_cache* cache, const sd_rows* rows, const sd_attend_params* prm) {
    const int rc = sd_check_cache(cache, rows);
    if (rc != SD_OK) return rc;
    if (!prm || prm->q_heads < 1 || prm->q_heads > 65536 || prm->q_heads % cache->kv_heads) return SD_ERR_INVALID_ARG;
    if (prm->window < 0 || prm->sinks < 0 || prm->shared < 0 || !(prm->scale - prm->scale == 0.f)) return SD_ERR_INVALID_ARG;
    for (int k = 0; k < 2; ++k)
        if (!sd_stride_ok(prm->q_stride[k]) || !sd_stride_ok(prm->out_stride[k])) return SD_ERR_INVALID_ARG;
    if (prm->q_heads / cache->kv_heads > 128) return SD_ERR_INVALID_ARG;
    if (rows->rows > 1 && prm->q_stride[0] <= 0 || prm->q_heads > 1 && prm->q_stride[1] <= 0) return SD_ERR_INVALID_ARG;
    if (!sd_out_strides_ok(prm->out_stride, rows->rows, prm->q_heads)) return SD_ERR_INVALID_ARG;
    if (prm->q_stride[0] >= 1ll << 38 || prm->q_stride[1] >= 1ll << 38) return SD_ERR_INVALID_ARG;
    for (int k = 1; k < 4; ++k)                                   // (tiled copies count bytes in 40 bits)
        if (cache->k_stride[k] >= 1ll << 38 || cache->v_stride[k] >= 1ll << 38) return SD_ERR_INVALID_ARG;
    return SD_OK;
}

struct Room {
    int blocks;
    bool planes;
    int64_t gave_up, cuts, part, part_lse, plane, plane_lse, all;          // bytes; begins of the parts
};

// Blocks and workspace of a call: as many blocks as multiprocessors, fewer where the longest lengths that the tables hold make less work than that.
int room_for(const sd_cache* c, const sd_rows* b, const sd_attend_params* p, Room* r) {
    int dev, sms;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return SD_ERR_CUDA;
    // all of the list, at the longest lengths that the tables hold
    const long long longest = ((long long)b->table_stride * c->page_size + TILE - 1) / TILE + 1, most = 2 * (128 / (p->q_heads / c->kv_heads));
    // (as many rows as each request can have: offsets that descend may give rows to more than one)
    const long long units = c->kv_heads * ((long long)b->n * ((b->max_draft + most) / most) + (b->rows + most - 1) / most);
    if (units > (1ll << 30) / (longest * WIDE + ENDS)) return SD_ERR_CAPACITY;
    r->planes = p->shared >= TILE && !p->window;
    r->blocks = (int)std::max(1ll, std::min((long long)std::min(sms, MOST_BLOCKS), (units * (longest * WIDE + ENDS) + LEAST - 1) / LEAST));
    int64_t at = 0;
    auto take = [&](int64_t bytes) { const int64_t was = at; at += (bytes + 255) / 256 * 256; return was; };
    r->gave_up = take(r->blocks * (int64_t)sizeof(int));
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

// Rows and the query heads of a head of the cache.
bool map_of_queries(CUtensorMap* m, const AttendArgs& a) {
    const EncodeTiled f = encode_tiled();
    if (!f) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)a.c.head_dim, (cuuint64_t)a.p.q_heads, (cuuint64_t)std::max(a.b.rows, 1)};
    const cuuint64_t bytes[2] = {(cuuint64_t)(a.p.q_heads > 1 ? a.p.q_stride[1] : a.c.head_dim) * 2, (cuuint64_t)(a.b.rows > 1 ? a.p.q_stride[0] : (int64_t)a.p.q_heads * a.c.head_dim) * 2};
    const cuuint32_t shape[3] = {64, (cuuint32_t)a.group, (cuuint32_t)a.tile_rows}, step[3] = {1, 1, 1};
    return f(m, a.c.dtype == SD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(a.b.rows ? a.q : a.c.d_k), dims, bytes, shape, step,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class T, int D>
int launch(const AttendArgs& a, const Room& r, cudaStream_t st) {
    CUtensorMap mk, mv, mq;
    if (!map_of(&mk, &a.c, a.c.d_k, a.c.k_stride, a.box) || !map_of(&mv, &a.c, a.c.d_v, a.c.v_stride, a.box) || !map_of_queries(&mq, a)) return SD_ERR_CUDA;
    // (At every call: a cudaDeviceReset takes the limit away.)
    SD_CUDA_OK(cudaFuncSetAttribute(attend_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes<D>()));
    SD_CUDA_OK(sd_launch(attend_kernel<T, D>, r.blocks, THREADS, smem_bytes<D>(), st, a, mk, mv, mq));
    if (a.b.rows == 0) return SD_OK;
    const long long rows = std::min((long long)a.b.rows, 2ll * a.tile_rows) * a.group;  // packed ones of a cut
    SD_CUDA_OK(sd_launch(join_cuts_kernel<T, D>, r.blocks * (unsigned)std::min((rows + JOIN_ROWS - 1) / JOIN_ROWS, (long long)JOIN_BLOCKS), 32 * JOIN_ROWS, 0, st, a, r.planes, r.blocks));
    if (r.planes) SD_CUDA_OK(sd_launch(join_planes_kernel<T, D>, a.b.rows, 256, 0, st, a, r.blocks));
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
    AttendArgs a = {*cache, *rows, *prm, d_q, d_out, d_lse};
    a.group = prm->q_heads / cache->kv_heads;
    a.tile_rows = 128 / a.group;
    // (A factor of 0: the least number keeps scores that are not seen, -inf, what they are.)
    a.scale = std::max(std::abs(prm->scale) * 1.4426950408889634f, 1.17549435e-38f);
    a.box = std::min(cache->page_size, TILE);
    a.limit = g_limit > 0 ? g_limit.load() : WAIT_LIMIT;
    a.gave_up = (int*)(w + r.gave_up); a.cuts = (Cut*)(w + r.cuts); a.part = (float*)(w + r.part); a.part_lse = (float*)(w + r.part_lse);
    a.plane[0] = (float*)(w + r.plane); a.plane[1] = a.plane[0] + lines * cache->head_dim;
    a.plane_lse[0] = (float*)(w + r.plane_lse); a.plane_lse[1] = a.plane_lse[0] + lines;
    cudaStream_t st = (cudaStream_t)stream;
    if (cache->dtype == SD_BF16) return cache->head_dim == 128 ? launch<__nv_bfloat16, 128>(a, r, st) : launch<__nv_bfloat16, 64>(a, r, st);
    return cache->head_dim == 128 ? launch<__half, 128>(a, r, st) : launch<__half, 64>(a, r, st);
}

extern "C" void sd_debug_attend_limit(int64_t cycles) { g_limit = cycles; }
