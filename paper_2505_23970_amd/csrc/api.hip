// Host side of the C ABI declared in include/greencache.h: argument checks,
// work-split policy, workspace layout and kernel launches. Every check runs
// before the first HIP call, so invalid calls enqueue nothing.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <mutex>

#include "gc_internal.h"
#include "greencache.h"

namespace {

struct Shape {
    int64_t total_tokens = 0;
    int group = 1;
    bool small = false;          // small-tile (decode) path
    bool wide = false;           // 8-wavefront prefill tiles
    int block_m = gc::kBlockM;   // query rows per tile
    int block_n = gc::kBlockN;   // keys per tile
    int tq = 1;                  // new tokens per query tile
};

struct Plan {
    int chunk = 0;  // key tiles per chunk, 0 = no split
    int64_t items = 0, combines = 0, partials = 0;
    int max_splits = 1;  // key chunks of the query tile with the most
    bool heaviest_decides = false;  // the heaviest work item ends the launch (see heaviest_decides)
    bool three = false;             // a third 128-row workgroup per compute unit pays (8-bit pools, d = 64)
    int group_cost = gc::kCostBuckets;  // work-list order (gc::PlanArgs)
    int buckets = gc::kCostBuckets;
    gc::WorkspaceLayout layout{};
};

gc_status check_common(const gc_geometry* geo, const gc_batch* b, Shape* sh) {
    if (geo == nullptr || b == nullptr) return GC_ERR_NULL_ARG;
    if (b->batch < 0) return GC_ERR_BAD_SHAPE;
    if (geo->num_q_heads <= 0 || geo->num_kv_heads <= 0 || geo->head_dim <= 0 ||
        geo->page_size <= 0 || geo->num_blocks < 0 || geo->max_blocks_per_seq < 0)
        return GC_ERR_BAD_SHAPE;
    if (geo->num_q_heads % geo->num_kv_heads != 0) return GC_ERR_BAD_SHAPE;
    const int group = geo->num_q_heads / geo->num_kv_heads;
    if (group > gc::kBlockM) return GC_ERR_UNSUPPORTED;
    if (geo->num_kv_heads > 65535) return GC_ERR_UNSUPPORTED;  // append grid dimension
    if (geo->head_dim != 64 && geo->head_dim != 128) return GC_ERR_UNSUPPORTED;
    if (geo->page_size != gc::kPage) return GC_ERR_UNSUPPORTED;
    sh->group = group;
    sh->tq = gc::tokens_per_tile(group, sh->block_m);
    sh->total_tokens = 0;
    if (b->batch == 0) return GC_OK;
    if (b->prefix_lens_host == nullptr || b->new_lens_host == nullptr) return GC_ERR_NULL_ARG;
    int64_t total = 0;
    for (int r = 0; r < b->batch; ++r) {
        const int64_t P = b->prefix_lens_host[r], n = b->new_lens_host[r];
        if (P < 0 || n < 0) return GC_ERR_BAD_SHAPE;
        if (P + n > (int64_t)INT32_MAX - gc::kBlockN) return GC_ERR_BAD_SHAPE;
        total += n;
    }
    if (total > (int64_t)INT32_MAX) return GC_ERR_BAD_SHAPE;
    for (int r = 0; r < b->batch; ++r) {
        const int64_t P = b->prefix_lens_host[r], n = b->new_lens_host[r];
        if (n > 0 && (P + n + gc::kPage - 1) / gc::kPage > geo->max_blocks_per_seq)
            return GC_ERR_BLOCK_TABLE;
    }
    sh->total_tokens = total;
    // the append grid: one workgroup per (page receiving new tokens, KV head), plus
    // the planner's in the combined launch
    if (gc::append_pages_host(b->prefix_lens_host, b->new_lens_host, b->batch) * geo->num_kv_heads >=
        (int64_t)INT32_MAX)
        return GC_ERR_UNSUPPORTED;
    if (total > 0) {
        if (geo->num_blocks <= 0) return GC_ERR_BAD_SHAPE;
        if (b->prefix_lens_dev == nullptr || b->cu_new_lens_dev == nullptr ||
            b->block_tables_dev == nullptr)
            return GC_ERR_NULL_ARG;
    }
    return GC_OK;
}

gc_status check_options(const gc_plan_options* o) {
    if (o == nullptr) return GC_OK;
    if (o->tiling != GC_TILES_AUTO && o->tiling != GC_TILES_PREFILL && o->tiling != GC_TILES_SMALL &&
        o->tiling != GC_TILES_WIDE)
        return GC_ERR_BAD_SHAPE;
    for (int i = 0; i < 6; ++i)
        if (o->reserved[i] != 0) return GC_ERR_BAD_SHAPE;
    return GC_OK;
}

// Tiling: small tiles (one wavefront per 16 query rows, K and V pages streamed through
// its own LDS ring) when every request's new tokens fit one such tile, which is the
// decode case. Otherwise LDS-staged prefill tiles, 128 rows (two workgroups per CU) or
// wide (256 rows, one workgroup per CU). Wide tiles copy each K/V tile once for twice the
// rows; over 8-bit pools, which share their plans with bf16 ones, they also widen it once for
// twice the rows. So at d = 128 and with wide tiles >= 85 % full they are taken, except
//   - between one and two per CU, where whole units leave the last round mostly idle (bf16,
//     128-row against wide: 965 us / 1072 at 288 wide tiles);
//   - below one per CU with fewer than kWideSplitTiles key tiles per CU: a wide launch that
//     short is one prologue, and two small workgroups cover each other's (20.2 / 23.6 at
//     1.4 tiles, 20.0 / 23.8 at 1.7; over 8-bit pools 24.9 / 25.7 and 24.2 / 25.3; at 2.5
//     22.0 / 23.9, but 26.4 / 25.4 over 8-bit pools).
// Above two per CU, 128-row tiles win over bf16 pools up to about 140 key tiles per CU (79 / 93
// at 19, 182 / 189 at 85) and lose 2 to 16 % over 8-bit pools at every size, so wide.
// Not at d = 64 (half the products for the same weights): three 128-row workgroups share a
// compute unit there (164 registers) and overlap better: 16 misses of 100 to 1500 tokens 120 us
// against 148 on wide tiles.
constexpr int kWideSplitTiles = 2;
int device_cus();

// f(key tiles) for every query tile of the batch (block_n: a power of two).
template <typename F>
inline void for_each_tile(const gc_batch* b, int tq, int block_n, F&& f) {
    const int shift = __builtin_ctz((unsigned)block_n);
    for (int r = 0; r < b->batch; ++r) {
        const uint32_t P = (uint32_t)b->prefix_lens_host[r], n = (uint32_t)b->new_lens_host[r];
        for (uint32_t q0 = 0; q0 < n; q0 += (uint32_t)tq) {
            const uint32_t end = q0 + (uint32_t)tq < n ? q0 + (uint32_t)tq : n;
            f((int)((P + end + (uint32_t)block_n - 1) >> shift));
        }
    }
}

gc_status choose_tiling(const gc_geometry* geo, const gc_batch* b, const gc_plan_options* o, Shape* sh) {
    const int want = o == nullptr ? GC_TILES_AUTO : o->tiling;
    bool small = false, wide = false;
    if (want == GC_TILES_SMALL) {
        if (sh->group > gc::kDecM) return GC_ERR_UNSUPPORTED;
        small = true;
    } else if (want == GC_TILES_WIDE) {
        wide = true;
    } else if (want == GC_TILES_AUTO) {
        if (sh->group <= gc::kDecM) {
            small = true;
            for (int r = 0; r < b->batch && small; ++r)
                small = (int64_t)b->new_lens_host[r] * sh->group <= gc::kDecM;
        }
        if (!small && geo->head_dim == 128) {
            const int tq = gc::tokens_per_tile(sh->group, gc::kWideM);
            int64_t units = 0, rows = 0;
            for (int r = 0; r < b->batch; ++r) {
                units += gc::ceil_div64(b->new_lens_host[r], tq);
                rows += (int64_t)b->new_lens_host[r] * sh->group;
            }
            const int64_t cus = device_cus();
            const int64_t grid = units * geo->num_kv_heads;
            if (rows * 100 >= units * gc::kWideM * 85) {
                wide = grid >= 2 * cus;
                if (grid <= cus) {
                    int64_t tiles = 0;
                    for_each_tile(b, tq, gc::kBlockN, [&](int kt) { tiles += kt; });
                    wide = tiles * geo->num_kv_heads >= kWideSplitTiles * cus;
                }
            }
        }
    }
    sh->small = small;
    sh->wide = wide;
    sh->block_m = small ? gc::kDecM : (wide ? gc::kWideM : gc::kBlockM);
    sh->block_n = small ? gc::kDecN : gc::kBlockN;
    sh->tq = gc::tokens_per_tile(sh->group, sh->block_m);
    return GC_OK;
}

// Compute units of the current device (cached per device id).
int device_cus() {
    static std::mutex mu;
    static int cache[64] = {0};
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0) return 256;
    if (dev < 64) {
        std::lock_guard<std::mutex> g(mu);
        if (cache[dev] > 0) return cache[dev];
    }
    int cus = 0;
    if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0)
        cus = 256;
    if (dev < 64) {
        std::lock_guard<std::mutex> g(mu);
        cache[dev] = cus;
    }
    return cus;
}

// Split policy: keep whole query tiles when there are at least as many work
// items as resident slots (per compute unit: two 128-row workgroups, one wide
// workgroup, or four small-tile wavefronts); otherwise cut the keys into chunks
// so that the launch fills those slots: the smallest chunk that makes no more items
// than slots (each query tile's chunks are rounded up, so equal shares of the key
// tiles make a few items more, which run a round of their own), unless the busiest slot
// ends 8 % sooner with equal shares; and at least 512 keys
// (384 for small tiles), below which the partial rows and a work item's fixed cost
// outweigh the shorter chunks.
// Measured on MI355X (attention and merge, 70B heads): one request of 4100 tokens
// 15.9 us with chunks of 384 keys (24.3 with 1024), four requests of 61 MB of codes
// 18.1 us (29.4 with 1024, 21.5 with 128); 32 requests of 791 MB 145 us with 1000
// items (155 with 1150, 162 with 4000). 16 requests of 4 to 64 new tokens on 4000
// cached ones: 85 us with 480 128-row items (103 with the 600 of equal shares, 97 with
// 1000); one request of 512 on 8000: 137 us with 256 wide items (165 with 288).
// Fitting against equal shares on batches of 0.4 to 1 query tile per slot (1000 of them), by the
// busiest slot of the shares over the fitting chunk, each with an item's fixed cost in key tiles.
// Below 0.92 (12/11) prefill tiles lose by fitting (wide: 114 us / 202 at 0.48, 145 / 220 at
// 0.60, 126 / 159 at 0.69, 66 / 74 at 0.77; 128-row: 230 / 287 at 0.78, 89 / 110 at 0.82), above it
// they gain (wide 45 / 38 at 1.09, 62 / 47 at 1.21; 128-row 89 / 70 at 0.97, 110 / 89 at 1.25),
// with an exception in 100 batches. Small tiles are bound by the memory, not by the slot that ends last, so
// a second item has to save much: 264 / 333 at 0.68, but 59 / 48 at 1.47 and 335 / 278 at 0.95
// (8-bit pools would gain up to 30 % between 0.8 and 1.1, and share their plans with bf16 ones).
constexpr int kSmallMinChunkKeys = 384;
constexpr int kItemTilesSmall = 64, kItemTiles = 16, kItemTilesWide = 5;
constexpr int64_t kMaxSlots = 2048;  // (of 256 compute units: 1024)
int64_t resident_slots(const Shape& sh) {
    const int64_t slots = (sh.small ? 4LL : (sh.wide ? 1LL : 2LL)) * device_cus();
    return slots < kMaxSlots ? slots : kMaxSlots;
}

// Key tiles, and `fixed` for each item, of the slot that ends last when the query tiles kts[0 .. units)
// are cut into chunks of c key tiles (every one `heads` times), more items than slots and at most
// twice as many, and run heaviest first: the items past the slots follow the lightest of the first
// round, the heaviest of the one after the lightest of the other. (Sizes in at most 512 steps.)
// partials: the chunks of the query tiles that are cut.
int busiest_slot(const int32_t* kts, int units, int c, int heads, int64_t slots, int fixed, int64_t* partials) {
    constexpr int kSizes = 512;
    int shift = 0;
    while ((c >> shift) >= kSizes) ++shift;
    const int top = c >> shift;
    int32_t count[kSizes];
    for (int s = 0; s <= top; ++s) count[s] = 0;
    int whole = 0, cut = 0;  // items of query tiles in one piece, and in several
    for (int i = 0; i < units; ++i) {
        if (kts[i] <= c) {
            count[kts[i] >> shift] += 1;
            whole += 1;
            continue;
        }
        const int ns = 1 + (int)((double)(kts[i] - 1) / (double)c);  // (exact, as in choose_chunk)
        const int lo = (int)((double)kts[i] / (double)ns), n_hi = kts[i] - lo * ns;
        count[lo >> shift] += ns - n_hi;
        if (n_hi > 0) count[(lo + 1) >> shift] += n_hi;
        cut += ns;
    }
    *partials = cut;
    int64_t past = (int64_t)(whole + cut) * heads - slots;
    // the size `a` at place slots - 1 of the list, then upwards; `b` from place slots downwards
    int a = top;
    int64_t in_a = (int64_t)count[a] * heads, first = slots;
    int alone = 0, two = 0;  // most tiles of a slot with one item, with two
    while (first > in_a && a > 0) {
        if (in_a > 0 && alone == 0) alone = a;
        first -= in_a;
        in_a = (int64_t)count[--a] * heads;
    }
    int b = a;
    int64_t in_b = in_a - first;  // those of size a past the slots
    in_a = first;
    while (past > 0) {
        while (in_a == 0 && a < top) in_a = (int64_t)count[++a] * heads;
        while (in_b == 0 && b > 0) in_b = (int64_t)count[--b] * heads;
        const int64_t m = in_a < in_b ? in_a : in_b;
        if (m <= 0) break;
        if (a + b > two) two = a + b;
        in_a -= m;
        in_b -= m;
        past -= m;
    }
    alone = (alone << shift) + fixed;
    two = (two << shift) + 2 * fixed;
    return alone > two ? alone : two;
}

int choose_chunk(const gc_geometry* geo, const gc_batch* b, const Shape& sh,
                 const gc_plan_options* o) {
    if (o != nullptr && o->kv_split_tiles != 0) return o->kv_split_tiles > 0 ? o->kv_split_tiles : 0;
    const int64_t target = resident_slots(sh), heads = geo->num_kv_heads;
    int64_t all_units = 0;
    for (int r = 0; r < b->batch; ++r) all_units += gc::ceil_div64(b->new_lens_host[r], sh.tq);
    if (all_units * heads >= target || all_units == 0) return 0;
    const int units = (int)all_units;  // fewer than slots
    int32_t kts[kMaxSlots];            // their key tiles
    int max_tiles = 1, at = 0;
    int64_t tiles = 0;
    for_each_tile(b, sh.tq, sh.block_n, [&](int kt) {
        kts[at++] = kt;
        tiles += kt;
        if (kt > max_tiles) max_tiles = kt;
    });
    const int64_t least = (tiles * heads + target - 1) / target;  // equal shares
    const int min_keys = sh.small ? kSmallMinChunkKeys : 512;
    int lo = least < min_keys / sh.block_n ? min_keys / sh.block_n : (int)least;  // (least <= max_tiles)
    if (lo >= max_tiles) return lo;  // unsplit
    // The smallest chunk whose items fit the slots, per KV head. A chunk of c makes fewer than
    // tiles / c + units items, which bounds the search from above.
    const int64_t slots = target / heads;
    auto items = [&](int c) {  // (exact: a double holds either operand, and quotients below 2^31 apart)
        int k = units;
        for (int i = 0; i < units; ++i) k += (int)((double)(kts[i] - 1) / (double)c);
        return (int64_t)k;
    };
    const int64_t shares = items(lo);
    if (shares <= slots) return lo;
    int hi = max_tiles;  // unsplit tiles: units < slots
    if (slots > units && (tiles + slots - units - 1) / (slots - units) < hi)
        hi = (int)((tiles + slots - units - 1) / (slots - units));
    // Near as many query tiles as slots, few of them can be cut: where the chunk that fits is far
    // above the load of the busiest slot with equal shares, those are better.
    // (That slot carries at least the mean load.)
    const int fixed = sh.small ? kItemTilesSmall : sh.wide ? kItemTilesWide : kItemTiles;
    auto limit = [&](int64_t load) { return load * 12 / 11 - fixed; };
    const int64_t mean = (tiles + shares * fixed) * heads / target;
    if (limit(mean) < hi && items((int)limit(mean)) <= slots) {
        hi = (int)limit(mean);
    } else if (limit(mean) < hi && shares < 2 * slots) {
        int64_t partials;
        const int64_t fits = limit(busiest_slot(kts, units, lo, (int)heads, target, fixed, &partials));
        // (partial rows within 60 MB, that the calls on the fixed scratch take the batch)
        if (fits < hi && partials * heads * sh.block_m * (geo->head_dim + 1) * 4 <= 60000000) {
            if (fits <= lo || items((int)fits) > slots) return lo;
            hi = (int)fits;
        }
    }
    lo += 1;
    while (lo < hi) {
        const int mid = lo + (hi - lo) / 2;
        if (items(mid) <= slots) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// Work-list order. Items run in list order, and a list in strict cost order,
// heaviest first, ends on its lightest items (longest-processing-time order).
// Only the end needs that order, though: before it the items are sorted by the
// length of their request instead, so that a request's query tiles, which read
// nearly the same keys, run side by side and share the K/V tiles in L2. In cost
// order the tiles of a long miss (one of every cost from 1 up) are spread over the
// whole launch and each fetches the same K/V again. The lightest items, two rounds
// of the resident slots, keep the strict order: items of fewer than group_cost
// key tiles; a list no longer than that is not grouped at all.
void choose_order(const gc_geometry* geo, const gc_batch* b, const Shape& sh, Plan* pl) {
    pl->group_cost = gc::kCostBuckets;
    const int64_t tail = (2 * resident_slots(sh) + geo->num_kv_heads - 1) / geo->num_kv_heads;  // items per KV head
    if (pl->items <= tail) return;
    int64_t hist[gc::kCostBuckets] = {};  // items per cost (clamped like the planner's buckets)
    for_each_tile(b, sh.tq, sh.block_n, [&](int kt) {
        const int ns = gc::num_splits(kt, pl->chunk);
        const int lo = ns == 1 ? kt : kt / ns, n_hi = kt - lo * ns;
        hist[lo < gc::kCostBuckets - 1 ? lo : gc::kCostBuckets - 1] += ns - n_hi;
        if (n_hi > 0) hist[lo + 1 < gc::kCostBuckets - 1 ? lo + 1 : gc::kCostBuckets - 1] += n_hi;
    });
    int64_t below = 0;
    int c = 0;
    while (c < gc::kCostBuckets && below < tail) below += hist[c++];
    pl->group_cost = c;  // the items of cost < c make up the tail
}

// Which 128-row workgroups the kernel prefers (attention_kernels.h): of the two that share a
// compute unit, the first round's, which hold the heaviest items, or the second's. The
// first where the heaviest item decides the end: in launches of one round, and beyond where its
// key tiles exceed the mean load of a slot by a quarter (an item's fixed cost counted as four
// tiles; below a quarter the lighter items had better end soon and make room). Preferring the
// second round against the first, bf16 / 8-bit pools, 200 ragged batches: one round 1.00 to
// 1.13 times the time (520 items, the longest of 63 tiles on a mean load of 41: 100.0 us / 89.2,
// 126.5 / 117.1); 1.25 to 3 times the mean load 0.92 to 1.15, two in three above 1.04; below,
// 0.84 to 1.06 (chat turns of 648 items, 62 tiles on 56: 117.1 / 120.4, 151.0 / 173.1).
bool heaviest_decides(int64_t items, int64_t tiles, int heaviest, int64_t slots) {
    constexpr int kItemTiles = 4;
    return items <= slots || (heaviest + kItemTiles) * slots * 4 >= (tiles + kItemTiles * items) * 5;
}

// 8-bit pools at d = 64: 128-row tiles run three workgroups per compute unit, at the price of spilled
// registers, where there is a third one and the mean load of a slot (two per unit) is long enough
// for the spills at an item's ends (three workgroups / two: 84.2 us / 95.0 at 58 tiles, 41.1 / 46.7
// at 28, 69.2 / 74.2 at 17, 30.4 / 30.9 at 15; 24.4 / 23.1 at 11, 22.2 / 21.1 at 9).
constexpr int kThirdTiles = 13;

gc_status make_plan(const gc_geometry* geo, const gc_batch* b, const Shape& sh,
                    const gc_plan_options* o, Plan* pl) {
    pl->chunk = choose_chunk(geo, b, sh, o);
    int longest = 0;  // key tiles of the longest query tile
    const int chunk = pl->chunk;
    int64_t units = 0, combines = 0, partials = 0, tiles = 0;
    for_each_tile(b, sh.tq, sh.block_n, [&](int kt) {
        units += 1;
        tiles += kt;
        if (kt > longest) longest = kt;
        if (chunk > 0 && kt > chunk) {
            combines += 1;
            partials += (uint32_t)(kt + chunk - 1) / (uint32_t)chunk;
        }
    });
    pl->items = units - combines + partials;
    pl->combines = combines;
    pl->partials = partials;
    pl->max_splits = gc::num_splits(longest, chunk);
    if (pl->items > (int64_t)INT32_MAX / geo->num_kv_heads) return GC_ERR_BAD_SHAPE;
    const int64_t slots = resident_slots(sh);
    pl->heaviest_decides = heaviest_decides(pl->items * geo->num_kv_heads, tiles * geo->num_kv_heads,
                                            chunk > 0 && longest > chunk ? chunk : longest, slots);
    pl->three = pl->items * geo->num_kv_heads > slots && tiles * geo->num_kv_heads >= kThirdTiles * slots;
    pl->layout = gc::workspace_layout(b->batch, pl->items, pl->combines, pl->partials,
                                      geo->num_kv_heads, geo->head_dim, sh.block_m);
    choose_order(geo, b, sh, pl);
    // the largest sort key: a request's key tiles where items are grouped, an item's otherwise
    int key = pl->group_cost < gc::kCostBuckets || pl->chunk <= 0 || longest < pl->chunk ? longest : pl->chunk;
    if (key > gc::kCostBuckets - 1) key = gc::kCostBuckets - 1;
    pl->buckets = (key / gc::kPlanThreads + 1) * gc::kPlanThreads;
    return GC_OK;
}

template <typename T>
T* at(void* ws, size_t off) {
    return reinterpret_cast<T*>(static_cast<char*>(ws) + off);
}

gc_status plan_checked(const gc_geometry* geo, const gc_batch* b, const gc_plan_options* o,
                       Shape* sh, Plan* pl) {
    gc_status st = check_common(geo, b, sh);
    if (st != GC_OK) return st;
    st = check_options(o);
    if (st != GC_OK) return st;
    st = choose_tiling(geo, b, o, sh);
    if (st != GC_OK) return st;
    if (sh->total_tokens == 0) return GC_OK;
    return make_plan(geo, b, *sh, o, pl);
}

gc::PlanArgs plan_args(const gc_geometry* geo, const gc_batch* b, const Shape& sh, const Plan& pl, void* ws) {
    gc::PlanArgs a{};
    a.prefix_lens = b->prefix_lens_dev;
    a.cu_new_lens = b->cu_new_lens_dev;
    a.scratch = at<int32_t>(ws, pl.layout.scratch_off);
    a.items = at<gc::WorkItem>(ws, pl.layout.items_off);
    a.combines = at<gc::CombineItem>(ws, pl.layout.combine_off);
    a.status = at<int32_t>(ws, pl.layout.status_off);
    a.queues = at<int32_t>(ws, pl.layout.queue_off);
    a.shared_mark = at<int32_t>(ws, gc::kMarkOffset);
    a.batch = b->batch;
    a.tq = sh.tq;
    a.chunk = pl.chunk;
    a.block_n = sh.block_n;
    a.expect_items = (int32_t)pl.items;
    a.expect_combines = (int32_t)pl.combines;
    a.expect_partials = (int32_t)pl.partials;
    a.total_tokens = (int32_t)sh.total_tokens;
    a.max_blocks = geo->max_blocks_per_seq;
    a.group_cost = pl.group_cost;
    a.buckets = pl.buckets;
    return a;
}

gc_status enqueue_plan(const gc_geometry* geo, const gc_batch* b, const Shape& sh, const Plan& pl,
                       void* ws, hipStream_t stream) {
    return gc::launch_plan(plan_args(geo, b, sh, pl, ws), stream) == hipSuccess ? GC_OK : GC_ERR_HIP;
}

// Wide tiles with at least two rounds of work items per compute unit run as a
// resident launch (one workgroup per CU taking items from per-XCD queues;
// attention_kernels.h): it removes the dispatch gaps between items and lets the XCDs that
// finish first take the last items of the others. A single round has nothing to
// balance. 0: the regular launch.
int resident_workgroups(const gc_geometry* geo, const Shape& sh, const Plan& pl) {
    if (!sh.wide) return 0;
    const int cus = device_cus();
    if (cus % gc::kQueues != 0) return 0;
    return pl.items * geo->num_kv_heads >= 2LL * cus ? cus : 0;
}

// Pools of bf16 elements (fp8 false, scales 1) or of E4M3 codes with one scale each.
struct PoolKind {
    bool fp8 = false;
    float k_scale = 1.f, v_scale = 1.f;
};

gc_status enqueue_run(const gc_geometry* geo, const gc_batch* b, const Shape& sh, const Plan& pl,
                      const void* q, const void* k_pool, const void* v_pool, float scale,
                      void* out, float* lse, void* ws, hipStream_t stream, const PoolKind& pk = PoolKind{}) {
    gc::AttnArgs a{};
    a.q = static_cast<const uint16_t*>(q);
    a.k_pool = static_cast<const uint16_t*>(k_pool);
    a.v_pool = static_cast<const uint16_t*>(v_pool);
    a.out = static_cast<uint16_t*>(out);
    a.lse = lse;
    a.part_o = at<float>(ws, pl.layout.part_o_off);
    a.part_lse = at<float>(ws, pl.layout.part_lse_off);
    a.block_tables = b->block_tables_dev;
    a.items = at<gc::WorkItem>(ws, pl.layout.items_off);
    a.queues = at<int32_t>(ws, pl.layout.queue_off);
    a.num_q_heads = geo->num_q_heads;
    a.num_kv_heads = geo->num_kv_heads;
    a.group = sh.group;
    a.tq = sh.tq;
    a.num_blocks = geo->num_blocks;
    a.max_blocks = geo->max_blocks_per_seq;
    a.scale_log2 = (float)((double)scale * (double)pk.k_scale * 1.4426950408889634074);
    a.v_scale = pk.v_scale;
    a.prefer_span = (uint32_t)device_cus();
    a.prefer_odd = pl.heaviest_decides ? 0 : 1;
    const hipError_t e = sh.small ? gc::launch_attention_small(a, geo->head_dim, pl.items, pk.fp8, stream)
                                  : gc::launch_attention(a, geo->head_dim, pl.items, sh.wide, pl.three, pk.fp8,
                                                         resident_workgroups(geo, sh, pl), stream);
    if (e != hipSuccess) return GC_ERR_HIP;
    if (pl.combines > 0) {
        gc::CombineArgs c{};
        c.out = a.out;
        c.lse = lse;
        c.part_o = a.part_o;
        c.part_lse = a.part_lse;
        c.cu_new_lens = b->cu_new_lens_dev;
        c.combines = at<gc::CombineItem>(ws, pl.layout.combine_off);
        c.num_q_heads = geo->num_q_heads;
        c.num_kv_heads = geo->num_kv_heads;
        c.group = sh.group;
        c.tq = sh.tq;
        c.batch = b->batch;
        c.num_partials = (int32_t)pl.partials;
        c.block_m = sh.block_m;
        if (gc::launch_combine(c, geo->head_dim, pl.combines, pl.max_splits, stream) != hipSuccess) return GC_ERR_HIP;
    }
    return GC_OK;
}

gc_status check_run_args(const void* q, const void* k_pool, const void* v_pool, float scale,
                         void* out) {
    if (q == nullptr || k_pool == nullptr || v_pool == nullptr || out == nullptr)
        return GC_ERR_NULL_ARG;
    if (!std::isfinite(scale) || !(scale > 0.f)) return GC_ERR_BAD_SHAPE;
    return GC_OK;
}

gc_status check_pool_scales(float k_scale, float v_scale) {
    if (!std::isfinite(k_scale) || !(k_scale > 0.f) || !std::isfinite(v_scale) || !(v_scale > 0.f))
        return GC_ERR_BAD_SHAPE;
    // the append multiplies by fl32(1 / scale), which must be finite as well
    if (!std::isfinite(1.f / k_scale) || !std::isfinite(1.f / v_scale)) return GC_ERR_BAD_SHAPE;
    return GC_OK;
}

gc_status check_workspace(const Plan& pl, const void* ws, size_t bytes) {
    if (ws == nullptr || bytes < pl.layout.total) return GC_ERR_WORKSPACE;
    return GC_OK;
}

gc::AppendArgs append_args(const gc_geometry* geo, const gc_batch* batch, const Shape& sh,
                           const void* k_new, const void* v_new, void* k_pool, void* v_pool,
                           const PoolKind& pk) {
    gc::AppendArgs a{};
    a.k_new = static_cast<const uint16_t*>(k_new);
    a.v_new = static_cast<const uint16_t*>(v_new);
    a.k_pool = k_pool;
    a.v_pool = v_pool;
    a.prefix_lens = batch->prefix_lens_dev;
    a.cu_new_lens = batch->cu_new_lens_dev;
    a.block_tables = batch->block_tables_dev;
    a.batch = batch->batch;
    a.total_tokens = (int32_t)sh.total_tokens;
    a.num_kv_heads = geo->num_kv_heads;
    a.num_blocks = geo->num_blocks;
    a.max_blocks = geo->max_blocks_per_seq;
    a.total_pages = (int32_t)gc::append_pages_host(batch->prefix_lens_host, batch->new_lens_host, batch->batch);
    a.k_inv = 1.f / pk.k_scale;  // IEEE division: the same fl32(1 / scale) the definition uses
    a.v_inv = 1.f / pk.v_scale;
    return a;
}

gc_status append(const gc_geometry* geo, const gc_batch* batch, const void* k_new, const void* v_new,
                 void* k_pool, void* v_pool, const PoolKind& pk, hipStream_t stream) {
    Shape sh;
    gc_status st = check_common(geo, batch, &sh);
    if (st != GC_OK) return st;
    if (sh.total_tokens == 0) return GC_OK;
    if (k_new == nullptr || v_new == nullptr || k_pool == nullptr || v_pool == nullptr)
        return GC_ERR_NULL_ARG;
    const gc::AppendArgs a = append_args(geo, batch, sh, k_new, v_new, k_pool, v_pool, pk);
    return gc::launch_append(a, geo->head_dim, pk.fp8, stream) == hipSuccess ? GC_OK : GC_ERR_HIP;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Bytes that T rows of `width` elements, `stride` elements apart, span from their first one.
int64_t span_bytes(int64_t T, int64_t stride, int64_t width) { return ((T - 1) * stride + width) * 2; }

bool overlap(const void* p, int64_t np, const void* q, int64_t nq) {
    const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
    return a < b + (uintptr_t)nq && b < a + (uintptr_t)np;
}

gc_status append_rotary(const gc_geometry* geo, const gc_batch* batch, const gc_rotary* rot, const gc_new_rows* rows,
                        void* q_out, void* k_pool, void* v_pool, const PoolKind& pk, hipStream_t stream) {
    Shape sh;
    gc_status st = check_common(geo, batch, &sh);
    if (st != GC_OK) return st;
    if (rot == nullptr || rows == nullptr) return GC_ERR_NULL_ARG;
    if (rot->rotary_dim < 16 || rot->rotary_dim > geo->head_dim || rot->rotary_dim % 16 != 0 || rot->num_positions < 0 ||
        (rot->pairs != GC_PAIRS_HALVES && rot->pairs != GC_PAIRS_INTERLEAVED))
        return GC_ERR_BAD_SHAPE;
    for (int i = 0; i < 5; ++i)
        if (rot->reserved[i] != 0) return GC_ERR_BAD_SHAPE;
    if (sh.total_tokens == 0) return GC_OK;
    if (rot->table_dev == nullptr || rows->k == nullptr || rows->v == nullptr || k_pool == nullptr || v_pool == nullptr)
        return GC_ERR_NULL_ARG;
    if ((rows->q == nullptr) != (q_out == nullptr)) return GC_ERR_NULL_ARG;
    const bool with_q = rows->q != nullptr;
    const int64_t T = sh.total_tokens, D = geo->head_dim;
    const int64_t q_row = geo->num_q_heads * D, kv_row = geo->num_kv_heads * D;
    // (the upper bound keeps byte offsets of 2^31 rows within 64 bits)
    auto bad_stride = [](int64_t stride, int64_t row) { return stride < row || stride % 8 != 0 || stride > (1LL << 28); };
    if (bad_stride(rows->k_stride, kv_row) || bad_stride(rows->v_stride, kv_row) ||
        (with_q && bad_stride(rows->q_stride, q_row)))
        return GC_ERR_BAD_SHAPE;
    if (!aligned16(rows->q) || !aligned16(rows->k) || !aligned16(rows->v) || !aligned16(q_out) || !aligned16(rot->table_dev))
        return GC_ERR_BAD_SHAPE;
    for (int r = 0; r < batch->batch; ++r)
        if (batch->new_lens_host[r] > 0 &&
            (int64_t)batch->prefix_lens_host[r] + batch->new_lens_host[r] > rot->num_positions)
            return GC_ERR_BAD_SHAPE;
    if (with_q) {
        const int64_t out = T * q_row * 2, pool = (int64_t)geo->num_blocks * gc::kPage * kv_row * (pk.fp8 ? 1 : 2);
        const bool in_place = q_out == rows->q && rows->q_stride == q_row;
        if ((!in_place && overlap(q_out, out, rows->q, span_bytes(T, rows->q_stride, q_row))) ||
            overlap(q_out, out, rows->k, span_bytes(T, rows->k_stride, kv_row)) ||
            overlap(q_out, out, rows->v, span_bytes(T, rows->v_stride, kv_row)) ||
            overlap(q_out, out, rot->table_dev, (int64_t)rot->num_positions * rot->rotary_dim * 4) ||
            overlap(q_out, out, k_pool, pool) || overlap(q_out, out, v_pool, pool))
            return GC_ERR_BAD_SHAPE;
    }
    gc::RotaryArgs ra{};
    ra.a = append_args(geo, batch, sh, rows->k, rows->v, k_pool, v_pool, pk);
    if (gc::rotary_workgroups(ra.a.total_pages, geo->num_q_heads, geo->num_kv_heads, geo->head_dim, with_q) > gc::kMaxWorkgroups)
        return GC_ERR_UNSUPPORTED;
    ra.q = static_cast<const uint16_t*>(rows->q);
    ra.q_out = static_cast<uint16_t*>(q_out);
    ra.table = rot->table_dev;
    ra.q_stride = rows->q_stride;
    ra.k_stride = rows->k_stride;
    ra.v_stride = rows->v_stride;
    ra.num_q_heads = geo->num_q_heads;
    ra.num_positions = rot->num_positions;
    ra.rotary_dim = rot->rotary_dim;
    ra.interleaved = rot->pairs == GC_PAIRS_INTERLEAVED;
    return gc::launch_append_rotary(ra, geo->head_dim, pk.fp8, stream) == hipSuccess ? GC_OK : GC_ERR_HIP;
}

// Append and plan in one launch (the plan reads only the lengths, so the two are
// independent).
gc_status prepare(const gc_geometry* geo, const gc_batch* batch, const gc_plan_options* opts,
                  const void* k_new, const void* v_new, void* k_pool, void* v_pool, void* workspace,
                  size_t workspace_bytes, hipStream_t stream, const PoolKind& pk) {
    Shape sh;
    Plan pl;
    gc_status st = plan_checked(geo, batch, opts, &sh, &pl);
    if (st != GC_OK || sh.total_tokens == 0) return st;
    if (k_new == nullptr || v_new == nullptr || k_pool == nullptr || v_pool == nullptr)
        return GC_ERR_NULL_ARG;
    if (pk.fp8) {
        st = check_pool_scales(pk.k_scale, pk.v_scale);
        if (st != GC_OK) return st;
    }
    st = check_workspace(pl, workspace, workspace_bytes);
    if (st != GC_OK) return st;
    const gc::AppendArgs aa = append_args(geo, batch, sh, k_new, v_new, k_pool, v_pool, pk);
    return gc::launch_prepare(aa, plan_args(geo, batch, sh, pl, workspace), geo->head_dim, pk.fp8, stream) ==
                   hipSuccess
               ? GC_OK
               : GC_ERR_HIP;
}

gc_status run(const gc_geometry* geo, const gc_batch* batch, const gc_plan_options* opts,
              const void* q, const void* k_pool, const void* v_pool, float scale, void* out,
              float* lse, void* workspace, size_t workspace_bytes, hipStream_t stream,
              bool with_plan, const PoolKind& pk) {
    Shape sh;
    Plan pl;
    gc_status st = plan_checked(geo, batch, opts, &sh, &pl);
    if (st != GC_OK || sh.total_tokens == 0) return st;
    st = check_run_args(q, k_pool, v_pool, scale, out);
    if (st != GC_OK) return st;
    if (pk.fp8) {
        st = check_pool_scales(pk.k_scale, pk.v_scale);
        if (st != GC_OK) return st;
    }
    st = check_workspace(pl, workspace, workspace_bytes);
    if (st != GC_OK) return st;
    if (with_plan) {
        st = enqueue_plan(geo, batch, sh, pl, workspace, stream);
        if (st != GC_OK) return st;
    }
    return enqueue_run(geo, batch, sh, pl, q, k_pool, v_pool, scale, out, lse, workspace, stream, pk);
}

// ---------------------------------------------------------------- no-allocation variant
// Workspace of gc_prefix_prefill_attention_noalloc: one file-scope device array per
// GPU the library runs on (held until the process ends). Host code never passes the
// array's name to a kernel or a copy: in host code it is a host-side stand-in, not
// a device address. The device address comes from hipGetSymbolAddress, taken once
// per device with that device current, and is kept per device.
static __device__ __align__(256) unsigned char scratch[GC_NOALLOC_SCRATCH_BYTES];

constexpr int kMaxDevices = 64;
struct DeviceScratch {
    std::once_flag once;
    void* ptr = nullptr;
    hipError_t err = hipSuccess;
};
DeviceScratch g_scratch[kMaxDevices];

// Device address of the current device's scratch array (nullptr and a status on failure).
void* scratch_address(gc_status* st) {
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0) {
        *st = GC_ERR_HIP;
        return nullptr;
    }
    if (dev >= kMaxDevices) {
        *st = GC_ERR_UNSUPPORTED;
        return nullptr;
    }
    DeviceScratch& d = g_scratch[dev];
    std::call_once(d.once, [&d]() { d.err = hipGetSymbolAddress(&d.ptr, HIP_SYMBOL(scratch)); });
    if (d.err != hipSuccess || d.ptr == nullptr) {
        *st = GC_ERR_HIP;
        return nullptr;
    }
    *st = GC_OK;
    return d.ptr;
}

// Append and run from a plan already in the workspace, as two launches. One launch that
// read the new keys from k_new / v_new and wrote them into the pool from LDS read the new keys'
// values through registers in every tile that holds some, and could not run as a resident
// launch. One / two launches, us a pass, on the same tiles: 16 chat requests of the 70B shape 214 /
// 195, 8 of the 8B shape 147 / 128, the mixed 70B batch 2547 / 2196, 6 mixed 8B requests 205 / 174;
// only the smallest calls lose the second launch (one request of 32 tokens 11.7 / 14.1).
gc_status run_with_append(const gc_geometry* geo, const gc_batch* batch, const gc_plan_options* opts,
                          const void* q, const void* k_new, const void* v_new, void* k_pool, void* v_pool,
                          float scale, void* out, float* lse, void* workspace, size_t workspace_bytes,
                          hipStream_t stream) {
    Shape sh;
    Plan pl;
    gc_status st = plan_checked(geo, batch, opts, &sh, &pl);
    if (st != GC_OK || sh.total_tokens == 0) return st;
    st = check_run_args(q, k_pool, v_pool, scale, out);
    if (st != GC_OK) return st;
    if (k_new == nullptr || v_new == nullptr) return GC_ERR_NULL_ARG;
    st = check_workspace(pl, workspace, workspace_bytes);
    if (st != GC_OK) return st;
    // (a limit of the interface: a request's new rows within 32-bit byte offsets)
    const int64_t row_bytes = (int64_t)geo->num_kv_heads * geo->head_dim * 2;
    for (int r = 0; r < batch->batch; ++r)
        if ((int64_t)batch->new_lens_host[r] * row_bytes > INT32_MAX) return GC_ERR_UNSUPPORTED;
    const gc::AppendArgs aa = append_args(geo, batch, sh, k_new, v_new, k_pool, v_pool, PoolKind{});
    if (gc::launch_append(aa, geo->head_dim, false, stream) != hipSuccess) return GC_ERR_HIP;
    return enqueue_run(geo, batch, sh, pl, q, k_pool, v_pool, scale, out, lse, workspace, stream);
}

// ---------------------------------------------------------------- shared prefixes
struct SharedPlan {
    bool any = false;  // some group's shared keys are taken once (else the plain attention runs)
    gc::SharedSizes z{};
    int64_t big = 0, big_slots = 0;         // 128-row items and their partial slots
    int64_t big_shared = 0;                 // those items of shared parts
    int64_t parts = 0, places = 0;          // small parts and their places in the sequence
    int64_t pieces = 0, runs = 0;           // of the small tiles' sequence
    int max_shared = 0, max_own = 0;        // the most chunks of a part
    gc::SharedLayout layout{};
    uint64_t mark = 0;                      // (see shared_mark)
};

gc_status check_shared(const gc_geometry* geo, const gc_batch* b, const gc_shared* s) {
    if (s == nullptr) return GC_ERR_NULL_ARG;
    if (s->groups < 0 || s->groups > b->batch || (s->groups == 0) != (b->batch == 0)) return GC_ERR_BAD_SHAPE;
    if (s->policy != GC_SHARE_AUTO && s->policy != GC_SHARE_ALWAYS) return GC_ERR_BAD_SHAPE;
    for (int i = 0; i < 6; ++i)
        if (s->reserved[i] != 0) return GC_ERR_BAD_SHAPE;
    if (b->batch == 0) return GC_OK;
    if (s->group_first_host == nullptr || s->shared_lens_host == nullptr) return GC_ERR_NULL_ARG;
    if (s->group_first_host[0] != 0 || s->group_first_host[s->groups] != b->batch) return GC_ERR_BAD_SHAPE;
    for (int g = 0; g < s->groups; ++g) {
        const int ra = s->group_first_host[g], rb = s->group_first_host[g + 1], S = s->shared_lens_host[g];
        if (ra < 0 || rb <= ra || rb > b->batch || S < 0 || S % gc::kPage != 0) return GC_ERR_BAD_SHAPE;
        if (S / gc::kPage > geo->max_blocks_per_seq) return GC_ERR_BLOCK_TABLE;
        for (int r = ra; r < rb; ++r)
            if (b->prefix_lens_host[r] < S) return GC_ERR_BAD_SHAPE;
    }
    return GC_OK;
}

// f(PartWork, shared, own) for every shared part, and then for every own part of the batch (shared: of a
// group whose shared keys are taken once).
template <typename F>
void for_each_part(const gc_batch* b, const gc_shared* s, const gc::SharedSizes& z, F&& f) {
    int64_t at = 0;
    auto part = [&](int keys, int n, bool shared, bool own) {
        const gc::PartWork w = gc::part_work(keys, n, (int)(at & INT32_MAX), z);  // (a longer sequence is refused)
        if (w.small) at += gc::kPieceCost + w.kt;
        f(w, shared, own);
    };
    for (int pass = 0; pass < 2; ++pass) {
        for (int g = 0; g < s->groups; ++g) {
            const int ra = s->group_first_host[g], rb = s->group_first_host[g + 1];
            const int S = z.taken(g, s->shared_lens_host[g], z.take);
            if (pass == 0) {
                int tokens = 0;
                for (int r = ra; r < rb; ++r) tokens += b->new_lens_host[r];
                part(S, tokens, S > 0, false);
                continue;
            }
            for (int r = ra; r < rb; ++r)
                part(b->prefix_lens_host[r] - S + b->new_lens_host[r], b->new_lens_host[r], S > 0, true);
        }
    }
}

// Which groups' shared keys are taken once: those that it saves time by the estimates below, if together they
// save more than the merge costs. The plain attention reads S keys for every request, its 16-row tiles from L2
// at about 20 TB/s over all heads (13 of 8-bit codes: 136 answers on 641 tokens 31.6 us, taken once 25.5), its
// 128-row tiles at the matrix cores' pace; taken once, they cost a read from HBM or the pace of the group's own
// 128-row tiles, and every row two fp32 partial rows, written and read. Paces: us of a compute unit per 128-row
// tile and 64 keys (48 requests of 20 tokens on 32768 shared ones, the plain attention / this one: 1316 us /
// 1074, 8-bit pools 1763 / 1206; at d = 64 533 / 288 and 665 / 341).
// Short launches of 128-row tiles are bound by their latency, which the finer chunks here make shorter: up to 64
// tiles over all heads and 4096 of their key tiles, groups of 256 shared keys or more are taken (16.0 us / 13.2
// for two requests of 3 tokens on 513, 18.8 / 15.5 for 27 on 796, 21.7 / 17.9 for 7 of 19 tokens; at 16384 key
// tiles 117 / 128).
// More than kTakeGroups groups (a choice of single ones would not fit the kernel's argument): all or none, by the
// sum of what each saves or loses, with the plain attention's reads at the memory's rate too: that many prefixes are not
// in L2 when the next request of a group comes (520 pairs of answers on 2000 tokens 1504 us / 1019). Against the better of
// both ways 60 such batches take 1.05 times the time, all taken 1.40, none 1.27.
constexpr double kShareGain = 2.0, kShareGainTiles = 6.0;  // us: batches of small tiles; with 128-row own parts
constexpr int kShortTiles = 64, kShortSteps = 4096, kShortKeys = 256;

void choose_groups(const gc_geometry* geo, const gc_batch* b, const gc_shared* s, const PoolKind& pk, gc::SharedSizes* z) {
    z->all = s->policy == GC_SHARE_ALWAYS;
    if (z->all) return;
    const bool many = s->groups > gc::kTakeGroups;
    const double heads = geo->num_kv_heads, D = geo->head_dim;
    const double key_bytes = heads * D * 2 * (pk.fp8 ? 1 : 2);
    const double hbm = 5.6e6;                                // bytes in a us
    const double l2 = many ? hbm : pk.fp8 ? 13e6 : 20e6;
    const double step = heads / device_cus() / gc::kBlockN;  // of a 128-row tile, per key
    const double plain_pace = D == 128 ? (pk.fp8 ? 1.13 : 0.85) : (pk.fp8 ? 0.86 : 0.69);
    const double shared_pace = D == 128 ? (pk.fp8 ? 1.03 : 0.95) : (pk.fp8 ? 0.71 : 0.62);
    double gain = 0;
    bool any_tiles = false;
    double all_tiles = 0, all_steps = 0;  // of all requests, over all heads
    uint64_t brief[gc::kTakeGroups / 64] = {};
    for (int g = 0; g < s->groups; ++g) {
        const int S = s->shared_lens_host[g];
        int64_t small = 0, tiles = 0, tokens = 0;
        for (int r = s->group_first_host[g]; r < s->group_first_host[g + 1]; ++r) {
            const int n = b->new_lens_host[r];
            tokens += n;
            if (n > z->tq_small) tiles += z->tq.ceil_of(n);
            else small += n > 0;
        }
        all_tiles += tiles * heads;
        all_steps += tiles * heads * S / gc::kBlockN;
        if (S <= 0 || tokens == 0) continue;
        if (!many && tiles >= 2 && S >= kShortKeys) brief[g / 64] |= 1ull << (g % 64);
        const double plain = S * (small * key_bytes / l2 + tiles * step * plain_pace);
        const double read = key_bytes / hbm;
        const double paced = tokens <= z->tq_small ? 0 : gc::ceil_div64(tokens, z->tq.d) * step * shared_pace;
        const double rows = tokens * geo->num_q_heads * D * 4 * 4 / 4e6;
        const double saved = plain - S * (read > paced ? read : paced) - rows;
        if (!many && saved < 0.2) continue;
        if (!many) z->take[g / 64] |= 1ull << (g % 64);
        gain += saved;
        any_tiles |= tiles > 0;
    }
    if (many) {
        z->all = gain >= (any_tiles ? kShareGainTiles : kShareGain);
        return;
    }
    if (gain < (any_tiles ? kShareGainTiles : kShareGain))
        for (uint64_t& t : z->take) t = 0;
    if (all_tiles <= kShortTiles && all_steps <= kShortSteps)
        for (int i = 0; i < gc::kTakeGroups / 64; ++i) z->take[i] |= brief[i];
}

// Chunks of the key axis.
//   - 128-row tiles at d = 128: one workgroup a compute unit, whose other half runs small tiles; alone, two would be
//     8 % faster and write twice the partial rows (64 answers on 8192 shared tokens and hardly any of their own:
//     33 us with 256 items, 36 with 512; 37 with 192). At d = 64 two (24 questions of 20 tokens on 4000: 40 us with
//     360 and 480 shared items, 48 with 240). So the smallest chunk whose items make a whole number of such
//     rounds: an item longer than two thirds of the chunk fills a slot, and all of them the slots by their
//     key tiles and kItemSteps more each. Where reading the small tiles takes longer than that, the load alone
//     decides (128 answers on 16k-token contexts: 304 items of 45 key tiles 132 us, 240 of 60 143), and an item
//     may take 0.7 of that reading (64 answers on 4000 tokens and 300 of their own 30.1 us, with the smallest such chunk
//     33.7; 135 on 6000 and 1500 243 / 274; 183 at d = 64 31.4 / 43.6).
//   - Without many small tiles, from kLongSteps key tiles a slot on, two workgroups a unit at d = 128 too: their partial
//     rows are few beside that (13 questions of 11 tokens on 13300 over 8-bit pools 69.0 us, one a unit 76.9; 57 answers on
//     26835 79.0 / 77.1).
//   - More query tiles than slots: no chunk longer than a third of the longest part, or than a fifth where that has
//     more than 64 key tiles. Whole parts run in step, two workgroups a unit at the same phase (48 questions of 20 tokens on 32768
//     1074 us, whole 1431; over 8-bit pools 1206 / 1626; 40 of 30 on 8000 at d = 64 113 / 119).
//   - A few items more than slots are a round more: up to a quarter longer chunks where that avoids it (16 questions of 10
//     tokens on 3000 at d = 64 21.8 us / 24.1, 5 of 29 on 13055 38.1 / 42.5).
//   - At least kMinChunk key tiles (16 answers of the 8B model on 2000 tokens: 16.4 us with 4, 15.8 with 3, 16.6 with
//     2, 17.4 with 6, 20.4 with 8).
//   - Small tiles: equal runs, one for each of the wavefronts that the remaining workgroup slots hold, of at least
//     kMinRun places. Where some units hold two 128-row workgroups, two thirds of that, because the rest of
//     the small workgroups follow when the first end (132 us; 145 with whole runs).
constexpr int kMinChunk = 4, kMinRun = 8, kItemSteps = 4, kLongSteps = 20;

// The batch's work: 128-row parts (the first kKept of them kept) and the places of the small ones.
struct SharedLoad {
    static constexpr int kKept = 512;
    struct {
        int tiles, kt;
    } part[kKept];
    int parts = 0, longest = 1;
    int64_t units = 0, steps = 0, places = 0, small_tiles = 0;  // 128-row tiles, their key tiles; small key tiles
};

void shared_load(const gc_batch* b, const gc_shared* s, const gc::SharedSizes& z, SharedLoad* l) {
    for_each_part(b, s, z, [&](const gc::PartWork& w, bool, bool) {
        if (w.small) {
            l->places += gc::kPieceCost + w.kt;
            l->small_tiles += w.kt;
        } else if (w.tiles > 0) {
            l->units += w.tiles;
            l->steps += (int64_t)w.tiles * w.kt;
            if (w.kt > l->longest) l->longest = w.kt;
            if (l->parts < SharedLoad::kKept) {
                l->part[l->parts].tiles = w.tiles;
                l->part[l->parts].kt = w.kt;
            }
            l->parts += 1;
        }
    });
}

void choose_shared_chunks(const gc_geometry* geo, const gc_batch* b, const gc_shared* s, const PoolKind& pk, gc::SharedSizes* z) {
    const int64_t cus = device_cus(), heads = geo->num_kv_heads;
    SharedLoad l;
    shared_load(b, s, *z, &l);
    int64_t slots = geo->head_dim == 128 ? cus : 2 * cus, big = 0;
    const double small_us = l.small_tiles * heads * (double)(gc::kDecN * geo->head_dim * 2 * (pk.fp8 ? 1 : 2)) / 5.6e6;
    const double big_us = l.steps * heads * 1.4 / cus;
    const bool by_load = small_us > big_us;  // reading the small tiles takes longer than the 128-row ones
    const bool rounds = l.units * heads > slots;
    if (rounds || (small_us < 0.1 * big_us && l.steps * heads >= 2 * cus * kLongSteps)) slots = 2 * cus;
    auto fits = [&](int c) {
        z->chunk = gc::divisor(c);
        big = 0;
        int64_t most = 0;  // items of about the longest chunk
        auto count = [&](int64_t tiles, int kt) {
            const int ns = z->chunk.ceil_of(kt);
            big += tiles * ns;
            if ((int64_t)kt * 3 >= (int64_t)c * 2 * ns) most += tiles * ns;
        };
        if (l.parts <= SharedLoad::kKept)
            for (int i = 0; i < l.parts; ++i) count(l.part[i].tiles, l.part[i].kt);
        else
            for_each_part(b, s, *z, [&](const gc::PartWork& w, bool, bool) {
                if (!w.small && w.tiles > 0) count(w.tiles, w.kt);
            });
        return (l.steps + big * kItemSteps) * heads <= slots * (c + kItemSteps) && (by_load || most * heads <= slots);
    };
    int lo = kMinChunk < l.longest ? kMinChunk : l.longest, hi = l.longest;
    while (lo < hi) {
        const int mid = lo + (hi - lo) / 2;
        if (fits(mid)) hi = mid;
        else lo = mid + 1;
    }
    fits(lo);
    if (rounds) {
        const int third = gc::ceil_div(l.longest, 3), fifth = gc::ceil_div(l.longest, 5);
        const int most = third < 64 ? third : fifth > 64 ? fifth : 64;
        if (lo > most) lo = most;
    }
    if (by_load) {
        const double as_long = 0.7 * small_us / (geo->head_dim == 128 ? 1.4 : 0.75);
        if (as_long > lo) lo = as_long < l.longest ? (int)as_long : l.longest;
    }
    fits(lo);
    if (!rounds && !by_load && slots == 2 * cus && big * heads > slots && big * heads <= slots * 5 / 4) {
        const int before = lo;
        while (big * heads > slots && lo < l.longest && lo * 4 < before * 5) fits(++lo);
        if (big * heads > slots) fits(before);
    }
    int64_t wgs = 2 * cus - big * heads;
    if (wgs < cus) wgs = cus;
    const int64_t waves = gc::shared_rings(pk.fp8) * wgs;
    int64_t run = waves >= heads ? gc::ceil_div64(l.places, waves / heads) : gc::ceil_div64(l.places * heads, waves);
    if (big * heads > cus) run = run * 2 / 3;
    // (long before the upper bound the places are more than a launch takes)
    z->run = gc::divisor((int)std::min<int64_t>(std::max<int64_t>(run, kMinRun), INT32_MAX / 2));
}

gc_status make_shared_plan(const gc_geometry* geo, const gc_batch* b, const gc_shared* s, const gc_plan_options* o,
                           const Shape& sh, const PoolKind& pk, SharedPlan* pl) {
    gc::SharedSizes& z = pl->z;
    z.tq = gc::divisor(gc::tokens_per_tile(sh.group, gc::kBlockM));
    z.chunk = gc::divisor(INT32_MAX / gc::kBlockN);  // whole
    z.tq_small = sh.group <= gc::kDecM ? gc::tokens_per_tile(sh.group, gc::kDecM) : 0;
    choose_groups(geo, b, s, pk, &z);
    pl->any = false;
    for_each_part(b, s, z, [&](const gc::PartWork&, bool shared, bool) { pl->any |= shared; });
    if (!pl->any) return GC_OK;
    if (o != nullptr && o->kv_split_tiles > 0) {
        z.chunk = z.run = gc::divisor(o->kv_split_tiles < (1 << 25) ? o->kv_split_tiles : 1 << 25);
    } else if (o != nullptr && o->kv_split_tiles < 0) {
        int longest = 1;
        for_each_part(b, s, z, [&](const gc::PartWork& w, bool, bool) {
            if (w.small && w.kt + gc::kPieceCost > longest) longest = w.kt + gc::kPieceCost;
        });
        z.run = gc::divisor(longest);
    } else {
        choose_shared_chunks(geo, b, s, pk, &z);
    }
    for_each_part(b, s, z, [&](const gc::PartWork& w, bool shared, bool own) {
        const int64_t items = w.small ? 0 : (int64_t)w.tiles * w.ns;
        pl->big += items;
        if (!own) pl->big_shared += items;
        int& most = own ? pl->max_own : pl->max_shared;
        if (w.ns > most) most = w.ns;
        if (shared || w.ns > 1) pl->big_slots += items;
        pl->parts += w.small;
        pl->places += w.small ? gc::kPieceCost + w.kt : 0;
    });
    if (pl->places > 0) {
        pl->pieces = pl->parts + (pl->places - 1) / z.run.d;
        pl->runs = gc::ceil_div64(pl->places, z.run.d);
    }
    const int64_t most = gc::kMaxWorkgroups / geo->num_kv_heads - 64;
    if (pl->big + pl->pieces > most || pl->places > (int64_t)INT32_MAX - z.run.d ||
        sh.total_tokens * geo->num_q_heads / 8 >= gc::kMaxWorkgroups ||
        gc::shared_merge_workgroups(sh.total_tokens * geo->num_q_heads, geo->head_dim, pl->max_shared + pl->max_own) >
            (int64_t)UINT32_MAX / gc::kCombineThreads)
        return GC_ERR_BAD_SHAPE;
    gc::SharedLayout& l = pl->layout;
    size_t off = 256;  // (the status word leads, as in the plain workspace)
    auto take = [&](size_t bytes) {
        const size_t at = off;
        off = gc::align_up(off + bytes, 256);
        return at;
    };
    const size_t heads = (size_t)geo->num_kv_heads, D = (size_t)geo->head_dim;
    l.reqs_off = take(sizeof(gc::SharedReq) * (size_t)b->batch);
    l.big_off = take(sizeof(gc::SharedItem) * (size_t)pl->big);
    l.small_off = take(sizeof(gc::SharedItem) * (size_t)pl->pieces);
    l.runs_off = take(sizeof(int32_t) * (size_t)pl->runs);
    l.scratch_off = take(sizeof(int32_t) * gc::shared_scratch_ints(b->batch));
    l.big_lse_off = take(sizeof(float) * (size_t)pl->big_slots * heads * gc::kBlockM);
    l.small_lse_off = take(sizeof(float) * (size_t)pl->pieces * heads * gc::kDecM);
    l.big_o_off = take(sizeof(float) * (size_t)pl->big_slots * heads * gc::kBlockM * D);
    l.small_o_off = take(sizeof(float) * (size_t)pl->pieces * heads * gc::kDecM * D);
    l.total = off;
    return GC_OK;
}

// What a plan is made for: a run finds the plan's mark in the workspace or does nothing, so that a workspace
// with another plan, or none, is no list of garbage items. A hash of every length and group (the next step of a
// decoding loop has the same totals, and its items end a key later), the pool kind and what the host chose.
uint64_t shared_mark(const gc_geometry* geo, const gc_batch* b, const gc_shared* s, const PoolKind& pk, const Shape& sh,
                     const SharedPlan& p) {
    uint64_t x = 0xcbf29ce484222325ull;
    auto add = [&](int64_t v) { x = (x ^ (uint64_t)v) * 0x100000001b3ull ^ (x >> 29); };
    auto add2 = [&](int32_t u, int32_t v) { add((int64_t)u << 32 | (uint32_t)v); };
    for (int64_t v : {(int64_t)geo->num_q_heads, (int64_t)geo->num_kv_heads, (int64_t)geo->head_dim,
                      (int64_t)geo->max_blocks_per_seq, (int64_t)b->batch, (int64_t)s->groups, (int64_t)pk.fp8, sh.total_tokens,
                      p.big, p.big_shared, p.big_slots, p.parts, p.places, p.pieces, p.runs, (int64_t)p.z.chunk.d,
                      (int64_t)p.z.run.d, (int64_t)p.layout.total})
        add(v);
    for (uint64_t t : p.z.take) add((int64_t)t);
    add(p.z.all);
    for (int r = 0; r < b->batch; ++r) add2(b->prefix_lens_host[r], b->new_lens_host[r]);
    for (int g = 0; g < s->groups; ++g) add2(s->group_first_host[g], s->shared_lens_host[g]);
    return x != 0 ? x : 1;
}

// Every check that needs no tensors, and the plan. Where no group shares, the plain attention's shape and plan.
gc_status shared_checked(const gc_geometry* geo, const gc_batch* b, const gc_shared* s, const gc_plan_options* o,
                         const PoolKind& pk, Shape* sh, SharedPlan* spl, Plan* pl) {
    gc_status st = check_common(geo, b, sh);
    if (st != GC_OK) return st;
    st = check_options(o);
    if (st != GC_OK) return st;
    if (o != nullptr && o->tiling != GC_TILES_AUTO) return GC_ERR_UNSUPPORTED;
    st = check_shared(geo, b, s);
    if (st != GC_OK || sh->total_tokens == 0) return st;
    if (s->group_first_dev == nullptr || s->shared_lens_dev == nullptr) return GC_ERR_NULL_ARG;
    st = make_shared_plan(geo, b, s, o, *sh, pk, spl);
    if (st != GC_OK && s->policy == GC_SHARE_ALWAYS) return st;
    if (st != GC_OK) spl->any = false;  // more work than its launches hold: the plain attention may take it
    if (!spl->any) return plan_checked(geo, b, o, sh, pl);
    spl->mark = shared_mark(geo, b, s, pk, *sh, *spl);
    return GC_OK;
}

gc_status check_shared_workspace(const SharedPlan& spl, const Plan& pl, const void* ws, size_t bytes) {
    if (!aligned16(ws)) return GC_ERR_WORKSPACE;
    if (!spl.any) return check_workspace(pl, ws, bytes);
    return ws == nullptr || bytes < spl.layout.total ? GC_ERR_WORKSPACE : GC_OK;
}

gc_status enqueue_shared_plan(const gc_geometry* geo, const gc_batch* b, const gc_shared* s, const Shape& sh,
                              const SharedPlan& spl, void* ws, hipStream_t stream) {
    gc::SharedPlanArgs a{};
    a.prefix_lens = b->prefix_lens_dev;
    a.cu_new_lens = b->cu_new_lens_dev;
    a.group_first = s->group_first_dev;
    a.shared_lens = s->shared_lens_dev;
    a.status = at<int32_t>(ws, gc::kStatusOffset);
    a.plan_mark = at<uint64_t>(ws, gc::kMarkOffset);
    a.mark = spl.mark;
    a.scratch = at<int32_t>(ws, spl.layout.scratch_off);
    a.reqs = at<gc::SharedReq>(ws, spl.layout.reqs_off);
    a.big_items = at<gc::SharedItem>(ws, spl.layout.big_off);
    a.small_items = at<gc::SharedItem>(ws, spl.layout.small_off);
    a.batch = b->batch;
    a.groups = s->groups;
    a.total_tokens = (int32_t)sh.total_tokens;
    a.max_blocks = geo->max_blocks_per_seq;
    a.run_first = at<int32_t>(ws, spl.layout.runs_off);
    a.expect_big = (int32_t)spl.big;
    a.expect_big_slots = (int32_t)spl.big_slots;
    a.expect_parts = (int32_t)spl.parts;
    a.expect_places = (int32_t)spl.places;
    a.pieces = (int32_t)spl.pieces;
    a.num_runs = (int32_t)spl.runs;
    a.z = spl.z;
    return gc::launch_shared_plan(a, stream) == hipSuccess ? GC_OK : GC_ERR_HIP;
}

gc_status enqueue_shared_run(const gc_geometry* geo, const gc_batch* b, const Shape& sh, const SharedPlan& spl, const void* q,
                             const void* k_pool, const void* v_pool, float scale, void* out, float* lse,
                             void* ws, hipStream_t stream, const PoolKind& pk) {
    gc::SharedAttnArgs a{};
    a.q = static_cast<const uint16_t*>(q);
    a.k_pool = static_cast<const uint16_t*>(k_pool);
    a.v_pool = static_cast<const uint16_t*>(v_pool);
    a.out = static_cast<uint16_t*>(out);
    a.lse = lse;
    a.part_o = at<float>(ws, spl.layout.big_o_off);
    a.part_lse = at<float>(ws, spl.layout.big_lse_off);
    a.block_tables = b->block_tables_dev;
    a.items = reinterpret_cast<const gc::WorkItem*>(at<gc::SharedItem>(ws, spl.layout.big_off));
    a.num_q_heads = geo->num_q_heads;
    a.num_kv_heads = geo->num_kv_heads;
    a.group = sh.group;
    a.tq = spl.z.tq.d;
    a.num_blocks = geo->num_blocks;
    a.max_blocks = geo->max_blocks_per_seq;
    a.scale_log2 = (float)((double)scale * (double)pk.k_scale * 1.4426950408889634074);
    a.v_scale = pk.v_scale;
    a.small_items = at<gc::SharedItem>(ws, spl.layout.small_off);
    a.small_o = at<float>(ws, spl.layout.small_o_off);
    a.small_lse = at<float>(ws, spl.layout.small_lse_off);
    a.shared_items = (int32_t)spl.big_shared;
    a.own_items = (int32_t)(spl.big - spl.big_shared);
    a.runs = at<int32_t>(ws, spl.layout.runs_off);
    a.small = (int32_t)(spl.runs * geo->num_kv_heads);
    a.pieces = (int32_t)spl.pieces;
    a.plan_mark = at<uint64_t>(ws, gc::kMarkOffset);
    a.mark = spl.mark;
    if (gc::launch_attention_shared(a, geo->head_dim, pk.fp8, stream) != hipSuccess) return GC_ERR_HIP;
    gc::SharedMergeArgs m{};
    m.out = a.out;
    m.lse = lse;
    m.big_o = a.part_o;
    m.big_lse = a.part_lse;
    m.small_o = a.small_o;
    m.small_lse = a.small_lse;
    m.cu_new_lens = b->cu_new_lens_dev;
    m.status = at<int32_t>(ws, gc::kStatusOffset);
    m.plan_mark = a.plan_mark;
    m.mark = a.mark;
    m.reqs = at<gc::SharedReq>(ws, spl.layout.reqs_off);
    m.rows = sh.total_tokens * geo->num_q_heads;
    m.batch = b->batch;
    m.num_kv_heads = geo->num_kv_heads;
    m.single = sh.total_tokens == b->batch && std::all_of(b->new_lens_host, b->new_lens_host + b->batch, [](int32_t n) { return n == 1; });
    m.hq = gc::divisor(geo->num_q_heads);
    m.group = gc::divisor(sh.group);
    m.tq = spl.z.tq;
    return gc::launch_shared_merge(m, geo->head_dim, spl.max_shared + spl.max_own, stream) == hipSuccess ? GC_OK : GC_ERR_HIP;
}

gc_status run_shared(const gc_geometry* geo, const gc_batch* batch, const gc_shared* shared, const gc_plan_options* opts,
                     const void* q, const void* k_pool, const void* v_pool, float scale, void* out, float* lse,
                     void* workspace, size_t workspace_bytes, hipStream_t stream, bool with_plan, const PoolKind& pk) {
    Shape sh;
    SharedPlan spl;
    Plan pl;
    gc_status st = shared_checked(geo, batch, shared, opts, pk, &sh, &spl, &pl);
    if (st != GC_OK || sh.total_tokens == 0) return st;
    st = check_run_args(q, k_pool, v_pool, scale, out);
    if (st != GC_OK) return st;
    if (!aligned16(q) || !aligned16(k_pool) || !aligned16(v_pool) || !aligned16(out)) return GC_ERR_BAD_SHAPE;
    if (pk.fp8) {
        st = check_pool_scales(pk.k_scale, pk.v_scale);
        if (st != GC_OK) return st;
    }
    st = check_shared_workspace(spl, pl, workspace, workspace_bytes);
    if (st != GC_OK) return st;
    if (with_plan) {
        st = spl.any ? enqueue_shared_plan(geo, batch, shared, sh, spl, workspace, stream)
                     : enqueue_plan(geo, batch, sh, pl, workspace, stream);
        if (st != GC_OK) return st;
    }
    return spl.any ? enqueue_shared_run(geo, batch, sh, spl, q, k_pool, v_pool, scale, out, lse, workspace, stream, pk)
                   : enqueue_run(geo, batch, sh, pl, q, k_pool, v_pool, scale, out, lse, workspace, stream, pk);
}

}  // namespace

extern "C" {

__attribute__((visibility("default")))
gc_status gc_kv_append(const gc_geometry* geo, const gc_batch* batch, const void* k_new,
                       const void* v_new, void* k_pool, void* v_pool, hipStream_t stream) {
    return append(geo, batch, k_new, v_new, k_pool, v_pool, PoolKind{}, stream);
}

__attribute__((visibility("default")))
gc_status gc_kv_append_fp8(const gc_geometry* geo, const gc_batch* batch, const void* k_new,
                           const void* v_new, float k_scale, float v_scale, void* k_pool,
                           void* v_pool, hipStream_t stream) {
    const gc_status st = check_pool_scales(k_scale, v_scale);
    if (st != GC_OK) return st;
    return append(geo, batch, k_new, v_new, k_pool, v_pool, PoolKind{true, k_scale, v_scale}, stream);
}

__attribute__((visibility("default")))
gc_status gc_kv_append_rotary(const gc_geometry* geo, const gc_batch* batch, const gc_rotary* rotary,
                              const gc_new_rows* rows, void* q_out, void* k_pool, void* v_pool,
                              hipStream_t stream) {
    return append_rotary(geo, batch, rotary, rows, q_out, k_pool, v_pool, PoolKind{}, stream);
}

__attribute__((visibility("default")))
gc_status gc_kv_append_rotary_fp8(const gc_geometry* geo, const gc_batch* batch, const gc_rotary* rotary,
                                  const gc_new_rows* rows, void* q_out, float k_scale, float v_scale,
                                  void* k_pool, void* v_pool, hipStream_t stream) {
    const gc_status st = check_pool_scales(k_scale, v_scale);
    if (st != GC_OK) return st;
    return append_rotary(geo, batch, rotary, rows, q_out, k_pool, v_pool, PoolKind{true, k_scale, v_scale}, stream);
}

__attribute__((visibility("default")))
gc_status gc_prefix_prefill_workspace_size(const gc_geometry* geo, const gc_batch* batch,
                                           const gc_plan_options* opts, size_t* bytes) {
    if (bytes == nullptr) return GC_ERR_NULL_ARG;
    Shape sh;
    Plan pl;
    gc_status st = plan_checked(geo, batch, opts, &sh, &pl);
    if (st != GC_OK) return st;
    *bytes = sh.total_tokens == 0 ? 0 : pl.layout.total;
    return GC_OK;
}

__attribute__((visibility("default")))
gc_status gc_prefix_prefill_plan(const gc_geometry* geo, const gc_batch* batch,
                                 const gc_plan_options* opts, void* workspace,
                                 size_t workspace_bytes, hipStream_t stream) {
    Shape sh;
    Plan pl;
    gc_status st = plan_checked(geo, batch, opts, &sh, &pl);
    if (st != GC_OK || sh.total_tokens == 0) return st;
    st = check_workspace(pl, workspace, workspace_bytes);
    if (st != GC_OK) return st;
    return enqueue_plan(geo, batch, sh, pl, workspace, stream);
}

__attribute__((visibility("default")))
gc_status gc_prefix_prefill_run(const gc_geometry* geo, const gc_batch* batch,
                                const gc_plan_options* opts, const void* q, const void* k_pool,
                                const void* v_pool, float scale, void* out, float* lse,
                                void* workspace, size_t workspace_bytes, hipStream_t stream) {
    return run(geo, batch, opts, q, k_pool, v_pool, scale, out, lse, workspace, workspace_bytes,
               stream, false, PoolKind{});
}

__attribute__((visibility("default")))
gc_status gc_prefix_prefill_attention(const gc_geometry* geo, const gc_batch* batch,
                                      const gc_plan_options* opts, const void* q,
                                      const void* k_pool, const void* v_pool, float scale,
                                      void* out, float* lse, void* workspace,
                                      size_t workspace_bytes, hipStream_t stream) {
    return run(geo, batch, opts, q, k_pool, v_pool, scale, out, lse, workspace, workspace_bytes,
               stream, true, PoolKind{});
}

__attribute__((visibility("default")))
gc_status gc_prefix_prefill_attention_noalloc(const gc_geometry* geo, const gc_batch* batch,
                                              const gc_plan_options* opts, const void* q,
                                              const void* k_pool, const void* v_pool, float scale,
                                              void* out, float* lse, hipStream_t stream) {
    // every host check first (workspace size included), then the device address
    Shape sh;
    Plan pl;
    gc_status st = plan_checked(geo, batch, opts, &sh, &pl);
    if (st != GC_OK || sh.total_tokens == 0) return st;
    st = check_run_args(q, k_pool, v_pool, scale, out);
    if (st != GC_OK) return st;
    if (pl.layout.total > (size_t)GC_NOALLOC_SCRATCH_BYTES) return GC_ERR_WORKSPACE;
    void* ws = scratch_address(&st);
    if (ws == nullptr) return st;
    return run(geo, batch, opts, q, k_pool, v_pool, scale, out, lse, ws, GC_NOALLOC_SCRATCH_BYTES, stream,
               true, PoolKind{});
}

__attribute__((visibility("default")))
gc_status gc_prefix_prefill_run_with_append(const gc_geometry* geo, const gc_batch* batch,
                                            const gc_plan_options* opts, const void* q, const void* k_new,
                                            const void* v_new, void* k_pool, void* v_pool, float scale,
                                            void* out, float* lse, void* workspace, size_t workspace_bytes,
                                            hipStream_t stream) {
    return run_with_append(geo, batch, opts, q, k_new, v_new, k_pool, v_pool, scale, out, lse, workspace,
                           workspace_bytes, stream);
}

__attribute__((visibility("default")))
gc_status gc_prefix_prefill_run_fp8(const gc_geometry* geo, const gc_batch* batch,
                                    const gc_plan_options* opts, const void* q, const void* k_pool,
                                    const void* v_pool, float k_scale, float v_scale, float scale,
                                    void* out, float* lse, void* workspace, size_t workspace_bytes,
                                    hipStream_t stream) {
    return run(geo, batch, opts, q, k_pool, v_pool, scale, out, lse, workspace, workspace_bytes,
               stream, false, PoolKind{true, k_scale, v_scale});
}

__attribute__((visibility("default")))
gc_status gc_prefix_prefill_attention_fp8(const gc_geometry* geo, const gc_batch* batch,
                                          const gc_plan_options* opts, const void* q,
                                          const void* k_pool, const void* v_pool, float k_scale,
                                          float v_scale, float scale, void* out, float* lse,
                                          void* workspace, size_t workspace_bytes,
                                          hipStream_t stream) {
    return run(geo, batch, opts, q, k_pool, v_pool, scale, out, lse, workspace, workspace_bytes,
               stream, true, PoolKind{true, k_scale, v_scale});
}

__attribute__((visibility("default")))
gc_status gc_prefix_prefill_prepare(const gc_geometry* geo, const gc_batch* batch,
                                    const gc_plan_options* opts, const void* k_new, const void* v_new,
                                    void* k_pool, void* v_pool, void* workspace, size_t workspace_bytes,
                                    hipStream_t stream) {
    return prepare(geo, batch, opts, k_new, v_new, k_pool, v_pool, workspace, workspace_bytes, stream,
                   PoolKind{});
}

__attribute__((visibility("default")))
gc_status gc_prefix_prefill_prepare_fp8(const gc_geometry* geo, const gc_batch* batch,
                                        const gc_plan_options* opts, const void* k_new, const void* v_new,
                                        float k_scale, float v_scale, void* k_pool8, void* v_pool8,
                                        void* workspace, size_t workspace_bytes, hipStream_t stream) {
    return prepare(geo, batch, opts, k_new, v_new, k_pool8, v_pool8, workspace, workspace_bytes, stream,
                   PoolKind{true, k_scale, v_scale});
}

__attribute__((visibility("default")))
gc_status gc_shared_prefix_workspace_size(const gc_geometry* geo, const gc_batch* batch, const gc_shared* shared,
                                          const gc_plan_options* opts, int32_t fp8, size_t* bytes) {
    if (bytes == nullptr) return GC_ERR_NULL_ARG;
    Shape sh;
    SharedPlan spl;
    Plan pl;
    const gc_status st = shared_checked(geo, batch, shared, opts, PoolKind{fp8 != 0}, &sh, &spl, &pl);
    if (st != GC_OK) return st;
    *bytes = sh.total_tokens == 0 ? 0 : spl.any ? spl.layout.total : pl.layout.total;
    return GC_OK;
}

__attribute__((visibility("default")))
gc_status gc_shared_prefix_plan(const gc_geometry* geo, const gc_batch* batch, const gc_shared* shared,
                                const gc_plan_options* opts, int32_t fp8, void* workspace, size_t workspace_bytes,
                                hipStream_t stream) {
    Shape sh;
    SharedPlan spl;
    Plan pl;
    gc_status st = shared_checked(geo, batch, shared, opts, PoolKind{fp8 != 0}, &sh, &spl, &pl);
    if (st != GC_OK || sh.total_tokens == 0) return st;
    st = check_shared_workspace(spl, pl, workspace, workspace_bytes);
    if (st != GC_OK) return st;
    return spl.any ? enqueue_shared_plan(geo, batch, shared, sh, spl, workspace, stream)
                   : enqueue_plan(geo, batch, sh, pl, workspace, stream);
}

__attribute__((visibility("default")))
gc_status gc_shared_prefix_run(const gc_geometry* geo, const gc_batch* batch, const gc_shared* shared,
                               const gc_plan_options* opts, const void* q, const void* k_pool, const void* v_pool,
                               float scale, void* out, float* lse, void* workspace, size_t workspace_bytes,
                               hipStream_t stream) {
    return run_shared(geo, batch, shared, opts, q, k_pool, v_pool, scale, out, lse, workspace, workspace_bytes, stream,
                      false, PoolKind{});
}

__attribute__((visibility("default")))
gc_status gc_shared_prefix_attention(const gc_geometry* geo, const gc_batch* batch, const gc_shared* shared,
                                     const gc_plan_options* opts, const void* q, const void* k_pool, const void* v_pool,
                                     float scale, void* out, float* lse, void* workspace, size_t workspace_bytes,
                                     hipStream_t stream) {
    return run_shared(geo, batch, shared, opts, q, k_pool, v_pool, scale, out, lse, workspace, workspace_bytes, stream,
                      true, PoolKind{});
}

__attribute__((visibility("default")))
gc_status gc_shared_prefix_run_fp8(const gc_geometry* geo, const gc_batch* batch, const gc_shared* shared,
                                   const gc_plan_options* opts, const void* q, const void* k_pool, const void* v_pool,
                                   float k_scale, float v_scale, float scale, void* out, float* lse, void* workspace,
                                   size_t workspace_bytes, hipStream_t stream) {
    return run_shared(geo, batch, shared, opts, q, k_pool, v_pool, scale, out, lse, workspace, workspace_bytes, stream,
                      false, PoolKind{true, k_scale, v_scale});
}

__attribute__((visibility("default")))
gc_status gc_shared_prefix_attention_fp8(const gc_geometry* geo, const gc_batch* batch, const gc_shared* shared,
                                         const gc_plan_options* opts, const void* q, const void* k_pool,
                                         const void* v_pool, float k_scale, float v_scale, float scale, void* out,
                                         float* lse, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    return run_shared(geo, batch, shared, opts, q, k_pool, v_pool, scale, out, lse, workspace, workspace_bytes, stream,
                      true, PoolKind{true, k_scale, v_scale});
}

__attribute__((visibility("default")))
gc_status gc_prefix_prefill_plan_status(const void* workspace, size_t workspace_bytes, hipStream_t stream) {
    if (workspace == nullptr) return GC_ERR_NULL_ARG;
    if (workspace_bytes < sizeof(int32_t)) return GC_ERR_WORKSPACE;
    static_assert(gc::kStatusOffset == 0, "the status word leads the workspace");
    int32_t word = 0;
    if (hipMemcpyAsync(&word, workspace, sizeof(word), hipMemcpyDeviceToHost, stream) != hipSuccess ||
        hipStreamSynchronize(stream) != hipSuccess)
        return GC_ERR_HIP;
    return word == 0 ? GC_OK : GC_ERR_LENGTHS;
}

__attribute__((visibility("default")))
gc_status gc_read_bandwidth_probe(const void* buf, size_t bytes, void* sink, hipStream_t stream) {
    if (buf == nullptr || sink == nullptr) return GC_ERR_NULL_ARG;
    if (bytes % 16 != 0) return GC_ERR_BAD_SHAPE;
    if (bytes == 0) return GC_OK;
    return gc::launch_read_probe(buf, bytes, static_cast<uint32_t*>(sink), stream) == hipSuccess ? GC_OK
                                                                                               : GC_ERR_HIP;
}

__attribute__((visibility("default")))
gc_status gc_mfma_peak_probe(int32_t iterations, void* sink, hipStream_t stream) {
    static_assert(GC_MFMA_PROBE_SINK_FLOATS == gc::kMfmaProbeBlocks * gc::kProbeThreads, "sink size");
    static_assert(GC_MFMA_PROBE_PRODUCTS_PER_ITERATION ==
                      gc::kMfmaProbeBlocks * (gc::kProbeThreads / 64) * gc::kMfmaProbeChains * gc::kMfmaProbePerChain,
                  "products per iteration");
    if (sink == nullptr) return GC_ERR_NULL_ARG;
    if (iterations < 0) return GC_ERR_BAD_SHAPE;
    if (iterations == 0) return GC_OK;
    return gc::launch_mfma_probe(iterations, static_cast<float*>(sink), stream) == hipSuccess ? GC_OK : GC_ERR_HIP;
}

__attribute__((visibility("default")))
const char* gc_status_string(gc_status s) {
    switch (s) {
        case GC_OK: return "GC_OK: success";
        case GC_ERR_NULL_ARG: return "GC_ERR_NULL_ARG: a required pointer is NULL";
        case GC_ERR_BAD_SHAPE: return "GC_ERR_BAD_SHAPE: invalid size, length or scale";
        case GC_ERR_UNSUPPORTED: return "GC_ERR_UNSUPPORTED: head_dim must be 64 or 128, page_size 16, Hq/Hkv <= 128 (<= 16 for small tiles)";
        case GC_ERR_BLOCK_TABLE: return "GC_ERR_BLOCK_TABLE: block table too short for a request";
        case GC_ERR_WORKSPACE: return "GC_ERR_WORKSPACE: workspace missing or too small";
        case GC_ERR_HIP: return "GC_ERR_HIP: a HIP launch failed";
        case GC_ERR_LENGTHS: return "GC_ERR_LENGTHS: the device length arrays disagree with the host's";
    }
    return "unknown gc_status";
}

}  // extern "C"
