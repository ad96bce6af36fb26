// Internal declarations shared by the host library and the gfx950 kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

namespace gc {

// Attention tiling, prefill path: a workgroup of 4 wavefronts owns 128 query
// rows (query heads of one KV head stacked over consecutive new tokens) and
// walks the request's keys in tiles of 64 (four 16-key pool pages).
constexpr int kRowsPerWave = 32;
constexpr int kWaves = 4;
constexpr int kBlockM = kRowsPerWave * kWaves;  // 128
constexpr int kBlockN = 64;
// Small-tile (decode) path: one wavefront owns 16 query rows and walks the keys
// in tiles of 32 (two pages) through an LDS ring of its own.
constexpr int kDecM = 16;
constexpr int kDecN = 32;
constexpr int kPage = 16;
constexpr int64_t kMaxWorkgroups = UINT32_MAX / 512;  // of up to 512 threads, in one launch
constexpr float kLn2 = 0.69314718055994530942f;
constexpr int kAttnThreads = kWaves * 64;
// Wide prefill tiles: 8 wavefronts, 256 query rows per work item (one workgroup
// per CU; every K/V tile copied into LDS feeds twice the rows).
constexpr int kWideWaves = 8;
constexpr int kWideM = kRowsPerWave * kWideWaves;  // 256
constexpr int kPlanThreads = 256;
constexpr int kAppendThreads = 256;
constexpr int kCostBuckets = 2048;  // counting-sort buckets of the work list (cost in tiles)
constexpr int kCombineThreads = 256;  // threads per split-merge workgroup
constexpr int kPlanLdsBatch = 512;    // batches up to this size are planned from LDS copies
constexpr int kProbeBlocks = 2048;    // read-probe grid
constexpr int kProbeThreads = 256;
constexpr int kMfmaProbeBlocks = 1024;   // matrix-core probe grid: four workgroups per CU
constexpr int kMfmaProbeChains = 4;      // independent accumulators per wavefront
constexpr int kMfmaProbePerChain = 4;    // products per accumulator per iteration

// One attention work item: query tile [q0, q0 + tq) of request r against key
// tiles [kt_begin, kt_end). part >= 0 marks a split item whose normalised
// partial output goes to partial slot `part`; -1 writes the output directly.
// r < 0 marks an empty item. P, cu and n repeat the request's prefix length,
// first new row and new-token count, so that one load gives all of an item's
// lengths.
struct WorkItem {
    int32_t r, q0, kt_begin, kt_end, part, P, cu, n;
};

// The same in a shared-prefix launch. Keys (and key tiles) count from page page0 of table row r:
// `keys` of them, of which row t of the tile sees the first P + q0 + t + 1, or all where full is set.
// part < 0: written to the output, else a partial slot of the tile's height. last: the last of a
// wavefront's small items.
struct SharedItem {
    int32_t r, q0, kt_begin, kt_end, part, P, cu, n;
    int32_t page0, keys, full, last;
};

// Keys of an item, its first page in the table row, and whether every row sees all of its keys.
__host__ __device__ inline int item_keys(const WorkItem& it) { return it.P + it.n; }
__host__ __device__ inline int item_keys(const SharedItem& it) { return it.keys; }
__host__ __device__ inline constexpr int item_page0(const WorkItem&) { return 0; }
__host__ __device__ inline int item_page0(const SharedItem& it) { return it.page0; }
__host__ __device__ inline constexpr bool item_full(const WorkItem&) { return false; }
__host__ __device__ inline bool item_full(const SharedItem& it) { return it.full != 0; }

// One query tile whose keys were split: partial slots [part_base, part_base + ns).
struct CombineItem {
    int32_t r, q0, part_base, ns;
};

// ---------------------------------------------------------------- plan math
// Used by the host (grid sizes, workspace) and the planner kernel (the list
// itself); both must agree exactly.

__host__ __device__ inline int ceil_div(int a, int b) { return (a + b - 1) / b; }
__host__ __device__ inline int64_t ceil_div64(int64_t a, int64_t b) { return (a + b - 1) / b; }

// new tokens per query tile of block_m rows for a GQA group of g query heads per KV head
__host__ __device__ inline int tokens_per_tile(int group, int block_m) { return block_m / group; }

__host__ __device__ inline int key_tiles(int prefix, int q0, int ntok, int block_n) {
    return ceil_div(prefix + q0 + ntok, block_n);
}

// number of key chunks of a query tile with kt key tiles; chunk <= 0 means never split
__host__ __device__ inline int num_splits(int kt, int chunk) {
    return (chunk <= 0 || kt <= chunk) ? 1 : ceil_div(kt, chunk);
}

// ---------------------------------------------------------------- shared prefixes
// Work of a shared-prefix launch, derived by the same functions on the host (grid sizes, workspace)
// and in the planner kernel (the list). Every group of requests whose prefix is taken once has one
// shared part: its requests' new tokens, adjacent in the packed order, against the S shared keys, all
// visible. Every request has an own part: its new tokens against its keys from S on, causal.
// (The planner is one workgroup and a chain of such arithmetic: an integer division by a variable, some
// 35 dependent instructions, is three here.)
struct Divisor {
    int d = 1;
    double inv = 1.0;  // fl64(1 / d)
    // a / d, exact for a < 2^32: (a + 1/2) / d is at least 1 / (2 d) from every integer, and its
    // computed value within 2^-20 / d of it.
    __host__ __device__ int of(uint32_t a) const {
#ifdef __HIP_DEVICE_COMPILE__
        return (int)fma((double)a, inv, 0.5 * inv);
#else
        return (int)(a / (uint32_t)d);
#endif
    }
    __host__ __device__ int ceil_of(int a) const { return of((uint32_t)a + (uint32_t)d - 1u); }
};
inline Divisor divisor(int d) { return Divisor{d, 1.0 / d}; }

// a / d for 0 <= a < 2^31, 0 < d < 2^31.
__host__ __device__ inline int quick_div(int a, int d) {
#ifdef __HIP_DEVICE_COMPILE__
    int q = (int)((float)a * __builtin_amdgcn_rcpf((float)d));
    int r = a - q * d;
    while (r < 0) {  // (a step or two where the quotient has more than 22 bits)
        --q;
        r += d;
    }
    while (r >= d) {
        ++q;
        r -= d;
    }
    return q;
#else
    return a / d;
#endif
}

constexpr int kTakeGroups = 512;  // (a batch of more groups takes all or none)
struct SharedSizes {
    Divisor tq;    // new tokens per 128-row query tile
    Divisor chunk; // 64-key tiles per chunk of a 128-row tile
    Divisor run;   // places of one wavefront's run over the small tiles (PartWork)
    int tq_small;  // new tokens per 16-row query tile (0: no small tiles)
    int all;       // every group's shared keys are taken once; else those of the groups in `take`
    uint64_t take[kTakeGroups / 64];
    // shared keys that are taken once for group g, which shares S (words: `take`, or a copy of it)
    __host__ __device__ int taken(int g, int S, const uint64_t* words) const {
        return all || (g < kTakeGroups && (words[g / 64] >> (g % 64) & 1)) ? S : 0;
    }
};

// What one group or request adds to the launch. 128-row tiles: `tiles` query tiles of `ns` key chunks
// each. Small: one query tile of kt key tiles. The small tiles of the batch form one sequence (per KV
// head), groups first, each part kPieceCost places for its start (its loads before the first tile, its
// results) and then its key tiles; wavefront j takes the key tiles at places [j run, (j + 1) run). So a
// part is cut into ns pieces where runs end, and its pieces have numbers of their own: the part's index
// among the small parts plus the run's (numbers in between may be nobody's).
struct PartWork {
    int keys, small, tiles, ns, kt;
};
constexpr int kPieceCost = 4;

// A part of n new tokens against `keys` keys; at: its first place in the sequence.
__host__ __device__ inline PartWork part_work(int keys, int n, int at, const SharedSizes& z) {
    PartWork w{keys, 0, 0, 0, 0};
    if (keys <= 0 || n <= 0) return w;
    w.small = n <= z.tq_small;
    w.tiles = w.small ? 1 : z.tq.ceil_of(n);
    w.kt = ceil_div(keys, w.small ? kDecN : kBlockN);
    w.ns = w.small ? z.run.of((uint32_t)at + kPieceCost + w.kt - 1) - z.run.of((uint32_t)at + kPieceCost) + 1 : z.chunk.ceil_of(w.kt);
    return w;
}
// Number of a small part's first piece; parts: small parts before it.
__host__ __device__ inline int first_piece(int parts, int at, const SharedSizes& z) {
    return parts + z.run.of(at + kPieceCost);
}

// Runs of small items that one workgroup takes: its tile buffers hold that many rings of two small tiles.
__host__ __device__ constexpr int shared_rings(bool fp8) { return fp8 ? 4 : 2; }

// Key tiles [begin, end) of chunk c of ns: the first kt % ns chunks take one more.
__host__ __device__ inline int chunk_begin(int kt, int ns, int c) {
    const int lo = quick_div(kt, ns), more = kt - lo * ns;
    return c * lo + (c < more ? c : more);
}

// What the merge has to know of a request (written by the planner).
struct SharedReq {
    int32_t cu, n, P, merge;              // first row, new tokens, own cached tokens; rows are merged
    int32_t own_small, own_ns, own_slot;  // chunks and first partial slot of its own part
    int32_t g_cu, g_small, g_ns, g_slot;  // the group's: first row, chunks (0: nothing shared), first slot
    int32_t pad[5];
};
static_assert(sizeof(SharedReq) == 64, "four 16-byte loads");

size_t shared_scratch_ints(int batch);  // the planner's scratch, for batches that do not fit its LDS

struct SharedLayout {
    size_t reqs_off, big_off, small_off, runs_off, scratch_off, big_lse_off, big_o_off, small_lse_off, small_o_off, total;
};

// Pool pages that receive new tokens over the batch (the append grid), from the
// host lengths: pages P_r / 16 .. (P_r + n_r - 1) / 16 of every request with n_r > 0.
inline int64_t append_pages_host(const int32_t* prefix, const int32_t* n, int batch) {
    int64_t u = 0;
    for (int r = 0; r < batch; ++r)
        if (n[r] > 0) u += ((int64_t)prefix[r] + n[r] + kPage - 1) / kPage - prefix[r] / kPage;
    return u;
}

// ---------------------------------------------------------------- workspace
constexpr size_t kStatusOffset = 0;  // byte offset of the planner's status word in the workspace
// A shared-prefix plan's mark in that block: a hash of what the plan was made for, never 0. A plain plan
// sets it to 0, since its items lie where a shared plan's records and items were.
constexpr size_t kMarkOffset = 128;
// Work queues of the resident attention launch: kQueues ticket counters and one exit
// counter (int32) in the workspace's leading 256-byte block, zeroed by the planner and
// left at zero by every launch that uses them.
constexpr size_t kQueueOffset = 64;
constexpr int kQueues = 8;  // one per XCD

struct WorkspaceLayout {
    size_t items_off, combine_off, scratch_off, part_lse_off, part_o_off, status_off, queue_off, total;
};

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

inline WorkspaceLayout workspace_layout(int batch, int64_t items, int64_t combines,
                                        int64_t partials, int num_kv_heads, int head_dim, int block_m) {
    WorkspaceLayout w{};
    size_t off = kStatusOffset;
    w.status_off = off;
    w.queue_off = off + kQueueOffset;
    off = align_up(off + 256, 256);
    w.items_off = off;
    off = align_up(off + sizeof(WorkItem) * (size_t)(items > 0 ? items : 1), 256);
    w.combine_off = off;
    off = align_up(off + sizeof(CombineItem) * (size_t)(combines > 0 ? combines : 1), 256);
    w.scratch_off = off;  // 3 int32 per request + 1
    off = align_up(off + sizeof(int32_t) * 3 * (size_t)(batch + 1), 256);
    w.part_lse_off = off;
    off = align_up(off + sizeof(float) * (size_t)partials * num_kv_heads * block_m, 256);
    w.part_o_off = off;
    off = align_up(off + sizeof(float) * (size_t)partials * num_kv_heads * block_m * head_dim, 256);
    w.total = off;
    return w;
}

// ---------------------------------------------------------------- kernel launch arguments
struct AppendArgs {
    const uint16_t* k_new;
    const uint16_t* v_new;
    void* k_pool;        // bf16 elements, or E4M3 codes for 8-bit pools
    void* v_pool;
    const int32_t* prefix_lens;
    const int32_t* cu_new_lens;
    const int32_t* block_tables;
    int32_t batch, total_tokens, num_kv_heads, num_blocks, max_blocks;
    int32_t total_pages;  // pool pages that receive new tokens (host count; the append grid)
    float k_inv, v_inv;  // 8-bit pools: fl32(1 / scale) of each pool
};

// Append with rotation: keys and queries of token rows `stride` elements apart.
struct RotaryArgs {
    AppendArgs a;
    const uint16_t* q;      // may be null: keys and values only
    uint16_t* q_out;        // [T][Hq][D]; may be q
    const float* table;     // [num_positions][rotary_dim / 2][cos, sin]
    int64_t q_stride, k_stride, v_stride;
    int32_t num_q_heads, num_positions, rotary_dim, interleaved;
    uint32_t jobs, by_page;  // workgroups of a page; launched page by page (else head by head)
};

struct PlanArgs {
    const int32_t* prefix_lens;
    const int32_t* cu_new_lens;
    int32_t* scratch;         // 3 * (batch + 1) int32
    WorkItem* items;          // [items], in launch order (see group_cost)
    CombineItem* combines;    // [combines]
    int32_t* status;          // status[0] = 0 when the device lengths matched the host's
    int32_t* queues;          // [kQueues + 1] work-queue counters, zeroed here
    int32_t* shared_mark;     // [2] the mark of a shared-prefix plan that was here before, zeroed here
    int32_t batch, tq, chunk, block_n;
    int32_t expect_items, expect_combines, expect_partials;
    int32_t total_tokens;     // the host's T (= cu_new_lens[batch] on the device)
    int32_t max_blocks;       // row length of the block tables
    // Items of at least group_cost key tiles are sorted by their request's key
    // tiles (so the items of one request stay together), lighter ones by their own
    // cost; kCostBuckets gives the plain cost order.
    int32_t group_cost;
    // Buckets of the counting sort that this batch can use: more than its largest sort
    // key, a multiple of kPlanThreads, at most kCostBuckets (clearing and scanning all
    // 2048 for a batch of short chunks took 0.5-1 of the plan's 5-12 us).
    int32_t buckets;
};

// (Integers first: the order decides how the compiler loads and holds the arguments. With the
// pointers first the wide kernel takes 485 us instead of 476 on 4 x 128 new tokens over 32768.)
struct AttnArgs {
    int32_t num_q_heads, num_kv_heads, group, tq;
    int32_t num_blocks, max_blocks;
    uint32_t prefer_span, prefer_odd;  // 128-row workgroups b with b / span % 2 == odd are preferred
    const uint16_t* q;
    const uint16_t* k_pool;
    const uint16_t* v_pool;
    uint16_t* out;
    float* lse;          // may be null
    float* part_o;       // [partials][Hkv][block_m][D]
    float* part_lse;     // [partials][Hkv][block_m]
    const int32_t* block_tables;
    const WorkItem* items;
    int32_t* queues;     // resident launch: [kQueues] ticket counters, then the exit counter
    float scale_log2;    // softmax scale * log2(e) (times the key scale for 8-bit pools)
    float v_scale;       // value scale of 8-bit pools, 1 for bf16 pools
};

// One launch of both kinds of items: workgroups of 128-row items first (rounded up to whole rounds of
// the XCDs), then workgroups whose wavefronts take one run of small items each.
struct SharedAttnArgs : AttnArgs {  // items: the 128-row items
    const SharedItem* small_items;  // by piece number
    const int32_t* runs;            // [runs] first piece of every run
    float* small_o;                 // [pieces][Hkv][16][D]
    float* small_lse;               // [pieces][Hkv][16]
    int32_t shared_items, own_items;      // 128-row items of either kind, the shared ones first
    int32_t shared_per_xcd, big_wgs;      // workgroups of the shared ones on an XCD; of both kinds
    int32_t small, pieces;          // runs times KV heads; pieces
    const uint64_t* plan_mark;      // what the plan was made for, in the workspace: not `mark`, no work
    uint64_t mark;
};

struct SharedPlanArgs {
    const int32_t* prefix_lens;
    const int32_t* cu_new_lens;
    const int32_t* group_first;   // [groups + 1]
    const int32_t* shared_lens;   // [groups]
    int32_t* status;
    uint64_t* plan_mark;          // receives `mark`
    uint64_t mark;
    int32_t* scratch;             // shared_scratch_ints(batch)
    SharedReq* reqs;
    SharedItem* big_items;
    SharedItem* small_items;
    int32_t* run_first;
    int32_t batch, groups, total_tokens, max_blocks;
    int32_t expect_big, expect_big_slots, expect_parts, expect_places;  // small parts and their places
    int32_t pieces, num_runs;
    SharedSizes z;
};

struct SharedMergeArgs {
    uint16_t* out;
    float* lse;
    const float *big_o, *big_lse, *small_o, *small_lse;
    const int32_t* cu_new_lens;
    const int32_t* status;
    const uint64_t* plan_mark;
    uint64_t mark;
    const SharedReq* reqs;
    int64_t rows;  // T * Hq
    int32_t batch, num_kv_heads;
    int32_t single;  // every request has one new token
    Divisor hq, group, tq;  // query heads; of a KV head; new tokens of a 128-row tile
};

struct CombineArgs {
    uint16_t* out;
    float* lse;
    const float* part_o;
    const float* part_lse;
    const int32_t* cu_new_lens;
    const CombineItem* combines;
    int32_t num_q_heads, num_kv_heads, group, tq;
    int32_t batch, num_partials, block_m;
};

hipError_t launch_append(const AppendArgs& a, int head_dim, bool fp8, hipStream_t s);
hipError_t launch_plan(const PlanArgs& a, hipStream_t s);
hipError_t launch_append_rotary(const RotaryArgs& ra, int head_dim, bool fp8, hipStream_t s);
// workgroups of that launch
int64_t rotary_workgroups(int64_t pages, int num_q_heads, int num_kv_heads, int head_dim, bool with_q);
// append (AppendArgs) and plan (PlanArgs) in one launch
hipError_t launch_prepare(const AppendArgs& aa, const PlanArgs& pa, int head_dim, bool fp8, hipStream_t s);
// resident > 0 (wide tiles only): that many resident workgroups take
// the items from the work queues instead of one workgroup per item
// (three: the 128-row kernel of three workgroups per compute unit over 8-bit pools at d = 64)
hipError_t launch_attention(const AttnArgs& a, int head_dim, int64_t num_items, bool wide, bool three, bool fp8,
                            int resident, hipStream_t s);
// the same over 8-bit pools (launch_attention forwards fp8 launches here)
hipError_t launch_attention_fp8(const AttnArgs& a, int head_dim, int64_t num_items, bool wide, bool three,
                                int resident, hipStream_t s);
hipError_t launch_attention_small(const AttnArgs& a, int head_dim, int64_t num_items, bool fp8,
                                  hipStream_t s);
hipError_t launch_read_probe(const void* buf, size_t bytes, uint32_t* sink, hipStream_t s);
hipError_t launch_mfma_probe(int iterations, float* sink, hipStream_t s);
hipError_t launch_shared_plan(const SharedPlanArgs& a, hipStream_t s);
hipError_t launch_attention_shared(const SharedAttnArgs& a, int head_dim, bool fp8, hipStream_t s);
// max_chunks: the most chunks of any row
int64_t shared_merge_workgroups(int64_t rows, int head_dim, int max_chunks);  // at most UINT32_MAX / kCombineThreads
hipError_t launch_shared_merge(const SharedMergeArgs& a, int head_dim, int max_chunks, hipStream_t s);
// max_splits: the most key chunks of any split query tile
hipError_t launch_combine(const CombineArgs& a, int head_dim, int64_t num_combines, int max_splits, hipStream_t s);

}  // namespace gc
