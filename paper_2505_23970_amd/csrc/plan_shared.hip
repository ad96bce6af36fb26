// Work lists of the shared-prefix attention, built on the device from the device copies of the lengths
// (no host-to-device copy, so a plan can be enqueued freely and captured in a graph). One workgroup:
//   1. the device lengths are checked before anything is derived from them;
//   2. scans over groups and then requests give each its items, partial slots and pieces, and every
//      request its record for the merge (which groups' shared keys are taken once, the host says);
//   3. every item, found from its index by a search of the scans.
// What bounds it is the chain of these steps, each a barrier and some reads of what the one before wrote:
// up to kPlanLdsBatch requests all of it stays in LDS.
// 128-row items of a shared part are ordered chunk by chunk, so that the query tiles that read one chunk
// of keys run side by side and share it in L2; a request's own query tiles longest first. Small items
// are pieces of one sequence, cut into equal runs (PartWork).
// Where the device lengths disagree with the host's, every item is emitted empty and status[0] set.
#include "gc_internal.h"

namespace gc {
namespace {

struct Quad {
    int x[4];
};
// (200 requests with 700 small pieces 7.6 us, 9.8 with 256 threads; fewer pieces the same)
constexpr int kSharedPlanThreads = 1024;
enum { kBigItems, kBigSlots, kParts, kPlaces };  // kParts, kPlaces: small parts and their places

// Inclusive scan over a wavefront: within rows of 16 lanes, then the rows' totals passed on (as lane
// exchanges in the additions themselves: a sixth of the time of exchanges through the LDS unit).
__device__ __forceinline__ int wave_scan(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);  // row_shr:1
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);  // row_shr:2
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);  // row_shr:4
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);  // row_shr:8
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15 into rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31 into rows 2 and 3
    return x;
}

// Exclusive scan of four values per thread over the workgroup, from `base`; base receives the totals on
// top. Values behind the first `waves` wavefronts are 0. (Each call has its own tmp, so that one barrier does.)
__device__ __forceinline__ Quad block_scan4(const Quad v, Quad (&tmp)[kSharedPlanThreads / 64], const int waves, Quad& base) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Quad s = v;
#pragma unroll
    for (int k = 0; k < 4; ++k) s.x[k] = wave_scan(s.x[k]);
    if (lane == 63) tmp[wave] = s;
    __syncthreads();
    Quad at = base;
#pragma nounroll
    for (int w = 0; w < waves; ++w)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int t = tmp[w].x[k];
            if (w < wave) at.x[k] += t;
            base.x[k] += t;
        }
#pragma unroll
    for (int k = 0; k < 4; ++k) at.x[k] += s.x[k] - v.x[k];
    return at;
}

__device__ __forceinline__ void add_part(Quad& q, const PartWork& w, bool slots) {
    const int n = w.small ? 0 : w.tiles * w.ns;
    q.x[kBigItems] += n;
    q.x[kBigSlots] += slots ? n : 0;
    q.x[kParts] += w.small;
    q.x[kPlaces] += w.small ? kPieceCost + w.kt : 0;
}

// largest i with a[i] <= v, in [0, n)
__device__ __forceinline__ int last_at_most(const int* a, int n, int v) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a[mid] <= v) lo = mid;
        else hi = mid;
    }
    return lo;
}

constexpr int kPlanArrays = 9;  // int32 per request of what the planner derives

template <int BATCH>
struct SharedPlanLds {
    Quad tmp[2][kSharedPlanThreads / 64];
    int bad, wave_bad[kSharedPlanThreads / 64];
    uint64_t take[kTakeGroups / 64];
    int cu[BATCH + 1], pre[BATCH + 1], first[BATCH + 1], share[BATCH + 1];
    int derived[kPlanArrays][BATCH + 1];
};

// LDS: batches of up to kPlanLdsBatch requests. (Pointers that may be either make every access a flat one:
// with one kernel for both the plan of 64 requests took 9.4 us instead of 8.7, before the scans changed.)
template <bool LDS>
__global__ __launch_bounds__(kSharedPlanThreads) void shared_plan_kernel(const SharedPlanArgs a) {
    __shared__ SharedPlanLds<LDS ? kPlanLdsBatch : 1> sm;
    const int tid = threadIdx.x, B = a.batch, G = a.groups;
    const SharedSizes& z = a.z;
    auto derived = [&](int k) -> int* {
        if constexpr (LDS) return sm.derived[k];
        else return a.scratch + (size_t)k * (B + 1);
    };
    auto either = [](int* in_lds, const int* global) -> const int* {
        if constexpr (LDS) return in_lds;
        else return global;
    };
    int* const group_of = derived(0);  // [B]
    int* const r_big = derived(1);     // [B] own 128-row items before it (after all shared ones)
    int* const r_slot = derived(2);    // [B] its first partial slot, of 128 rows
    int* const r_piece = derived(3);   // [B] number of its first piece, if it were small
    int* const r_at = derived(4);      // [B] its first place, if it were small
    int* const g_big = derived(5);     // [G] the same of the groups' shared parts
    int* const g_piece = derived(6);
    int* const g_at = derived(7);
    int* const g_taken = derived(8);   // [G] shared keys that are taken once
    const int* const cu = either(sm.cu, a.cu_new_lens);
    const int* const pre = either(sm.pre, a.prefix_lens);
    const int* const first = either(sm.first, a.group_first);
    const int* const share = either(sm.share, a.shared_lens);

    auto empty_all = [&] {
        const SharedItem none{-1, 0, 0, 0, -1, 0, 0, 0, 0, 0, 0, 1};
        for (int i = tid; i < a.expect_big; i += kSharedPlanThreads) a.big_items[i] = none;
        for (int i = tid; i < a.pieces; i += kSharedPlanThreads) a.small_items[i] = none;
        for (int i = tid; i < a.num_runs; i += kSharedPlanThreads) a.run_first[i] = 0;
        if (tid == 0) a.status[0] = 1;
    };

    // 1. the lengths must describe the batch the host checked (up to kPlanLdsBatch requests they go to LDS on the way)
    // (from LDS: indexed by a lane's group, the arguments would be copied to private memory first, 1.0 us)
    if (tid < kTakeGroups / 64) sm.take[tid] = z.take[tid];
    if (tid == 0) {
        sm.bad = 0;
        *a.plan_mark = a.mark;
    }
    {
        bool bad = false;
#pragma nounroll
        for (int r = tid; r <= B; r += kSharedPlanThreads) {  // (and group r: 1 <= G <= B)
            // (all loads before the first use: one round trip)
            const int c = a.cu_new_lens[r], next = a.cu_new_lens[min(r + 1, B)], P = a.prefix_lens[min(r, B - 1)];
            const int f = a.group_first[min(r, G)], f_next = a.group_first[min(r + 1, G)], S = a.shared_lens[min(r, G - 1)];
            const uint32_t n = (uint32_t)next - (uint32_t)c, keys = (uint32_t)P + n;
            bad |= (r == 0 && c != 0) || (r == B && c != a.total_tokens) || (r == 0 && f != 0) || (r == G && f != B);
            bad |= r < B && (P < 0 || c < 0 || next < c || keys > (uint32_t)(INT32_MAX - kBlockN) ||
                             (n > 0 && (keys + kPage - 1) / kPage > (uint32_t)a.max_blocks));
            bad |= r < G && (S < 0 || S % kPage != 0 || S / kPage > a.max_blocks || f < 0 || f_next <= f || f_next > B);
            if constexpr (LDS) {
                sm.cu[r] = c;
                if (r < B) sm.pre[r] = P;
                if (r <= G) sm.first[r] = f;
                if (r < G) sm.share[r] = S;
            }
        }
        const int any = __any(bad);
        if ((tid & 63) == 0) sm.wave_bad[tid / 64] = any;
    }
    __syncthreads();
    int bad = 0;
#pragma unroll
    for (int w = 0; w < kSharedPlanThreads / 64; ++w) bad |= sm.wave_bad[w];
    if (bad) return empty_all();

    // 2. (A thread owns consecutive requests, and groups.)
    const int per = ceil_div(B, kSharedPlanThreads), r0 = min(B, tid * per), r1 = min(B, r0 + per);
    const int per_g = ceil_div(G, kSharedPlanThreads), g0 = min(G, tid * per_g), g1 = min(G, g0 + per_g);
    auto tokens_of = [&](int g) { return cu[first[g + 1]] - cu[first[g]]; };

    //    groups: what each shares, its items, slots and pieces
    Quad total{{0, 0, 0, 0}};
    {
        Quad v{{0, 0, 0, 0}};
#pragma nounroll
        for (int g = g0; g < g1; ++g) {
            const int S = z.taken(g, share[g], sm.take);
            g_taken[g] = S;
            add_part(v, part_work(S, tokens_of(g), 0, z), true);
        }
        Quad at = block_scan4(v, sm.tmp[0], ceil_div(G, 64 * per_g), total);
#pragma nounroll
        for (int g = g0; g < g1; ++g) {
            g_big[g] = at.x[kBigItems];  // (and its first slot: every shared item has one)
            g_piece[g] = first_piece(at.x[kParts], at.x[kPlaces], z);
            g_at[g] = at.x[kPlaces];
            add_part(at, part_work(g_taken[g], tokens_of(g), 0, z), true);
        }
    }
    const Quad shared_total = total;
    __threadfence_block();
    __syncthreads();

    //    requests: own items, slots and pieces, and the record for the merge
    {
        // (a small part alone is merged where runs cut it, which its place in the sequence decides; only
        // 128-row parts have slots counted here)
        Quad v{{0, 0, 0, 0}};
#pragma nounroll
        for (int r = r0; r < r1; ++r) {
            const int g = last_at_most(first, G, r), S = g_taken[g];
            group_of[r] = g;
            if (pre[r] < share[g]) sm.bad = 1;
            const PartWork w = part_work(pre[r] - S + cu[r + 1] - cu[r], cu[r + 1] - cu[r], 0, z);
            add_part(v, w, S > 0 || w.ns > 1);
        }
        Quad at = block_scan4(v, sm.tmp[1], ceil_div(B, 64 * per), total);
#pragma nounroll
        for (int r = r0; r < r1; ++r) {
            const int g = group_of[r], S = g_taken[g], n = cu[r + 1] - cu[r];
            const PartWork sw = part_work(S, tokens_of(g), g_at[g], z);
            const PartWork w = part_work(pre[r] - S + n, n, at.x[kPlaces], z);
            const int piece = first_piece(at.x[kParts], at.x[kPlaces], z);
            SharedReq q{};
            q.cu = cu[r];
            q.n = n;
            q.P = pre[r] - S;
            q.merge = S > 0 || w.ns > 1;
            q.own_small = w.small;
            q.own_ns = w.ns;
            q.own_slot = w.small ? piece : at.x[kBigSlots];
            q.g_cu = cu[first[g]];
            q.g_small = sw.small;
            q.g_ns = sw.ns;
            q.g_slot = sw.small ? g_piece[g] : g_big[g];
            a.reqs[r] = q;
            r_big[r] = at.x[kBigItems] - shared_total.x[kBigItems];
            r_slot[r] = at.x[kBigSlots];
            r_piece[r] = piece;
            r_at[r] = at.x[kPlaces];
            add_part(at, w, q.merge);
        }
    }
    if (sm.bad || total.x[kBigItems] != a.expect_big || total.x[kBigSlots] != a.expect_big_slots || total.x[kParts] != a.expect_parts ||
        total.x[kPlaces] != a.expect_places)
        return empty_all();
    __threadfence_block();
    __syncthreads();

    // 3. items (positions are in range when the totals agree; never write outside all the same)
#pragma nounroll
    for (int i = tid; i < a.expect_big; i += kSharedPlanThreads) {
        SharedItem it;
        if (i < shared_total.x[kBigItems]) {
            const int g = last_at_most(g_big, G, i), S = g_taken[g], tokens = tokens_of(g);
            const PartWork w = part_work(S, tokens, 0, z);
            if (w.tiles <= 0) continue;  // (not reached: the group has items)
            const int local = i - g_big[g], c = quick_div(local, w.tiles), tile = local - c * w.tiles;
            it = SharedItem{first[g], tile * z.tq.d, chunk_begin(w.kt, w.ns, c), chunk_begin(w.kt, w.ns, c + 1), g_big[g] + tile * w.ns + c,
                            0, cu[first[g]], tokens, 0, S, 1, 0};
        } else {
            const int own = i - shared_total.x[kBigItems], r = last_at_most(r_big, B, own), S = g_taken[group_of[r]];
            const int P = pre[r] - S, n = cu[r + 1] - cu[r];
            const PartWork w = part_work(P + n, n, 0, z);
            if (w.ns <= 0) continue;  // (not reached)
            const int local = own - r_big[r], t = quick_div(local, w.ns), c = local - t * w.ns;
            const int tile = w.tiles - 1 - t, q0 = tile * z.tq.d;
            const int kt = key_tiles(P, q0, min(z.tq.d, n - q0), kBlockN), ns = min(w.ns, kt);
            it = SharedItem{r, q0, 0, 0, S > 0 || w.ns > 1 ? r_slot[r] + tile * w.ns + c : -1, P, cu[r], n, S / kPage, w.keys, 0, 0};
            if (c < ns) {
                it.kt_begin = chunk_begin(kt, ns, c);
                it.kt_end = chunk_begin(kt, ns, c + 1);
            } else {
                it.r = -1;
            }
        }
        if (it.part >= a.expect_big_slots) it.r = -1;
        a.big_items[i] = it;
    }
    for (int i = tid; i < a.num_runs; i += kSharedPlanThreads) a.run_first[i] = -1;  // (a run may hold no key tile)
    __syncthreads();
    const int shared_pieces = shared_total.x[kParts] > 0 ? first_piece(shared_total.x[kParts], shared_total.x[kPlaces], z) : 0;
#pragma nounroll
    for (int i = tid; i < a.pieces; i += kSharedPlanThreads) {
        // the last part whose first piece is at most i (a number may be nobody's)
        const bool shared = i < shared_pieces;
        const int o = shared ? last_at_most(g_piece, G, i) : last_at_most(r_piece, B, i);
        const int g = shared ? o : group_of[o], S = g_taken[g];
        const int n = shared ? tokens_of(g) : cu[o + 1] - cu[o], P = shared ? 0 : pre[o] - S;
        const int at = shared ? g_at[o] : r_at[o];
        const PartWork w = part_work(shared ? S : P + n, n, at, z);
        const int c = i - (shared ? g_piece[o] : r_piece[o]);
        if (!w.small || c < 0 || c >= w.ns) continue;
        const int run = z.run.of(at + kPieceCost) + c;
        // key tiles of the run, from the part's first one
        const int64_t begin = (int64_t)run * z.run.d - at - kPieceCost, end = begin + z.run.d;
        // the run ends with this piece: the part goes on in the next, or the next part's first tile lies there
        const int64_t next = (int64_t)at + kPieceCost + w.kt;
        const bool last = c + 1 < w.ns || next >= a.expect_places || z.run.of(next + kPieceCost) != run;
        SharedItem it{shared ? first[g] : o, 0, (int)max(begin, (int64_t)0), (int)min(end, (int64_t)w.kt), i, P, shared ? cu[first[g]] : cu[o], n,
                      shared ? 0 : S / kPage, w.keys, shared, last};
        if (!shared && S == 0 && w.ns == 1) it.part = -1;
        a.small_items[i] = it;
        // the run's first piece: the part began in an earlier run, or the part before ended in one
        const bool begins = c > 0 || at == 0 || z.run.of(at - 1) != run;
        if (begins && run < a.num_runs) a.run_first[run] = i;
    }
    if (tid == 0) a.status[0] = 0;
}

}  // namespace

size_t shared_scratch_ints(int batch) { return batch <= kPlanLdsBatch ? 1 : (size_t)kPlanArrays * ((size_t)batch + 1); }

hipError_t launch_shared_plan(const SharedPlanArgs& a, hipStream_t s) {
    if (a.batch <= kPlanLdsBatch)
        shared_plan_kernel<true><<<1, kSharedPlanThreads, 0, s>>>(a);
    else
        shared_plan_kernel<false><<<1, kSharedPlanThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace gc
