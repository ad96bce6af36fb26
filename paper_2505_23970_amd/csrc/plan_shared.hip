// Work lists of the shared-prefix attention, built on the device from the device copies of the lengths
// (no host-to-device copy, so a plan can be enqueued freely and captured in a graph). One workgroup:
//   1. the device lengths are checked before anything is derived from them;
//   2. per-request prefix sums (requests with new tokens, own 128-row query tiles) give every group its
//      rows and whether its shared keys are taken once; scans over groups and then requests give each
//      its items and partial slots;
//   3. every request's record for the merge; every item, found from its index by a search of the scans.
// Items of a shared part are ordered chunk by chunk, so that the query tiles that read one chunk of keys
// run side by side and share it in L2; a request's own query tiles longest first.
// Where the device lengths disagree with the host's, every item is emitted empty and status[0] set.
#include "gc_internal.h"

namespace gc {
namespace {

struct Quad {
    int x[4];
};
enum { kBigItems, kSmallItems, kBigSlots, kSmallSlots };

// Exclusive scan of four values per thread over the workgroup, from `base`; base receives the totals on top.
__device__ Quad block_scan4(const Quad v, Quad (&tmp)[kPlanThreads / 64], Quad& base) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Quad s = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int y = __shfl_up(s.x[k], d);
            if (lane >= d) s.x[k] += y;
        }
    if (lane == 63) tmp[wave] = s;
    __syncthreads();
    Quad at = base;
#pragma unroll
    for (int w = 0; w < kPlanThreads / 64; ++w)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (w < wave) at.x[k] += tmp[w].x[k];
            base.x[k] += tmp[w].x[k];
        }
    __syncthreads();  // tmp is reused
#pragma unroll
    for (int k = 0; k < 4; ++k) at.x[k] += s.x[k] - v.x[k];
    return at;
}

__device__ __forceinline__ Quad quad_of(const PartWork& w, bool slots) {
    Quad q{{0, 0, 0, 0}};
    q.x[w.small ? kSmallItems : kBigItems] = w.items();
    if (slots) q.x[w.small ? kSmallSlots : kBigSlots] = w.items();
    return q;
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

struct SharedPlanLds {
    Quad tmp[kPlanThreads / 64];
    int bad;
    int cu[kPlanLdsBatch + 1], pre[kPlanLdsBatch], first[kPlanLdsBatch + 1], share[kPlanLdsBatch];
    int active[kPlanLdsBatch + 1], tiles[kPlanLdsBatch + 1], r_items[kPlanLdsBatch + 1], g_items[kPlanLdsBatch + 1];
};

// A group's record while the plan is made (kept in the workspace behind the requests' scratch).
struct GroupRec {
    int taken, r, cu, tokens, slot, big, small_, ns;  // big, small_: position of its first item of that kind
};

__global__ __launch_bounds__(kPlanThreads) void shared_plan_kernel(const SharedPlanArgs a) {
    __shared__ SharedPlanLds sm;
    const int tid = threadIdx.x, B = a.batch, G = a.groups;
    const bool lds = B <= kPlanLdsBatch;  // (G <= B)
    int* const s = a.scratch;
    int* const active = lds ? sm.active : s;
    int* const tiles = lds ? sm.tiles : s + (B + 1);
    int* const r_items = lds ? sm.r_items : s + 2 * (B + 1);
    int* const g_items = lds ? sm.g_items : s + 3 * (B + 1);
    GroupRec* const groups = reinterpret_cast<GroupRec*>(s + 4 * (B + 1));
    int* const r_at = s + 4 * (B + 1) + 8 * B;  // position of a request's first own item of its kind
    if (tid == 0) sm.bad = 0;
    if (lds) {
        for (int r = tid; r <= B; r += kPlanThreads) {
            sm.cu[r] = a.cu_new_lens[r];
            if (r < B) sm.pre[r] = a.prefix_lens[r];
            if (r <= G) sm.first[r] = a.group_first[r];
            if (r < G) sm.share[r] = a.shared_lens[r];
        }
    }
    __syncthreads();
    const int* const cu = lds ? sm.cu : a.cu_new_lens;
    const int* const pre = lds ? sm.pre : a.prefix_lens;
    const int* const first = lds ? sm.first : a.group_first;
    const int* const share = lds ? sm.share : a.shared_lens;

    auto empty_all = [&] {
        const SharedItem none{-1, 0, 0, 0, -1, 0, 0, 0, 0, 0, 0, 0};
        for (int i = tid; i < a.expect_big; i += kPlanThreads) a.big_items[i] = none;
        for (int i = tid; i < a.expect_small; i += kPlanThreads) a.small_items[i] = none;
        if (tid == 0) a.status[0] = 1;
    };

    // 1. the lengths must describe the batch the host checked
    {
        bool bad = tid == 0 && (cu[0] != 0 || cu[B] != a.total_tokens || first[0] != 0 || first[G] != B);
        for (int r = tid; r < B; r += kPlanThreads) {
            const int64_t P = pre[r], n = (int64_t)cu[r + 1] - cu[r];
            bad |= P < 0 || n < 0 || P + n > (int64_t)INT32_MAX - kBlockN || (n > 0 && ceil_div64(P + n, kPage) > a.max_blocks);
        }
        for (int g = tid; g < G; g += kPlanThreads) {
            const int S = share[g];
            bad |= S < 0 || S % kPage != 0 || S / kPage > a.max_blocks || first[g] < 0 || first[g + 1] <= first[g] || first[g + 1] > B;
        }
        if (bad) sm.bad = 1;
    }
    __syncthreads();
    if (sm.bad) return empty_all();
    {
        bool bad = false;  // (in a pass of its own: group bounds are known to be good)
        for (int r = tid; r < B; r += kPlanThreads) bad |= pre[r] < share[last_at_most(first, G, r)];
        if (bad) sm.bad = 1;
    }
    __syncthreads();
    if (sm.bad) return empty_all();

    // 2. prefix sums over requests: those with new tokens, and own 128-row tiles
    const int per = ceil_div(B, kPlanThreads), r0 = min(B, tid * per), r1 = min(B, r0 + per);
    {
        Quad v{{0, 0, 0, 0}}, total{{0, 0, 0, 0}};
        for (int r = r0; r < r1; ++r) {
            const int n = cu[r + 1] - cu[r];
            v.x[0] += n > 0;
            v.x[1] += ceil_div(n, a.z.tq);
        }
        Quad at = block_scan4(v, sm.tmp, total);
        for (int r = r0; r < r1; ++r) {
            const int n = cu[r + 1] - cu[r];
            active[r] = at.x[0];
            tiles[r] = at.x[1];
            at.x[0] += n > 0;
            at.x[1] += ceil_div(n, a.z.tq);
        }
        if (tid == 0) {
            active[B] = total.x[0];
            tiles[B] = total.x[1];
        }
    }
    __threadfence_block();
    __syncthreads();

    //    groups: what each shares, its items and slots
    Quad total{{0, 0, 0, 0}};
    auto taken_of = [&](int g, int& tokens) {
        const int ra = first[g], rb = first[g + 1];
        tokens = cu[rb] - cu[ra];
        return shared_taken(share[g], active[rb] - active[ra], tokens, tiles[rb] - tiles[ra], a.z);
    };
    const int per_g = ceil_div(G, kPlanThreads), g0 = min(G, tid * per_g), g1 = min(G, g0 + per_g);
    {
        Quad v{{0, 0, 0, 0}};
        for (int g = g0; g < g1; ++g) {
            int tokens;
            const int S = taken_of(g, tokens);
            const Quad q = quad_of(shared_part(S, tokens, a.z), true);
            for (int k = 0; k < 4; ++k) v.x[k] += q.x[k];
        }
        Quad at = block_scan4(v, sm.tmp, total);
        for (int g = g0; g < g1; ++g) {
            int tokens;
            const int S = taken_of(g, tokens);
            const PartWork w = shared_part(S, tokens, a.z);
            groups[g] = GroupRec{S, first[g], cu[first[g]], tokens, at.x[w.small ? kSmallSlots : kBigSlots], at.x[kBigItems], at.x[kSmallItems], w.ns};
            g_items[g] = at.x[kBigItems] + at.x[kSmallItems];
            const Quad q = quad_of(w, true);
            for (int k = 0; k < 4; ++k) at.x[k] += q.x[k];
        }
    }
    const int shared_items = total.x[kBigItems] + total.x[kSmallItems];
    __threadfence_block();
    __syncthreads();

    //    requests: own items and slots, and the record for the merge
    {
        Quad v{{0, 0, 0, 0}};
        for (int r = r0; r < r1; ++r) {
            const int S = groups[last_at_most(first, G, r)].taken;
            const PartWork w = own_part(pre[r] - S, cu[r + 1] - cu[r], a.z);
            const Quad q = quad_of(w, S > 0 || w.ns > 1);
            for (int k = 0; k < 4; ++k) v.x[k] += q.x[k];
        }
        Quad at = block_scan4(v, sm.tmp, total);
        for (int r = r0; r < r1; ++r) {
            const GroupRec g = groups[last_at_most(first, G, r)];
            const PartWork sw = shared_part(g.taken, g.tokens, a.z);
            const int n = cu[r + 1] - cu[r];
            const PartWork w = own_part(pre[r] - g.taken, n, a.z);
            const bool merge = g.taken > 0 || w.ns > 1;
            SharedReq q{};
            q.cu = cu[r];
            q.n = n;
            q.P = pre[r] - g.taken;
            q.merge = merge;
            q.own_small = w.small;
            q.own_ns = w.ns;
            q.own_slot = at.x[w.small ? kSmallSlots : kBigSlots];
            q.g_cu = g.cu;
            q.g_small = sw.small;
            q.g_ns = g.taken > 0 ? sw.ns : 0;
            q.g_slot = g.slot;
            a.reqs[r] = q;
            r_at[r] = at.x[w.small ? kSmallItems : kBigItems];
            r_items[r] = at.x[kBigItems] + at.x[kSmallItems] - shared_items;
            const Quad add = quad_of(w, merge);
            for (int k = 0; k < 4; ++k) at.x[k] += add.x[k];
        }
    }
    const int own_items = total.x[kBigItems] + total.x[kSmallItems] - shared_items;
    __threadfence_block();
    __syncthreads();
    if (total.x[kBigItems] != a.expect_big || total.x[kSmallItems] != a.expect_small ||
        total.x[kBigSlots] != a.expect_big_slots || total.x[kSmallSlots] != a.expect_small_slots)
        return empty_all();

    // 3. items (positions and slots are in range when the totals agree; never write outside all the same)
    auto put = [&](bool small, int pos, SharedItem it) {
        const int most = small ? a.expect_small : a.expect_big, slots = small ? a.expect_small_slots : a.expect_big_slots;
        if (pos < 0 || pos >= most) return;
        if (it.part >= slots) it.r = -1;
        (small ? a.small_items : a.big_items)[pos] = it;
    };
    for (int i = tid; i < shared_items; i += kPlanThreads) {
        const int g = last_at_most(g_items, G, i);
        const GroupRec q = groups[g];
        const PartWork w = shared_part(q.taken, q.tokens, a.z);
        if (w.tiles <= 0) continue;
        const int local = i - g_items[g], c = local / w.tiles, tile = local - c * w.tiles;
        const int kt = ceil_div(q.taken, w.small ? kDecN : kBlockN);
        put(w.small, (w.small ? q.small_ : q.big) + local,
            SharedItem{q.r, tile * a.z.tq, chunk_begin(kt, w.ns, c), chunk_begin(kt, w.ns, c + 1), q.slot + tile * w.ns + c, 0,
                       q.cu, q.tokens, 0, q.taken, 1, 0});
    }
    for (int i = tid; i < own_items; i += kPlanThreads) {
        const int r = last_at_most(r_items, B, i);
        const SharedReq q = a.reqs[r];
        const PartWork w = own_part(q.P, q.n, a.z);
        if (w.tiles <= 0) continue;
        const int local = i - r_items[r], c = local % w.ns, tile = w.tiles - 1 - local / w.ns;
        const int q0 = tile * a.z.tq;
        const int kt = w.small ? ceil_div(w.keys, kDecN) : key_tiles(q.P, q0, min(a.z.tq, q.n - q0), kBlockN);
        const int ns = min(w.ns, kt);
        SharedItem it{r, q0, 0, 0, q.merge ? q.own_slot + tile * w.ns + c : -1, q.P, q.cu, q.n, (pre[r] - q.P) / kPage, w.keys, 0, 0};
        if (c < ns) {
            it.kt_begin = chunk_begin(kt, ns, c);
            it.kt_end = chunk_begin(kt, ns, c + 1);
        } else {
            it.r = -1;
        }
        put(w.small, r_at[r] + local, it);
    }
    if (tid == 0) a.status[0] = 0;
}

}  // namespace

hipError_t launch_shared_plan(const SharedPlanArgs& a, hipStream_t s) {
    shared_plan_kernel<<<1, kPlanThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace gc
