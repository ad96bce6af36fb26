// Attention of a batch whose requests share long prefixes (GreenCache §2.2: many requests reuse one
// context, a system prompt or a document): the shared keys and values are read once for all of a
// group's queries.
//
// Mathematics. A row's softmax over its keys is joined from two sets, the S keys that its group shares
// and its own (the rest of its cached prefix and its new tokens): with the partial outputs o_c and
// log-sum-exps l_c of any split of the keys into chunks c,
//     m = max_c l_c,   o = sum_c exp(l_c - m) o_c / sum_c exp(l_c - m),   lse = m + ln sum_c exp(l_c - m),
// so the shared set may be computed for all rows of the group at once: rows of other requests are
// further rows of the same matrix products, with no mask.
//
// Rounding. As everywhere in this framework the weights enter the second product as bf16, the row sums (fp32) add the
// rounded ones, partial rows and log-sum-exps are fp32. 128-row items keep the offset of a row's first tile
// (attention_kernels.h), so that its heaviest weight is rounded too, where the plain attention of single tokens
// (16-row tiles, the running maximum) has it at exactly 1. With the running maximum here as well, relative error
// against 64 bits and time, without / with: 64 answers on 8192 tokens 0.0021 / 0.0018, 52.6 / 53.7 us; 200 on 32768 at
// 8 heads 0.0021 / 0.0017, 46.8 / 52.1; 100 over 8-bit pools 0.0018 / 0.0017, 65.2 / 65.3; 24 questions at d = 64
// 0.0021 / 0.0018, 44.5 / 50.4, prompts whose plain attention has 0.0021 too. Rounding the output to bf16 alone
// is 0.0016, so the time was kept.
//
// Work. Three launches: plan (once a batch), items, merge. One launch runs both kinds of items, so that
// they overlap: 128-row items (64-key tiles through LDS; the shared parts, and own parts of many new
// tokens), bound by the matrix cores and the softmax, and small items (one wavefront, 16 rows; own parts
// of single tokens), bound by reading K and V. A compute unit holds two workgroups, and the hardware
// deals them out in index order, unit after unit: the 128-row ones come first, so that each gets a unit's one
// half and small ones the other (mixed evenly instead, some units get two 128-row workgroups and others
// none: 64 answers on 8192 shared tokens of the 70B heads, 400 of their own, 46 us, so 38).
// What bounds it there, per launch: 256 128-row items of 16 key tiles take 26 us alone (1.4 us a tile; 1.0
// with half the units at work, and a sixth less on zeros, so part of it is the power limit), the small items'
// 126 MB 26 us at 4.9 TB/s; together 29 us where the pools are in the last-level cache (162 MB at 5.6 TB/s take
// 29) and 47 where they come from HBM, where the two slow each other down: the 128-row items load each key
// tile once per query tile, 134 MB through the same path as the small ones' 126.
#include "attention_kernels.h"

namespace gc {
namespace {

// Wavefronts of a workgroup, for 128-row tiles: 4 of 32 rows, or 8 of 16. With 8, the wavefronts that share a SIMD
// compute products and weights in turn where only one such workgroup is on the unit, and 512 threads share
// the widening of a tile's codes; every key and value is read from LDS twice as often, and 128 registers must do,
// which spills around the items. Over 8-bit pools at d = 128 (8 wavefronts / 4): 100 answers on four documents 59.3 us / 67.1,
// 48 questions of 20 tokens on 32768 shared ones 988 / 1065, 8 of 60 tokens on 4096 62.7 / 74.2. Over bf16 pools
// 64 answers on 8192 tokens 55.2 / 54.1, 128 on 16384 142 / 133, 200 on 32768 at 8 heads 44.9 / 45.9; at d = 64 in 8 bits 40 single
// tokens on 6000 26.8 / 26.2, 24 questions of 20 tokens in bf16 39.0 / 40.7 and 48 on 32768 632 / 599.
template <int D, bool FP8, int W>
__global__ __launch_bounds__(W * 64, W / 2) void attention_shared_kernel(const SharedAttnArgs a) {
    attention_body<D, W, FP8, 2, true, kBlockM / W>(a, blockIdx.x);
}

template <int D, bool FP8>
void launch_items(const SharedAttnArgs& a, unsigned workgroups, hipStream_t s) {
    constexpr int W = FP8 && D == 128 ? 8 : kWaves;
    attention_shared_kernel<D, FP8, W><<<workgroups, W * 64, 0, s>>>(a);
}

// Merge: a thread owns four consecutive output elements of one row; its chunks' log-sum-exps and
// values are read B at a time in one pass with a running maximum, in a fixed order (deterministic).
// What bounds it is the chain of dependent loads: the request (a search of the new-token offsets, 64 at
// a step), its record, the chunks. With G > 1 a row's chunks are dealt to G groups of threads (chunk c to
// group c % G), whose results are joined through LDS in group order: for few rows of many chunks.
template <int D, int G, int B>
__global__ __launch_bounds__(kCombineThreads) void shared_merge_kernel(const SharedMergeArgs a) {
    constexpr int CPR = D / 4;                          // threads per row and group
    constexpr int kRows = kCombineThreads / (CPR * G);  // rows per workgroup
    __shared__ f32x4 s_acc[G > 1 ? kCombineThreads : 1];
    __shared__ float s_max[G > 1 ? kCombineThreads / CPR : 1], s_tot[G > 1 ? kCombineThreads / CPR : 1];
    // (looked at below, so that the search does not wait for them)
    const bool planned = a.status[0] == 0 && *a.plan_mark == a.mark;
    const int lane = threadIdx.x & 63;
    const int c4 = (int)threadIdx.x % CPR;
    const int lane_row = (int)threadIdx.x / CPR;  // (row, group) of this thread
    const int sub = lane_row % G;
    const int64_t row = (int64_t)blockIdx.x * kRows + lane_row / G;
    const bool in_range = row < a.rows;
    const int64_t row_or_last = in_range ? row : a.rows - 1;
    const int t = a.rows <= UINT32_MAX ? a.hq.of((uint32_t)row_or_last) : (int)(row_or_last / a.hq.d);
    // the request of the wavefront's first row: the last r with cu[r] <= t0 (one token each: t0 itself, a load less)
    const int t0 = __builtin_amdgcn_readfirstlane(t);
    int lo = a.single ? t0 : 0, hi = a.single ? t0 + 1 : a.batch;  // cu[lo] <= t0 < cu[hi]
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64;
        const int at = lo + step * (lane + 1);
        const bool past = at >= hi || a.cu_new_lens[at < hi ? at : hi] > t0;
        lo += step * __builtin_popcountll(__ballot(!past));
        hi = min(lo + step, hi);
    }
    int r = lo;
    SharedReq q = a.reqs[r];
    while (planned && t >= q.cu + q.n && r + 1 < a.batch) q = a.reqs[++r];  // (later rows of the wavefront)
    const int i = t - q.cu;
    const bool row_ok = planned && in_range && q.merge && i >= 0 && i < q.n;
    if (G == 1 && !row_ok) return;
    const int h = (int)(row_or_last - (int64_t)t * a.hq.d);
    const int kvh = a.group.of((uint32_t)h), hl = h - kvh * a.group.d;

    float mx = -INFINITY, tot = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (row_ok) {
        // row of this row's first partial, and the distance to the next chunk's
        auto locate = [&](int i, bool small, int slot, int ns, int64_t& first, int64_t& stride) -> int {
            const int tile = small ? 0 : a.tq.of((uint32_t)i), bm = small ? kDecM : kBlockM;  // (a small part is one tile)
            stride = (int64_t)a.num_kv_heads * bm;
            first = ((int64_t)(slot + tile * ns) * a.num_kv_heads + kvh) * bm + (i - tile * a.tq.d) * a.group.d + hl;
            return tile;
        };
        int64_t g_row = 0, g_stride = 0, o_row, o_stride;
        if (q.g_ns > 0) locate(t - q.g_cu, q.g_small, q.g_slot, q.g_ns, g_row, g_stride);
        const int tile = locate(i, q.own_small, q.own_slot, q.own_ns, o_row, o_stride);
        int own = q.own_ns;  // (a tile of fewer key tiles has fewer chunks)
        if (!q.own_small) own = min(own, key_tiles(q.P, tile * a.tq.d, min(a.tq.d, q.n - tile * a.tq.d), kBlockN));
        const int total = q.g_ns + own;  // the shared chunks first
        const float* const g_o = q.g_small ? a.small_o : a.big_o;
        const float* const g_l = q.g_small ? a.small_lse : a.big_lse;
        const float* const o_o = q.own_small ? a.small_o : a.big_o;
        const float* const o_l = q.own_small ? a.small_lse : a.big_lse;

        for (int s0 = sub; s0 < total; s0 += B * G) {
            float l[B];
            f32x4 v[B];
#pragma unroll
            for (int u = 0; u < B; ++u) {
                const int c = s0 + u * G;
                l[u] = -INFINITY;
                v[u] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (c < total) {
                    const bool shared = c < q.g_ns;
                    const int64_t pr = shared ? g_row + c * g_stride : o_row + (c - q.g_ns) * o_stride;
                    l[u] = (shared ? g_l : o_l)[pr];
                    v[u] = *reinterpret_cast<const f32x4*>((shared ? g_o : o_o) + pr * D + 4 * c4);
                }
            }
            float mn = mx;
#pragma unroll
            for (int u = 0; u < B; ++u) mn = fmaxf(mn, l[u]);
            const float off = mn == -INFINITY ? 0.f : mn;
            const float alpha = expf(mx - off);
            tot *= alpha;
            acc *= alpha;
            mx = mn;
#pragma unroll
            for (int u = 0; u < B; ++u) {
                const float w = expf(l[u] - off);  // 0 for the padding entries
                tot += w;
                acc += w * v[u];
            }
        }
    }
    if constexpr (G > 1) {
        s_acc[threadIdx.x] = acc;
        if (c4 == 0) {
            s_max[lane_row] = mx;
            s_tot[lane_row] = tot;
        }
        __syncthreads();
        if (sub != 0 || !row_ok) return;
        const float mx0 = mx;
#pragma unroll
        for (int g = 1; g < G; ++g) mx = fmaxf(mx, s_max[lane_row + g]);
        const float off = mx == -INFINITY ? 0.f : mx;
        const float w0 = expf(mx0 - off);
        tot *= w0;
        acc *= w0;
#pragma unroll
        for (int g = 1; g < G; ++g) {
            const float w = expf(s_max[lane_row + g] - off);
            tot += w * s_tot[lane_row + g];
            acc += w * s_acc[threadIdx.x + g * CPR];
        }
    }
    // as in an unsplit item: weights that are all 0 give 0, a NaN sum gives NaN, both with lse -inf
    const float lse_tot = tot > 0.f ? mx + logf(tot) : -INFINITY;
    acc *= tot > 0.f ? 1.f / tot : 0.f;
    u32x2 w2;
    w2[0] = pack_bf16x2(acc[0], acc[1]);
    w2[1] = pack_bf16x2(acc[2], acc[3]);
    *reinterpret_cast<u32x2*>(a.out + row * D + 4 * c4) = w2;
    if (a.lse != nullptr && c4 == 0) a.lse[row] = lse_tot;
}

}  // namespace

hipError_t launch_attention_shared(const SharedAttnArgs& args, int head_dim, bool fp8, hipStream_t s) {
    SharedAttnArgs a = args;
    const int64_t heads = a.num_kv_heads;
    a.shared_per_xcd = (int)ceil_div64(a.shared_items * heads, kQueues);
    a.big_wgs = (int)((a.shared_per_xcd + ceil_div64(a.own_items * heads, kQueues)) * kQueues);
    const int64_t small = ceil_div64(a.small, shared_rings(fp8));
    if (a.big_wgs + small == 0) return hipSuccess;
    const unsigned grid = (unsigned)(a.big_wgs + small);
    if (head_dim == 128)
        fp8 ? launch_items<128, true>(a, grid, s) : launch_items<128, false>(a, grid, s);
    else
        fp8 ? launch_items<64, true>(a, grid, s) : launch_items<64, false>(a, grid, s);
    return hipGetLastError();
}

// Thread groups of a row in the merge: eight where the trips of loads saved (16 chunks a trip, or 64) are worth the
// rows' additional workgroups. One group / eight, attention and merge: 64 rows of 131 chunks 32.3 us / 18.5, 512 of
// 38 20.2 / 17.0, 1200 of 28 22.6 / 22.3, 1600 of 25 23.9 / 25.1, 4096 of 12 53.7 / 57.7.
static int merge_groups(int64_t rows, int max_chunks) {
    const int trips_saved = ceil_div(max_chunks, 16) - ceil_div(max_chunks, 64);
    return rows <= 1536LL * trips_saved ? 8 : 1;
}

int64_t shared_merge_workgroups(int64_t rows, int head_dim, int max_chunks) {
    return ceil_div64(rows, kCombineThreads / (head_dim / 4 * merge_groups(rows, max_chunks)));
}

template <int D>
static void launch_merge(const SharedMergeArgs& a, int max_chunks, hipStream_t s) {
    const unsigned grid = (unsigned)shared_merge_workgroups(a.rows, D, max_chunks);
    // Six chunks at a time where a compute unit has more than one workgroup (fewer registers, more of them at
    // once), 16 where each row's loads are on their own. Attention and merge, 6 / 16: 64 workgroups 16.8 us / 16.6, 200
    // of 25 chunks 46.2 / 45.3, 256 18.5 / 18.6, 448 22.7 / 23.2, 800 51.6 / 53.3, 960 of five chunks 37.4 / 39.5, 2360 66.3 / 71.2.
    if (merge_groups(a.rows, max_chunks) > 1)
        shared_merge_kernel<D, 8, 8><<<grid, kCombineThreads, 0, s>>>(a);
    else if (grid > 256)
        shared_merge_kernel<D, 1, 6><<<grid, kCombineThreads, 0, s>>>(a);
    else
        shared_merge_kernel<D, 1, 16><<<grid, kCombineThreads, 0, s>>>(a);
}

hipError_t launch_shared_merge(const SharedMergeArgs& a, int head_dim, int max_chunks, hipStream_t s) {
    if (head_dim == 128)
        launch_merge<128>(a, max_chunks, s);
    else
        launch_merge<64>(a, max_chunks, s);
    return hipGetLastError();
}

}  // namespace gc
