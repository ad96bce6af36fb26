// KV append into 4-bit pools (GreenCache §2.2, Fig. 1a step 1; the numbers are in fp4.h): the new tokens' rows are
// quantised on the way. A workgroup owns one destination page (up to 16 tokens of one request, found as in append_body.h)
// of kHeads KV heads or groups of heads; thread (slot s, chunk c) takes eight elements of a key row and of a value row of each,
// four neighbouring lanes a block.
// What bounds it: memory, and for a few tokens the chain lengths -> block id, rows -> codes. A workgroup of one head has 8 KB in
// flight and starts too often: from kManyWorkgroups of them on, a workgroup takes four (32000 tokens of 8 heads, d = 64, 96 MB:
// 29.8 -> 19.6 us; two 20.9, eight 22.1). Rows of more than the last-level cache keeps, 192 MB, are read past it (66000 tokens,
// d = 128, 340 MB: 59.8 us, else 68.4; but 96 MB 20.1 / 19.6).
#include "append_body.h"
#include "fp4.h"

namespace gc {
namespace {

constexpr int64_t kManyWorkgroups = 4096;

template <int D, int HEADS, bool STREAM>
__global__ __launch_bounds__(kAppendThreads) void append_fp4_kernel(const AppendArgs a, uint8_t* scales, uint32_t jobs) {
    __shared__ AppendLds<D> lds;
    constexpr int CPR = D / 8;
    constexpr int kPer = kPage * CPR;  // threads per head
    constexpr int kBeside = AppendLds<D>::kHeads;
    const unsigned u = blockIdx.x / jobs, hg = blockIdx.x - u * jobs;
    PageUnit at;
    if (!locate_page<D>(a, lds, (int)u, (int)gridDim.x, at)) return;
    const int lp = at.P / kPage + at.k;
    const int s0 = max(at.P - lp * kPage, 0);
    const int s1 = min(at.P + at.n - lp * kPage, kPage);
    if (lp >= a.max_blocks) return;
    const int blk = a.block_tables[(int64_t)at.r * a.max_blocks + lp];
    const int tid = threadIdx.x % kPer;
    const int s = tid / CPR, c = tid % CPR;
    const int64_t row = (int64_t)at.cu + (int64_t)lp * kPage - at.P + s;
    const int h0 = (int)hg * (HEADS * kBeside) + threadIdx.x / kPer;
    const bool ok = s >= s0 && s < s1 && row >= 0 && row < a.total_tokens;
    u32x4 k[HEADS], v[HEADS];
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
        const int h = h0 + i * kBeside;
        k[i] = v[i] = u32x4{0u, 0u, 0u, 0u};
        if (ok && h < a.num_kv_heads) {  // (before the block id is looked at, so that the loads run beside its own)
            const int64_t src = (row * a.num_kv_heads + h) * D + c * 8;
            const u32x4* const kp = reinterpret_cast<const u32x4*>(a.k_new + src);
            const u32x4* const vp = reinterpret_cast<const u32x4*>(a.v_new + src);
            k[i] = STREAM ? __builtin_nontemporal_load(kp) : *kp;
            v[i] = STREAM ? __builtin_nontemporal_load(vp) : *vp;
        }
    }
    if (blk < 0 || blk >= a.num_blocks) return;
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
        const int h = h0 + i * kBeside;
        float x[8], y[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[2 * j] = bf16_lo(k[i][j]);
            x[2 * j + 1] = bf16_hi(k[i][j]);
            y[2 * j] = bf16_lo(v[i][j]);
            y[2 * j + 1] = bf16_hi(v[i][j]);
        }
        fp4_store<D>(static_cast<uint8_t*>(a.k_pool), static_cast<uint8_t*>(a.v_pool), scales,
                     ((int64_t)blk * a.num_kv_heads + h) * kPage + s, c, x, y, ok && h < a.num_kv_heads);
    }
}

template <int D>
void launch(const AppendArgs& a, uint8_t* scales, hipStream_t s) {
    const int64_t one = head_page_workgroups(a.total_pages, a.num_kv_heads, D);
    const int groups = ceil_div(a.num_kv_heads, append_heads(D));
    if (one >= kManyWorkgroups) {
        const uint32_t jobs = (uint32_t)ceil_div(groups, 4);
        const unsigned grid = jobs * (unsigned)a.total_pages;
        if ((int64_t)a.total_tokens * a.num_kv_heads * D * 4 >= (192LL << 20))
            append_fp4_kernel<D, 4, true><<<grid, kAppendThreads, 0, s>>>(a, scales, jobs);
        else
            append_fp4_kernel<D, 4, false><<<grid, kAppendThreads, 0, s>>>(a, scales, jobs);
    } else {
        append_fp4_kernel<D, 1, false><<<(unsigned)one, kAppendThreads, 0, s>>>(a, scales, (uint32_t)groups);
    }
}

}  // namespace

int64_t head_page_workgroups(int64_t pages, int num_kv_heads, int head_dim) {
    return pages * ceil_div(num_kv_heads, append_heads(head_dim));
}

hipError_t launch_append_fp4(const AppendArgs& a, uint8_t* scales, int head_dim, hipStream_t s) {
    if (a.total_pages <= 0) return hipSuccess;
    if (head_dim == 128)
        launch<128>(a, scales, s);
    else
        launch<64>(a, scales, s);
    return hipGetLastError();
}

}  // namespace gc
