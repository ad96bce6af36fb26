// Rows out of a paged pool (GreenCache §2.2, Fig. 1a: a context's KV on its way to the cache's host tier, or to a
// pool of another kind): the inverse of the append. For every request r, new token i of the batch and KV head h
// the element values that the pool holds at position P_r + i go to row cu_r + i of k_out and v_out as bf16.
//
// A workgroup owns one page (up to 16 tokens of one request) of one KV head (two at D = 64), as in the append,
// with the same search; thread (slot s, chunk c) writes eight elements, 16 bytes, of a row of keys and of one of values:
//   - bf16 pools: the bits; 8-bit pools: bf16(fl32(code value * scale));
//     4-bit pools: exact (every value is a bf16 number).
//   - keys, and the values of 4-bit pools, lie as rows; value pages of the other pools are transposed
//     ([D][16 slots]): thread (value row d, half of the slots) reads eight slots, which reach their rows through LDS.
// Rows whose page has a block id outside the pool keep their contents.
// What bounds it: memory; for a few tokens the chain lengths -> block id -> codes -> rows. From kManyWorkgroups workgroups of
// one head each on, a workgroup takes four heads of a page, or eight of 4-bit pools, whose loads run side by side (66000 tokens
// of 8 heads out of 4-bit pools, 340 MB: 85.6 -> 71.6 us). The rows are written around the caches' retention (non-temporal): 50.9 us,
// 6.7 TB/s with a part of the codes in the last-level cache; out of 8-bit pools 53.6 -> 41.6 (256 MB), bf16 51.1 -> 45.6 (244 MB).
// To pinned host memory PCIe: 270 MB of rows 5.06 ms, 53.5 GB/s (a copy of them 4.76).
#include "append_body.h"
#include "fp4.h"

namespace gc {
namespace {

constexpr int64_t kManyWorkgroups = 4096;  // (workgroups of one head each)

// Eight E4M3 codes times scale as eight bf16 values.
__device__ __forceinline__ u32x4 widen_fp8x8(const u32x2 w, float scale) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false);
        const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
        const fp4_bf16x2 a = {(__bf16)(lo[0] * scale), (__bf16)(lo[1] * scale)};
        const fp4_bf16x2 b = {(__bf16)(hi[0] * scale), (__bf16)(hi[1] * scale)};
        r[2 * i] = __builtin_bit_cast(uint32_t, a);
        r[2 * i + 1] = __builtin_bit_cast(uint32_t, b);
    }
    return r;
}

template <int D, Pool KIND, int HEADS>
__global__ __launch_bounds__(kAppendThreads) void read_kernel(const ReadArgs ra) {
    const AppendArgs& a = ra.a;
    constexpr int CPR = D / 8;
    constexpr int kPer = kPage * CPR;  // threads per head
    constexpr int kBeside = AppendLds<D>::kHeads;
    constexpr int kStride = AppendLds<D>::kStride;
    constexpr bool kRows = KIND == Pool::kFp4;  // values lie as rows
    __shared__ union {
        AppendLds<D> search;
        uint16_t v[kRows ? 1 : HEADS][kRows ? 1 : kBeside][kRows ? 1 : kPage * kStride];
    } lds;
    const unsigned u = blockIdx.x / ra.jobs, hg = blockIdx.x - u * ra.jobs;
    PageUnit at;
    if (!locate_page<D>(a, lds.search, (int)u, (int)gridDim.x, at)) return;
    const int lp = at.P / kPage + at.k;
    const int s0 = max(at.P - lp * kPage, 0);
    const int s1 = min(at.P + at.n - lp * kPage, kPage);
    if (lp >= a.max_blocks) return;
    const int blk = a.block_tables[(int64_t)at.r * a.max_blocks + lp];
    if (blk < 0 || blk >= a.num_blocks) return;
    const int tid = threadIdx.x % kPer, sub = threadIdx.x / kPer;
    const int s = tid / CPR, c = tid % CPR;
    const int64_t row = (int64_t)at.cu + (int64_t)lp * kPage - at.P + s;
    const int h0 = (int)hg * (HEADS * kBeside) + sub;
    const bool ok = s >= s0 && s < s1 && row >= 0 && row < a.total_tokens;
    const int64_t page0 = (int64_t)blk * a.num_kv_heads;
    u32x4 k[HEADS], v[HEADS];
    if constexpr (kRows) {
        uint32_t kw[HEADS], vw[HEADS], sc[HEADS];
        if (!ok) return;
#pragma unroll
        for (int i = 0; i < HEADS; ++i) {
            const int h = min(h0 + i * kBeside, a.num_kv_heads - 1);  // (a head twice rather than none)
            const int64_t slot = (page0 + h) * kPage + s;
            kw[i] = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(a.k_pool) + slot * (D / 2) + c * 4);
            vw[i] = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(a.v_pool) + slot * (D / 2) + c * 4);
            sc[i] = *reinterpret_cast<const uint16_t*>(ra.scales + (slot * (D / kFp4Block) + c / 4) * 2);
        }
#pragma unroll
        for (int i = 0; i < HEADS; ++i) {
            uint32_t w[4];
            fp4_widen8(kw[i], fp4_scale(sc[i] & 255), w);
            k[i] = u32x4{w[0], w[1], w[2], w[3]};
            fp4_widen8(vw[i], fp4_scale(sc[i] >> 8), w);
            v[i] = u32x4{w[0], w[1], w[2], w[3]};
        }
    } else {
        // Value pages are transposed: thread (value row d, half of the slots) brings eight slots, through LDS.
        const int d = tid >> 1, x0 = 8 * (tid & 1);
#pragma unroll
        for (int i = 0; i < HEADS; ++i) {
            const int h = min(h0 + i * kBeside, a.num_kv_heads - 1);
            const int64_t from = ((page0 + h) * kPage + s) * D + c * 8, v_from = ((page0 + h) * D + d) * kPage + x0;
            if constexpr (KIND == Pool::kFp8) {
                k[i] = widen_fp8x8(*reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(a.k_pool) + from), ra.k_scale);
                v[i] = widen_fp8x8(*reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(a.v_pool) + v_from), ra.v_scale);
            } else {
                k[i] = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.k_pool) + from);
                v[i] = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.v_pool) + v_from);
            }
        }
        __syncthreads();  // (the search is over)
#pragma unroll
        for (int i = 0; i < HEADS; ++i)
#pragma unroll
            for (int x = 0; x < 8; ++x) lds.v[i][sub][(x0 + x) * kStride + d] = (uint16_t)(v[i][x / 2] >> (16 * (x % 2)));
        __syncthreads();
        if (!ok) return;
#pragma unroll
        for (int i = 0; i < HEADS; ++i) v[i] = *reinterpret_cast<const u32x4*>(&lds.v[i][sub][s * kStride + c * 8]);
    }
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
        const int h = h0 + i * kBeside;
        if (h >= a.num_kv_heads) return;
        const int64_t dst = (row * a.num_kv_heads + h) * D + c * 8;
        __builtin_nontemporal_store(k[i], reinterpret_cast<u32x4*>(ra.k_out + dst));
        __builtin_nontemporal_store(v[i], reinterpret_cast<u32x4*>(ra.v_out + dst));
    }
}

template <int D, Pool KIND, int MOST>
void launch_kind(ReadArgs ra, hipStream_t s) {
    const int64_t one = head_page_workgroups(ra.a.total_pages, ra.a.num_kv_heads, D);
    const int groups = ceil_div(ra.a.num_kv_heads, append_heads(D));
    if (one >= kManyWorkgroups) {
        ra.jobs = (uint32_t)ceil_div(groups, MOST);
        read_kernel<D, KIND, MOST><<<ra.jobs * (unsigned)ra.a.total_pages, kAppendThreads, 0, s>>>(ra);
    } else {
        ra.jobs = (uint32_t)groups;
        read_kernel<D, KIND, 1><<<(unsigned)one, kAppendThreads, 0, s>>>(ra);
    }
}

template <int D>
void launch(const ReadArgs& ra, Pool kind, hipStream_t s) {
    if (kind == Pool::kFp4)
        launch_kind<D, Pool::kFp4, 8>(ra, s);
    else if (kind == Pool::kFp8)
        launch_kind<D, Pool::kFp8, 4>(ra, s);
    else
        launch_kind<D, Pool::kBf16, 4>(ra, s);
}

}  // namespace

hipError_t launch_read(const ReadArgs& ra, int head_dim, Pool kind, hipStream_t s) {
    if (ra.a.total_pages <= 0) return hipSuccess;
    if (head_dim == 128)
        launch<128>(ra, kind, s);
    else
        launch<64>(ra, kind, s);
    return hipGetLastError();
}

}  // namespace gc
