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
// What bounds it: memory; for a few tokens the chain lengths -> block id -> codes -> rows.
#include "append_body.h"
#include "fp4.h"

namespace gc {
namespace {

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

template <int D, Pool KIND>
__global__ __launch_bounds__(kAppendThreads) void read_kernel(const ReadArgs ra) {
    __shared__ AppendLds<D> lds;
    const AppendArgs& a = ra.a;
    constexpr int CPR = D / 8;
    constexpr int kPer = kPage * CPR;  // threads per head
    const unsigned u = blockIdx.x / ra.jobs, hg = blockIdx.x - u * ra.jobs;
    PageUnit at;
    if (!locate_page<D>(a, lds, (int)u, (int)gridDim.x, at)) return;
    const int lp = at.P / kPage + at.k;
    const int s0 = max(at.P - lp * kPage, 0);
    const int s1 = min(at.P + at.n - lp * kPage, kPage);
    if (lp >= a.max_blocks) return;
    const int blk = a.block_tables[(int64_t)at.r * a.max_blocks + lp];
    if (blk < 0 || blk >= a.num_blocks) return;
    const int tid = threadIdx.x % kPer, sub = threadIdx.x / kPer;
    const int h = (int)hg * AppendLds<D>::kHeads + sub;
    const bool head_ok = h < a.num_kv_heads;
    const int s = tid / CPR, c = tid % CPR;
    const int64_t row = (int64_t)at.cu + (int64_t)lp * kPage - at.P + s;
    const bool ok = head_ok && s >= s0 && s < s1 && row >= 0 && row < a.total_tokens;
    const int64_t page = (int64_t)blk * a.num_kv_heads + h;
    const int64_t slot = page * kPage + s;
    u32x4 k = u32x4{0u, 0u, 0u, 0u}, v = k;
    if constexpr (KIND == Pool::kFp4) {
        if (!ok) return;
        const uint32_t kw = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(a.k_pool) + slot * (D / 2) + c * 4);
        const uint32_t vw = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(a.v_pool) + slot * (D / 2) + c * 4);
        const uint32_t sc = *reinterpret_cast<const uint16_t*>(ra.scales + (slot * (D / kFp4Block) + c / 4) * 2);
        uint32_t w[4];
        fp4_widen8(kw, fp4_scale(sc & 255), w);
        k = u32x4{w[0], w[1], w[2], w[3]};
        fp4_widen8(vw, fp4_scale(sc >> 8), w);
        v = u32x4{w[0], w[1], w[2], w[3]};
    } else {
        if (ok) {
            if constexpr (KIND == Pool::kFp8)
                k = widen_fp8x8(*reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(a.k_pool) + slot * D + c * 8), ra.k_scale);
            else
                k = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.k_pool) + slot * D + c * 8);
        }
        constexpr int kStride = AppendLds<D>::kStride;
        uint16_t* const sv = lds.v[sub];
        if (head_ok) {
            const int d = tid >> 1, x0 = 8 * (tid & 1);
            const int64_t src = (page * D + d) * kPage + x0;
            u32x4 w;
            if constexpr (KIND == Pool::kFp8)
                w = widen_fp8x8(*reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(a.v_pool) + src), ra.v_scale);
            else
                w = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.v_pool) + src);
#pragma unroll
            for (int x = 0; x < 8; ++x) sv[(x0 + x) * kStride + d] = (uint16_t)(w[x / 2] >> (16 * (x % 2)));
        }
        __syncthreads();
        if (!ok) return;
        v = *reinterpret_cast<const u32x4*>(&sv[s * kStride + c * 8]);
    }
    const int64_t dst = (row * a.num_kv_heads + h) * D + c * 8;
    *reinterpret_cast<u32x4*>(ra.k_out + dst) = k;
    *reinterpret_cast<u32x4*>(ra.v_out + dst) = v;
}

template <int D>
void launch_kind(const ReadArgs& ra, Pool kind, unsigned grid, hipStream_t s) {
    if (kind == Pool::kFp4)
        read_kernel<D, Pool::kFp4><<<grid, kAppendThreads, 0, s>>>(ra);
    else if (kind == Pool::kFp8)
        read_kernel<D, Pool::kFp8><<<grid, kAppendThreads, 0, s>>>(ra);
    else
        read_kernel<D, Pool::kBf16><<<grid, kAppendThreads, 0, s>>>(ra);
}

}  // namespace

int64_t read_workgroups(int64_t pages, int num_kv_heads, int head_dim) {
    return pages * ceil_div(num_kv_heads, append_heads(head_dim));
}

hipError_t launch_read(const ReadArgs& args, int head_dim, Pool kind, hipStream_t s) {
    ReadArgs ra = args;
    if (ra.a.total_pages <= 0) return hipSuccess;
    ra.jobs = (uint32_t)read_workgroups(1, ra.a.num_kv_heads, head_dim);
    const unsigned grid = ra.jobs * (unsigned)ra.a.total_pages;
    if (head_dim == 128)
        launch_kind<128>(ra, kind, grid, s);
    else
        launch_kind<64>(ra, kind, grid, s);
    return hipGetLastError();
}

}  // namespace gc
