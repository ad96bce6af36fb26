// Attention kernels over 4-bit pools and their launcher (the device code is in attention_fp4_body.h).
#include "attention_fp4_body.h"

namespace gc {
namespace {

template <int D>
__global__ __launch_bounds__(kFp4SmallWaves * 64, 4) void attention_fp4_small_kernel(const Fp4AttnArgs a) {
    __shared__ Fp4SmallLds<D> lds;
    const int kvh = (int)(blockIdx.x % (unsigned)a.num_kv_heads);
    fp4_small_body<D>(a, a.items[blockIdx.x / (unsigned)a.num_kv_heads], kvh, lds);
}

template <int D, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 8 / WAVES) void attention_fp4_kernel(const Fp4AttnArgs a) {
    __shared__ Fp4Lds<D, WAVES> lds;
    fp4_attention_body<D, WAVES>(a, blockIdx.x, lds);
}

// Resident launch of wide tiles, as over the other pools (attention_kernels.h): one workgroup per compute unit takes
// work items from its XCD's queue, and from the others' when that is empty.
template <int D>
__global__ __launch_bounds__(kWideWaves * 64, 1) void attention_fp4_resident_kernel(const Fp4AttnArgs a, int total) {
    __shared__ Fp4Lds<D, kWideWaves> lds;
    __shared__ int s_tk, s_empty;
    const int x = (int)(blockIdx.x % (unsigned)kQueues);
    if (threadIdx.x == 0) s_empty = 0;
    for (;;) {
        if (threadIdx.x == 0) {
            int b = -1, empty = s_empty;
            for (int j = 0; j < kQueues && b < 0; ++j) {
                const int y = (x + j) % kQueues;
                if (empty & (1 << y)) continue;
                const int k = __hip_atomic_fetch_add(&a.queues[y], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                if ((int64_t)k * kQueues + y < total) b = k * kQueues + y;
                else empty |= 1 << y;
            }
            s_empty = empty;
            s_tk = b;
        }
        __syncthreads();
        const int b = s_tk;
        __syncthreads();  // every wavefront has read the ticket, and the stage, before the next item
        if (b < 0) break;
        fp4_attention_body<D, kWideWaves>(a, (unsigned)b, lds);
    }
    if (threadIdx.x == 0) {
        const int out = __hip_atomic_fetch_add(&a.queues[kQueues], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (out == (int)gridDim.x - 1)
            for (int y = 0; y <= kQueues; ++y)
                __hip_atomic_store(&a.queues[y], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
}

template <int D>
void launch_fp4(const Fp4AttnArgs& a, int64_t num_items, bool small, bool wide, int resident, hipStream_t s) {
    const int64_t total = num_items * a.num_kv_heads;
    const dim3 grid((unsigned)total);
    if (small)
        attention_fp4_small_kernel<D><<<grid, kFp4SmallWaves * 64, 0, s>>>(a);
    else if (wide && resident > 0)
        attention_fp4_resident_kernel<D><<<dim3((unsigned)resident), kWideWaves * 64, 0, s>>>(a, (int)total);
    else if (wide)
        attention_fp4_kernel<D, kWideWaves><<<grid, kWideWaves * 64, 0, s>>>(a);
    else
        attention_fp4_kernel<D, kWaves><<<grid, kWaves * 64, 0, s>>>(a);
}

}  // namespace

hipError_t launch_attention_fp4(const Fp4AttnArgs& a, int head_dim, int64_t num_items, bool small, bool wide,
                                int resident, hipStream_t s) {
    if (head_dim == 128)
        launch_fp4<128>(a, num_items, small, wide, resident, s);
    else
        launch_fp4<64>(a, num_items, small, wide, resident, s);
    return hipGetLastError();
}

}  // namespace gc
