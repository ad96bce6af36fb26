// Small-tile attention kernel and its launcher (the device code is in attention_small_body.h).
#include "attention_small_body.h"

namespace gc {
namespace {

template <int D, bool FP8>
__global__ __launch_bounds__(64, 2) void attention_small_kernel(const AttnArgs a) {
    __shared__ __align__(1024) unsigned char ring[2 * kSmallTileBytes<D, FP8>];
    const int kvh = (int)(blockIdx.x % (unsigned)a.num_kv_heads);
    small_body<D, FP8, false>(a, a.items[blockIdx.x / (unsigned)a.num_kv_heads], kvh, ring, ring + kSmallTileBytes<D, FP8>);
}

}  // namespace

hipError_t launch_attention_small(const AttnArgs& a, int head_dim, int64_t num_items, bool fp8,
                                  hipStream_t s) {
    const dim3 grid((unsigned)(num_items * a.num_kv_heads));
    if (fp8) {
        if (head_dim == 128)
            attention_small_kernel<128, true><<<grid, 64, 0, s>>>(a);
        else
            attention_small_kernel<64, true><<<grid, 64, 0, s>>>(a);
    } else {
        if (head_dim == 128)
            attention_small_kernel<128, false><<<grid, 64, 0, s>>>(a);
        else
            attention_small_kernel<64, false><<<grid, 64, 0, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace gc
