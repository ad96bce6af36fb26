// Launchers of the attention kernels over 8-bit pools and of the split merge (the
// kernels are in attention_kernels.h).
#include "attention_kernels.h"

namespace gc {

hipError_t launch_attention_fp8(const AttnArgs& a, int head_dim, int64_t num_items, bool wide, bool three,
                                int resident, hipStream_t s) {
    const dim3 grid((unsigned)(num_items * a.num_kv_heads));
    if (resident > 0 && wide) {
        const int total = (int)(num_items * a.num_kv_heads);
        const dim3 rg((unsigned)resident), rb(kWideWaves * 64);
        if (head_dim == 128)
            hipLaunchKernelGGL((attention_resident_kernel<128, true>), rg, rb, 0, s, a, total);
        else
            hipLaunchKernelGGL((attention_resident_kernel<64, true>), rg, rb, 0, s, a, total);
        return hipGetLastError();
    }
    if (wide) {
        if (head_dim == 128)
            attention_kernel<128, kWideWaves, true><<<grid, kWideWaves * 64, 0, s>>>(a);
        else
            attention_kernel<64, kWideWaves, true><<<grid, kWideWaves * 64, 0, s>>>(a);
    } else {
        if (head_dim == 128)
            attention_kernel<128, kWaves, true><<<grid, kWaves * 64, 0, s>>>(a);
        else if (three)
            attention_kernel<64, kWaves, true, 3><<<grid, kWaves * 64, 0, s>>>(a);
        else
            attention_kernel<64, kWaves, true><<<grid, kWaves * 64, 0, s>>>(a);
    }
    return hipGetLastError();
}

// Eight thread groups per row save round trips (32 chunks each instead of 8, about
// 1 us a trip) and cost workgroups (one per row instead of one per eight, about 0.7 ns
// each to start), so they are for few rows: 16.3 -> 15.1 us (attention and merge) for
// 128 rows of 17 chunks, but 28.6 -> 31.0 for 4096 rows of 9 and 93 -> 105 for 16384.
static int combine_groups(int64_t num_combines, int num_kv_heads, int block_m, int max_splits) {
    const int trips_saved = ceil_div(max_splits, 8) - ceil_div(max_splits, 32);
    return num_combines * num_kv_heads * block_m <= 1536LL * trips_saved ? 8 : 1;
}

int64_t combine_workgroups(int64_t num_combines, int num_kv_heads, int block_m, int head_dim, int max_splits) {
    const int rows = kCombineThreads / (head_dim / 4 * combine_groups(num_combines, num_kv_heads, block_m, max_splits));
    return num_combines * num_kv_heads * ceil_div(block_m, rows);
}

hipError_t launch_combine(const CombineArgs& a, int head_dim, int64_t num_combines, int max_splits, hipStream_t s) {
    const int groups_of = combine_groups(num_combines, a.num_kv_heads, a.block_m, max_splits);
    const dim3 grid((unsigned)combine_workgroups(num_combines, a.num_kv_heads, a.block_m, head_dim, max_splits));
    if (head_dim == 128) {
        if (groups_of > 1)
            combine_kernel<128, 8><<<grid, kCombineThreads, 0, s>>>(a);
        else
            combine_kernel<128, 1><<<grid, kCombineThreads, 0, s>>>(a);
    } else {
        if (groups_of > 1)
            combine_kernel<64, 8><<<grid, kCombineThreads, 0, s>>>(a);
        else
            combine_kernel<64, 1><<<grid, kCombineThreads, 0, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace gc
