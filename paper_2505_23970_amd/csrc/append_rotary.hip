// KV append with the rotary position applied on the way (GreenCache §2.2, Fig. 1a step 1, for a program
// whose projections hand over keys and queries without their position): the new tokens' keys are rotated
// and saved with their values, the queries are rotated into q_out, in one launch.
//
// Mathematics. Token i of request r stands at position p = P_r + i. Its head vector's first R elements
// form R / 2 pairs, (j, j + R/2) or (2j, 2j + 1), and pair j is turned by the angle whose cosine and sine
// the caller's table holds:
//     y_a = x_a cos - x_b sin,   y_b = x_b cos + x_a sin,
// in fp32 (one product and one fused multiply-add), rounded once: to bf16, or for keys of 8-bit pools
// straight to the E4M3 code nearest to y / scale (rounding to bf16 in between would add half as much
// again as a bf16 ulp to a code's own error for nothing). Elements from R on pass through bit for bit.
// The table is fp32 [position][pair][cos, sin]: angles of far positions need 64 bits, which the kernel
// would have to spend per token and head; the table costs 4 R bytes a token, read once per workgroup.
//
// Work. A workgroup owns one destination page (up to 16 tokens of one request) of either
//   - one KV head (two at D = 64): keys in 16-byte chunks, one per thread, whose partner chunk in the other
//     half comes from the lane that holds it; values as in the plain append (append_body.h);
//   - or kRotQHeads query heads: a thread owns two 16-byte chunks (elements j .. j + 7 and their
//     partners, or two that need no other), holds the eight (cos, sin) of its token in registers and goes through
//     the heads, so it may write q_out over q. Pages with few new tokens (decode) put their threads on heads
//     instead. Neighbouring lanes take neighbouring chunks and then heads, whatever the pairs (pairs side by side:
//     16000 tokens of the 70B heads 92 us, 121 with a thread's two chunks adjacent and slots before heads).
// What bounds it: memory for prompts; for decode the chain lengths -> block id, rows and table -> stores.
//   - Prompts: the workgroups of a page (its KV heads, its query heads) are launched side by side, on all
//     XCDs, so that a token's projections are read in one sweep (30000 tokens of the 70B heads 243 us, page
//     after page for each head 277, pages dealt to the XCDs 273). Decode batches, a token a page, are launched
//     head by head: the workgroups of a page then share an XCD's L2 (96 tokens 5.0 us, 5.6 the other way).
//   - q_out is written around the caches' retention (non-temporal): 1290 MB 231 us (243), 359 MB 61 (74), 46 MB
//     9.8 (10.8). The queries are read that way as well where they exceed what the last-level cache keeps from one
//     pass to the next: from 192 MB of them on (1290 MB 210 us against 231, 550 MB 94 / 99; but 359 MB 66 / 61,
//     183 MB at d = 64 41 / 32).
// At 1290 MB it moves 5.7 TB/s (228 us), and 6.1 where the last-level cache holds a part of the inputs; a copy of as
// many bytes by the framework's tensor library 4.8 to 5.3.
#include "append_body.h"
#include "fp4.h"

namespace gc {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kRotQHeads = 16;  // query heads of a workgroup

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __bf16 a = (__bf16)lo, b = (__bf16)hi;
    return (uint32_t)__builtin_bit_cast(uint16_t, a) | ((uint32_t)__builtin_bit_cast(uint16_t, b) << 16);
}

__device__ __forceinline__ uint32_t quantise4f(float x0, float x1, float x2, float x3, float inv) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(clamp448(x0 * inv), clamp448(x1 * inv), 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(clamp448(x2 * inv), clamp448(x3 * inv), r, true);
    return (uint32_t)r;
}

// Eight bf16 values (a 16-byte chunk) in fp32.
__device__ __forceinline__ void widen8(const u32x4 w, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = bf16_lo(w[i]);
        x[2 * i + 1] = bf16_hi(w[i]);
    }
}
__device__ __forceinline__ u32x4 pack8(const float (&y)[8]) {
    return u32x4{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7])};
}

// (cos, sin) of N consecutive pairs.
template <int N>
__device__ __forceinline__ void load_angles(const float* at, float* cs, float* sn) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        const f32x4 w = *reinterpret_cast<const f32x4*>(at + 4 * i);
        cs[2 * i] = w[0];
        sn[2 * i] = w[1];
        cs[2 * i + 1] = w[2];
        sn[2 * i + 1] = w[3];
    }
}

// Pairs side by side: elements 2j and 2j + 1 of a chunk.
__device__ __forceinline__ void turn_adjacent(float (&x)[8], const float* cs, const float* sn) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float a = x[2 * j], b = x[2 * j + 1];
        x[2 * j] = fmaf(a, cs[j], -(b * sn[j]));
        x[2 * j + 1] = fmaf(b, cs[j], a * sn[j]);
    }
}

// Keys and values of one page and KV head (group hg of heads).
template <int D, bool FP8>
__device__ __forceinline__ void rotary_kv(const RotaryArgs& ra, AppendLds<D>& sm, const PageUnit& at, int lp, int s0,
                                          int s1, int hg) {
    const AppendArgs& a = ra.a;
    constexpr int CPR = D / 8;
    constexpr int kStride = AppendLds<D>::kStride;
    constexpr int kPer = kPage * CPR;
    const int tid = threadIdx.x % kPer;
    const int sub = threadIdx.x / kPer;
    const int h = hg * AppendLds<D>::kHeads + sub;
    const bool head_ok = h < a.num_kv_heads;
    const int blk = a.block_tables[(int64_t)at.r * a.max_blocks + lp];
    const int s = tid / CPR, c = tid % CPR;
    const int64_t row = (int64_t)at.cu + (int64_t)lp * kPage - at.P + s;
    const int pos = lp * kPage + s;
    const bool ok = head_ok && s >= s0 && s < s1 && row >= 0 && row < a.total_tokens && pos < ra.num_positions;
    const int half = ra.rotary_dim / 16;  // chunks of half the rotated elements
    const bool turned = c < 2 * half;
    u32x4 key = u32x4{0u, 0u, 0u, 0u}, v = key;
    float cs[8] = {}, sn[8] = {};
    if (ok) {  // (before the block id is looked at, so that the loads run beside its own)
        key = *reinterpret_cast<const u32x4*>(a.k_new + row * ra.k_stride + h * D + c * 8);
        v = *reinterpret_cast<const u32x4*>(a.v_new + row * ra.v_stride + h * D + c * 8);
        if (turned) {
            const float* table = ra.table + (int64_t)pos * ra.rotary_dim;
            if (ra.interleaved)
                load_angles<4>(table + 8 * c, cs, sn);
            else
                load_angles<8>(table + 16 * (c < half ? c : c - half), cs, sn);
        }
    }
    float x[8];
    widen8(key, x);
    if (ra.interleaved) {
        if (turned) turn_adjacent(x, cs, sn);
    } else {
        // the partner chunk, from the lane that holds it (a row's chunks lie in one wavefront)
        const int lane = threadIdx.x & 63;
        const int from = turned ? lane + (c < half ? half : -half) : lane;
        u32x4 other;
#pragma unroll
        for (int i = 0; i < 4; ++i) other[i] = (uint32_t)__shfl((int)key[i], from);
        if (turned) {
            float y[8];
            widen8(other, y);
            // the upper half adds the product that the lower half subtracts
            const bool low = c < half;
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = fmaf(x[j], cs[j], low ? -(y[j] * sn[j]) : y[j] * sn[j]);
        }
    }
    if (blk < 0 || blk >= a.num_blocks) return;
    const int64_t page = (int64_t)blk * a.num_kv_heads + h;
    if (ok) {
        const int64_t dst = (page * kPage + s) * D + c * 8;
        if constexpr (FP8) {
            *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.k_pool) + dst) =
                u32x2{quantise4f(x[0], x[1], x[2], x[3], a.k_inv), quantise4f(x[4], x[5], x[6], x[7], a.k_inv)};
        } else {
            *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.k_pool) + dst) = turned ? pack8(x) : key;
        }
    }
    uint16_t* const sv = sm.v[sub];
    *reinterpret_cast<u32x4*>(&sv[s * kStride + c * 8]) = v;
    __syncthreads();
    if (head_ok) store_values<D, FP8>(a, sv, page, tid, s0, s1);
}

// The same into 4-bit pools (fp4.h), whose pages hold whole rows of keys and of values: a token's codes share
// no byte with another token's. Four lanes hold the 32 elements of a block. Rotated keys are computed in 64
// bits and rounded to 32 (the products of a bf16 and an fp32 number are exact there, so that the codes are those
// of the definition, next to a border too): the conversions and products cost nothing that shows beside the memory (16 prompts
// of 1900 tokens, 64 heads on 8, d = 128, 1200 MB: 209 us, 5.7 TB/s; 96 single tokens 5.3 us, one 3.7).
template <int D>
__device__ __forceinline__ void rotary_kv_fp4(const RotaryArgs& ra, const PageUnit& at, int lp, int s0, int s1, int hg) {
    const AppendArgs& a = ra.a;
    constexpr int CPR = D / 8;
    constexpr int kPer = kPage * CPR;
    const int tid = threadIdx.x % kPer;
    const int h = hg * AppendLds<D>::kHeads + threadIdx.x / kPer;
    const bool head_ok = h < a.num_kv_heads;
    const int blk = a.block_tables[(int64_t)at.r * a.max_blocks + lp];
    const int s = tid / CPR, c = tid % CPR;
    const int64_t row = (int64_t)at.cu + (int64_t)lp * kPage - at.P + s;
    const int pos = lp * kPage + s;
    const bool ok = head_ok && s >= s0 && s < s1 && row >= 0 && row < a.total_tokens && pos < ra.num_positions;
    const int half = ra.rotary_dim / 16;
    const bool turned = c < 2 * half;
    u32x4 key = u32x4{0u, 0u, 0u, 0u}, v = key;
    float cs[8] = {}, sn[8] = {};
    if (ok) {
        key = *reinterpret_cast<const u32x4*>(a.k_new + row * ra.k_stride + h * D + c * 8);
        v = *reinterpret_cast<const u32x4*>(a.v_new + row * ra.v_stride + h * D + c * 8);
        if (turned) {
            const float* table = ra.table + (int64_t)pos * ra.rotary_dim;
            if (ra.interleaved)
                load_angles<4>(table + 8 * c, cs, sn);
            else
                load_angles<8>(table + 16 * (c < half ? c : c - half), cs, sn);
        }
    }
    float x[8], y[8];
    widen8(key, x);
    widen8(v, y);
    if (ra.interleaved) {
        if (turned) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const double p = x[2 * j], q = x[2 * j + 1], co = cs[j], si = sn[j];
                x[2 * j] = (float)fma(p, co, -(q * si));
                x[2 * j + 1] = (float)fma(q, co, p * si);
            }
        }
    } else {
        const int lane = threadIdx.x & 63;
        const int from = turned ? lane + (c < half ? half : -half) : lane;
        u32x4 other;
#pragma unroll
        for (int i = 0; i < 4; ++i) other[i] = (uint32_t)__shfl((int)key[i], from);
        if (turned) {
            float z[8];
            widen8(other, z);
            const double low = c < half ? -1.0 : 1.0;
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = (float)fma((double)x[j], (double)cs[j], low * ((double)z[j] * (double)sn[j]));
        }
    }
    const int64_t slot = ((int64_t)blk * a.num_kv_heads + h) * kPage + s;
    fp4_store<D>(static_cast<uint8_t*>(a.k_pool), static_cast<uint8_t*>(a.v_pool), ra.scales, slot, c, x, y,
                 ok && blk >= 0 && blk < a.num_blocks);
}

// kRotQHeads query heads (group qg) of the tokens of one page.
template <int D, bool STREAM>
__device__ __forceinline__ void rotary_q(const RotaryArgs& ra, const PageUnit& at, int lp, int s0, int s1, int qg) {
    constexpr int U = D / 16;  // pairs of chunks per head
    constexpr int kBatch = 4;  // heads whose loads a thread keeps in flight
    const int slots = s1 - s0;
    // Threads go over the slots, each over heads `step` apart: a head's lanes side by side, then `step` heads.
    const int span = slots <= 1 ? 1 : slots <= 2 ? 2 : slots <= 4 ? 4 : slots <= 8 ? 8 : 16;
    const int u = threadIdx.x % U;
    const int rest = threadIdx.x / U;
    const int step = kAppendThreads / (U * span);
    const int s = s0 + rest / step;
    const int64_t row = (int64_t)at.cu + (int64_t)lp * kPage - at.P + s;
    const int pos = lp * kPage + s;
    if (s >= s1 || row < 0 || row >= ra.a.total_tokens || pos >= ra.num_positions) return;
    const int half = ra.rotary_dim / 16;
    // This thread's two chunks, 8 elements each: so that the lanes of a head read and write adjacent ones.
    // Halves: the partners, or two of the rest; side by side: one of the head's lower half and one of its upper.
    const int c0 = ra.interleaved || u < half ? u : u + half;
    const int c1 = c0 + (ra.interleaved ? U : u < half ? half : U - half);
    const bool turned0 = c0 < 2 * half, turned1 = c1 < 2 * half;
    float cs[8] = {}, sn[8] = {};
    const float* const table = ra.table + (int64_t)pos * ra.rotary_dim;
    if (!ra.interleaved) {
        if (turned0) load_angles<8>(table + 16 * u, cs, sn);
    } else {
        if (turned0) load_angles<4>(table + 8 * c0, cs, sn);
        if (turned1) load_angles<4>(table + 8 * c1, cs + 4, sn + 4);
    }
    const int h_end = min((qg + 1) * kRotQHeads, ra.num_q_heads);
    const uint16_t* src = ra.q + row * ra.q_stride;
    uint16_t* dst = ra.q_out + row * ra.num_q_heads * D;
    for (int h0 = qg * kRotQHeads + rest % step; h0 < h_end; h0 += kBatch * step) {
        u32x4 w0[kBatch], w1[kBatch];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            const int h = h0 + b * step;
            if (h < h_end) {
                const u32x4* const p0 = reinterpret_cast<const u32x4*>(src + h * D + 8 * c0);
                const u32x4* const p1 = reinterpret_cast<const u32x4*>(src + h * D + 8 * c1);
                w0[b] = STREAM ? __builtin_nontemporal_load(p0) : *p0;
                w1[b] = STREAM ? __builtin_nontemporal_load(p1) : *p1;
            }
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            const int h = h0 + b * step;
            if (h >= h_end) break;
            float x[8], y[8];
            widen8(w0[b], x);
            widen8(w1[b], y);
            if (ra.interleaved) {
                turn_adjacent(x, cs, sn);
                turn_adjacent(y, cs + 4, sn + 4);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float lo = x[j], hi = y[j];
                    x[j] = fmaf(lo, cs[j], -(hi * sn[j]));
                    y[j] = fmaf(hi, cs[j], lo * sn[j]);
                }
            }
            if (turned0) w0[b] = pack8(x);
            if (turned1) w1[b] = pack8(y);
            __builtin_nontemporal_store(w0[b], reinterpret_cast<u32x4*>(dst + h * D + 8 * c0));
            __builtin_nontemporal_store(w1[b], reinterpret_cast<u32x4*>(dst + h * D + 8 * c1));
        }
    }
}

template <int D, Pool KIND, bool STREAM>
__global__ __launch_bounds__(kAppendThreads) void append_rotary_kernel(const RotaryArgs ra) {
    __shared__ AppendLds<D> lds;
    const AppendArgs& a = ra.a;
    // blockIdx.x = page jobs + job, or job pages + page
    const unsigned inner = ra.by_page ? ra.jobs : (unsigned)a.total_pages;
    const unsigned hi = blockIdx.x / inner, lo = blockIdx.x - hi * inner;
    const int u = (int)(ra.by_page ? hi : lo), job = (int)(ra.by_page ? lo : hi);
    PageUnit at;
    if (!locate_page<D>(a, lds, u, (int)gridDim.x, at)) return;
    const int lp = at.P / kPage + at.k;
    const int s0 = max(at.P - lp * kPage, 0);
    const int s1 = min(at.P + at.n - lp * kPage, kPage);
    if (lp >= a.max_blocks) return;
    const int kv_jobs = ceil_div(a.num_kv_heads, append_heads(D));
    if (job >= kv_jobs)
        rotary_q<D, STREAM>(ra, at, lp, s0, s1, job - kv_jobs);
    else if constexpr (KIND == Pool::kFp4)
        rotary_kv_fp4<D>(ra, at, lp, s0, s1, job);
    else
        rotary_kv<D, KIND == Pool::kFp8>(ra, lds, at, lp, s0, s1, job);
}

}  // namespace

int64_t rotary_workgroups(int64_t pages, int num_q_heads, int num_kv_heads, int head_dim, bool with_q) {
    return pages * (ceil_div(num_kv_heads, append_heads(head_dim)) + (with_q ? ceil_div(num_q_heads, kRotQHeads) : 0));
}

template <int D, Pool KIND>
static void launch_rotary(const RotaryArgs& ra, bool stream, unsigned grid, hipStream_t s) {
    if (stream)
        append_rotary_kernel<D, KIND, true><<<grid, kAppendThreads, 0, s>>>(ra);
    else
        append_rotary_kernel<D, KIND, false><<<grid, kAppendThreads, 0, s>>>(ra);
}

template <int D>
static void launch_rotary_kind(const RotaryArgs& ra, Pool kind, bool stream, unsigned grid, hipStream_t s) {
    if (kind == Pool::kFp4)
        launch_rotary<D, Pool::kFp4>(ra, stream, grid, s);
    else if (kind == Pool::kFp8)
        launch_rotary<D, Pool::kFp8>(ra, stream, grid, s);
    else
        launch_rotary<D, Pool::kBf16>(ra, stream, grid, s);
}

hipError_t launch_append_rotary(const RotaryArgs& args, int head_dim, Pool kind, hipStream_t s) {
    RotaryArgs ra = args;
    if (ra.a.total_pages <= 0) return hipSuccess;
    const bool with_q = ra.q != nullptr;
    ra.jobs = (unsigned)rotary_workgroups(1, ra.num_q_heads, ra.a.num_kv_heads, head_dim, with_q);
    ra.by_page = ra.a.total_tokens >= 2LL * ra.a.total_pages;
    const bool stream = with_q && (int64_t)ra.a.total_tokens * ra.num_q_heads * head_dim * 2 >= (192LL << 20);
    const unsigned grid = ra.jobs * (unsigned)ra.a.total_pages;
    if (head_dim == 128)
        launch_rotary_kind<128>(ra, kind, stream, grid, s);
    else
        launch_rotary_kind<64>(ra, kind, stream, grid, s);
    return hipGetLastError();
}

}  // namespace gc
