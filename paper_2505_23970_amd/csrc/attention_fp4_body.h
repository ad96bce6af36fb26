// Attention over 4-bit pools for gfx950 (device code of the small, 128-row and wide tiles): the same causal
// attention, work lists and merge as over the other pools (attention_small_body.h, attention_kernels.h), with the
// operands made for pages of E2M1 codes and block scales (fp4.h).
//
// Scores. The matrix cores take the key codes and their scales as they lie in the pool: a scaled product of
// 16 keys by 16 query rows over 128 elements, whose first operand is E2M1 with one scale per row and 32 elements.
// Its second operand has 8 bits at most, so a query row goes in twice, as two E4M3 numbers per element: with
// 2^E the row's scale (largest magnitude in [128, 256)),
//     h = E4M3(q 2^-E),   l = E4M3((q 2^-E - h) 2^5),   q = (h + l 2^-5) 2^E
// h has 4 significant bits and the rest of a bf16 number has 4, so the sum is q itself for elements from
// 2^-14 of the row's largest on, and off by at most 2^-22 of the largest below.
// Sums are fp32 but for one step inside the product: of the eight elements of a word of codes, those bits of each element's product are
// dropped (towards zero) that lie 2^-13 below the largest product of the eight (2^-12 where its code is 0.5; measured over
// codes, and by one element beside a larger one). Products have 6 bits, so only those under 2^-8 of the eight's largest lose any, and h's part
// of a score is off by at most the sum over its groups of eight of 7 * 2^-12 max |q k|, l's, at most 2^-4 of h, by 2^-4 of that; q's
// own error above adds 2^-22 max |q| sum |k|. That is less than the rounding to bf16 of the queries that make
// these maxima (2^-8 of them each). On random rows it is 2^-16 of sum |q k| at most (over bf16 pools 2^-24). Taken because the
// alternative is bf16 keys: a widening of every key, four times the LDS reads, for numbers that are 4-bit.
// Two such products take the time of the four bf16 ones they replace, and the keys need no conversion:
// with D = 64 one product takes both, keys twice along k against h and l.
// Operand layout of the product (lane group G = lane / 16, row or column lane % 16): the codes are elements
// 32 G .. + 31, with that lane's scale; the 8-bit operand's bytes are elements 16 G .. + 15 and 64 + 16 G .. + 15,
// with the scale of elements 32 G .. + 31 in lane group G.
// Values are widened to bf16 (exact) once per workgroup and tile, scales included, into rows of LDS,
// and read transposed (each 16 lanes a 16 x 4 block) as the V^T operand, with
//     O^T (D x rows) += V^T . P^T   in 16x16x32 bf16 products, as over the other pools.
// A value block that held a NaN makes the rows NaN that see its token and no other: in tiles where some row sees
// some key not, such blocks are zeroed and the rows that see them get the NaN afterwards.
#pragma once
#include "attention_kernels.h"
#include "fp4.h"

namespace gc {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) unsigned char lds_byte;

__device__ __forceinline__ f32x4 mfma_fp4_fp8(const u32x4 k, const i32x8 q, const f32x4 c, uint32_t k_scale, uint32_t q_scale) {
    const i32x8 a = {(int)k[0], (int)k[1], (int)k[2], (int)k[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q, c, 4, 0, 0, (int)k_scale, 0, (int)q_scale);
}

// A query row as operands of those products. D = 128: w[0] the h, w[1] the l; D = 64: both in w[0].
template <int D>
struct QueryRow {
    static constexpr int kParts = D / 64;
    i32x8 w[kParts];
    uint32_t scale[kParts];  // of the product's 32 elements of this lane group

    // q: the row (head_dim bf16 values); ok: false gives zeros
    __device__ __forceinline__ void load(const uint16_t* q, bool ok, int g4) {
        u32x4 x[2 * kParts];
#pragma unroll
        for (int i = 0; i < 2 * kParts; ++i)
            x[i] = ok ? *reinterpret_cast<const u32x4*>(q + 64 * (i >> 1) + 16 * g4 + 8 * (i & 1)) : u32x4{0u, 0u, 0u, 0u};
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 2 * kParts; ++i)
#pragma unroll
            for (int v = 0; v < 4; ++v) top = max(top, max(x[i][v] & 0x7FFFu, (x[i][v] >> 16) & 0x7FFFu));
        top = max(top, (uint32_t)__shfl_xor((int)top, 16));
        top = max(top, (uint32_t)__shfl_xor((int)top, 32));
        // largest magnitude 2^7 .. 2^8 in units of the scale; the l's scale is 2^-5 of it
        const uint32_t e = (uint32_t)max((int)(top >> 7) - 7, 6);
        const float inv = __uint_as_float((254u - e) << 23);
        uint32_t hi[4 * kParts], lo[4 * kParts];
#pragma unroll
        for (int i = 0; i < 4 * kParts; ++i) {
            // four elements
            const uint32_t w0 = x[i >> 1][2 * (i & 1)], w1 = x[i >> 1][2 * (i & 1) + 1];
            const float f0 = __uint_as_float(w0 << 16) * inv, f1 = __uint_as_float(w0 & 0xFFFF0000u) * inv;
            const float f2 = __uint_as_float(w1 << 16) * inv, f3 = __uint_as_float(w1 & 0xFFFF0000u) * inv;
            int h = __builtin_amdgcn_cvt_pk_fp8_f32(f0, f1, 0, false);
            h = __builtin_amdgcn_cvt_pk_fp8_f32(f2, f3, h, true);
            const auto b0 = __builtin_amdgcn_cvt_pk_f32_fp8(h, false);
            const auto b1 = __builtin_amdgcn_cvt_pk_f32_fp8(h, true);
            int l = __builtin_amdgcn_cvt_pk_fp8_f32((f0 - b0[0]) * 32.f, (f1 - b0[1]) * 32.f, 0, false);
            l = __builtin_amdgcn_cvt_pk_fp8_f32((f2 - b1[0]) * 32.f, (f3 - b1[1]) * 32.f, l, true);
            hi[i] = (uint32_t)h;
            lo[i] = (uint32_t)l;
        }
        if constexpr (D == 128) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[0][i] = (int)hi[i];
                w[kParts - 1][i] = (int)lo[i];
            }
            scale[0] = e;
            scale[kParts - 1] = e - 5;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[0][i] = (int)hi[i];
                w[0][4 + i] = (int)lo[i];
            }
            scale[0] = g4 < 2 ? e : e - 5;
        }
    }
    // scores of 16 keys (codes k and their scales, as this lane's operand)
    __device__ __forceinline__ f32x4 scores(const u32x4 k, uint32_t k_scale) const {
        f32x4 s = mfma_fp4_fp8(k, w[0], f32x4{0.f, 0.f, 0.f, 0.f}, k_scale, scale[0]);
        if constexpr (kParts == 2) s = mfma_fp4_fp8(k, w[1], s, k_scale, scale[1]);
        return s;
    }
};

// Value rows of a tile in LDS: row `key`, D bf16 values, whose 16-byte chunk `chunk` lies at this offset. Pieces of 32 bytes
// are swizzled by the row, so that the eight rows that 32 lanes read transposed lie in different banks, and their halves,
// so that eight lanes that write a chunk of eight rows (at D = 64: all even, or odd, ones of two) fall on different parts of
// 128 bytes (else a write takes twice as long).
template <int D>
__device__ __forceinline__ uint32_t value_at(int key, int chunk) {
    return (uint32_t)(key * 2 * D + (chunk ^ (D == 128 ? 2 * (key & 7) + (key >> 2 & 1) : key & 7)) * 16);
}
// Where a lane reads four elements of element block db (transposed, see below) of rows 4 (lane / 16) .. + 3.
template <int D>
__device__ __forceinline__ uint32_t value_from(int lane, int db) {
    return value_at<D>(4 * (lane >> 4) + ((lane & 15) >> 2), 2 * db + ((lane & 3) >> 1)) + 8 * (lane & 1);
}

// Four elements (keys) of one value column: lane i of 16 gives the address of elements 4 (i % 4) .. + 3 of row i / 4
// and gets column i of the four rows.
__device__ __forceinline__ u32x2 read_transposed(const unsigned char* at) {
    typedef __attribute__((address_space(3))) i16x4* lds_i16x4;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)(lds_byte*)at));
}

// Direct global->LDS copies with an address of their own per lane: lane i's 16 (4) bytes land at lds + 16 i (4 i).
// As dma16 (attention_kernels.h): the compiler does not track them, every wait is explicit.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy16(const unsigned char* from, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" :: "v"(from), "s"(lds) : "memory", "m0");
}
__device__ __forceinline__ void dma4(const unsigned char* base, uint32_t off, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" :: "v"(off), "s"(base), "s"(lds) : "memory", "m0");
}
__device__ __forceinline__ void copy4(const unsigned char* from, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" :: "v"(from), "s"(lds) : "memory", "m0");
}
#pragma clang diagnostic pop

// Codes of a page in LDS (D = 128): 16-byte block `block` of row `row` lies at block ^ code_swizzle(row) of it, so that
// the sixteen lanes of a 16-byte read (see value_at) lie in different banks, and the 32 of an 8-byte one (at D = 64
// they do without): 0, 2, 3, 1 for the rows 4 i .. 4 i + 3.
template <int D>
__device__ __forceinline__ int code_swizzle(int row) {
    const int q = row >> 2 & 3;
    return D == 128 ? q >> 1 | ((q ^ q >> 1) & 1) << 1 : 0;
}

// ---------------------------------------------------------------- small tiles
// Query tiles of 16 rows, key tiles of 32 (two pages), as over the other pools, but kFp4SmallWaves wavefronts a work item,
// which take its key tiles in turn and join their rows in LDS at the end: a tile is a chain of some thousand
// cycles (copies, widening, products, weights, transposition, products) for 4.3 KB, and one wavefront a SIMD waits through it
// (32 requests of 6500 tokens, 64 heads on 8, d = 128, 238 MB, with the merge: one wavefront an item 74.6 us, four 54).
// What bounds it: HBM, 49 us and 4.9 TB/s there (the copies alone, without the work: 44 us, 5.4), 4.4 for one request of 120000 tokens
// (131 MB, 30 us with the start and the end of the launch). A wavefront's next tile (pages of codes, 1 KiB at D = 128, and their scales) is copied into LDS
// while it works on the present one in registers: of the keys lane (row j, group G) holds block G of key j, 16 bytes and
// their scale, as the products take them; of the values 16 elements of key j for every 64 elements of a row, which
// go through 4 KiB of LDS for their transposition, 64 elements of the rows at a time.
constexpr int kFp4SmallWaves = 4;
template <int D>
struct Fp4SmallLds {
    static constexpr int kCodeBytes = kDecN * D / 2;  // of a tile's keys, or values
    static constexpr int kScaleBytes = 256;
    static constexpr int kTileBytes = 2 * kCodeBytes + kScaleBytes;
    static constexpr int kValueBytes = kDecN * 64 * 2;
    static_assert(kTileBytes + kValueBytes >= kDecM * D * 4, "the sums of 16 rows, at the end");
    __align__(16) unsigned char wave[kFp4SmallWaves][kTileBytes + kValueBytes];
    float m[kFp4SmallWaves][kDecM], l[kFp4SmallWaves][kDecM];
};

template <int D>
__device__ __forceinline__ void fp4_small_body(const Fp4AttnArgs& a, const WorkItem it, const int kvh, Fp4SmallLds<D>& lds) {
    constexpr int DB = D / 16;
    constexpr int NB = D / kFp4Block;
    constexpr int kPageCodes = kPage * D / 2;
    constexpr int kPageScales = kPage * NB * 2;
    constexpr int kCodeBytes = Fp4SmallLds<D>::kCodeBytes;
    constexpr int W = kFp4SmallWaves;
    constexpr int NH = D / 64;  // halves of a row, 64 elements each
    const int lane = threadIdx.x & 63;
    if (it.r < 0 || it.kt_begin >= it.kt_end) return;
    const int P = it.P, cu = it.cu, n = it.n;
    const int L = item_keys(it);
    const int ntok = min(a.tq, n - it.q0);
    const int g4 = lane >> 4, j = lane & 15;
    const int t = (int)((unsigned)j / (unsigned)a.group);
    const int hl = j - t * a.group;
    const bool row_ok = t < ntok;
    const int lim = P + it.q0 + (row_ok ? t : 0);
    const int64_t qrow = (int64_t)(cu + it.q0 + t) * a.num_q_heads + kvh * a.group + hl;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    unsigned char* const tile = lds.wave[wave];
    unsigned char* const vbuf = tile + Fp4SmallLds<D>::kTileBytes;
    const int kt_begin = it.kt_begin + wave, kt_end = it.kt_end;  // this wavefront's tiles: kt_begin, + W, ..

    const scalar_i32p table = (scalar_i32p)(a.block_tables + (int64_t)it.r * a.max_blocks);
    const uint32_t code_at = (uint32_t)(j * (D / 2) + ((g4 % NB) ^ code_swizzle<D>(j)) * 16);
    const uint32_t scale_at = (uint32_t)((j * NB + g4 % NB) * 2);
    uint32_t vcode_at[NH];  // elements 64 h + 16 g4 .. + 15
#pragma unroll
    for (int h = 0; h < NH; ++h) vcode_at[h] = (uint32_t)(j * (D / 2) + ((2 * h + (g4 >> 1)) ^ code_swizzle<D>(j)) * 16 + 8 * (g4 & 1));
    const uint32_t vscale_at = (uint32_t)((j * NB + (g4 >> 1)) * 2 + 1);  // + 4 h
    const unsigned char* const kbase = reinterpret_cast<const unsigned char*>(a.k_pool) + (int64_t)kvh * kPageCodes;
    const unsigned char* const vbase = reinterpret_cast<const unsigned char*>(a.v_pool) + (int64_t)kvh * kPageCodes;
    const unsigned char* const sbase = a.scales + (int64_t)kvh * kPageScales;
    // where each lane of a copy reads
    const int copy_row = lane / NB % kPage;
    const uint32_t code_from = (uint32_t)(copy_row * (D / 2) + ((lane % NB) ^ code_swizzle<D>(copy_row)) * 16);
    const uint32_t scale_from = (uint32_t)(lane % (kPageScales / 4) * 4);
    const uint32_t tile_at = __builtin_amdgcn_readfirstlane(lds_address(tile));

    // Block ids of a tile's two pages (scalar loads, fetched a tile ahead of their use). A page behind the last one (which
    // the table row holds: the plan has seen to that) stands for it, one with an id outside the pool is copied from
    // block 0: the keys behind the end are masked, their values zeroed.
    struct Ids {
        int b0, b1;
    };
    const int last_page = min((L - 1) / kPage, a.max_blocks - 1);
    auto fetch_ids = [&](int kt) -> Ids { return Ids{table[min(kt * 2, last_page)], table[min(kt * 2 + 1, last_page)]}; };
    const int64_t block_codes = (int64_t)a.num_kv_heads * kPageCodes;
    auto copy_tile = [&](const Ids& ids) {
        int64_t b[2];  // byte offsets of the pages' codes; of their scales an eighth
        static_assert(kPageScales * 8 == kPageCodes, "scales");
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const uint32_t id = (uint32_t)(p ? ids.b1 : ids.b0);
            b[p] = (int64_t)(id < (uint32_t)a.num_blocks ? id : 0u) * block_codes;
        }
        const uint32_t at = tile_at;
        if constexpr (D == 128) {
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                dma16(kbase + b[p], code_from, at + p * kPageCodes);
                dma16(vbase + b[p], code_from, at + kCodeBytes + p * kPageCodes);
            }
            copy4(sbase + (lane < 32 ? b[0] / 8 : b[1] / 8) + scale_from, at + 2 * kCodeBytes);
        } else {
            const int64_t mine = lane < 32 ? b[0] : b[1];
            copy16(kbase + mine + code_from, at);
            copy16(vbase + mine + code_from, at + kCodeBytes);
            copy4(sbase + (lane & 16 ? b[1] / 8 : b[0] / 8) + scale_from, at + 2 * kCodeBytes);  // (twice over)
        }
    };

    Ids next = fetch_ids(kt_begin);
    if (kt_begin < kt_end) copy_tile(next);
    next = fetch_ids(kt_begin + W);
    QueryRow<D> q;
    q.load(a.q + qrow * D, row_ok, g4);

    // where this lane puts 8 elements and reads transposed ones, of 64
    uint32_t v_to[2], v_from[4];
#pragma unroll
    for (int w = 0; w < 2; ++w) v_to[w] = value_at<64>(j, 2 * g4 + w);
#pragma unroll
    for (int db = 0; db < 4; ++db) v_from[db] = value_from<64>(lane, db);

    f32x4 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;
    const float c = a.scale_log2;
    const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};

    for (int kt = kt_begin; kt < kt_end; kt += W) {
        wait_copies<0>();
        u32x4 xk[2];
        u32x2 xv[NH][2];
        uint32_t xs[2], vs[NH][2];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            xk[p] = *reinterpret_cast<const u32x4*>(tile + p * kPageCodes + code_at);
            xs[p] = *reinterpret_cast<const uint16_t*>(tile + 2 * kCodeBytes + p * kPageScales + scale_at);
        }
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                xv[h][p] = *reinterpret_cast<const u32x2*>(tile + kCodeBytes + p * kPageCodes + vcode_at[h]);
                vs[h][p] = (tile + 2 * kCodeBytes + p * kPageScales)[vscale_at + 4 * h];
            }
        wait_lds_reads();
        if (kt + W < kt_end) {
            copy_tile(next);
            next = fetch_ids(kt + 2 * W);
        }

        const int key0 = kt * kDecN;
        const bool masked = key0 + kDecN - 1 > P + it.q0;  // some row does not see some key
        uint64_t nan[NH][2] = {};                          // lanes whose value block is NaN and within the sequence
        if (masked) {                                      // (values behind the end, and NaN, as zeros)
#pragma unroll
            for (int h = 0; h < NH; ++h)
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const bool in = key0 + kPage * p + j < L;
                    nan[h][p] = __ballot(in && vs[h][p] == kFp4Nan);
                    if (!in || vs[h][p] == kFp4Nan) {
                        xv[h][p] = u32x2{0u, 0u};
                        vs[h][p] = 127;
                    }
                }
        }
        // s[p][v] is the score of tile key 16 p + 4 g4 + v
        f32x4 s[2];
#pragma unroll
        for (int p = 0; p < 2; ++p) s[p] = q.scores(xk[p], xs[p]);
        auto put_values = [&](int h) {  // widened, into LDS
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    uint32_t b[4];
                    fp4_widen8(xv[h][p][w], fp4_scale(vs[h][p]), b);
                    *reinterpret_cast<u32x4*>(vbuf + v_to[w] + p * kPage * 128) = u32x4{b[0], b[1], b[2], b[3]};
                }
        };
        put_values(0);
        const int rel = lim - key0;
        if (masked) {
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int v = 0; v < 4; ++v) s[p][v] = (16 * p + 4 * g4 + v > rel) ? -INFINITY : s[p][v];
        }
        // (maxima that pass a NaN on, as it is the row's anyway, take three operands an instruction)
        float mx = s[0][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) mx = __builtin_elementwise_maximum(mx, s[e >> 2][e & 3]);
        {
            const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
            mx = __builtin_elementwise_maximum(__uint_as_float(x[0]), __uint_as_float(x[1]));
            const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
            mx = __builtin_elementwise_maximum(__uint_as_float(y[0]), __uint_as_float(y[1]));
        }
        const float m_new = __builtin_elementwise_maximum(m_run, mx * c);
        if (__any(m_new > m_run)) {
            const float alpha = m_new == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m_new);
            m_run = m_new;
            l_run *= alpha;
#pragma unroll
            for (int db = 0; db < DB; ++db) o[db] *= alpha;
        }
        const float m_use = (m_run == -INFINITY) ? 0.f : m_run;
        u32x4 pw;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float p0 = __builtin_amdgcn_exp2f(fmaf(s[i >> 1][2 * (i & 1)], c, -m_use));
            const float p1 = __builtin_amdgcn_exp2f(fmaf(s[i >> 1][2 * (i & 1) + 1], c, -m_use));
            const bf16x2 pair = {(__bf16)p0, (__bf16)p1};
            l_run = __builtin_amdgcn_fdot2_f32_bf16(pair, ones, l_run, false);
            pw[i] = __builtin_bit_cast(uint32_t, pair);
        }
        const bf16x8 pf = __builtin_bit_cast(bf16x8, pw);
#pragma unroll
        for (int h = 0; h < NH; ++h) {
            if (h > 0) put_values(h);
            wave_lds_sync();
#pragma unroll
            for (int db = 0; db < 4; ++db) {
                const u32x2 lo = read_transposed(vbuf + v_from[db]);
                const u32x2 hi = read_transposed(vbuf + v_from[db] + kPage * 128);
                const bf16x8 vf = __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
                o[4 * h + db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf, o[4 * h + db], 0, 0, 0);
            }
            wave_lds_sync();
        }
        if (masked) {
            // value blocks that held a NaN: bit 16 g + j of nan[h][p] is key 16 p + j, block 2 h + g / 2
#pragma unroll
            for (int h = 0; h < NH; ++h)
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    if (nan[h][p] == 0) continue;
                    const int seen = rel - kPage * p;  // keys 0 .. seen of the page
                    const uint32_t sees = seen < 0 ? 0u : 0xFFFFu >> (15 - min(seen, 15));
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const float add = ((uint32_t)(nan[h][p] >> (32 * b)) & sees) != 0 ? __builtin_nanf("") : 0.f;
#pragma unroll
                        for (int v = 0; v < 4; ++v) {
                            o[4 * h + 2 * b][v] += add;
                            o[4 * h + 2 * b + 1][v] += add;
                        }
                    }
                }
        }
    }

    float l_tot = row_sum4(l_run);
    constexpr int kOwn = DB / W;  // element blocks whose sums this wavefront joins and writes: from kOwn wave on
    f32x4 mine[kOwn];
    if constexpr (W == 1) {
#pragma unroll
        for (int db = 0; db < DB; ++db) mine[db] = o[db];
    } else {
        // rows in units of 2^m of their own: joined in wavefront order
        f32x4* const at = reinterpret_cast<f32x4*>(tile);
#pragma unroll
        for (int db = 0; db < DB; ++db) at[db * 64 + lane] = o[db];
        if (g4 == 0) {
            lds.m[wave][j] = m_run;
            lds.l[wave][j] = l_tot;
        }
        __syncthreads();
        float m = lds.m[0][j];
#pragma unroll
        for (int w = 1; w < W; ++w) m = fmaxf(m, lds.m[w][j]);
        m_run = m;
        l_tot = 0.f;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) mine[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(lds.m[w][j] - m);
            l_tot = fmaf(lds.l[w][j], alpha, l_tot);
            const f32x4* const from = reinterpret_cast<const f32x4*>(lds.wave[w]) + kOwn * wave * 64 + lane;
#pragma unroll
            for (int i = 0; i < kOwn; ++i) mine[i] += from[i * 64] * alpha;
        }
    }
    const float inv = l_tot > 0.f ? 1.f / l_tot : 0.f;
    // (a split item passes a NaN sum on to the merge)
    const float lse_v = l_tot > 0.f ? (m_run + log2f(l_tot)) * kLn2 : (it.part >= 0 && l_tot != l_tot ? l_tot : -INFINITY);
    // mine[i][v] is element d = 16 (kOwn wave + i) + 4 g4 + v of row j
    if (!row_ok) return;
    const int d0 = 16 * kOwn * wave + 4 * g4;
    const bool first = wave == 0 && g4 == 0;
    if (it.part < 0) {
        uint16_t* op = a.out + qrow * D + d0;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            u32x2 w;
            w[0] = pack_pair(mine[i][0] * inv, mine[i][1] * inv);
            w[1] = pack_pair(mine[i][2] * inv, mine[i][3] * inv);
            *reinterpret_cast<u32x2*>(op + 16 * i) = w;
        }
        if (a.lse != nullptr && first) a.lse[qrow] = lse_v;
    } else {
        const int64_t prow = ((int64_t)it.part * a.num_kv_heads + kvh) * kDecM + j;
        float* po = a.part_o + prow * D + d0;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) *reinterpret_cast<f32x4*>(po + 16 * i) = mine[i] * inv;
        if (first) a.part_lse[prow] = lse_v;
    }
}

// ---------------------------------------------------------------- 128-row and wide tiles
// Query tiles of 32 rows a wavefront, key tiles of 64 (four pages). Pages of codes and of scales are copied straight into
// LDS, two tiles ahead; keys are multiplied as they are, values are widened from there into rows of bf16, a tile ahead.
// What bounds it: the matrix cores and, beside them, the softmax's vector instructions. 6 prompts of 800 tokens on 9000, 64 heads
// on 8, d = 128 (wide tiles, 1.09 TFLOP): 805-833 us by card, 1310-1360 TFLOP/s, matrix cores busy 60-62 % of the time (830 where bf16 pools take 881).
// 8 requests of 288 on 2560, 32 heads on 8 (128-row tiles): 102-105 us by card, of which the slot that ends last has 60 key tiles on a mean
// of 46. At d = 64 (24 requests of 20 on 3000) 35-36 us: matrix cores busy 29 % of the cycles, the vector unit about half,
// little of it at once with two wavefronts a SIMD; copies three tiles ahead, or three workgroups a compute unit, change nothing.
template <int D, int WAVES>
struct Fp4Lds {
    static constexpr int kSlots = 4;  // tiles t to t + 2 are in use, and the scales of t - 1
    static constexpr int kValueBuffers = WAVES == kWideWaves ? 3 : 2;
    static constexpr int kValueBytes = kBlockN * D * 2;
    static constexpr int kCodeBytes = kBlockN * D / 2;
    static constexpr int kScaleBytes = kBlockN * (D / kFp4Block) * 2;
    __align__(16) unsigned char v[kValueBuffers][kValueBytes];
    __align__(16) unsigned char kc[kSlots][kCodeBytes], vc[kSlots][kCodeBytes];  // codes of keys and of values
    __align__(16) unsigned char s[kSlots][kScaleBytes];
};

// Work item `it` by this wavefront, which has RB 16-row blocks of the tile. Wavefronts with one block and with two meet at the same
// barriers.
template <int D, int WAVES, int RB>
__device__ __forceinline__ void fp4_attention_rows(const Fp4AttnArgs& a, const WorkItem it, const int kvh, Fp4Lds<D, WAVES>& lds) {
    constexpr int ROWS = 16 * RB;
    constexpr int KB = kBlockN / 16;   // key blocks (pages) of a tile
    constexpr int DB = D / 16;
    constexpr int NB = D / kFp4Block;
    constexpr int kPageCodes = kPage * D / 2;
    constexpr int kPageScales = kPage * NB * 2;
    constexpr int kTileLog2Thresh = 8;
    // Value fragments read ahead of their products (wide tiles: 2 and 3 take 830 us on the prompts above, 4 844, 5 860, 1 835;
    // 128-row tiles: 2 to 4 the same).
    constexpr int kAhead = 3;

    int tid_opaque = (int)threadIdx.x;  // (lane constants per work item, not held across a resident launch's items)
    asm volatile("" : "+v"(tid_opaque));
    const int tid = tid_opaque, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g4 = lane >> 4, j16 = lane & 15;
    const int P = it.P, cu = it.cu, n = it.n;
    const int L = item_keys(it);
    const int ntok = min(a.tq, n - it.q0);

    // row of the tile of this wavefront's row
    auto row_of = [&](int row) { return WAVES == kWideWaves ? wave * ROWS + row : 16 * (wave + (row >> 4) * WAVES) + (row & 15); };
    bool row_ok[RB];
    int lim[RB];  // last key the row may see
    int64_t qrow[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int m = row_of(16 * rb + j16);
        const int t = (int)((unsigned)m / (unsigned)a.group);
        row_ok[rb] = t < ntok;
        lim[rb] = P + it.q0 + (row_ok[rb] ? t : 0);
        qrow[rb] = (int64_t)(cu + it.q0 + t) * a.num_q_heads + kvh * a.group + (m - t * a.group);
    }

    // Block ids: lane l of `ids` holds that of page 64 i + l of the item (from its first tile on), of `ids_next` the next 64.
    // A page behind the last one (which the table row holds: the plan has seen to that) stands for it, one with an id
    // outside the pool is taken from block 0: the keys behind the end are masked, their values zeroed.
    const int32_t* const table = a.block_tables + (int64_t)it.r * a.max_blocks;
    const int last_page = min((L - 1) / kPage, a.max_blocks - 1);
    auto fetch_ids = [&](int i) -> int { return table[(uint32_t)min(it.kt_begin * 4 + 64 * i + lane, last_page)]; };
    const int64_t block_codes = (int64_t)a.num_kv_heads * kPageCodes;
    int ids = fetch_ids(0), ids_next = ids;

    QueryRow<D> q[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) q[rb].load(a.q + qrow[rb] * D, row_ok[rb], g4);

    // Copies of a tile (its number counts from the item's first): a wavefront brings parts of page w % 4: codes, lane i the
    // 16-byte block i % NB (swizzled) of row i / NB, of its keys and of its values, and its scales. Of 8 wavefronts the first four,
    // which are half a tile ahead (see turns), bring what is needed first, values and scales, the others the keys.
    const unsigned char* const kbase = reinterpret_cast<const unsigned char*>(a.k_pool) + (int64_t)kvh * kPageCodes;
    const unsigned char* const vbase = reinterpret_cast<const unsigned char*>(a.v_pool) + (int64_t)kvh * kPageCodes;
    const unsigned char* const sbase = a.scales + (int64_t)kvh * kPageScales;
    using Lds = Fp4Lds<D, WAVES>;
    const uint32_t kc_lds = __builtin_amdgcn_readfirstlane(lds_address(lds.kc[0]) + (wave & 3) * kPageCodes);
    const uint32_t vc_lds = __builtin_amdgcn_readfirstlane(lds_address(lds.vc[0]) + (wave & 3) * kPageCodes);
    const uint32_t s_lds = __builtin_amdgcn_readfirstlane(lds_address(lds.s[0]) + (wave & 3) * kPageScales);
    const int copy_row = lane / NB % kPage;
    const uint32_t code_from = (uint32_t)(copy_row * (D / 2) + ((lane % NB) ^ code_swizzle<D>(copy_row)) * 16);
    auto copy_tile = [&](int tile) {
        const uint32_t id = (uint32_t)__builtin_amdgcn_readlane(ids, tile * 4 % 64 + (wave & 3));
        const int64_t at = (int64_t)(id < (uint32_t)a.num_blocks ? id : 0u) * block_codes;
        const uint32_t to = (uint32_t)(tile % Lds::kSlots);
        static_assert(kPageScales * 8 == kPageCodes, "offsets of scales");
        if (lane < kPageCodes / 16) {
            if (WAVES == 4 || wave < 4) dma16(vbase + at, code_from, vc_lds + to * Lds::kCodeBytes);
            if (WAVES == 4 || wave >= 4) dma16(kbase + at, code_from, kc_lds + to * Lds::kCodeBytes);
        }
        if ((WAVES == 4 || wave < 4) && lane < kPageScales / 4) dma4(sbase + at / 8, 4u * lane, s_lds + to * Lds::kScaleBytes);
        if (tile % 16 == 15) {
            ids = ids_next;
            ids_next = fetch_ids(tile / 16 + 2);
        }
    };
    // Values: a thread widens kPer elements of one row and block; at D = 128 neighbouring lanes take neighbouring rows (value_at).
    constexpr int kPer = kBlockN * D / (WAVES * 64);  // 32, 16 or 8
    constexpr int kWords = kPer / 8;
    constexpr int kRowsOfWave = 64 * kPer / D;
    const int v_key = D == 128 ? wave * kRowsOfWave + lane % kRowsOfWave : tid * kPer / D;
    const int v_el = D == 128 ? lane / kRowsOfWave * kPer : tid * kPer % D;
    const uint32_t vc_at = (uint32_t)(v_key * (D / 2) + ((v_el / 32) ^ code_swizzle<D>(v_key)) * 16 + v_el % 32 / 2);
    const uint32_t vs_at = (uint32_t)((v_key * NB + v_el / kFp4Block) * 2 + 1);
    uint32_t v_to[kWords];
#pragma unroll
    for (int w = 0; w < kWords; ++w) v_to[w] = value_at<D>(v_key, v_el / 8 + w);
    uint32_t vc[kWords], vs = 0;
    auto read_codes = [&](int tile) {
        const unsigned char* const from = lds.vc[0] + tile % Lds::kSlots * Lds::kCodeBytes + vc_at;
        if constexpr (kWords == 4) {
            const u32x4 w = *reinterpret_cast<const u32x4*>(from);
#pragma unroll
            for (int i = 0; i < 4; ++i) vc[i] = w[i];
        } else if constexpr (kWords == 2) {
            const u32x2 w = *reinterpret_cast<const u32x2*>(from);
            vc[0] = w[0];
            vc[1] = w[1];
        } else {
            vc[0] = *reinterpret_cast<const uint32_t*>(from);
        }
        vs = (lds.s[0] + tile % Lds::kSlots * Lds::kScaleBytes)[vs_at];
    };
    const int first_masked = P + it.q0;  // tiles that reach past this key hide some key from some row
    auto put_values = [&](int buf, int tile) {
        const int key0 = (it.kt_begin + tile) * kBlockN;
        if (key0 + kBlockN - 1 > first_masked && (key0 + v_key >= L || vs == kFp4Nan)) {
#pragma unroll
            for (int w = 0; w < kWords; ++w) vc[w] = 0;  // (values behind the end, and NaN, as zeros)
            vs = 127;
        }
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
            uint32_t b[4];
            fp4_widen8(vc[w], fp4_scale(vs), b);
            *reinterpret_cast<u32x4*>(lds.v[0] + buf * Lds::kValueBytes + v_to[w]) = u32x4{b[0], b[1], b[2], b[3]};
        }
    };

    f32x4 o[RB][DB];
    float m_run[RB], neg_off[RB];
    bool need_max, exact = false;  // (the exponent offset, as in attention_kernels.h)
    const float c = a.scale_log2;
    // Row sums of the (rounded) weights by products with ones: every element of l_run[rb] is its column's sum. Dot products
    // of the vector unit share the matrix cores: one took 54 to 86 cycles beside another wavefront's products.
    const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u});
    f32x4 l_run[RB];

    const uint32_t k_at = (uint32_t)(j16 * (D / 2) + ((g4 % NB) ^ code_swizzle<D>(j16)) * 16);
    const uint32_t s_at = (uint32_t)((j16 * NB + g4 % NB) * 2);
    uint32_t v_from[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) v_from[db] = value_from<D>(lane, db);

    f32x4 s[RB][KB];     // s[rb][b][v] is the score of row 16 rb + j16 and tile key 16 b + 4 g4 + v
    bf16x8 pf[RB][2];    // the weights, as operands of the products with the values
    bf16x8 vf[2 * DB];   // value fragment i: keys 32 (i / DB) .. + 31, elements 16 (i % DB) .. + 15
    u32x4 kf[KB];        // key fragments and their scales
    uint32_t ks[KB];
    auto kread = [&](int tile) {
        const uint32_t in = (uint32_t)(tile % Lds::kSlots);
#pragma unroll
        for (int b = 0; b < KB; ++b) {
            kf[b] = *reinterpret_cast<const u32x4*>(lds.kc[0] + in * Lds::kCodeBytes + b * kPageCodes + k_at);
            ks[b] = *reinterpret_cast<const uint16_t*>(lds.s[0] + in * Lds::kScaleBytes + b * kPageScales + s_at);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto scores = [&]() {
#pragma unroll
        for (int part = 0; part < QueryRow<D>::kParts; ++part)
#pragma unroll
            for (int b = 0; b < KB; ++b) {
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
                    s[rb][b] = mfma_fp4_fp8(kf[b], q[rb].w[part], part == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[rb][b], ks[b], q[rb].scale[part]);
                __builtin_amdgcn_sched_barrier(0);
            }
    };
    auto vread = [&](int buf, int i) {
        const unsigned char* const at = lds.v[0] + buf * Lds::kValueBytes + v_from[i % DB] + (i / DB) * 2 * kPage * 2 * D;
        const u32x2 lo = read_transposed(at), hi = read_transposed(at + kPage * 2 * D);
        vf[i] = __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
    };
    // masks the tile's scores and, where a row has no exponent offset yet (or in the exact pass), takes it
    auto offsets = [&](int tile) {
        const int key0 = (it.kt_begin + tile) * kBlockN;
        if (key0 + kBlockN - 1 > first_masked) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                const int rel = lim[rb] - key0 - 4 * g4;
#pragma unroll
                for (int b = 0; b < KB; ++b)
#pragma unroll
                    for (int v = 0; v < 4; ++v) s[rb][b][v] = (16 * b + v > rel) ? -INFINITY : s[rb][b][v];
            }
        }
        if (need_max) {
            need_max = exact;
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                float mx = s[rb][0][0];
#pragma unroll
                for (int e = 1; e < 4 * KB; ++e) mx = __builtin_elementwise_maximum(mx, s[rb][e >> 2][e & 3]);
                {
                    const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
                    mx = __builtin_elementwise_maximum(__uint_as_float(x[0]), __uint_as_float(x[1]));
                    const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
                    mx = __builtin_elementwise_maximum(__uint_as_float(y[0]), __uint_as_float(y[1]));
                }
                const float m_tile = mx * c;
                if (__any(m_tile > m_run[rb] + kTileLog2Thresh)) {
                    const float m_new = fmaxf(m_run[rb], m_tile);
                    const float alpha = m_new == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run[rb] - m_new);
                    m_run[rb] = m_new;
                    l_run[rb] *= alpha;
#pragma unroll
                    for (int db = 0; db < DB; ++db) o[rb][db] *= alpha;
                }
                need_max |= __any(m_run[rb] == -INFINITY);
                neg_off[rb] = m_run[rb] == -INFINITY ? 0.f : -m_run[rb];
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // pair x of a half's eight weights of a row, as bf16
    auto w_pair = [&](int rb, int hb, int x) {
        const f32x4 y = s[rb][2 * hb + (x >> 1)];
        const bf16x2 pq = {(__bf16)__builtin_amdgcn_exp2f(fmaf(y[2 * (x & 1)], c, neg_off[rb])),
                           (__bf16)__builtin_amdgcn_exp2f(fmaf(y[2 * (x & 1) + 1], c, neg_off[rb]))};
        pf[rb][hb][2 * x] = pq[0];
        pf[rb][hb][2 * x + 1] = pq[1];
    };
    auto weights = [&](int hb) {
#pragma unroll
        for (int x = 0; x < 4 * RB; ++x) w_pair(x % RB, hb, x / RB);
    };
    auto value_products = [&](int buf, int i) {
        if (i + kAhead < 2 * DB) vread(buf, i + kAhead);
        if (i % DB == 0) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) l_run[rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[rb][i / DB], l_run[rb], 0, 0, 0);
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
            o[rb][i % DB] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[i], pf[rb][i / DB], o[rb][i % DB], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    // value blocks that held a NaN, in a tile where some row sees some key not (lane = key of the tile)
    auto nan_values = [&](int tile) {
        const int key0 = (it.kt_begin + tile) * kBlockN;
        if (key0 + kBlockN - 1 <= first_masked) return;
        const unsigned char* const sb = lds.s[0] + tile % Lds::kSlots * Lds::kScaleBytes;
        uint64_t nan[NB];
        uint64_t any = 0;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            nan[b] = __ballot(key0 + lane < L && sb[(lane * NB + b) * 2 + 1] == kFp4Nan);
            any |= nan[b];
        }
        if (any != 0) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                const int seen = lim[rb] - key0;  // keys 0 .. seen of the tile
                const uint64_t sees = seen < 0 ? 0ull : ~0ull >> (63 - min(seen, 63));
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    const float add = (nan[db / 2] & sees) != 0 ? __builtin_nanf("") : 0.f;
#pragma unroll
                    for (int v = 0; v < 4; ++v) o[rb][db][v] += add;
                }
            }
        }
    };

    const int tiles = it.kt_end - it.kt_begin;
    int tile = 0;
    // 4 wavefronts: tile after tile, another workgroup's wavefronts beside them. The first half's weights as a block, a
    // quarter of the second half's after every quarter of the products with the first (attention_kernels.h).
    auto step = [&](const int cur) {
        kread(tile);
        if (tile + 1 < tiles) read_codes(tile + 1);
        if (tile + 2 < tiles) copy_tile(tile + 2);
        __builtin_amdgcn_sched_barrier(0);
        scores();
#pragma unroll
        for (int i = 0; i < kAhead; ++i) vread(cur, i);
        __builtin_amdgcn_sched_barrier(0);
        if (tile + 1 < tiles) put_values(1 - cur, tile + 1);
        __builtin_amdgcn_sched_barrier(0);
        offsets(tile);
        weights(0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 2 * DB; ++i) {
            value_products(cur, i);
            if (i < DB && i % (DB / 4) == DB / 4 - 1) {
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) w_pair(rb, 1, i / (DB / 4));
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        nan_values(tile);
        wait_vmem<0>();
        __syncthreads();
    };
    // 8 wavefronts: in turns. The two wavefronts of a SIMD are half a tile apart: while one multiplies (the values of
    // tile t, then the keys of tile t + 1), the other computes weights and widens the values of the next tile, and at a barrier
    // they change. In the turns 0, 1, .. the wavefronts ahead multiply in 2 t + 2 and weigh tile t in 2 t + 1, those behind a
    // turn later. So
    //   - values of t + 1 are written in turns 2 t + 1 and 2 t + 2, and read in 2 t + 4 and 2 t + 5: three buffers;
    //   - codes of tile t + 2 are asked for in turn 2 t + 1 (values, scales) and 2 t + 2 (keys), waited for at the end of the
    //     turn after, and needed from turn 2 t + 3 (values, scales) and 2 t + 4 (keys) on; what lay there was tile t - 2's,
    //     whose scales were read last in turn 2 t - 1.
    // Both halves pass the same number of barriers. The last one of those ahead comes before the last products of those
    // behind: whoever writes to the value buffers after turns() needs a barrier of its own.
    auto change = [&]() {  // (this wavefront's writes to LDS are over; the reads of the first value fragments may go on)
        static_assert(2 * kAhead == 6, "the wait");
        asm volatile("s_waitcnt lgkmcnt(6)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    auto turns = [&]() {
        int buf = 0;
        if (wave >= WAVES / 2) change();
        __builtin_amdgcn_s_setprio(2);
        kread(0);
        scores();
        wait_vmem<0>();
        change();
        while (true) {
            __builtin_amdgcn_s_setprio(0);
            const int next = buf == 2 ? 0 : buf + 1;
            const bool more = tile + 1 < tiles;
            if (more) read_codes(tile + 1);
            if (tile + 2 < tiles) copy_tile(tile + 2);
            offsets(tile);
            if (more) put_values(next, tile + 1);
            weights(0);
            weights(1);
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) asm volatile("" : "+v"(pf[rb][0]), "+v"(pf[rb][1]));  // (in this turn)
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) vread(buf, i);
            change();
            __builtin_amdgcn_s_setprio(2);
#pragma unroll
            for (int i = 0; i < 2 * DB; ++i) {
                value_products(buf, i);
                if (i == 2 * DB - kAhead && more) kread(tile + 1);
            }
            nan_values(tile);
            buf = next;
            ++tile;
            if (!more) break;
            scores();
            wait_vmem<0>();
            change();
        }
        __builtin_amdgcn_s_setprio(0);
        if (wave < WAVES / 2) change();
    };
    for (;;) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
            for (int db = 0; db < DB; ++db) o[rb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
            m_run[rb] = -INFINITY;
            neg_off[rb] = 0.f;
            l_run[rb] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        need_max = true;
        tile = 0;
        if (exact) ids = fetch_ids(0);
        ids_next = fetch_ids(1);
        copy_tile(0);
        wait_vmem<0>();
        __syncthreads();
        read_codes(0);
        if (tiles > 1) copy_tile(1);
        put_values(0, 0);
        wait_vmem<0>();
        __syncthreads();
        if constexpr (WAVES == kWideWaves) {
            turns();
        } else {
            while (true) {
                step(0);
                if (++tile >= tiles) break;
                step(1);
                if (++tile >= tiles) break;
            }
        }
        // (A barrier after either pass: wavefronts behind leave turns() with value reads that no barrier has followed, of the
        // buffers that the others then stage their output rows in.)
        if (exact) {
            __syncthreads();
            break;
        }
        if (!__syncthreads_or(!(l_run[0][0] <= 0x1p100f) || !(l_run[RB - 1][0] <= 0x1p100f))) break;
        exact = true;
    }

    float inv[RB], lse_v[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const float l = l_run[rb][0];
        inv[rb] = l > 0.f ? 1.f / l : 0.f;
        lse_v[rb] = l > 0.f ? (m_run[rb] + log2f(l)) * kLn2 : (it.part >= 0 && l != l ? l : -INFINITY);
    }
    // o[rb][db][v] is element d = 16 db + 4 g4 + v of row 16 rb + j16. Rows go through LDS (the values' buffers, no longer
    // read), so that a store covers whole rows: each wavefront a part of its own, as many of its rows at a time as fit.
    constexpr int kStage = 2 * Fp4Lds<D, WAVES>::kValueBytes / WAVES;  // (two of the buffers)
    unsigned char* const stage = lds.v[0] + wave * kStage;
    auto through_stage = [&](auto out_bytes, auto&& put, auto&& get) {
        constexpr int kOutRow = decltype(out_bytes)::value;
        constexpr int CH = kOutRow / 16;
        constexpr int kRows = kStage / kOutRow < ROWS ? kStage / kOutRow : ROWS;
        constexpr int kSw = (CH < 16 ? CH : 16) - 1;  // chunk swizzle
        static_assert(ROWS % kRows == 0 && kRows * CH % 64 == 0, "stage");
#pragma unroll
        for (int r0 = 0; r0 < ROWS; r0 += kRows) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                const int sr = 16 * rb + j16 - r0;
                if (sr < 0 || sr >= kRows) continue;
#pragma unroll
                for (int db = 0; db < DB; ++db)
                    put(rb, db, [&](int ch) { return stage + sr * kOutRow + (ch ^ (sr & kSw)) * 16; });
            }
            wave_lds_sync();
#pragma unroll
            for (int i = 0; i < kRows * CH / 64; ++i) {
                const int x = i * 64 + lane, sr = x / CH, ch = x % CH;
                get(r0 + sr, ch, *reinterpret_cast<const u32x4*>(stage + sr * kOutRow + (ch ^ (sr & kSw)) * 16));
            }
            wave_lds_sync();
        }
    };
    if (it.part < 0) {
        through_stage(std::integral_constant<int, 2 * D>{},
            [&](int rb, int db, auto&& at) {
                u32x2 w;
                w[0] = pack_bf16x2(o[rb][db][0] * inv[rb], o[rb][db][1] * inv[rb]);
                w[1] = pack_bf16x2(o[rb][db][2] * inv[rb], o[rb][db][3] * inv[rb]);
                *reinterpret_cast<u32x2*>(at(2 * db + (g4 >> 1)) + 8 * (g4 & 1)) = w;
            },
            [&](int row, int ch, const u32x4 w) {
                const int m = row_of(row);
                const int t = (int)((unsigned)m / (unsigned)a.group);
                if (t < ntok)
                    *reinterpret_cast<u32x4*>(a.out + ((int64_t)(cu + it.q0 + t) * a.num_q_heads + kvh * a.group + (m - t * a.group)) * D + ch * 8) = w;
            });
        if (a.lse != nullptr && g4 == 0) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
                if (row_ok[rb]) a.lse[qrow[rb]] = lse_v[rb];
        }
    } else {
        const int64_t prow0 = ((int64_t)it.part * a.num_kv_heads + kvh) * (WAVES * kRowsPerWave);
        through_stage(std::integral_constant<int, 4 * D>{},
            [&](int rb, int db, auto&& at) { *reinterpret_cast<f32x4*>(at(4 * db + g4)) = o[rb][db] * inv[rb]; },
            [&](int row, int ch, const u32x4 w) {
                const int m = row_of(row);
                if (m < ntok * a.group) *reinterpret_cast<u32x4*>(a.part_o + (prow0 + m) * D + ch * 4) = w;
            });
        if (g4 == 0) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) a.part_lse[prow0 + row_of(16 * rb + j16)] = lse_v[rb];
        }
    }
}

// Rows of a tile: 8 wavefronts take 32 in a row each. Of 4, wavefront w takes the 16-row blocks w and w + 4, and only the first where
// the second is empty: a tile of up to 64 rows costs half (24 requests of 10 tokens, 32 heads on 8, d = 64: 33.5 -> 23.8 us; of 20
// tokens 38 -> 36). Full tiles pay for it: with the merge, one card, 8 requests of 288, d = 128, 102.7 -> 105.0.
template <int D, int WAVES>
__device__ __forceinline__ void fp4_attention_body(const Fp4AttnArgs& a, const unsigned bid, Fp4Lds<D, WAVES>& lds) {
    constexpr int RB = kRowsPerWave / 16;
    // (4 wavefronts: one of the two workgroups on a compute unit is preferred, attention_kernels.h)
    if (WAVES != kWideWaves && D == 128 && (bid / a.prefer_span & 1) == a.prefer_odd) __builtin_amdgcn_s_setprio(2);
    const int kvh = (int)(bid % (unsigned)a.num_kv_heads);
    const WorkItem it = a.items[bid / (unsigned)a.num_kv_heads];
    asm volatile("" ::"s"(it.r), "s"(it.q0), "s"(it.kt_begin), "s"(it.kt_end), "s"(it.part), "s"(it.P), "s"(it.cu), "s"(it.n));
    if (it.r < 0 || it.kt_begin >= it.kt_end) return;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if constexpr (WAVES == kWideWaves) {
        fp4_attention_rows<D, WAVES, RB>(a, it, kvh, lds);
    } else {
        static_assert(RB == 2, "row blocks");
        if (__builtin_expect(16 * (wave + WAVES) < min(a.tq, it.n - it.q0) * a.group, 1)) fp4_attention_rows<D, WAVES, 2>(a, it, kvh, lds);
        else fp4_attention_rows<D, WAVES, 1>(a, it, kvh, lds);
    }
}

}  // namespace
}  // namespace gc
