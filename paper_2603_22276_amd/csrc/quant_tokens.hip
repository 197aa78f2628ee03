// Forward of a few tokens over a 4-bit weight (decode):  y = g (.) (x W^T + s h B^T) (+ bias), h summed from its slices, in one
// launch behind the one that forms those.  Bound: reading W once (d_out d_in / 2 bytes and the scales), and latency.
//
// A workgroup owns 16 MR rows of W; its waves take the blocks of 128 columns in turn, each with an LDS ring of its own for codes
// and token rows (buffer_load ... lds, no barrier: only its own vmcnt).  Codes become 16-bit integers (or E2M1 floats) exactly,
// products are summed in fp32 within a group, and the group's sum is multiplied by the scale in fp32: no weight is rounded,
// whatever the scale.  A zero point enters as the addend of the group's first MFMA, its negative times the sum of x over the group,
// which one more MFMA against a constant gives for all rows (-8 times it where the zero point is the same everywhere).  Which columns
// a lane multiplies in a k-step is free as long as the x fragments take the same ones and a k-step stays within a group: a lane's share
// of a group is consecutive, so it is one read of 16, 8 or 4 bytes of codes.
//
// Codes and x straight from memory in the MFMA's own layout, without the LDS: sixteen lanes in a row then are sixteen rows, each
// a line of its own to the L1 (14336 x 4096, r 8, 27 tokens, codes from memory 25 us, 20 this way).  Scales and zero points one at
// a time from memory cost the same way; they come through the LDS, a piece of the columns at a time.
#include "quant_codes.hpp"

namespace dora {
namespace {

// all LDS reads so far, these fragments among them
template <int TB>
__device__ __forceinline__ void landed(bf16x8_t (&f)[TB])
{
    static_assert(TB == 1 || TB == 2, "blocks of tokens");
    if constexpr (TB == 1) asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(f[0]));
    else asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(f[0]), "+v"(f[1]));
}

// A wave's ring slot: MR blocks of 16 rows of W, 64 bytes of codes each, then XR token rows of 256 bytes, in chunks of 16 bytes.
// Chunks are swizzled so that the sixteen rows of a fragment lie in different banks.
template <int MR, int XR>
struct Slot {
    static constexpr int W_BYTES = MR * 1024, BYTES = W_BYTES + XR * 256;
    static constexpr int LOADS = MR + XR / 4;          // wave-wide, 1 KB each
    static __device__ __forceinline__ int w_chunk(int row, int chunk) { return chunk ^ ((row >> 2) & 3); }
    static __device__ __forceinline__ int x_chunk(int row, int chunk) { return chunk ^ (row & 15); }
};

// TB: blocks of 16 tokens; XR: token rows that are loaded (4, or all); MR: blocks of 16 rows of W; NW: waves; D: ring slots of a
// wave; SUB: k-steps of 32 to a scale
template <int TB, int XR, int MR, int NW, int D, int CODE, int SUB, bool ZERO, int DT>
__global__ __launch_bounds__(64 * NW) void quant_tokens_kernel(QuantTokensArgs p)
{
    typedef Elem16<DT> E;
    typedef Slot<MR, XR> S;
    constexpr int ROWS = MR * 16, TOK = TB * 16, NS = 4 / SUB, LPS = S::LOADS;
    constexpr bool INT = CODE == DORA_QUANT_INT4;
    constexpr int RED_LD = ROWS + 4, RED_BYTES = NW * XR * RED_LD * 4;
    constexpr int RING_BYTES = NW * D * S::BYTES, TOP_BYTES = RING_BYTES > RED_BYTES ? RING_BYTES : RED_BYTES;
    // h comes through LDS, H_RANKS of it at a time
    constexpr int H_RANKS = TB == 1 ? 512 : 256, H_LD = H_RANKS * 2 + 16, H_BYTES = XR * H_LD;
    // scales (low half) and zero points (high) of a piece of the columns, a multiple of what the waves take in a round: rows of
    // an odd number of words, so that the sixteen of a fragment lie in different banks
    constexpr int SCALES_LD = (MR == 1 ? 4096 : 6144) / ROWS - 1;
    __shared__ __attribute__((aligned(1024))) char smem[TOP_BYTES + H_BYTES + ROWS * SCALES_LD * 4];
    static_assert(sizeof(smem) <= 160 * 1024, "LDS of a gfx950 CU");
    static_assert((D - 1) * LPS <= 63, "vmcnt is a 6-bit counter");

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, lq = lane >> 4;
    const int n0 = (int)blockIdx.x * ROWS;
    const int T = p.T, N = p.w.d_out, K = p.w.d_in, r = p.r;
    const int rows = N - n0 < ROWS ? N - n0 : ROWS;
    const int blocks = (K + BLOCK_K - 1) / BLOCK_K, whole = K / BLOCK_K;   // of columns
    const uint32_t row_bytes = (uint32_t)K / 2;
    const uint32_t smem_lds = (uint32_t)(uintptr_t)(lds_cptr_t)smem;
    const uint32_t h_lds = smem_lds + TOP_BYTES, scales_lds = h_lds + H_BYTES;

    // What the low-rank part and the scales need is asked for ahead of the first codes: loads complete in order, and one latency
    // covers them all.  Item of a piece of h: eight ranks of one token, `per` of them to a token, ranks past r among them as far
    // as a k-step reaches.
    constexpr int SLICES = 8 / TB, PRE = (H_RANKS / 32 + NW - 1) / NW;
    u32x4_t hs[SLICES][2];
    auto load_h = [&](int t, int l) {
        const uint32_t at = t < T && l < r ? ((uint32_t)t * (uint32_t)r + (uint32_t)l) * 4u : OUTSIDE;
#pragma unroll
        for (int z = 0; z < SLICES; ++z) {
            const __amdgpu_buffer_rsrc_t rh = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(p.h_part + (int64_t)(z < p.h_slices ? z : 0) * T * r), 0,
                                                                                z < p.h_slices ? (int)((uint32_t)T * (uint32_t)r * 4u) : 0, 0x00020000);
            hs[z][0] = __builtin_amdgcn_raw_buffer_load_b128(rh, at, 0, 0);
            hs[z][1] = __builtin_amdgcn_raw_buffer_load_b128(rh, at, 16, 0);
        }
    };
    const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(p.b + (int64_t)n0 * r), 0,
                                                                        (int)(uint32_t)((int64_t)rows * r * 2), 0x00020000);
    u32x4_t bpre[PRE][MR];
    auto load_b = [&](int c0) {
#pragma unroll
        for (int q = 0; q < PRE; ++q)
#pragma unroll
            for (int i = 0; i < MR; ++i) {
                const int l = c0 + (wave + q * NW) * 32 + lq * 8, row = i * 16 + l16;
                bpre[q][i] = __builtin_amdgcn_raw_buffer_load_b128(rb, l < r && row < rows ? ((uint32_t)row * (uint32_t)r + (uint32_t)l) * 2u : OUTSIDE, 0, 0);
            }
    };
    const int per0 = ((r < H_RANKS ? r : H_RANKS) + 31) / 32 * 4;
    load_h((int)threadIdx.x / per0, (int)threadIdx.x % per0 * 8);
    load_b(0);
    // a wave takes every NW-th row of the scales, 64 groups of it at a time
    constexpr int ROUND = D * NW, SROWS = ROWS / NW;
    static_assert(ROWS % NW == 0, "rows of scales of a wave");
    const int64_t fit = (((int64_t)SCALES_LD - 1) << p.w.group_shift) / BLOCK_K / ROUND * ROUND;   // (one group more where a piece begins inside one)
    const int piece = fit < blocks ? (int)fit : (blocks + ROUND - 1) / ROUND * ROUND;              // blocks of columns
    const uint16_t* const scale = static_cast<const uint16_t*>(p.w.scale);
    const uint16_t* const zero = static_cast<const uint16_t*>(p.w.zero);
    uint32_t sc[SROWS], zc[SROWS];
    auto load_scales = [&](int first, int count, int g0) {
        const int g = g0 + lane < count ? g0 + lane : count - 1;
#pragma unroll
        for (int i = 0; i < SROWS; ++i) {
            const int row = wave + i * NW;
            const int64_t at = (int64_t)(n0 + (row < rows ? row : rows - 1)) * p.w.groups + first + g;
            sc[i] = scale[at];
            zc[i] = ZERO ? zero[at] : 0u;
        }
    };
    auto put_scales = [&](int count, int g0) {
#pragma unroll
        for (int i = 0; i < SROWS; ++i) {
            if (g0 + lane < count) lds_write_b32(scales_lds + (uint32_t)((wave + i * NW) * SCALES_LD + g0 + lane) * 4u, sc[i] | zc[i] << 16);
        }
    };
    auto groups_of = [&](int b0, int& first) {
        first = (int)(((int64_t)b0 * BLOCK_K) >> p.w.group_shift);
        const int64_t end = (int64_t)(b0 + piece) * BLOCK_K < K ? (int64_t)(b0 + piece) * BLOCK_K : K;
        return (int)((end - 1) >> p.w.group_shift) - first + 1;
    };
    int first0;
    const int count0 = groups_of(0, first0);
    load_scales(first0, count0, 0);
    // as are the norm, the magnitude and the bias of the two columns that a thread stores, which would cost a latency at the end (4096 x
    // 4096, r 384, 1 token 11.3 -> 10.9 us); 64 rows with a scale to every k-step leave no registers for them
    constexpr bool EARLY = MR < 4 || SUB > 1;
    constexpr int PAIRS = ROWS / 2;
    static_assert(64 * NW % PAIRS == 0, "a thread keeps its columns");
    const int c = (int)threadIdx.x % PAIRS * 2, n = n0 + (c < rows ? c : 0);
    float2 cj, mj;
    uint32_t bias;
    auto load_columns = [&] {
        cj = *reinterpret_cast<const float2*>(p.c + n);
        mj = *reinterpret_cast<const float2*>(p.m + n);
        bias = p.bias ? *reinterpret_cast<const uint32_t*>(p.bias + n) : 0u;
    };
    if constexpr (EARLY) load_columns();
    __builtin_amdgcn_sched_barrier(0);

    __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint32_t*>(p.w.q + (int64_t)n0 * (K / 8)), 0, (int)(uint32_t)((int64_t)rows * row_bytes), 0x00020000);
    __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(p.x), 0, (int)(uint32_t)((int64_t)T * K * 2),
                                                                        0x00020000);
    // load i of a slot brings rows 16 i + lane / 4 of W, then token rows 4 (i - MR) + lane / 16; everything but the block's place in the
    // row travels in the vector offset, which alone is range checked
    uint32_t vo[LPS];
#pragma unroll
    for (int i = 0; i < LPS; ++i) {
        if (i < MR) {
            const int row = i * 16 + (lane >> 2);
            vo[i] = row < rows ? (uint32_t)row * row_bytes + (uint32_t)S::w_chunk(row, lane & 3) * 16u : OUTSIDE;
        } else {
            const int t = (i - MR) * 4 + (lane >> 4);
            vo[i] = t < T ? (uint32_t)t * (uint32_t)K * 2u + (uint32_t)S::x_chunk(t, lane & 15) * 16u : OUTSIDE;
        }
    }
    char* const ring = smem + wave * (D * S::BYTES);
    auto issue = [&](int b, int slot) {
        char* const at = ring + slot * S::BYTES;
        const bool in = b < whole;                     // a block past the end brings zeros
        const uint32_t k0 = in ? (uint32_t)b * BLOCK_K : 0u;
        static_for<LPS>([&](auto it) {
            constexpr int i = decltype(it)::value;
            load_1k(at + i * 1024, i < MR ? rw : rx, in ? vo[i] : OUTSIDE, i < MR ? k0 / 2 : k0 * 2);
        });
    };
    f32x4_t acc[MR][TB], accl[MR][TB];
#pragma unroll
    for (int i = 0; i < MR; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) { acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f}; accl[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f}; }
#pragma unroll
    for (int d = 0; d < D; ++d) issue(wave + d * NW, d);
    __builtin_amdgcn_sched_barrier(0);

    // low-rank part while the first codes are on their way: h summed in slice order and rounded once to the storage type, as
    // the saved tensor is; the waves share its k-steps of 32
    for (int c0 = 0; c0 < r; c0 += H_RANKS) {
        const int left = r - c0 < H_RANKS ? r - c0 : H_RANKS, per = (left + 31) / 32 * 4;
        if (c0 > 0) {
            __builtin_amdgcn_s_barrier();              // the ranks before have been read
            load_b(c0);
        }
        for (int e = threadIdx.x; e < T * per; e += 64 * NW) {
            const int t = e / per, k = e % per * 8;
            if (c0 > 0 || e >= 64 * NW) load_h(t, c0 + k);
            float a[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int z = 0; z < SLICES; ++z)
                if (z < p.h_slices) {
#pragma unroll
                    for (int u = 0; u < 8; ++u) a[u] += __uint_as_float(hs[z][u / 4][u % 4]);
                }
            uint4 o;
            o.x = E::pack2(a[0], a[1]); o.y = E::pack2(a[2], a[3]); o.z = E::pack2(a[4], a[5]); o.w = E::pack2(a[6], a[7]);
            if (p.h_out && blockIdx.x == 0 && k < left) *reinterpret_cast<uint4*>(p.h_out + (int64_t)t * r + c0 + k) = o;
            lds_write_b128(h_lds + (uint32_t)(t * H_LD + k * 2), o);
        }
        if (c0 == 0) {
            put_scales(count0, 0);
            for (int g0 = 64; g0 < count0; g0 += 64) {
                load_scales(first0, count0, g0);
                put_scales(count0, g0);
            }
        }
        wait_lgkmcnt<0>();
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int q = 0; q < PRE; ++q) {
            const int st = wave + q * NW;
            if (st * 32 >= left) continue;
            bf16x8_t hf[TB];
#pragma unroll
            for (int j = 0; j < TB; ++j) {
                const int t = j * 16 + l16 < T ? j * 16 + l16 : T - 1;   // (tokens past T: not stored)
                hf[j] = lds_read_b128<0>(h_lds + (uint32_t)(t * H_LD + (st * 32 + lq * 8) * 2));
            }
            landed(hf);
#pragma unroll
            for (int i = 0; i < MR; ++i)
#pragma unroll
                for (int j = 0; j < TB; ++j) accl[i][j] = E::mfma16(hf[j], __builtin_bit_cast(bf16x8_t, bpre[q][i]), accl[i][j]);
        }
    }

    // LDS reads of a lane, relative to the slot: k-step q of token block j, 16 / NS bytes of codes of row block i
    const uint32_t ring_lds = smem_lds + (uint32_t)(wave * (D * S::BYTES));
    uint32_t rx_at[4], rw_at[NS];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int n = q / SUB, u = q % SUB;
        const int row = l16 < XR ? l16 : 0;            // (token rows that were not loaded: not stored)
        rx_at[q] = (uint32_t)(S::W_BYTES + row * 256 + S::x_chunk(row, n * (SUB * 4) + lq * SUB + u) * 16);
        if (u == 0) rw_at[n] = (uint32_t)(l16 * 64 + S::w_chunk(l16, SUB == 4 ? lq : SUB == 2 ? n * 2 + (lq >> 1) : n) * 16 + (SUB == 2 ? (lq & 1) * 8 : SUB == 1 ? lq * 4 : 0));
    }
    const uint32_t addend = INT && !ZERO ? (DT == DT_BF16 ? 0xc100c100u : 0xc800c800u) : (DT == DT_BF16 ? 0x3f803f80u : 0x3c003c00u);   // -8, 1
    const bf16x8_t constant = __builtin_bit_cast(bf16x8_t, u32x4_t{addend, addend, addend, addend});
    // the block in `slot`: codes, x and scales out of the LDS, then (refill) the slot's next loads, then the products
    auto multiply = [&](int b, int g_first, uint32_t slot_lds, auto&& refill) {
        bf16x8_t x[4][TB];
        uint32_t w[MR][4], sz[MR][NS];
        static_for<4 * TB>([&](auto it) {
            constexpr int q = decltype(it)::value / TB, j = decltype(it)::value % TB;
            x[q][j] = lds_read_b128<j * 4096>(slot_lds + rx_at[q]);
        });
        static_for<MR>([&](auto it) {
            constexpr int i = decltype(it)::value;
            if constexpr (SUB == 4) {
                const u32x4_t v = __builtin_bit_cast(u32x4_t, lds_read_b128<i * 1024>(slot_lds + rw_at[0]));
                w[i][0] = v[0]; w[i][1] = v[1]; w[i][2] = v[2]; w[i][3] = v[3];
            } else if constexpr (SUB == 2) {
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const uint64_t v = lds_read_b64<i * 1024>(slot_lds + rw_at[n]);
                    w[i][2 * n] = (uint32_t)v; w[i][2 * n + 1] = (uint32_t)(v >> 32);
                }
            } else {
#pragma unroll
                for (int n = 0; n < 4; ++n) w[i][n] = lds_read_b32<i * 1024>(slot_lds + rw_at[n]);
            }
#pragma unroll
            for (int n = 0; n < NS; ++n) {
                int g = (b * BLOCK_K + n * SUB * 32) >> p.w.group_shift;
                g = (g < p.w.groups ? g : p.w.groups - 1) - g_first;   // (past the end: times a sum of zeros)
                sz[i][n] = lds_read_b32<i * 64 * SCALES_LD>(scales_lds + (uint32_t)(l16 * SCALES_LD + g) * 4u);
            }
        });
        wait_lgkmcnt<0>();
        __builtin_amdgcn_sched_barrier(0);
        refill();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            f32x4_t first[TB];                         // what the products are added to: -8 (or 1) times the sum of x
#pragma unroll
            for (int j = 0; j < TB; ++j) {
                first[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                if constexpr (INT) {
#pragma unroll
                    for (int q = n * SUB; q < (n + 1) * SUB; ++q) first[j] = E::mfma16(x[q][j], constant, first[j]);
                }
            }
#pragma unroll
            for (int i = 0; i < MR; ++i) {
                const float s = E::lo(sz[i][n]);
                f32x4_t part[TB];
#pragma unroll
                for (int j = 0; j < TB; ++j) {
                    part[j] = first[j];
                    if constexpr (ZERO) {
                        const float z = -E::hi(sz[i][n]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) part[j][e] *= z;
                    }
                }
#pragma unroll
                for (int q = n * SUB; q < (n + 1) * SUB; ++q) {
                    const bf16x8_t wf = decode_fragment<CODE, DT>(w[i][q]);
#pragma unroll
                    for (int j = 0; j < TB; ++j) part[j] = E::mfma16(x[q][j], wf, part[j]);
                }
#pragma unroll
                for (int j = 0; j < TB; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(s, part[j][e], acc[i][j][e]);
            }
        }
    };
    int slot = 0;
    for (int b0 = 0; b0 < blocks; b0 += piece) {
        int first = first0;
        if (b0 > 0) {
            __builtin_amdgcn_s_barrier();              // the scales before have been read
            const int count = groups_of(b0, first);
            for (int g0 = 0; g0 < count; g0 += 64) {
                load_scales(first, count, g0);
                put_scales(count, g0);
            }
            wait_lgkmcnt<0>();
            __builtin_amdgcn_s_barrier();
        }
        const int end = b0 + piece < whole ? b0 + piece : whole;
        for (int b = b0 + wave; b < end; b += NW) {
            __builtin_amdgcn_sched_barrier(0);
            wait_vmcnt<(D - 1) * LPS>();               // the oldest slot has landed
            __builtin_amdgcn_sched_barrier(0);
            multiply(b, first, ring_lds + slot * S::BYTES, [&] { issue(b + ROUND, slot); });
            slot = slot + 1 == D ? 0 : slot + 1;
        }
        if (b0 + piece >= blocks && whole < blocks && whole % NW == wave) {
            // The block that the rows end in, a word of codes at a time (a chunk may end past the tensor); what is past the end of
            // the rows is zeros.
            wait_vmcnt<0>();
            const uint32_t at = ring_lds + slot * S::BYTES;
#pragma unroll
            for (int i = 0; i < LPS; ++i) {
                const int chunk = i < MR ? S::w_chunk(i * 16 + (lane >> 2), lane & 3) : S::x_chunk((i - MR) * 4 + (lane >> 4), lane & 15);
                u32x4_t v;
                if (i < MR) {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        v[q] = __builtin_amdgcn_raw_buffer_load_b32(rw, vo[i] != OUTSIDE && whole * BLOCK_K + chunk * 32 + q * 8 < K ? vo[i] + q * 4 : OUTSIDE,
                                                                    (uint32_t)whole * (BLOCK_K / 2), 0);
                } else {
                    v = __builtin_amdgcn_raw_buffer_load_b128(rx, whole * BLOCK_K + chunk * 8 < K ? vo[i] : OUTSIDE, (uint32_t)whole * (BLOCK_K * 2), 0);
                }
                lds_write_b128(at + i * 1024 + lane * 16, make_uint4(v[0], v[1], v[2], v[3]));
            }
            wait_lgkmcnt<0>();
            __builtin_amdgcn_sched_barrier(0);
            multiply(whole, first, at, [] {});
        }
    }
    wait_vmcnt<0>();                                   // the loads past the end have written their zeros
    __syncthreads();

    // lane: tokens 4 lq .. +3 of block j, row l16 of block i.  The waves' tiles meet in LDS.
    float* const red = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int i = 0; i < MR; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (XR == TOK || lq * 4 + e < XR)
                    red[(wave * XR + j * 16 + lq * 4 + e) * RED_LD + i * 16 + l16] = fmaf(p.s, accl[i][j][e], acc[i][j][e]);
    __syncthreads();
    if (c >= rows) return;                             // d_out is a multiple of 8
    if constexpr (!EARLY) load_columns();
    const float g0 = mj.x / ((cj.x < p.eps) ? p.eps : cj.x), g1 = mj.y / ((cj.y < p.eps) ? p.eps : cj.y);
    for (int t = (int)threadIdx.x / PAIRS; t < T; t += 64 * NW / PAIRS) {
        float v0 = 0.f, v1 = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float2 u = *reinterpret_cast<const float2*>(red + (w * XR + t) * RED_LD + c);
            v0 += u.x; v1 += u.y;
        }
        const int64_t at = (int64_t)t * N + n;
        *reinterpret_cast<uint32_t*>(p.y + at) = E::pack2(fmaf(g0, v0, E::lo(bias)), fmaf(g1, v1, E::hi(bias)));
        if (p.inner) *reinterpret_cast<uint32_t*>(p.inner + at) = E::pack2(v0, v1);
    }
}

// Rows of a workgroup and ring slots: us of a forward, one after the other over as many sets of weights and inputs as make 600 MB.
//  - 16 rows make 256 workgroups of 4096 rows of W.  Beyond, they would read x once more for every round, so 32 of them up to
//    8192 rows and 64 past that: 8192 x 8192, r 64, 32 tokens 31.5, 22.7 and 26.9 us with 16, 32 and 64 rows, 16 tokens 24.4, 20.4,
//    25.2; 14336 x 4096, 27 tokens 35.6, 24.9, 21.3.  Up to four tokens x hardly counts, and 16 rows do up to 8192 (8192 x 8192, 1
//    token 16.1, 16.1 and 18.6 us; 14336 x 4096 20.3, 18.7, 15.4).
//  - One ring slot to each of eight waves: more LDS leaves room for one workgroup on a CU, and the other's prologue no longer stands
//    beside this one's products (27648 x 5120, 16 tokens 36.3 us with three slots to each of four waves, 33.5 this way; 1 token 30.1
//    with two slots to each of eight, 28.2).  Two slots where they are small enough (4096 x 4096, r 384, 1 token 11.8 and 11.1).
template <int CODE, int SUB, bool ZERO, int DT>
hipError_t launch_shape(const QuantTokensArgs& a, hipStream_t st)
{
#define DORA_QUANT_TOKENS(TB, XR, MR, D) \
    quant_tokens_kernel<TB, XR, MR, 8, D, CODE, SUB, ZERO, DT><<<dim3((unsigned)((a.w.d_out + MR * 16 - 1) / (MR * 16))), dim3(512), 0, st>>>(a)
    const bool narrow = a.w.d_out <= 4096, wide = a.w.d_out > 8192;
    if (a.T <= 4) { if (wide) DORA_QUANT_TOKENS(1, 4, 4, 1); else DORA_QUANT_TOKENS(1, 4, 1, 2); }
    else if (a.T <= 16) { if (wide) DORA_QUANT_TOKENS(1, 16, 4, 1); else if (narrow) DORA_QUANT_TOKENS(1, 16, 1, 1); else DORA_QUANT_TOKENS(1, 16, 2, 1); }
    else { if (wide) DORA_QUANT_TOKENS(2, 32, 4, 1); else if (narrow) DORA_QUANT_TOKENS(2, 32, 1, 1); else DORA_QUANT_TOKENS(2, 32, 2, 1); }
#undef DORA_QUANT_TOKENS
    return hipGetLastError();
}
template <int SUB, int DT>
hipError_t launch_code(const QuantTokensArgs& a, hipStream_t st)
{
    if (a.w.code == DORA_QUANT_FP4) return launch_shape<DORA_QUANT_FP4, SUB, false, DT>(a, st);
    return a.w.zero ? launch_shape<DORA_QUANT_INT4, SUB, true, DT>(a, st) : launch_shape<DORA_QUANT_INT4, SUB, false, DT>(a, st);
}
template <int DT>
hipError_t launch(const QuantTokensArgs& a, hipStream_t st)
{
    if (a.w.group_shift >= 7) return launch_code<4, DT>(a, st);
    return a.w.group_shift == 6 ? launch_code<2, DT>(a, st) : launch_code<1, DT>(a, st);
}

}  // namespace

hipError_t launch_quant_tokens(const QuantTokensArgs& a, int dt, hipStream_t st)
{
    TraceScope ts(DORA_K_QUANT_TOKENS, st);
    return dt == DT_F16 ? launch<DT_F16>(a, st) : launch<DT_BF16>(a, st);
}

}  // namespace dora
