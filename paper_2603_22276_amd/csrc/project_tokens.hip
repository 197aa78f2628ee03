// h = x A^T of a few hundred tokens in one launch, in front of a product over a 4-bit weight.  An output tile of 16 tokens x 16 ranks is
// all that a workgroup has; its sixteen waves share the columns, 64 at a time (a row's 128 bytes, two MFMA k-steps), hold their sums in
// fp32 and add them in LDS in wave order.  Fragments come straight from memory: a wave asks for four such pieces of both operands
// before it multiplies the first, so 4096 columns cost one latency.  h, and s h for the K-concatenated product, are rounded once each from
// those sums: they are operands of a 16-bit product.
//
// Bound: the latency of the first loads and the L1, which looks up sixteen rows for a load (16 cycles and more).  Tiles of 128 x 128 with K
// in slices and a launch that sums them, which other sizes take, are 6.8 and 4.0 us of 4096 columns and a launch more between them.
#include "quant_codes.hpp"

namespace dora {
namespace {

constexpr int NW = 16, U = 4, PIECE = 64;              // waves, pieces in flight, columns of a piece

template <int DT>
__global__ __launch_bounds__(NW * 64) void project_tokens_kernel(ProjectTokensArgs p)
{
    typedef Elem16<DT> E;
    __shared__ float red[NW][16][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, lq = lane >> 4;
    const int K = p.d_in, rank_tiles = (p.r + 15) / 16;
    const int t0 = (int)blockIdx.x / rank_tiles * 16, l0 = (int)blockIdx.x % rank_tiles * 16;
    const int toks = p.T - t0 < 16 ? p.T - t0 : 16, ranks = p.r - l0 < 16 ? p.r - l0 : 16;
    const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(p.x + (int64_t)t0 * K), 0,
                                                                        (int)(uint32_t)((int64_t)toks * K * 2), 0x00020000);
    const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(p.a + (int64_t)l0 * K), 0,
                                                                        (int)(uint32_t)((int64_t)ranks * K * 2), 0x00020000);
    f32x4_t acc = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const int pieces = (K + PIECE - 1) / PIECE;
    for (int first = wave; first < pieces; first += NW * U) {
        u32x4_t xv[U][2], av[U][2];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                // (a piece past the last one, and what lies past the end of the rows, is zeros)
                const int64_t k = (int64_t)(first + u * NW) * PIECE + q * 32 + lq * 8;
                const bool in = k < K;
                xv[u][q] = __builtin_amdgcn_raw_buffer_load_b128(rx, in && l16 < toks ? ((uint32_t)l16 * (uint32_t)K + (uint32_t)k) * 2u : OUTSIDE, 0, 0);
                av[u][q] = __builtin_amdgcn_raw_buffer_load_b128(ra, in && l16 < ranks ? ((uint32_t)l16 * (uint32_t)K + (uint32_t)k) * 2u : OUTSIDE, 0, 0);
            }
        __builtin_amdgcn_sched_barrier(0);             // (all of them asked for before the first is used)
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int q = 0; q < 2; ++q)
                acc = E::mfma16(__builtin_bit_cast(bf16x8_t, xv[u][q]), __builtin_bit_cast(bf16x8_t, av[u][q]), acc);
    }
    // lane: tokens 4 lq .. +3, rank l16
#pragma unroll
    for (int e = 0; e < 4; ++e) red[wave][lq * 4 + e][l16] = acc[e];
    __syncthreads();
    const int t = (int)threadIdx.x / 8, l = (int)threadIdx.x % 8 * 2;
    if (t >= toks || l >= ranks) return;               // r is a multiple of 8
    float v0 = 0.f, v1 = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) { v0 += red[w][t][l]; v1 += red[w][t][l + 1]; }
    const int64_t at = (int64_t)(t0 + t) * p.r + l0 + l;
    *reinterpret_cast<uint32_t*>(p.h + at) = E::pack2(v0, v1);
    if (p.hs) *reinterpret_cast<uint32_t*>(p.hs + at) = E::pack2(p.s * v0, p.s * v1);
}

}  // namespace

hipError_t launch_project_tokens(const ProjectTokensArgs& a, int dt, hipStream_t st)
{
    TraceScope ts(DORA_K_GEMM_H, st);
    const dim3 grid((unsigned)((a.T + 15) / 16 * ((a.r + 15) / 16))), block(NW * 64);
    if (dt == DT_F16) project_tokens_kernel<DT_F16><<<grid, block, 0, st>>>(a);
    else project_tokens_kernel<DT_BF16><<<grid, block, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace dora
