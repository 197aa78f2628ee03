// The row norm over a 4-bit weight, ranks up to NORM_ROWS_MAX_RANK: the kernels of norm_rows_body.hpp with the codes, a quarter of the
// bytes, in the ring, and with w = scale * (q - zero) formed in fp32 where it is used.  No weight is rounded, and none is written.  The
// terms of Eq. 5 are not asked for over codes, so an element is one square: (w + s v)^2 in fp32, in three multiply-adds beside the
// decoding (five for three sums).
//
// Bound: the matrix cores from r about 200 on (8192 x 8192, r 384: 52 GFLOP, 0.9 PFLOP/s of them in the launch); below, the vector
// instructions of the sum, about 350 to the 32 S matrix instructions of a wave's tile.  Against reading the weight back first and forming
// the three sums over that, and against the three sums over codes, us of a norm with Eq. 5, weights from memory: 8192 x 8192, r 384
// 97 / 73 / 66, r 64 60 / 31 / 28; 4096 x 4096, r 384 36 / 24 / 20; 1024 x 4096, r 64 15.7 / 9.5 / 7.8; 27648 x 5120, r 384 195 /
// 142 / 134.
#include "norm_rows_body.hpp"

namespace dora {
namespace {

template <int WK, int DT>
hipError_t launch(const NormRowsArgs& a, hipStream_t st)
{
    const dim3 grid((unsigned)((a.d_out + BM - 1) / BM * a.slices)), block(256);
    switch ((a.r + 63) / 64) {
        case 1: norm_rows_kernel<1, WK, DT><<<grid, block, 0, st>>>(a); break;
        case 2: norm_rows_kernel<2, WK, DT><<<grid, block, 0, st>>>(a); break;
        case 3: norm_rows_deep_kernel<3, WK, DT><<<grid, block, 0, st>>>(a); break;
        case 4: norm_rows_deep_kernel<4, WK, DT><<<grid, block, 0, st>>>(a); break;
        case 5: norm_rows_deep_kernel<5, WK, DT><<<grid, block, 0, st>>>(a); break;
        case 6: norm_rows_deep_kernel<6, WK, DT><<<grid, block, 0, st>>>(a); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}
template <int DT>
hipError_t launch_code(const NormRowsArgs& a, hipStream_t st)
{
    return a.q.code == DORA_QUANT_FP4 ? launch<W_FP4, DT>(a, st) : launch<W_INT4, DT>(a, st);
}

}  // namespace

hipError_t launch_norm_quant(const NormRowsArgs& a, int dt, hipStream_t st)
{
    TraceScope ts(DORA_K_NORM_CROSS, st);
    return dt == DT_F16 ? launch_code<DT_F16>(a, st) : launch_code<DT_BF16>(a, st);
}

}  // namespace dora
