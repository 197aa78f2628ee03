// The three sums of the row norm over a 4-bit weight, ranks up to NORM_ROWS_MAX_RANK: the kernels of norm_rows_body.hpp with the
// codes, a quarter of the bytes, in the ring, and with scale * (q - zero) formed in fp32 where a value is used.  No weight is rounded,
// and none is written.
//
// Bound: the matrix cores from r about 200 on (8192 x 8192, r 384: 52 GFLOP, 1.0 PFLOP/s of them); below, the latency of a tile's
// loads.  Against reading the weight back first and summing over that, us of a norm with Eq. 5, weights from memory: 8192 x 8192,
// r 384 97 -> 73, r 64 60 -> 31; 4096 x 4096, r 384 36 -> 24; 1024 x 4096, r 64 15.7 -> 9.5; 27648 x 5120, r 384 195 -> 142.
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
