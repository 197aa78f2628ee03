// The three sums of the row norm over a 16-bit weight: the kernels of norm_rows_body.hpp and their choice by the rank.
#include "norm_rows_body.hpp"

namespace dora {
namespace {

template <int DT>
hipError_t launch(const NormRowsArgs& a, hipStream_t st)
{
    const dim3 grid((unsigned)((a.d_out + BM - 1) / BM * a.slices)), block(256);
    switch ((a.r + 63) / 64) {
        case 1: norm_rows_kernel<1, W_16, DT><<<grid, block, 0, st>>>(a); break;
        case 2: norm_rows_kernel<2, W_16, DT><<<grid, block, 0, st>>>(a); break;
        case 3: norm_rows_deep_kernel<3, W_16, DT><<<grid, block, 0, st>>>(a); break;
        case 4: norm_rows_deep_kernel<4, W_16, DT><<<grid, block, 0, st>>>(a); break;
        case 5: norm_rows_deep_kernel<5, W_16, DT><<<grid, block, 0, st>>>(a); break;
        case 6: norm_rows_deep_kernel<6, W_16, DT><<<grid, block, 0, st>>>(a); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_rows(const NormRowsArgs& a, int dt, hipStream_t st)
{
    TraceScope ts(DORA_K_NORM_CROSS, st);
    return dt == DT_F16 ? launch<DT_F16>(a, st) : launch<DT_BF16>(a, st);
}

}  // namespace dora
