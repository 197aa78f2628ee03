// Dropout of the adapter's input and of its gradient (dora_dropout, dora_dropout_backward).  The mask is never stored: it is a
// function of (seed, offset, place), drawn again wherever it is needed.
//
// Philox 4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): ten rounds of two 32 x 32 ->
// 64 bit products over a counter of 128 bits give 128 random bits that depend on key and counter alone.  Sixteen of them decide
// an element, so one call serves eight: a 16-byte vector of a 16-bit type.  With 32 bits to an element the products alone (a
// quarter of the vector rate) would take as long as the memory; sixteen leave p a resolution of 2^-16, and the scale is that of
// the p that is used, so the mean is kept exactly.  Bound: memory.
#include "quant_codes.hpp"

namespace dora {
namespace {

__device__ __forceinline__ uint4 philox(uint32_t c0, uint32_t c1, uint32_t k0, uint32_t k1)
{
    uint32_t c2 = 0u, c3 = 0u;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t p0 = (uint64_t)c0 * 0xD2511F53u, p1 = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(p1 >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)p1;
        c2 = (uint32_t)(p0 >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)p0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

// out = (add +) (kept ? v * scale : 0); n elements, a multiple of four
template <typename T, bool ADD>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs p)
{
    typedef Eight<T> V;
    const uint32_t b = blockIdx.x * 256u + threadIdx.x;
    const int64_t first = (int64_t)b * 8;
    if (first >= p.n) return;
    const uint64_t at = p.offset + (p.counter ? *p.counter : 0) + b;
    const T* const src = static_cast<const T*>(p.v) + first;
    const T* const add = static_cast<const T*>(p.add) + first;
    T* const out = static_cast<T*>(p.out) + first;
    float f[8], a[8];
    const bool whole = first + 8 <= p.n;
    if (whole) {
        V::load(src, f);
        if constexpr (ADD) V::load(add, a);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            f[j] = j < 4 ? V::one(src, j) : 0.f;
            a[j] = ADD && j < 4 ? V::one(add, j) : 0.f;
        }
    }
    const uint4 r = philox((uint32_t)at, (uint32_t)(at >> 32), (uint32_t)p.seed, (uint32_t)(p.seed >> 32));
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t u = j % 2 ? w[j / 2] >> 16 : w[j / 2] & 0xffffu;
        const float v = u >= p.threshold ? f[j] * p.scale : 0.f;     // (chosen, not multiplied by 0: what is dropped may be NaN)
        f[j] = ADD ? a[j] + v : v;
    }
    if (whole) V::store(out, f);
    else {
#pragma unroll
        for (int j = 0; j < 4; ++j) V::put(out, j, f[j]);
    }
}

template <typename T>
hipError_t dropout_t(const DropoutArgs& a, hipStream_t st)
{
    const dim3 grid((unsigned)(((a.n + 7) / 8 + 255) / 256)), block(256);
    if (a.add) dropout_kernel<T, true><<<grid, block, 0, st>>>(a);
    else dropout_kernel<T, false><<<grid, block, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(int dtype, const DropoutArgs& a, hipStream_t st)
{
    TraceScope ts(DORA_K_DROPOUT, st);
    if (dtype == DORA_F32) return dropout_t<float>(a, st);
    return dtype == DORA_F16 ? dropout_t<f16_t>(a, st) : dropout_t<bf16_t>(a, st);
}

}  // namespace dora
