// A frozen weight into 4 bits and back (dora_quantize, dora_dequantize).  Both are streams over the weight: 2 bytes an element
// (16-bit storage) one way, half a byte and a scale per group the other.
#include "quant_codes.hpp"

#include <type_traits>

namespace dora {
namespace {

// Nearest number of four significant bits, ties to even.
__device__ __forceinline__ float four_bits(float v)
{
    const uint32_t u = __float_as_uint(v);
    return __uint_as_float((u + 0x7ffffu + ((u >> 20) & 1u)) & ~0xfffffu);
}
// Smallest number of four significant bits that is not below v >= 0.
__device__ __forceinline__ float four_bits_up(float v) { return __uint_as_float((__float_as_uint(v) + 0xfffffu) & ~0xfffffu); }

struct QuantizeArgs {
    const void* w;
    uint32_t* q;
    void *scale, *zero;
    int d_out, d_in, group_shift, groups;
};

// A group belongs to `lanes` = min(64, group / 8) lanes of a wave, eight weights to a lane at a time; the extremes of the group
// meet by lane exchanges, so a weight is read once (groups above 512: twice, the second time from the L2).  Bound: memory.
//
// Scales have four significant bits.  A symmetric code (at most 3 bits of odd part, 4 with a zero point) times such a scale
// has 8 at most, so the weight that codes and scale stand for is a bf16 and an fp16 number without rounding, and every path
// (streamed, tiled, backward) multiplies with the same one.  The step grows by up to 1/16 for it.
template <typename T, int CODE, bool ZERO>
__global__ __launch_bounds__(256) void quantize_kernel(QuantizeArgs p)
{
    typedef Eight<T> V;
    const int group = 1 << p.group_shift;
    const int lane_shift = p.group_shift - 3 < 6 ? p.group_shift - 3 : 6, lanes = 1 << lane_shift;
    const uint32_t unit = (uint32_t)(((uint64_t)blockIdx.x * 256 + threadIdx.x) >> lane_shift);
    const uint32_t row = unit / (uint32_t)p.groups, g = unit - row * (uint32_t)p.groups;
    if (row >= (uint32_t)p.d_out) return;              // (the lanes of a group leave together)
    const int k_first = (int)(g << p.group_shift) + (int)(threadIdx.x & (lanes - 1)) * 8;
    const int k_end = (int)((int64_t)(g + 1) << p.group_shift < p.d_in ? (g + 1) << p.group_shift : p.d_in);
    const T* const src = static_cast<const T*>(p.w) + (int64_t)row * p.d_in;
    float f[8];
    float lo = 0.f, hi = 0.f;
    int odd = 0;                                       // NaN or infinity seen
    for (int k = k_first; k < k_end; k += 512) {
        V::load(src + k, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            lo = fminf(lo, f[j]); hi = fmaxf(hi, f[j]);
            odd |= !(fabsf(f[j]) <= 3.402823466e38f);
        }
    }
    for (int m = 1; m < lanes; m <<= 1) {
        lo = fminf(lo, __shfl_xor(lo, m)); hi = fmaxf(hi, __shfl_xor(hi, m)); odd |= __shfl_xor(odd, m);
    }
    float s, z = 0.f;
    if constexpr (ZERO) s = four_bits_up((hi - lo) / 15.f);
    else s = four_bits(fmaxf(hi, -lo) / (CODE == DORA_QUANT_INT4 ? 7.f : 6.f));
    // What is read back stays finite in fp16: 6 x 10240 is, and a code is not taken past 65504.
    if constexpr (std::is_same<T, f16_t>::value && CODE == DORA_QUANT_FP4) s = fminf(s, 10240.f);
    if (odd || !(s <= 3.402823466e38f)) s = __uint_as_float(0x7fc00000u);
    const int64_t at = (int64_t)row * p.groups + g;
    const bool first = (threadIdx.x & (lanes - 1)) == 0;
    if constexpr (sizeof(T) == 2) {                    // as stored (fp16: small ones lose bits)
        uint32_t bits = 0;
        V::put(&bits, 0, s);
        s = V::one(&bits, 0);
    }
    const float most = std::is_same<T, f16_t>::value ? floorf(65504.f / s) : 15.f;
    const bool some = s > 0.f;                         // neither 0 nor NaN: otherwise the code of 0 everywhere
    if constexpr (ZERO) z = some ? fminf(fmaxf(rintf(-lo / s), 0.f), 15.f) : 0.f;
    if (first) {
        V::put(p.scale, at, s);
        if constexpr (ZERO) V::put(p.zero, at, z);
    }
    for (int k = k_first; k < k_end; k += 512) {
        if (group > 512) V::load(src + k, f);
        uint32_t word = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t q;
            if constexpr (CODE == DORA_QUANT_INT4) {
                const float offset = ZERO ? z : 8.f;
                q = (uint32_t)(some ? fminf(fmaxf(offset + fminf(fmaxf(rintf(f[j] / s), -most), most), 0.f), 15.f) : offset);
            } else {
                // against the seven midpoints, exact products; halfway goes to the even code
                const float a = fabsf(f[j]);
                q = (uint32_t)(a > 0.25f * s) + (uint32_t)(a >= 0.75f * s) + (uint32_t)(a > 1.25f * s) + (uint32_t)(a >= 1.75f * s) +
                    (uint32_t)(a > 2.5f * s) + (uint32_t)(a >= 3.5f * s) + (uint32_t)(a > 5.f * s) + (f[j] < 0.f ? 8u : 0u);
                q = some ? q : 0u;
            }
            word |= q << (4 * j);
        }
        p.q[((int64_t)row * p.d_in + k) >> 3] = word;
    }
}

// Eight weights to a thread, four times: 4 bytes of codes in, 16 (32) out.
template <typename T, int CODE, bool ZERO>
__global__ __launch_bounds__(256) void dequantize_kernel(QuantWeight w, T* out, uint32_t words, uint32_t per_row)
{
    typedef Eight<T> V;
    constexpr int U = 4;
    const uint32_t first = blockIdx.x * (256u * U) + threadIdx.x;
    uint32_t q[U];
    float s[U], z[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t i = first + u * 256u < words ? first + u * 256u : words - 1;
        const uint32_t row = i / per_row, k = (i - row * per_row) * 8;
        const int64_t at = (int64_t)row * w.groups + (k >> w.group_shift);
        q[u] = w.q[i];
        s[u] = V::one(w.scale, at);
        z[u] = CODE == DORA_QUANT_INT4 ? (ZERO ? V::one(w.zero, at) : 8.f) : 0.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t i = first + u * 256u;
        if (i >= words) return;
        float f[8];
        decode8<CODE>(q[u], f);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = (f[j] - z[u]) * s[u];
        V::store(out + (int64_t)i * 8, f);
    }
}

template <typename T>
hipError_t quantize_t(const QuantizeArgs& a, int code, hipStream_t st)
{
    const int lane_shift = a.group_shift - 3 < 6 ? a.group_shift - 3 : 6;
    const int64_t threads = ((int64_t)a.d_out * a.groups) << lane_shift;
    const dim3 grid((unsigned)((threads + 255) / 256)), block(256);
    if (code == DORA_QUANT_FP4) quantize_kernel<T, DORA_QUANT_FP4, false><<<grid, block, 0, st>>>(a);
    else if (a.zero) quantize_kernel<T, DORA_QUANT_INT4, true><<<grid, block, 0, st>>>(a);
    else quantize_kernel<T, DORA_QUANT_INT4, false><<<grid, block, 0, st>>>(a);
    return hipGetLastError();
}

template <typename T>
hipError_t dequantize_t(const QuantWeight& w, void* out, hipStream_t st)
{
    const uint32_t per_row = (uint32_t)w.d_in / 8, words = (uint32_t)w.d_out * per_row;   // (d_out d_in < 2^31)
    const dim3 grid((words + 1023) / 1024), block(256);
    T* const o = static_cast<T*>(out);
    if (w.code == DORA_QUANT_FP4) dequantize_kernel<T, DORA_QUANT_FP4, false><<<grid, block, 0, st>>>(w, o, words, per_row);
    else if (w.zero) dequantize_kernel<T, DORA_QUANT_INT4, true><<<grid, block, 0, st>>>(w, o, words, per_row);
    else dequantize_kernel<T, DORA_QUANT_INT4, false><<<grid, block, 0, st>>>(w, o, words, per_row);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize(int dtype, const void* W, int d_out, int d_in, int code, int group_shift, void* q, void* scale, void* zero,
                           hipStream_t st)
{
    TraceScope ts(DORA_K_QUANTIZE, st);
    const QuantizeArgs a{W, static_cast<uint32_t*>(q), scale, zero, d_out, d_in, group_shift, quant_groups(d_in, group_shift)};
    if (dtype == DORA_F32) return quantize_t<float>(a, code, st);
    return dtype == DORA_F16 ? quantize_t<f16_t>(a, code, st) : quantize_t<bf16_t>(a, code, st);
}

hipError_t launch_dequantize(int dtype, const QuantWeight& w, void* out, hipStream_t st)
{
    TraceScope ts(DORA_K_DEQUANTIZE, st);
    if (dtype == DORA_F32) return dequantize_t<float>(w, out, st);
    return dtype == DORA_F16 ? dequantize_t<f16_t>(w, out, st) : dequantize_t<bf16_t>(w, out, st);
}

}  // namespace dora
