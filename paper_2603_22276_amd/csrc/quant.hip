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
    int d_out, d_in, group_shift, groups, lane_shift;
};

// The largest of 16-bit pairs, both halves at once, over `lanes` (a power of two from 4 on) lanes in a row.
typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pair_max(uint32_t a, uint32_t b)
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, a), __builtin_bit_cast(u16x2_t, b)));
}
typedef int16_t s16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pair_max_signed(uint32_t a, uint32_t b)
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(s16x2_t, a), __builtin_bit_cast(s16x2_t, b)));
}
__device__ __forceinline__ uint32_t lanes_pair_max(uint32_t v, int lanes)
{
    v = pair_max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, true));                     // lanes 1 apart
    v = pair_max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, true));                     // 2
    if (lanes > 4) v = pair_max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, true));     // the other four of eight
    if (lanes > 8) v = pair_max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xf, 0xf, true));     // the other eight of sixteen
    for (int m = 16; m < lanes; m <<= 1) v = pair_max(v, (uint32_t)__shfl_xor((int)v, m));
    return v;
}

// A group belongs to `lanes` = min(64, group / 8) lanes of a wave (fewer where the row is shorter), eight weights to a lane at a time;
// the extremes of the group meet by lane exchanges, so a weight is read once (groups above 512: twice, the second time from the L2).
// 16-bit floats are ordered as their bits are: the extremes are found two at a time, the largest positive as it is and the most
// negative as the largest number with the sign bit; exponents of ones show infinities and NaN.  Bound: memory, and the vector
// instructions of rounding beside it: 14336 x 4104 in fp16 with zero points, groups of 64, 43 us, 3.5 TB/s (65 with the extremes, the
// eight quotients and the eight codes of a thread one by one).
//
// Scales have four significant bits.  A symmetric code (at most 3 bits of odd part, 4 with a zero point) times such a scale
// has 8 at most, so the weight that codes and scale stand for is a bf16 and an fp16 number without rounding, and every path
// (streamed, tiled, backward) multiplies with the same one.  The step grows by up to 1/16 for it.  In fp32 the same, so that codes and
// scales of a weight serve a module of any storage type.
template <typename T, int CODE, bool ZERO>
__global__ __launch_bounds__(256) void quantize_kernel(QuantizeArgs p)
{
    typedef Eight<T> V;
    const int group = 1 << p.group_shift;
    const int lanes = 1 << p.lane_shift;
    const uint32_t unit = (uint32_t)(((uint64_t)blockIdx.x * 256 + threadIdx.x) >> p.lane_shift);
    const uint32_t row = unit / (uint32_t)p.groups, g = unit - row * (uint32_t)p.groups;
    if (row >= (uint32_t)p.d_out) return;              // (the lanes of a group leave together)
    const int k_first = (int)(g << p.group_shift) + (int)(threadIdx.x & (lanes - 1)) * 8;
    const int k_end = (int)((int64_t)(g + 1) << p.group_shift < p.d_in ? (g + 1) << p.group_shift : p.d_in);
    const T* const src = static_cast<const T*>(p.w) + (int64_t)row * p.d_in;
    float f[8];
    float lo = 0.f, hi = 0.f;
    bool odd = false;                                  // NaN or infinity seen
    if constexpr (sizeof(T) == 2) {
        uint4 raw = make_uint4(0u, 0u, 0u, 0u);
        uint32_t up = 0u, down = 0u;                   // pairs: largest as signed numbers (symmetric: of magnitudes), as unsigned ones
        for (int k = k_first; k < k_end; k += 512) {
            raw = *reinterpret_cast<const uint4*>(src + k);
            const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (ZERO) { up = pair_max_signed(up, w[j]); down = pair_max(down, w[j]); }
                else up = pair_max(up, w[j] & 0x7fff7fffu);
            }
        }
        up = pair_max(up, up >> 16) & 0xffffu;
        down = pair_max(down, down >> 16) & 0xffffu;
        uint32_t most16 = up | (down & 0x8000u ? down & 0x7fffu : 0u) << 16;
        most16 = lanes_pair_max(most16, lanes);
        const uint32_t infinity = std::is_same<T, f16_t>::value ? 0x7c00u : 0x7f80u;
        odd = (most16 & 0xffffu) >= infinity || (ZERO && most16 >> 16 >= infinity);
        hi = V::E::lo(most16 & 0xffffu);
        lo = ZERO ? -V::E::lo(most16 >> 16) : -hi;
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) { f[2 * j] = V::E::lo(w[j]); f[2 * j + 1] = V::E::hi(w[j]); }
    } else {
        for (int k = k_first; k < k_end; k += 512) {
            V::load(src + k, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                lo = fminf(lo, f[j]); hi = fmaxf(hi, f[j]);
                odd |= !(fabsf(f[j]) <= 3.402823466e38f);
            }
        }
        for (int m = 1; m < lanes; m <<= 1) {
            lo = fminf(lo, __shfl_xor(lo, m)); hi = fmaxf(hi, __shfl_xor(hi, m)); odd |= (bool)__shfl_xor((int)odd, m);
        }
    }
    constexpr bool HALF = std::is_same<T, f16_t>::value;
    float s, z = 0.f;
    // Weights so large that their span, or a code times the scale, may pass the largest float (fp16: always looked after): the waves
    // that hold none do without what these need (14336 x 4104, bf16, 42.9 us, 43.8 with it in every wave).
    const bool vast = ZERO && !HALF && __builtin_amdgcn_ballot_w64(hi - lo > 0x1p120f) != 0;
    if constexpr (ZERO) {
        s = four_bits_up((hi - lo) / 15.f);
        if (vast && hi - lo > 0x1p120f) s = 2.f * four_bits_up((0.5f * hi - 0.5f * lo) / 15.f);
    } else s = four_bits(fmaxf(hi, -lo) / (CODE == DORA_QUANT_INT4 ? 7.f : 6.f));
    // What is read back stays finite: six times the largest number of four bits that allows it, and no code past the largest weight.
    if constexpr (CODE == DORA_QUANT_FP4) s = fminf(s, HALF ? 0x1.4p13f : 0x1.4p125f);
    if (odd) s = __uint_as_float(0x7fc00000u);
    const int64_t at = (int64_t)row * p.groups + g;
    const bool first = (threadIdx.x & (lanes - 1)) == 0;
    if constexpr (sizeof(T) == 2) {                    // as stored (fp16: small ones lose bits)
        uint32_t bits = 0;
        V::put(&bits, 0, s);
        s = V::one(&bits, 0);
    }
    const bool some = s > 0.f;                         // neither 0 nor NaN: otherwise the code of 0 everywhere
    // w / s is the product with 1 / s and one correction by its remainder, which is exact: the quotient rounded to nearest, a tie
    // between two codes among them.  Scales whose reciprocal or remainders would leave the normal range are lifted with their weights.
    const bool tiny = !HALF && some && s < 0x1p-100f;
    const float by = tiny ? s * 0x1p100f : s, inv = some ? 1.f / by : 0.f;
    auto over_s = [&](float v) { const float t = v * inv; return fmaf(fmaf(-t, by, v), inv, t); };
    const float most = HALF && some ? floorf(over_s(65504.f)) : 15.f;
    if constexpr (ZERO) z = some ? fminf(fmaxf(rintf(over_s(tiny ? -lo * 0x1p100f : -lo)), 0.f), 15.f) : 0.f;
    if (first) {
        V::put(p.scale, at, s);
        if constexpr (ZERO) V::put(p.zero, at, z);
    }
    const float offset = ZERO ? z : 8.f;
    float least = fmaxf(-offset, -most), largest = fminf(15.f - offset, most);
    if (vast && s > 0x1p100f) {
        const float whole = floorf(over_s(std::is_same<T, bf16_t>::value ? 0x1.fep127f : 0x1.fffffep127f));
        least = fmaxf(least, -whole); largest = fminf(largest, whole);
        asm volatile("" : "+v"(least), "+v"(largest));   // (a branch, not a choice between values)
    }
    for (int k = k_first; k < k_end; k += 512) {
        if (group > 512) V::load(src + k, f);
        if (tiny) {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] *= 0x1p100f;
        }
        uint32_t word = 0;
        float t[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = over_s(f[j]);
        if constexpr (CODE == DORA_QUANT_INT4) {
            // four codes are one number, exact in fp32 (a scale of 0 has t = 0)
            float four[2] = {0.f, 0.f};
#pragma unroll
            for (int j = 7; j >= 0; --j)
                four[j / 4] = fmaf(four[j / 4], 16.f, __builtin_amdgcn_fmed3f(rintf(t[j]), least, largest) + offset);
            word = (uint32_t)four[0] | (uint32_t)four[1] << 16;
        } else if (some) {                             // the converter rounds to nearest, halfway to the even code, and ends at 6
            word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, t[0], t[1], 1.f, 0);
            word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, t[2], t[3], 1.f, 1);
            word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, t[4], t[5], 1.f, 2);
            word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, t[6], t[7], 1.f, 3);
        }
        p.q[((int64_t)row * p.d_in + k) >> 3] = word;
    }
}

// Eight weights to a thread, four times: 4 bytes of codes in, 16 (32) out.  Bound: memory (14336 x 4104, groups of 64, fp16: 24 us, 6.2
// TB/s).  The workgroups past those form Eq. 6 for the caller, a launch of its own otherwise (4.7 us of 14336 rows).
template <typename T, int CODE, bool ZERO>
__global__ __launch_bounds__(256) void dequantize_kernel(QuantWeight w, T* out, uint32_t words, uint32_t per_row, MagScaleArgs mag)
{
    typedef Eight<T> V;
    constexpr int U = 4;
    const uint32_t own = (words + 256u * U - 1) / (256u * U);
    if (blockIdx.x >= own) {
        const int64_t j = (int64_t)(blockIdx.x - own) * 256 + threadIdx.x;
        if (j >= w.d_out) return;
        const float c = mag.c[j], cc = (c < mag.eps) ? mag.eps : c, m = mag.m[j];
        if (mag.g) mag.g[j] = m / cc;
        if (mag.gm1) mag.gm1[j] = (m - cc) / cc;
        return;
    }
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
hipError_t quantize_t(QuantizeArgs a, int code, hipStream_t st)
{
    // (no more lanes than a short row has use for: 64 to each of 2^26 rows of 8 weights would be 2^32 threads, more than a launch takes)
    a.lane_shift = a.group_shift - 3 < 6 ? a.group_shift - 3 : 6;
    while (a.lane_shift > 2 && a.d_in <= 4 << a.lane_shift) --a.lane_shift;
    const int64_t threads = ((int64_t)a.d_out * a.groups) << a.lane_shift;
    const dim3 grid((unsigned)((threads + 255) / 256)), block(256);
    if (code == DORA_QUANT_FP4) quantize_kernel<T, DORA_QUANT_FP4, false><<<grid, block, 0, st>>>(a);
    else if (a.zero) quantize_kernel<T, DORA_QUANT_INT4, true><<<grid, block, 0, st>>>(a);
    else quantize_kernel<T, DORA_QUANT_INT4, false><<<grid, block, 0, st>>>(a);
    return hipGetLastError();
}

template <typename T>
hipError_t dequantize_t(const QuantWeight& w, void* out, const MagScaleArgs& mag, hipStream_t st)
{
    const uint32_t per_row = (uint32_t)w.d_in / 8, words = (uint32_t)w.d_out * per_row;   // (d_out d_in < 2^31)
    const dim3 grid((words + 1023) / 1024 + (mag.m ? (unsigned)(w.d_out + 255) / 256 : 0)), block(256);
    T* const o = static_cast<T*>(out);
    if (w.code == DORA_QUANT_FP4) dequantize_kernel<T, DORA_QUANT_FP4, false><<<grid, block, 0, st>>>(w, o, words, per_row, mag);
    else if (w.zero) dequantize_kernel<T, DORA_QUANT_INT4, true><<<grid, block, 0, st>>>(w, o, words, per_row, mag);
    else dequantize_kernel<T, DORA_QUANT_INT4, false><<<grid, block, 0, st>>>(w, o, words, per_row, mag);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize(int dtype, const void* W, int d_out, int d_in, int code, int group_shift, void* q, void* scale, void* zero,
                           hipStream_t st)
{
    TraceScope ts(DORA_K_QUANTIZE, st);
    const QuantizeArgs a{W, static_cast<uint32_t*>(q), scale, zero, d_out, d_in, group_shift, quant_groups(d_in, group_shift), 0};
    if (dtype == DORA_F32) return quantize_t<float>(a, code, st);
    return dtype == DORA_F16 ? quantize_t<f16_t>(a, code, st) : quantize_t<bf16_t>(a, code, st);
}

hipError_t launch_dequantize(int dtype, const QuantWeight& w, void* out, hipStream_t st, const MagScaleArgs& mag)
{
    TraceScope ts(DORA_K_DEQUANTIZE, st);
    if (dtype == DORA_F32) return dequantize_t<float>(w, out, mag, st);
    return dtype == DORA_F16 ? dequantize_t<f16_t>(w, out, mag, st) : dequantize_t<bf16_t>(w, out, mag, st);
}

}  // namespace dora
