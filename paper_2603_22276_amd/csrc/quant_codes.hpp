// 4-bit frozen weights: what a word of codes stands for, and eight elements of a storage type at a time.
#pragma once

#include "lds_tile.hpp"

namespace dora {
namespace {

// Eight consecutive elements of a row, aligned to 16 bytes.
template <typename T> struct Eight;
template <int DT>
struct Eight16 {
    typedef Elem16<DT> E;
    static __device__ __forceinline__ void load(const void* p, float (&f)[8])
    {
        const uint4 r = *reinterpret_cast<const uint4*>(p);
        f[0] = E::lo(r.x); f[1] = E::hi(r.x); f[2] = E::lo(r.y); f[3] = E::hi(r.y);
        f[4] = E::lo(r.z); f[5] = E::hi(r.z); f[6] = E::lo(r.w); f[7] = E::hi(r.w);
    }
    static __device__ __forceinline__ void store(void* p, const float (&f)[8])
    {
        uint4 r;
        r.x = E::pack2(f[0], f[1]); r.y = E::pack2(f[2], f[3]); r.z = E::pack2(f[4], f[5]); r.w = E::pack2(f[6], f[7]);
        *reinterpret_cast<uint4*>(p) = r;
    }
    static __device__ __forceinline__ float one(const void* p, int64_t i) { return E::lo(static_cast<const uint16_t*>(p)[i]); }
    static __device__ __forceinline__ void put(void* p, int64_t i, float v) { static_cast<uint16_t*>(p)[i] = (uint16_t)E::pack2(v, 0.f); }
};
template <> struct Eight<bf16_t> : Eight16<DT_BF16> {};
template <> struct Eight<f16_t> : Eight16<DT_F16> {};
template <> struct Eight<float> {
    static __device__ __forceinline__ void load(const void* p, float (&f)[8])
    {
        const float4 a = static_cast<const float4*>(p)[0], b = static_cast<const float4*>(p)[1];
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
    static __device__ __forceinline__ void store(void* p, const float (&f)[8])
    {
        static_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
        static_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
    }
    static __device__ __forceinline__ float one(const void* p, int64_t i) { return static_cast<const float*>(p)[i]; }
    static __device__ __forceinline__ void put(void* p, int64_t i, float v) { static_cast<float*>(p)[i] = v; }
};

// The values of the eight codes of a word (before zero point and scale), in the order of their columns.
template <int CODE>
__device__ __forceinline__ void decode8(uint32_t w, float (&f)[8])
{
    if constexpr (CODE == DORA_QUANT_FP4) {
        const f32x2_hw_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 1);
        const f32x2_hw_t c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 3);
        f[0] = a[0]; f[1] = a[1]; f[2] = b[0]; f[3] = b[1]; f[4] = c[0]; f[5] = c[1]; f[6] = d[0]; f[7] = d[1];
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = (float)((w >> (4 * j)) & 15u);
    }
}

// The same as one MFMA fragment: eight 16-bit numbers, exact (the codes of DORA_QUANT_INT4 as 0 .. 15).  A nibble q is the E4M3
// float q 2^-9 (its lowest sixteen codes run linearly through the subnormals), so the converter of that type, with a scale of
// 512, makes two integers of two bytes; nibbles are sorted into column order on the way.
template <int CODE, int DT>
__device__ __forceinline__ bf16x8_t decode_fragment(uint32_t w)
{
    typedef uint32_t u32x4_frag_t __attribute__((ext_vector_type(4)));
    u32x4_frag_t v;
    if constexpr (CODE == DORA_QUANT_FP4) {
        if constexpr (DT == DT_BF16) {
            v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 0));
            v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 1));
            v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 2));
            v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 3));
        } else {
            v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.f, 0));
            v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.f, 1));
            v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.f, 2));
            v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.f, 3));
        }
    } else {
        const uint32_t even = w & 0x0f0f0f0fu, odd = (w >> 4) & 0x0f0f0f0fu;
        const uint32_t a = __builtin_amdgcn_perm(odd, even, 0x05010400u), b = __builtin_amdgcn_perm(odd, even, 0x07030602u);
        if constexpr (DT == DT_BF16) {
            v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 512.f, false));
            v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 512.f, true));
            v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 512.f, false));
            v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 512.f, true));
        } else {
            v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 512.f, false));
            v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 512.f, true));
            v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 512.f, false));
            v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 512.f, true));
        }
    }
    return __builtin_bit_cast(bf16x8_t, v);
}

// ---- what the kernels that multiply with codes share ------------------------------------------------
constexpr uint32_t OUTSIDE = 0xFFFFFFFFu;              // beyond every descriptor: loads zeros
constexpr int BLOCK_K = 128;                           // columns of a step of the kernels that multiply with codes

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) const char* lds_cptr_t;

template <int OFF>
__device__ __forceinline__ uint64_t lds_read_b64(uint32_t addr)
{
    static_assert(OFF >= 0 && OFF < 65536, "ds_read offset field is 16 bits");
    uint64_t v;
    asm volatile("ds_read_b64 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF));
    return v;
}
template <int OFF>
__device__ __forceinline__ uint32_t lds_read_b32(uint32_t addr)
{
    static_assert(OFF >= 0 && OFF < 65536, "ds_read offset field is 16 bits");
    uint32_t v;
    asm volatile("ds_read_b32 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF));
    return v;
}
template <int OFF>
__device__ __forceinline__ uint32_t lds_read_u16(uint32_t addr)
{
    static_assert(OFF >= 0 && OFF < 65536, "ds_read offset field is 16 bits");
    uint32_t v;
    asm volatile("ds_read_u16 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF));
    return v;
}
// (the writes too: the compiler would have them wait for the loads to the LDS that are in flight)
__device__ __forceinline__ void lds_write_b128(uint32_t addr, const uint4& v)
{
    asm volatile("ds_write_b128 %0, %1" ::"v"(addr), "v"(__builtin_bit_cast(bf16x8_t, v)) : "memory");
}
__device__ __forceinline__ void lds_write_b32(uint32_t addr, uint32_t v) { asm volatile("ds_write_b32 %0, %1" ::"v"(addr), "v"(v) : "memory"); }

// 16 bytes per lane from memory into 1 KB of LDS
__device__ __forceinline__ void load_1k(char* lds, __amdgpu_buffer_rsrc_t rs, uint32_t off, uint32_t soffset)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void_ptr_t)lds, 16, off, soffset, 0, 0);
}
}  // namespace
}  // namespace dora
