// What the calls on a paged cache in 8 bits share: the checks of the cache, the way from a position to its codes and scale, the two formats.
#pragma once
#include "mfma.h"
#include "paged.h"

namespace el {

constexpr int kMaxPage8 = 1 << 16;       // positions of a page: a quotient by a block's size is then a product with kMagic / block (Quotient)

// Host: EL_OK if the cache is one that the kernels cover (el_attn.h states the rules).
el_status check_pages8(const el_attn_pages8 *c);
PageView page_view8(const el_attn_pages8 &c, const int32_t *table, int64_t table_stride, int table_pages);

// x / by for x and by up to 2^16: x times the quotient 2^32 / by rounded up is off by less than x by, which 2^32 exceeds unless both are 2^16 (exact then).
struct Quotient {
    uint64_t factor;
    __host__ __device__ __forceinline__ unsigned of(unsigned x) const { return (unsigned)(x * factor >> 32); }
};
inline Quotient quotient(int by) { return Quotient{(((uint64_t)1 << 32) + by - 1) / by}; }

struct ScaleView {
    float *K, *V;                        // [pages, kv_heads, per]
    int block, per;                      // positions that share a scale; scales of a page and head
    Quotient by_block;
};
inline ScaleView scale_view(const el_attn_pages8 &c) { return ScaleView{c.K_scale, c.V_scale, c.block, c.page_size / c.block, quotient(c.block)}; }

// Codes of 8 bits: the largest, and the nearest to y, |y| beyond the largest taken as that.  A NaN stays one in e4m3 and is 0 among integers.
template <int FMT> struct Code;
template <> struct Code<EL_E4M3> {
    static constexpr float most = 448.f;
    static __device__ __forceinline__ float clamped(float y) { return y > most ? most : y < -most ? -most : y; }
    // four at once, the first in the lowest byte (the instruction rounds to the nearest, ties to even)
    static __device__ __forceinline__ unsigned of4(float a, float b, float c, float d)
    {
        const int low = __builtin_amdgcn_cvt_pk_fp8_f32(clamped(a), clamped(b), 0, false);
        return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(clamped(c), clamped(d), low, true);
    }
    // (none of them NaN or beyond the largest by more than a quarter of a step)
    static __device__ __forceinline__ unsigned of4_inside(float a, float b, float c, float d)
    {
        const int low = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, low, true);
    }
    static __device__ __forceinline__ f4 values(unsigned w)
    {
        const f2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        return f4{a[0], a[1], b[0], b[1]};
    }
};
template <> struct Code<EL_INT8> {
    static constexpr float most = 127.f;
    static __device__ __forceinline__ unsigned one(float y) { return y != y ? 0u : (unsigned)(int)rintf(fminf(fmaxf(y, -most), most)) & 0xffu; }
    static __device__ __forceinline__ unsigned of4(float a, float b, float c, float d) { return one(a) | one(b) << 8 | one(c) << 16 | one(d) << 24; }
    // (as above; the sum with 1.5 2^23 is rounded to an integer, whose last byte is the code)
    static __device__ __forceinline__ unsigned of4_inside(float a, float b, float c, float d)
    {
        auto bits = [](float y) __attribute__((always_inline)) {
#pragma clang fp contract(off)               // (y is rounded before it is added)
            return __float_as_uint(y + 0x1.8p23f);
        };
        const unsigned low = __builtin_amdgcn_perm(bits(b), bits(a), 0x0c0c0400u), high = __builtin_amdgcn_perm(bits(d), bits(c), 0x04000c0cu);
        return low | high;
    }
    static __device__ __forceinline__ f4 values(unsigned w)
    {
        return f4{(float)(int8_t)w, (float)(int8_t)(w >> 8), (float)(int8_t)(w >> 16), (float)(int8_t)(w >> 24)};
    }
};

} // namespace el
