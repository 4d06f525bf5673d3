// Rows in microscaled 4-bit floating point (OCP Microscaling Formats v1.0: E2M1
// elements in blocks of 32 that share a power of two, E8M0).
//
// A row of `cols` elements is g = ceil(cols / 128) groups of 128:
//   bytes [0, 64 g)        codes, element 2 i in the low half of byte i
//   bytes [64 g, 68 g)     scale bytes, one per 32 elements
//   up to a multiple of 16 zeros
// so that a row starts 16-byte aligned, a 128-deep slice of it is 64 bytes of codes
// and one word of scales (what one scaled matrix instruction takes), and a row is
// one run of bytes for the calls that move rows (gather, split, host placement).
// Codes past `cols` are zero.  A code's sign is bit 3, its magnitude one of
// 0, 1/2, 1, 3/2, 2, 3, 4, 6; its value that times 2^(s - 127), s the scale byte;
// s = 255 makes the block NaN.
#pragma once

#include "scone_internal.h"

namespace scone {
namespace mx4 {

constexpr int64_t kMaxCols = (int64_t)1 << 22;  // byte offsets inside 512 rows fit 31 bits

__host__ __device__ constexpr int64_t groups(int64_t cols) { return (cols + 127) / 128; }
__host__ __device__ constexpr int64_t row_bytes(int64_t cols) {
    return (68 * groups(cols) + 15) / 16 * 16;
}

inline bool cols_ok(int64_t cols) { return cols >= 1 && cols <= kMaxCols; }

// Bytes of an element of a scone_type, 0 for any other value (SCONE_MX4 among them).
inline int elem_bytes(int32_t type) {
    return type == SCONE_BF16 || type == SCONE_FP16 ? 2 : type == SCONE_FP32 ? 4 : 0;
}

// 16 bytes at an address aligned to a 2-byte element only (global memory takes
// unaligned dwordx4 accesses).
typedef uint32_t u32x4_elem __attribute__((ext_vector_type(4), aligned(2)));

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// By value: a bit cast of a vector's element reads the vector's first.
template <typename T>
__device__ __forceinline__ T as(uint32_t w) {
    return __builtin_bit_cast(T, w);
}

// The conversions take the scale as a float and use its exponent field only, so a
// scale byte s is s << 23 (0 is 2^-127 and 255 NaN: checked on gfx950 over every
// scale and code, and the roundings at, above and below each midpoint).
__device__ __forceinline__ float scale_of(uint32_t s) { return __uint_as_float(s << 23); }

// Element types: eight elements as they lie in memory, their largest magnitude's
// exponent, and the conversions of eight elements.
template <int kType>
struct Elem;

template <>
struct Elem<SCONE_BF16> {
    typedef uint16_t type;
    typedef u32x4 vec;  // eight elements
    // The largest magnitude of two vectors' halves, as bits (they order like integers).
    __device__ __forceinline__ static uint32_t top(const vec& v) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = v[i] & 0x7FFFu, hi = (v[i] >> 16) & 0x7FFFu;
            m = m > lo ? m : lo;
            m = m > hi ? m : hi;
        }
        return m;
    }
    __device__ __forceinline__ static uint32_t field(uint32_t m) { return m >> 7; }
    __device__ __forceinline__ static uint32_t quantize(const vec& v, float scale) {
        uint32_t q = 0;
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, as<bf16x2>(v[0]), scale, 0);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, as<bf16x2>(v[1]), scale, 1);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, as<bf16x2>(v[2]), scale, 2);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, as<bf16x2>(v[3]), scale, 3);
        return q;
    }
    __device__ __forceinline__ static vec values(uint32_t q, float scale) {
        vec v;
        v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, scale, 0));
        v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, scale, 1));
        v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, scale, 2));
        v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, scale, 3));
        return v;
    }
};

template <>
struct Elem<SCONE_FP16> {
    typedef uint16_t type;
    typedef u32x4 vec;
    __device__ __forceinline__ static uint32_t top(const vec& v) { return Elem<SCONE_BF16>::top(v); }
    __device__ __forceinline__ static uint32_t field(uint32_t m) {
        const _Float16 h = __builtin_bit_cast(_Float16, (uint16_t)m);
        return __float_as_uint((float)h) >> 23;  // exact, subnormals too
    }
    __device__ __forceinline__ static uint32_t quantize(const vec& v, float scale) {
        uint32_t q = 0;
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(q, as<f16x2>(v[0]), scale, 0);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(q, as<f16x2>(v[1]), scale, 1);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(q, as<f16x2>(v[2]), scale, 2);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(q, as<f16x2>(v[3]), scale, 3);
        return q;
    }
    __device__ __forceinline__ static vec values(uint32_t q, float scale) {
        vec v;
        v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(q, scale, 0));
        v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(q, scale, 1));
        v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(q, scale, 2));
        v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(q, scale, 3));
        return v;
    }
};

template <>
struct Elem<SCONE_FP32> {
    typedef uint32_t type;
    typedef uint32_t vec __attribute__((ext_vector_type(8)));
    __device__ __forceinline__ static uint32_t top(const vec& v) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t a = v[i] & 0x7FFFFFFFu;
            m = m > a ? m : a;
        }
        return m;
    }
    __device__ __forceinline__ static uint32_t field(uint32_t m) { return m >> 23; }
    __device__ __forceinline__ static uint32_t quantize(const vec& v, float scale) {
        uint32_t q = 0;
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __uint_as_float(v[0]), __uint_as_float(v[1]), scale, 0);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __uint_as_float(v[2]), __uint_as_float(v[3]), scale, 1);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __uint_as_float(v[4]), __uint_as_float(v[5]), scale, 2);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __uint_as_float(v[6]), __uint_as_float(v[7]), scale, 3);
        return q;
    }
};

// The scale byte of a block whose largest magnitude has this exponent field (that of
// a float): 2^(floor(log2 top) - 2), so that the largest element lies in [4, 8) steps
// of it (those above 6 round to 6); the smallest scale below 2^-125; NaN with an
// infinity or a NaN in the block.
__device__ __forceinline__ uint32_t scale_byte(uint32_t field) {
    return field == 255 ? 255u : field < 2 ? 0u : field - 2;
}

// Codes of eight elements, 16 lanes in a row holding a group of 128: each block of 32 is
// four lanes, whose largest magnitudes are joined by two exchanges; the group's four
// scale bytes are joined to a word the same way.
template <int kType>
__device__ __forceinline__ uint32_t quantize8(const typename Elem<kType>::vec& v,
                                              uint32_t& word) {
    typedef Elem<kType> E;
    uint32_t top = E::top(v);
    uint32_t o = __shfl_xor(top, 1);
    top = top > o ? top : o;
    o = __shfl_xor(top, 2);
    top = top > o ? top : o;
    const uint32_t s = scale_byte(E::field(top));
    word = s << (8 * ((threadIdx.x >> 2) & 3));
    word |= __shfl_xor(word, 4);
    word |= __shfl_xor(word, 8);
    return s == 255 ? 0u : E::quantize(v, scale_of(s));
}

// Eight elements from address p, of which the first n are there (n < 8: one by one).
template <int kType>
__device__ __forceinline__ typename Elem<kType>::vec load8(
    const typename Elem<kType>::type* p, int64_t n) {
    typedef typename Elem<kType>::vec vec;
    vec v{};
    if (n >= 8) {
        const u32x4_elem* q = reinterpret_cast<const u32x4_elem*>(p);
        if constexpr (sizeof(vec) == 16) {
            v = q[0];
        } else {
            const u32x4 a = q[0], b = q[1];
            v = vec{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        }
        return v;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t e = i < n ? (uint32_t)p[i] : 0u;
        if constexpr (sizeof(typename Elem<kType>::type) == 4) v[i] = e;
        else v[i / 2] |= e << (16 * (i & 1));
    }
    return v;
}

// A lane's share of a row on its way out: 16 bytes, so that the lanes of a store cover
// whole lines (two halves of 32 bytes of fp32, eight elements, took 450 us for the values
// of 131,072 rows of 2,048 where pieces of four take 163).
template <int kType>
struct Out {
    static constexpr int kElems = sizeof(typename Elem<kType>::type) == 4 ? 4 : 8;
    // The piece's codes in their word (fp32: the low half of it).
    __device__ __forceinline__ static uint32_t load(const uint8_t* row, int64_t c) {
        if constexpr (kElems == 8) return reinterpret_cast<const uint32_t*>(row)[c];
        else return reinterpret_cast<const uint16_t*>(row)[c];
    }
    __device__ __forceinline__ static u32x4 values(uint32_t q, uint32_t s) {
        const float scale = scale_of(s);
        if constexpr (kElems == 8) return Elem<kType>::values(q, scale);
        else {
            const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, scale, 0);
            const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, scale, 1);
            return u32x4{__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x),
                         __float_as_uint(b.y)};
        }
    }
    // The first n elements of a piece to address p.
    __device__ __forceinline__ static void store(typename Elem<kType>::type* p, int64_t n,
                                                 const u32x4& v) {
        if (n >= kElems) {
            __builtin_nontemporal_store(v, reinterpret_cast<u32x4_elem*>(p));
            return;
        }
#pragma unroll
        for (int i = 0; i < kElems; ++i) {
            if (i < n) {
                if constexpr (kElems == 4) p[i] = v[i];
                else p[i] = (uint16_t)(v[i / 2] >> (16 * (i & 1)));
            }
        }
    }
};

// Quantise rows (the whole of scone_quantize_mx4 after its argument checks).
hipError_t quantize(const void* x, int32_t type, int64_t n_rows, int64_t cols, int64_t ld,
                    void* rows, hipStream_t st);

}  // namespace mx4
}  // namespace scone
