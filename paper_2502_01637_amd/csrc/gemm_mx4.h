// Linear map with 4-bit weights and activations on the gfx950 matrix cores:
//
//   out[m, n] = act(sum_k x[m, k] w[n, k] + bias[n]) + residual[m, n]
//
// x and w are 4-bit rows (mx4.h); an x of another type is quantised first.  One
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 rows of w by 16 of x over a group of
// 128: lane l holds the 16 bytes of codes of row l % 16, block l / 16, and that block's
// scale byte, which the instruction applies.  Products of two codes are exact and the
// sums are fp32.  w is the first operand, so a lane's four accumulators are four
// consecutive n of one row m.
#pragma once

#include "gemm_bf16.h"
#include "mx4.h"

namespace scone {
namespace mx4 {

using gemm::f32x4;
typedef int i32x8 __attribute__((ext_vector_type(8)));

// What follows the sums.
struct Epilogue {
    const void* bias;      // [N] of bias_type, or null
    const void* residual;  // like out, or null
    void* out;
    int64_t ld;
    int64_t M, N;
    int32_t bias_type, out_type;
    bool gelu;
};

__device__ __forceinline__ float load_elem(const void* p, int32_t type, int64_t i) {
    if (type == SCONE_FP32) return static_cast<const float*>(p)[i];
    if (type == SCONE_BF16) return gemm::bf16_to_f32(static_cast<const uint16_t*>(p)[i]);
    return (float)static_cast<const _Float16*>(p)[i];
}

__device__ __forceinline__ void store_elem(void* p, int32_t type, int64_t i, float v) {
    if (type == SCONE_FP32) static_cast<float*>(p)[i] = v;
    else if (type == SCONE_BF16) static_cast<__bf16*>(p)[i] = (__bf16)v;
    else static_cast<_Float16*>(p)[i] = (_Float16)v;
}

__device__ __forceinline__ f32x4 mfma_mx4(const u32x4& a, const u32x4& b, const f32x4& c,
                                          uint32_t sa, uint32_t sb) {
    const i32x8 av = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
    const i32x8 bv = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, bv, c, 4, 4, 0, (int)sa, 0,
                                                            (int)sb);
}

// A workgroup of four wavefronts computes 64 x 64 of out, each 32 x 32 of it straight
// from memory.  Rows past the end read the last row and are not stored.
__global__ __launch_bounds__(256) void k_linear(const uint8_t* __restrict__ x,
                                                const uint8_t* __restrict__ w, int64_t K,
                                                Epilogue ep, int64_t tiles_n, int64_t block0) {
    const int64_t blk = block_index(block0);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t m0 = blk / tiles_n * 64 + (wave >> 1) * 32;
    const int64_t n0 = blk % tiles_n * 64 + (wave & 1) * 32;
    const int fr = lane & 15, q = lane >> 4;
    const int64_t rb = row_bytes(K), g = groups(K);
    const uint8_t *px[2], *pw[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int64_t m = m0 + i * 16 + fr, n = n0 + i * 16 + fr;
        px[i] = x + (m < ep.M ? m : ep.M - 1) * rb;
        pw[i] = w + (n < ep.N ? n : ep.N - 1) * rb;
    }
    f32x4 acc[2][2] = {};
    for (int64_t k = 0; k < g; ++k) {
        u32x4 a[2], b[2];
        uint32_t sa[2], sb[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            a[i] = *reinterpret_cast<const u32x4*>(pw[i] + k * 64 + q * 16);
            b[i] = *reinterpret_cast<const u32x4*>(px[i] + k * 64 + q * 16);
            sa[i] = pw[i][g * 64 + k * 4 + q];
            sb[i] = px[i][g * 64 + k * 4 + q];
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = mfma_mx4(a[i], b[j], acc[i][j], sa[i], sb[j]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t n = n0 + i * 16 + q * 4 + r, m = m0 + j * 16 + fr;
                if (m >= ep.M || n >= ep.N) continue;
                float v = acc[i][j][r];
                if (ep.bias) v += load_elem(ep.bias, ep.bias_type, n);
                if (ep.gelu) v = gemm::gelu_erf(v);
                if (ep.residual) v += load_elem(ep.residual, ep.out_type, m * ep.ld + n);
                store_elem(ep.out, ep.out_type, m * ep.ld + n, v);
            }
}

typedef float f32x16 __attribute__((ext_vector_type(16)));
using gemm::lds_ptr_t;

// Four values to or from consecutive elements of a type.
template <int kType>
__device__ __forceinline__ f32x4 load4(const void* p, int64_t i) {
    if constexpr (kType == SCONE_FP32) {
        typedef float f32x4_elem __attribute__((ext_vector_type(4), aligned(4)));
        return *reinterpret_cast<const f32x4_elem*>(static_cast<const float*>(p) + i);
    } else {
        typedef uint32_t u32x2_elem __attribute__((ext_vector_type(2), aligned(2)));
        const u32x2 v = *reinterpret_cast<const u32x2_elem*>(static_cast<const uint16_t*>(p) + i);
        f32x4 f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t h = (v[k / 2] >> (16 * (k & 1))) & 0xFFFFu;
            f[k] = kType == SCONE_BF16 ? gemm::bf16_to_f32(h)
                                       : (float)__builtin_bit_cast(_Float16, (uint16_t)h);
        }
        return f;
    }
}

template <int kType>
__device__ __forceinline__ void put4(void* p, int64_t i, const f32x4& v) {
    if constexpr (kType == SCONE_FP32) {
        typedef float f32x4_elem __attribute__((ext_vector_type(4), aligned(4)));
        __builtin_nontemporal_store(v, reinterpret_cast<f32x4_elem*>(static_cast<float*>(p) + i));
    } else {
        typedef uint32_t u32x2_elem __attribute__((ext_vector_type(2), aligned(2)));
        u32x2 o;
        if constexpr (kType == SCONE_BF16) {
            o.x = gemm::pack_bf16x2(v[0], v[1]);
            o.y = gemm::pack_bf16x2(v[2], v[3]);
        } else {
            o.x = __builtin_bit_cast(uint32_t, f16x2{(_Float16)v[0], (_Float16)v[1]});
            o.y = __builtin_bit_cast(uint32_t, f16x2{(_Float16)v[2], (_Float16)v[3]});
        }
        __builtin_nontemporal_store(o, reinterpret_cast<u32x2_elem*>(static_cast<uint16_t*>(p) + i));
    }
}

// s_waitcnt immediates as in gemm_bf16.h.
using gemm::kWaitLds;
using gemm::waitcnt_vm;

// A tile of 64 TM x 64 TN on four wavefronts, 32 TM x 32 TN each, in 32 x 32 x 64 scaled
// products (measured from registers 9,550 TFLOP/s against 7,190 for 16 x 16 x 128).
//
// A slab is one group of 128: 64 bytes of codes per row, which go from memory
// straight into a ring of three LDS stages.  One barrier per slab: behind it every
// wavefront's copies of the slab have landed and its reads of the slab before are done,
// so the stage of that one takes the copies of the slab after next.  A row's four
// 16-byte chunks lie at slot chunk ^ ((row >> 1) & 3), so that eight lanes that read
// one chunk of eight rows touch all banks.  Lane l of a product holds row l % 32 and
// block l / 32 of its 64-deep half; the scale bytes of four slabs come into a lane's
// registers as one load of its row, a group of four slabs ahead, shifted so that the
// lane's block is byte 0 or 2 for either half.
//
// Two such workgroups share a compute unit (128 accumulators a lane of 128 x 256), one
// of which can store its results while the other multiplies.
//
// Results go through LDS as fp32, 32 rows at a time in each wavefront's own part of the
// ring, and leave it by whole rows: a lane takes four consecutive n, adds the bias, and
// rounds once behind activation and residual.
template <int TM, int TN, int kOut, bool kResid>
__global__ __launch_bounds__(256, 2) void k_linear_tiles(const uint8_t* __restrict__ x,
                                                         const uint8_t* __restrict__ w, int g,
                                                         int rb, Epilogue ep, int64_t tiles_m,
                                                         int64_t tiles_n, int64_t block0) {
#if defined(__HIP_DEVICE_COMPILE__)  // the host has no buffer resources
    constexpr int BM = 64 * TM, BN = 64 * TN;
    constexpr int STAGE = (BM + BN) * 64;
    constexpr int PITCH = 32 * TN * 4 + 16;  // a staged row and 16 bytes against conflicts
    static_assert(4 * 32 * PITCH <= 3 * STAGE, "the staged rows take the ring's place");
    __shared__ __attribute__((aligned(1024))) uint8_t smem[3 * STAGE];

    int64_t m0, n0;
    {
        // As gemm::tile_at: each XCD a run of tiles, eight rows of tiles a group.
        const int64_t nb = tiles_m * tiles_n, b = block_index(block0), per = nb / 8;
        const int64_t t = b < per * 8 ? (b % 8) * per + b / 8 : b;
        const int64_t group = t / (8 * tiles_n), first = group * 8;
        const int64_t gm = tiles_m - first < 8 ? tiles_m - first : 8;
        const int64_t tr = t - group * 8 * tiles_n;
        m0 = (first + tr % gm) * BM;
        n0 = tr / gm * BN;
    }
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    // Rows past the end read the last row; their results are not stored.
    const int rows_m = (int)(ep.M - m0 < BM ? ep.M - m0 : BM);
    const int rows_n = (int)(ep.N - n0 < BN ? ep.N - n0 : BN);
    // Buffers: the slab's place is a scalar offset, so copies take no vector arithmetic.
    const auto px = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(x + m0 * rb), 0,
                                                      rows_m * rb, 0x20000);
    const auto pw = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(w + n0 * rb), 0,
                                                      rows_n * rb, 0x20000);
    // Copies: an instruction fills 16 rows, lane l slot l % 4 of row l / 4.
    int cx[TM], cw[TN];
    {
        const int chunk = ((lane & 3) ^ ((lane >> 3) & 3)) * 16;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int r = (wave * TM + i) * 16 + (lane >> 2);
            cx[i] = (r < rows_m ? r : rows_m - 1) * rb + chunk;
        }
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            const int r = (wave * TN + i) * 16 + (lane >> 2);
            cw[i] = (r < rows_n ? r : rows_n - 1) * rb + chunk;
        }
    }
    auto issue = [&](int slab) {
        uint8_t* at = smem + slab % 3 * STAGE + wave * TM * 1024;
#pragma unroll
        for (int i = 0; i < TM; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(px, (lds_ptr_t)(at + i * 1024), 16, cx[i],
                                                     slab * 64, 0, 0);
        at = smem + slab % 3 * STAGE + BM * 64 + wave * TN * 1024;
#pragma unroll
        for (int i = 0; i < TN; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(pw, (lds_ptr_t)(at + i * 1024), 16, cw[i],
                                                     slab * 64, 0, 0);
    };
    const int fr = lane & 31, half = lane >> 5;
    int sx[TM], sw[TN];  // where the lane's scale bytes are
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int r = wm * 32 * TM + i * 32 + fr;
        sx[i] = (r < rows_m ? r : rows_m - 1) * rb + 64 * g;
    }
#pragma unroll
    for (int i = 0; i < TN; ++i) {
        const int r = wn * 32 * TN + i * 32 + fr;
        sw[i] = (r < rows_n ? r : rows_n - 1) * rb + 64 * g;
    }
    u32x4 nx[TM], nw[TN], vx[TM], vw[TN];  // scales of the next and of this group of slabs
    auto load_scales = [&](int slab) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
            nx[i] = __builtin_bit_cast(
                u32x4, __builtin_amdgcn_raw_buffer_load_b128(px, sx[i], slab * 4, 0));
#pragma unroll
        for (int i = 0; i < TN; ++i)
            nw[i] = __builtin_bit_cast(
                u32x4, __builtin_amdgcn_raw_buffer_load_b128(pw, sw[i], slab * 4, 0));
    };

    f32x16 acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

    const int swz = (fr >> 1) & 3;
    const uint8_t* fx = smem + (wm * 32 * TM + fr) * 64;
    const uint8_t* fw = smem + BM * 64 + (wn * 32 * TN + fr) * 64;
    constexpr int kCopies = TM + TN;

    // Slab k, the j-th of its group.  kWhole: slabs k + 1 and k + 2 and the next group's
    // scales exist; otherwise that is looked up.
    auto step = [&](int k, auto j_c, bool more, auto whole_c) {
        constexpr int j = decltype(j_c)::value;
        constexpr bool kWhole = decltype(whole_c)::value;
        // What may be outstanding behind slab k: the copies of slab k + 1 and, until
        // the last slab of the group, the next scales.
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(kWaitLds);
        if (kWhole || (k + 1 < g && more))
            __builtin_amdgcn_s_waitcnt(waitcnt_vm(j == 1 || j == 2 ? 2 * kCopies : kCopies));
        else if (k + 1 < g)
            __builtin_amdgcn_s_waitcnt(waitcnt_vm(kCopies));
        else
            __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        if (j == 0) {
#pragma unroll
            for (int i = 0; i < TM; ++i) vx[i] = nx[i] >> (8 * half);
#pragma unroll
            for (int i = 0; i < TN; ++i) vw[i] = nw[i] >> (8 * half);
        }
        if (kWhole || k + 2 < g) issue(k + 2);
        if (j == 0 && (kWhole || more)) {
            __builtin_amdgcn_sched_barrier(0);  // the waits count on this order
            load_scales(k + 4);
            __builtin_amdgcn_sched_barrier(0);
        }
        const int at = k % 3 * STAGE;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int slot = at + ((h * 2 + half) ^ swz) * 16;
            i32x8 a[TN], b[TM];
#pragma unroll
            for (int i = 0; i < TN; ++i) {
                const u32x4 v = *reinterpret_cast<const u32x4*>(fw + slot + i * 2048);
                a[i] = i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
            }
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const u32x4 v = *reinterpret_cast<const u32x4*>(fx + slot + i * 2048);
                b[i] = i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
            }
#pragma unroll
            for (int i = 0; i < TN; ++i)
#pragma unroll
                for (int m = 0; m < TM; ++m) {
                    const int sa = (int)vw[i][j], sb = (int)vx[m][j];
                    acc[i][m] = h == 0 ? __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                                             a[i], b[m], acc[i][m], 4, 4, 0, sa, 0, sb)
                                       : __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                                             a[i], b[m], acc[i][m], 4, 4, 2, sa, 2, sb);
                }
        }
    };
    using std::integral_constant;
    load_scales(0);
    issue(0);
    if (g > 1) issue(1);
    int k0 = 0;
    for (; k0 + 5 < g; k0 += 4) {
        step(k0, integral_constant<int, 0>{}, true, std::true_type{});
        step(k0 + 1, integral_constant<int, 1>{}, true, std::true_type{});
        step(k0 + 2, integral_constant<int, 2>{}, true, std::true_type{});
        step(k0 + 3, integral_constant<int, 3>{}, true, std::true_type{});
    }
    for (; k0 < g; k0 += 4) {
        const bool more = k0 + 4 < g;
        step(k0, integral_constant<int, 0>{}, more, std::false_type{});
        if (k0 + 1 < g) step(k0 + 1, integral_constant<int, 1>{}, more, std::false_type{});
        if (k0 + 2 < g) step(k0 + 2, integral_constant<int, 2>{}, more, std::false_type{});
        if (k0 + 3 < g) step(k0 + 3, integral_constant<int, 3>{}, more, std::false_type{});
    }

    // acc[i][m][r] is out[row m * 32 + lane % 32, n i * 32 + 8 (r / 4) + 4 (lane / 32) + r % 4].
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(kWaitLds);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    uint8_t* part = smem + wave * 32 * PITCH;
    constexpr int LPR = 8 * TN;     // lanes a row, four n each
    constexpr int RPI = 64 / LPR;   // rows an instruction
    constexpr int kBatch = 4;       // instructions whose residuals are in flight together
    const int er = lane / LPR, ec = lane % LPR * 4;
    const int64_t n = n0 + wn * 32 * TN + ec;
    const int left = (int)(ep.N - n < 4 ? (ep.N - n < 0 ? 0 : ep.N - n) : 4);
    f32x4 bias = {0.f, 0.f, 0.f, 0.f};
    if (ep.bias)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) bias[e] = load_elem(ep.bias, ep.bias_type, n + e);
#pragma unroll
    for (int m = 0; m < TM; ++m) {
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<f32x4*>(part + fr * PITCH + (i * 32 + q * 8 + half * 4) * 4) =
                    f32x4{acc[i][m][q * 4], acc[i][m][q * 4 + 1], acc[i][m][q * 4 + 2],
                          acc[i][m][q * 4 + 3]};
        const int64_t row0 = m0 + (wm * TM + m) * 32 + er;
#pragma unroll
        for (int it = 0; it < 32 / RPI; it += kBatch) {
            f32x4 res[kBatch];
            if constexpr (kResid) {
#pragma unroll
                for (int u = 0; u < kBatch; ++u) {
                    const int64_t row = row0 + (it + u) * RPI;
                    res[u] = f32x4{0.f, 0.f, 0.f, 0.f};
                    if (row < ep.M) {
                        if (left == 4) res[u] = load4<kOut>(ep.residual, row * ep.ld + n);
                        else
#pragma unroll
                            for (int e = 0; e < 3; ++e)
                                if (e < left) res[u][e] = load_elem(ep.residual, kOut, row * ep.ld + n + e);
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int64_t row = row0 + (it + u) * RPI;
                f32x4 v = *reinterpret_cast<const f32x4*>(part + ((it + u) * RPI + er) * PITCH + ec * 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += bias[e];
                if (ep.gelu)
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = gemm::gelu_erf(v[e]);
                if constexpr (kResid)
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] += res[u][e];
                if (row < ep.M) {
                    if (left == 4) put4<kOut>(ep.out, row * ep.ld + n, v);
                    else
#pragma unroll
                        for (int e = 0; e < 3; ++e)
                            if (e < left) store_elem(ep.out, kOut, row * ep.ld + n + e, v[e]);
                }
            }
        }
    }
#endif
}

template <int TM, int TN, int kOut, bool kResid>
inline hipError_t launch_tiles(const uint8_t* x, const uint8_t* w, int64_t K, const Epilogue& ep,
                               hipStream_t st) {
    const int64_t tiles_m = (ep.M + 64 * TM - 1) / (64 * TM);
    const int64_t tiles_n = (ep.N + 64 * TN - 1) / (64 * TN);
    return launch_blocks(tiles_m * tiles_n, 256, [&](int64_t b0, dim3 grid) {
        hipLaunchKernelGGL((k_linear_tiles<TM, TN, kOut, kResid>), grid, dim3(256), 0, st, x, w,
                           (int)groups(K), (int)row_bytes(K), ep, tiles_m, tiles_n, b0);
    });
}

template <int TM, int TN>
inline hipError_t launch_tiles(const uint8_t* x, const uint8_t* w, int64_t K, const Epilogue& ep,
                               hipStream_t st) {
    const bool r = ep.residual != nullptr;
    switch (ep.out_type) {
        case SCONE_BF16:
            return r ? launch_tiles<TM, TN, SCONE_BF16, true>(x, w, K, ep, st)
                     : launch_tiles<TM, TN, SCONE_BF16, false>(x, w, K, ep, st);
        case SCONE_FP16:
            return r ? launch_tiles<TM, TN, SCONE_FP16, true>(x, w, K, ep, st)
                     : launch_tiles<TM, TN, SCONE_FP16, false>(x, w, K, ep, st);
        default:
            return r ? launch_tiles<TM, TN, SCONE_FP32, true>(x, w, K, ep, st)
                     : launch_tiles<TM, TN, SCONE_FP32, false>(x, w, K, ep, st);
    }
}

inline hipError_t linear(const uint8_t* x, const uint8_t* w, int64_t K, const Epilogue& ep,
                         hipStream_t st) {
    if (ep.M > 64) {
        const int64_t big = ((ep.M + 127) / 128) * ((ep.N + 255) / 256);
        return big >= 256 ? launch_tiles<2, 4>(x, w, K, ep, st) : launch_tiles<1, 2>(x, w, K, ep, st);
    }
    const int64_t tiles_m = (ep.M + 63) / 64, tiles_n = (ep.N + 63) / 64;
    return launch_blocks(tiles_m * tiles_n, 256, [&](int64_t b0, dim3 grid) {
        hipLaunchKernelGGL(k_linear, grid, dim3(256), 0, st, x, w, K, ep, tiles_n, b0);
    });
}

}  // namespace mx4
}  // namespace scone
