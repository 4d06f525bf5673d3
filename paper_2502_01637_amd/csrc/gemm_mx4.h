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

inline hipError_t linear(const uint8_t* x, const uint8_t* w, int64_t K, const Epilogue& ep,
                  hipStream_t st) {
    const int64_t tiles_m = (ep.M + 63) / 64, tiles_n = (ep.N + 63) / 64;
    return launch_blocks(tiles_m * tiles_n, 256, [&](int64_t b0, dim3 grid) {
        hipLaunchKernelGGL(k_linear, grid, dim3(256), 0, st, x, w, K, ep, tiles_n, b0);
    });
}

}  // namespace mx4
}  // namespace scone
