// Linear map with 4-bit weights and activations on the gfx950 matrix cores:
//
//   out[m, n] = act(sum_k x[m, k] w[n, k] + bias[n]) + residual[m, n]
//
// x and w are 4-bit rows (mx4.h); an x of another type is quantised on the way.  A scaled
// matrix instruction multiplies codes by blocks of 32 and applies the two blocks' scale
// bytes: v_mfma_scale_f32_16x16x128_f8f6f4 takes 16 rows of each operand over a group of
// 128, lane l holding the 16 bytes of codes of row l % 16, block l / 16, and that block's
// scale byte; 32x32x64 takes 32 rows over two blocks, row l % 32 and block l / 32.
// Products of two codes are exact and the sums are fp32.  w is the first operand, so
// that four accumulators of a lane in a row are four consecutive n of one row m.
//
// With few rows of x the weights bound the time and go straight into the lanes
// (k_linear_few); beyond them both operands are laid out for tiles (k_slabs) that go through
// LDS (k_linear_tiles).
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

typedef float f32x16 __attribute__((ext_vector_type(16)));
using gemm::lds_ptr_t;

// 16 bytes of a type as floats: four of fp32, eight of the others.
template <int kType>
constexpr int kPer16 = kType == SCONE_FP32 ? 4 : 8;

template <int kType>
__device__ __forceinline__ void widen(const u32x4& v, float (&f)[kPer16<kType>]) {
#pragma unroll
    for (int i = 0; i < kPer16<kType>; ++i) {
        if constexpr (kType == SCONE_FP32) f[i] = __uint_as_float(v[i]);
        else if constexpr (kType == SCONE_BF16)
            f[i] = __uint_as_float(i & 1 ? v[i / 2] & 0xFFFF0000u : v[i / 2] << 16);
        else f[i] = (float)__builtin_bit_cast(_Float16, (uint16_t)(v[i / 2] >> (16 * (i & 1))));
    }
}

// The values are fp32 before they are rounded: without the empty asm the compiler joins
// a multiply-add that computes one with its rounding to fp16 (v_fma_mix) where no branch
// lies between, and a value's last bit went by the tile that it lay in.
template <int kType>
__device__ __forceinline__ u32x4 narrow(const float (&f)[kPer16<kType>]) {
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (kType == SCONE_FP32) v[i] = __float_as_uint(f[i]);
        else if constexpr (kType == SCONE_BF16) v[i] = gemm::pack_bf16x2(f[2 * i], f[2 * i + 1]);
        else {
            float a = f[2 * i], b = f[2 * i + 1];
            asm("" : "+v"(a), "+v"(b));
            v[i] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)a, (_Float16)b});
        }
    }
    return v;
}

// Few rows of x: the weights are read once, from memory straight into the lanes, and
// bound the time.  A workgroup of kFewWaves wavefronts takes 16 rows of w; a round is
// kFewWaves groups, one a wavefront, whose weights are on their way kFewAhead rounds
// ahead.  The workgroup quantises x itself, a chunk of rounds at a time into LDS, so that
// there is one launch and no scratch.  The sums of the wavefronts are joined in LDS in
// their order.
//
// In LDS a row's four 16-byte blocks of a group lie at slot block ^ s with s = -(row / 4)
// mod 4: the 16 lanes of a read that are served at once (k_linear_tiles) are then four
// rows at one block and the other twelve at the same or the next, each in its own banks.
constexpr int kFewWaves = 8, kFewAhead = 4;

// Rounds in LDS at once for MT * 16 rows: 34 KiB.  Registers bound the workgroups of a
// compute unit to three (up to 80: MT = 1, 2 of 16-bit types without kEnd) or two; 64, for
// a fourth, spill: 22.4 us where 20.9 without (16 rows of 16,384 x 4,096).
constexpr int few_rounds(int mt) { return 4 / mt; }

// Eight elements without the first d of them (d < 8), zeros behind.
template <int kType>
__device__ __forceinline__ typename Elem<kType>::vec drop(typename Elem<kType>::vec v, uint32_t d) {
    constexpr int W = sizeof(v) / 4, kPerWord = 8 / W;  // words, elements in each
#pragma unroll
    for (int step = W / 2; step >= 1; step /= 2) {
        const bool on = d & (step * kPerWord);
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = on ? (i + step < W ? v[i + step] : 0u) : v[i];
    }
    if constexpr (kPerWord == 2) {
#pragma unroll
        for (int i = 0; i < W; ++i)
            v[i] = d & 1 ? (v[i] >> 16) | (i + 1 < W ? v[i + 1] << 16 : 0u) : v[i];
    }
    return v;
}

// Codes and scale byte of a block of 32, elements e on of the K that begin at x[row].
// kEnd: K is no multiple of 32.  Eights that pass the row's end are loaded from K - 8 on
// and moved, so that every lane has its loads on their way at once: element by element,
// behind a branch, 16 rows of 4,001 x 1,500 took 6.7 us, now 5.1 (K = 1,536 4.4), 32 rows
// 9.1 and 7.1.  It needs 17 to 41 registers more, so whole blocks have kernels without it,
// where a branch keeps the loads from being moved further up, which costs as many.
template <int kType, bool kEnd>
__device__ __forceinline__ u32x4 quantize32(const void* __restrict__ x, int64_t row, int64_t e,
                                            int64_t K, uint32_t& s) {
    typedef Elem<kType> E;
    const typename E::type* p = static_cast<const typename E::type*>(x) + row;
    typename E::vec v[4];
    if constexpr (!kEnd) {
        if (e + 32 <= K) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = load8<kType>(p + e + i * 8, 8);
        } else {
            for (int i = 0; i < 4; ++i) v[i] = typename E::vec{};
        }
    } else if (K >= 8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t from = e + i * 8;
            v[i] = load8<kType>(p + (from < K - 8 ? from : K - 8), 8);
        }
        if (e + 32 > K) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t d = e + i * 8 - (K - 8);
                if (d > 0) v[i] = d < 8 ? drop<kType>(v[i], (uint32_t)d) : typename E::vec{};
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = load8<kType>(p, e + i * 8 == 0 ? K : 0);
    }
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t t = E::top(v[i]);
        top = top > t ? top : t;
    }
    s = scale_byte(E::field(top));
    u32x4 codes;
#pragma unroll
    for (int i = 0; i < 4; ++i) codes[i] = s == 255 ? 0u : E::quantize(v[i], scale_of(s));
    return codes;
}

template <int kType, int MT, bool kEnd>
__global__ __launch_bounds__(64 * kFewWaves) void k_linear_few(const void* __restrict__ x,
                                                               int64_t ld,
                                                               const uint8_t* __restrict__ w,
                                                               int64_t K, Epilogue ep,
                                                               int64_t block0) {
    constexpr int kRows = 16 * MT, kRounds = few_rounds(MT), kChunk = kRounds * kFewWaves;
    constexpr bool kQuantize = kType != SCONE_MX4;
    // x's codes [group of the chunk][row][64] and scale words behind them; then the sums
    // [wavefront][row][16 n]
    constexpr int kCodes = kQuantize ? kChunk * kRows * 64 : 0;
    constexpr int kLds = kQuantize ? kCodes + kChunk * kRows * 4 : 0;
    constexpr int kSums = kFewWaves * kRows * 64;
    __shared__ __attribute__((aligned(16))) uint8_t smem[kLds > kSums ? kLds : kSums];
    const int lane = threadIdx.x & 63;
    // Known to be one per wavefront: what depends on it branches as a whole (a matrix
    // instruction takes no notice of lanes that are switched off).
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t n0 = block_index(block0) * 16;
    const int fr = lane & 15, q = lane >> 4;
    const int g = (int)groups(K), rb = (int)row_bytes(K);
    // Rows past the end read the last row and are not stored.
    const uint8_t* const pw = w + (n0 + fr < ep.N ? n0 + fr : ep.N - 1) * rb;
    const uint8_t* px[MT];
    if constexpr (!kQuantize)
#pragma unroll
        for (int i = 0; i < MT; ++i)
            px[i] = static_cast<const uint8_t*>(x) +
                    (i * 16 + fr < ep.M ? i * 16 + fr : ep.M - 1) * rb;
    u32x4 a[kFewAhead];
    uint32_t sa[kFewAhead];
    auto load = [&](int round, u32x4& v, uint32_t& s) {
        const int k = round * kFewWaves + wave;
        if (k >= g) return;
        v = *reinterpret_cast<const u32x4*>(pw + k * 64 + q * 16);
        s = pw[64 * (int64_t)g + k * 4 + q];
    };
    // Rows of x beyond M stay as they are in LDS: they reach only rows that are not stored.
    auto fill = [&](int k0) {
        if constexpr (kQuantize) {
            const int n = (g - k0 < kChunk ? g - k0 : kChunk) * 4;  // blocks of a row
            for (int u = threadIdx.x; u < (int)ep.M * n; u += 64 * kFewWaves) {
                const int r = u / n, c = u - r * n, k = c >> 2;
                uint32_t s;
                const u32x4 codes = quantize32<kType, kEnd>(x, r * ld, (int64_t)(k0 * 4 + c) * 32, K, s);
                const int slot = (c & 3) ^ (-(r >> 2) & 3);
                *reinterpret_cast<u32x4*>(smem + (k * kRows + r) * 64 + slot * 16) = codes;
                smem[kCodes + (k * kRows + r) * 4 + (c & 3)] = (uint8_t)s;
            }
        }
    };
    f32x4 acc[MT] = {};
    auto step = [&](int round, const u32x4& v, uint32_t s) {
        const int k = round * kFewWaves + wave;
        if (k >= g) return;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            u32x4 b;
            uint32_t sb;
            if constexpr (kQuantize) {
                const int at = k % kChunk * kRows + i * 16 + fr;
                b = *reinterpret_cast<const u32x4*>(smem + at * 64 +
                                                    ((q ^ (-(fr >> 2) & 3)) * 16));
                sb = *reinterpret_cast<const uint32_t*>(smem + kCodes + at * 4) >> (8 * q);
            } else {
                b = *reinterpret_cast<const u32x4*>(px[i] + k * 64 + q * 16);
                sb = px[i][64 * (int64_t)g + k * 4 + q];
            }
            acc[i] = mfma_mx4(v, b, acc[i], s, sb);
        }
    };
    const int rounds = (g + kFewWaves - 1) / kFewWaves;
#pragma unroll
    for (int j = 0; j < kFewAhead; ++j) load(j, a[j], sa[j]);
    for (int r0 = 0; r0 < rounds; r0 += kFewAhead) {
#pragma unroll
        for (int j = 0; j < kFewAhead; ++j) {
            const int r = r0 + j;
            if (r >= rounds) break;
            if (kQuantize && r % kRounds == 0) {
                if (r > 0) __syncthreads();
                fill(r * kFewWaves);
                __syncthreads();
            }
            step(r, a[j], sa[j]);
            load(r + kFewAhead, a[j], sa[j]);
        }
    }
    // acc[i][r] is out[i * 16 + lane % 16, n0 + 4 (lane / 16) + r].
    __syncthreads();
    float* const sums = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int i = 0; i < MT; ++i)
        *reinterpret_cast<f32x4*>(sums + ((wave * kRows + i * 16 + fr) * 16 + q * 4)) = acc[i];
    __syncthreads();
    for (int t = threadIdx.x; t < kRows * 16; t += 64 * kFewWaves) {
        const int64_t row = t >> 4, n = n0 + (t & 15);
        if (row >= ep.M || n >= ep.N) continue;
        float v = 0.f;
#pragma unroll
        for (int j = 0; j < kFewWaves; ++j) v += sums[j * kRows * 16 + t];
        if (ep.bias) v += load_elem(ep.bias, ep.bias_type, n);
        if (ep.gelu) v = gemm::gelu_erf(v);
        if (ep.residual) v += load_elem(ep.residual, ep.out_type, row * ep.ld + n);
        store_elem(ep.out, ep.out_type, row * ep.ld + n, v);
    }
}

template <int kType, int MT, bool kEnd>
inline hipError_t launch_few(const void* x, int64_t ld, const uint8_t* w, int64_t K,
                             const Epilogue& ep, hipStream_t st) {
    return launch_blocks((ep.N + 15) / 16, 64 * kFewWaves, [&](int64_t b0, dim3 grid) {
        hipLaunchKernelGGL((k_linear_few<kType, MT, kEnd>), grid, dim3(64 * kFewWaves), 0, st, x,
                           ld, w, K, ep, b0);
    });
}

template <int kType, int MT>
inline hipError_t launch_few(const void* x, int64_t ld, const uint8_t* w, int64_t K,
                             const Epilogue& ep, hipStream_t st) {
    if constexpr (kType != SCONE_MX4)
        if (K % 32 != 0) return launch_few<kType, MT, true>(x, ld, w, K, ep, st);
    return launch_few<kType, MT, false>(x, ld, w, K, ep, st);
}

template <int kType>
inline hipError_t launch_few(const void* x, int64_t ld, const uint8_t* w, int64_t K,
                             const Epilogue& ep, hipStream_t st) {
    if (ep.M <= 16) return launch_few<kType, 1>(x, ld, w, K, ep, st);
    if (ep.M <= 32) return launch_few<kType, 2>(x, ld, w, K, ep, st);
    return launch_few<kType, 4>(x, ld, w, K, ep, st);
}

using gemm::kWaitLds;
using gemm::waitcnt_vm;

// A matrix by groups, as the tiles read it: group k's codes of row r at byte
// (k ld + r) 64, its word of scales at k ld + r, so that a slab of a tile is one run of
// bytes.  The copies into LDS reach 37 TB/s on such runs, 13 to 16 on 64-byte pieces of
// 4-bit rows (whose pitch is no multiple of 128) and 20 to 32 on 128-byte pieces: with
// the rows' own layout an 8,192^3 product took 307 us, 204 of them without its copies.
struct Slabs {
    uint8_t* codes;
    uint32_t* scales;
    int64_t ld;
    float* bias;  // w's: what is added to row r's products
};

// Rows are laid out up to a multiple of the largest tile, and 320 more, which a tile's
// copy of 256 scale words may reach and which keep the groups of a row off powers of two;
// what lies past the last row is never written, and only feeds results that are never
// stored.
inline int64_t slabs_ld(int64_t n) { return (n + 255) / 256 * 256 + 320; }
inline int64_t slabs_bytes(int64_t n, int64_t K) { return slabs_ld(n) * (groups(K) * 68 + 4); }
inline Slabs slabs_at(uint8_t* at, int64_t n, int64_t K) {
    const int64_t ld = slabs_ld(n);
    uint8_t* const words = at + ld * groups(K) * 64;
    return {at, reinterpret_cast<uint32_t*>(words), ld,
            reinterpret_cast<float*>(words + ld * groups(K) * 4)};
}

// 16 rows by four groups a workgroup, from 4-bit rows: a wavefront copies the codes of
// one group, four lanes a row.
__device__ __forceinline__ void slabs_of_rows(const uint8_t* __restrict__ rows, int64_t n, int g,
                                              int rb, const Slabs& s, int64_t r0, int k0) {
    const int lane = threadIdx.x & 63, k = k0 + (threadIdx.x >> 6);
    const int64_t r = r0 + (lane >> 2);
    if (r >= n || k >= g) return;
    const uint8_t* row = rows + r * rb;
    const u32x4 v = *reinterpret_cast<const u32x4*>(row + k * 64 + (lane & 3) * 16);
    *reinterpret_cast<u32x4*>(s.codes + (k * s.ld + r) * 64 + (lane & 3) * 16) = v;
    if ((lane & 3) == 0)
        s.scales[k * s.ld + r] = *reinterpret_cast<const uint32_t*>(row + 64 * (int64_t)g + k * 4);
}

// The same from rows to quantise: 16 lanes hold a group of one row, as in k_quantize,
// a wavefront four rows and, one after another, four groups of them.
template <int kType>
__device__ __forceinline__ void slabs_of_elements(const typename Elem<kType>::type* __restrict__ x,
                                                  int64_t n, int64_t cols, int64_t ld, int g,
                                                  const Slabs& s, int64_t r0, int k0) {
    typedef Elem<kType> E;
    const int64_t r = r0 + (threadIdx.x >> 4);
    const int c = threadIdx.x & 15;
    typename E::vec v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int64_t e = (int64_t)(k0 + u) * 128 + c * 8;
        v[u] = load8<kType>(x + (r < n ? r * ld + e : 0), r < n ? cols - e : 0);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        uint32_t word;
        const uint32_t codes = quantize8<kType>(v[u], word);
        if (r >= n || k0 + u >= g) continue;
        const int64_t at = (k0 + u) * s.ld + r;
        reinterpret_cast<uint32_t*>(s.codes)[at * 16 + c] = codes;
        if (c == 0) s.scales[at] = word;
    }
}

inline int64_t slab_blocks(int64_t n, int64_t K) {
    return (n + 15) / 16 * ((groups(K) + 3) / 4);
}

// x's slabs (kType: its type) and then w's, with the biases as floats.
template <int kType>
__global__ __launch_bounds__(256) void k_slabs(const void* __restrict__ x, int64_t ld, int64_t M,
                                               Slabs sx, const uint8_t* __restrict__ w, int64_t N,
                                               Slabs sw, const void* __restrict__ bias,
                                               int32_t bias_type, int64_t K, int64_t x_blocks,
                                               int64_t block0) {
    const int g = (int)groups(K), quads = (g + 3) / 4;
    int64_t b = block_index(block0);
    const bool of_x = b < x_blocks;
    if (!of_x) b -= x_blocks;
    const int64_t r0 = b / quads * 16;
    const int k0 = (int)(b % quads) * 4;
    if (!of_x) {
        const int64_t r = r0 + threadIdx.x;
        if (k0 == 0 && threadIdx.x < 16 && r < N)
            sw.bias[r] = bias ? load_elem(bias, bias_type, r) : 0.f;
        slabs_of_rows(w, N, g, (int)row_bytes(K), sw, r0, k0);
    } else if constexpr (kType == SCONE_MX4)
        slabs_of_rows(static_cast<const uint8_t*>(x), M, g, (int)row_bytes(K), sx, r0, k0);
    else
        slabs_of_elements<kType>(static_cast<const typename Elem<kType>::type*>(x), M, K, ld, g,
                                 sx, r0, k0);
}

// A stage of the ring, and the workgroups of a compute unit that its 160 KiB hold.
constexpr int stage_bytes(int tm, int tn) { return 64 * (tm + tn) * 64 + 2048; }
constexpr int workgroups(int tm, int tn) {
    const int n = (160 << 10) / (3 * stage_bytes(tm, tn));
    return n < 4 ? n : 4;
}

// A tile of 64 TM x 64 TN on four wavefronts, 32 TM x 32 TN each, in 32 x 32 x 64 scaled
// products (measured from registers 9,550 TFLOP/s against 7,190 for 16 x 16 x 128).
//
// A slab is one group of 128: 64 bytes of codes and a word of scales per row (Slabs),
// which go from memory straight into a ring of three LDS stages.  A row's four 16-byte chunks
// lie at slot chunk ^ ((row >> 2) & 3): the 16 lanes that the LDS serves at once in a
// 16-byte read (0-3, 12-15, 20-23, 24-27, and the like) then touch every bank once.
// Lane l of a product holds row l % 32 and block l / 32 of its 64-deep half.
//
// A slab is two halves, whose fragments are double buffered in registers: the reads of
// one half run under the products of the other.  Between the halves lies the slab's one
// barrier: behind it every wavefront holds the whole slab in registers, so its stage
// takes the copies of the slab three further on, and the next slab has landed.
//
// Two such workgroups share a compute unit (128 accumulators a lane of 128 x 256), one
// of which can store its results while the other multiplies.
//
// Results go through LDS as fp32, 32 rows at a time in each wavefront's own part of the
// ring, and leave it by whole rows: a lane takes four consecutive n, adds the bias, and
// rounds once behind activation and residual.
//
// kLines: results pass by the caches.  So where rows are whole runs of 64 bytes;
// elsewhere the caches join what two workgroups write of one (36,827 x 2,507 x 804 to
// fp32 142 us past them, 127 through; x 2,544, 159 runs, 100 and 110; x 2,560 95 and 106;
// where all of the results fit the caches the two are within 5 % of each other).
template <int TM, int TN, int kOut, bool kResid, bool kLines>
__global__ __launch_bounds__(256, workgroups(TM, TN)) void k_linear_tiles(
    Slabs x, Slabs w, int g, Epilogue ep, uint32_t tiles_m, uint32_t tiles_n, int64_t block0) {
    constexpr int BM = 64 * TM, BN = 64 * TN;
    constexpr int SX = (BM + BN) * 64, SW = SX + 1024;  // the scales behind the codes
    constexpr int STAGE = stage_bytes(TM, TN);
    constexpr int PITCH = 32 * TN * 4 + 16;  // a staged row and 16 bytes against conflicts
    static_assert(4 * 32 * PITCH <= 3 * STAGE, "the staged rows take the ring's place");
    __shared__ __attribute__((aligned(1024))) uint8_t smem[3 * STAGE];

    int64_t m0, n0;
    {
        // As gemm::tile_at: each XCD a run of tiles, eight rows of tiles a group.
        const uint32_t nb = tiles_m * tiles_n, b = (uint32_t)block_index(block0), per = nb / 8;
        const uint32_t t = b < per * 8 ? (b % 8) * per + b / 8 : b;
        const uint32_t group = t / (8 * tiles_n), first = group * 8;
        const uint32_t gm = tiles_m - first < 8 ? tiles_m - first : 8;
        const uint32_t tr = t - group * 8 * tiles_n, tn = tr / gm;
        m0 = (int64_t)(first + tr - tn * gm) * BM;
        n0 = (int64_t)tn * BN;
    }
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    // Copies: an instruction fills 16 rows, lane l slot l % 4 of row l / 4.  Wavefronts 0
    // and 2 copy 256 words of x's scales, 1 and 3 of w's (twice, so that every wavefront
    // counts the same copies; as words of 64 lanes each they cost a fifth more: 98.8 us
    // against 118 for the sums of 65,459 x 1,024 x 4,096).
    constexpr int kCopies = TM + TN + 1;
    const bool odd = wave & 1;
    const uint8_t* const cx = x.codes + (m0 + wave * TM * 16) * 64;
    const uint8_t* const cw = w.codes + (n0 + wave * TN * 16) * 64;
    const uint32_t piece = (lane >> 2) * 64 + ((lane & 3) ^ ((lane >> 4) & 3)) * 16;
    auto issue = [&](int slab, int stage) {
        uint8_t* const at = smem + stage * STAGE;
        const uint8_t* const fx = cx + slab * x.ld * 64;
        const uint8_t* const fw = cw + slab * w.ld * 64;
#pragma unroll
        for (int i = 0; i < TM; ++i)
            __builtin_amdgcn_global_load_lds((gemm::gbl_ptr_t)(fx + i * 1024 + piece),
                                             (lds_ptr_t)(at + (wave * TM + i) * 1024), 16, 0, 0);
#pragma unroll
        for (int i = 0; i < TN; ++i)
            __builtin_amdgcn_global_load_lds(
                (gemm::gbl_ptr_t)(fw + i * 1024 + piece),
                (lds_ptr_t)(at + BM * 64 + (wave * TN + i) * 1024), 16, 0, 0);
        const uint32_t* const fs = odd ? w.scales + slab * w.ld + n0 : x.scales + slab * x.ld + m0;
        __builtin_amdgcn_global_load_lds((gemm::gbl_ptr_t)(fs + lane * 4),
                                         (lds_ptr_t)(at + (odd ? SW : SX)), 16, 0, 0);
    };

    // The sums begin with the biases; acc[i][m][r] is out[row m * 32 + lane % 32,
    // n i * 32 + 8 (r / 4) + 4 (lane / 32) + r % 4] of the wavefront's part.
    const int fr = lane & 31, half = lane >> 5;
    // Three slabs in flight (the last again where there are fewer).
    issue(0, 0);
    f32x4 bias[TN][4];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            bias[i][q] = *reinterpret_cast<const f32x4*>(w.bias + n0 + (wn * TN + i) * 32 + q * 8 +
                                                         half * 4);
    issue(g > 1 ? 1 : 0, 1);
    issue(g > 2 ? 2 : g - 1, 2);
    f32x16 acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = bias[i][r / 4][r % 4];

    const int swz = (fr >> 2) & 3;
    const int slots[2] = {(half ^ swz) * 16, ((2 + half) ^ swz) * 16};
    const uint8_t* const fx = smem + (wm * 32 * TM + fr) * 64;
    const uint8_t* const fw = smem + BM * 64 + (wn * 32 * TN + fr) * 64;
    const uint8_t* const gx = smem + SX + (wm * 32 * TM + fr) * 4;
    const uint8_t* const gw = smem + SW + (wn * 32 * TN + fr) * 4;
    u32x4 a0[TN], b0[TM], a1[TN], b1[TM];    // fragments of halves 0 and 1
    uint32_t va[TN], vb[TM], na[TN], nb[TM];  // scales of this slab and the next
    auto read = [&](int stage, int h, u32x4 (&a)[TN], u32x4 (&b)[TM]) {
        const int at = stage * STAGE + slots[h];
#pragma unroll
        for (int i = 0; i < TN; ++i) a[i] = *reinterpret_cast<const u32x4*>(fw + at + i * 2048);
#pragma unroll
        for (int i = 0; i < TM; ++i) b[i] = *reinterpret_cast<const u32x4*>(fx + at + i * 2048);
    };
    auto read_scales = [&](int stage) {
#pragma unroll
        for (int i = 0; i < TN; ++i)
            na[i] = *reinterpret_cast<const uint32_t*>(gw + stage * STAGE + i * 128);
#pragma unroll
        for (int i = 0; i < TM; ++i)
            nb[i] = *reinterpret_cast<const uint32_t*>(gx + stage * STAGE + i * 128);
    };
    auto take_scales = [&]() {  // the lane's blocks become bytes 0 and 2
#pragma unroll
        for (int i = 0; i < TN; ++i) va[i] = na[i] >> (8 * half);
#pragma unroll
        for (int i = 0; i < TM; ++i) vb[i] = nb[i] >> (8 * half);
    };
    auto multiply = [&](auto h_c, const u32x4 (&a)[TN], const u32x4 (&b)[TM]) {
        constexpr int kByte = decltype(h_c)::value * 2;
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            const i32x8 av = {(int)a[i][0], (int)a[i][1], (int)a[i][2], (int)a[i][3], 0, 0, 0, 0};
#pragma unroll
            for (int m = 0; m < TM; ++m) {
                const i32x8 bv = {(int)b[m][0], (int)b[m][1], (int)b[m][2], (int)b[m][3], 0, 0, 0, 0};
                acc[i][m] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                    av, bv, acc[i][m], 4, 4, kByte, (int)va[i], kByte, (int)vb[m]);
            }
        }
    };
    using std::integral_constant;
    constexpr int kMfma = 0x008, kVmemRead = 0x020, kDsRead = 0x100;
    // Slab k in stage `st`, its first half's fragments and scales in registers.
    // kMore: how many of the slabs behind it exist, up to three.
    auto step = [&](int k, int st, auto more_c) {
        constexpr int kMore = decltype(more_c)::value;
        const int next = st == 2 ? 0 : st + 1;
        take_scales();
        read(st, 1, a1, b1);
        multiply(integral_constant<int, 0>{}, a0, b0);
#pragma unroll
        for (int i = 0; i < TM + TN; ++i) {
            __builtin_amdgcn_sched_group_barrier(kDsRead, 1, 0);
            __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (kMore >= 1) {
            __builtin_amdgcn_s_waitcnt(kWaitLds);
            __builtin_amdgcn_s_waitcnt(waitcnt_vm(kMore >= 2 ? kCopies : 0));
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (kMore >= 3) issue(k + 3, st);
            read_scales(next);
            read(next, 0, a0, b0);
        }
        multiply(integral_constant<int, 1>{}, a1, b1);
        if constexpr (kMore >= 1) {
#pragma unroll
            for (int i = 0; i < TN * TM; ++i) {
                if constexpr (kMore >= 3) __builtin_amdgcn_sched_group_barrier(kVmemRead, 1, 1);
                __builtin_amdgcn_sched_group_barrier(kDsRead, 2, 1);
                __builtin_amdgcn_sched_group_barrier(kMfma, 1, 1);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(2 * kCopies));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    read_scales(0);
    read(0, 0, a0, b0);
    int k = 0, st = 0;
    for (; k + 3 < g; ++k) {
        step(k, st, integral_constant<int, 3>{});
        st = st == 2 ? 0 : st + 1;
    }
    if (k + 2 < g) {
        step(k++, st, integral_constant<int, 2>{});
        st = st == 2 ? 0 : st + 1;
    }
    if (k + 1 < g) {
        step(k++, st, integral_constant<int, 1>{});
        st = st == 2 ? 0 : st + 1;
    }
    step(k, st, integral_constant<int, 0>{});

    // With a single slab the copies of the other two stages may still be on their way
    // to where the results are staged; otherwise nothing is outstanding.
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
    __builtin_amdgcn_sched_barrier(0);
    // On the way out an instruction takes RPI rows, LPR lanes a row, V n (16 bytes) a lane;
    // NB batches of NI of them, whose residuals are loaded a batch ahead.
    constexpr int V = kPer16<kOut>, LPR = 32 * TN / V, RPI = 64 / LPR;
    constexpr int NI = 32 / RPI < 8 ? 32 / RPI : 8, NB = TM * (32 / RPI / NI);
    typedef uint32_t u32x4_out __attribute__((ext_vector_type(4), aligned(2)));
    constexpr int kSize = 16 / V;
    const int er = lane / LPR, ec = lane % LPR * V;
    const int64_t row0 = m0 + wm * TM * 32 + er, n = n0 + wn * 32 * TN + ec;
    const int64_t at0 = row0 * ep.ld + n;
    const bool inside = m0 + BM <= ep.M && n0 + BN <= ep.N;
    const int rows = (int)(ep.M - row0 < 32 * TM ? ep.M - row0 : 32 * TM);  // from row0 on
    const int left = (int)(ep.N - n < V ? ep.N - n : V);                     // and columns
    u32x4 res[2][kResid ? NI : 1];
    auto load_residuals = [&](int batch, u32x4 (&v)[kResid ? NI : 1]) {
        if constexpr (kResid) {
            const uint8_t* p = static_cast<const uint8_t*>(ep.residual) +
                               (at0 + (int64_t)batch * NI * RPI * ep.ld) * kSize;
#pragma unroll
            for (int u = 0; u < NI; ++u, p += RPI * ep.ld * kSize) {
                if (inside) {
                    v[u] = *reinterpret_cast<const u32x4_out*>(p);
                } else {
                    v[u] = u32x4{0, 0, 0, 0};
                    if ((batch * NI + u) * RPI >= rows) continue;
                    if (left == V) {
                        v[u] = *reinterpret_cast<const u32x4_out*>(p);
                        continue;
                    }
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        if (e >= left) continue;
                        if constexpr (kSize == 4) v[u][e] = reinterpret_cast<const uint32_t*>(p)[e];
                        else v[u][e / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[e] << (16 * (e & 1));
                    }
                }
            }
        }
    };
    load_residuals(0, res[0]);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(kWaitLds);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    uint8_t* const part = smem + wave * 32 * PITCH;
    // kInside, kGelu: known (0, 1) or looked up (2).  Known, the way out is straight code
    // that reads the next sums while others leave (65,459 x 4,096 x 1,024 with GELU 287 ->
    // 279 us, to fp32 320 -> 303; without it 65,459 x 4,096 x 512 157 -> 147, x 1,024 231 ->
    // 235).  With residuals that was slower (196 -> 216 us, x 1,024 x 4,096):
    // more of them in flight hold up the copies of the other workgroup.
    // In tiles over an edge the lanes whose columns are all there still move 16 bytes
    // (by elements 1,000 x 16,384 x 4,096 took 58.7 us, now 50.2).
    auto store = [&](const u32x4& o, uint8_t* to) {
        if constexpr (kLines) __builtin_nontemporal_store(o, reinterpret_cast<u32x4_out*>(to));
        else *reinterpret_cast<u32x4_out*>(to) = o;
    };
    auto leave = [&](auto inside_c, auto gelu_c) {
        constexpr int kInside = decltype(inside_c)::value, kGelu = decltype(gelu_c)::value;
        uint8_t* po = static_cast<uint8_t*>(ep.out) + at0 * kSize;
#pragma unroll
        for (int batch = 0; batch < NB; ++batch) {
            constexpr int kPerRowSet = NB / TM;  // batches per 32 rows
            if (batch % kPerRowSet == 0) {
                const int m = batch / kPerRowSet;
#pragma unroll
                for (int i = 0; i < TN; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *reinterpret_cast<f32x4*>(part + fr * PITCH + (i * 32 + q * 8 + half * 4) * 4) =
                            f32x4{acc[i][m][q * 4], acc[i][m][q * 4 + 1], acc[i][m][q * 4 + 2],
                                  acc[i][m][q * 4 + 3]};
            }
            if (batch + 1 < NB) load_residuals(batch + 1, res[(batch + 1) & 1]);
#pragma unroll
            for (int u = 0; u < NI; ++u, po += RPI * ep.ld * kSize) {
                const int r = (batch % kPerRowSet * NI + u) * RPI + er;
                float v[V];
#pragma unroll
                for (int e = 0; e < V; e += 4) {
                    const f32x4 s = *reinterpret_cast<const f32x4*>(part + r * PITCH + (ec + e) * 4);
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[e + k] = s[k];
                }
                if (kGelu == 2 ? ep.gelu : kGelu == 1)
#pragma unroll
                    for (int e = 0; e < V; ++e) v[e] = gemm::gelu_erf(v[e]);
                if constexpr (kResid) {
                    float f[V];
                    widen<kOut>(res[batch & 1][u], f);
#pragma unroll
                    for (int e = 0; e < V; ++e) v[e] += f[e];
                }
                const u32x4 o = narrow<kOut>(v);
                if (kInside == 2 ? inside : kInside == 1) {
                    store(o, po);
                } else if ((batch * NI + u) * RPI < rows) {
                    if (left == V) {
                        store(o, po);
                        continue;
                    }
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        if (e >= left) continue;
                        if constexpr (kSize == 4) reinterpret_cast<uint32_t*>(po)[e] = o[e];
                        else reinterpret_cast<uint16_t*>(po)[e] = (uint16_t)(o[e / 2] >> (16 * (e & 1)));
                    }
                }
            }
        }
    };
    if constexpr (kResid) {
        leave(integral_constant<int, 2>{}, integral_constant<int, 2>{});
    } else {
        if (!inside) leave(integral_constant<int, 0>{}, integral_constant<int, 2>{});
        else if (ep.gelu) leave(integral_constant<int, 1>{}, integral_constant<int, 1>{});
        else leave(integral_constant<int, 1>{}, integral_constant<int, 0>{});
    }
}

template <int TM, int TN, int kOut, bool kResid, bool kLines>
inline hipError_t launch_tiles(const Slabs& x, const Slabs& w, int64_t K, const Epilogue& ep,
                               hipStream_t st) {
    const int64_t tiles_m = (ep.M + 64 * TM - 1) / (64 * TM);
    const int64_t tiles_n = (ep.N + 64 * TN - 1) / (64 * TN);
    // the kernel counts tiles in 32 bits (2^28 of them hold a terabyte of results)
    if (tiles_m * tiles_n > ((int64_t)1 << 28)) return hipErrorInvalidConfiguration;
    return launch_blocks(tiles_m * tiles_n, 256, [&](int64_t b0, dim3 grid) {
        hipLaunchKernelGGL((k_linear_tiles<TM, TN, kOut, kResid, kLines>), grid, dim3(256), 0, st, x,
                           w, (int)groups(K), ep, (uint32_t)tiles_m,
                           (uint32_t)tiles_n, b0);
    });
}

template <int TM, int TN, int kOut, bool kResid>
inline hipError_t launch_tiles(const Slabs& x, const Slabs& w, int64_t K, const Epilogue& ep,
                               hipStream_t st) {
    const uintptr_t row = (uintptr_t)ep.ld * (16 / kPer16<kOut>);
    return ((uintptr_t)ep.out | row) % 64 == 0
               ? launch_tiles<TM, TN, kOut, kResid, true>(x, w, K, ep, st)
               : launch_tiles<TM, TN, kOut, kResid, false>(x, w, K, ep, st);
}

template <int TM, int TN, int kOut>
inline hipError_t launch_tiles(const Slabs& x, const Slabs& w, int64_t K, const Epilogue& ep,
                               hipStream_t st) {
    return ep.residual ? launch_tiles<TM, TN, kOut, true>(x, w, K, ep, st)
                       : launch_tiles<TM, TN, kOut, false>(x, w, K, ep, st);
}

template <int TM, int TN>
inline hipError_t launch_tiles(const Slabs& x, const Slabs& w, int64_t K, const Epilogue& ep,
                               hipStream_t st) {
    switch (ep.out_type) {
        case SCONE_BF16: return launch_tiles<TM, TN, SCONE_BF16>(x, w, K, ep, st);
        case SCONE_FP16: return launch_tiles<TM, TN, SCONE_FP16>(x, w, K, ep, st);
        default: return launch_tiles<TM, TN, SCONE_FP32>(x, w, K, ep, st);
    }
}

// Whether a product takes the tiles.  Up to 64 rows k_linear_few has one launch and no
// layout of w, but every workgroup brings all rows of x to 4 bits again, or reads their
// codes.  Rows count by what that costs (4-bit 1, 16-bit 2, fp32 4), and the more there
// are, the fewer groups and workgroups it pays for.  Us, k_linear_few / tiles:
//   N x K            4-bit x, M = 32, 64     bf16, M = 16, 32, 64           fp32, M = 16, 32
//   4,096 x 1,024    3.9/8.7  5.0/8.4        4.0/8.7  5.0/8.9   7.2/9.0     5.2/9.2  7.2/9.3
//   4,001 x 1,500    4.1/10.6 5.6/10.5       5.2/10.2 7.2/10.8 10.3/11.3             10.1/10.8
//   1,024 x 4,096    8.0/13.3 12.0/13.2      7.4/13.7 10.8/13.9 18.0/13.8  11.8/14.0 19.8/14.3
//   16,384 x 1,024   6.7/12.8 11.1/12.6               9.4/12.8  16.8/12.7  12.3/12.6 19.2/13.1
//   8,192 x 4,096    14.0/21.0 22.4/21.4              17.7/21.4 30.0/21.2  21.4/21.1
//   16,384 x 4,096   25.3/27.2 48.6/26.6    21.0/27.5 30.2/26.8 53.6/26.7  39.4/27.8
inline bool tiled(int64_t M, int64_t N, int64_t K, int32_t type) {
    if (M > 64) return true;
    const int64_t rows = M * (type == SCONE_MX4 ? 1 : type == SCONE_FP32 ? 4 : 2);
    const int64_t g = groups(K), workgroups = (N + 15) / 16;
    return rows <= 32   ? false
           : rows <= 64 ? g * workgroups > 16384
                        : rows > 128 || g > 16 || workgroups > 512;
}

// Scratch of a linear map: the slabs of x and w.
inline int64_t linear_workspace(int64_t M, int64_t N, int64_t K, int32_t type) {
    return tiled(M, N, K, type) && N > 0 ? slabs_bytes(M, K) + slabs_bytes(N, K) : 0;
}

template <int kType>
inline hipError_t launch_slabs(const void* x, int64_t ld, const Slabs& sx, const uint8_t* w,
                               const Slabs& sw, int64_t K, const Epilogue& ep, hipStream_t st) {
    const int64_t bx = slab_blocks(ep.M, K);
    return launch_blocks(bx + slab_blocks(ep.N, K), 256, [&](int64_t b0, dim3 grid) {
        hipLaunchKernelGGL(k_slabs<kType>, grid, dim3(256), 0, st, x, ld, ep.M, sx, w, ep.N, sw,
                           ep.bias, ep.bias_type, K, bx, b0);
    });
}

// x: 4-bit rows, or (type not SCONE_MX4) rows to quantise.
inline hipError_t linear(const void* x, int32_t type, int64_t ld, const uint8_t* w, int64_t K,
                         const Epilogue& ep, uint8_t* ws, hipStream_t st) {
    if (!tiled(ep.M, ep.N, K, type)) {
        switch (type) {
            case SCONE_BF16: return launch_few<SCONE_BF16>(x, ld, w, K, ep, st);
            case SCONE_FP16: return launch_few<SCONE_FP16>(x, ld, w, K, ep, st);
            case SCONE_FP32: return launch_few<SCONE_FP32>(x, ld, w, K, ep, st);
            default: return launch_few<SCONE_MX4>(x, ld, w, K, ep, st);
        }
    }
    const Slabs sx = slabs_at(ws, ep.M, K), sw = slabs_at(ws + slabs_bytes(ep.M, K), ep.N, K);
    hipError_t e;
    switch (type) {
        case SCONE_BF16: e = launch_slabs<SCONE_BF16>(x, ld, sx, w, sw, K, ep, st); break;
        case SCONE_FP16: e = launch_slabs<SCONE_FP16>(x, ld, sx, w, sw, K, ep, st); break;
        case SCONE_FP32: e = launch_slabs<SCONE_FP32>(x, ld, sx, w, sw, K, ep, st); break;
        default: e = launch_slabs<SCONE_MX4>(x, ld, sx, w, sw, K, ep, st);
    }
    if (e != hipSuccess) return e;
    // The small tiles, four for a large one, as long as they run in one round (three a
    // compute unit, 768); over a long loop the large ones from two small ones a compute
    // unit on.  Us, large / small, at 128, 160, 192, 224, 256 and 512 large tiles:
    //   4,096 x 1,024         14.7/13.7 15.6/15.6 16.1/16.2 16.7/17.9 17.4/18.4 25.4/27.5
    //   the same, GELU        18.6/15.0 19.4/17.2 19.8/17.8 20.3/20.2 21.0/20.5 29.8/31.0
    //   4,096 x 2,048         20.3/20.2 21.7/23.1 22.3/23.6 23.6/26.8 24.9/27.4
    //   the same, GELU        24.3/20.9 25.5/24.8 26.2/25.2 27.5/28.6 28.7/29.5
    //   2,048 x 2,048, fp32 residual 24.6/20.8 24.1/23.1 25.6/24.0 27.9/29.1 28.9/28.6
    //   4,096 x 4,096, GELU   32.9/28.7 32.2/33.8 33.4/34.9 35.3/39.8 37.1/41.1
    //   1,024 x 4,096, fp32 residual 32.5/28.5 34.8/35.4 37.6/37.9 40.8/43.9 44.3/47.2 77.0/86.3
    //   16,384 x 4,096        34.4/33.5           36.7/40.0           39.8/46.0 58.2/71.4
    const int64_t big = ((ep.M + 127) / 128) * ((ep.N + 255) / 256);
    return big > (groups(K) < 32 ? 192 : 128) ? launch_tiles<2, 4>(sx, sw, K, ep, st)
                                              : launch_tiles<1, 2>(sx, sw, K, ep, st);
}

}  // namespace mx4
}  // namespace scone
