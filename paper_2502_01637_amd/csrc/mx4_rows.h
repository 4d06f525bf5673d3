// Rows to 4 bits and back: quantisation, and the gather of 4-bit rows by id (mx4.h has
// the format).
//
// Both are streams bound by memory: a lane takes a piece of a row, consecutive lanes
// consecutive pieces, and rows follow one another in a flat array of pieces, so that any
// width fills the lanes.  On the way in a piece is eight elements (a word of codes), on
// the way out 16 bytes.
#pragma once

#include "mx4.h"
#include "row_copy.h"

namespace scone {
namespace mx4 {

constexpr int kThreads = 256;

// Quantisation.  A row's 16 g pieces are a multiple of 16, so a group lies inside one
// row and one aligned run of 16 lanes, as quantize8 takes it.
template <int kType, int U>
__global__ __launch_bounds__(kThreads) void k_quantize(
    const typename Elem<kType>::type* __restrict__ x, int64_t n_rows, int64_t cols,
    int64_t ld, RowUnits pieces, uint8_t* __restrict__ rows, int64_t row_bytes, int64_t block0) {
    typedef Elem<kType> E;
    const int64_t base = block_index(block0) * (kThreads * U);
    const int64_t r0 = pieces.div64(base);
    const uint32_t c0 = (uint32_t)(base - r0 * pieces.upr);
    typename E::vec v[U];
    int64_t r[U];
    uint32_t c[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t k = c0 + u * kThreads + threadIdx.x;
        const uint32_t q = pieces.div(k);
        r[u] = r0 + q;
        c[u] = k - q * pieces.upr;
        const int64_t e = (int64_t)c[u] * 8;
        v[u] = load8<kType>(x + (r[u] < n_rows ? r[u] * ld + e : 0),
                                 r[u] < n_rows ? cols - e : 0);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        uint32_t word;
        const uint32_t codes = quantize8<kType>(v[u], word);
        if (r[u] >= n_rows) continue;
        uint8_t* row = rows + r[u] * row_bytes;
        reinterpret_cast<uint32_t*>(row)[c[u]] = codes;
        if ((threadIdx.x & 15) == 0) {
            // pieces.upr words of codes, a word of scales per 16, zeros
            uint32_t* tail = reinterpret_cast<uint32_t*>(row) + pieces.upr;
            tail[c[u] / 16] = word;
            if (c[u] + 16 == pieces.upr)
                for (uint32_t w = pieces.upr / 16; w < row_bytes / 4 - pieces.upr; ++w) tail[w] = 0;
        }
    }
}

template <int kType, int U>
hipError_t launch_quantize(const void* x, int64_t n_rows, int64_t cols, int64_t ld, void* rows,
                           hipStream_t st) {
    const RowUnits pieces = row_units(16 * groups(cols), 1);
    const int64_t total = n_rows * pieces.upr;
    return launch_blocks((total + kThreads * U - 1) / (kThreads * U), kThreads,
                         [&](int64_t b0, dim3 grid) {
                             hipLaunchKernelGGL(
                                 (k_quantize<kType, U>), grid, dim3(kThreads), 0, st,
                                 static_cast<const typename Elem<kType>::type*>(x), n_rows,
                                 cols, ld, pieces, static_cast<uint8_t*>(rows),
                                 row_bytes(cols), b0);
                         });
}

// Gather: out[k] = the values of row ids[k], or of row k where there are no ids.  An
// id outside the table writes zeros.
template <int kType, int U>
__global__ __launch_bounds__(kThreads) void k_gather_values(
    const int32_t* __restrict__ ids, int64_t n_tok, const uint8_t* __restrict__ rows,
    int64_t n_rows, int64_t cols, RowUnits pieces, int64_t row_bytes, int64_t scale_at,
    typename Elem<kType>::type* __restrict__ out, unsigned* __restrict__ err,
    int64_t block0) {
    typedef Out<kType> O;
    const int64_t base = block_index(block0) * (kThreads * U);
    const int64_t r0 = pieces.div64(base);
    const uint32_t c0 = (uint32_t)(base - r0 * pieces.upr);
    int64_t r[U], id[U];
    uint32_t c[U], codes[U], s[U];
    bool in[U], ok[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t k = c0 + u * kThreads + threadIdx.x;
        const uint32_t q = pieces.div(k);
        r[u] = r0 + q;
        c[u] = k - q * pieces.upr;
        in[u] = r[u] < n_tok;
        if (!in[u]) r[u] = n_tok - 1;
        id[u] = ids ? (int64_t)ids[r[u]] : r[u];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        ok[u] = (id[u] >= 0) & (id[u] < n_rows);
        const uint8_t* row = rows + (ok[u] ? id[u] : 0) * row_bytes;
        codes[u] = O::load(row, c[u]);
        s[u] = row[scale_at + c[u] / (32 / O::kElems)];
    }
    bool bad = false;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        bad |= in[u] & !ok[u];
        if (!in[u]) continue;
        const u32x4 v = ok[u] ? O::values(codes[u], s[u]) : u32x4{};
        const int64_t e = (int64_t)c[u] * O::kElems;
        O::store(out + r[u] * cols + e, cols - e, v);
    }
    if (bad) atomicOr(err, err_bit(SCONE_EROW));
}

template <int kType, int U>
hipError_t launch_gather(const int32_t* ids, int64_t n_tok, const void* rows, int64_t n_rows,
                             int64_t cols, void* out, unsigned* err, hipStream_t st) {
    constexpr int E = Out<kType>::kElems;
    const RowUnits pieces = row_units((cols + E - 1) / E, 1);
    const int64_t total = n_tok * pieces.upr;
    return launch_blocks((total + kThreads * U - 1) / (kThreads * U), kThreads,
                         [&](int64_t b0, dim3 grid) {
                             hipLaunchKernelGGL(
                                 (k_gather_values<kType, U>), grid, dim3(kThreads), 0, st, ids,
                                 n_tok, static_cast<const uint8_t*>(rows), n_rows, cols, pieces,
                                 row_bytes(cols), 64 * groups(cols),
                                 static_cast<typename Elem<kType>::type*>(out), err, b0);
                         });
}

// Four pieces a thread in flight, two where the rows come over PCIe (the lines of rows
// that repeat are then in the caches more often): 131,072 rows of 2,048 as bf16 from
// 10.9 GB 130 us with four, 142 with two, 135 with eight; from host memory 1,744 with
// two, 1,786 with four.
template <int kType>
inline hipError_t gather(const int32_t* ids, int64_t n_tok, const void* rows, int64_t n_rows,
                         int64_t cols, void* out, int32_t placement, unsigned* err,
                         hipStream_t st) {
    return placement == SCONE_PLACE_HOST
               ? launch_gather<kType, 2>(ids, n_tok, rows, n_rows, cols, out, err, st)
               : launch_gather<kType, 4>(ids, n_tok, rows, n_rows, cols, out, err, st);
}

inline hipError_t gather(const int32_t* ids, int64_t n_tok, const void* rows, int64_t n_rows,
                         int64_t cols, void* out, int32_t type, int32_t placement, unsigned* err,
                         hipStream_t st) {
    switch (type) {
        case SCONE_BF16:
            return gather<SCONE_BF16>(ids, n_tok, rows, n_rows, cols, out, placement, err, st);
        case SCONE_FP16:
            return gather<SCONE_FP16>(ids, n_tok, rows, n_rows, cols, out, placement, err, st);
        default:
            return gather<SCONE_FP32>(ids, n_tok, rows, n_rows, cols, out, placement, err, st);
    }
}

}  // namespace mx4
}  // namespace scone
