// Rows to 4 bits and back: quantisation, and the gather of 4-bit rows by id (mx4.h has
// the format).
//
// Both are streams bound by memory: a lane takes eight elements (16 bytes of bf16 or
// fp16, 32 of fp32, one word of codes), consecutive lanes consecutive pieces of a row, and
// rows follow one another in a flat array of pieces, so that any width fills the lanes.
#include "mx4.h"
#include "row_copy.h"

namespace scone {
namespace {

constexpr int kThreads = 256;

// Quantisation: each block of 32 is four lanes, whose largest magnitudes are joined
// by two exchanges; sixteen lanes hold a group of 128, whose four scale bytes are
// joined to a word the same way.  A row's 16 g pieces are a multiple of 16, so blocks
// and groups lie inside one row and one aligned run of lanes.
template <int kType, int U>
__global__ __launch_bounds__(kThreads) void k_quantize(
    const typename mx4::Elem<kType>::type* __restrict__ x, int64_t n_rows, int64_t cols,
    int64_t ld, RowUnits pieces, uint8_t* __restrict__ rows, int64_t row_bytes, int64_t block0) {
    typedef mx4::Elem<kType> E;
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
        v[u] = mx4::load8<kType>(x + (r[u] < n_rows ? r[u] * ld + e : 0),
                                 r[u] < n_rows ? cols - e : 0);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        uint32_t top = E::top(v[u]);
        uint32_t o = __shfl_xor(top, 1);
        top = top > o ? top : o;
        o = __shfl_xor(top, 2);
        top = top > o ? top : o;
        const uint32_t s = mx4::scale_byte(E::field(top));
        const uint32_t codes = s == 255 ? 0u : E::quantize(v[u], mx4::scale_of(s));
        uint32_t word = s << (8 * ((threadIdx.x >> 2) & 3));
        word |= __shfl_xor(word, 4);
        word |= __shfl_xor(word, 8);
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
    const RowUnits pieces = row_units(16 * mx4::groups(cols), 1);
    const int64_t total = n_rows * pieces.upr;
    return launch_blocks((total + kThreads * U - 1) / (kThreads * U), kThreads,
                         [&](int64_t b0, dim3 grid) {
                             hipLaunchKernelGGL(
                                 (k_quantize<kType, U>), grid, dim3(kThreads), 0, st,
                                 static_cast<const typename mx4::Elem<kType>::type*>(x), n_rows,
                                 cols, ld, pieces, static_cast<uint8_t*>(rows),
                                 mx4::row_bytes(cols), b0);
                         });
}

// Gather: out[k] = the values of row ids[k], or of row k where there are no ids.  An
// id outside the table writes zeros.
template <int kType, int U>
__global__ __launch_bounds__(kThreads) void k_gather_mx4(
    const int32_t* __restrict__ ids, int64_t n_tok, const uint8_t* __restrict__ rows,
    int64_t n_rows, int64_t cols, RowUnits pieces, int64_t row_bytes, int64_t scale_at,
    typename mx4::Elem<kType>::type* __restrict__ out, unsigned* __restrict__ err,
    int64_t block0) {
    typedef mx4::Elem<kType> E;
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
        codes[u] = reinterpret_cast<const uint32_t*>(row)[c[u]];
        s[u] = row[scale_at + (c[u] >> 2)];
    }
    bool bad = false;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        bad |= in[u] & !ok[u];
        if (!in[u]) continue;
        typename E::vec v = E::values(codes[u], mx4::scale_of(s[u]));
        if (!ok[u]) v = typename E::vec{};
        const int64_t e = (int64_t)c[u] * 8;
        mx4::store8<kType>(out + r[u] * cols + e, cols - e, v);
    }
    if (bad) atomicOr(err, err_bit(SCONE_EROW));
}

template <int kType, int U>
hipError_t launch_gather_mx4(const int32_t* ids, int64_t n_tok, const void* rows, int64_t n_rows,
                             int64_t cols, void* out, unsigned* err, hipStream_t st) {
    const RowUnits pieces = row_units((cols + 7) / 8, 1);
    const int64_t total = n_tok * pieces.upr;
    return launch_blocks((total + kThreads * U - 1) / (kThreads * U), kThreads,
                         [&](int64_t b0, dim3 grid) {
                             hipLaunchKernelGGL(
                                 (k_gather_mx4<kType, U>), grid, dim3(kThreads), 0, st, ids,
                                 n_tok, static_cast<const uint8_t*>(rows), n_rows, cols, pieces,
                                 mx4::row_bytes(cols), 64 * mx4::groups(cols),
                                 static_cast<typename mx4::Elem<kType>::type*>(out), err, b0);
                         });
}

}  // namespace

namespace mx4 {

hipError_t quantize(const void* x, int32_t type, int64_t n_rows, int64_t cols, int64_t ld,
                    void* rows, hipStream_t st) {
    switch (type) {
        case SCONE_BF16: return launch_quantize<SCONE_BF16, 4>(x, n_rows, cols, ld, rows, st);
        case SCONE_FP16: return launch_quantize<SCONE_FP16, 4>(x, n_rows, cols, ld, rows, st);
        default: return launch_quantize<SCONE_FP32, 2>(x, n_rows, cols, ld, rows, st);
    }
}

}  // namespace mx4
}  // namespace scone

extern "C" int64_t scone_mx4_row_bytes(int64_t cols) {
    return scone::mx4::cols_ok(cols) ? scone::mx4::row_bytes(cols) : -1;
}

extern "C" int scone_quantize_mx4(const void* x, int32_t x_type, int64_t n_rows, int64_t cols,
                                  int64_t ld, void* rows, void* stream) {
    using namespace scone;
    const int64_t eb = mx4::elem_bytes(x_type);
    if (eb == 0 || n_rows < 0 || !mx4::cols_ok(cols) || ld < cols) return SCONE_EINVAL;
    if (ld > ((int64_t)1 << 56) || (n_rows > 0 && ld > ((int64_t)1 << 60) / n_rows))
        return SCONE_EINVAL;
    if (n_rows == 0) return SCONE_OK;
    const int64_t rb = mx4::row_bytes(cols);
    if (!x || !rows || (uintptr_t)x % eb != 0 || (uintptr_t)rows % 16 != 0) return SCONE_EINVAL;
    // Rows are written while others are read.
    if (overlaps(rows, span_bytes(n_rows, rb), x, ((n_rows - 1) * ld + cols) * eb))
        return SCONE_EINVAL;
    return status_of(mx4::quantize(x, x_type, n_rows, cols, ld, rows,
                                   static_cast<hipStream_t>(stream)));
}

extern "C" int scone_gather_mx4(const int32_t* fgram_ids, int64_t n_tok, const void* rows,
                                int64_t n_rows, int64_t cols, void* out, int32_t out_type,
                                int32_t placement, void* stream) {
    using namespace scone;
    const int64_t eb = mx4::elem_bytes(out_type);
    if (eb == 0 || n_tok < 0 || n_rows < 0 || !mx4::cols_ok(cols)) return SCONE_EINVAL;
    if (placement != SCONE_PLACE_HBM && placement != SCONE_PLACE_HOST) return SCONE_EINVAL;
    if (n_tok > ((int64_t)1 << 58) / cols) return SCONE_EINVAL;
    if (!fgram_ids && n_tok > n_rows) return SCONE_EINVAL;
    if (n_tok == 0) return SCONE_OK;
    if (!out || (!rows && n_rows > 0)) return SCONE_EINVAL;
    if ((uintptr_t)out % eb != 0 || (uintptr_t)rows % 16 != 0) return SCONE_EINVAL;
    // Rows are written while other wavefronts still read their ids and rows.
    const int64_t out_b = n_tok * cols * eb;
    if (overlaps(out, out_b, fgram_ids, span_bytes(n_tok, 4)) ||
        overlaps(out, out_b, rows, span_bytes(n_rows, mx4::row_bytes(cols))))
        return SCONE_EINVAL;
    unsigned* err = device_error_word();
    if (!err) return SCONE_EHIP;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (n_rows == 0) return status_of(launch_zero_rows(out, out_b, err, st));
    switch (out_type) {
        case SCONE_BF16:
            return status_of(launch_gather_mx4<SCONE_BF16, 4>(fgram_ids, n_tok, rows, n_rows,
                                                              cols, out, err, st));
        case SCONE_FP16:
            return status_of(launch_gather_mx4<SCONE_FP16, 4>(fgram_ids, n_tok, rows, n_rows,
                                                              cols, out, err, st));
        default:
            return status_of(launch_gather_mx4<SCONE_FP32, 4>(fgram_ids, n_tok, rows, n_rows,
                                                              cols, out, err, st));
    }
}
