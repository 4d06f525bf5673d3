// One decoding step for many sequences: shift the new token into each
// sequence's rolling context, find the longest f-gram ending at it, and copy
// its row (Algorithm 1 applied to the newest position only; decoding emits one
// token per step, Section 4.3 and the resource summary in the appendix).
//
// One wavefront owns one sequence.  Lanes 0..G-1 probe the suffix lengths
// max_n .. 2 of (context + new token) in parallel and a ballot picks the
// longest hit; the wave then rewrites the context (the last ctx_cap tokens)
// and copies the chosen row with 16-byte vectors.  Because the context keeps
// the last max_n - 1 tokens, the step's result equals the prefill lookup at
// the same position of the whole sequence.
#include "mx4.h"
#include "row_copy.h"
#include "tile_lookup.h"

namespace scone {
namespace {

constexpr int kDecodeThreads = 64;  // one wavefront, one sequence

// The step of one wavefront's sequence up to the row: rewrites its context, writes
// the id and the match length, and returns the row's id.
template <int SB, int G>
__device__ __forceinline__ int32_t decode_find(
    const typename SlotOps<SB>::Slot* __restrict__ slots, uint64_t mask, int32_t* __restrict__ ctx,
    int32_t* __restrict__ ctx_len, int ctx_cap, const int32_t* __restrict__ new_tok, int max_n,
    int64_t s, int lane, int32_t* __restrict__ ids_out, int8_t* __restrict__ len_out,
    unsigned* __restrict__ err) {
    int32_t* my_ctx = ctx + s * ctx_cap;
    // The length, the new token and the whole context are loaded at once (the
    // context without waiting for its length); probe windows then come from
    // the lanes holding the context, so a step has three dependent memory
    // round trips: inputs, one hash bucket, the row.
    int L = ctx_len[s];
    const int32_t nt = new_tok[s];
    const int32_t cv_raw = lane < ctx_cap ? my_ctx[lane] : 0;
    L = L < 0 ? 0 : (L > ctx_cap ? ctx_cap : L);
    // seq[0..L] = context (oldest first) followed by the new token
    const int32_t cv = lane < L ? cv_raw : 0;

    bool hit = false;
    int32_t id = 0;
    const int n = max_n - lane;
    int32_t win[SCONE_MAX_FGRAM_LEN];
#pragma unroll
    for (int i = 0; i < SCONE_MAX_FGRAM_LEN; ++i) {
        const int k = L + 1 - n + i;  // position of window token i in seq
        const int32_t c = __shfl(cv, k & 63);
        win[i] = k < L ? c : nt;
    }
    if (lane < G && n >= 2 && n <= L + 1) {
        bool ok = true;
#pragma unroll
        for (int i = 0; i < SCONE_MAX_FGRAM_LEN; ++i)
            if (i < n) ok &= (win[i] >= 0) & (win[i] < SCONE_TOKEN_LIMIT);
        if (ok) hit = probe<SB>(slots, mask, pack_key(win, n), id);
    }
    const unsigned long long m = __ballot(hit);
    const unsigned gm = (unsigned)m & ((1u << G) - 1u);
    const int jb = gm ? __ffs(gm) - 1 : 0;
    const int32_t best = __shfl(id, jb);
    const int32_t rid = gm ? best : nt;

    // New context: the last min(ctx_cap, L + 1) tokens of seq.
    const int Lp = L + 1 < ctx_cap ? L + 1 : ctx_cap;
    const int d = L + 1 - Lp;
    const int32_t moved = __shfl(cv, (lane + d) & 63);
    if (lane < Lp) my_ctx[lane] = (lane + d < L) ? moved : nt;
    if (lane == 0) {
        ctx_len[s] = Lp;
        if (nt < 0 || nt >= SCONE_TOKEN_LIMIT) atomicOr(err, err_bit(SCONE_ETOKEN));
        if (ids_out) ids_out[s] = rid;
        if (len_out) len_out[s] = (int8_t)(gm ? max_n - jb : 1);
    }
    return rid;
}

template <int SB, int G, typename V, int U, bool kPow2>
__global__ __launch_bounds__(kDecodeThreads) void k_decode(
    const typename SlotOps<SB>::Slot* __restrict__ slots, uint64_t mask, int32_t* __restrict__ ctx,
    int32_t* __restrict__ ctx_len, int ctx_cap, const int32_t* __restrict__ new_tok, int max_n,
    const V* __restrict__ rows, int64_t n_rows, int64_t upr, int shift, V* __restrict__ out,
    int32_t* __restrict__ ids_out, int8_t* __restrict__ len_out, unsigned* __restrict__ err,
    int64_t block0) {
    const int64_t s = block_index(block0);
    const int lane = threadIdx.x;
    const int32_t rid = decode_find<SB, G>(slots, mask, ctx, ctx_len, ctx_cap, new_tok, max_n, s,
                                           lane, ids_out, len_out, err);

    // Copy the row: aligned rows of a power of two of 16-byte units by shifts, any
    // other width in 16-byte units at any alignment (row_copy.h) or, below 16
    // bytes, in bytes.  The first path is 0.25 to 0.55 us of 3.1 to 4.5 faster than
    // the second on its rows; the others took single bytes: 256 rows of 3,072
    // bytes 8.1 us a step, now 3.3, 1,024 rows of 6,000 bytes 15.3, now 4.7.
    const bool ok = (rid >= 0) & ((int64_t)rid < n_rows);
    if (!ok && lane == 0) atomicOr(err, err_bit(SCONE_EROW));
    if constexpr (!kPow2) {  // upr holds the row's bytes
        const int64_t row_bytes = upr, last = row_bytes - (int64_t)sizeof(V);
        uint8_t* __restrict__ to = reinterpret_cast<uint8_t*>(out) + s * row_bytes;
        const uint8_t* __restrict__ from =
            reinterpret_cast<const uint8_t*>(rows) + (ok ? rid : 0) * row_bytes;
        for (int64_t o0 = lane * (int64_t)sizeof(V); o0 < row_bytes;
             o0 += (int64_t)kDecodeThreads * U * sizeof(V)) {
            V v[U];
            if (ok) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int64_t o = o0 + (int64_t)u * kDecodeThreads * sizeof(V);
                    if (o < row_bytes)
                        v[u] = *reinterpret_cast<const V*>(from + (o < last ? o : last));
                }
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u) v[u] = V{};
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t o = o0 + (int64_t)u * kDecodeThreads * sizeof(V);
                if (o < row_bytes)
                    __builtin_nontemporal_store(v[u],
                                                reinterpret_cast<V*>(to + (o < last ? o : last)));
            }
        }
        return;
    }
    V* __restrict__ dst = out + s * upr;
    const V* __restrict__ src = rows + ((int64_t)rid << shift);
    for (int64_t c0 = lane; c0 < upr; c0 += (int64_t)kDecodeThreads * U) {
        V v[U];
        if (ok) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t c = c0 + (int64_t)u * kDecodeThreads;
                if (c < upr) v[u] = src[c];
            }
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = V{};
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t c = c0 + (int64_t)u * kDecodeThreads;
            if (c < upr) __builtin_nontemporal_store(v[u], dst + c);
        }
    }
}

template <int SB, int G, typename V, bool kPow2>
hipError_t launch(const scone_table* tb, int32_t* ctx, int32_t* ctx_len, int ctx_cap,
                  const int32_t* new_tok, int64_t S, int max_n, const void* rows,
                  int64_t n_rows, int64_t upr, int shift, void* out, int32_t* ids, int8_t* lens,
                  unsigned* err, hipStream_t st) {
    using Slot = typename SlotOps<SB>::Slot;
    return launch_blocks(S, kDecodeThreads, [&](int64_t b0, dim3 grid) {
        hipLaunchKernelGGL((k_decode<SB, G, V, 4, kPow2>), grid, dim3(kDecodeThreads), 0, st,
                           static_cast<const Slot*>(tb->slots), (uint64_t)tb->capacity - 1, ctx,
                           ctx_len, ctx_cap, new_tok, max_n, static_cast<const V*>(rows), n_rows,
                           upr, shift, static_cast<V*>(out), ids, lens, err, b0);
    });
}

template <int SB, typename V, bool kPow2>
hipError_t dispatch(const scone_table* tb, int32_t* ctx, int32_t* ctx_len, int ctx_cap,
                    const int32_t* new_tok, int64_t S, int max_n, const void* rows,
                    int64_t n_rows, int64_t upr, int shift, void* out, int32_t* ids,
                    int8_t* lens, unsigned* err, hipStream_t st) {
    switch (lanes_for(max_n)) {
        case 1:
            return launch<SB, 1, V, kPow2>(tb, ctx, ctx_len, ctx_cap, new_tok, S, max_n, rows,
                                           n_rows, upr, shift, out, ids, lens, err, st);
        case 2:
            return launch<SB, 2, V, kPow2>(tb, ctx, ctx_len, ctx_cap, new_tok, S, max_n, rows,
                                           n_rows, upr, shift, out, ids, lens, err, st);
        case 4:
            return launch<SB, 4, V, kPow2>(tb, ctx, ctx_len, ctx_cap, new_tok, S, max_n, rows,
                                           n_rows, upr, shift, out, ids, lens, err, st);
        default:
            return launch<SB, 8, V, kPow2>(tb, ctx, ctx_len, ctx_cap, new_tok, S, max_n, rows,
                                           n_rows, upr, shift, out, ids, lens, err, st);
    }
}

template <typename V, bool kPow2>
hipError_t dispatch_slots(const scone_table* tb, int32_t* ctx, int32_t* ctx_len, int ctx_cap,
                          const int32_t* new_tok, int64_t S, int max_n, const void* rows,
                          int64_t n_rows, int64_t upr, int shift, void* out, int32_t* ids,
                          int8_t* lens, unsigned* err, hipStream_t st) {
    return tb->slot_bytes == 16
               ? dispatch<16, V, kPow2>(tb, ctx, ctx_len, ctx_cap, new_tok, S, max_n, rows,
                                        n_rows, upr, shift, out, ids, lens, err, st)
               : dispatch<32, V, kPow2>(tb, ctx, ctx_len, ctx_cap, new_tok, S, max_n, rows,
                                        n_rows, upr, shift, out, ids, lens, err, st);
}

// The same step with the values of a 4-bit row (mx4.h) for the row: a lane takes
// 16 bytes of them at a time, the codes and scale bytes of kMx4Pieces in flight.
constexpr int kMx4Pieces = 4;

template <int SB, int G, int kType>
__global__ __launch_bounds__(kDecodeThreads) void k_decode_mx4(
    const typename SlotOps<SB>::Slot* __restrict__ slots, uint64_t mask, int32_t* __restrict__ ctx,
    int32_t* __restrict__ ctx_len, int ctx_cap, const int32_t* __restrict__ new_tok, int max_n,
    const uint8_t* __restrict__ rows, int64_t n_rows, int cols,
    typename mx4::Elem<kType>::type* __restrict__ out, int32_t* __restrict__ ids_out,
    int8_t* __restrict__ len_out, unsigned* __restrict__ err, int64_t block0) {
    typedef mx4::Out<kType> O;
    const int64_t s = block_index(block0);
    const int lane = threadIdx.x;
    const int32_t rid = decode_find<SB, G>(slots, mask, ctx, ctx_len, ctx_cap, new_tok, max_n, s,
                                           lane, ids_out, len_out, err);
    const bool ok = (rid >= 0) & ((int64_t)rid < n_rows);
    if (!ok && lane == 0) atomicOr(err, err_bit(SCONE_EROW));
    const int pieces = (cols + O::kElems - 1) / O::kElems;
    const uint8_t* row = rows + (ok ? rid : 0) * mx4::row_bytes(cols);
    const uint8_t* scales = row + 64 * mx4::groups(cols);
    auto* dst = out + s * cols;
    for (int c0 = lane; c0 < pieces; c0 += kDecodeThreads * kMx4Pieces) {
        uint32_t codes[kMx4Pieces] = {}, sc[kMx4Pieces] = {};
        if (ok) {
#pragma unroll
            for (int u = 0; u < kMx4Pieces; ++u) {
                const int c = c0 + u * kDecodeThreads;
                if (c < pieces) {
                    codes[u] = O::load(row, c);
                    sc[u] = scales[c / (32 / O::kElems)];
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kMx4Pieces; ++u) {
            const int c = c0 + u * kDecodeThreads;
            if (c < pieces)
                O::store(dst + c * O::kElems, cols - c * O::kElems, O::values(codes[u], sc[u]));
        }
    }
}

struct Mx4Call {
    const scone_table* tb;
    int32_t *ctx, *ctx_len;
    int ctx_cap;
    const int32_t* new_tok;
    int64_t S;
    int max_n;
    const void* rows;
    int64_t n_rows;
    int cols;
    void* out;
    int32_t* ids;
    int8_t* lens;
    unsigned* err;
    hipStream_t st;
};

template <int SB, int G, int kType>
hipError_t launch_mx4(const Mx4Call& c) {
    using Slot = typename SlotOps<SB>::Slot;
    return launch_blocks(c.S, kDecodeThreads, [&](int64_t b0, dim3 grid) {
        hipLaunchKernelGGL((k_decode_mx4<SB, G, kType>), grid, dim3(kDecodeThreads), 0, c.st,
                           static_cast<const Slot*>(c.tb->slots), (uint64_t)c.tb->capacity - 1,
                           c.ctx, c.ctx_len, c.ctx_cap, c.new_tok, c.max_n,
                           static_cast<const uint8_t*>(c.rows), c.n_rows, c.cols,
                           static_cast<typename mx4::Elem<kType>::type*>(c.out), c.ids, c.lens,
                           c.err, b0);
    });
}

template <int SB, int kType>
hipError_t dispatch_mx4(const Mx4Call& c) {
    switch (lanes_for(c.max_n)) {
        case 1: return launch_mx4<SB, 1, kType>(c);
        case 2: return launch_mx4<SB, 2, kType>(c);
        case 4: return launch_mx4<SB, 4, kType>(c);
        default: return launch_mx4<SB, 8, kType>(c);
    }
}

template <int kType>
hipError_t dispatch_mx4_slots(const Mx4Call& c) {
    return c.tb->slot_bytes == 16 ? dispatch_mx4<16, kType>(c) : dispatch_mx4<32, kType>(c);
}

// The argument checks of a decoding step whose table rows take row_bytes and output
// rows out_bytes; `eff` receives the effective window.  SCONE_OK with S = 0 means that
// there is nothing to do.
int check_step(const scone_table_t* table, const int32_t* ctx, const int32_t* ctx_len,
               int32_t ctx_cap, const int32_t* new_tok, int64_t S, int32_t max_n,
               const void* rows, int64_t n_rows, int64_t row_bytes, int32_t placement,
               const void* out, int64_t out_bytes, const int32_t* fgram_ids,
               const int8_t* match_len, int& eff) {
    if (!table || S < 0 || max_n < 1 || n_rows < 0 || row_bytes <= 0) return SCONE_EINVAL;
    if (placement != SCONE_PLACE_HBM && placement != SCONE_PLACE_HOST) return SCONE_EINVAL;
    eff = max_n < table->max_len ? max_n : table->max_len;
    if (ctx_cap < eff - 1 || ctx_cap > 63 || ctx_cap < 0) return SCONE_EINVAL;
    if (S > ((int64_t)1 << 62) / out_bytes) return SCONE_EINVAL;
    if (S == 0) return SCONE_OK;
    if (!ctx_len || !new_tok || !out || (!ctx && ctx_cap > 0) || (!rows && n_rows > 0))
        return SCONE_EINVAL;
    // Each wavefront rewrites its own sequence's context in place; the other
    // outputs must not alias any input or each other.
    const void* outs[3] = {out, fgram_ids, match_len};
    const int64_t outs_b[3] = {S * out_bytes, span_bytes(S, 4), S};
    const void* ins[4] = {ctx, ctx_len, new_tok, rows};
    const int64_t ins_b[4] = {span_bytes(S, 4 * (int64_t)ctx_cap), span_bytes(S, 4),
                              span_bytes(S, 4), span_bytes(n_rows, row_bytes)};
    for (int i = 0; i < 3; ++i) {
        for (int j = 0; j < 4; ++j)
            if (overlaps(outs[i], outs_b[i], ins[j], ins_b[j])) return SCONE_EINVAL;
        for (int j = i + 1; j < 3; ++j)
            if (overlaps(outs[i], outs_b[i], outs[j], outs_b[j])) return SCONE_EINVAL;
    }
    if (overlaps(ctx, ins_b[0], ctx_len, ins_b[1]) || overlaps(ctx, ins_b[0], new_tok, ins_b[2]) ||
        overlaps(ctx_len, ins_b[1], new_tok, ins_b[2]))
        return SCONE_EINVAL;
    return SCONE_OK;
}

}  // namespace
}  // namespace scone

extern "C" int scone_decode_step(const scone_table_t* table, int32_t* ctx, int32_t* ctx_len,
                                 int32_t ctx_cap, const int32_t* new_tok, int64_t S,
                                 int32_t max_n, const void* rows, int64_t n_rows,
                                 int64_t row_bytes, int32_t placement, void* out,
                                 int32_t* fgram_ids, int8_t* match_len, void* stream) {
    using namespace scone;
    int eff = 0;
    const int rc = check_step(table, ctx, ctx_len, ctx_cap, new_tok, S, max_n, rows, n_rows,
                              row_bytes, placement, out, row_bytes, fgram_ids, match_len, eff);
    if (rc != SCONE_OK || S == 0) return rc;
    int dev = 0;
    SCONE_HIP_TRY(hipGetDevice(&dev));
    if (dev != table->device) return SCONE_EINVAL;
    unsigned* err = device_error_word();
    if (!err) return SCONE_EHIP;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const uintptr_t align = (uintptr_t)rows | (uintptr_t)out | (uintptr_t)row_bytes;
    hipError_t e;
    if ((align & 15) == 0 && ((row_bytes / 16) & (row_bytes / 16 - 1)) == 0) {
        const int64_t upr = row_bytes / 16;
        int shift = 0;
        while (((int64_t)1 << shift) < upr) ++shift;
        e = dispatch_slots<u32x4, true>(table, ctx, ctx_len, ctx_cap, new_tok, S, eff, rows,
                                        n_rows, upr, shift, out, fgram_ids, match_len, err, st);
    } else if (row_bytes >= 16) {
        e = dispatch_slots<u32x4_any, false>(table, ctx, ctx_len, ctx_cap, new_tok, S, eff, rows,
                                             n_rows, row_bytes, 0, out, fgram_ids, match_len, err,
                                             st);
    } else {
        e = dispatch_slots<uint8_t, false>(table, ctx, ctx_len, ctx_cap, new_tok, S, eff, rows,
                                           n_rows, row_bytes, 0, out, fgram_ids, match_len, err,
                                           st);
    }
    return status_of(e);
}

extern "C" int scone_decode_step_mx4(const scone_table_t* table, int32_t* ctx, int32_t* ctx_len,
                                     int32_t ctx_cap, const int32_t* new_tok, int64_t S,
                                     int32_t max_n, const void* rows, int64_t n_rows,
                                     int64_t cols, int32_t placement, void* out,
                                     int32_t out_type, int32_t* fgram_ids, int8_t* match_len,
                                     void* stream) {
    using namespace scone;
    const int64_t eb = mx4::elem_bytes(out_type);
    if (eb == 0 || !mx4::cols_ok(cols)) return SCONE_EINVAL;
    int eff = 0;
    const int rc = check_step(table, ctx, ctx_len, ctx_cap, new_tok, S, max_n, rows, n_rows,
                              mx4::row_bytes(cols), placement, out, cols * eb, fgram_ids,
                              match_len, eff);
    if (rc != SCONE_OK || S == 0) return rc;
    if ((uintptr_t)out % eb != 0 || (uintptr_t)rows % 16 != 0) return SCONE_EINVAL;
    int dev = 0;
    SCONE_HIP_TRY(hipGetDevice(&dev));
    if (dev != table->device) return SCONE_EINVAL;
    unsigned* err = device_error_word();
    if (!err) return SCONE_EHIP;
    const Mx4Call c{table, ctx, ctx_len, ctx_cap, new_tok, S, eff, rows, n_rows, (int)cols, out,
                    fgram_ids, match_len, err, static_cast<hipStream_t>(stream)};
    switch (out_type) {
        case SCONE_BF16: return status_of(dispatch_mx4_slots<SCONE_BF16>(c));
        case SCONE_FP16: return status_of(dispatch_mx4_slots<SCONE_FP16>(c));
        default: return status_of(dispatch_mx4_slots<SCONE_FP32>(c));
    }
}
