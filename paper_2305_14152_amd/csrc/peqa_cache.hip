// New tokens into the paged cache (peqa_rope_append, peqa_norm_rope_append), and the host's check of the cache's descriptor.
#include "peqa_cache.h"
#include "peqa_heads.h"
#include "peqa_host.h"

using namespace peqa::host;

namespace peqa {

namespace {

struct AppendArgs {
    CacheArgs cache;
    const int32_t *pos, *place, *seq;      // place: null where it is pos
    const float *cos_table, *sin_table;
    const float *q_weight, *k_weight;      // of the norms, or null: ones
    const uint16_t *q, *k, *v;
    uint16_t *q_out;
    long long q_stride, k_stride, v_stride, q_out_stride;
    int T, heads, n_pos;
    int units;            // of 16 elements, per token: queries, keys, values
    uint32_t units_inverse;   // floor(2^32 / units)
    int head_shift;       // units per head = 1 << head_shift
    int rot_units;        // rotated units of a head: rot / 16
    float eps;            // of the norms
};

// NORM: queries and keys times one over their head's root mean square and the norm's weights first; the lanes that have a head's units
// are neighbours in one row of 16, so its sum of squares takes two to four lane exchanges and no memory.
// A thread has a unit of 16 elements of one head of a token: where halves are paired, eight of each half; else, and
// of what is not rotated, 16 neighbours.  Every element is loaded and stored once, 16 bytes at a time; the tables' rows (4 rot bytes
// a token) are shared by the token's heads.  Bound by memory for prompts (5555 tokens, 32 + 2 x 8 heads of 256, 8-bit cache: 48.8 us, 5.2 TB/s)
// and by three loads after one another, position, page and tables, for single tokens (16 of 32 + 2 x 32 heads of 128: 3.4 us).  With norms 5003
// tokens, 40 + 2 x 8 heads of 128, half rotated in neighbouring pairs, 8-bit cache: 32.5 us, 4.1 TB/s; 16 tokens of 32 + 2 x 8 heads 3.4 us.
template <bool FP8, bool INTERLEAVED, bool NORM>
__global__ __launch_bounds__(256) void rope_append_kernel(AppendArgs a)
{
    const unsigned idx = blockIdx.x * 256u + threadIdx.x;
    int t = (int)__umulhi(idx, a.units_inverse), u = (int)(idx - (unsigned)t * (unsigned)a.units);    // (t: one too small at most)
    if (u >= a.units) { ++t; u -= a.units; }
    if (t >= a.T) return;
    const CacheArgs &C = a.cache;
    const int pos = a.pos[t], at = NORM && a.place ? a.place[t] : pos, seq = a.seq ? a.seq[t] : t;
    const int q_units = a.q ? a.heads << a.head_shift : 0;
    const bool is_q = u < q_units;
    const int w = is_q ? u : u - q_units;
    int h = w >> a.head_shift;
    const int part = w & ((1 << a.head_shift) - 1), dim = 16 << a.head_shift;
    const bool is_v = !is_q && h >= C.kv_heads;
    if (is_v) h -= C.kv_heads;
    const bool rotated = !is_v && part < a.rot_units;
    // where the unit's two groups of eight are
    int at0 = part * 16, at1 = at0 + 8;
    if (!INTERLEAVED && rotated) { at0 = part * 8; at1 = at0 + a.rot_units * 8; }

    // asked for before the page is known: the place in the table follows from the position, the page from the table
    const uint16_t *x = (is_q ? a.q + t * a.q_stride : is_v ? a.v + t * a.v_stride : a.k + t * a.k_stride) + h * dim;
    const u32x4 raw0 = *reinterpret_cast<const u32x4 *>(x + at0), raw1 = *reinterpret_cast<const u32x4 *>(x + at1);
    int page = -1;
    if (pos >= 0 && (a.rot_units == 0 || pos < a.n_pos) && at >= 0 && seq >= 0 && seq < C.n_seqs && (at >> C.page_shift) < C.n_blocks)
        page = C.table[seq * C.table_stride + (at >> C.page_shift)];
    const bool there = page >= 0 && page < C.n_pages;
    if (!there) {
        if (is_q) {
            uint16_t *o = a.q_out + t * a.q_out_stride + h * dim;
            *reinterpret_cast<u32x4 *>(o + at0) = u32x4{0, 0, 0, 0};
            *reinterpret_cast<u32x4 *>(o + at1) = u32x4{0, 0, 0, 0};
        }
        return;
    }
    Eight e0 = eight(raw0), e1 = eight(raw1);
    if (NORM && !is_v) {
        const float r = inverse_rms(e0, e1, a.head_shift, a.eps);
        const float *w = is_q ? a.q_weight : a.k_weight;
        const Eight w0 = weights_at(w, at0), w1 = weights_at(w, at1);
#pragma unroll
        for (int i = 0; i < 8; ++i) { e0.x[i] *= r * w0.x[i]; e1.x[i] *= r * w1.x[i]; }
    }
    if (rotated) turn<INTERLEAVED>(e0, e1, angles(a.cos_table, a.sin_table, pos, a.rot_units, part));
    if (is_q) {
        uint16_t *o = a.q_out + t * a.q_out_stride + h * dim;
        *reinterpret_cast<u32x4 *>(o + at0) = to_bf16(e0);
        *reinterpret_cast<u32x4 *>(o + at1) = to_bf16(e1);
        return;
    }
    const long long place = page * C.page_stride + h * C.head_stride + (at & C.page_mask) * C.slot_stride;
    if (FP8) {
        const float *scales = is_v ? C.v_scale : C.k_scale;
        const float scale = scales ? scales[h] : 1.f, inverse = 1.f / scale;
        uint8_t *o = static_cast<uint8_t *>(is_v ? C.v : C.k) + place;
        *reinterpret_cast<u32x2 *>(o + at0) = to_fp8(e0, scale, inverse);
        *reinterpret_cast<u32x2 *>(o + at1) = to_fp8(e1, scale, inverse);
    } else {
        uint16_t *o = static_cast<uint16_t *>(is_v ? C.v : C.k) + place;
        *reinterpret_cast<u32x4 *>(o + at0) = to_bf16(e0);
        *reinterpret_cast<u32x4 *>(o + at1) = to_bf16(e1);
    }
}

template <bool NORM> hipError_t launch_append(bool fp8, bool interleaved, const AppendArgs &a, unsigned blocks, hipStream_t stream)
{
    auto kernel = fp8 ? (interleaved ? rope_append_kernel<true, true, NORM> : rope_append_kernel<true, false, NORM>)
                      : (interleaved ? rope_append_kernel<false, true, NORM> : rope_append_kernel<false, false, NORM>);
    constexpr int id = NORM ? KID_NORM_ROPE_APPEND : KID_ROPE_APPEND;
    trace_before(id, stream);
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), 0, stream, a);
    trace_after(id, stream);
    return hipGetLastError();
}

// The arguments that both calls have, checked and, where they are right, in `a`.
peqa_status append_args(const peqa_kv_cache *C, int32_t T, const int32_t *pos, const int32_t *seq, const float *cos_table,
                        const float *sin_table, int32_t n_pos, int32_t rot, int32_t heads, const uint16_t *q, int64_t q_stride,
                        const uint16_t *k, int64_t k_stride, const uint16_t *v, int64_t v_stride, uint16_t *q_out, int64_t q_out_stride,
                        AppendArgs &a)
{
    const peqa_status st = peqa_check_cache(C);
    if (st != PEQA_OK) return st;
    if (!pos || !k || !v || (q != nullptr) != (q_out != nullptr)) return PEQA_ERR_NULL;
    const int D = C->head_dim;
    if (T < 1 || (q && (heads < 1 || heads > 65536)) || (!seq && T > C->n_seqs)) return PEQA_ERR_SHAPE;
    if (rot < 0 || rot > D || rot % 16 || (rot > 0 && n_pos < 1)) return PEQA_ERR_PARAM;
    if (rot > 0 && (!cos_table || !sin_table)) return PEQA_ERR_NULL;
    const int64_t q_width = (int64_t)heads * D, kv_width = (int64_t)C->kv_heads * D;
    if (k_stride < kv_width || v_stride < kv_width || (q && (q_stride < q_width || q_out_stride < q_width))) return PEQA_ERR_SHAPE;
    if (!aligned16(k) || !aligned16(v) || !aligned16(q) || !aligned16(q_out) || k_stride % 8 || v_stride % 8 ||
        (q && (q_stride % 8 || q_out_stride % 8)))
        return PEQA_ERR_ALIGN;
    if (rot > 0 && (!aligned16(cos_table) || !aligned16(sin_table))) return PEQA_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(pos) | reinterpret_cast<uintptr_t>(seq)) & 3) return PEQA_ERR_ALIGN;
    const int64_t units = ((q ? heads : 0) + 2 * (int64_t)C->kv_heads) * (D / 16);
    if (units * T > (int64_t)INT32_MAX - 256) return PEQA_ERR_SHAPE;    // 32-bit indexes of units in there
    a.cache = cache_args(C);
    a.pos = pos; a.seq = seq; a.cos_table = cos_table; a.sin_table = sin_table;
    a.q = q; a.k = k; a.v = v; a.q_out = q_out;
    a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.q_out_stride = q_out_stride;
    a.T = T; a.heads = heads; a.n_pos = n_pos;
    a.units = (int)units;                                      // (two at least)
    a.units_inverse = (uint32_t)((1ull << 32) / (uint64_t)units);
    a.head_shift = __builtin_ctz((unsigned)(D / 16));
    a.rot_units = rot / 16;
    return PEQA_OK;
}

}  // namespace
}  // namespace peqa

extern "C" {

peqa_status peqa_check_cache(const peqa_kv_cache *C)
{
    if (!C || !C->k || !C->v || !C->table) return PEQA_ERR_NULL;
    if (C->dtype != PEQA_CACHE_BF16 && C->dtype != PEQA_CACHE_FP8) return PEQA_ERR_PARAM;
    if (C->reserved != 0 || (C->dtype == PEQA_CACHE_BF16 && (C->k_scale || C->v_scale))) return PEQA_ERR_PARAM;
    if (C->page_size < 8 || C->page_size > 1024 || (C->page_size & (C->page_size - 1))) return PEQA_ERR_SHAPE;
    if (C->head_dim != 64 && C->head_dim != 128 && C->head_dim != 256) return PEQA_ERR_SHAPE;
    if (C->n_pages < 1 || C->kv_heads < 1 || C->kv_heads > 4096 || C->n_seqs < 1 || C->n_blocks < 1) return PEQA_ERR_SHAPE;
    if ((int64_t)C->n_blocks * C->page_size > (1 << 30) || C->table_stride < C->n_blocks) return PEQA_ERR_SHAPE;    // positions are 32-bit numbers
    if (C->page_stride < 0 || C->head_stride < 0 || C->slot_stride < C->head_dim) return PEQA_ERR_SHAPE;
    const int64_t unit = C->dtype == PEQA_CACHE_FP8 ? 16 : 8;
    if (C->slot_stride > (INT32_MAX / 2) / C->page_size) return PEQA_ERR_SHAPE;    // a head's slots of a page: 32-bit offsets in kernels
    if (!aligned16(C->k) || !aligned16(C->v) || C->page_stride % unit || C->head_stride % unit || C->slot_stride % unit)
        return PEQA_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(C->table) | reinterpret_cast<uintptr_t>(C->k_scale) | reinterpret_cast<uintptr_t>(C->v_scale)) & 3)
        return PEQA_ERR_ALIGN;
    return PEQA_OK;
}

peqa_status peqa_rope_append(const peqa_kv_cache *C, int32_t T, const int32_t *pos, const int32_t *seq, const float *cos_table,
                             const float *sin_table, int32_t n_pos, int32_t rot, int32_t interleaved, int32_t heads, const uint16_t *q,
                             int64_t q_stride, const uint16_t *k, int64_t k_stride, const uint16_t *v, int64_t v_stride, uint16_t *q_out,
                             int64_t q_out_stride, void *stream)
{
    peqa::AppendArgs a{};
    const peqa_status st = peqa::append_args(C, T, pos, seq, cos_table, sin_table, n_pos, rot, heads, q, q_stride, k, k_stride, v, v_stride,
                                             q_out, q_out_stride, a);
    if (st != PEQA_OK) return st;
    return dev_status(peqa::launch_append<false>(C->dtype == PEQA_CACHE_FP8, interleaved != 0, a, (unsigned)(((int64_t)a.units * T + 255) / 256),
                                                 static_cast<hipStream_t>(stream)));
}

peqa_status peqa_norm_rope_append(const peqa_kv_cache *C, int32_t T, const int32_t *pos, const int32_t *place, const int32_t *seq,
                                  const float *cos_table, const float *sin_table, int32_t n_pos, int32_t rot, int32_t interleaved,
                                  const float *q_weight, const float *k_weight, float eps, int32_t heads, const uint16_t *q,
                                  int64_t q_stride, const uint16_t *k, int64_t k_stride, const uint16_t *v, int64_t v_stride,
                                  uint16_t *q_out, int64_t q_out_stride, void *stream)
{
    peqa::AppendArgs a{};
    const peqa_status st = peqa::append_args(C, T, pos, seq, cos_table, sin_table, n_pos, rot, heads, q, q_stride, k, k_stride, v, v_stride,
                                             q_out, q_out_stride, a);
    if (st != PEQA_OK) return st;
    if (!(eps > 0.f) || eps > 3.402823466e38f) return PEQA_ERR_PARAM;
    if (!aligned16(q_weight) || !aligned16(k_weight) || (reinterpret_cast<uintptr_t>(place) & 3)) return PEQA_ERR_ALIGN;
    a.place = place; a.q_weight = q_weight; a.k_weight = k_weight; a.eps = eps;
    return dev_status(peqa::launch_append<true>(C->dtype == PEQA_CACHE_FP8, interleaved != 0, a, (unsigned)(((int64_t)a.units * T + 255) / 256),
                                                static_cast<hipStream_t>(stream)));
}

}  // extern "C"
