// New tokens into the paged cache (peqa_rope_append), and the host's check of the cache's descriptor.
#include "peqa_cache.h"
#include "peqa_host.h"

using namespace peqa::host;

namespace peqa {

namespace {

struct AppendArgs {
    CacheArgs cache;
    const int32_t *pos, *seq;
    const float *cos_table, *sin_table;
    const uint16_t *q, *k, *v;
    uint16_t *q_out;
    long long q_stride, k_stride, v_stride, q_out_stride;
    int T, heads, n_pos;
    int units;            // of 16 elements, per token: queries, keys, values
    uint32_t units_inverse;   // floor(2^32 / units)
    int head_shift;       // units per head = 1 << head_shift
    int rot_units;        // rotated units of a head: rot / 16
};

struct Eight {
    float x[8];
};

__device__ __forceinline__ Eight eight(u32x4 v)
{
    Eight e;
#pragma unroll
    for (int i = 0; i < 4; ++i) { e.x[2 * i] = bf16_lo(v[i]); e.x[2 * i + 1] = bf16_hi(v[i]); }
    return e;
}

__device__ __forceinline__ u32x4 to_bf16(const Eight &e)
{
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pack_bf16x2(e.x[2 * i], e.x[2 * i + 1]);
    return v;
}

// x / scale to 8-bit floats, nearest even, past the largest finite value to it; NaN stays NaN.  The quotient is the product with the
// reciprocal and one correction by its remainder, three instructions for the eleven of a division (half of the vector instructions of
// keys and values); a quotient that is infinite has no remainder.
__device__ __forceinline__ u32x2 to_fp8(const Eight &e, float scale, float inverse)
{
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float first = e.x[i] * inverse, d = fabsf(first) < 1024.f ? fmaf(fmaf(-first, scale, e.x[i]), inverse, first) : first;
        y[i] = d != d ? d : fminf(fmaxf(d, -448.f), 448.f);
    }
    u32x2 v;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
        v[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], w, true);
    }
    return v;
}

// Pair i of the rotated elements: (a, b) -> (a c - b s, a s + b c), c and s from the tables at the token's position.
// A thread has a unit of 16 elements of one head of a token: where halves are paired, eight of each half; else, and
// of what is not rotated, 16 neighbours.  Every element is loaded and stored once, 16 bytes at a time; the tables' rows (4 rot bytes
// a token) are shared by the token's heads.  Bound by memory for prompts (5555 tokens, 32 + 2 x 8 heads of 256, 8-bit cache: 48.8 us, 5.2 TB/s)
// and by three loads after one another, position, page and tables, for single tokens (16 of 32 + 2 x 32 heads of 128: 3.4 us).
template <bool FP8, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rope_append_kernel(AppendArgs a)
{
    const unsigned idx = blockIdx.x * 256u + threadIdx.x;
    int t = (int)__umulhi(idx, a.units_inverse), u = (int)(idx - (unsigned)t * (unsigned)a.units);    // (t: one too small at most)
    if (u >= a.units) { ++t; u -= a.units; }
    if (t >= a.T) return;
    const CacheArgs &C = a.cache;
    const int pos = a.pos[t], seq = a.seq ? a.seq[t] : t;
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
    if (pos >= 0 && (a.rot_units == 0 || pos < a.n_pos) && seq >= 0 && seq < C.n_seqs && (pos >> C.page_shift) < C.n_blocks)
        page = C.table[seq * C.table_stride + (pos >> C.page_shift)];
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
    if (rotated) {
        const size_t row = (size_t)pos * (size_t)(a.rot_units * 8) + (size_t)(part * 8);
        float c[8], s[8];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const f32x4 cv = *reinterpret_cast<const f32x4 *>(a.cos_table + row + 4 * i);
            const f32x4 sv = *reinterpret_cast<const f32x4 *>(a.sin_table + row + 4 * i);
#pragma unroll
            for (int j = 0; j < 4; ++j) { c[4 * i + j] = cv[j]; s[4 * i + j] = sv[j]; }
        }
        if (INTERLEAVED) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a0 = e0.x[2 * i], b0 = e0.x[2 * i + 1], a1 = e1.x[2 * i], b1 = e1.x[2 * i + 1];
                e0.x[2 * i] = a0 * c[i] - b0 * s[i];
                e0.x[2 * i + 1] = a0 * s[i] + b0 * c[i];
                e1.x[2 * i] = a1 * c[4 + i] - b1 * s[4 + i];
                e1.x[2 * i + 1] = a1 * s[4 + i] + b1 * c[4 + i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float p = e0.x[i], r = e1.x[i];
                e0.x[i] = p * c[i] - r * s[i];
                e1.x[i] = p * s[i] + r * c[i];
            }
        }
    }
    if (is_q) {
        uint16_t *o = a.q_out + t * a.q_out_stride + h * dim;
        *reinterpret_cast<u32x4 *>(o + at0) = to_bf16(e0);
        *reinterpret_cast<u32x4 *>(o + at1) = to_bf16(e1);
        return;
    }
    const long long place = page * C.page_stride + h * C.head_stride + (pos & C.page_mask) * C.slot_stride;
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

hipError_t launch_rope_append(bool fp8, bool interleaved, const AppendArgs &a, unsigned blocks, hipStream_t stream)
{
    auto kernel = fp8 ? (interleaved ? rope_append_kernel<true, true> : rope_append_kernel<true, false>)
                      : (interleaved ? rope_append_kernel<false, true> : rope_append_kernel<false, false>);
    trace_before(KID_ROPE_APPEND, stream);
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), 0, stream, a);
    trace_after(KID_ROPE_APPEND, stream);
    return hipGetLastError();
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
    peqa::AppendArgs a{};
    a.cache = peqa::cache_args(C);
    a.pos = pos; a.seq = seq; a.cos_table = cos_table; a.sin_table = sin_table;
    a.q = q; a.k = k; a.v = v; a.q_out = q_out;
    a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.q_out_stride = q_out_stride;
    a.T = T; a.heads = heads; a.n_pos = n_pos;
    a.units = (int)units;                                      // (two at least)
    a.units_inverse = (uint32_t)((1ull << 32) / (uint64_t)units);
    a.head_shift = __builtin_ctz((unsigned)(D / 16));
    a.rot_units = rot / 16;
    return dev_status(peqa::launch_rope_append(C->dtype == PEQA_CACHE_FP8, interleaved != 0, a, (unsigned)((units * T + 255) / 256),
                                               static_cast<hipStream_t>(stream)));
}

}  // extern "C"
