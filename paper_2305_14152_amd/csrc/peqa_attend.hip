// Attention of single query tokens over the paged cache (peqa_paged_attention).
//
// For a row and one of its key heads, with the heads that share it as columns:
//   x[j][h] = scale <k_j, q_h>;   out[h] = sum_j e^(x[j][h]) v_j / sum_j e^(x[j][h])
// in one pass over the positions j with the running maximum and sum of every head, all in powers of two (the scale carries
// log2 e).  Both products are matrix instructions that take their operands as they come from memory: the scores as keys x
// queries, so that a lane ends with eight scores of ONE head, which are the weights' operand of the second product as they
// stand, and values^T x weights, for which a lane loads whole 16-byte pieces of eight positions and turns the 8 x 8 elements
// in registers.
// Positions are split twice: tiles of 32 over the waves of a workgroup, chunks over workgroups; what the waves have is
// joined in LDS, and what the chunks have by a second kernel.
#include "peqa_cache.h"
#include "peqa_host.h"

using namespace peqa::host;

namespace peqa {

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr int TILE = 32;                 // positions per step of a wave
constexpr int WAVES = 4;
constexpr int CHUNK_MAX = 4096;          // positions of a workgroup at most (its pages' numbers are in LDS)
constexpr float LOWEST = -3.0e38f;       // finite stand-in for the maximum of nothing: e^(-inf - LOWEST) is 0, not NaN
constexpr float LN2 = 0.693147180559945309f, LOG2E = 1.44269504088896341f;

struct AttendArgs {
    CacheArgs cache;
    const uint16_t *q;
    const int32_t *lens, *seq;
    uint16_t *out;
    float *lse;
    float *part;               // [rows, heads, splits, head_dim] sums of the chunks, relative to their maxima
    float *part_ml;            // [rows, heads, splits, 2] maximum (of powers of two) and sum
    long long q_stride, out_stride;
    float scale;               // times log2 e
    int rows, heads, group;    // heads per key head
    int max_len, window;
    int chunk, splits, blocks; // positions of a chunk, chunks of the longest row, workgroups per key head
};

// What of a row there is: positions [lo, len), of which chunk s has [from + s chunk, ..) (from: lo rounded down to a tile).
struct RowRange {
    int seq, lo, from, len;
};
__device__ __forceinline__ RowRange row_range(const AttendArgs &a, int row)
{
    RowRange r;
    r.seq = a.seq ? a.seq[row] : row;
    int len = a.lens[row];
    len = len < a.max_len ? len : a.max_len;
    if (r.seq < 0 || r.seq >= a.cache.n_seqs || len < 0) len = 0;
    r.len = len;
    r.lo = a.window > 0 && len > a.window ? len - a.window : 0;
    r.from = r.lo & ~(TILE - 1);
    return r;
}

__device__ __forceinline__ f32x4 mfma_bf16(u32x4 x, u32x4 y, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma_f16(u32x4 x, u32x4 y, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0, 0, 0);
}

// Four 8-bit floats as bf16, or two as fp16: exact.
template <bool HI> __device__ __forceinline__ uint32_t fp8_bf16(uint32_t v)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, 1.f, HI));
}
template <bool HI> __device__ __forceinline__ uint32_t fp8_f16(uint32_t v)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v, 1.f, HI));
}

template <int D, bool FP8, int HB>
__global__ __launch_bounds__(64 * WAVES) void attend_kernel(AttendArgs a)
{
    // Columns of the matrix instructions: 16 heads with 8-bit values, whose weights are fp16; with bf16 values eight heads twice,
    // the upper ones with what rounding the weights to bf16 leaves, so that they have 16 bits.
    constexpr int COLS = FP8 ? 16 : 8;
    constexpr int QK = D / 32;                        // steps of the scores' product
    constexpr int SEG = D > 128 ? D / 128 : 1;        // segments of 128 elements of a value
    constexpr int W = D / 16 / SEG;                   // neighbouring elements of a segment that a lane has: 4 or 8
    constexpr int KB = FP8 ? D / 64 : D / 32;         // 16-byte pieces of a key that a lane loads
    constexpr int VR = FP8 ? W / 4 : W / 2;           // registers of a value's segment
    __shared__ int32_t pages[CHUNK_MAX / 8 + 8];
    __shared__ float wave_m[WAVES][HB][16], wave_l[WAVES][HB][16];
    __shared__ f32x4 joined[WAVES / 2][HB * SEG * W][64];

    const CacheArgs &C = a.cache;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, g = lane >> 4;
    unsigned idx = blockIdx.x;
    const unsigned per_split = (unsigned)(C.kv_heads * a.blocks);
    const int hb = (int)(idx % per_split);
    idx /= per_split;
    const int split = (int)(idx % (unsigned)a.splits), row = (int)(idx / (unsigned)a.splits);
    const int kv_head = hb / a.blocks, first = (hb - kv_head * a.blocks) * COLS * HB;    // of the heads that share kv_head
    const RowRange range = row_range(a, row);
    const int begin = range.from + split * a.chunk;
    const int end = begin + a.chunk < range.len ? begin + a.chunk : range.len;
    if (begin >= range.len && split > 0) return;
    const bool alone = range.len - range.from <= a.chunk;

    // this lane's head in every block of columns
    int head[HB];
    bool live[HB];
#pragma unroll
    for (int b = 0; b < HB; ++b) {
        const int i = first + b * COLS + (c & (COLS - 1));
        live[b] = i < a.group;
        head[b] = kv_head * a.group + (live[b] ? i : 0);
    }

    // numbers of the chunk's pages
    const int block0 = begin >> C.page_shift, nblocks = end > begin ? ((end - 1) >> C.page_shift) - block0 + 1 : 0;
    for (int i = threadIdx.x; i < nblocks; i += 64 * WAVES) {
        const int p = C.table[range.seq * C.table_stride + block0 + i];
        pages[i] = p >= 0 && p < C.n_pages ? p : -1;
    }
    u32x4 q[HB][QK];
#pragma unroll
    for (int b = 0; b < HB; ++b) {
        const uint16_t *src = a.q + row * a.q_stride + (long long)head[b] * D;
#pragma unroll
        for (int s = 0; s < QK; ++s) {
            // the keys' pieces decide which elements a step has
            const int at = FP8 ? 64 * (s >> 1) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g;
            q[b][s] = *reinterpret_cast<const u32x4 *>(src + at);
            if (!live[b]) q[b][s] = u32x4{0, 0, 0, 0};
        }
    }
    __syncthreads();

    const float k_scale = FP8 && C.k_scale ? C.k_scale[kv_head] : 1.f;
    const float scale = a.scale * k_scale;
    const uint8_t *kbase = static_cast<const uint8_t *>(C.k) + kv_head * C.head_stride * (FP8 ? 1 : 2);
    const uint8_t *vbase = static_cast<const uint8_t *>(C.v) + kv_head * C.head_stride * (FP8 ? 1 : 2);
    constexpr int EL = FP8 ? 1 : 2;

    float m[HB], l[HB];
    f32x4 acc[HB][SEG * W];
#pragma unroll
    for (int b = 0; b < HB; ++b) {
        m[b] = LOWEST;
        l[b] = 0.f;
#pragma unroll
        for (int e = 0; e < SEG * W; ++e) acc[b][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    for (int t0 = begin + wave * TILE; t0 < end; t0 += WAVES * TILE) {
        // addresses: of the keys at t0 + c, t0 + 16 + c, of the values at t0 + 4 g .. and t0 + 16 + 4 g ..; positions past the
        // end read the last one
        bool whole = t0 >= range.lo && t0 + TILE <= end;
        long long kat[2], vat[2][4];
        bool vthere[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int kp = t0 + 16 * s + c, kq = kp < end ? kp : end - 1;
            const int page = pages[(kq >> C.page_shift) - block0];
            whole = whole && page >= 0;
            kat[s] = ((page < 0 ? 0 : page) * C.page_stride + (kq & C.page_mask) * C.slot_stride + (FP8 ? 16 : 8) * g) * EL;
            const int vp = t0 + 16 * s + 4 * g, vq = vp < end ? vp : end - 1;
            const int vpage = pages[(vq >> C.page_shift) - block0];
            vthere[s] = vpage >= 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = vp + i < end ? vp + i : end - 1;
                vat[s][i] = ((vpage < 0 ? 0 : vpage) * C.page_stride + (at & C.page_mask) * C.slot_stride + W * c) * EL;
            }
        }
        u32x4 k[2][KB];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int j = 0; j < KB; ++j)
                k[s][j] = *reinterpret_cast<const u32x4 *>(kbase + kat[s] + 64 * j);
        uint32_t v[8][SEG][VR];
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int s = 0; s < SEG; ++s) {
                const uint8_t *src = vbase + vat[i >> 2][i & 3] + 128 * EL * s;
                if constexpr (VR == 4) {
                    const u32x4 x = *reinterpret_cast<const u32x4 *>(src);
#pragma unroll
                    for (int r = 0; r < VR; ++r) v[i][s][r] = x[r];
                } else if constexpr (VR == 2) {
                    const u32x2 x = *reinterpret_cast<const u32x2 *>(src);
#pragma unroll
                    for (int r = 0; r < VR; ++r) v[i][s][r] = x[r];
                } else {
                    v[i][s][0] = *reinterpret_cast<const uint32_t *>(src);
                }
            }
        const bool full = __ballot(!whole) == 0;
        if (!full) {
            // what masked positions hold must not meet a weight of 0: NaN and infinities would stay
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int p = t0 + 16 * (i >> 2) + 4 * g + (i & 3);
                const bool in = p >= range.lo && p < end && vthere[i >> 2];
#pragma unroll
                for (int s = 0; s < SEG; ++s)
#pragma unroll
                    for (int r = 0; r < VR; ++r) v[i][s][r] = in ? v[i][s][r] : 0u;
            }
        }

        u32x4 weight[HB];
#pragma unroll
        for (int b = 0; b < HB; ++b) {
            f32x4 x[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int j = 0; j < QK; ++j) {
                    u32x4 kj;
                    if constexpr (FP8) {
                        const uint32_t lo = k[s][j >> 1][2 * (j & 1)], hi = k[s][j >> 1][2 * (j & 1) + 1];
                        kj = u32x4{fp8_bf16<false>(lo), fp8_bf16<true>(lo), fp8_bf16<false>(hi), fp8_bf16<true>(hi)};
                    } else {
                        kj = k[s][j];
                    }
                    x[s] = mfma_bf16(kj, q[b][j], x[s]);
                }
            float y[8], top = LOWEST;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                y[i] = x[i >> 2][i & 3] * scale;
                if (!full) {
                    const int p = t0 + 16 * (i >> 2) + 4 * g + (i & 3);
                    y[i] = p >= range.lo && p < end && vthere[i >> 2] ? y[i] : -__builtin_inff();
                }
                top = fmaxf(top, y[i]);
            }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float mn = fmaxf(m[b], top), fall = __builtin_amdgcn_exp2f(m[b] - mn);
            m[b] = mn;
            float p[8], sum = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                p[i] = __builtin_amdgcn_exp2f(y[i] - mn);
                sum += p[i];
            }
            l[b] = l[b] * fall + sum;
#pragma unroll
            for (int e = 0; e < SEG * W; ++e) acc[b][e] *= fall;
            if constexpr (FP8) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    weight[b][i] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)p[2 * i], (_Float16)p[2 * i + 1]});
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t near = pack_bf16x2(p[2 * i], p[2 * i + 1]);
                    const uint32_t rest = pack_bf16x2(p[2 * i] - bf16_lo(near), p[2 * i + 1] - bf16_hi(near));
                    weight[b][i] = c < 8 ? near : rest;
                }
            }
        }
#pragma unroll
        for (int s = 0; s < SEG; ++s)
#pragma unroll
            for (int r = 0; r < VR; ++r) {
                if constexpr (FP8) {
                    // elements 4 r .. 4 r + 3: bytes of two positions next to each other, then to fp16
                    uint32_t lo[4], hi[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        lo[i] = __builtin_amdgcn_perm(v[2 * i + 1][s][r], v[2 * i][s][r], 0x05010400u);
                        hi[i] = __builtin_amdgcn_perm(v[2 * i + 1][s][r], v[2 * i][s][r], 0x07030602u);
                    }
                    const u32x4 e0 = {fp8_f16<false>(lo[0]), fp8_f16<false>(lo[1]), fp8_f16<false>(lo[2]), fp8_f16<false>(lo[3])};
                    const u32x4 e1 = {fp8_f16<true>(lo[0]), fp8_f16<true>(lo[1]), fp8_f16<true>(lo[2]), fp8_f16<true>(lo[3])};
                    const u32x4 e2 = {fp8_f16<false>(hi[0]), fp8_f16<false>(hi[1]), fp8_f16<false>(hi[2]), fp8_f16<false>(hi[3])};
                    const u32x4 e3 = {fp8_f16<true>(hi[0]), fp8_f16<true>(hi[1]), fp8_f16<true>(hi[2]), fp8_f16<true>(hi[3])};
#pragma unroll
                    for (int b = 0; b < HB; ++b) {
                        acc[b][s * W + 4 * r] = mfma_f16(e0, weight[b], acc[b][s * W + 4 * r]);
                        acc[b][s * W + 4 * r + 1] = mfma_f16(e1, weight[b], acc[b][s * W + 4 * r + 1]);
                        acc[b][s * W + 4 * r + 2] = mfma_f16(e2, weight[b], acc[b][s * W + 4 * r + 2]);
                        acc[b][s * W + 4 * r + 3] = mfma_f16(e3, weight[b], acc[b][s * W + 4 * r + 3]);
                    }
                } else {
                    u32x4 e0, e1;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        e0[i] = __builtin_amdgcn_perm(v[2 * i + 1][s][r], v[2 * i][s][r], 0x05040100u);
                        e1[i] = __builtin_amdgcn_perm(v[2 * i + 1][s][r], v[2 * i][s][r], 0x07060302u);
                    }
#pragma unroll
                    for (int b = 0; b < HB; ++b) {
                        acc[b][s * W + 2 * r] = mfma_bf16(e0, weight[b], acc[b][s * W + 2 * r]);
                        acc[b][s * W + 2 * r + 1] = mfma_bf16(e1, weight[b], acc[b][s * W + 2 * r + 1]);
                    }
                }
            }
    }

    // the waves' maxima and sums, then their accumulators in a tree
#pragma unroll
    for (int b = 0; b < HB; ++b) {
        l[b] += __shfl_xor(l[b], 16);
        l[b] += __shfl_xor(l[b], 32);
        if (g == 0) { wave_m[wave][b][c] = m[b]; wave_l[wave][b][c] = l[b]; }
    }
    __syncthreads();
    float total[HB], top[HB];
#pragma unroll
    for (int b = 0; b < HB; ++b) {
        top[b] = LOWEST;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top[b] = fmaxf(top[b], wave_m[w][b][c]);
        total[b] = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) total[b] += wave_l[w][b][c] * __builtin_amdgcn_exp2f(wave_m[w][b][c] - top[b]);
        const float mine = __builtin_amdgcn_exp2f(m[b] - top[b]);
#pragma unroll
        for (int e = 0; e < SEG * W; ++e) acc[b][e] *= mine;
    }
#pragma unroll
    for (int half = WAVES / 2; half >= 1; half /= 2) {
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int b = 0; b < HB; ++b)
#pragma unroll
                for (int e = 0; e < SEG * W; ++e) joined[wave - half][b * SEG * W + e][lane] = acc[b][e];
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int b = 0; b < HB; ++b)
#pragma unroll
                for (int e = 0; e < SEG * W; ++e) acc[b][e] += joined[wave][b * SEG * W + e][lane];
        __syncthreads();
    }
    if (wave != 0) return;

    const float v_scale = FP8 && C.v_scale ? C.v_scale[kv_head] : 1.f;
#pragma unroll
    for (int b = 0; b < HB; ++b) {
        if constexpr (!FP8)
#pragma unroll
            for (int e = 0; e < SEG * W; ++e)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[b][e][r] += __shfl_xor(acc[b][e][r], 8);
        if (!live[b] || c >= COLS) continue;
        // this lane: elements 128 s + W (4 g + r) + e
        const size_t rh = (size_t)row * a.heads + head[b];
        if (alone) {
            const float by = total[b] > 0.f || total[b] != total[b] ? v_scale / total[b] : 0.f;
            uint16_t *o = a.out + row * a.out_stride + (long long)head[b] * D;
#pragma unroll
            for (int s = 0; s < SEG; ++s)
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int e = 0; e < W; e += 4) {
                        const u32x2 x = {pack_bf16x2(acc[b][s * W + e][r] * by, acc[b][s * W + e + 1][r] * by),
                                         pack_bf16x2(acc[b][s * W + e + 2][r] * by, acc[b][s * W + e + 3][r] * by)};
                        *reinterpret_cast<u32x2 *>(o + 128 * s + W * (4 * g + r) + e) = x;
                    }
            if (a.lse && g == 0)
                a.lse[rh] = total[b] > 0.f || total[b] != total[b] ? (top[b] + __builtin_amdgcn_logf(total[b])) * LN2 : -__builtin_inff();
        } else {
            const size_t at = rh * a.splits + split;
            float *o = a.part + at * D;
#pragma unroll
            for (int s = 0; s < SEG; ++s)
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int e = 0; e < W; e += 4)
                        *reinterpret_cast<f32x4 *>(o + 128 * s + W * (4 * g + r) + e) =
                            f32x4{acc[b][s * W + e][r], acc[b][s * W + e + 1][r], acc[b][s * W + e + 2][r], acc[b][s * W + e + 3][r]};
            if (g == 0) {
                a.part_ml[2 * at] = top[b];
                a.part_ml[2 * at + 1] = total[b];
            }
        }
    }
}

// Joins the chunks of the rows that have several: one workgroup per row and head.  A group of D / 4 lanes reads the
// sums of a chunk, 16 bytes a lane; the groups take the chunks in turn, four loads of a lane in flight, and meet in LDS.
template <int D, bool FP8>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a)
{
    constexpr int LANES = D / 4, GROUPS = 256 / LANES, BATCH = 256;
    __shared__ float weight[BATCH], wave_x[4];
    __shared__ f32x4 sums[GROUPS][LANES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row = (int)(blockIdx.x / (unsigned)a.heads), head = (int)(blockIdx.x - (unsigned)row * (unsigned)a.heads);
    const RowRange range = row_range(a, row);
    const int n = (range.len - range.from + a.chunk - 1) / a.chunk;
    if (n < 2) return;
    const size_t rh = (size_t)row * a.heads + head;
    const float *ml = a.part_ml + 2 * rh * a.splits;
    float top = LOWEST;
    for (int s = tid; s < n; s += 256) top = fmaxf(top, ml[2 * s]);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    if (lane == 0) wave_x[wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(wave_x[0], wave_x[1]), fmaxf(wave_x[2], wave_x[3]));
    const int at = tid % LANES, group = tid / LANES;
    const f32x4 *part = reinterpret_cast<const f32x4 *>(a.part + rh * a.splits * D) + at;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    float total = 0.f;
    for (int s0 = 0; s0 < n; s0 += BATCH) {
        const int here = n - s0 < BATCH ? n - s0 : BATCH;
        __syncthreads();                                       // (also: everyone has read wave_x)
        float w = 0.f;
        if (tid < here) {
            w = __builtin_amdgcn_exp2f(ml[2 * (s0 + tid)] - top);
            total += w * ml[2 * (s0 + tid) + 1];
        }
        weight[tid] = w;
        __syncthreads();
        for (int i = group; i < here; i += 4 * GROUPS) {
            f32x4 x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = part[(size_t)(s0 + (i + k * GROUPS < here ? i + k * GROUPS : i)) * LANES];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float wk = i + k * GROUPS < here ? weight[i + k * GROUPS] : 0.f;
                if (i + k * GROUPS < here) sum += x[k] * wk;
            }
        }
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) total += __shfl_xor(total, o);
    if (lane == 0) wave_x[wave] = total;
    sums[group][at] = sum;
    __syncthreads();
    if (tid >= LANES) return;
    total = (wave_x[0] + wave_x[1]) + (wave_x[2] + wave_x[3]);
#pragma unroll
    for (int k = 1; k < GROUPS; ++k) sum += sums[k][at];
    const bool any = total > 0.f || total != total;
    const float v_scale = FP8 && a.cache.v_scale ? a.cache.v_scale[head / a.group] : 1.f;
    const float by = any ? v_scale / total : 0.f;
    uint16_t *o = a.out + row * a.out_stride + (long long)head * D + 4 * at;
    *reinterpret_cast<u32x2 *>(o) = u32x2{pack_bf16x2(sum[0] * by, sum[1] * by), pack_bf16x2(sum[2] * by, sum[3] * by)};
    if (a.lse && tid == 0) a.lse[rh] = any ? (top + __builtin_amdgcn_logf(total)) * LN2 : -__builtin_inff();
}

template <int D, bool FP8>
hipError_t launch_attend(const AttendArgs &a, int hb, hipStream_t stream)
{
    const unsigned grid = (unsigned)a.rows * (unsigned)a.splits * (unsigned)(a.cache.kv_heads * a.blocks);
    trace_before(KID_ATTEND, stream);
    if constexpr (D <= 128) {
        if (hb == 2)
            hipLaunchKernelGGL((attend_kernel<D, FP8, 2>), dim3(grid), dim3(64 * WAVES), 0, stream, a);
        else
            hipLaunchKernelGGL((attend_kernel<D, FP8, 1>), dim3(grid), dim3(64 * WAVES), 0, stream, a);
    } else {
        hipLaunchKernelGGL((attend_kernel<D, FP8, 1>), dim3(grid), dim3(64 * WAVES), 0, stream, a);
    }
    trace_after(KID_ATTEND, stream);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    trace_before(KID_ATTEND_JOIN, stream);
    hipLaunchKernelGGL((attend_join_kernel<D, FP8>), dim3((unsigned)a.rows * (unsigned)a.heads), dim3(256), 0, stream, a);
    trace_after(KID_ATTEND_JOIN, stream);
    return hipGetLastError();
}

// How a call is cut: column blocks of a workgroup, workgroups per key head, chunk and chunks of the longest row.
struct AttendPlan {
    int hb, blocks, chunk, splits;
    size_t part_bytes, ml_bytes;
};

AttendPlan attend_plan(const peqa_kv_cache *C, int rows, int heads, int max_len, int window)
{
    AttendPlan p{};
    const int group = heads / C->kv_heads, cols = C->dtype == PEQA_CACHE_FP8 ? 16 : 8;
    p.hb = C->head_dim <= 128 && group > cols ? 2 : 1;
    p.blocks = (group + cols * p.hb - 1) / (cols * p.hb);
    const long long span = window > 0 && (long long)window + TILE - 1 < max_len ? (long long)window + TILE - 1 : max_len;
    const long long items = (long long)rows * C->kv_heads * p.blocks;
    // workgroups for every unit several times over, but no chunk under two tiles a wave
#ifndef WANT
#define WANT 8
#endif
    long long want = (PLAN_UNITS * (long long)WANT + items - 1) / items;
    long long chunk = (span + want - 1) / want;
#ifndef LEAST
#define LEAST 2
#endif
    const long long least = LEAST * WAVES * TILE;
    if (chunk < least) chunk = least;
    if (chunk > CHUNK_MAX) chunk = CHUNK_MAX;
    p.chunk = (int)((chunk + TILE * WAVES - 1) / (TILE * WAVES) * (TILE * WAVES));
    p.splits = (int)((span + p.chunk - 1) / p.chunk);
    if (p.splits < 1) p.splits = 1;
    if (p.splits > 1) {
        const size_t parts = (size_t)rows * (size_t)heads * (size_t)p.splits;
        p.part_bytes = round256(parts * (size_t)C->head_dim * sizeof(float));
        p.ml_bytes = round256(parts * 2 * sizeof(float));
    }
    return p;
}

peqa_status check_attend(const peqa_kv_cache *C, int32_t rows, int32_t heads, int32_t max_len, int32_t window)
{
    const peqa_status st = peqa_check_cache(C);
    if (st != PEQA_OK) return st;
    if (rows < 1 || heads < 1 || heads > 65536 || heads % C->kv_heads || max_len < 0) return PEQA_ERR_SHAPE;
    if ((int64_t)max_len > (int64_t)C->n_blocks * C->page_size) return PEQA_ERR_SHAPE;
    if (window < 0) return PEQA_ERR_PARAM;
    const AttendPlan p = attend_plan(C, rows, heads, max_len, window);
    const int64_t wgs = (int64_t)C->kv_heads * p.blocks * p.splits;
    if (wgs > INT32_MAX / rows || (int64_t)rows * heads > INT32_MAX) return PEQA_ERR_SHAPE;
    return PEQA_OK;
}

}  // namespace
}  // namespace peqa

extern "C" {

size_t peqa_paged_attention_workspace_bytes(const peqa_kv_cache *C, int32_t rows, int32_t heads, int32_t max_len, int32_t window)
{
    if (peqa::check_attend(C, rows, heads, max_len, window) != PEQA_OK) return 0;
    const peqa::AttendPlan p = peqa::attend_plan(C, rows, heads, max_len, window);
    const size_t bytes = p.part_bytes + p.ml_bytes;
    return bytes ? bytes : 256;                                // (0 would read as "invalid")
}

peqa_status peqa_paged_attention(const peqa_kv_cache *C, int32_t rows, int32_t heads, const uint16_t *q, int64_t q_stride,
                                 const int32_t *lens, const int32_t *seq, int32_t max_len, int32_t window, float scale, uint16_t *out,
                                 int64_t out_stride, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    const peqa_status st = peqa::check_attend(C, rows, heads, max_len, window);
    if (st != PEQA_OK) return st;
    if (!q || !lens || !out) return PEQA_ERR_NULL;
    if (!seq && rows > C->n_seqs) return PEQA_ERR_SHAPE;
    const int64_t width = (int64_t)heads * C->head_dim;
    if (q_stride < width || out_stride < width) return PEQA_ERR_SHAPE;
    if (!aligned16(q) || !aligned16(out) || q_stride % 8 || out_stride % 8) return PEQA_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(lens) | reinterpret_cast<uintptr_t>(seq) | reinterpret_cast<uintptr_t>(lse)) & 3) return PEQA_ERR_ALIGN;
    const peqa::AttendPlan p = peqa::attend_plan(C, rows, heads, max_len, window);
    if (p.splits > 1) {
        if (!workspace || workspace_bytes < p.part_bytes + p.ml_bytes) return PEQA_ERR_WORKSPACE;
        if (!aligned16(workspace)) return PEQA_ERR_ALIGN;
    }
    peqa::AttendArgs a{};
    a.cache = peqa::cache_args(C);
    a.q = q; a.lens = lens; a.seq = seq; a.out = out; a.lse = lse;
    a.part = static_cast<float *>(workspace);
    a.part_ml = p.splits > 1 ? reinterpret_cast<float *>(static_cast<char *>(workspace) + p.part_bytes) : nullptr;
    a.q_stride = q_stride; a.out_stride = out_stride;
    a.scale = scale * peqa::LOG2E;
    a.rows = rows; a.heads = heads; a.group = heads / C->kv_heads;
    a.max_len = max_len; a.window = window;
    a.chunk = p.chunk; a.splits = p.splits; a.blocks = p.blocks;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool fp8 = C->dtype == PEQA_CACHE_FP8;
    hipError_t e;
    switch (C->head_dim) {
    case 64: e = fp8 ? peqa::launch_attend<64, true>(a, p.hb, s) : peqa::launch_attend<64, false>(a, p.hb, s); break;
    case 128: e = fp8 ? peqa::launch_attend<128, true>(a, p.hb, s) : peqa::launch_attend<128, false>(a, p.hb, s); break;
    default: e = fp8 ? peqa::launch_attend<256, true>(a, p.hb, s) : peqa::launch_attend<256, false>(a, p.hb, s); break;
    }
    return dev_status(e);
}

}  // extern "C"
