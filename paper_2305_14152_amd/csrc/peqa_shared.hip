// Attention of single query tokens whose sequences begin with the same positions (peqa_shared_attention): those are read once for all rows.
//
// For a key head the queries of all rows and of the heads that share it are the columns of one product with the shared positions; what
// a row has of its own is a product with its heads alone.  Both are cut into chunks of positions, a workgroup each, in one launch, and every
// column's parts (running maximum, sum, weighted values) are joined by a second one.  A workgroup has up to 64 columns (heads of 128) in blocks of 16, its four
// waves take tiles of 32 positions in turn and have all columns of each, so that a key or a value that is loaded is used for every column
// without passing through LDS; the products and their operands are those of the paged attention (scores as keys x queries, whose result is the
// weights' operand of values^T x weights as it stands; values are turned 8 x 8 in registers).
#include "peqa_attend.h"
#include "peqa_cache.h"
#include "peqa_host.h"

using namespace peqa::host;

namespace peqa {

namespace {

constexpr int TILE = 32, WAVES = 4, STEP = TILE * WAVES;   // positions of a wave's step, and of a workgroup's

struct SharedArgs {
    CacheArgs cache;
    const uint16_t *q;
    const int32_t *lens, *seq;
    uint16_t *out;
    float *lse;
    float *part, *part_ml;     // [slots, head_dim] weighted sums, [slots, 2] reference (of powers of two) and sum: a slot is a column's part
    long long q_stride, out_stride;
    float scale;               // times log2 e
    int rows, heads, group;    // heads per key head
    int max_len, prefix, shared;
    int columns, tiles;        // of the shared positions' workgroups: columns of one, and how many have all
    int chunk, chunks;         // positions of one, and how many have the shared ones
    int prefix_wgs;
    int own_chunk, own_splits; // positions of a row's own at least, and workgroups of a row and a block of heads
    int own_blocks, own_columns;   // blocks of a key head's heads, and heads in one
};

// A row's own positions [lo, len): those behind the shared ones, or, of a row that ends among those, all of them by itself.
struct RowInfo {
    int len, lo, seq;
    bool follows;              // sees all shared positions
};
__device__ __forceinline__ RowInfo row_info(const SharedArgs &a, int row)
{
    RowInfo r;
    r.seq = a.seq ? a.seq[row] : row;
    r.len = a.lens[row];
    r.len = r.len < a.max_len ? r.len : a.max_len;
    if (r.seq < 0 || r.seq >= a.cache.n_seqs || r.len < 0) r.len = 0;
    r.follows = r.len >= a.shared && r.len > 0;
    r.lo = r.follows ? a.shared : 0;
    if (!r.follows) r.seq = a.prefix;
    return r;
}
// Chunks of a row's own positions: `length` positions each from `from` on (lo rounded down to a tile).
struct OwnChunks {
    int from, length, n;
};
__device__ __forceinline__ OwnChunks own_chunks(const SharedArgs &a, const RowInfo &r)
{
    OwnChunks o;
    o.from = r.lo & ~(TILE - 1);
    const int span = r.len > r.lo ? r.len - o.from : 0;
    o.length = ((span + a.own_splits - 1) / a.own_splits + STEP - 1) & ~(STEP - 1);
    o.length = o.length > a.own_chunk ? o.length : a.own_chunk;
    o.n = (span + o.length - 1) / o.length;
    return o;
}

// What a workgroup does: columns of a key head against positions [lo, end), walked from `begin` on, of the sequence of one row of the table.
struct Item {
    int kv_head, first, n;     // queries first .. first + n - 1: number row * group + head of the key head's
    int lo, begin, end;
    const int32_t *table;
    long long slot;            // of the first column
};

// The pages of a tile of 32 positions: four at most, neighbouring entries of the table (the last ones of an item again past its end).
struct Pages {
    long long at[4];           // in bytes
    uint32_t there;            // bit i: the page is there
};

typedef const __attribute__((address_space(4))) int32_t *scalar_ints;

template <int D> struct Shape {
    static constexpr int SEG = D > 128 ? D / 128 : 1, DS = D / SEG;
};

template <int D, bool FP8, int HB>
__device__ __forceinline__ void attend_item(const SharedArgs &a, const Item &it, u32x4 *lds_q, float (*wave_m)[16], float (*wave_l)[16],
                                            float (*joined)[16][Shape<D>::DS + 4])
{
    constexpr int QK = D / 32;                        // steps of the scores' product
    constexpr int SEG = Shape<D>::SEG, DS = Shape<D>::DS;
    constexpr int W = D / 16 / SEG;                   // neighbouring elements of a segment that a lane has: 4 or 8
    constexpr int KB = FP8 ? D / 64 : D / 32;         // 16-byte pieces of a key that a lane loads
    constexpr int VR = FP8 ? W / 4 : W / 2;           // registers of a value's segment
    constexpr int EL = FP8 ? 1 : 2;
    constexpr bool QUERIES_IN_LDS = HB > 2;
    constexpr bool AHEAD = HB * D < 512 || (FP8 && D <= 128);       // registers for two tiles
    const CacheArgs &C = a.cache;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, g = lane >> 4;
    const int slot_bytes = (int)C.slot_stride * EL;

    // a negative scale turns the queries' sign, so that the largest score is that of the largest product
    float scale = a.scale * (FP8 && C.k_scale ? C.k_scale[it.kv_head] : 1.f);
    const uint32_t turn = scale < 0.f ? 0x80008000u : 0u;
    scale = fabsf(scale);
    auto query = [&](int b, int s) __attribute__((always_inline)) {
        int i = 16 * b + c;
        i = it.first + (i < it.n ? i : 0);
        const int row = i / a.group, head = it.kv_head * a.group + (i - row * a.group);
        // the keys' pieces decide which elements a step has
        const int at = FP8 ? 64 * (s >> 1) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g;
        u32x4 x = *reinterpret_cast<const u32x4 *>(a.q + row * a.q_stride + (long long)head * D + at);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] ^= turn;
        return x;
    };
    u32x4 q[QUERIES_IN_LDS ? 1 : HB][QUERIES_IN_LDS ? 1 : QK];
    if constexpr (QUERIES_IN_LDS) {
#pragma unroll
        for (int b = 0; b < HB / WAVES; ++b)
#pragma unroll
            for (int s = 0; s < QK; ++s) lds_q[((b * WAVES + wave) * QK + s) * 64 + lane] = query(b * WAVES + wave, s);
        __syncthreads();
    } else {
#pragma unroll
        for (int b = 0; b < HB; ++b)
#pragma unroll
            for (int s = 0; s < QK; ++s) q[b][s] = query(b, s);
    }

    const int last = it.end - 1, last_block = last >> C.page_shift;
    scalar_ints table = (scalar_ints)(uintptr_t)it.table;
    auto read_pages = [&](int t0) __attribute__((always_inline)) {
        Pages p;
        p.there = 0;
        const int block = t0 >> C.page_shift;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            int entry;
            if (i > 0 && C.page_shift >= 5) {
                p.at[i] = p.at[0];
                p.there |= (p.there & 1u) << i;
                continue;
            }
            entry = table[block + i < last_block ? block + i : last_block];
            const bool ok = entry >= 0 && entry < C.n_pages;
            p.at[i] = ok ? entry * C.page_stride * EL : 0ll;
            p.there |= ok ? 1u << i : 0u;
        }
        return p;
    };
    auto page_of = [&](const Pages &p, int which) __attribute__((always_inline)) {
        long long at = which & 1 ? p.at[1] : p.at[0];
        const long long high = which & 1 ? p.at[3] : p.at[2];
        return which & 2 ? high : at;
    };
    // A tile in registers: pieces of the keys at t0 + c and t0 + 16 + c, of the values at t0 + 4 g .. + 3 and t0 + 16 + 4 g .. + 3 (a page
    // has whole quads of positions).  Positions past the end are read from the last one's place, quads from the last one's.
    struct Tile {
        u32x4 k[2][KB];
        uint32_t v[8][SEG][VR];
        uint32_t there;
    };
    const uint8_t *kbase = static_cast<const uint8_t *>(C.k) + it.kv_head * C.head_stride * EL + 16 * g;
    const uint8_t *vbase = static_cast<const uint8_t *>(C.v) + it.kv_head * C.head_stride * EL + W * EL * c;
    auto load = [&](Tile &t, const Pages &p, int t0) __attribute__((always_inline)) {
        const int block = t0 >> C.page_shift;
        t.there = p.there;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int pos = t0 + 16 * s + c, at = pos < last ? pos : last;
            const uint8_t *src = kbase + page_of(p, (at >> C.page_shift) - block) + (uint32_t)((at & C.page_mask) * slot_bytes);
#pragma unroll
            for (int j = 0; j < KB; ++j) t.k[s][j] = *reinterpret_cast<const u32x4 *>(src + 64 * j);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int pos = t0 + 16 * s + 4 * g, quad = last & ~3, at = pos < quad ? pos : quad;
            const uint8_t *src = vbase + page_of(p, (at >> C.page_shift) - block) + (uint32_t)((at & C.page_mask) * slot_bytes);
#pragma unroll
            for (int i = 0; i < 4; ++i, src += slot_bytes)
#pragma unroll
                for (int e = 0; e < SEG; ++e) {
                    uint32_t *v = t.v[4 * s + i][e];
                    if constexpr (VR == 4) {
                        const u32x4 x = *reinterpret_cast<const u32x4 *>(src + 128 * EL * e);
#pragma unroll
                        for (int r = 0; r < VR; ++r) v[r] = x[r];
                    } else if constexpr (VR == 2) {
                        const u32x2 x = *reinterpret_cast<const u32x2 *>(src + 128 * EL * e);
#pragma unroll
                        for (int r = 0; r < VR; ++r) v[r] = x[r];
                    } else {
                        v[0] = *reinterpret_cast<const uint32_t *>(src + 128 * EL * e);
                    }
                }
        }
    };

    float m[HB], l[HB];
    f32x4 acc[HB][SEG * W];
#pragma unroll
    for (int b = 0; b < HB; ++b) {
        m[b] = LOWEST;
        l[b] = 0.f;
#pragma unroll
        for (int e = 0; e < SEG * W; ++e) acc[b][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    auto step = [&](Tile &t, int t0) __attribute__((always_inline)) {
        const bool full = t0 >= it.lo && t0 + TILE <= it.end && t.there == 15u;
        auto seen = [&](int i) {
            const int pos = t0 + 16 * (i >> 2) + 4 * g + (i & 3);
            return pos >= it.lo && pos < it.end && (t.there >> ((pos >> C.page_shift) - (t0 >> C.page_shift) & 3) & 1u);
        };
        if (!full) {
            // what masked positions hold must not meet a weight of 0: NaN and infinities would stay
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool in = seen(i);
#pragma unroll
                for (int s = 0; s < SEG; ++s)
#pragma unroll
                    for (int r = 0; r < VR; ++r) t.v[i][s][r] = in ? t.v[i][s][r] : 0u;
            }
        }
        // the values' operands: element W (lane's row) + e of eight positions
        u32x4 vt[SEG][W];
#pragma unroll
        for (int s = 0; s < SEG; ++s)
#pragma unroll
            for (int r = 0; r < VR; ++r) {
                auto &v = t.v;
                if constexpr (FP8) {
                    // elements 4 r .. 4 r + 3: bytes of two positions next to each other, then to fp16
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t lo = __builtin_amdgcn_perm(v[2 * i + 1][s][r], v[2 * i][s][r], 0x05010400u);
                        const uint32_t hi = __builtin_amdgcn_perm(v[2 * i + 1][s][r], v[2 * i][s][r], 0x07030602u);
                        vt[s][4 * r][i] = fp8_f16<false>(lo);
                        vt[s][4 * r + 1][i] = fp8_f16<true>(lo);
                        vt[s][4 * r + 2][i] = fp8_f16<false>(hi);
                        vt[s][4 * r + 3][i] = fp8_f16<true>(hi);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        vt[s][2 * r][i] = __builtin_amdgcn_perm(v[2 * i + 1][s][r], v[2 * i][s][r], 0x05040100u);
                        vt[s][2 * r + 1][i] = __builtin_amdgcn_perm(v[2 * i + 1][s][r], v[2 * i][s][r], 0x07060302u);
                    }
                }
            }
        u32x4 key[2][QK];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int j = 0; j < QK; ++j) {
                if constexpr (FP8) {
                    const uint32_t lo = t.k[s][j >> 1][2 * (j & 1)], hi = t.k[s][j >> 1][2 * (j & 1) + 1];
                    key[s][j] = u32x4{fp8_bf16<false>(lo), fp8_bf16<true>(lo), fp8_bf16<false>(hi), fp8_bf16<true>(hi)};
                } else {
                    key[s][j] = t.k[s][j];
                }
            }
#pragma unroll
        for (int b = 0; b < HB; ++b) {
            f32x4 x[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
            for (int j = 0; j < QK; ++j) {
                u32x4 qj;
                if constexpr (QUERIES_IN_LDS) qj = lds_q[(b * QK + j) * 64 + lane];
                else qj = q[b][j];
#pragma unroll
                for (int s = 0; s < 2; ++s) x[s] = mfma_bf16(key[s][j], qj, x[s]);
            }
            float y[8], top = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                y[i] = x[i >> 2][i & 3];
                if (!full) y[i] = seen(i) ? y[i] : -__builtin_inff();
                top = fmaxf(top, y[i]);
            }
            // The reference follows the maximum only when that is 2^GROWTH past it, so that the sums are seldom carried over; weights are then up to
            // that, and as fp16 (relative to 2^6 below the maximum that was met) up to 2^14.
            constexpr float GROWTH = 8.f;
            top *= scale;
            if (__ballot(top > m[b] + (FP8 ? GROWTH + 6.f : GROWTH)) != 0) {
                top = across_groups(top, [](float x, float y) { return fmaxf(x, y); });
                if constexpr (FP8) top -= 6.f;
                const float mn = fmaxf(m[b], top), fall = __builtin_amdgcn_exp2f(m[b] - mn);
                m[b] = mn;
                l[b] *= fall;
#pragma unroll
                for (int e = 0; e < SEG * W; ++e) acc[b][e] *= fall;
            }
            float p[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                p[i] = __builtin_amdgcn_exp2f(fmaf(y[i], scale, -m[b]));
                if (!full) p[i] = seen(i) ? p[i] : 0.f;        // (a scale of 0 times -inf)
                l[b] += p[i];
            }
            if constexpr (FP8) {
                u32x4 w;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f16x2 h = {(_Float16)p[2 * i], (_Float16)p[2 * i + 1]};
                    w[i] = __builtin_bit_cast(uint32_t, h);
                }
#pragma unroll
                for (int s = 0; s < SEG; ++s)
#pragma unroll
                    for (int e = 0; e < W; ++e) acc[b][s * W + e] = mfma_f16(vt[s][e], w, acc[b][s * W + e]);
            } else {
                // Weights in two bf16 parts, 16 bits.  The first is cut, so that the second is not negative, and not 0: an infinite value then
                // gives infinities of one sign.
                u32x4 near, rest;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t p0 = __float_as_uint(p[2 * i]), p1 = __float_as_uint(p[2 * i + 1]);
                    near[i] = __builtin_amdgcn_perm(p1, p0, 0x07060302u);
                    rest[i] = pack_bf16x2(fmaxf(p[2 * i] - __uint_as_float(p0 & 0xFFFF0000u), 1.2e-38f),
                                          fmaxf(p[2 * i + 1] - __uint_as_float(p1 & 0xFFFF0000u), 1.2e-38f));
                }
#pragma unroll
                for (int s = 0; s < SEG; ++s)
#pragma unroll
                    for (int e = 0; e < W; ++e) {
                        acc[b][s * W + e] = mfma_bf16(vt[s][e], near, acc[b][s * W + e]);
                        acc[b][s * W + e] = mfma_bf16(vt[s][e], rest, acc[b][s * W + e]);
                    }
            }
        }
    };

    // Pages are known two tiles ahead, a tile is asked for one ahead.
    int t0 = it.begin + wave * TILE;
    if (t0 < it.end) {
        Tile x;
        Pages next = read_pages(t0);
        load(x, next, t0);
        if (t0 + STEP < it.end) next = read_pages(t0 + STEP);
        for (;;) {
            const bool more = t0 + STEP < it.end;
            if constexpr (AHEAD) {
                Tile y;
                if (more) {
                    load(y, next, t0 + STEP);
                    if (t0 + 2 * STEP < it.end) next = read_pages(t0 + 2 * STEP);
                }
                step(x, t0);
                x = y;
            } else {
                step(x, t0);
                if (more) {
                    load(x, next, t0 + STEP);
                    if (t0 + 2 * STEP < it.end) next = read_pages(t0 + 2 * STEP);
                }
            }
            if (!more) break;
            t0 += STEP;
        }
    }

    // The waves' sums: everything goes to LDS as it is, and every thread scales and adds four elements of a column.
    const float v_scale = FP8 && C.v_scale ? C.v_scale[it.kv_head] : 1.f;
#pragma unroll
    for (int b = 0; b < HB; ++b) {
        if (16 * b >= it.n) break;                             // (uniform)
        l[b] = across_groups(l[b], [](float x, float y) { return x + y; });
#pragma unroll
        for (int s = 0; s < SEG; ++s) {
            if (b + s > 0) __syncthreads();
            if (s == 0 && g == 0) { wave_m[wave][c] = m[b]; wave_l[wave][c] = l[b]; }
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int e = 0; e < W; e += 4) {
                    f32x4 x;
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = acc[b][s * W + e + i][r];
                    *reinterpret_cast<f32x4 *>(&joined[wave][c][W * (4 * g + r) + e]) = x;
                }
            __syncthreads();
            for (int u = threadIdx.x; u < 16 * DS / 4; u += 64 * WAVES) {
                const int col = u / (DS / 4), at = 4 * (u % (DS / 4));
                if (16 * b + col >= it.n) break;
                float top = LOWEST, total = 0.f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) top = fmaxf(top, wave_m[w][col]);
                f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < WAVES; ++w) {
                    const float by = __builtin_amdgcn_exp2f(wave_m[w][col] - top);
                    total += wave_l[w][col] * by;
                    x += *reinterpret_cast<const f32x4 *>(&joined[w][col][at]) * by;
                }
                const size_t place = (size_t)it.slot + 16 * b + col;
                *reinterpret_cast<f32x4 *>(a.part + place * D + 128 * s + at) = x * v_scale;
                if (at == 0 && s == 0) {
                    a.part_ml[2 * place] = top;
                    a.part_ml[2 * place + 1] = total;
                }
            }
        }
    }
}

// Workgroups of a unit: two, of one wave per SIMD each, with up to 256 registers a lane, or one with up to 512.
constexpr int wgs_per_unit(int D, int HB) { return HB * D <= 128 ? 2 : 1; }

template <int D, bool FP8, int HB>
__global__ __launch_bounds__(64 * WAVES, wgs_per_unit(D, HB)) void shared_kernel(SharedArgs a)
{
    __shared__ u32x4 lds_q[HB > 2 ? HB * (D / 32) * 64 : 1];
    __shared__ float wave_m[WAVES][16], wave_l[WAVES][16];
    __shared__ __attribute__((aligned(16))) float joined[WAVES][16][Shape<D>::DS + 4];
    const CacheArgs &C = a.cache;
    Item it;
    if ((int)blockIdx.x < a.prefix_wgs) {
        // The workgroups of a chunk that have different columns read the same positions: they are eight apart, on one XCD, at the same time.
        const int per = 8 * a.tiles, eight = (int)blockIdx.x / per, in = (int)blockIdx.x - eight * per, tile = in / 8, unit = 8 * eight + in - 8 * tile;
        if (unit >= a.chunks * C.kv_heads) return;
        const int chunk = unit / C.kv_heads;
        it.kv_head = unit - chunk * C.kv_heads;
        it.first = tile * a.columns;
        it.n = a.rows * a.group - it.first;
        it.n = it.n < a.columns ? it.n : a.columns;
        it.lo = it.begin = chunk * a.chunk;
        it.end = a.shared - it.begin < a.chunk ? a.shared : it.begin + a.chunk;
        it.table = C.table + a.prefix * C.table_stride;
        it.slot = ((long long)unit * a.tiles + tile) * a.columns;
        attend_item<D, FP8, HB>(a, it, lds_q, wave_m, wave_l, joined);
    } else {
        const int number = (int)blockIdx.x - a.prefix_wgs, item = number / a.own_splits, split = number - item * a.own_splits;
        const int of_row = item / a.own_blocks, block = item - of_row * a.own_blocks, row = of_row / C.kv_heads;
        RowInfo r = row_info(a, row);
        r.len = __builtin_amdgcn_readfirstlane(r.len);
        r.lo = __builtin_amdgcn_readfirstlane(r.lo);
        r.seq = __builtin_amdgcn_readfirstlane(r.seq);
        const OwnChunks o = own_chunks(a, r);
        if (split >= o.n) return;
        it.kv_head = of_row - row * C.kv_heads;
        it.first = row * a.group + block * a.own_columns;
        it.n = a.group - block * a.own_columns;
        it.n = it.n < a.own_columns ? it.n : a.own_columns;
        it.lo = r.lo;
        it.begin = o.from + split * o.length;
        it.end = r.len - it.begin < o.length ? r.len : it.begin + o.length;
        it.table = C.table + r.seq * C.table_stride;
        it.slot = (long long)a.chunks * C.kv_heads * a.tiles * a.columns + (long long)number * a.own_columns;
        attend_item<D, FP8, 1>(a, it, lds_q, wave_m, wave_l, joined);
    }
}

// Joins a column's parts: a workgroup per row and head.  A group of D / 4 lanes has some of the parts, 16 bytes of a part's sums a lane, four
// parts in flight; the groups' results meet in LDS.
template <int D> __global__ __launch_bounds__(256) void shared_join_kernel(SharedArgs a)
{
    constexpr int LANES = D / 4, GROUPS = 256 / LANES, FLIGHT = 4;
    __shared__ float group_m[GROUPS], group_l[GROUPS];
    __shared__ f32x4 sums[GROUPS][LANES];
    const CacheArgs &C = a.cache;
    const int row = (int)(blockIdx.x / (unsigned)a.heads), head = (int)(blockIdx.x - (unsigned)row * (unsigned)a.heads);
    const int kv_head = head / a.group, of_group = head - kv_head * a.group;
    const RowInfo r = row_info(a, row);
    const int shared = r.follows ? a.chunks : 0, n = shared + own_chunks(a, r).n;
    const int query = row * a.group + of_group, tile = query / a.columns, block = of_group / a.own_columns;
    const long long own0 = (long long)a.chunks * C.kv_heads * a.tiles * a.columns +
                           ((long long)(row * C.kv_heads + kv_head) * a.own_blocks + block) * a.own_splits * a.own_columns + (of_group - block * a.own_columns);
    const long long shared0 = ((long long)kv_head * a.tiles + tile) * a.columns + (query - tile * a.columns);
    const int at = threadIdx.x % LANES, group = threadIdx.x / LANES;
    float m = LOWEST, l = 0.f;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = group; s0 < n; s0 += FLIGHT * GROUPS) {
        f32x4 x[FLIGHT];
        float pm[FLIGHT], pl[FLIGHT], top = m;
#pragma unroll
        for (int k = 0; k < FLIGHT; ++k) {
            const int s = s0 + k * GROUPS < n ? s0 + k * GROUPS : s0;
            const size_t slot = (size_t)(s < shared ? shared0 + (long long)s * C.kv_heads * a.tiles * a.columns : own0 + (long long)(s - shared) * a.own_columns);
            x[k] = *reinterpret_cast<const f32x4 *>(a.part + slot * D + 4 * at);
            pm[k] = a.part_ml[2 * slot];
            pl[k] = a.part_ml[2 * slot + 1];
        }
#pragma unroll
        for (int k = 0; k < FLIGHT; ++k) top = fmaxf(top, pm[k]);
        const float fall = __builtin_amdgcn_exp2f(m - top);
        m = top;
        l *= fall;
        sum *= fall;
#pragma unroll
        for (int k = 0; k < FLIGHT; ++k) {
            if (s0 + k * GROUPS >= n) continue;
            const float by = __builtin_amdgcn_exp2f(pm[k] - top);
            l += pl[k] * by;
            sum += x[k] * by;
        }
    }
    sums[group][at] = sum;
    if (at == 0) { group_m[group] = m; group_l[group] = l; }
    __syncthreads();
    if (threadIdx.x >= LANES) return;
    float top = LOWEST, total = 0.f;
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) top = fmaxf(top, group_m[k]);
    sum = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) {
        const float by = __builtin_amdgcn_exp2f(group_m[k] - top);
        total += group_l[k] * by;
        sum += sums[k][at] * by;
    }
    const bool any = total > 0.f || total != total;
    const float by = any ? 1.f / total : 0.f;
    uint16_t *o = a.out + row * a.out_stride + (long long)head * D + 4 * at;
    *reinterpret_cast<u32x2 *>(o) = u32x2{pack_bf16x2(sum[0] * by, sum[1] * by), pack_bf16x2(sum[2] * by, sum[3] * by)};
    if (a.lse && at == 0) a.lse[(size_t)row * a.heads + head] = any ? (top + __builtin_amdgcn_logf(total)) * LN2 : -__builtin_inff();
}

// How a call is cut.
struct SharedPlan {
    int hb, columns, tiles, chunk, chunks, own_chunk, own_splits, own_blocks, own_columns;
    long long prefix_wgs, own_wgs;
    size_t part_bytes, ml_bytes;
};

SharedPlan shared_plan(const peqa_kv_cache *C, int rows, int heads, int max_len, int shared)
{
    SharedPlan p{};
    const int group = heads / C->kv_heads;
    if (max_len < shared) shared = 0;                          // (every row ends among the shared positions, and has them by itself)
    const long long queries = (long long)rows * group;
    const int most = 512 / C->head_dim;                        // (as many as there are registers for)
    p.hb = 1;
    while (p.hb < most && 16 * p.hb < queries) p.hb *= 2;
    p.columns = 16 * p.hb;
    p.tiles = (int)((queries + p.columns - 1) / p.columns);
    p.own_columns = group < 16 ? group : 16;
    p.own_blocks = (group + p.own_columns - 1) / p.own_columns;
    const long long own = max_len > shared ? max_len - shared + TILE - 1 : 0;
    const long long items = (long long)rows * C->kv_heads * p.own_blocks, units = (long long)C->kv_heads * p.tiles;
    // all that there is to walk, over as many workgroups as have room at once, 128 positions at least
    const int wgs = PLAN_UNITS * wgs_per_unit(C->head_dim, p.hb);
    const long long all = units * shared + items * own;
    long long chunk = (all + wgs - 1) / wgs;
    chunk = (chunk + STEP - 1) / STEP * STEP;
    if (chunk < STEP) chunk = STEP;
    p.chunks = (int)((shared + chunk - 1) / chunk);
    p.chunk = p.chunks > 0 ? (int)(((shared + p.chunks - 1) / p.chunks + TILE - 1) / TILE * TILE) : TILE;
    p.chunks = (shared + p.chunk - 1) / p.chunk;
    p.own_splits = (int)((own + chunk - 1) / chunk);
    if (p.own_splits < 1) p.own_splits = 1;                    // (rows that end among the shared positions)
    p.own_chunk = STEP;
    p.prefix_wgs = ((long long)p.chunks * C->kv_heads + 7) / 8 * 8 * p.tiles;
    p.own_wgs = items * p.own_splits;
    const size_t slots = (size_t)p.chunks * (size_t)units * (size_t)p.columns + (size_t)p.own_wgs * (size_t)p.own_columns;
    p.part_bytes = round256(slots * (size_t)C->head_dim * sizeof(float));
    p.ml_bytes = round256(slots * 2 * sizeof(float));
    return p;
}

template <int D, bool FP8> hipError_t launch_shared(const SharedArgs &a, const SharedPlan &p, hipStream_t stream)
{
    auto kernel = p.hb == 1 ? shared_kernel<D, FP8, 1> : shared_kernel<D, FP8, 2>;
    if constexpr (D <= 128)
        if (p.hb == 4) kernel = shared_kernel<D, FP8, 4>;
    if constexpr (D <= 64)
        if (p.hb == 8) kernel = shared_kernel<D, FP8, 8>;
    trace_before(KID_SHARED, stream);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(p.prefix_wgs + p.own_wgs)), dim3(64 * WAVES), 0, stream, a);
    trace_after(KID_SHARED, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    trace_before(KID_SHARED_JOIN, stream);
    hipLaunchKernelGGL(shared_join_kernel<D>, dim3((unsigned)a.rows * (unsigned)a.heads), dim3(256), 0, stream, a);
    trace_after(KID_SHARED_JOIN, stream);
    return hipGetLastError();
}

peqa_status check_shared(const peqa_kv_cache *C, int32_t rows, int32_t heads, int32_t max_len, int32_t shared)
{
    const peqa_status st = peqa_check_cache(C);
    if (st != PEQA_OK) return st;
    if (rows < 1 || heads < 1 || heads > 65536 || heads % C->kv_heads || max_len < 0 || shared < 0) return PEQA_ERR_SHAPE;
    const int64_t room = (int64_t)C->n_blocks * C->page_size;
    if (max_len > room || shared > room) return PEQA_ERR_SHAPE;
    if ((int64_t)rows * heads > (1 << 23)) return PEQA_ERR_SHAPE;             // workgroups of a launch
    const SharedPlan p = shared_plan(C, rows, heads, max_len, shared);
    if (p.prefix_wgs + p.own_wgs > (1 << 23)) return PEQA_ERR_SHAPE;
    return PEQA_OK;
}

}  // namespace
}  // namespace peqa

extern "C" {

size_t peqa_shared_attention_workspace_bytes(const peqa_kv_cache *C, int32_t rows, int32_t heads, int32_t max_len, int32_t shared)
{
    if (peqa::check_shared(C, rows, heads, max_len, shared) != PEQA_OK) return 0;
    const peqa::SharedPlan p = peqa::shared_plan(C, rows, heads, max_len, shared);
    return p.part_bytes + p.ml_bytes;
}

peqa_status peqa_shared_attention(const peqa_kv_cache *C, int32_t rows, int32_t heads, const uint16_t *q, int64_t q_stride, const int32_t *lens,
                                  const int32_t *seq, int32_t max_len, int32_t prefix, int32_t shared, float scale, uint16_t *out,
                                  int64_t out_stride, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    const peqa_status st = peqa::check_shared(C, rows, heads, max_len, shared);
    if (st != PEQA_OK) return st;
    if (!q || !lens || !out) return PEQA_ERR_NULL;
    if ((!seq && rows > C->n_seqs) || prefix < 0 || prefix >= C->n_seqs) return PEQA_ERR_SHAPE;
    const int64_t width = (int64_t)heads * C->head_dim;
    if (q_stride < width || out_stride < width) return PEQA_ERR_SHAPE;
    if (!aligned16(q) || !aligned16(out) || q_stride % 8 || out_stride % 8) return PEQA_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(lens) | reinterpret_cast<uintptr_t>(seq) | reinterpret_cast<uintptr_t>(lse)) & 3) return PEQA_ERR_ALIGN;
    const peqa::SharedPlan p = peqa::shared_plan(C, rows, heads, max_len, shared);
    if (!workspace || workspace_bytes < p.part_bytes + p.ml_bytes) return PEQA_ERR_WORKSPACE;
    if (!aligned16(workspace)) return PEQA_ERR_ALIGN;
    peqa::SharedArgs a{};
    a.cache = peqa::cache_args(C);
    a.q = q; a.lens = lens; a.seq = seq; a.out = out; a.lse = lse;
    a.part = static_cast<float *>(workspace);
    a.part_ml = reinterpret_cast<float *>(static_cast<char *>(workspace) + p.part_bytes);
    a.q_stride = q_stride; a.out_stride = out_stride;
    a.scale = scale * peqa::LOG2E;
    a.rows = rows; a.heads = heads; a.group = heads / C->kv_heads;
    a.max_len = max_len; a.prefix = prefix; a.shared = shared;
    a.columns = p.columns; a.tiles = p.tiles; a.chunk = p.chunk; a.chunks = p.chunks;
    a.prefix_wgs = (int)p.prefix_wgs;
    a.own_chunk = p.own_chunk; a.own_splits = p.own_splits; a.own_blocks = p.own_blocks; a.own_columns = p.own_columns;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool fp8 = C->dtype == PEQA_CACHE_FP8;
    hipError_t e;
    switch (C->head_dim) {
    case 64: e = fp8 ? peqa::launch_shared<64, true>(a, p, s) : peqa::launch_shared<64, false>(a, p, s); break;
    case 128: e = fp8 ? peqa::launch_shared<128, true>(a, p, s) : peqa::launch_shared<128, false>(a, p, s); break;
    default: e = fp8 ? peqa::launch_shared<256, true>(a, p, s) : peqa::launch_shared<256, false>(a, p, s); break;
    }
    return dev_status(e);
}

}  // extern "C"
