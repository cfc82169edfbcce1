// Attention of single query tokens whose sequences begin with the same positions (peqa_shared_attention): those are read once for all rows.
//
// For a key head the queries of all rows and of the heads that share it are the columns of one product with the shared positions; what
// a row has of its own is a product with its heads alone:
//   x[j][c] = scale <k_j, q_c>;   m_c = max_j x[j][c];   l_c = sum_j e^(x[j][c] - m_c);   o_c = sum_j e^(x[j][c] - m_c) v_j
// Both are cut into chunks of positions, a workgroup each, in one launch, and every column's parts (m, l, o) are joined by a second one: with
// M = max m, out = sum e^(m - M) o / sum e^(m - M) l.  The products and their operands are those of the paged attention (scores as keys x
// queries, whose result is the weights' operand of values^T x weights as it stands; values are turned 8 x 8 in registers).
//
// Up to 64 columns (32 of heads of 256) are in every wave: four waves take tiles of 32 positions in turn, and a key or a value that is loaded is used
// for every column without passing through LDS.  More have waves of their own, 16 or 32 each of eight, and keys and values come to LDS once,
// as operands, for all of them.
//
// Bound by memory where columns are few: 3 rows x 32 heads behind 555 positions 5.2 us and the join 3.5, launches and loads after one another;  16
// rows x 32 heads behind 2048 with up to 512 of their own 20.4 us, 4.8 TB/s of the cache.  Where they are many, by three things that overlap in part and
// are about 1000 cycles each for a tile of 32 positions and 256 columns, of the 2800 that it takes: matrix instructions, vector instructions of the softmax and
// of the operands, and the operands' way out of LDS, 16 KB for each of eight waves.  65537 positions of 8 bits, 8 key heads, 256 columns
// 94.5 us, 0.73 PFLOP/s; more columns a wave than 32, which would halve the last, do not fit its registers.  Heads of 256 have no such form: every 32
// columns walk the shared positions anew (32 rows x 4 key heads x 8 behind 8000: 52 us, 8 bits 38).  A row that ends among the shared positions
// has them to itself, in as many workgroups as the rows' own positions are given: one where those are few (32 rows x 64 heads behind 65536 with 333 of
// their own, one of them 65535 long: 672 us for 146, 8 bits 360 for 100).
#include "peqa_attend.h"
#include "peqa_cache.h"
#include "peqa_host.h"

using namespace peqa::host;

namespace peqa {

// How a call is cut.
struct SharedPlan {
    bool wide;
    int hb, columns, tiles, chunk, chunks, own_chunk, own_splits, own_blocks, own_columns, join_each;
    long long prefix_wgs, own_items;
    size_t part_bytes, ml_bytes;
};
SharedPlan shared_plan(const peqa_kv_cache *C, int rows, int heads, int max_len, int shared);

namespace {

constexpr int TILE = 32;       // positions of a wave's step
constexpr int UNIT = 128;      // that chunks are counted in

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
    int prefix_wgs, own_items;
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
    o.length = ((span + a.own_splits - 1) / a.own_splits + UNIT - 1) & ~(UNIT - 1);
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

typedef const __attribute__((address_space(4))) int32_t *scalar_ints;

// The pages of a tile of 32 positions: four at most, neighbouring entries of the table.  They are read (scalar loads) a step before they
// are used, the last one of the positions up to `last` again past its end.
struct Entries {
    int page[4];
};
__device__ __forceinline__ Entries read_entries(const CacheArgs &C, const int32_t *row, int last, int t0)
{
    scalar_ints table = (scalar_ints)(uintptr_t)row;
    const int block = t0 >> C.page_shift, last_block = last >> C.page_shift, next = C.page_shift < 5 ? 1 : 0;
    Entries e;
#pragma unroll
    for (int i = 0; i < 4; ++i) e.page[i] = table[block + i * next < last_block ? block + i * next : last_block];
    return e;
}
struct Pages {
    long long at[4];           // in bytes
    uint32_t there;            // bit i: the page is there
};
__device__ __forceinline__ Pages pages_of(const CacheArgs &C, const Entries &e, int el)
{
    Pages p;
    p.there = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool ok = (unsigned)e.page[i] < (unsigned)C.n_pages;
        p.at[i] = (ok ? e.page[i] : 0) * C.page_stride * el;
        p.there |= (ok ? 1u : 0u) << i;
    }
    return p;
}
__device__ __forceinline__ long long page_of(const Pages &p, int which)
{
    const long long low = which & 1 ? p.at[1] : p.at[0], high = which & 1 ? p.at[3] : p.at[2];
    return which & 2 ? high : low;
}
// Where a position of a tile is: the last one's place past the end.
__device__ __forceinline__ long long place_of(const CacheArgs &C, const Pages &p, int t0, int pos, int last, int slot_bytes)
{
    const int at = pos < last ? pos : last;
    return page_of(p, (at >> C.page_shift) - (t0 >> C.page_shift)) + (uint32_t)((at & C.page_mask) * slot_bytes);
}
// Whether a position of the tile at t0 is in [lo, end) and its page there.
__device__ __forceinline__ bool seen_at(const CacheArgs &C, uint32_t there, int t0, int pos, int lo, int end)
{
    return pos >= lo && pos < end && (there >> ((pos >> C.page_shift) - (t0 >> C.page_shift) & 3) & 1u);
}
// What the scores' sums begin with: 0, or of positions that are not seen -inf.  (Score i of a lane is of position t0 + 16 (i / 4) + 4 g + i % 4.)
struct Start {
    f32x4 x[2];
};
__device__ __forceinline__ Start start_of(const CacheArgs &C, uint32_t there, int t0, int g, int lo, int end)
{
    Start s;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        s.x[i >> 2][i & 3] = seen_at(C, there, t0, t0 + 16 * (i >> 2) + 4 * g + (i & 3), lo, end) ? 0.f : -__builtin_inff();
    return s;
}

// Values of eight positions, 2 VR or 4 VR elements each (bf16; 8 bits), turned: operand e has element e of all eight, 8-bit ones as fp16 (exact).
template <bool FP8, int VR> __device__ __forceinline__ void turn_values(const uint32_t (&v)[8][VR], u32x4 *vt)
{
#pragma unroll
    for (int r = 0; r < VR; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (FP8) {
                // bytes of two positions next to each other, then to fp16
                const uint32_t lo = __builtin_amdgcn_perm(v[2 * i + 1][r], v[2 * i][r], 0x05010400u);
                const uint32_t hi = __builtin_amdgcn_perm(v[2 * i + 1][r], v[2 * i][r], 0x07030602u);
                vt[4 * r][i] = fp8_f16<false>(lo);
                vt[4 * r + 1][i] = fp8_f16<true>(lo);
                vt[4 * r + 2][i] = fp8_f16<false>(hi);
                vt[4 * r + 3][i] = fp8_f16<true>(hi);
            } else {
                vt[2 * r][i] = __builtin_amdgcn_perm(v[2 * i + 1][r], v[2 * i][r], 0x05040100u);
                vt[2 * r + 1][i] = __builtin_amdgcn_perm(v[2 * i + 1][r], v[2 * i][r], 0x07060302u);
            }
        }
}

// Weights of 8 positions and a column as operands: bf16 in two parts, fp16 in one.  (A second fp16 part, 22 bits for 11, is as many matrix instructions again as
// the values have: 65537 positions of 8 bits, 256 columns 118.3 us for 93.9, 8192 of heads of 64 31.5 for 26.5, 40000 and 64 columns 29.4 for 27.5.  Values of
// 8 bits are off by 2^-4 themselves, and a weight's 2^-12 is of any sign.)
template <bool FP8> struct Weights {
    u32x4 near, rest;
};
// The reference of a column follows the maximum of its scores only when that is 2^GROWTH past it, so that the sums are seldom carried over; weights are
// then up to that, and as fp16 (relative to 2^6 below the maximum that was met) up to 2^14.  x: a lane's eight scores, to be multiplied with
// scale > 0; m, l and acc: the reference, the lane's sum of weights, and what is carried over.
// A weight is 2 to the power of x scale - m in one operation, which does not round the product, as the reference is: by half of its last place, 32 of
// 2^29, and that would be in the weight's exponent.  Where one of a wave's references reaches FAR, every tile comes here, its scores become what
// their rounded products are past the reference, never more than 8, and stand for themselves: x scale less 0.  (Equal scores before and
// behind that point differ by what rounding one of FAR is, 2^-12 of a weight.)  Returned: what weights are relative to.
// limit: what a score must pass to come here.  (It takes a register for the addition that it saves: heads of 256, bf16, 32 columns, 20000 positions 29.7 us, 28.0
// without, 65537 of 8 bits, 256 columns 93.2 and 92.9.  A flag beside the addition: 28.7 and 96.2.)
template <bool FP8, int ACC> __device__ __forceinline__ float follow(f32x4 (&x)[2], float scale, float &m, float &l, float &limit, f32x4 (&acc)[ACC])
{
    constexpr float GROWTH = FP8 ? 14.f : 8.f, FAR = 4096.f;
    float top = x[0][0], from = m;
#pragma unroll
    for (int i = 1; i < 8; ++i) top = fmaxf(top, x[i >> 2][i & 3]);
    top *= scale;
    if (__ballot(top > limit) != 0) {
        top = across_groups(top, [](float x, float y) { return fmaxf(x, y); });
        if constexpr (FP8) top -= 6.f;
        const float mn = fmaxf(m, top), fall = __builtin_amdgcn_exp2f(m - mn);
        m = from = mn;
        l *= fall;
#pragma unroll
        for (int e = 0; e < ACC; ++e) acc[e] *= fall;
        limit = m + GROWTH;
        if (__builtin_expect(__ballot(fabsf(m) >= FAR && m > LOWEST) != 0, 0)) {
#pragma clang fp contract(off)
            const float back = 1.f / scale;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float y = x[i >> 2][i & 3] * scale;
                x[i >> 2][i & 3] = (y - m) * back;
            }
            from = 0.f;
            limit = -__builtin_inff();
        }
    }
    return from;
}
// The weights of eight scores; their sum is added to l.
struct Eights {
    float p[8];
};
__device__ __forceinline__ Eights powers(const f32x4 (&x)[2], float scale, float m, float &l)
{
    Eights e;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        e.p[i] = __builtin_amdgcn_exp2f(fmaf(x[i >> 2][i & 3], scale, -m));
        l += e.p[i];
    }
    return e;
}
// As operands.  Two bf16 parts have 16 bits: the first is cut, so that the second is not negative, and not 0: an infinite value then gives
// infinities of one sign, and a finite one of 10^34 counts for 10^-4 at least.
template <bool FP8> __device__ __forceinline__ Weights<FP8> operands(const Eights &e)
{
    const auto &p = e.p;
    Weights<FP8> w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (FP8) {
            const f16x2 h = {(_Float16)p[2 * i], (_Float16)p[2 * i + 1]};
            w.near[i] = __builtin_bit_cast(uint32_t, h);
        } else {
            const uint32_t p0 = __float_as_uint(p[2 * i]), p1 = __float_as_uint(p[2 * i + 1]);
            w.near[i] = __builtin_amdgcn_perm(p1, p0, 0x07060302u);
            w.rest[i] = pack_bf16x2(fmaxf(p[2 * i] - __uint_as_float(p0 & 0xFFFF0000u), 1.2e-38f),
                                    fmaxf(p[2 * i + 1] - __uint_as_float(p1 & 0xFFFF0000u), 1.2e-38f));
        }
    }
    return w;
}
// acc[e] += values' operand e x weights, for COUNT operands: no two neighbouring instructions add to the same sums.
template <bool FP8, int COUNT> __device__ __forceinline__ void add_weighted(const u32x4 *vt, const Weights<FP8> &w, f32x4 *acc)
{
#pragma unroll
    for (int e = 0; e < COUNT; ++e) acc[e] = FP8 ? mfma_f16(vt[e], w.near, acc[e]) : mfma_bf16(vt[e], w.near, acc[e]);
    if constexpr (!FP8) {
#pragma unroll
        for (int e = 0; e < COUNT; ++e) acc[e] = mfma_bf16(vt[e], w.rest, acc[e]);
    }
}

// What the products of a key head's queries and keys are multiplied with, made positive: a negative one turns the queries' signs, so that the largest
// score is that of the largest product, and for 0 a number stands that no product makes anything of (and -inf stays).
template <bool FP8> __device__ __forceinline__ float scale_of(const SharedArgs &a, int kv_head, uint32_t &turn)
{
    const float scale = a.scale * (FP8 && a.cache.k_scale ? a.cache.k_scale[kv_head] : 1.f);
    turn = scale < 0.f ? 0x80008000u : 0u;
    const float size = fabsf(scale);
    return size < 1e-36f ? 1e-36f : size;                      // (NaN stays)
}

// A piece of the query of a column: 16 bytes of step s of the scores' product, whose elements the keys' pieces decide.
template <int D, bool FP8> __device__ __forceinline__ u32x4 query_piece(const SharedArgs &a, const Item &it, int column, int s, int g, uint32_t turn)
{
    const int i = it.first + (column < it.n ? column : 0);
    const int row = i / a.group, head = it.kv_head * a.group + (i - row * a.group);
    const int at = FP8 ? 64 * (s >> 1) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g;
    u32x4 x = *reinterpret_cast<const u32x4 *>(a.q + row * a.q_stride + (long long)head * D + at);
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] ^= turn;
    return x;
}
// Eight elements of a key for step j, of the pieces that were loaded.
template <bool FP8, int KB> __device__ __forceinline__ u32x4 key_piece(const u32x4 (&k)[KB], int j)
{
    if constexpr (FP8) {
        const uint32_t lo = k[j >> 1][2 * (j & 1)], hi = k[j >> 1][2 * (j & 1) + 1];
        return u32x4{fp8_bf16<false>(lo), fp8_bf16<true>(lo), fp8_bf16<false>(hi), fp8_bf16<true>(hi)};
    } else {
        return k[j];
    }
}
// VR registers from memory.
template <int VR> __device__ __forceinline__ void load_value(const uint8_t *src, uint32_t (&v)[VR])
{
    if constexpr (VR == 4) {
        const u32x4 x = *reinterpret_cast<const u32x4 *>(src);
#pragma unroll
        for (int r = 0; r < VR; ++r) v[r] = x[r];
    } else if constexpr (VR == 2) {
        const u32x2 x = *reinterpret_cast<const u32x2 *>(src);
#pragma unroll
        for (int r = 0; r < VR; ++r) v[r] = x[r];
    } else {
        v[0] = *reinterpret_cast<const uint32_t *>(src);
    }
}

template <int D> struct Shape {
    static constexpr int SEG = D > 128 ? D / 128 : 1, DS = D / SEG;
};

// All columns in every wave, which take the tiles in turn.
template <int D, bool FP8, int HB, int WAVES>
__device__ __forceinline__ void attend_item(const SharedArgs &a, const Item &it, int tid, u32x4 *lds_q, float (*wave_m)[16], float (*wave_l)[16],
                                            float (*joined)[16][Shape<D>::DS + 4])
{
    constexpr int STEP = TILE * WAVES;                // positions of a workgroup's step
    constexpr int QK = D / 32;                        // steps of the scores' product
    constexpr int SEG = Shape<D>::SEG, DS = Shape<D>::DS;
    constexpr int W = D / 16 / SEG;                   // neighbouring elements of a segment that a lane has: 4 or 8
    constexpr int KB = FP8 ? D / 64 : D / 32;         // 16-byte pieces of a key that a lane loads
    constexpr int VR = FP8 ? W / 4 : W / 2;           // registers of a value's segment
    constexpr int EL = FP8 ? 1 : 2;
    constexpr bool QUERIES_IN_LDS = HB > 2;
    constexpr bool AHEAD = HB * D < 512 || (FP8 && D <= 128);       // registers for two tiles
    const CacheArgs &C = a.cache;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;
    const int slot_bytes = (int)C.slot_stride * EL;

    uint32_t turn;
    const float scale = scale_of<FP8>(a, it.kv_head, turn);
    u32x4 q[QUERIES_IN_LDS ? 1 : HB][QUERIES_IN_LDS ? 1 : QK];
    if constexpr (QUERIES_IN_LDS) {
#pragma unroll
        for (int b = 0; b < HB / WAVES; ++b)
#pragma unroll
            for (int s = 0; s < QK; ++s)
                lds_q[((b * WAVES + wave) * QK + s) * 64 + lane] = query_piece<D, FP8>(a, it, 16 * (b * WAVES + wave) + c, s, g, turn);
        __syncthreads();
    } else {
#pragma unroll
        for (int b = 0; b < HB; ++b)
#pragma unroll
            for (int s = 0; s < QK; ++s) q[b][s] = query_piece<D, FP8>(a, it, 16 * b + c, s, g, turn);
    }

    const int last = it.end - 1;
    // A tile in registers: pieces of the keys at t0 + c and t0 + 16 + c, of the values at t0 + 4 g .. + 3 and t0 + 16 + 4 g .. + 3 (a page
    // has whole quads of positions).  Positions past the end are read from the last one's place, quads from the last one's.
    struct Tile {
        u32x4 k[2][KB];
        uint32_t v[SEG][8][VR];
        uint32_t there;
    };
    const uint8_t *kbase = static_cast<const uint8_t *>(C.k) + it.kv_head * C.head_stride * EL + 16 * g;
    const uint8_t *vbase = static_cast<const uint8_t *>(C.v) + it.kv_head * C.head_stride * EL + W * EL * c;
    auto entries_at = [&](int t0) __attribute__((always_inline)) { return read_entries(C, it.table, last, t0); };
    auto load = [&](Tile &t, const Entries &e, int t0) __attribute__((always_inline)) {
        const Pages p = pages_of(C, e, EL);
        t.there = p.there;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const uint8_t *src = kbase + place_of(C, p, t0, t0 + 16 * s + c, last, slot_bytes);
#pragma unroll
            for (int j = 0; j < KB; ++j) t.k[s][j] = *reinterpret_cast<const u32x4 *>(src + 64 * j);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const uint8_t *src = vbase + place_of(C, p, t0, t0 + 16 * s + 4 * g, last & ~3, slot_bytes);
#pragma unroll
            for (int i = 0; i < 4; ++i, src += slot_bytes)
#pragma unroll
                for (int e = 0; e < SEG; ++e) load_value<VR>(src + 128 * EL * e, t.v[e][4 * s + i]);
        }
    };

    float m[HB], l[HB], limit[HB];
    f32x4 acc[HB][SEG * W];
#pragma unroll
    for (int b = 0; b < HB; ++b) {
        m[b] = limit[b] = LOWEST;
        l[b] = 0.f;
#pragma unroll
        for (int e = 0; e < SEG * W; ++e) acc[b][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    auto step = [&](Tile &t, int t0) __attribute__((always_inline)) {
        Start start{};
        if (!(t0 >= it.lo && t0 + TILE <= it.end && t.there == 15u)) {
            // what positions that are not seen hold must not meet a 0 or -inf: NaN and infinities would stay
            start = start_of(C, t.there, t0, g, it.lo, it.end);
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const bool in = seen_at(C, t.there, t0, t0 + 16 * s + c, it.lo, it.end);
#pragma unroll
                for (int j = 0; j < KB; ++j) t.k[s][j] = in ? t.k[s][j] : u32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool in = seen_at(C, t.there, t0, t0 + 16 * (i >> 2) + 4 * g + (i & 3), it.lo, it.end);
#pragma unroll
                for (int s = 0; s < SEG; ++s)
#pragma unroll
                    for (int r = 0; r < VR; ++r) t.v[s][i][r] = in ? t.v[s][i][r] : 0u;
            }
        }
        u32x4 vt[SEG * W], key[2][QK];                         // (element W (lane's row) + e of eight positions)
#pragma unroll
        for (int s = 0; s < SEG; ++s) turn_values<FP8, VR>(t.v[s], vt + s * W);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int j = 0; j < QK; ++j) key[s][j] = key_piece<FP8, KB>(t.k[s], j);
#pragma unroll
        for (int b = 0; b < HB; ++b) {
            f32x4 x[2] = {start.x[0], start.x[1]};
#pragma unroll
            for (int j = 0; j < QK; ++j) {
                u32x4 qj;
                if constexpr (QUERIES_IN_LDS) qj = lds_q[(b * QK + j) * 64 + lane];
                else qj = q[b][j];
#pragma unroll
                for (int s = 0; s < 2; ++s) x[s] = mfma_bf16(key[s][j], qj, x[s]);
            }
            const float from = follow<FP8>(x, scale, m[b], l[b], limit[b], acc[b]);
            add_weighted<FP8, SEG * W>(vt, operands<FP8>(powers(x, scale, from, l[b])), acc[b]);
        }
    };
    // Pages are known two tiles ahead, a tile is asked for one ahead.
    int t0 = it.begin + wave * TILE;
    if (t0 < it.end) {
        Tile x;
        Entries next = entries_at(t0);
        load(x, next, t0);
        if (t0 + STEP < it.end) next = entries_at(t0 + STEP);
        for (;;) {
            const bool more = t0 + STEP < it.end;
            if constexpr (AHEAD) {
                Tile y;
                if (more) {
                    load(y, next, t0 + STEP);
                    if (t0 + 2 * STEP < it.end) next = entries_at(t0 + 2 * STEP);
                }
                step(x, t0);
                x = y;
            } else {
                step(x, t0);
                if (more) {
                    load(x, next, t0 + STEP);
                    if (t0 + 2 * STEP < it.end) next = entries_at(t0 + 2 * STEP);
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
            for (int u = tid; u < 16 * DS / 4; u += 64 * WAVES) {
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

// Columns of their own for every wave, HB blocks of 16: keys and values come to LDS once, as operands, 64 positions (a stage) at a time, those of
// the next two stages on their way to registers meanwhile.  Of a tile of 32 two waves bring keys (KEYS), two turn values (where they have two
// registers each at least).
template <int D, bool FP8, int HB, bool KEYS>
__device__ __forceinline__ void attend_columns(const SharedArgs &a, const Item &it, u32x4 *lds, uint32_t (*there)[2])
{
    constexpr int QK = D / 32, W = D / 16, KB = FP8 ? D / 64 : D / 32, VR = FP8 ? W / 4 : W / 2, EL = FP8 ? 1 : 2;
    constexpr int SUB = 2, STEP = TILE * SUB;         // tiles of a stage
    constexpr int FRAGS = 2 * QK + W;                 // operands of a tile: of the keys, then of the values
    // Registers, and neighbouring elements, of a value that a lane of a wave turns; waves for it, each with a half of the elements (whole lines of
    // memory: 150 us -> 136 of 65537 positions, 8 key heads, 256 columns, where both waves had 8 bytes of every 16).  Operand e of the values has
    // element e / WH * D / HALVES + WH * row + e % WH.
    constexpr int VH = VR > 1 ? VR / 2 : 1, WH = VH * (FP8 ? 4 : 2), HALVES = W / WH;
    const CacheArgs &C = a.cache;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, g = lane >> 4;
    const int slot_bytes = (int)C.slot_stride * EL, last = it.end - 1;
    uint32_t turn;
    const float scale = scale_of<FP8>(a, it.kv_head, turn);
    const bool idle = !KEYS && VR == 1 && (wave & 1);
    const int sub = wave >> 1 & 1, half = wave & 1;   // tile of a stage; which keys, or elements, of it
    const uint8_t *pool = static_cast<const uint8_t *>(KEYS ? C.k : C.v) + it.kv_head * C.head_stride * EL;
    const int in_head = KEYS ? 16 * g : (WH * c + (idle ? 0 : half * (D / HALVES))) * EL;
    const uint8_t *base = pool + in_head;
    const uint32_t lane_at = (uint32_t)((KEYS ? 16 * half + c : 4 * g) * slot_bytes + in_head);       // in a page of 32 positions or more
    // This wave's tile of a stage; past the last one, that again (as many loads in every stage: what is waited for is counted).
    auto tile_at = [&](int t0) __attribute__((always_inline)) {
        const int t = t0 + TILE * sub, most = it.begin + ((last - it.begin) & ~(TILE - 1));
        return t < most ? t : most;
    };
    Entries next;
    auto entries_at = [&](int t0) __attribute__((always_inline)) { next = read_entries(C, it.table, last, tile_at(t0)); };
    struct Raw {
        uint32_t r[8][2];                             // pieces of a key, or VH registers of eight values
        uint32_t there;
    };
    Raw raw[2];                                       // of the stages after this one, by their number's last bit
    static_assert(KB * 4 <= 16 && VH <= 2);
    auto fetch = [&](Raw &raw, int t0) __attribute__((always_inline)) {
        const int t = tile_at(t0);
        const Pages pages = pages_of(C, next, EL);
        raw.there = pages.there;
        if (C.page_shift >= 5 && t + TILE <= it.end) {
            // of one page, all of it: what differs between lanes stays as it is
            const uint8_t *src = pool + pages.at[0] + (uint32_t)((t & C.page_mask) * slot_bytes);
            if constexpr (KEYS) {
#pragma unroll
                for (int j = 0; j < KB; ++j) {
                    const u32x4 k = *reinterpret_cast<const u32x4 *>(src + 64 * j + lane_at);
#pragma unroll
                    for (int r = 0; r < 4; ++r) raw.r[2 * j + (r >> 1)][r & 1] = k[r];
                }
            } else {
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t v[VH];
                        load_value<VH>(src + (uint32_t)((16 * s + i) * slot_bytes) + lane_at, v);
#pragma unroll
                        for (int r = 0; r < VH; ++r) raw.r[4 * s + i][r] = v[r];
                    }
            }
        } else if constexpr (KEYS) {
            const uint8_t *src = base + place_of(C, pages, t, t + 16 * half + c, last, slot_bytes);
#pragma unroll
            for (int j = 0; j < KB; ++j) {
                const u32x4 k = *reinterpret_cast<const u32x4 *>(src + 64 * j);
#pragma unroll
                for (int r = 0; r < 4; ++r) raw.r[2 * j + (r >> 1)][r & 1] = k[r];
            }
        } else {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const uint8_t *src = base + place_of(C, pages, t, t + 16 * s + 4 * g, last & ~3, slot_bytes);
#pragma unroll
                for (int i = 0; i < 4; ++i, src += slot_bytes) {
                    uint32_t v[VH];
                    load_value<VH>(src, v);
#pragma unroll
                    for (int r = 0; r < VH; ++r) raw.r[4 * s + i][r] = v[r];
                }
            }
        }
    };
    auto keep = [&](Raw &raw, int buffer, int t0) __attribute__((always_inline)) {
        const int t = t0 + TILE * sub;
        if (t >= it.end || idle) return;
        u32x4 *to = lds + ((buffer * SUB + sub) * FRAGS) * 64 + lane;
        constexpr int USED = KEYS ? 2 * KB : 8;
        if (t + TILE > it.end || raw.there != 15u) {
            // what positions that are not seen hold must not meet a 0 or -inf: NaN and infinities would stay
            const bool key_in = seen_at(C, raw.there, t, t + 16 * half + c, it.lo, it.end);
#pragma unroll
            for (int i = 0; i < USED; ++i) {
                const bool in = KEYS ? key_in : seen_at(C, raw.there, t, t + 16 * (i >> 2) + 4 * g + (i & 3), it.lo, it.end);
#pragma unroll
                for (int r = 0; r < (KEYS ? 2 : VH); ++r) raw.r[i][r] = in ? raw.r[i][r] : 0u;
            }
        }
        if constexpr (KEYS) {
            if (lane == 0) there[buffer][sub] = raw.there;
            u32x4 k[KB];
#pragma unroll
            for (int j = 0; j < KB; ++j) k[j] = u32x4{raw.r[2 * j][0], raw.r[2 * j][1], raw.r[2 * j + 1][0], raw.r[2 * j + 1][1]};
#pragma unroll
            for (int j = 0; j < QK; ++j) to[(half * QK + j) * 64] = key_piece<FP8, KB>(k, j);
        } else {
            uint32_t v[8][VH];
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int r = 0; r < VH; ++r) v[i][r] = raw.r[i][r];
            u32x4 vt[WH];
            turn_values<FP8, VH>(v, vt);
#pragma unroll
            for (int e = 0; e < WH; ++e) to[(2 * QK + WH * half + e) * 64] = vt[e];
        }
    };

    u32x4 q[HB][QK];
    float m[HB], l[HB], limit[HB];
    f32x4 acc[HB][W];
#pragma unroll
    for (int b = 0; b < HB; ++b) {
        m[b] = limit[b] = LOWEST;
        l[b] = 0.f;
#pragma unroll
        for (int s = 0; s < QK; ++s) q[b][s] = query_piece<D, FP8>(a, it, 16 * (wave * HB + b) + c, s, g, turn);
#pragma unroll
        for (int e = 0; e < W; ++e) acc[b][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // A step is a block of columns of a tile; the next one's scores are begun while this one's become weights.  (A block's values x weights held back
    // until the next one's exponentials, each matrix instruction between vector instructions: 96.0 us for 93.5 of 65537 positions of 8 bits, 71.0
    // for 71.4 of 30000 of bf16.)
    u32x4 key[2 * QK], vt[W];
    uint32_t next_pages = 15u;                        // of the tile whose keys were read, and where it begins
    int next_t0 = it.begin;
    f32x4 x[2];
    int t0 = it.begin;                                // of the present tile
    auto operands_of = [&](int stage, int tile) __attribute__((always_inline)) { return lds + (stage * SUB + tile) * FRAGS * 64 + lane; };
    auto read_keys = [&](int stage, int tile, int t) __attribute__((always_inline)) {
        const u32x4 *from = operands_of(stage, tile);
#pragma unroll
        for (int j = 0; j < 2 * QK; ++j) key[j] = from[j * 64];
        next_pages = there[stage][tile];
        next_t0 = t;
    };
    // Scores of positions that are not seen (their keys are zeros in LDS) become -inf.
    auto hide = [&]() __attribute__((always_inline)) {
        const uint32_t pages = __builtin_amdgcn_readfirstlane(next_pages);
        if (next_t0 + TILE > it.end || pages != 15u) {
            const Start start = start_of(C, pages, next_t0, g, it.lo, it.end);
            x[0] += start.x[0];
            x[1] += start.x[1];
        }
    };
    // (stage: its number's last bit.  Past the last tile everything goes on, so that the loads in flight are always as many; those scores are not used.)
    auto next_keys = [&](int stage, int tile) __attribute__((always_inline)) {
        const int next_tile = t0 + TILE;
        if (tile == SUB - 1) {
            keep(raw[stage ^ 1], stage ^ 1, next_tile);
            __syncthreads();
            fetch(raw[stage ^ 1], next_tile + 2 * STEP);
            entries_at(next_tile + 3 * STEP);
            read_keys(stage ^ 1, 0, next_tile);
        } else {
            read_keys(stage, tile + 1, next_tile);
        }
    };
    auto step = [&](int stage, int tile, int b) __attribute__((always_inline)) {
        hide();
        if (b == 0) {
            const u32x4 *from = operands_of(stage, tile);
#pragma unroll
            for (int k = 0; k < W; ++k) vt[k] = from[(2 * QK + k) * 64];
        }
        if (b == HB - 1) next_keys(stage, tile);
        const float from = follow<FP8>(x, scale, m[b], l[b], limit[b], acc[b]);
        const Eights e = powers(x, scale, from, l[b]);
        x[0] = x[1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 2 * QK; ++j) x[j & 1] = mfma_bf16(key[(j & 1) * QK + (j >> 1)], q[b + 1 < HB ? b + 1 : 0][j >> 1], x[j & 1]);
        add_weighted<FP8, W>(vt, operands<FP8>(e), acc[b]);
    };
    entries_at(it.begin);
    fetch(raw[0], it.begin);
    entries_at(it.begin + STEP);
    fetch(raw[1], it.begin + STEP);
    entries_at(it.begin + 2 * STEP);
    keep(raw[0], 0, it.begin);
    __syncthreads();
    fetch(raw[0], it.begin + 2 * STEP);
    entries_at(it.begin + 3 * STEP);
    read_keys(0, 0, t0);
    x[0] = x[1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 2 * QK; ++j) x[j & 1] = mfma_bf16(key[(j & 1) * QK + (j >> 1)], q[0][j >> 1], x[j & 1]);
    for (bool more = true; more;) {
#pragma unroll
        for (int tile = 0; tile < 2 * SUB; ++tile) {
            if (!more) break;
#pragma unroll
            for (int b = 0; b < HB; ++b) step(tile / SUB, tile % SUB, b);
            t0 += TILE;
            more = t0 < it.end;
        }
    }
    // A block's sums through the wave's part of LDS, so that whole rows are stored (16 bytes a lane, each of another row: 11 us of the 24 that 128
    // positions take, of 256 workgroups; pieces of a row change places by its column's last bits, for the banks).
    const float v_scale = FP8 && C.v_scale ? C.v_scale[it.kv_head] : 1.f;
    constexpr int PIECES = D / 4;                     // of 16 bytes, of a column
    f32x4 *own = reinterpret_cast<f32x4 *>(lds) + wave * 16 * PIECES;
    __syncthreads();                                  // (the last operands have been read)
#pragma unroll
    for (int b = 0; b < HB; ++b) {
        const int column0 = 16 * (wave * HB + b);
        l[b] = across_groups(l[b], [](float x, float y) { return x + y; });
        if (g == 0 && column0 + c < it.n) {
            a.part_ml[2 * ((size_t)it.slot + column0 + c)] = m[b];
            a.part_ml[2 * ((size_t)it.slot + column0 + c) + 1] = l[b];
        }
#pragma unroll
        for (int h = 0; h < HALVES; ++h)
#pragma unroll
            for (int k = 0; k < WH; ++k) {                     // four elements: of one row of the operand, or of two neighbouring ones
                f32x4 x;
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = acc[b][WH * h + i % WH][k * 4 / WH + i / WH] * v_scale;
                own[c * PIECES + ((PIECES / HALVES * h + WH * g + k) ^ (c & 7))] = x;
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int k = 0; k < 16 * PIECES / 64; ++k) {
            const int u = 64 * k + lane, column = u / PIECES, piece = u % PIECES;
            const f32x4 x = own[column * PIECES + (piece ^ (column & 7))];
            if (column0 + column < it.n) *reinterpret_cast<f32x4 *>(a.part + ((size_t)it.slot + column0 + column) * D + 4 * piece) = x;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// The item of a workgroup: true, of the shared positions; it.n < 1: none.  Of rows' own positions a workgroup has EACH items, this is one of them.
template <int EACH> __device__ __forceinline__ bool item_of(const SharedArgs &a, int of_wg, Item &it)
{
    const CacheArgs &C = a.cache;
    it.n = 0;
    if ((int)blockIdx.x < a.prefix_wgs) {
        // The workgroups of a chunk that have different columns read the same positions: they are eight apart, on one XCD, at the same time.
        const int per = 8 * a.tiles, eight = (int)blockIdx.x / per, in = (int)blockIdx.x - eight * per, tile = in / 8, unit = 8 * eight + in - 8 * tile;
        if (unit >= a.chunks * C.kv_heads) return true;
        const int chunk = unit / C.kv_heads;
        it.kv_head = unit - chunk * C.kv_heads;
        it.first = tile * a.columns;
        it.n = a.rows * a.group - it.first;
        it.n = it.n < a.columns ? it.n : a.columns;
        it.lo = it.begin = chunk * a.chunk;
        it.end = a.shared - it.begin < a.chunk ? a.shared : it.begin + a.chunk;
        it.table = C.table + a.prefix * C.table_stride;
        it.slot = ((long long)unit * a.tiles + tile) * a.columns;
        return true;
    }
    const int number = ((int)blockIdx.x - a.prefix_wgs) * EACH + of_wg, item = number / a.own_splits, split = number - item * a.own_splits;
    if (number >= a.own_items) return false;
    const int of_row = item / a.own_blocks, block = item - of_row * a.own_blocks, row = of_row / C.kv_heads;
    RowInfo r = row_info(a, row);
    r.len = __builtin_amdgcn_readfirstlane(r.len);
    r.lo = __builtin_amdgcn_readfirstlane(r.lo);
    r.seq = __builtin_amdgcn_readfirstlane(r.seq);
    const OwnChunks o = own_chunks(a, r);
    if (split >= o.n) return false;
    it.kv_head = of_row - row * C.kv_heads;
    it.first = row * a.group + block * a.own_columns;
    it.n = a.group - block * a.own_columns;
    it.n = it.n < a.own_columns ? it.n : a.own_columns;
    it.lo = r.lo;
    it.begin = o.from + split * o.length;
    it.end = r.len - it.begin < o.length ? r.len : it.begin + o.length;
    it.table = C.table + r.seq * C.table_stride;
    it.slot = (long long)a.chunks * C.kv_heads * a.tiles * a.columns + (long long)number * a.own_columns;
    return false;
}

// Workgroups of a unit: two, of one wave per SIMD each, with up to 256 registers a lane, or one with up to 512.
constexpr int wgs_per_unit(int D, int HB) { return HB * D <= 128 ? 2 : 1; }

template <int D, bool FP8, int HB>
__global__ __launch_bounds__(256, wgs_per_unit(D, HB)) void shared_kernel(SharedArgs a)
{
    __shared__ u32x4 lds_q[HB > 2 ? HB * (D / 32) * 64 : 1];
    __shared__ float wave_m[4][16], wave_l[4][16];
    __shared__ __attribute__((aligned(16))) float joined[4][16][Shape<D>::DS + 4];
    Item it;
    const bool of_prefix = item_of<1>(a, 0, it);
    if (it.n < 1) return;
    if (of_prefix) attend_item<D, FP8, HB, 4>(a, it, threadIdx.x, lds_q, wave_m, wave_l, joined);
    else attend_item<D, FP8, 1, 4>(a, it, threadIdx.x, lds_q, wave_m, wave_l, joined);
}

// The shared positions of many columns, 128 HB of a workgroup of eight waves; behind those two items of rows' own positions a workgroup, by four
// waves each (one by eight: 200 rows x 32 heads of up to 300 own positions 152 us for 144).
template <int D, bool FP8, int HB>
__global__ __launch_bounds__(512, 1) void shared_wide_kernel(SharedArgs a)
{
    __shared__ union {
        u32x4 operands[2 * 2 * (D / 8) * 64];
        float joined[2][4][16][D + 4];
    } lds;
    __shared__ uint32_t there[2][2];
    __shared__ float wave_m[2][4][16], wave_l[2][4][16];
    Item it;
    const int half = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
    if (!item_of<2>(a, half, it)) {
        // (one barrier in either)
        if (it.n > 0) attend_item<D, FP8, 1, 4>(a, it, threadIdx.x & 255, nullptr, wave_m[half], wave_l[half], lds.joined[half]);
        else __syncthreads();
        return;
    }
    if (it.n < 1) return;
    if (half == 0) attend_columns<D, FP8, HB, true>(a, it, lds.operands, there);
    else attend_columns<D, FP8, HB, false>(a, it, lds.operands, there);
}

// Joins a column's parts: a workgroup, or a wave of one (EACH = 4), per row and head.  A group of D / 4 lanes has some of the parts, 16 bytes of a
// part's sums a lane, four or eight parts in flight; the groups' results meet in LDS.
template <int D, int EACH> __global__ __launch_bounds__(256) void shared_join_kernel(SharedArgs a)
{
    constexpr int LANES = D / 4, GROUPS = 256 / EACH / LANES, FLIGHT = EACH > 1 ? 8 : 4;
    __shared__ float all_m[EACH][GROUPS], all_l[EACH][GROUPS];
    __shared__ f32x4 all_sums[EACH][GROUPS][LANES];
    const CacheArgs &C = a.cache;
    const int of_wg = EACH > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0, tid = EACH > 1 ? threadIdx.x & 63 : threadIdx.x;
    auto &group_m = all_m[of_wg], &group_l = all_l[of_wg];
    auto &sums = all_sums[of_wg];
    const unsigned number = blockIdx.x * EACH + of_wg, items = (unsigned)a.rows * (unsigned)a.heads, item = number < items ? number : items - 1;   // (the last again)
    const int row = (int)(item / (unsigned)a.heads), head = (int)(item - (unsigned)row * (unsigned)a.heads);
    const int kv_head = head / a.group, of_group = head - kv_head * a.group;
    const RowInfo r = row_info(a, row);
    const int shared = r.follows ? a.chunks : 0, n = shared + own_chunks(a, r).n;
    const int query = row * a.group + of_group, tile = query / a.columns, block = of_group / a.own_columns;
    const long long own0 = (long long)a.chunks * C.kv_heads * a.tiles * a.columns +
                           ((long long)(row * C.kv_heads + kv_head) * a.own_blocks + block) * a.own_splits * a.own_columns + (of_group - block * a.own_columns);
    const long long shared0 = ((long long)kv_head * a.tiles + tile) * a.columns + (query - tile * a.columns);
    const int at = tid % LANES, group = tid / LANES;
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
    if (tid >= LANES) return;
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

}  // namespace

SharedPlan shared_plan(const peqa_kv_cache *C, int rows, int heads, int max_len, int shared)
{
    SharedPlan p{};
    const int group = heads / C->kv_heads;
    if (max_len < shared) shared = 0;                          // (every row ends among the shared positions, and has them by itself)
    const long long queries = (long long)rows * group;
    const int most = C->head_dim > 128 ? 2 : 4;                // (as many as there are registers for)
    p.hb = 1;
    while (p.hb < most && 16 * p.hb < queries) p.hb *= 2;
    p.columns = 16 * p.hb;
    // (up to 64 columns all in every wave / each wave its own, us: 8 key heads x 32, 40000 positions 39.8 / 57.6;  4 x 64 28.5 / 33.9, 8 bits 27.0 / 29.5;
    // 4 x 80 36.3 / 34.4;  4 x 128 37.3 / 35.5, 8 bits 36.0 / 31.4, heads of 64 29.6 / 27.9;  4 x 160 72 / 50;  8 x 256 81 / 72.5;  8192 positions
    // 4 x 80 18.8 / 18.7, 4 x 128 19.6 / 19.8)
    p.wide = C->head_dim <= 128 && queries > 64;
    if (p.wide) {
        // 256 columns halve what comes through LDS for each, 128 the parts, which count where few positions are walked; neither leaves columns
        // empty that the other does not (us, 256 / 128: 8 key heads x 512, 8192 shared and up to 1024 own 73 / 87.5;  8 x 256, 30000 72.5 / 76.6;
        // 4 x 160, 40000 50 / 54;  8 x 256, 8192 (8 bits) 29.0 / 27.9;  4 x 160, 8192 25.8 / 22.8;  4 x 320, 30000 68 / 58)
        p.hb = (queries + 127) / 128 % 2 == 0 && (queries + 255) / 256 * C->kv_heads * shared >= 2 * UNIT * PLAN_UNITS ? 2 : 1;
        p.columns = 128 * p.hb;
    }
    p.tiles = (int)((queries + p.columns - 1) / p.columns);
    p.own_columns = group < 16 ? group : 16;
    p.own_blocks = (group + p.own_columns - 1) / p.own_columns;
    const long long own = max_len > shared ? max_len - shared + TILE - 1 : 0;
    const long long items = (long long)rows * C->kv_heads * p.own_blocks, units = (long long)C->kv_heads * p.tiles;
    // all that there is to walk, over as many workgroups as have room at once, 128 positions at least; rows' own positions are half of the longest's on average
    auto per_workgroup = [](long long all, int wgs) {
        const long long chunk = ((all + wgs - 1) / wgs + UNIT - 1) / UNIT * UNIT;
        return chunk < UNIT ? (long long)UNIT : chunk;
    };
    long long chunk, own_chunk;
    if (p.wide) {
        // Many columns of a position are two of a row's own: then the units that the shared positions leave read the rows' own meanwhile, matrix
        // instructions beside loads (64 rows x 8 key heads x 8, 8192 shared and up to 1024 own: 65 us, 79 with the shared ones on all units; with three
        // or four for two 80, rows' own cut finer 67 to 72).
        chunk = per_workgroup(units * shared + items * own / 4, PLAN_UNITS);
        own_chunk = per_workgroup(items * own, 2 * PLAN_UNITS);
    } else {
        // (rows' own cut finer: 40 rows x 8 heads, 4096 shared and up to 2000 own 47.4 -> 41.8 us)
        chunk = per_workgroup(units * shared + items * own / 2, PLAN_UNITS * wgs_per_unit(C->head_dim, p.hb));
        own_chunk = chunk / 2 > UNIT ? chunk / 2 : UNIT;
    }
    p.chunks = (int)((shared + chunk - 1) / chunk);
    p.chunk = p.chunks > 0 ? (int)(((shared + p.chunks - 1) / p.chunks + TILE - 1) / TILE * TILE) : TILE;
    p.chunks = (shared + p.chunk - 1) / p.chunk;
    p.own_splits = (int)((own + own_chunk - 1) / own_chunk);
    if (p.own_splits < 1) p.own_splits = 1;                    // (rows that end among the shared positions)
    p.own_chunk = UNIT;
    p.prefix_wgs = ((long long)p.chunks * C->kv_heads + 7) / 8 * 8 * p.tiles;
    p.own_items = items * p.own_splits;
    // A wave a column where columns are many and its parts all in flight at once (us, and by four waves: 64 rows x 64 heads of 10 parts 70.4, 74.5;  100 x 32
    // of 64 elements 21.1, 22.6;  200 x 32 133, 136;  but 32 x 64 of 33 parts 96.2, 95.0, 8 x 64 of 64 38.2, 36.5)
    p.join_each = (long long)rows * heads >= 4 * PLAN_UNITS && p.chunks + p.own_splits <= 2048 / C->head_dim ? 4 : 1;
    const size_t slots = (size_t)p.chunks * (size_t)units * (size_t)p.columns + (size_t)p.own_items * (size_t)p.own_columns;
    p.part_bytes = round256(slots * (size_t)C->head_dim * sizeof(float));
    p.ml_bytes = round256(slots * 2 * sizeof(float));
    return p;
}

namespace {

template <int D, bool FP8> hipError_t launch_shared(const SharedArgs &a, const SharedPlan &p, hipStream_t stream)
{
    auto run = [&](auto kernel, const SharedArgs &args, long long wgs, int threads) {
        trace_before(KID_SHARED, stream);
        hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(threads), 0, stream, args);
        trace_after(KID_SHARED, stream);
        return hipGetLastError();
    };
    hipError_t e = hipSuccess;
    if constexpr (D <= 128) {
        if (p.wide) {
            e = run(p.hb == 1 ? shared_wide_kernel<D, FP8, 1> : shared_wide_kernel<D, FP8, 2>, a, p.prefix_wgs + (p.own_items + 1) / 2, 512);
        } else if (p.hb == 4) {
            e = run(shared_kernel<D, FP8, 4>, a, p.prefix_wgs + p.own_items, 256);
        }
    }
    if (!p.wide && p.hb < 4) e = run(p.hb == 1 ? shared_kernel<D, FP8, 1> : shared_kernel<D, FP8, 2>, a, p.prefix_wgs + p.own_items, 256);
    if (e != hipSuccess) return e;
    trace_before(KID_SHARED_JOIN, stream);
    const unsigned items = (unsigned)a.rows * (unsigned)a.heads;
    if (p.join_each > 1) hipLaunchKernelGGL((shared_join_kernel<D, 4>), dim3((items + 3) / 4), dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((shared_join_kernel<D, 1>), dim3(items), dim3(256), 0, stream, a);
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
    if (p.prefix_wgs + p.own_items > (1 << 23)) return PEQA_ERR_SHAPE;
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
    a.prefix_wgs = (int)p.prefix_wgs; a.own_items = (int)p.own_items;
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
