// Attention of single query tokens over the paged cache (peqa_paged_attention), and with what every position was given of it
// (peqa_paged_attention_weights).
//
// For a row and one of its key heads, with the heads that share it as columns:
//   x[j][h] = scale <k_j, q_h>;   out[h] = sum_j e^(x[j][h]) v_j / sum_j e^(x[j][h])
// in one pass over the positions j with the running maximum and sum of every head, all in powers of two (the scale carries
// log2 e).  Both products are matrix instructions that take their operands as they come from memory: the scores as keys x
// queries, so that a lane ends with eight scores of ONE head, which are the weights' operand of the second product as they
// stand, and values^T x weights, for which a lane loads whole 16-byte pieces of eight positions and turns the 8 x 8 elements
// in registers.
// Positions are split over the waves of a workgroup in tiles of 32, whose sums meet in LDS, and over workgroups, joined by a second
// kernel (attend_plan): a workgroup has a whole item (a row with the heads of one key head), a chunk of one, or an equal share
// of all items laid end to end.
// Every key and value is read once, and the matrix and vector instructions of a tile (a third and less of the time) run beside the loads of
// the next: bound by what a unit has in flight, and for short rows by the start of a launch and the latency of its three dependent
// loads (length, page, tile).  Measured, the kernel alone:  one row of 131072 positions, 8 key heads of 128, 8 heads to each  93.5 us,
// 5.7 TB/s;  64 rows of up to 8192 on 8 bits, as many heads  107 us, 5.2 TB/s;  16 rows of up to 2048, 32 key heads  53.5 us, 4.8 TB/s;
// one row of 333, 32 key heads  9 us.
#include "peqa_attend.h"
#include "peqa_cache.h"
#include "peqa_host.h"

using namespace peqa::host;

namespace peqa {

// How a call is cut: column blocks of a workgroup, workgroups' worth of heads per key head, heads of a workgroup, chunks or shares.
struct AttendPlan {
    int hb, waves, blocks, per_wg, splits, chunk_units, shares, entries;
    long long grid;
    size_t part_bytes, ml_bytes, parts_bytes;
};
AttendPlan attend_plan(const peqa_kv_cache *C, int rows, int heads, int max_len, int window);

namespace {

constexpr int TILE = 32;                 // positions per step of a wave
constexpr int UNIT = 64;                 // positions that shares are counted in
constexpr int SCAN_ROWS = 1024;          // rows of a launch of equal shares at most: every workgroup adds up their lengths

// An item in several workgroups, for the join (n < 2: none): the slots of its n parts are first, next, next + step, ...
struct ItemParts {
    int row, item, n, first, next, step;
};

// What the scores of a row and a head are weighted with: 2^(score - reference) / total (0 of a row that saw no position).  The logarithm of the sum would be one
// number, but rounded to 2^-24 of itself: 2^-11 of every weight where scores are around 10^4.
struct RowSum {
    float reference, total;
};
constexpr int SUM_ROOM = 4;              // floats for it in front of a row's and a head's scores
__device__ __forceinline__ RowSum &sum_of(const float *scores) { return *reinterpret_cast<RowSum *>(const_cast<float *>(scores) - SUM_ROOM); }

struct AttendArgs {
    CacheArgs cache;
    const uint16_t *q;
    const int32_t *lens, *seq;
    uint16_t *out;
    float *lse;
    // Parts of items that are in several workgroups: a slot has the heads of one workgroup.
    float *part;               // [slots, per_wg, head_dim] weighted sums, relative to the reference
    float *part_ml;            // [slots, per_wg, 2] reference (the maximum, or 14 below it; of powers of two) and sum
    ItemParts *parts;          // [rows * items of a row], or [shares]: of the item that ends in a share and began before it
    float *scores;             // [rows, heads, score_stride] of powers of two, for the positions' weights, a RowSum in front of each; or null
    const float *weights;      // of an item's positions, where the workgroup that has all of it adds what they were given
    float *weights_out;        // (null: attend_weights_kernel does)
    long long q_stride, out_stride, score_stride, weights_seq_stride, weights_head_stride;
    float scale;               // times log2 e
    int rows, heads, group;    // heads per key head
    int max_len, window;
    int blocks, per_wg;        // workgroups' worth of heads per key head, and heads in one
    int splits, chunk_units;   // chunks of the longest row, and units in one
    int shares;                // workgroups of a launch of equal shares; 0: workgroups of chunks
};

// What of a row there is: positions [lo, len), walked from `from` on (lo rounded down to a unit), in `units`.
struct RowRange {
    int lo, from, len, units;
};
__device__ __forceinline__ RowRange row_range(const AttendArgs &a, int len)
{
    RowRange r;
    r.len = len;
    r.lo = a.window > 0 && len > a.window ? len - a.window : 0;
    r.from = r.lo & ~(UNIT - 1);
    r.units = (len - r.from + UNIT - 1) / UNIT;
    if (r.units == 0) r.units = 1;                         // an empty row is an item too: of zeros
    return r;
}
// A row's sequence and the positions it has.
struct RowInfo {
    int seq, len;
};
__device__ __forceinline__ RowInfo row_info(const AttendArgs &a, int row)
{
    RowInfo r;
    r.seq = a.seq ? a.seq[row] : row;
    r.len = a.lens[row];
    r.len = r.len < a.max_len ? r.len : a.max_len;
    if (r.seq < 0 || r.seq >= a.cache.n_seqs || r.len < 0) { r.len = 0; r.seq = 0; }
    return r;
}

// What a workgroup does: units [at, until) of all items laid end to end; `at` is in row `row`, whose first unit is `row_at`.
// Shares are cut at multiples of `length` from a line on which every item has START more units in front: what a workgroup
// takes to begin one and to leave its result.
constexpr int START = 3;
struct Share {
    int at, until, length, row, row_at;
};

// Share number `share` of a launch of equal shares; leaves what all rows have in `info`.  scan: WAVES + 6 numbers of LDS.
template <int WAVES>
__device__ __forceinline__ Share share_of(const AttendArgs &a, int share, int per_row, RowInfo *info, int *scan)
{
    constexpr int EACH = SCAN_ROWS / (64 * WAVES);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int units[EACH], sum = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int row = i * 64 * WAVES + tid;
        units[i] = 0;
        if (row < a.rows) info[row] = row_info(a, row);
    }
    __syncthreads();
    const int each = (a.rows + 64 * WAVES - 1) / (64 * WAVES);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int row = tid * each + i;
        if (i < each && row < a.rows) units[i] = (row_range(a, info[row].len).units + START) * per_row;
        sum += units[i];
    }
    int upto = sum;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const int other = __shfl_up(upto, o);
        if (lane >= o) upto += other;
    }
    if (lane == 63) scan[wave] = upto;
    __syncthreads();
    int before = upto - sum, total = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        before += w < wave ? scan[w] : 0;
        total += scan[w];
    }
    Share s;
    s.length = __builtin_amdgcn_readfirstlane((total + a.shares - 1) / a.shares);
    const int cut[2] = {share * s.length, share * s.length + s.length};
    int *found = scan + WAVES;                             // row, its first unit, unit: of both cuts
    if (tid < 6) found[tid] = tid % 3 == 0 ? a.rows : total - START * per_row * a.rows;    // cuts past the end
    __syncthreads();
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (cut[k] >= before && cut[k] < before + units[i]) {
                const int row = tid * each + i, of_item = units[i] / per_row, in = cut[k] - before, item = in / of_item;
                const int unit = in - item * of_item - START, row_at = before - START * per_row * row;
                found[3 * k] = row;
                found[3 * k + 1] = row_at;
                found[3 * k + 2] = row_at + item * (of_item - START) + (unit > 0 ? unit : 0);
            }
        before += units[i];
    }
    __syncthreads();
    // (all that a share is, is the same for the whole workgroup)
    s.row = __builtin_amdgcn_readfirstlane(found[0]);
    s.row_at = __builtin_amdgcn_readfirstlane(found[1]);
    s.at = __builtin_amdgcn_readfirstlane(found[2]);
    s.until = __builtin_amdgcn_readfirstlane(found[5]);
    return s;
}

// A piece of a share: at most CHUNK positions [begin, end) of an item.  A segment is what a share has of an item: one or more pieces.
struct Piece {
    int row, item, kv_head, first_head, seq, lo, begin, end, slot;    // first_head: of the heads that share kv_head
    bool first, last, alone;                               // of its segment; alone: the segment is the whole item
};

// What four positions were given by a row's heads of a key head, FLIGHT heads in flight, added in their order: of those in [lo, end).  (Scores of positions that
// are not seen are -inf, references finite.)
template <int FLIGHT>
__device__ __forceinline__ void add_given(f32x4 &sum, const float *scores, long long stride, int heads, int pos, int lo, int end)
{
    for (int i0 = 0; i0 < heads; i0 += FLIGHT) {
        f32x4 x[FLIGHT];
        RowSum of[FLIGHT];
#pragma unroll
        for (int i = 0; i < FLIGHT; ++i) {
            const int at = i0 + i < heads ? i0 + i : i0;
            x[i] = *reinterpret_cast<const f32x4 *>(scores + at * stride + pos);
            of[i] = sum_of(scores + at * stride);
        }
#pragma unroll
        for (int i = 0; i < FLIGHT; ++i) {
            if (i0 + i >= heads) continue;
            const float by = of[i].total != 0.f ? __builtin_amdgcn_rcpf(of[i].total) : 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) sum[k] += pos + k >= lo && pos + k < end ? __builtin_amdgcn_exp2f(x[i][k] - of[i].reference) * by : 0.f;
        }
    }
}
__device__ __forceinline__ void store_given(const float *weights, float *weights_out, f32x4 sum, int pos, int end)
{
    if (pos + 4 <= end) {
        if (weights) sum += *reinterpret_cast<const f32x4 *>(weights + pos);
        *reinterpret_cast<f32x4 *>(weights_out + pos) = sum;
    } else {
        for (int k = 0; k < end - pos; ++k) weights_out[pos + k] = (weights ? weights[pos + k] : 0.f) + sum[k];
    }
}

// The sum of lanes c and c + 8 of every 16, in both.
__device__ __forceinline__ float add_halves(float v)
{
    return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x128 /* row_ror:8 */, 0xF, 0xF, true));
}

// Workgroups of a unit: two, of one wave per SIMD each, with up to 256 registers a lane; of the widest heads, whose two tiles
// alone are as many, one with up to 512.
constexpr int wgs_per_unit(int D, bool fp8) { return D > 128 && !fp8 ? 1 : 2; }

template <int D, bool FP8, int HB, int WAVES, bool TWICE, bool SCORES>
__global__ __launch_bounds__(64 * WAVES, wgs_per_unit(D, FP8)) void attend_kernel(AttendArgs a)
{
    // Columns of the matrix instructions: eight heads twice, the upper ones with what rounding the weights leaves, so that they have 16 bits
    // against bf16 values and 22, as fp16, against 8-bit ones (64 rows of up to 8192 with eight heads to a key head 115.5 us with one part,
    // 115.9 with two, three caches in turn).  More than eight heads on 8-bit values have a column each and weights of 11 bits: with eight at
    // a time 12 heads take 132 us for 120, 128 rows of up to 200 with 8 x 12 heads 19.7 for 14.5.
    static_assert(TWICE || FP8);
    constexpr int COLS = TWICE ? 8 : 16;
    constexpr int QK = D / 32;                        // steps of the scores' product
    constexpr int SEG = D > 128 ? D / 128 : 1;        // segments of 128 elements of a value
    constexpr int W = D / 16 / SEG;                   // neighbouring elements of a segment that a lane has: 4 or 8
    constexpr int KB = FP8 ? D / 64 : D / 32;         // 16-byte pieces of a key that a lane loads
    constexpr int DS = D / SEG;
    constexpr int VR = FP8 ? W / 4 : W / 2;           // registers of a value's segment
    constexpr int EL = FP8 ? 1 : 2;                   // bytes of an element
    constexpr bool AHEAD = HB * D <= 128 || (HB == 1 && wgs_per_unit(D, FP8) == 1);    // registers for two tiles (of 16 heads of 256: for their queries and sums)
    // Positions of a piece, whose pages are in LDS at a time: few where a wave has an item to itself, whose rows are short (5 KB of LDS for a
    // workgroup instead of 21: 119 rows x 64 heads of up to 8 positions 25.0 -> 20.6 us, 128 x 8 of up to 200 16.0 -> 13.5; 17.0 and 13.8 with
    // 8-bit weights in two parts).
    constexpr int CHUNK = WAVES == 1 ? 512 : 4096;
    __shared__ long long page_at[2][CHUNK / 8];             // where a piece's pages begin, in bytes; -1: not there
    __shared__ RowInfo info[WAVES == 4 ? SCAN_ROWS : 1];
    __shared__ int scan[WAVES + 6];
    __shared__ float wave_m[WAVES][HB][16], wave_l[WAVES][HB][16];
    __shared__ __attribute__((aligned(16))) float joined[WAVES][8][DS + 4];

    const CacheArgs &C = a.cache;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, g = lane >> 4;
    const int per_row = C.kv_heads * a.blocks;
    const int slot_bytes = (int)C.slot_stride * EL;

    Share share;
    int info_row = 0;                                      // the row of info[0]
    int parts_at = (int)blockIdx.x, chunk_slot = 0;
    const bool shares = WAVES == 4 && a.shares > 0;        // (others are launched with whole items)
    if (shares) {
        share = share_of<WAVES>(a, (int)blockIdx.x, per_row, info, scan);
        if (threadIdx.x == 0) a.parts[parts_at].n = 0;
        if (share.at >= share.until) return;
    } else {
        // workgroups by row, chunk and item: the items of a row at the same time, whose heads' places in a page are neighbours
        const int of_row = (int)(blockIdx.x / (unsigned)per_row), item = (int)(blockIdx.x - (unsigned)of_row * (unsigned)per_row);
        share.row = (int)((unsigned)of_row / (unsigned)a.splits);
        const int split = of_row - share.row * a.splits;
        const RowInfo here = row_info(a, share.row);
        const int units = __builtin_amdgcn_readfirstlane(row_range(a, here.len).units);
        if (split * a.chunk_units >= units) return;
        if (threadIdx.x == 0) info[0] = here;
        __syncthreads();
        info_row = share.row;
        share.row_at = 0;
        share.length = a.chunk_units;
        share.at = item * units + split * a.chunk_units;
        share.until = item * units + ((split + 1) * a.chunk_units < units ? (split + 1) * a.chunk_units : units);
        parts_at = share.row * per_row + item;
        chunk_slot = parts_at * a.splits + split;
        if (a.splits > 1 && split == 0 && threadIdx.x == 0)
            a.parts[parts_at] = ItemParts{share.row, item, (units + a.chunk_units - 1) / a.chunk_units, chunk_slot, chunk_slot + 1, 1};
    }
    const int share_begin = share.at;

    int segment_from = 0;                                  // the unit of its item that the segment began at
    auto next_piece = [&]() __attribute__((always_inline)) {
        Piece p;
        p.row = share.row;
        p.seq = __builtin_amdgcn_readfirstlane(info[p.row - info_row].seq);
        const RowRange range = row_range(a, __builtin_amdgcn_readfirstlane(info[p.row - info_row].len));
        const int in_row = share.at - share.row_at;
        p.item = in_row / range.units;
        p.kv_head = p.item / a.blocks;
        p.first_head = (p.item - p.kv_head * a.blocks) * COLS * HB;
        const int from = in_row - p.item * range.units, left = share.until - share.at;
        int n = range.units - from < left ? range.units - from : left;
        n = n < CHUNK / UNIT ? n : CHUNK / UNIT;
        p.lo = range.lo;
        p.begin = range.from + from * UNIT;
        const bool over = from + n == range.units;         // the item ends here
        p.end = over ? range.len : p.begin + n * UNIT;
        p.first = share.at == share_begin || from == 0;
        if (p.first) segment_from = from;
        p.last = over || n == left;
        p.alone = over && segment_from == 0;               // (of a chunk: segment_from is its first unit)
        if (!shares) {
            p.slot = chunk_slot;
        } else {
            // of the share's first segment, where an item goes on, and of its last one
            p.slot = 2 * (int)blockIdx.x + (share.at - from + segment_from == share_begin ? 0 : 1);
            if (over && segment_from > 0 && threadIdx.x == 0) {
                // the item's first unit on the line of the cuts, and the share that has it
                const int start = share.row_at + START * per_row * p.row + p.item * (range.units + START), w = (start + START) / share.length;
                a.parts[blockIdx.x] = ItemParts{p.row, p.item, (int)blockIdx.x - w + 1, 2 * w + (w * share.length >= start ? 0 : 1), 2 * w + 2, 2};
            }
        }
        share.at += n;
        if (in_row + n == range.units * per_row) { share.row_at = share.at; ++share.row; }
        return p;
    };
    constexpr int ENTRIES = CHUNK / 8 / (64 * WAVES);      // of a piece's part of the table, per thread
    int32_t entry[ENTRIES];
    auto read_table = [&](const Piece &p) __attribute__((always_inline)) {
        const int block0 = p.begin >> C.page_shift, blocks = p.end > p.begin ? ((p.end - 1) >> C.page_shift) - block0 + 1 : 0;
        const int32_t *table = C.table + p.seq * C.table_stride + block0;
#pragma unroll
        for (int i = 0; i < ENTRIES; ++i) {
            const int at = i * 64 * WAVES + (int)threadIdx.x;
            entry[i] = at < blocks ? table[at] : -1;
        }
    };
    auto keep_table = [&](int buffer) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < ENTRIES; ++i)
            page_at[buffer][i * 64 * WAVES + threadIdx.x] = entry[i] >= 0 && entry[i] < C.n_pages ? entry[i] * C.page_stride * EL : -1ll;
    };

    int buffer = 0;
    u32x4 q[HB][QK];
    auto read_queries = [&](const Piece &p) __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < HB; ++b) {
            const int i = p.first_head + b * COLS + (c & (COLS - 1));
            const uint16_t *src = a.q + p.row * a.q_stride + (long long)(p.kv_head * a.group + (i < a.group ? i : 0)) * D;
#pragma unroll
            for (int s = 0; s < QK; ++s) {
                // the keys' pieces decide which elements a step has
                const int at = FP8 ? 64 * (s >> 1) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g;
                q[b][s] = *reinterpret_cast<const u32x4 *>(src + at);
            }
        }
    };
    float m[HB], l[HB], scale = 0.f;
    f32x4 acc[HB][SEG * W];
    Piece cur{};
    // A tile in registers: pieces of the keys at t0 + c and t0 + 16 + c, of the values at t0 + 4 g .. + 3 and t0 + 16 + 4 g .. + 3 (a page
    // has whole quads of positions).  Positions past the end are read from the last one's place, quads from the last one's.
    struct Tile {
        u32x4 k[2][KB];
        uint32_t v[8][SEG][VR];
        uint32_t there;                                // bits 0, 1: the quads' pages are there; 2: the keys' too
    };
    auto load = [&](Tile &t, const Piece &p, int t0) __attribute__((always_inline)) {
        const int last = p.end - 1, block0 = p.begin >> C.page_shift;
        const uint8_t *kbase = static_cast<const uint8_t *>(C.k) + p.kv_head * C.head_stride * EL + 16 * g;
        const uint8_t *vbase = static_cast<const uint8_t *>(C.v) + p.kv_head * C.head_stride * EL + W * EL * c;
        const long long *pages = page_at[buffer];
        t.there = 4;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int pos = t0 + 16 * s + c, at = pos < last ? pos : last;
            long long page = pages[(at >> C.page_shift) - block0];
            if (page < 0) { page = 0; t.there &= ~4u; }
            const uint8_t *src = kbase + page + (uint32_t)((at & C.page_mask) * slot_bytes);
#pragma unroll
            for (int j = 0; j < KB; ++j) t.k[s][j] = *reinterpret_cast<const u32x4 *>(src + 64 * j);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int pos = t0 + 16 * s + 4 * g, quad = last & ~3, at = pos < quad ? pos : quad;
            long long page = pages[(at >> C.page_shift) - block0];
            if (page < 0) page = 0; else t.there |= 1u << s;
            const uint8_t *src = vbase + page + (uint32_t)((at & C.page_mask) * slot_bytes);
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
    auto step = [&](Tile &t, int t0) __attribute__((always_inline)) {
        auto &k = t.k;
        auto &v = t.v;
        const bool full = t0 >= cur.lo && t0 + TILE <= cur.end && __ballot(t.there != 7u) == 0;
        auto seen = [&](int i) {
            const int p = t0 + 16 * (i >> 2) + 4 * g + (i & 3);
            return p >= cur.lo && p < cur.end && (t.there >> (i >> 2) & 1u);
        };
        if (!full) {
            // what masked positions hold must not meet a weight of 0: NaN and infinities would stay
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool in = seen(i);
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
                if (!full) y[i] = seen(i) ? y[i] : -__builtin_inff();
                top = fmaxf(top, y[i]);
            }
            if constexpr (SCORES) {
                // (the columns of a head's remainders have the same scores)
                const int of_group = cur.first_head + b * COLS + c;
                if (c < COLS && of_group < a.group) {
                    float *o = a.scores + ((size_t)cur.row * a.heads + cur.kv_head * a.group + of_group) * a.score_stride + t0 + 4 * g;
                    if (t0 + 4 * g < cur.end) *reinterpret_cast<f32x4 *>(o) = f32x4{y[0], y[1], y[2], y[3]};
                    if (t0 + 16 + 4 * g < cur.end) *reinterpret_cast<f32x4 *>(o + 16) = f32x4{y[4], y[5], y[6], y[7]};
                }
            }
            top = across_groups(top, [](float x, float y) { return fmaxf(x, y); });
            // relative to 2^14 below the maximum, weights down to 2^-28 of the largest are normal fp16 numbers (scores past 2^24 have no bits for it)
            if constexpr (FP8) top = fabsf(top) < 16777216.f ? top - 14.f : top;
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
                for (int i = 0; i < 4; ++i) {
                    const f16x2 near = {(_Float16)p[2 * i], (_Float16)p[2 * i + 1]};
                    if constexpr (TWICE) {
                        const f16x2 rest = {(_Float16)(p[2 * i] - (float)near[0]), (_Float16)(p[2 * i + 1] - (float)near[1])};
                        weight[b][i] = __builtin_bit_cast(uint32_t, c < 8 ? near : rest);
                    } else {
                        weight[b][i] = __builtin_bit_cast(uint32_t, near);
                    }
                }
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
    };

    // The waves' sums: everything goes to LDS as it is, and every thread scales and adds four elements of a head.
    auto join_waves = [&](bool more) __attribute__((always_inline)) {
        if constexpr (!FP8) {
            // Of an infinite value the product with the weight is the answer: the remainder's sign is any, and 0 times infinity is NaN.  (One
            // instruction a sum to see that there are none: 110 x 64 rows of 5 positions, heads of 256, 45.5 -> 46.7 us; choosing for every
            // sum 49.)
            constexpr int CHAINS = HB == 1 ? 4 : 2;        // (as many as there are registers for)
            float zero[4] = {0.f, 0.f, 0.f, 0.f};          // NaN where a sum is not finite
#pragma unroll
            for (int b = 0; b < HB; ++b)
#pragma unroll
                for (int e = 0; e < SEG * W; ++e)
#pragma unroll
                    for (int r = 0; r < 4; ++r) zero[r % CHAINS] = fmaf(acc[b][e][r], 0.f, zero[r % CHAINS]);
            if (__builtin_expect(__ballot(zero[0] + zero[1] + (zero[2] + zero[3]) != 0.f) != 0, 0)) {
#pragma unroll
                for (int b = 0; b < HB; ++b)
#pragma unroll
                    for (int e = 0; e < SEG * W; ++e)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            // (the remainders' lanes become 0 where the weights' are infinite)
                            const float other = __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(acc[b][e][r]), 0x128, 0xF, 0xF, true));
                            acc[b][e][r] = c >= 8 && fabsf(other) == __builtin_inff() ? 0.f : acc[b][e][r];
                            __builtin_amdgcn_sched_barrier(0);
                        }
            }
        }
        const float v_scale = FP8 && C.v_scale ? C.v_scale[cur.kv_head] : 1.f;
        int tid = threadIdx.x, c = lane & 15, g = lane >> 4;
        if constexpr (D > 128) {
            // what follows from the thread's number is found anew, not kept in registers over the tiles
            asm volatile("" : "+v"(tid));
            c = tid & 15;
            g = tid >> 4 & 3;
        }
#pragma unroll
        for (int b = 0; b < HB; ++b) {
            l[b] = across_groups(l[b], [](float x, float y) { return x + y; });
            if (g == 0) { wave_m[wave][b][c] = m[b]; wave_l[wave][b][c] = l[b]; }
#pragma unroll
            for (int half = 0; half < COLS / 8; ++half) {
                const int first = cur.first_head + b * COLS + 8 * half;       // of the heads that share the key head: eight columns
                if (b + half > 0 && first >= a.group) break;                  // (uniform)
#pragma unroll
                for (int s = 0; s < SEG; ++s) {
                    if (b + half + s > 0) __syncthreads();
#pragma unroll
                    for (int r = 0; r < 4; ++r)
#pragma unroll
                        for (int e = 0; e < W; e += 4) {
                            f32x4 x;
#pragma unroll
                            for (int i = 0; i < 4; ++i) x[i] = TWICE ? add_halves(acc[b][s * W + e + i][r]) : acc[b][s * W + e + i][r];
                            // this lane: elements 128 s + W (4 g + r) + e
                            if (c >> 3 == half) *reinterpret_cast<f32x4 *>(&joined[wave][c & 7][W * (4 * g + r) + e]) = x;
                        }
                    __syncthreads();
                    for (int u = tid; u < 8 * DS / 4; u += 64 * WAVES) {
                        const int col = u / (DS / 4), at = 4 * (u % (DS / 4)), of_group = first + col;
                        if (of_group >= a.group) break;
                        float top = LOWEST, total = 0.f;
#pragma unroll
                        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, wave_m[w][b][8 * half + col]);
                        f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int w = 0; w < WAVES; ++w) {
                            const float by = __builtin_amdgcn_exp2f(wave_m[w][b][8 * half + col] - top);
                            total += wave_l[w][b][8 * half + col] * by;
                            x += *reinterpret_cast<const f32x4 *>(&joined[w][col][at]) * by;
                        }
                        const int head = cur.kv_head * a.group + of_group;
                        if (cur.alone) {
                            const bool any = total > 0.f || total != total;
                            const float by = any ? v_scale / total : 0.f;
                            uint16_t *o = a.out + cur.row * a.out_stride + (long long)head * D + 128 * s + at;
                            *reinterpret_cast<u32x2 *>(o) = u32x2{pack_bf16x2(x[0] * by, x[1] * by), pack_bf16x2(x[2] * by, x[3] * by)};
                            if (at == 0 && s == 0) {
                                const float lse = any ? top + __builtin_amdgcn_logf(total) : -__builtin_inff();
                                if constexpr (SCORES) sum_of(a.scores + ((size_t)cur.row * a.heads + head) * a.score_stride) = RowSum{top, total};
                                if (a.lse) a.lse[(size_t)cur.row * a.heads + head] = lse * LN2;
                            }
                        } else {
                            const size_t place = (size_t)cur.slot * a.per_wg + b * COLS + 8 * half + col;
                            *reinterpret_cast<f32x4 *>(a.part + place * D + 128 * s + at) = x;
                            if (at == 0 && s == 0) {
                                a.part_ml[2 * place] = top;
                                a.part_ml[2 * place + 1] = total;
                            }
                        }
                    }
                }
            }
        }
        if constexpr (SCORES) {
            if (a.weights_out) {
                // (the item, of one piece or several, is this workgroup's only one and has all heads of its key head)
                __syncthreads();
                const long long at = cur.seq * a.weights_seq_stride + cur.kv_head * a.weights_head_stride;
                for (int pos = 4 * tid; pos < cur.end; pos += 256 * WAVES) {
                    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
                    const float *scores = a.scores + ((size_t)cur.row * a.heads + (size_t)cur.kv_head * a.group) * a.score_stride;
                    if (pos + 4 > cur.lo) {
                        if (a.group > 1) add_given<4>(sum, scores, a.score_stride, a.group, pos, cur.lo, cur.end);
                        else add_given<1>(sum, scores, a.score_stride, 1, pos, cur.lo, cur.end);
                    }
                    store_given(a.weights ? a.weights + at : nullptr, a.weights_out + at, sum, pos, cur.end);
                }
            }
        }
        if (more) __syncthreads();
    };

    // While a piece is computed, the next one's part of the table is on its way; its first tile and queries are while a segment's sums are
    // joined.  Two tiles of a wave are in flight where they fit in the registers.  The first piece is a next one like the others: a
    // kernel's instructions come from memory when they are first met, and those of a short call are met once.
    constexpr int STEP = WAVES * TILE;
    Tile x;
    bool begun = false;
    for (;;) {
        const bool more = share.at < share.until;
        Piece next = cur;
        if (more) {
            next = next_piece();
            read_table(next);
        }
        if (begun) {
            int t0 = cur.begin + wave * TILE;
            if constexpr (AHEAD) {
                Tile y;
                while (t0 < cur.end) {
                    if (t0 + STEP < cur.end) load(y, cur, t0 + STEP);
                    step(x, t0);
                    x = y;
                    t0 += STEP;
                }
            } else {
                while (t0 < cur.end) {
                    step(x, t0);
                    t0 += STEP;
                    if (t0 < cur.end) load(x, cur, t0);
                }
            }
        }
        if (more) {
            buffer ^= 1;
            keep_table(buffer);
            __syncthreads();
            if (next.first) read_queries(next);
            if (next.begin + wave * TILE < next.end) load(x, next, next.begin + wave * TILE);
        }
        if (begun && cur.last) join_waves(more);
        if (!more) return;
        cur = next;
        begun = true;
        if (cur.first) {
            scale = a.scale * (FP8 && C.k_scale ? C.k_scale[cur.kv_head] : 1.f);
#pragma unroll
            for (int b = 0; b < HB; ++b) {
                m[b] = LOWEST;
                l[b] = 0.f;
#pragma unroll
                for (int e = 0; e < SEG * W; ++e) acc[b][e] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
        }
    }
}

// Joins the parts of an item that is in several workgroups: a workgroup per entry of `parts` and head.  A group of D / 4 lanes has some of
// the parts, 16 bytes of a part's sums a lane with their maximum beside them, four parts in flight, and joins them as the tiles are
// joined; the groups' results meet in LDS.  Bound by the latency of two loads after one another, the entry and the parts: 4.7 us where
// 512 shares have few parts each.
template <int D, bool FP8>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a)
{
    constexpr int LANES = D / 4, GROUPS = 256 / LANES, FLIGHT = 4;
    __shared__ float group_m[GROUPS], group_l[GROUPS];
    __shared__ f32x4 sums[GROUPS][LANES];
    const int heads = a.group < a.per_wg ? a.group : a.per_wg;
    const int entry = (int)(blockIdx.x / (unsigned)heads), i = (int)(blockIdx.x - (unsigned)entry * (unsigned)heads);
    const ItemParts item = a.parts[entry];
    const int n = item.n;
    if (n < 2) return;
    const int kv_head = item.item / a.blocks, of_group = (item.item - kv_head * a.blocks) * a.per_wg + i;
    if (of_group >= a.group) return;
    const int head = kv_head * a.group + of_group;
    const float v_scale = FP8 && a.cache.v_scale ? a.cache.v_scale[kv_head] : 1.f;
    const int at = threadIdx.x % LANES, group = threadIdx.x / LANES;
    float m = LOWEST, l = 0.f;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = group; s0 < n; s0 += FLIGHT * GROUPS) {
        f32x4 x[FLIGHT];
        float pm[FLIGHT], pl[FLIGHT], top = m;
#pragma unroll
        for (int k = 0; k < FLIGHT; ++k) {
            const int s = s0 + k * GROUPS < n ? s0 + k * GROUPS : s0;
            const size_t slot = (size_t)(s == 0 ? item.first : item.next + (s - 1) * item.step) * a.per_wg + i;
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
    const float by = any ? v_scale / total : 0.f;
    uint16_t *o = a.out + item.row * a.out_stride + (long long)head * D + 4 * at;
    *reinterpret_cast<u32x2 *>(o) = u32x2{pack_bf16x2(sum[0] * by, sum[1] * by), pack_bf16x2(sum[2] * by, sum[3] * by)};
    if (a.lse && at == 0) a.lse[(size_t)item.row * a.heads + head] = any ? (top + __builtin_amdgcn_logf(total)) * LN2 : -__builtin_inff();
    if (a.scores && at == 0) sum_of(a.scores + ((size_t)item.row * a.heads + head) * a.score_stride) = RowSum{top, total};
}

template <int D, bool FP8, bool SCORES>
hipError_t launch_attend(const AttendArgs &a, const AttendPlan &p, hipStream_t stream)
{
    auto kernel = p.waves == 1 ? attend_kernel<D, FP8, 1, 1, true, SCORES> : attend_kernel<D, FP8, 1, 4, true, SCORES>;
    if constexpr (D <= 128)
        if (p.waves == 8) kernel = attend_kernel<D, FP8, 1, 8, true, SCORES>;
    if constexpr (FP8) {
        if (p.per_wg > 8) {
            kernel = p.waves == 1 ? attend_kernel<D, true, 1, 1, false, SCORES> : attend_kernel<D, true, 1, 4, false, SCORES>;
            if constexpr (D <= 128) {
                if (p.waves == 8) kernel = attend_kernel<D, true, 1, 8, false, SCORES>;
                if (p.hb == 2) kernel = p.waves == 1 ? attend_kernel<D, true, 2, 1, false, SCORES> : attend_kernel<D, true, 2, 4, false, SCORES>;
            }
        }
    } else {
        if (p.hb == 2) kernel = p.waves == 1 ? attend_kernel<D, false, 2, 1, true, SCORES> : attend_kernel<D, false, 2, 4, true, SCORES>;
    }
    trace_before(KID_ATTEND, stream);
    hipLaunchKernelGGL(kernel, dim3((unsigned)p.grid), dim3(64 * p.waves), 0, stream, a);
    trace_after(KID_ATTEND, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.entries == 0) return e;
    trace_before(KID_ATTEND_JOIN, stream);
    hipLaunchKernelGGL((attend_join_kernel<D, FP8>), dim3((unsigned)(p.entries * (a.group < p.per_wg ? a.group : p.per_wg))),
                       dim3(256), 0, stream, a);
    trace_after(KID_ATTEND_JOIN, stream);
    return hipGetLastError();
}

template <bool SCORES> hipError_t launch_attend(const peqa_kv_cache *C, const AttendArgs &a, const AttendPlan &p, hipStream_t s)
{
    const bool fp8 = C->dtype == PEQA_CACHE_FP8;
    switch (C->head_dim) {
    case 64: return fp8 ? launch_attend<64, true, SCORES>(a, p, s) : launch_attend<64, false, SCORES>(a, p, s);
    case 128: return fp8 ? launch_attend<128, true, SCORES>(a, p, s) : launch_attend<128, false, SCORES>(a, p, s);
    default: return fp8 ? launch_attend<256, true, SCORES>(a, p, s) : launch_attend<256, false, SCORES>(a, p, s);
    }
}

// What the positions were given: weights_out = weights + the sum over a row's heads of a key head, and over the rows of a sequence, of
// 2^(score - log2 of the sum of powers), of the scores that the attention left: a score is known long before its row's sum is, and 4 bytes written
// and read again for a head and a position are less than reading its keys again (where 8 heads share 256 bytes of a key, an eighth).  A workgroup has
// 1024 positions of a key head, four a thread, of the first row with its sequence, and adds the others' after one another, so that no sum
// depends on an order of workgroups.  Bound by memory: 32 rows of up to 8192, 64 heads, 8 key heads  11.4 us for 33 MB of scores, which are
// still cached in part; the attention that writes them takes 125 us for 109.  Rows of one sequence are added by few workgroups, one for 1024 positions and a key
// head: a prompt of 512 tokens with 32 heads on 8 takes 679 us, its attention alone 71, of 2048 4.7 ms (in calls of 256 rows 3.8) for 0.66.
struct WeightArgs {
    const int32_t *lens, *seq;
    const float *scores, *weights;
    float *weights_out;
    long long score_stride, seq_stride, head_stride;
    int rows, heads, kv_heads, group, n_seqs, max_len, window, chunks;
};
constexpr int WEIGHT_POSITIONS = 1024;

template <int FLIGHT> __global__ __launch_bounds__(256) void attend_weights_kernel(WeightArgs a)
{
    unsigned b = blockIdx.x;
    const int chunk = (int)(b % (unsigned)a.chunks);
    b /= (unsigned)a.chunks;
    const int row = (int)(b / (unsigned)a.kv_heads), h = (int)(b - (unsigned)row * (unsigned)a.kv_heads);
    const int seq = a.seq ? a.seq[row] : row, lane = threadIdx.x & 63;
    if (seq < 0 || seq >= a.n_seqs) return;
    if (a.seq) {
        for (int r0 = 0; r0 < row; r0 += 64) {
            const int r = r0 + lane;
            if (__ballot(r < row && a.seq[r < row ? r : 0] == seq) != 0) return;
        }
    }
    const int pos = chunk * WEIGHT_POSITIONS + 4 * (int)threadIdx.x;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    int longest = 0;
    auto add_row = [&](int r) {
        int len = a.lens[r];
        len = len < a.max_len ? len : a.max_len;
        if (len > longest) longest = len;
        const int lo = a.window > 0 && len > a.window ? len - a.window : 0;
        if (pos >= len || pos + 4 <= lo) return;
        const size_t head = (size_t)r * a.heads + (size_t)h * a.group;
        add_given<FLIGHT>(sum, a.scores + head * a.score_stride, a.score_stride, a.group, pos, lo, len);
    };
    add_row(row);
    if (a.seq) {
        for (int r0 = row + 1; r0 < a.rows; r0 += 64) {
            const int r = r0 + lane;
            uint64_t same = __ballot(r < a.rows && a.seq[r < a.rows ? r : row] == seq);
            while (same) {
                add_row(r0 + __builtin_ctzll(same));
                same &= same - 1;
            }
        }
    }
    if (pos >= longest) return;
    const long long at = seq * a.seq_stride + h * a.head_stride;
    store_given(a.weights ? a.weights + at : nullptr, a.weights_out + at, sum, pos, longest);
}

}  // namespace

AttendPlan attend_plan(const peqa_kv_cache *C, int rows, int heads, int max_len, int window)
{
    AttendPlan p{};
    const int group = heads / C->kv_heads, cols = C->dtype == PEQA_CACHE_FP8 && group > 8 ? 16 : 8;
    p.hb = (C->head_dim <= 128 || C->dtype == PEQA_CACHE_BF16) && group > cols ? 2 : 1;    // (16 heads of 256 with 8 bits fill the registers)
    p.per_wg = cols * p.hb;
    p.blocks = (group + p.per_wg - 1) / p.per_wg;
    const long long span = window > 0 && (long long)window + UNIT - 1 < max_len ? (long long)window + UNIT - 1 : max_len;
    const long long items = (long long)rows * C->kv_heads * p.blocks, units = items * ((span + UNIT - 1) / UNIT + START);
    p.grid = items;
    p.waves = 4;
    p.splits = 1;
    p.chunk_units = (int)((span + UNIT - 1) / UNIT);
    if (p.chunk_units < 1) p.chunk_units = 1;
    // Measured, us (lengths are spread from 2 % to 100 % of the longest; "n x kv, group, length"; bf16, head_dim 128 unless stated):
    //   whole items, four waves / one     101 rows x 32, 1, 12 (8 bits)  35.6 / 10.6;  101 x 32, 1, 60  32.5 / 16.6;  40 x 16, 8, 40  10.1 / 7.5;
    //                                     128 x 4, 8, 128 (8 bits, 64)  5.9 / 7.3;  16 x 32, 1, 500  18.7 / 27.8
    //   whole items / shares              64 x 8, 4, 1000  35.7 / 39.1;  128 x 8, 8, 2000 (8 bits)  65 / 69;  16 x 8, 8, 4096  57.3 / 35.6;
    //                                     64 x 8, 8, 8192 (8 bits)  123 / 116
    //   chunks of 128, 256, 512 / whole   8 x 4, 4, 960  8.9, 10.7, 14.2 / 16.9;  1 x 8, 8, 2048  9.2, 10.5, 13.6 / 28.8
    //   chunks of 256, 512 / shares       2 x 8, 8, 8192  17.5, 17.8 / 19.7;  1 x 8, 8, 16384 (8 bits)  15.1, 14.5 / 17.8
    //   chunks of 1024, 512 / shares      16 x 8, 8, 4096  41.5, 41.9 / 35.6;  4 x 8, 8, 32768  69.8, 66.3 / 62.0
    // "up to": lengths spread, "of": all alike:
    //   whole items, four waves / one     82 x 64, 1, up to 151 (8 bits)  66.4 / 28.2;  82 x 64, 1, of 200  108.8 / 104.2;  128 x 8, 8, up to 200 (8
    //                                     bits)  18.1 / 13.9;  63 x 64, 2, up to 250 (256)  163 / 109;  82 x 64, 1, up to 300  89.7 / 85.4;
    //                                     60 x 40, 1, up to 300  47.7 / 47.0;  but 128 x 8, 8, up to 400  30.9 / 32.3;  82 x 64, 1, up to 500  128 / 135
    //   whole items, four waves / eight   1 x 32, 1, of 333  9.0 / 8.4;  4 x 32, 2, up to 500 (8 bits)  9.7 / 8.8;  8 x 16, 4, of 200  8.4 / 8.0
    //   of 256 elements: whole / chunks   14 x 1, 8, up to 465  18.6 / 12.3;  4 x 8, 1, of 400 (8 bits)  12.4 / 9.9;  but 100 x 2, 4, of 400
    //                                     (8 bits)  14.8 / 22.9;  250 x 1, 4, of 500  29.9 / 38.8
    //   of 256 elements, bf16: chunks of 512 / shares  16 x 8, 1, up to 1500  26.7 / 27.7, of 1500  52.6 / 47.7;  20 x 5, 2, of 2000  55.4 / 49.5
    //   heads of 256, bf16, in two workgroups / one with 16 columns twice  4 x 1, 16, of 66436  100 / 69;  50 x 8, 12, of 488  88.8 / 61.7
    const int fit = wgs_per_unit(C->head_dim, C->dtype == PEQA_CACHE_FP8) * PLAN_UNITS;
    // Of bf16 rows of 256 bytes one workgroup has two tiles of every wave, 128 KB of a unit, in flight, which is enough; where a second one
    // has no more items to pass it only makes everything wait longer.  512 / 256 of them: 32 x 8, 8, 4096 (all that long)  109.5 / 102.4;
    // 16 x 8, 8, 4096  36.8 / 35.0;  8 x 32, 1, 8192  98.2 / 100.1;  of 512 items (16 x 32, 1, 2048)  59.9 / 57.7, and of 8 bits 64 x 8, 8, 8192
    // 115.8 / 119.5.
    const int wgs = C->dtype == PEQA_CACHE_BF16 && C->head_dim >= 128 && items <= PLAN_UNITS ? PLAN_UNITS : fit;
    long long slots = 0;
    if (items >= 2 * fit || (items >= fit && span <= 1024) || span <= 256 || (span <= 512 && (C->head_dim <= 128 || items > PLAN_UNITS / 2))) {
        // whole items: many, or of one length, or short.  Of many short ones a wave each; of few all tiles at once, two of each of eight waves
        if (items > fit && span <= (items >= 4 * fit ? 384 : 256)) p.waves = 1;
        else if (span > 128 && span <= 512 && items <= PLAN_UNITS && p.hb == 1 && C->head_dim <= 128) p.waves = 8;
    } else if (rows == 1 || rows > SCAN_ROWS || span * items < (fit == PLAN_UNITS ? 480ll : 960ll) * fit || units >= (1ll << 30)) {
        // chunks: of one row, or as many as there is room for workgroups, of a tile a wave at least
        long long chunk = span * items / wgs;
        chunk = chunk < 128 ? 128 : chunk;
        const long long splits = (span + chunk / 2) / chunk;   // of the longest row, all alike
        p.chunk_units = (int)((span + splits * UNIT - 1) / (splits * UNIT));
        p.splits = (int)((span + p.chunk_units * UNIT - 1) / (p.chunk_units * UNIT));
        p.grid = items * p.splits;
        if (p.splits > 1) {
            p.entries = (int)items;                            // (under 2 fit)
            slots = items * p.splits;
        }
    } else {
        p.shares = wgs;
        p.grid = p.entries = wgs;
        slots = 2 * wgs;
    }
    if (slots > 0) {
        p.part_bytes = round256((size_t)(slots * p.per_wg) * (size_t)C->head_dim * sizeof(float));
        p.ml_bytes = round256((size_t)(slots * p.per_wg) * 2 * sizeof(float));
        p.parts_bytes = round256((size_t)p.entries * sizeof(ItemParts));
    }
    return p;
}

namespace {

peqa_status check_attend(const peqa_kv_cache *C, int32_t rows, int32_t heads, int32_t max_len, int32_t window)
{
    const peqa_status st = peqa_check_cache(C);
    if (st != PEQA_OK) return st;
    if (rows < 1 || heads < 1 || heads > 65536 || heads % C->kv_heads || max_len < 0) return PEQA_ERR_SHAPE;
    if ((int64_t)max_len > (int64_t)C->n_blocks * C->page_size) return PEQA_ERR_SHAPE;
    if (window < 0) return PEQA_ERR_PARAM;
    const AttendPlan p = attend_plan(C, rows, heads, max_len, window);
    if ((int64_t)C->kv_heads * p.blocks * (((int64_t)max_len + UNIT - 1) / UNIT + START) > (1 << 30)) return PEQA_ERR_SHAPE;    // units of a row
    if (p.grid * 64 * p.waves > (int64_t)UINT32_MAX) return PEQA_ERR_SHAPE;    // threads of a launch
    return PEQA_OK;
}

// The arguments that both calls have, checked and, where they are right, in `a`; part_bytes: what the parts of split items need.
peqa_status attend_args(const peqa_kv_cache *C, int32_t rows, int32_t heads, const uint16_t *q, int64_t q_stride, const int32_t *lens,
                        const int32_t *seq, int32_t max_len, int32_t window, float scale, uint16_t *out, int64_t out_stride, float *lse,
                        void *workspace, size_t workspace_bytes, AttendArgs &a, AttendPlan &p)
{
    const peqa_status st = check_attend(C, rows, heads, max_len, window);
    if (st != PEQA_OK) return st;
    if (!q || !lens || !out) return PEQA_ERR_NULL;
    if (!seq && rows > C->n_seqs) return PEQA_ERR_SHAPE;
    const int64_t width = (int64_t)heads * C->head_dim;
    if (q_stride < width || out_stride < width) return PEQA_ERR_SHAPE;
    if (!aligned16(q) || !aligned16(out) || q_stride % 8 || out_stride % 8) return PEQA_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(lens) | reinterpret_cast<uintptr_t>(seq) | reinterpret_cast<uintptr_t>(lse)) & 3) return PEQA_ERR_ALIGN;
    p = attend_plan(C, rows, heads, max_len, window);
    if (p.entries > 0) {
        if (!workspace || workspace_bytes < p.part_bytes + p.ml_bytes + p.parts_bytes) return PEQA_ERR_WORKSPACE;
        if (!aligned16(workspace)) return PEQA_ERR_ALIGN;
    }
    a.cache = cache_args(C);
    a.q = q; a.lens = lens; a.seq = seq; a.out = out; a.lse = lse;
    if (p.entries > 0) {
        char *w = static_cast<char *>(workspace);
        a.part = reinterpret_cast<float *>(w);
        a.part_ml = reinterpret_cast<float *>(w + p.part_bytes);
        a.parts = reinterpret_cast<ItemParts *>(w + p.part_bytes + p.ml_bytes);
    }
    a.q_stride = q_stride; a.out_stride = out_stride;
    a.scale = scale * LOG2E;
    a.rows = rows; a.heads = heads; a.group = heads / C->kv_heads;
    a.max_len = max_len; a.window = window;
    a.blocks = p.blocks; a.per_wg = p.per_wg;
    a.splits = p.splits; a.chunk_units = p.chunk_units; a.shares = p.shares;
    return PEQA_OK;
}

// Room of a call that says what the positions were given, behind the parts' own: scores, and what the rows' sums were in front of them.
struct ScoreRoom {
    size_t parts, scores;
    long long stride;
};
ScoreRoom score_room(const peqa_kv_cache *C, int rows, int heads, int max_len, int window)
{
    const AttendPlan p = attend_plan(C, rows, heads, max_len, window);
    ScoreRoom r{};
    r.stride = (((long long)max_len + 3) & ~3ll) + SUM_ROOM;
    r.parts = p.part_bytes + p.ml_bytes + p.parts_bytes;
    r.scores = round256((size_t)rows * (size_t)heads * (size_t)r.stride * sizeof(float));
    return r;
}

}  // namespace
}  // namespace peqa

extern "C" {

size_t peqa_paged_attention_workspace_bytes(const peqa_kv_cache *C, int32_t rows, int32_t heads, int32_t max_len, int32_t window)
{
    if (peqa::check_attend(C, rows, heads, max_len, window) != PEQA_OK) return 0;
    const peqa::AttendPlan p = peqa::attend_plan(C, rows, heads, max_len, window);
    const size_t bytes = p.part_bytes + p.ml_bytes + p.parts_bytes;
    return bytes ? bytes : 256;                                // (0 would read as "invalid")
}

peqa_status peqa_paged_attention(const peqa_kv_cache *C, int32_t rows, int32_t heads, const uint16_t *q, int64_t q_stride,
                                 const int32_t *lens, const int32_t *seq, int32_t max_len, int32_t window, float scale, uint16_t *out,
                                 int64_t out_stride, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    peqa::AttendArgs a{};
    peqa::AttendPlan p{};
    const peqa_status st = peqa::attend_args(C, rows, heads, q, q_stride, lens, seq, max_len, window, scale, out, out_stride, lse, workspace,
                                             workspace_bytes, a, p);
    if (st != PEQA_OK) return st;
    return dev_status(peqa::launch_attend<false>(C, a, p, static_cast<hipStream_t>(stream)));
}

size_t peqa_paged_attention_weights_workspace_bytes(const peqa_kv_cache *C, int32_t rows, int32_t heads, int32_t max_len, int32_t window)
{
    if (peqa::check_attend(C, rows, heads, max_len, window) != PEQA_OK) return 0;
    const peqa::ScoreRoom r = peqa::score_room(C, rows, heads, max_len, window);
    return r.parts + r.scores;
}

peqa_status peqa_paged_attention_weights(const peqa_kv_cache *C, int32_t rows, int32_t heads, const uint16_t *q, int64_t q_stride,
                                         const int32_t *lens, const int32_t *seq, int32_t max_len, int32_t window, float scale, uint16_t *out,
                                         int64_t out_stride, float *lse, const float *weights, float *weights_out,
                                         int64_t weights_seq_stride, int64_t weights_head_stride, void *workspace, size_t workspace_bytes,
                                         void *stream)
{
    peqa_status st = peqa::check_attend(C, rows, heads, max_len, window);
    if (st != PEQA_OK) return st;
    if (!weights_out) return PEQA_ERR_NULL;
    if (!aligned16(weights) || !aligned16(weights_out) || weights_head_stride % 4 || weights_seq_stride % 4) return PEQA_ERR_ALIGN;
    if (!peqa::weights_apart(C, max_len, weights_seq_stride, weights_head_stride)) return PEQA_ERR_SHAPE;
    const peqa::ScoreRoom r = peqa::score_room(C, rows, heads, max_len, window);
    const long long chunks = ((long long)max_len + peqa::WEIGHT_POSITIONS - 1) / peqa::WEIGHT_POSITIONS;
    if (chunks * rows * C->kv_heads > (1 << 23)) return PEQA_ERR_SHAPE;       // workgroups of a launch
    if (!workspace || workspace_bytes < r.parts + r.scores) return PEQA_ERR_WORKSPACE;
    if (!aligned16(workspace)) return PEQA_ERR_ALIGN;
    char *w = static_cast<char *>(workspace);
    peqa::AttendArgs a{};
    peqa::AttendPlan p{};
    st = peqa::attend_args(C, rows, heads, q, q_stride, lens, seq, max_len, window, scale, out, out_stride, lse, workspace, workspace_bytes, a, p);
    if (st != PEQA_OK) return st;
    a.scores = reinterpret_cast<float *>(w + r.parts) + peqa::SUM_ROOM;
    a.score_stride = r.stride;
    // An item that one workgroup has is finished there, without a launch of its own (1 row x 32, 1, of 333  10.5 us, 12.4 with; 16 x 32, 1, of 500
    // 26.1, 28.5;  64 x 8, 8, up to 1000 (8 bits)  23.0, 26.8;  128 x 8, 8, up to 400  32.5, 34.8); rows of one sequence add to the same sums.
    const bool within = !seq && p.blocks == 1 && p.splits == 1 && p.shares == 0;
    if (within) {
        a.weights = weights; a.weights_out = weights_out;
        a.weights_seq_stride = weights_seq_stride; a.weights_head_stride = weights_head_stride;
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = peqa::launch_attend<true>(C, a, p, s);
    if (e != hipSuccess || chunks == 0 || within) return dev_status(e);
    peqa::WeightArgs g{};
    g.lens = lens; g.seq = seq; g.scores = a.scores; g.weights = weights; g.weights_out = weights_out;
    g.score_stride = r.stride; g.seq_stride = weights_seq_stride; g.head_stride = weights_head_stride;
    g.rows = rows; g.heads = heads; g.kv_heads = C->kv_heads; g.group = a.group; g.n_seqs = C->n_seqs;
    g.max_len = max_len; g.window = window; g.chunks = (int)chunks;
    peqa::trace_before(peqa::KID_ATTEND_WEIGHTS, s);
    // Few workgroups have more in flight each (both calls, us, four heads / two: 1 row of 30000, 8 key heads x 8 32.4, 33.7;  16 rows of up to 4096
    // 37.1, 38.2;  32 of up to 8192 145.4, 142.9)
    const long long wgs = chunks * rows * C->kv_heads;
    auto kernel = a.group == 1 ? peqa::attend_weights_kernel<1> : wgs <= 4 * peqa::PLAN_UNITS ? peqa::attend_weights_kernel<4> : peqa::attend_weights_kernel<2>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(256), 0, s, g);
    peqa::trace_after(peqa::KID_ATTEND_WEIGHTS, s);
    return dev_status(hipGetLastError());
}

}  // extern "C"
