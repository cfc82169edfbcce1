// Positions that leave the paged cache (peqa_cache_evict): of a sequence and a key head the first `sinks`, the last `recent` and, of those
// between, the ones with the largest weights stay, in order, at the first `keep` places.
#include "peqa_cache.h"
#include "peqa_host.h"

using namespace peqa::host;

namespace peqa {

namespace {

struct EvictArgs {
    CacheArgs from, to;
    const int32_t *seq, *lens;
    const float *weights;
    float *weights_out;
    long long seq_stride, head_stride;     // of both, in elements
    int32_t *kept, *new_lens;              // [n, kv_heads, keep]; new_lens or null
    int32_t *moved;                        // [n] positions that an entry keeps and the move kernel looks at
    int n, max_len, keep, sinks, recent;
    int splits, chunks, chunk;             // of the move: workgroups for the bytes of a position, for the positions of a head, and positions of one
    int row_bytes;                         // bytes of a head's position
    bool in_place;
};

// A sequence's entry: the sequence, its length, and whether an earlier entry has the same one (uniform in a workgroup).
struct Entry {
    int seq, len;
    bool again;
};
__device__ __forceinline__ Entry entry_of(const EvictArgs &a, int i)
{
    Entry e;
    e.seq = a.seq ? a.seq[i] : i;
    e.again = false;
    int first = i;
    if (a.seq) {
        // the first entry with this sequence (in one pass: entries are few)
        __shared__ int least;
        if (threadIdx.x == 0) least = i;
        __syncthreads();
        for (int j = threadIdx.x; j < i; j += blockDim.x)
            if (a.seq[j] == e.seq) atomicMin(&least, j);
        __syncthreads();
        first = least;
        e.again = first < i;
    }
    e.len = a.lens[first];
    e.len = e.len < a.max_len ? e.len : a.max_len;
    if (e.seq < 0 || e.seq >= a.from.n_seqs || e.len < 0) { e.len = 0; e.seq = 0; }
    return e;
}

// A weight's place in the order: larger is kept; NaN is less than everything, the two zeros are the same.
__device__ __forceinline__ uint32_t order_of(float w)
{
    const uint32_t b = __float_as_uint(w + 0.f);
    return w != w ? 0u : b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}

// One workgroup for a sequence and a key head.  The least weight that stays is found digit by digit, 11, 11 and 10 bits, each by a
// histogram of the weights that have the digits found so far (counts: no order of adding matters); then, as many positions as there
// are threads at a time and in order, those above it and as many equal ones as there is room for get their places.  A sort would move every weight
// log n times for an order among those that stay that nobody asks for.  Bound by the latency of its barriers, three for a digit and one for
// as many positions as there are threads: 8 heads of 1501 positions 7.0 us, 512 of up to 2048 10 us, 8 of 30000 47.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void evict_select_kernel(EvictArgs a)
{
    constexpr int WAVES = THREADS / 64, OWN = 2048 / THREADS;
    constexpr int FIRST = 4096 / THREADS, FLIGHT = 8;      // weights of a thread that stay in registers; of the others, in flight
    __shared__ __attribute__((aligned(16))) uint32_t bins[3][2048];       // of a pass each
    __shared__ uint32_t scan[2][WAVES][2];
    __shared__ uint32_t found[3][2];                       // the digit, and how many of its weights stay
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int i = (int)(blockIdx.x / (unsigned)a.from.kv_heads), h = (int)blockIdx.x - i * a.from.kv_heads;
    const Entry e = entry_of(a, i);
    const int stays = e.len < a.keep ? e.len : a.keep;
    int32_t *kept = a.kept + ((size_t)i * a.from.kv_heads + h) * (size_t)a.keep;
    if (h == 0 && tid == 0) {
        if (a.new_lens) a.new_lens[i] = stays;
        a.moved[i] = e.again ? 0 : stays;
    }
    if (e.again || e.len == 0) {
        for (int j = tid; j < a.keep; j += THREADS) kept[j] = -1;
        return;
    }
    for (int j = tid; j < 3 * 512; j += THREADS) reinterpret_cast<u32x4 *>(bins)[j] = u32x4{0, 0, 0, 0};
    const float *in = a.weights + e.seq * a.seq_stride + h * a.head_stride;
    float *out = a.weights_out + e.seq * a.seq_stride + h * a.head_stride;
    const int lo = a.sinks, hi = e.len - a.recent;         // those that have to be chosen from, where some leave
    const bool all = e.len <= a.keep;
    // the first weights' orders stay in registers over the passes, the others (past 4096 positions) are read again
    uint32_t order[FIRST];
    float first_w[FIRST];
#pragma unroll
    for (int k = 0; k < FIRST; ++k) {
        const int j = k * THREADS + tid;
        first_w[k] = j < e.len ? in[j] : 0.f;
        order[k] = order_of(first_w[k]);
    }
    uint32_t least = 0, equal = 0;                         // the least order that stays, and how many of it
    if (!all) {
        __syncthreads();                                   // (the bins are empty)
        uint32_t room = (uint32_t)(a.keep - a.sinks - a.recent), known = 0, mask = 0;
        if (room == 0) {
            least = 0xFFFFFFFFu;                           // (of NaN only, which no weight has)
        } else {
#pragma unroll 1
            for (int pass = 0; pass < 3; ++pass) {
                const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, digits = pass == 2 ? 1024 : 2048;
                auto count = [&](int j, uint32_t o) {
                    if (j >= lo && j < hi && (o & mask) == known) atomicAdd(&bins[pass][(o >> shift) & (digits - 1)], 1u);
                };
#pragma unroll
                for (int k = 0; k < FIRST; ++k) count(k * THREADS + tid, order[k]);
                for (int j0 = FIRST * THREADS + tid; j0 < hi; j0 += FLIGHT * THREADS) {
                    float w[FLIGHT];
#pragma unroll
                    for (int k = 0; k < FLIGHT; ++k) w[k] = in[j0 + k * THREADS < hi ? j0 + k * THREADS : j0];
#pragma unroll
                    for (int k = 0; k < FLIGHT; ++k) count(j0 + k * THREADS, order_of(w[k]));
                }
                __syncthreads();
                // from the top: thread t has the OWN digits up to 2047 - OWN t
                uint32_t own[OWN], mine = 0;
#pragma unroll
                for (int d = 0; d < OWN; ++d) {
                    own[d] = bins[pass][2047 - OWN * tid - d];
                    mine += own[d];
                }
                uint32_t upto = mine;
#pragma unroll
                for (int o = 1; o < 64; o *= 2) {
                    const uint32_t other = __shfl_up(upto, o);
                    if (lane >= o) upto += other;
                }
                if (lane == 63) scan[0][wave][0] = upto;
                __syncthreads();
                uint32_t before = upto - mine;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) before += w < wave ? scan[0][w][0] : 0;
                if (before < room && room <= before + mine) {
#pragma unroll
                    for (int d = 0; d < OWN; ++d) {
                        if (before < room && room <= before + own[d]) {
                            found[pass][0] = 2047 - OWN * tid - d;
                            found[pass][1] = room - before;
                        }
                        before += own[d];
                    }
                }
                __syncthreads();
                known |= found[pass][0] << shift;
                mask |= (uint32_t)(digits - 1) << shift;
                room = found[pass][1];
            }
            least = known;
            equal = room;
        }
    }
    uint32_t larger_before = 0, equal_before = 0;
    auto place = [&](int from, int k, float w, uint32_t o) __attribute__((always_inline)) {
        const int j = from + tid;
        const bool held = all || j < lo || j >= hi;
        const bool is_larger = j < e.len && (held || o > least), is_equal = j < e.len && !held && o == least;
        const uint64_t larger = __ballot(is_larger), same = __ballot(is_equal), below = (1ull << lane) - 1;
        if (lane == 0) {
            scan[k][wave][0] = (uint32_t)__popcll(larger);
            scan[k][wave][1] = (uint32_t)__popcll(same);
        }
        __syncthreads();                                   // (and every weight of these positions is read: they may be overwritten)
        uint32_t l = larger_before + (uint32_t)__popcll(larger & below), q = equal_before + (uint32_t)__popcll(same & below);
#pragma unroll
        for (int v = 0; v < WAVES; ++v) {
            const uint32_t nl = scan[k][v][0], nq = scan[k][v][1];
            l += v < wave ? nl : 0;
            q += v < wave ? nq : 0;
            larger_before += nl;
            equal_before += nq;
        }
        if (is_larger || (is_equal && q < equal)) {
            const uint32_t at = l + (q < equal ? q : equal);
            kept[at] = j;
            out[at] = w;
        }
    };
#pragma unroll
    for (int k = 0; k < FIRST; ++k)
        if (k * THREADS < e.len) place(k * THREADS, k & 1, first_w[k], order[k]);
    for (int from = FIRST * THREADS; from < e.len; from += FLIGHT * THREADS) {
        float w[FLIGHT];                                   // (read before any of their places is written)
#pragma unroll
        for (int k = 0; k < FLIGHT; ++k) w[k] = from + k * THREADS + tid < e.len ? in[from + k * THREADS + tid] : 0.f;
#pragma unroll
        for (int k = 0; k < FLIGHT; ++k)
            if (from + k * THREADS < e.len) place(from + k * THREADS, k & 1, w[k], order_of(w[k]));
    }
    __syncthreads();
    for (int j = stays + tid; j < a.keep; j += THREADS) kept[j] = -1;
    for (int j = stays + tid; j < a.max_len; j += THREADS) out[j] = 0.f;
}

constexpr int SECTION = 1024;          // positions whose places are looked up at a time
// Positions that a thread has in flight.  (Both kernels, us.  Large workgroups with 2, 4, 6, 8: 1 x 8 heads, 1501 -> 1001 14.1, 13.7, 14.4, 15.3;  30000 ->
// 20000 162, 141, 147, 181;  25 x 8, 2000 -> 1000 27, 30, 31, 41;  small ones with 4, 8: 16 x 32, 2048 -> 1024 68, 60.)
constexpr int each_of(int threads) { return threads > 512 ? 4 : 8; }

// Keys or values of a sequence and a key head, or some of the bytes of each, to their places.  Where they come from and go to is found for a
// section first (two loads after one another for all of it); then the next positions' bytes are asked for before the present ones are stored.
// In place a workgroup goes over all positions in order: no position moves up, so what is written lies at or below what the
// workgroup has read when it writes, what is read next lies above, and no other workgroup has these bytes.  To another cache the positions
// are split over workgroups too.
// Bound by memory where there are many heads: 16 sequences x 32 heads of up to 2048 positions to 1024 53.8 us, 4.5 TB/s of what moves; by what
// a workgroup has in flight between two barriers where there are few: 8 heads of 1501 to 1001 6.2 us, of 30000 to 20000 95
// (32 workgroups, 55 GB/s of what moves each: a place must not be written before all that was there is read).
template <int THREADS>
__global__ __launch_bounds__(THREADS) void evict_move_kernel(EvictArgs a)
{
    constexpr int EACH = each_of(THREADS);
    __shared__ long long from_at[SECTION], to_at[SECTION];  // in bytes; -1: from nowhere (zeros), to nowhere
    unsigned b = blockIdx.x;
    const int chunk = (int)(b % (unsigned)a.chunks);
    b /= (unsigned)a.chunks;
    const int split = (int)(b % (unsigned)a.splits);
    b /= (unsigned)a.splits;
    const bool is_v = b & 1;
    b >>= 1;
    const int i = (int)(b / (unsigned)a.from.kv_heads), h = (int)(b - (unsigned)i * (unsigned)a.from.kv_heads);
    const int32_t *kept = a.kept + ((size_t)i * a.from.kv_heads + h) * (size_t)a.keep;
    const int first = chunk * a.chunk;
    // (the first section's, asked for before it is known how many there are)
    int32_t old_at[SECTION / THREADS];
#pragma unroll
    for (int k = 0; k < SECTION / THREADS; ++k) {
        const int j = first + k * THREADS + (int)threadIdx.x;
        old_at[k] = j < a.keep ? kept[j] : -1;
    }
    const int n = a.moved[i], seq = a.seq ? a.seq[i] : i;
    const int bytes = a.row_bytes / a.splits, lanes = bytes / 16, rows = THREADS / lanes;
    const int row = (int)threadIdx.x / lanes, at = split * bytes + 16 * ((int)threadIdx.x - row * lanes);
    const int step = EACH * rows;
    const uint8_t *src = static_cast<const uint8_t *>(is_v ? a.from.v : a.from.k) + h * a.from.head_stride + at;
    uint8_t *dst = static_cast<uint8_t *>(is_v ? a.to.v : a.to.k) + h * a.to.head_stride + at;
    const int32_t *table = a.from.table + seq * a.from.table_stride, *to_table = a.to.table + seq * a.to.table_stride;
    const int until = a.in_place ? n : first + a.chunk < n ? first + a.chunk : n;
    for (int j0 = first; j0 < until; j0 += SECTION) {
        const int count = until - j0 < SECTION ? until - j0 : SECTION;
        if (j0 > first) __syncthreads();                    // (the last section's places have been read)
#pragma unroll
        for (int k = 0; k < SECTION / THREADS; ++k) {
            const int u = k * THREADS + (int)threadIdx.x, j = j0 + u;
            if (u < count) {
                const int old = j0 == first ? old_at[k] : kept[j];
                const bool moves = old >= 0 && !(a.in_place && old == j);
                const int page = moves ? table[old >> a.from.page_shift] : -1, goal = moves ? to_table[j >> a.to.page_shift] : -1;
                const bool there = page >= 0 && page < a.from.n_pages, room = goal >= 0 && goal < a.to.n_pages;
                from_at[u] = there ? page * a.from.page_stride + (old & a.from.page_mask) * a.from.slot_stride : -1ll;
                to_at[u] = room ? goal * a.to.page_stride + (j & a.to.page_mask) * a.to.slot_stride : -1ll;
            }
        }
        __syncthreads();
        u32x4 x[EACH], y[EACH];
        auto read = [&](u32x4 (&x)[EACH], int u0) __attribute__((always_inline)) {
#pragma unroll
            for (int k = 0; k < EACH; ++k) {
                const int u = u0 + k * rows + row;
                x[k] = u32x4{0, 0, 0, 0};
                const long long from = u < count ? from_at[u] : -1ll;
                if (from >= 0) x[k] = *reinterpret_cast<const u32x4 *>(src + from);
            }
        };
        read(x, 0);
        for (int u0 = 0; u0 < count; u0 += step) {
            if (a.in_place) {
                // every thread has what it read
#pragma unroll
                for (int k = 0; k < EACH; ++k) asm volatile("" : "+v"(x[k]));
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                __syncthreads();
            }
            read(y, u0 + step);
#pragma unroll
            for (int k = 0; k < EACH; ++k) {
                const int u = u0 + k * rows + row;
                const long long to = u < count ? to_at[u] : -1ll;
                if (to >= 0) *reinterpret_cast<u32x4 *>(dst + to) = x[k];
            }
#pragma unroll
            for (int k = 0; k < EACH; ++k) x[k] = y[k];
        }
    }
}

struct EvictPlan {
    size_t kept_bytes, moved_bytes;
    bool few;                              // heads in place: large workgroups of the move, `splits` for a position's bytes
    int splits, chunks, chunk;             // of the move
};
EvictPlan evict_plan(const peqa_kv_cache *C, int n, int max_len, int keep, bool in_place)
{
    EvictPlan p{};
    const int heads = n * C->kv_heads, most = max_len < keep ? max_len : keep;
    const int row_bytes = C->head_dim * (C->dtype == PEQA_CACHE_FP8 ? 1 : 2);
    // In place a head's positions are one workgroup's, or its lines': of few heads 16 waves that have 128 bytes of each, which keep more in flight.
    // (us, and as of many heads: 1 x 8 heads, 1501 -> 1001 positions 14.6, 23.5;  5 x 8, 3000 -> 2000 22, 45;  2 x 8 of 256 elements, 6000 -> 4000
    // 39, 138;  25 x 8, 2000 -> 1000 30.6, 31.7;  40 x 8 43.9, 44.2;  64 x 8 of 64 bytes 30.9, 27.6.  Pieces of 64 bytes 14.7, 23.5, 39.3, 41.7.  To
    // another cache 2 x 8 of 256 elements 46.7, 41.9;  4 x 8 20.2, 18.6.)
    p.few = in_place && heads < PLAN_UNITS;
    p.splits = p.few && row_bytes > 128 ? row_bytes / 128 : 1;
    // to another cache a step each, or, of many heads, up to a section
    const int threads = p.few ? 1024 : 256, step = each_of(threads) * (threads * 16 * p.splits / row_bytes);
    long long chunk = in_place ? SECTION : (long long)most * heads * 2 * p.splits / (8 * PLAN_UNITS) / step * step;
    chunk = chunk < step ? step : chunk > SECTION ? SECTION : chunk;
    p.chunk = (int)chunk;
    p.chunks = in_place ? 1 : (int)((most + chunk - 1) / chunk);
    if (p.chunks < 1) p.chunks = 1;
    p.kept_bytes = round256((size_t)n * (size_t)C->kv_heads * (size_t)keep * sizeof(int32_t));
    p.moved_bytes = round256((size_t)n * sizeof(int32_t));
    return p;
}

peqa_status check_evict(const peqa_kv_cache *C, int32_t n, int32_t max_len, int32_t keep)
{
    const peqa_status st = peqa_check_cache(C);
    if (st != PEQA_OK) return st;
    if (n < 1 || max_len < 0 || (int64_t)max_len > (int64_t)C->n_blocks * C->page_size) return PEQA_ERR_SHAPE;
    if (keep < 1 || keep > (1 << 30)) return PEQA_ERR_PARAM;
    if ((int64_t)n * C->kv_heads > (1 << 20)) return PEQA_ERR_SHAPE;          // workgroups of a launch, here and of the move
    const EvictPlan p = evict_plan(C, n, max_len, keep, false);
    if ((int64_t)n * C->kv_heads * 2 * p.splits * p.chunks > (1 << 23)) return PEQA_ERR_SHAPE;
    return PEQA_OK;
}

// Strides in bytes, as the move takes them.
CacheArgs in_bytes(const peqa_kv_cache *C)
{
    CacheArgs a = cache_args(C);
    const int el = C->dtype == PEQA_CACHE_FP8 ? 1 : 2;
    a.page_stride *= el;
    a.head_stride *= el;
    a.slot_stride *= el;
    return a;
}

}  // namespace
}  // namespace peqa

extern "C" {

size_t peqa_cache_evict_workspace_bytes(const peqa_kv_cache *C, int32_t n, int32_t max_len, int32_t keep)
{
    if (peqa::check_evict(C, n, max_len, keep) != PEQA_OK) return 0;
    const peqa::EvictPlan p = peqa::evict_plan(C, n, max_len, keep, true);
    return p.kept_bytes + p.moved_bytes;
}

peqa_status peqa_cache_evict(const peqa_kv_cache *C, const peqa_kv_cache *to, int32_t n, const int32_t *seq, const int32_t *lens, int32_t max_len,
                             const float *weights, float *weights_out, int64_t weights_seq_stride, int64_t weights_head_stride, int32_t keep,
                             int32_t sinks, int32_t recent, int32_t *kept, int32_t *new_lens, void *workspace, size_t workspace_bytes,
                             void *stream)
{
    peqa_status st = peqa::check_evict(C, n, max_len, keep);
    if (st != PEQA_OK) return st;
    const bool in_place = !to || (to->table == C->table && to->k == C->k && to->v == C->v);
    if (to) {
        st = peqa_check_cache(to);
        if (st != PEQA_OK) return st;
        if (to->kv_heads != C->kv_heads || to->head_dim != C->head_dim || to->n_seqs != C->n_seqs) return PEQA_ERR_SHAPE;
        if (to->dtype != C->dtype) return PEQA_ERR_PARAM;
        if ((int64_t)to->n_blocks * to->page_size < (max_len < keep ? max_len : keep)) return PEQA_ERR_SHAPE;
        if (in_place && (to->page_size != C->page_size || to->page_stride != C->page_stride || to->head_stride != C->head_stride ||
                         to->slot_stride != C->slot_stride || to->table_stride != C->table_stride))
            return PEQA_ERR_PARAM;                         // the same places by other numbers
    }
    if (!lens || !weights || !weights_out) return PEQA_ERR_NULL;
    if (!seq && n > C->n_seqs) return PEQA_ERR_SHAPE;
    if (sinks < 0 || recent < 0 || (int64_t)sinks + recent > keep) return PEQA_ERR_PARAM;
    if (!peqa::weights_apart(C, max_len, weights_seq_stride, weights_head_stride)) return PEQA_ERR_SHAPE;
    if ((reinterpret_cast<uintptr_t>(lens) | reinterpret_cast<uintptr_t>(seq) | reinterpret_cast<uintptr_t>(weights) |
         reinterpret_cast<uintptr_t>(weights_out) | reinterpret_cast<uintptr_t>(kept) | reinterpret_cast<uintptr_t>(new_lens)) & 3)
        return PEQA_ERR_ALIGN;
    const intptr_t behind = (intptr_t)new_lens - (intptr_t)lens;
    if (new_lens && behind < n * 4ll && -behind < n * 4ll) return PEQA_ERR_PARAM;             // (the heads' workgroups read lens)
    const peqa::EvictPlan p = peqa::evict_plan(C, n, max_len, keep, in_place);
    if (!workspace || workspace_bytes < p.kept_bytes + p.moved_bytes) return PEQA_ERR_WORKSPACE;
    if (!aligned16(workspace)) return PEQA_ERR_ALIGN;
    char *w = static_cast<char *>(workspace);
    peqa::EvictArgs a{};
    a.from = peqa::in_bytes(C);
    a.to = peqa::in_bytes(in_place ? C : to);
    a.seq = seq; a.lens = lens; a.weights = weights; a.weights_out = weights_out;
    a.seq_stride = weights_seq_stride; a.head_stride = weights_head_stride;
    a.kept = kept ? kept : reinterpret_cast<int32_t *>(w);
    a.moved = reinterpret_cast<int32_t *>(w + p.kept_bytes);
    a.new_lens = new_lens;
    a.n = n; a.max_len = max_len; a.keep = keep; a.sinks = sinks; a.recent = recent;
    a.in_place = in_place;
    a.row_bytes = C->head_dim * (C->dtype == PEQA_CACHE_FP8 ? 1 : 2);
    const int heads = n * C->kv_heads;
    a.splits = p.splits;
    a.chunk = p.chunk;
    a.chunks = p.chunks;
    hipStream_t s = static_cast<hipStream_t>(stream);
    peqa::trace_before(peqa::KID_EVICT_SELECT, s);
    // (512 and 1024 threads, us: 16 x 32 heads of up to 2048 positions 8.5 and 12.6, 512 of 300 5.8 and 11.7;  8 of 30000 77 and 58 with a weight of a
    // thread in flight)
    const bool many = max_len > 4096;
    hipLaunchKernelGGL((many ? peqa::evict_select_kernel<1024> : peqa::evict_select_kernel<512>), dim3((unsigned)heads), dim3(many ? 1024 : 512), 0, s, a);
    peqa::trace_after(peqa::KID_EVICT_SELECT, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return dev_status(e);
    peqa::trace_before(peqa::KID_EVICT_MOVE, s);
    auto move = p.few ? peqa::evict_move_kernel<1024> : peqa::evict_move_kernel<256>;
    hipLaunchKernelGGL(move, dim3((unsigned)heads * 2u * (unsigned)a.splits * (unsigned)a.chunks), dim3(p.few ? 1024 : 256), 0, s, a);
    peqa::trace_after(peqa::KID_EVICT_MOVE, s);
    return dev_status(hipGetLastError());
}

}  // extern "C"
