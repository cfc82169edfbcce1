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
    int splits, chunks;                    // of the move: workgroups for the bytes of a position, and for the positions of a head
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

constexpr int SELECT_THREADS = 1024, WAVES = SELECT_THREADS / 64;

// One workgroup for a sequence and a key head.  The least weight that stays is found digit by digit, 11, 11 and 10 bits, each by a
// histogram of the weights that have the digits found so far (counts: no order of adding matters); then, 1024 positions at a time and
// in order, those above it and as many equal ones as there is room for get their places.
__global__ __launch_bounds__(SELECT_THREADS) void evict_select_kernel(EvictArgs a)
{
    __shared__ uint32_t bins[2048];
    __shared__ uint32_t scan[2][WAVES][2];
    __shared__ uint32_t found[2];                          // the digit, and how many of its weights stay
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
        for (int j = tid; j < a.keep; j += SELECT_THREADS) kept[j] = -1;
        return;
    }
    const float *in = a.weights + e.seq * a.seq_stride + h * a.head_stride;
    float *out = a.weights_out + e.seq * a.seq_stride + h * a.head_stride;
    const int lo = a.sinks, hi = e.len - a.recent;         // those that have to be chosen from, where some leave
    const bool all = e.len <= a.keep;
    uint32_t least = 0, equal = 0;                         // the least order that stays, and how many of it
    if (!all) {
        uint32_t room = (uint32_t)(a.keep - a.sinks - a.recent), known = 0, mask = 0;
        if (room == 0) {
            least = 0xFFFFFFFFu;                           // (of NaN only, which no weight has)
        } else {
#pragma unroll 1
            for (int pass = 0; pass < 3; ++pass) {
                const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, digits = pass == 2 ? 1024 : 2048;
                for (int j = tid; j < 2048; j += SELECT_THREADS) bins[j] = 0;
                __syncthreads();
                for (int j = lo + tid; j < hi; j += SELECT_THREADS) {
                    const uint32_t o = order_of(in[j]);
                    if ((o & mask) == known) atomicAdd(&bins[(o >> shift) & (digits - 1)], 1u);
                }
                __syncthreads();
                // from the top: thread t has the digits 2047 - 2 t and 2046 - 2 t
                const uint32_t high = bins[2047 - 2 * tid], low = bins[2046 - 2 * tid];
                uint32_t upto = high + low;
#pragma unroll
                for (int o = 1; o < 64; o *= 2) {
                    const uint32_t other = __shfl_up(upto, o);
                    if (lane >= o) upto += other;
                }
                if (lane == 63) scan[0][wave][0] = upto;
                __syncthreads();
                uint32_t before = upto - high - low;
                for (int w = 0; w < wave; ++w) before += scan[0][w][0];
                if (before < room && room <= before + high + low) {
                    const bool first = room <= before + high;
                    found[0] = first ? 2047 - 2 * tid : 2046 - 2 * tid;
                    found[1] = first ? room - before : room - before - high;
                }
                __syncthreads();
                known |= found[0] << shift;
                mask |= (uint32_t)(digits - 1) << shift;
                room = found[1];
                __syncthreads();
            }
            least = known;
            equal = room;
        }
    }
    uint32_t larger_before = 0, equal_before = 0;
    for (int from = 0, k = 0; from < e.len; from += SELECT_THREADS, k ^= 1) {
        const int j = from + tid;
        const float w = j < e.len ? in[j] : 0.f;
        const bool held = all || j < lo || j >= hi;
        const uint32_t o = order_of(w);
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
    }
    __syncthreads();
    for (int j = stays + tid; j < a.keep; j += SELECT_THREADS) kept[j] = -1;
    for (int j = stays + tid; j < a.max_len; j += SELECT_THREADS) out[j] = 0.f;
}

constexpr int MOVE_THREADS = 256, EACH = 4;                // positions that a thread has in flight

// Keys or values of a sequence and a key head, or some of the bytes of each, to their places.  In place a workgroup goes over all
// positions in order: no position moves up, so what is written lies at or below what the workgroup has read, and no other workgroup has
// these bytes.  To another cache the positions are split over workgroups too.
__global__ __launch_bounds__(MOVE_THREADS) void evict_move_kernel(EvictArgs a)
{
    unsigned b = blockIdx.x;
    const int chunk = (int)(b % (unsigned)a.chunks);
    b /= (unsigned)a.chunks;
    const int split = (int)(b % (unsigned)a.splits);
    b /= (unsigned)a.splits;
    const bool is_v = b & 1;
    b >>= 1;
    const int i = (int)(b / (unsigned)a.from.kv_heads), h = (int)(b - (unsigned)i * (unsigned)a.from.kv_heads);
    const int n = a.moved[i], seq = a.seq ? a.seq[i] : i;
    const int bytes = a.row_bytes / a.splits, lanes = bytes / 16, rows = MOVE_THREADS / lanes;
    const int row = (int)threadIdx.x / lanes, at = split * bytes + 16 * ((int)threadIdx.x - row * lanes);
    const int step = EACH * rows;
    const int32_t *kept = a.kept + ((size_t)i * a.from.kv_heads + h) * (size_t)a.keep;
    const uint8_t *src = static_cast<const uint8_t *>(is_v ? a.from.v : a.from.k) + h * a.from.head_stride + at;
    uint8_t *dst = static_cast<uint8_t *>(is_v ? a.to.v : a.to.k) + h * a.to.head_stride + at;
    const int32_t *table = a.from.table + seq * a.from.table_stride, *to_table = a.to.table + seq * a.to.table_stride;
    for (int j0 = chunk * step; j0 < n; j0 += a.chunks * step) {
        u32x4 x[EACH];
        int goal[EACH];
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            const int j = j0 + k * rows + row;
            const int old = j < n ? kept[j] : -1;
            goal[k] = old < 0 || (a.in_place && old == j) ? -1 : j;
            x[k] = u32x4{0, 0, 0, 0};
            if (goal[k] >= 0) {
                const int page = table[old >> a.from.page_shift];
                if (page >= 0 && page < a.from.n_pages)
                    x[k] = *reinterpret_cast<const u32x4 *>(src + page * a.from.page_stride + (old & a.from.page_mask) * a.from.slot_stride);
            }
        }
        if (a.in_place) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
        }
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            if (goal[k] < 0) continue;
            const int page = to_table[goal[k] >> a.to.page_shift];
            if (page >= 0 && page < a.to.n_pages)
                *reinterpret_cast<u32x4 *>(dst + page * a.to.page_stride + (goal[k] & a.to.page_mask) * a.to.slot_stride) = x[k];
        }
    }
}

struct EvictPlan {
    size_t kept_bytes, moved_bytes;
};
EvictPlan evict_plan(const peqa_kv_cache *C, int n, int keep)
{
    EvictPlan p{};
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
    if ((int64_t)n * C->kv_heads > (1 << 20)) return PEQA_ERR_SHAPE;          // workgroups of a launch
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
    const peqa::EvictPlan p = peqa::evict_plan(C, n, keep);
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
    if (new_lens == lens) return PEQA_ERR_PARAM;           // (the heads' workgroups read it)
    if (weights_head_stride < max_len || weights_seq_stride < max_len) return PEQA_ERR_SHAPE;
    if ((reinterpret_cast<uintptr_t>(lens) | reinterpret_cast<uintptr_t>(seq) | reinterpret_cast<uintptr_t>(weights) |
         reinterpret_cast<uintptr_t>(weights_out) | reinterpret_cast<uintptr_t>(kept) | reinterpret_cast<uintptr_t>(new_lens)) & 3)
        return PEQA_ERR_ALIGN;
    const peqa::EvictPlan p = peqa::evict_plan(C, n, keep);
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
    const int heads = n * C->kv_heads, most = max_len < keep ? max_len : keep;
    a.splits = a.row_bytes >= 256 && heads < peqa::PLAN_UNITS ? a.row_bytes / 128 : 1;
    const int step = peqa::EACH * (peqa::MOVE_THREADS * 16 * a.splits / a.row_bytes);
    a.chunks = in_place ? 1 : (most + step - 1) / step;
    if (a.chunks < 1) a.chunks = 1;
    hipStream_t s = static_cast<hipStream_t>(stream);
    peqa::trace_before(peqa::KID_EVICT_SELECT, s);
    hipLaunchKernelGGL(peqa::evict_select_kernel, dim3((unsigned)heads), dim3(peqa::SELECT_THREADS), 0, s, a);
    peqa::trace_after(peqa::KID_EVICT_SELECT, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return dev_status(e);
    peqa::trace_before(peqa::KID_EVICT_MOVE, s);
    hipLaunchKernelGGL(peqa::evict_move_kernel, dim3((unsigned)heads * 2u * (unsigned)a.splits * (unsigned)a.chunks), dim3(peqa::MOVE_THREADS), 0, s, a);
    peqa::trace_after(peqa::KID_EVICT_MOVE, s);
    return dev_status(hipGetLastError());
}

}  // extern "C"
