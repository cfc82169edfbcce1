// Log probabilities of given words, entropy and the largest alternatives (peqa_token_logprobs), and the gradient of the
// first two with respect to the logits (peqa_token_logprobs_bwd).
//
// With m the largest of a row, s = sum e^(x - m) and u = sum e^(x - m) (x - m):
//   lse = m + log s,   logp = (x_target - m) - log s,   entropy = log s - u / s
// m, s and u are kept per thread over one pass; when a larger m' is met, s and u are carried over to it:
//   u' = e^(m - m') (u + s (m - m')),  s' = e^(m - m') s.
// Alternatives: see take_top.
#include "peqa_device.h"
#include "peqa_host.h"

using namespace peqa::host;

namespace peqa {

namespace {

constexpr float LOG2E = 1.44269504088896341f;
constexpr float LOWEST = -3.402823466e38f;   // the lowest finite float: the maximum of a row without a finite logit
constexpr float FAR = -1e4f;                 // e^FAR is 0; products with differences are kept finite by it
constexpr int CANDIDATES = 1024;             // alternatives that are gathered before their order is found

struct LogprobArgs {
    const void *logits;
    const int32_t *targets;
    float *logp, *entropy, *lse, *top_logp;
    int32_t *top_ids;
    float *part;                // [T, slices, 4] m, s, u of the slices of a row
    unsigned long long *part_keys;   // [T, slices, top]
    long long stride;
    int T, V, top;
    int slices, slice;          // slices of a row, and vectors of eight logits in one
};

struct GradArgs {
    const void *logits;
    const int32_t *targets;
    const float *lse, *entropy, *d_logp, *d_entropy;
    void *d_logits;
    long long stride, d_stride;
    int T, V, blocks;           // workgroups per row
};

__device__ __forceinline__ float exp_of(float y) { return __builtin_amdgcn_exp2f(y * LOG2E); }

// A row as vectors of eight elements from the 16-byte boundary at or before its start on: `off` elements of the first vector
// are not the row's.
template <bool F32> struct Row {
    typedef typename std::conditional<F32, float, uint16_t>::type T;
    const T *base;
    int off;
    __device__ __forceinline__ Row(const void *logits, long long row, long long stride)
    {
        const T *p = static_cast<const T *>(logits) + row * stride;
        off = (int)((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T));
        base = p - off;
    }
    __device__ __forceinline__ float one(int j) const
    {
        if constexpr (F32) return base[off + j];
        else return __uint_as_float((uint32_t)base[off + j] << 16);
    }
    __device__ __forceinline__ int vectors(int V) const { return (V + off + 7) >> 3; }
    __device__ __forceinline__ bool edge(int v, int V) const { return 8 * v < off || 8 * v + 8 > V + off; }
};

struct Raw {
    u32x4 a, b;     // b: fp32 only
};
template <bool F32> __device__ __forceinline__ Raw load_vector(const Row<F32> &r, int v)
{
    Raw w;
    const u32x4 *p = reinterpret_cast<const u32x4 *>(r.base + 8ll * v);
    w.a = p[0];
    if constexpr (F32) w.b = p[1];
    return w;
}
template <bool F32> __device__ __forceinline__ void floats(const Raw &w, float x[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (F32) {
            x[i] = __uint_as_float(w.a[i]);
            x[4 + i] = __uint_as_float(w.b[i]);
        } else {
            x[2 * i] = bf16_lo(w.a[i]);
            x[2 * i + 1] = bf16_hi(w.a[i]);
        }
    }
}
template <bool F32> __device__ __forceinline__ Raw nothing()
{
    constexpr uint32_t inf = F32 ? 0xFF800000u : 0xFF80FF80u;
    Raw w;
    w.a = u32x4{inf, inf, inf, inf};
    if constexpr (F32) w.b = w.a;
    return w;
}
// Element i of a vector, i not a constant.
template <bool F32> __device__ __forceinline__ float element(const Raw &w, int i)
{
    if constexpr (F32) {
        const uint32_t lo = i & 2 ? (i & 1 ? w.a[3] : w.a[2]) : (i & 1 ? w.a[1] : w.a[0]);
        const uint32_t hi = i & 2 ? (i & 1 ? w.b[3] : w.b[2]) : (i & 1 ? w.b[1] : w.b[0]);
        return __uint_as_float(i & 4 ? hi : lo);
    }
    const uint32_t pair = i & 4 ? (i & 2 ? w.a[3] : w.a[2]) : (i & 2 ? w.a[1] : w.a[0]);
    return i & 1 ? bf16_hi(pair) : bf16_lo(pair);
}
// A vector that is not all the row's, the rest of it as -inf; nothing but the row's elements is read.
template <bool F32> __device__ __forceinline__ Raw read_edge(const Row<F32> &r, int v, int V)
{
    uint32_t x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int j = 8 * v + i - r.off, inside = j < 0 ? 0 : j < V ? j : V - 1;
        const uint32_t bits = __float_as_uint(r.one(inside));
        x[i] = j == inside ? bits : 0xFF800000u;
    }
    Raw w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (F32) { w.a[i] = x[i]; w.b[i] = x[4 + i]; }
        else w.a[i] = x[2 * i] >> 16 | (x[2 * i + 1] & 0xFFFF0000u);
    }
    return w;
}
template <bool F32> __device__ __forceinline__ Raw read_vector(const Row<F32> &r, int v, int V)
{
    return r.edge(v, V) ? read_edge<F32>(r, v, V) : load_vector<F32>(r, v);
}

// Order of the alternatives as unsigned numbers: by logit, then the lower index first.  -0 counts as 0, NaN as -inf.
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t b = __float_as_uint(x != x ? -__builtin_inff() : x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ unsigned long long key_of(float x, int j)
{
    return (unsigned long long)order_of(x) << 32 | (uint32_t)~j;
}
__device__ __forceinline__ int key_index(unsigned long long key) { return (int)~(uint32_t)key; }
__device__ __forceinline__ float key_logit(unsigned long long key)
{
    const uint32_t b = (uint32_t)(key >> 32);
    return __uint_as_float(b & 0x80000000u ? b & 0x7FFFFFFFu : ~b);
}

struct Stats {
    float m, s, u;
    // the state as seen from a maximum that is no smaller
    __device__ __forceinline__ void move_to(float to)
    {
        const float d = fmaxf(m - to, FAR), f = exp_of(d);
        u = f * (u + s * d);
        s *= f;
        m = to;
    }
};

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

struct Answer {
    float logp, entropy, lse, log_s, m;
};
__device__ __forceinline__ Answer answer_of(float m, float s, float u)
{
    Answer r;
    r.m = m;
    r.log_s = logf(s);
    const bool none = s == 0.f;              // a row without a finite logit
    r.lse = none ? -__builtin_inff() : m + r.log_s;
    r.entropy = none ? 0.f : r.log_s - u / s;
    return r;
}
__device__ __forceinline__ float logp_of(const Answer &r, float x) { return r.lse == -__builtin_inff() ? r.lse : (x - r.m) - r.log_s; }

// The target and its logit: asked for before the pass over the row, used after it.
struct Target {
    bool live;
    float x;
};
template <bool F32> __device__ __forceinline__ Target target_of(const LogprobArgs &a, int row, const Row<F32> &r)
{
    const int t = a.logp ? a.targets[row] : -1;
    const bool live = t >= 0 && t < a.V;
    return Target{live, live ? r.one(t) : 0.f};
}
__device__ __forceinline__ void write_row(const LogprobArgs &a, int row, const Target &t, const Answer &n)
{
    if (a.logp) a.logp[row] = t.live ? logp_of(n, t.x) : 0.f;
    if (a.entropy) a.entropy[row] = n.entropy;
    if (a.lse) a.lse[row] = n.lse;
}

// A lane's key, the same for the whole wave.
__device__ __forceinline__ unsigned long long lane_key(unsigned long long key, int lane)
{
    return (unsigned long long)(uint32_t)__builtin_amdgcn_readlane((int)(key >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)key, lane);
}

// out(rank, key) for the `top` largest of `count` different keys in LDS (all, of fewer), by the first wave, with a key in every lane that it
// compares with one after the other.  Of more than 64 (words that are masked alike are candidates together, and so are the slices'
// answers) it first leaves those that are no smaller than the top-th largest of its lanes' largest ones, which takes away the keys of
// 64 - top lanes at least, mostly most of them, until there are 64 or less.  1174 rows of 1002 words, all but one masked, 20 alternatives
// 13.2 us (30.8 where a wave took a key and counted by ballots how many are larger), 9 rows of 245236 words 14.4 us (19.4).
template <typename Out> __device__ __forceinline__ void rank_keys(unsigned long long *keys, int count, int top, Out out)
{
    if (threadIdx.x >= 64) return;
    const int lane = threadIdx.x;
    while (count > 64) {
        unsigned long long largest = 0;
        for (int i = lane; i < count; i += 64) largest = keys[i] > largest ? keys[i] : largest;
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < 64; ++j) rank += lane_key(largest, j) > largest;
        const unsigned long long least = lane_key(largest, __builtin_ctzll(__ballot(rank == top - 1)));
        int left = 0;
        for (int i = 0; i < count; i += 64) {
            const unsigned long long key = i + lane < count ? keys[i + lane] : 0, stays = __ballot(key >= least);
            if (key >= least) keys[left + __popcll(stays & ((1ull << lane) - 1))] = key;      // (a place that has been read)
            left += __popcll(stays);
        }
        count = left;
    }
    const unsigned long long mine = lane < count ? keys[lane] : 0;
    int rank = 0;
    for (int j = 0; j < count; ++j) rank += lane_key(mine, j) > mine;
    if (lane < count && rank < top) out(rank, mine);
}

// One workgroup of NT threads per slice of a row.  The logits pass once, BATCH vectors of a thread in flight; per batch one maximum is
// found and one carry-over done.  With TOP every thread also keeps the vector with its largest logit.
// Bound by memory and the latency of a batch: 2048 rows of 32000 bf16 logits 27.8 us, 4.7 TB/s (11 vector instructions a logit; a
// form with 8, that looks for a new maximum only where a batch's sum gets large, is no faster), 333 rows of 100003 fp32 logits with five
// alternatives 33.5 us, 4.0 TB/s.  16 rows of 32000 with 20 alternatives, 9.7 us, are a launch, two batches and the steps of the search one
// after the other.
//
// Alternatives.  The threads with the same lane are a group.  At least `top` groups have an element no smaller than the top-th
// largest of the 64 groups' largest ones: what is no smaller than this bound, a few more than `top` if the large logits lie
// anywhere, contains the answer, and lies with the few threads whose own largest is no smaller.  Their vectors are looked at once
// more by all threads, the keys gathered in LDS and ranked.  The order in which they are gathered does not matter: keys are different
// and ranks are counts.
constexpr int BATCH = 4;
template <bool F32, int NT, bool TOP>
__global__ __launch_bounds__(NT) void logprobs_kernel(LogprobArgs a)
{
    constexpr int WAVES = NT / 64;
    __shared__ float wave_m[WAVES], wave_s[WAVES], wave_u[WAVES];
    __shared__ unsigned long long best[TOP ? NT : 1], list[TOP ? CANDIDATES : 1], bound;
    __shared__ int gathered, n_owners;
    __shared__ short owner[TOP ? NT : 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = (int)(blockIdx.x / (unsigned)a.slices), slice = (int)(blockIdx.x - (unsigned)row * (unsigned)a.slices);
    const Row<F32> r(a.logits, row, a.stride);
    const int all = r.vectors(a.V);
    const int v0 = slice * a.slice < all ? slice * a.slice : all, v1 = slice + 1 < a.slices && v0 + a.slice < all ? v0 + a.slice : all;

    const Target target = a.slices == 1 ? target_of(a, row, r) : Target{false, 0.f};
    Stats st{LOWEST, 0.f, 0.f};
    float most = -__builtin_inff();
    int at = -1;                                           // TOP: the vector with the first of this thread's largest
    // vectors that are all the row's; a first and a last one that are not are threads 0's and 1's
    const int f0 = v0 < v1 && r.edge(v0, a.V) ? v0 + 1 : v0, f1 = v1 > f0 && r.edge(v1 - 1, a.V) ? v1 - 1 : v1;
    const int edge = tid == 0 && f0 > v0 ? v0 : tid == 1 && f1 < v1 ? f1 : -1;
    Raw w[BATCH], ahead[BATCH], largest = nothing<F32>();
    float top = LOWEST;
    auto look = [&](const Raw &raw, int v) __attribute__((always_inline)) {
        float x[8];
        floats<F32>(raw, x);
        float vm = -__builtin_inff();                      // (stays of eight NaN)
#pragma unroll
        for (int i = 0; i < 8; ++i) vm = fmaxf(vm, x[i]);
        top = fmaxf(top, vm);
        if constexpr (TOP) {
            const bool more = vm > most || (vm == most && (unsigned)v < (unsigned)at);      // (at = -1: none yet)
            most = more ? vm : most;
            at = more ? v : at;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                largest.a[i] = more ? raw.a[i] : largest.a[i];
                if constexpr (F32) largest.b[i] = more ? raw.b[i] : largest.b[i];
            }
        }
    };
    auto add = [&](const Raw &raw) __attribute__((always_inline)) {
        float x[8];
        floats<F32>(raw, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float y = x[i] - st.m, e = exp_of(y);
            st.s += e;
            st.u += e * fmaxf(y, FAR);
        }
    };
    auto read = [&](int vb) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            const int v = vb + k * NT + tid;
            ahead[k] = v >= f0 && v < f1 ? load_vector<F32>(r, v) : nothing<F32>();
        }
    };
    // the next batch is in flight while one is added up (2048 rows of 32000 bf16 logits: 31.6 -> 29.5 us); with TOP the registers that
    // it takes cost more (20 alternatives: 38.3 -> 39.4)
    read(v0);
    for (int vb = v0; vb < v1; vb += BATCH * NT) {
        if (TOP && vb > v0) read(vb);
#pragma unroll
        for (int k = 0; k < BATCH; ++k) w[k] = ahead[k];
        if (!TOP && vb + BATCH * NT < v1) read(vb + BATCH * NT);
        top = st.m;
#pragma unroll
        for (int k = 0; k < BATCH; ++k)
            if (vb + k * NT + wave * 64 < v1) look(w[k], vb + k * NT + tid);       // (uniform)
        st.move_to(top);
#pragma unroll
        for (int k = 0; k < BATCH; ++k)
            if (vb + k * NT + wave * 64 < v1) add(w[k]);
    }

    Raw part = nothing<F32>();
    if (edge >= 0) {
        part = read_edge<F32>(r, edge, a.V);
        top = st.m;
        look(part, edge);
        st.move_to(top);
        add(part);
    }

    unsigned long long mine = 0;                           // this thread's largest key
    if constexpr (TOP) {
        if (at >= 0 && (at < f1 || at == edge)) {         // (else a place past the slice: no element)
            float x[8];
            floats<F32>(largest, x);
            const int begin = r.off - 8 * at > 0 ? r.off - 8 * at : 0;      // elements before are not the row's
            int i0 = begin;
#pragma unroll
            for (int i = 7; i >= 0; --i)
                if (fmaxf(x[i], -__builtin_inff()) == most && i >= begin) i0 = i;
            mine = key_of(most, 8 * at + i0 - r.off);
        }
        best[tid] = mine;
        if (tid == 0) { gathered = 0; n_owners = 0; bound = 0; }
    }
    float m = st.m;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    if (lane == 0) wave_m[wave] = m;
    __syncthreads();
    m = wave_m[0];
#pragma unroll
    for (int k = 1; k < WAVES; ++k) m = fmaxf(m, wave_m[k]);
    st.move_to(m);
    st.s = wave_sum(st.s);
    st.u = wave_sum(st.u);
    if (lane == 0) { wave_s[wave] = st.s; wave_u[wave] = st.u; }
    if constexpr (TOP) {
        // every wave looks at some of the groups' largest
        unsigned long long column = 0;
#pragma unroll
        for (int k = 0; k < WAVES; ++k) column = best[k * 64 + lane] > column ? best[k * 64 + lane] : column;
#pragma unroll
        for (int i = 0; i < 64 / WAVES; ++i) {
            const unsigned long long key = lane_key(column, wave * (64 / WAVES) + i);
            if (key != 0 && __popcll(__ballot(column > key)) == a.top - 1 && lane == 0) bound = key;
        }
    }
    __syncthreads();
    float s = 0.f, u = 0.f;
#pragma unroll
    for (int k = 0; k < WAVES; ++k) { s += wave_s[k]; u += wave_u[k]; }
    const Answer n = answer_of(m, s, u);
    if (tid == 0) {
        if (a.slices == 1) {
            write_row(a, row, target, n);
        } else {
            float *p = a.part + 4 * ((size_t)row * a.slices + slice);
            p[0] = m;
            p[1] = s;
            p[2] = u;
        }
    }
    if constexpr (TOP) {
        const unsigned long long least = bound;            // 0: fewer than `top` groups have elements
        const float least_x = least != 0 ? key_logit(least) : -__builtin_inff();
        const int least_j = least != 0 ? key_index(least) : 1 << 30;
        // which of a vector's eight elements are no smaller than the bound
        auto above = [&](const Raw &raw, int v) __attribute__((always_inline)) {
            float x[8];
            floats<F32>(raw, x);
            uint32_t mask = 0, ties = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float y = fmaxf(x[i], -__builtin_inff());           // (NaN counts as -inf)
                mask |= y > least_x ? 1u << i : 0u;
                ties |= y == least_x ? 1u << i : 0u;
            }
            const int before = r.off - 8 * v, upto = least_j + 1 + before, end = a.V + before;   // elements of the row, of ties
            mask |= upto >= 8 ? ties : upto > 0 ? ties & ((1u << upto) - 1u) : 0u;
            if (before > 0) mask &= 0xFFu << before;
            return end < 8 ? mask & ((1u << end) - 1u) : mask;
        };
        auto gather = [&](const Raw &raw, int v) __attribute__((always_inline)) {
            uint32_t mask = above(raw, v);
#pragma unroll 1
            while (mask != 0) {
                const int i = __builtin_ctz(mask), place = atomicAdd(&gathered, 1);
                mask &= mask - 1;
                if (place < CANDIDATES) list[place] = key_of(element<F32>(raw, i), 8 * v + i - r.off);
            }
        };
        const bool owns = mine != 0 && mine >= least;
        if (owns) owner[atomicAdd(&n_owners, 1)] = (short)tid;
        __syncthreads();
        const int owners = n_owners, rounds = (v1 - v0 + NT - 1) / NT;
        for (int i = tid; i < owners * rounds; i += NT) {
            const int round = i / owners, v = v0 + round * NT + owner[i - round * owners];
            if (v >= f0 && v < f1) gather(load_vector<F32>(r, v), v);
        }
        if (owns && edge >= 0) gather(part, edge);
        __syncthreads();
        int count = gathered;
        if (count > CANDIDATES) {
            // Many large logits in few groups: the answer one by one, the largest key below the last one found.
            unsigned long long below = ~0ull;
            for (int k = 0; k < a.top; ++k) {
                unsigned long long top = 0;
                for (int v = v0 + tid; v < v1; v += NT) {
                    float x[8];
                    floats<F32>(read_vector<F32>(r, v, a.V), x);
                    for (int i = 0; i < 8; ++i) {
                        const int j = 8 * v + i - r.off;
                        if (j < 0 || j >= a.V) continue;
                        const unsigned long long key = key_of(x[i], j);
                        if (key < below && key > top) top = key;
                    }
                }
#pragma unroll
                for (int o = 32; o >= 1; o >>= 1) {
                    const unsigned long long other = __shfl_xor(top, o);
                    top = other > top ? other : top;
                }
                __syncthreads();
                if (lane == 0) best[wave] = top;
                __syncthreads();
                below = best[0];
#pragma unroll
                for (int q = 1; q < WAVES; ++q) below = best[q] > below ? best[q] : below;
                if (tid == 0) list[k] = below;
            }
            count = a.top;
            __syncthreads();
        }
        if (a.slices == 1) {
            rank_keys(list, count, a.top, [&](int rank, unsigned long long key) {
                a.top_ids[(size_t)row * a.top + rank] = key_index(key);
                a.top_logp[(size_t)row * a.top + rank] = logp_of(n, key_logit(key));
            });
        } else {
            unsigned long long *keys = a.part_keys + ((size_t)row * a.slices + slice) * a.top;
            rank_keys(list, count, a.top, [&](int rank, unsigned long long key) { keys[rank] = key; });
            for (int k = count + tid; k < a.top; k += NT) keys[k] = 0;
        }
    }
}

// Joins the slices of a row: at most 32 of at most 32 keys.
constexpr int SLICES_MAX = 32;
template <bool F32>
__global__ __launch_bounds__(256) void logprobs_join_kernel(LogprobArgs a)
{
    __shared__ unsigned long long keys[SLICES_MAX * PEQA_MAX_TOP];
    __shared__ int gathered;
    const int row = blockIdx.x;
    const Target target = target_of(a, row, Row<F32>(a.logits, row, a.stride));
    // a lane per slice
    const int lane = threadIdx.x & 63, count = a.slices * a.top;
    const unsigned long long *from = a.part_keys + (size_t)row * count;
    Stats st{LOWEST, 0.f, 0.f};
    if (lane < a.slices) {
        const f32x4 p = *reinterpret_cast<const f32x4 *>(a.part + 4 * ((size_t)row * a.slices + lane));
        st = Stats{p[0], p[1], p[2]};
    }
    // Every slice's keys fall, and each has at least ceil(top / slices) keys no smaller than the least of the slices' keys with that
    // number: `top` in all, so what is smaller is not looked at.  (0: a slice has fewer.)
    unsigned long long least = a.top > 0 && lane < a.slices ? from[lane * a.top + (a.top + a.slices - 1) / a.slices - 1] : ~0ull;
    float m = st.m;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    st.move_to(m);
    const float s = wave_sum(st.s), u = wave_sum(st.u);
    const Answer n = answer_of(m, s, u);
    if (threadIdx.x == 0) write_row(a, row, target, n);
    if (a.top == 0) return;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        const unsigned long long other = __shfl_xor(least, o);
        least = other < least ? other : least;
    }
    if (threadIdx.x == 0) gathered = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < count; i += 256) {
        const unsigned long long key = from[i];
        if (key != 0 && key >= least) keys[atomicAdd(&gathered, 1)] = key;
    }
    __syncthreads();
    rank_keys(keys, gathered, a.top, [&](int rank, unsigned long long key) {
        a.top_ids[(size_t)row * a.top + rank] = key_index(key);
        a.top_logp[(size_t)row * a.top + rank] = logp_of(n, key_logit(key));
    });
}

// d_j = g ([j = target] - p_j) - h p_j (log p_j + H): one read and one write of the logits.  Bound by memory: 2048 rows of 32000 bf16
// logits, a tenth of them ignored and not read, at 5.7 TB/s.  A thread has 32 bytes of a row, one vector of eight or two (fp32: 1000 rows
// of 32000 48 us with one, 52 with two; bf16: the 2048 rows 51.9 and 46.1).  The target's place is looked for a vector at a time and the
// entropy's terms are left out where there are none, else it is 19.5 vector instructions a logit and 47.7 us.
//
// p_j = e^(x_j - lse) is off by the rounding of lse to fp32, 2^-17 of p_j for an lse under 256.  Of a row whose lse is further from zero
// (all words masked with the lowest value: nothing is left of log V in it) one workgroup first adds up the row: r = log sum e^(x - lse) is
// what the rounding left, p_j = e^((x_j - lse) - r).  It reads the whole row before it writes any of it, so the gradient may still
// replace the logits.  Such rows cost two to three times as much (2048 of 32000 bf16 logits 134 us, 1000 of 50257 fp32 ones 151 for 74), the
// others nothing.
constexpr float LSE_FAR = 256.f;
constexpr int grad_vectors(bool f32) { return f32 ? 1 : 2; }
template <bool F32, bool ENTROPY>
__global__ __launch_bounds__(256) void logprobs_bwd_kernel(GradArgs a)
{
    constexpr int GRAD_VECTORS = grad_vectors(F32);
    int row = (int)(blockIdx.x / (unsigned)a.blocks);
    asm("" : "+s"(row));                                   // (and all that follows from it; else 12 vector instructions a logit, not 8: 4000 rows of 2000 7.9 us, not 7.6)
    const int block = (int)(blockIdx.x - (unsigned)row * (unsigned)a.blocks);
    const Row<F32> r(a.logits, row, a.stride);
    typedef typename Row<F32>::T E;
    const int t = a.targets ? a.targets[row] : -1;
    const bool live = t >= 0 && t < a.V;
    const float lse = a.lse[row];
    const float g = live && a.d_logp ? a.d_logp[row] : 0.f, h = ENTROPY ? a.d_entropy[row] : 0.f, H = ENTROPY ? a.entropy[row] : 0.f;
    const bool none = (g == 0.f && h == 0.f) || lse == -__builtin_inff();
    E *out = static_cast<E *>(a.d_logits) + row * a.d_stride;
    const bool aligned = (int)((reinterpret_cast<uintptr_t>(out) & 15u) / sizeof(E)) == r.off;
    const int all = r.vectors(a.V);
    // vector v of the row, whose logits are `raw`; rest: what lse lacks (REST), else 0
    auto write = [&](int v, const Raw &raw, float rest, auto REST) __attribute__((always_inline)) {
        float x[8];
        if (none) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = 0.f;
        } else {
            floats<F32>(raw, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float logp = REST ? (x[i] - lse) - rest : x[i] - lse, p = exp_of(logp);
                x[i] = ENTROPY ? -p * (g + h * (fmaxf(logp, FAR) + H)) : -p * g;
            }
            const int target = t + r.off - 8 * v;              // its place in this vector
            if (live && target >= 0 && target < 8) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] += i == target ? g : 0.f;
            }
        }
        if (aligned && !r.edge(v, a.V)) {
            u32x4 *o = reinterpret_cast<u32x4 *>(out + (8ll * v - r.off));
            if constexpr (F32) {
                o[0] = u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
                o[1] = u32x4{__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7])};
            } else {
                o[0] = u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int j = 8 * v + i - r.off;
                if (j < 0 || j >= a.V) continue;
                if constexpr (F32) out[j] = x[i];
                else out[j] = (uint16_t)float_to_bf16_bits(x[i]);
            }
        }
    };
    if (__builtin_expect(!none && fabsf(lse) >= LSE_FAR && fabsf(lse) < __builtin_inff(), 0)) {
        // (the same for all workgroups of the row; not the first of every one, which can all be on one die)
        if (block != (int)((unsigned)row % (unsigned)a.blocks)) return;
        __shared__ float wave_s[4];
        constexpr int FLIGHT = 4;
        auto walk = [&](auto each) __attribute__((always_inline)) {
#pragma unroll 1
            for (int v0 = (int)threadIdx.x; v0 < all; v0 += FLIGHT * 256) {
                Raw w[FLIGHT];
#pragma unroll
                for (int k = 0; k < FLIGHT; ++k) w[k] = v0 + k * 256 < all ? read_vector<F32>(r, v0 + k * 256, a.V) : nothing<F32>();
#pragma unroll
                for (int k = 0; k < FLIGHT; ++k) each(v0 + k * 256, w[k]);
            }
        };
        float s = 0.f;
        walk([&](int, const Raw &raw) {
            float x[8], sum = 0.f;
            floats<F32>(raw, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += exp_of(x[i] - lse);
            s += sum;
        });
        s = wave_sum(s);
        if ((threadIdx.x & 63) == 0) wave_s[threadIdx.x >> 6] = s;
        __syncthreads();
        float rest = logf(wave_s[0] + wave_s[1] + wave_s[2] + wave_s[3]);
        // an lse that is off by more than rounding is not this row's alone (words in several pieces), and is taken as it is
        if (!(fabsf(rest) <= fabsf(lse) * 0x1p-22f)) rest = 0.f;
        walk([&](int v, const Raw &raw) {
            if (v < all) write(v, raw, rest, std::true_type{});
        });
        return;
    }
    const int v0 = block * GRAD_VECTORS * 256 + (int)threadIdx.x;
#pragma unroll
    for (int k = 0; k < GRAD_VECTORS; ++k) {
        if (v0 + k * 256 >= all) return;
        const int v = v0 + k * 256;
        write(v, none ? Raw{} : read_vector<F32>(r, v, a.V), 0.f, std::false_type{});
    }
}

// Slices of a row (0: the whole row by one workgroup) and vectors in one.
struct LogprobPlan {
    int slices, slice;
    size_t part_bytes, key_bytes;
};
LogprobPlan logprob_plan(int T, int V, int top)
{
    LogprobPlan p{};
    const int vectors = (V + 7 + 7) / 8;                       // with any offset of the row
    // Few long rows are cut, if the slices are not so short that the join outlasts what they save: slices of 8192, 16384, 32768 logits, us:
    // 16 rows of 128256 6.4, 7.2, 8.5 (fp32, no alternatives) and 17.7, 14.1, 15.1 (bf16, 20); one of 250000 10.1, 10.4, 11.8 (26.9 uncut).
    int slices = PLAN_UNITS / T;
    const int most = vectors / (top > 0 ? 2048 : 1024);
    slices = slices < most ? slices : most;
    slices = slices < SLICES_MAX ? slices : SLICES_MAX;
    p.slices = slices > 1 ? slices : 1;
    p.slice = (vectors + p.slices - 1) / p.slices;
    if (p.slices > 1) {
        p.part_bytes = round256((size_t)T * p.slices * 4 * sizeof(float));
        p.key_bytes = round256((size_t)T * p.slices * top * sizeof(unsigned long long));
    }
    return p;
}

peqa_status check_logits(int32_t dtype, int32_t T, int32_t vocab)
{
    if (dtype != PEQA_LOGITS_BF16 && dtype != PEQA_LOGITS_F32) return PEQA_ERR_PARAM;
    if (T < 1 || vocab < 1 || vocab > (1 << 30)) return PEQA_ERR_SHAPE;
    return PEQA_OK;
}

inline bool aligned_to(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

}  // namespace
}  // namespace peqa

extern "C" {

size_t peqa_token_logprobs_workspace_bytes(int32_t T, int32_t vocab, int32_t top)
{
    if (peqa::check_logits(PEQA_LOGITS_BF16, T, vocab) != PEQA_OK || top < 0 || top > PEQA_MAX_TOP || top > vocab) return 0;
    const peqa::LogprobPlan p = peqa::logprob_plan(T, vocab, top);
    const size_t bytes = p.part_bytes + p.key_bytes;
    return bytes ? bytes : 256;
}

peqa_status peqa_token_logprobs(const void *logits, int32_t dtype, int32_t T, int32_t vocab, int64_t stride, const int32_t *targets,
                                int32_t top, float *logp, float *entropy, float *lse, float *top_logp, int32_t *top_ids, void *workspace,
                                size_t workspace_bytes, void *stream)
{
    const peqa_status st = peqa::check_logits(dtype, T, vocab);
    if (st != PEQA_OK) return st;
    if (top < 0 || top > PEQA_MAX_TOP || top > vocab) return PEQA_ERR_PARAM;
    if (!logits || (logp && !targets) || (top > 0 && (!top_logp || !top_ids))) return PEQA_ERR_NULL;
    if (!logp && !entropy && !lse && top == 0) return PEQA_ERR_NULL;
    if (stride < vocab || (int64_t)T * 512 > (int64_t)UINT32_MAX) return PEQA_ERR_SHAPE;    // (threads of a launch)
    if (!peqa::aligned_to(logits, dtype == PEQA_LOGITS_F32 ? 4 : 2) || !peqa::aligned_to(targets, 4) || !peqa::aligned_to(logp, 4) ||
        !peqa::aligned_to(entropy, 4) || !peqa::aligned_to(lse, 4) || !peqa::aligned_to(top_logp, 4) || !peqa::aligned_to(top_ids, 4))
        return PEQA_ERR_ALIGN;
    const peqa::LogprobPlan p = peqa::logprob_plan(T, vocab, top);
    if (p.slices > 1) {
        if (!workspace || workspace_bytes < p.part_bytes + p.key_bytes) return PEQA_ERR_WORKSPACE;
        if (!aligned16(workspace)) return PEQA_ERR_ALIGN;
    }
    peqa::LogprobArgs a{};
    a.logits = logits; a.targets = targets; a.logp = logp; a.entropy = entropy; a.lse = lse; a.top_logp = top_logp; a.top_ids = top_ids;
    a.part = static_cast<float *>(workspace);
    a.part_keys = p.slices > 1 ? reinterpret_cast<unsigned long long *>(static_cast<char *>(workspace) + p.part_bytes) : nullptr;
    a.stride = stride;
    a.T = T; a.V = vocab; a.top = top; a.slices = p.slices; a.slice = p.slice;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const unsigned grid = (unsigned)T * (unsigned)p.slices;
    peqa::trace_before(peqa::KID_LOGPROBS, s);
    const bool f32 = dtype == PEQA_LOGITS_F32;
    // Short rows: 128 threads, of few vectors each.  Else 256 (of fp32, and of many rows), or 512, which end a row sooner where there are
    // not rows enough to fill the machine.  128 / 256 / 512, us: 4000 rows of 2000  7.2 / 9.4 / 14.9, with 20 alternatives 15.8 / 19.1 / 31.6;
    // 64 of 4000 with 32  9.9 / 7.7 / 8.0;  16 of 32000 with 20  - / 11.2 / 9.1;  512 of 50257 with one  29.9 / 19.7 / 18.4;  2048 of 32000
    // with 20  43.8 / 38.4 / 38.7;  fp32: 300 of 100000  35.3 / 28.8 / 30.8.
    const int vectors = (vocab + 14) / 8, threads = vectors <= 512 && T >= peqa::PLAN_UNITS ? 128 : T >= (f32 ? 256 : 1024) ? 256 : 512;
    auto pick = [&](auto n) {
        constexpr int NT = decltype(n)::value;
        return top > 0 ? (f32 ? peqa::logprobs_kernel<true, NT, true> : peqa::logprobs_kernel<false, NT, true>)
                       : (f32 ? peqa::logprobs_kernel<true, NT, false> : peqa::logprobs_kernel<false, NT, false>);
    };
    auto kernel = threads == 128 ? pick(std::integral_constant<int, 128>{}) : threads == 256 ? pick(std::integral_constant<int, 256>{})
                                                                                           : pick(std::integral_constant<int, 512>{});
    hipLaunchKernelGGL(kernel, dim3(grid), dim3((unsigned)threads), 0, s, a);
    peqa::trace_after(peqa::KID_LOGPROBS, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.slices == 1) return dev_status(e);
    peqa::trace_before(peqa::KID_LOGPROBS_JOIN, s);
    auto join = f32 ? peqa::logprobs_join_kernel<true> : peqa::logprobs_join_kernel<false>;
    hipLaunchKernelGGL(join, dim3((unsigned)T), dim3(256), 0, s, a);
    peqa::trace_after(peqa::KID_LOGPROBS_JOIN, s);
    return dev_status(hipGetLastError());
}

peqa_status peqa_token_logprobs_bwd(const void *logits, int32_t dtype, int32_t T, int32_t vocab, int64_t stride, const int32_t *targets,
                                    const float *lse, const float *entropy, const float *d_logp, const float *d_entropy, void *d_logits,
                                    int64_t d_stride, void *stream)
{
    const peqa_status st = peqa::check_logits(dtype, T, vocab);
    if (st != PEQA_OK) return st;
    if (!logits || !lse || !d_logits || (!d_logp && !d_entropy) || (d_logp && !targets) || (d_entropy && !entropy)) return PEQA_ERR_NULL;
    if (stride < vocab || d_stride < vocab || (d_logits == logits && d_stride != stride)) return PEQA_ERR_SHAPE;
    const size_t el = dtype == PEQA_LOGITS_F32 ? 4 : 2;
    if (!peqa::aligned_to(logits, el) || !peqa::aligned_to(d_logits, el) || !peqa::aligned_to(targets, 4) || !peqa::aligned_to(lse, 4) ||
        !peqa::aligned_to(entropy, 4) || !peqa::aligned_to(d_logp, 4) || !peqa::aligned_to(d_entropy, 4))
        return PEQA_ERR_ALIGN;
    peqa::GradArgs a{};
    a.logits = logits; a.targets = targets; a.lse = lse; a.entropy = entropy; a.d_logp = d_logp; a.d_entropy = d_entropy;
    a.d_logits = d_logits; a.stride = stride; a.d_stride = d_stride; a.T = T; a.V = vocab;
    const int vectors = (vocab + 7 + 7) / 8;
    const int per_block = 256 * peqa::grad_vectors(dtype == PEQA_LOGITS_F32);
    a.blocks = (vectors + per_block - 1) / per_block;
    if ((int64_t)a.blocks * T * 256 > (int64_t)UINT32_MAX) return PEQA_ERR_SHAPE;    // threads of a launch
    hipStream_t s = static_cast<hipStream_t>(stream);
    const unsigned grid = (unsigned)T * (unsigned)a.blocks;
    peqa::trace_before(peqa::KID_LOGPROBS_BWD, s);
    auto kernel = dtype == PEQA_LOGITS_F32 ? (d_entropy ? peqa::logprobs_bwd_kernel<true, true> : peqa::logprobs_bwd_kernel<true, false>)
                                           : (d_entropy ? peqa::logprobs_bwd_kernel<false, true> : peqa::logprobs_bwd_kernel<false, false>);
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, s, a);
    peqa::trace_after(peqa::KID_LOGPROBS_BWD, s);
    return dev_status(hipGetLastError());
}

}  // extern "C"
