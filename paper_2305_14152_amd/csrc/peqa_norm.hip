// Norms of queries and keys for each head with the rotation by the position, without a cache (peqa_norm_rope), and its gradients
// (peqa_norm_rope_bwd).  With r = (mean x^2 + eps)^(-1/2) of a head, z = r x, w the norm's weights and R the rotation:
//   y = R (z w);   g = R^T dy,   dw = sum over tokens and heads of g z,   dx = r (u - z mean(u z)),  u = g w
#include "peqa_heads.h"
#include "peqa_host.h"

using namespace peqa::host;

namespace peqa {

namespace {

// Of queries (0) and keys (1); the heads of all tokens are numbered through, queries' first.
struct NormArgs {
    const int32_t *pos;
    const float *cos_table, *sin_table;
    const float *weight[2];
    const uint16_t *x[2], *dy[2];
    uint16_t *y[2];                        // what the forward or the backward writes
    float *part[2];                        // [workgroups, head_dim]: sums of a workgroup for the weights' gradients, or null
    float *dw[2];
    long long x_stride[2], dy_stride[2], y_stride[2];
    int heads[2], items[2], blocks[2];     // items: heads of all tokens; workgroups of queries and of keys
    uint32_t inverse_heads[2];             // floor((2^32 - 1) / heads)
    int n_pos, head_shift, rot_units;      // units of 16 elements in a head: 1 << head_shift, of which rotated
    float eps;
};

// Token and head of an item (the product is one too small at most: items are under 2^31).
struct Item {
    int t, h;
};
__device__ __forceinline__ Item item_at(const NormArgs &a, int side, int i)
{
    const int heads = a.heads[side];
    Item m;
    m.t = (int)__umulhi((unsigned)i, a.inverse_heads[side]);
    m.h = i - m.t * heads;
    if (m.h >= heads) { ++m.t; m.h -= heads; }
    return m;
}

// A lane's two groups of eight elements of a head.
struct Places {
    int at0, at1;
    bool rotated;
};
template <bool INTERLEAVED> __device__ __forceinline__ Places places(const NormArgs &a, int part)
{
    Places p;
    p.rotated = part < a.rot_units;
    p.at0 = part * 16;
    p.at1 = p.at0 + 8;
    if (!INTERLEAVED && p.rotated) { p.at0 = part * 8; p.at1 = p.at0 + a.rot_units * 8; }
    return p;
}

// A unit of 16 elements a thread, as in the cache's append kernel: a head's sum of squares is two to four lane exchanges, and everything is read
// and written once.  Products and sums are fp32; the output is rounded to bf16 once, the type of its readers.  Bound by
// memory: 2048 tokens of 2 x 32 heads of 128 14.7 us, 4.6 TB/s; 129 of 10 heads of 256 3.4 us, a launch and three loads after one another.
template <bool INTERLEAVED>
__global__ __launch_bounds__(256) void norm_rope_kernel(NormArgs a)
{
    const int side = blockIdx.x >= (unsigned)a.blocks[0];
    const int block = (int)blockIdx.x - (side ? a.blocks[0] : 0);
    const int part = threadIdx.x & ((1 << a.head_shift) - 1), dim = 16 << a.head_shift;
    const int i = block * (256 >> a.head_shift) + ((int)threadIdx.x >> a.head_shift);
    if (i >= a.items[side]) return;
    const Item m = item_at(a, side, i);
    const Places p = places<INTERLEAVED>(a, part);
    const uint16_t *x = a.x[side] + m.t * a.x_stride[side] + m.h * dim;
    uint16_t *y = a.y[side] + m.t * a.y_stride[side] + m.h * dim;
    const int pos = a.pos[m.t];
    Eight e0 = eight(*reinterpret_cast<const u32x4 *>(x + p.at0)), e1 = eight(*reinterpret_cast<const u32x4 *>(x + p.at1));
    const Eight w0 = weights_at(a.weight[side], p.at0), w1 = weights_at(a.weight[side], p.at1);
    const float r = inverse_rms(e0, e1, a.head_shift, a.eps);
    if (pos < 0 || (a.rot_units > 0 && pos >= a.n_pos)) {
        *reinterpret_cast<u32x4 *>(y + p.at0) = u32x4{0, 0, 0, 0};
        *reinterpret_cast<u32x4 *>(y + p.at1) = u32x4{0, 0, 0, 0};
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) { e0.x[j] *= r * w0.x[j]; e1.x[j] *= r * w1.x[j]; }
    if (p.rotated) turn<INTERLEAVED>(e0, e1, angles(a.cos_table, a.sin_table, pos, a.rot_units, part));
    *reinterpret_cast<u32x4 *>(y + p.at0) = to_bf16(e0);
    *reinterpret_cast<u32x4 *>(y + p.at1) = to_bf16(e1);
}

// The same units.  TRAINED: a workgroup goes over several items, so that a thread adds up the weights' gradients of the elements it always
// has, its heads meet in LDS and few rows of sums are left for norm_weights_kernel, all in a fixed order (atomics would change the bits from
// call to call).  x is normalised again from its bf16 rather than kept: that is 4 bytes an element less than storing z, and r costs a few
// lane exchanges.  Bound by memory: 2048 tokens of 2 x 32 heads of 128 20.0 us, 5.0 TB/s.
template <bool INTERLEAVED, bool TRAINED>
__global__ __launch_bounds__(256) void norm_rope_bwd_kernel(NormArgs a)
{
    __shared__ f32x4 sums[TRAINED ? 4 : 1][256];
    const int side = blockIdx.x >= (unsigned)a.blocks[0];
    const int block = (int)blockIdx.x - (side ? a.blocks[0] : 0);
    const int part = threadIdx.x & ((1 << a.head_shift) - 1), dim = 16 << a.head_shift, each = 256 >> a.head_shift;
    const Places p = places<INTERLEAVED>(a, part);
    const Eight w0 = weights_at(a.weight[side], p.at0), w1 = weights_at(a.weight[side], p.at1);
    Eight dw0{}, dw1{};
    for (int i = block * each + ((int)threadIdx.x >> a.head_shift); i < a.items[side]; i += a.blocks[side] * each) {
        const Item m = item_at(a, side, i);
        const uint16_t *x = a.x[side] + m.t * a.x_stride[side] + m.h * dim, *dy = a.dy[side] + m.t * a.dy_stride[side] + m.h * dim;
        uint16_t *dx = a.y[side] + m.t * a.y_stride[side] + m.h * dim;
        const int pos = a.pos[m.t];
        const bool there = pos >= 0 && (a.rot_units == 0 || pos < a.n_pos);
        Eight z0 = eight(*reinterpret_cast<const u32x4 *>(x + p.at0)), z1 = eight(*reinterpret_cast<const u32x4 *>(x + p.at1));
        Eight g0 = eight(*reinterpret_cast<const u32x4 *>(dy + p.at0)), g1 = eight(*reinterpret_cast<const u32x4 *>(dy + p.at1));
        if (p.rotated) turn<INTERLEAVED, true>(g0, g1, angles(a.cos_table, a.sin_table, there ? pos : 0, a.rot_units, part));
        const float r = inverse_rms(z0, z1, a.head_shift, a.eps);
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            z0.x[j] *= r;
            z1.x[j] *= r;
            if constexpr (TRAINED) {
                if (there) { dw0.x[j] = fmaf(g0.x[j], z0.x[j], dw0.x[j]); dw1.x[j] = fmaf(g1.x[j], z1.x[j], dw1.x[j]); }
            }
            g0.x[j] *= w0.x[j];
            g1.x[j] *= w1.x[j];
            sum = fmaf(g0.x[j], z0.x[j], fmaf(g1.x[j], z1.x[j], sum));
        }
        const float mean = over_head(sum, a.head_shift) * (1.f / (float)dim);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            g0.x[j] = there ? r * (g0.x[j] - z0.x[j] * mean) : 0.f;
            g1.x[j] = there ? r * (g1.x[j] - z1.x[j] * mean) : 0.f;
        }
        *reinterpret_cast<u32x4 *>(dx + p.at0) = to_bf16(g0);
        *reinterpret_cast<u32x4 *>(dx + p.at1) = to_bf16(g1);
    }
    if constexpr (TRAINED) {
        if (!a.part[side]) return;
        // element e of a lane's 16 is at [e / 4][thread][e % 4]; lanes with the same part are 1 << head_shift apart
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            sums[j][threadIdx.x] = f32x4{dw0.x[4 * j], dw0.x[4 * j + 1], dw0.x[4 * j + 2], dw0.x[4 * j + 3]};
            sums[2 + j][threadIdx.x] = f32x4{dw1.x[4 * j], dw1.x[4 * j + 1], dw1.x[4 * j + 2], dw1.x[4 * j + 3]};
        }
        __syncthreads();
        const int quads = dim / 4;                         // four per lane of a head
        if ((int)threadIdx.x < quads) {
            const int of = threadIdx.x & ((1 << a.head_shift) - 1), quad = (int)threadIdx.x >> a.head_shift;
            f32x4 total = {0.f, 0.f, 0.f, 0.f};
            for (int k = of; k < 256; k += 1 << a.head_shift) total += sums[quad][k];
            const Places mine = places<INTERLEAVED>(a, of);
            const int at = (quad < 2 ? mine.at0 : mine.at1) + 4 * (quad & 1);
            *reinterpret_cast<f32x4 *>(a.part[side] + (size_t)block * dim + at) = total;
        }
    }
}

// dw = the sum of all workgroups' rows.  A workgroup has 32 columns of one side: eight lanes of four columns, 32 rows at a time.  Bound by latency
// (512 KB of rows, 3.8 us of 8 workgroups; a last workgroup that does it would need a counter cleared before every call).
__global__ __launch_bounds__(256) void norm_weights_kernel(NormArgs a)
{
    __shared__ f32x4 sums[32][8];
    const int dim = 16 << a.head_shift, of_side = dim / 32;
    const int side = (int)blockIdx.x / of_side, lane = threadIdx.x & 7, row = threadIdx.x >> 3;
    if (!a.part[side]) return;
    const int at = ((int)blockIdx.x - side * of_side) * 32 + 4 * lane;
    f32x4 total = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int b = row; b < a.blocks[side]; b += 32) total += *reinterpret_cast<const f32x4 *>(a.part[side] + (size_t)b * dim + at);
    sums[row][lane] = total;
    __syncthreads();
    if (threadIdx.x >= 8) return;
    for (int k = 1; k < 32; ++k) total += sums[k][lane];
    *reinterpret_cast<f32x4 *>(a.dw[side] + at) = total;
}

// Workgroups of a backward that adds up the weights' gradients, at most: fewer have less in flight, more leave more rows (forward and backward of
// 2048 tokens, 2 x 32 heads, us: 512 workgroups 39.2, 1024 37.6, 2048 40.6;  8192 tokens of 40 + 8 heads 108.5, 104.3, 108.6).
constexpr int TRAINED_BLOCKS = 4 * PLAN_UNITS;

// Workgroups of queries and keys: one for as many heads as it has room for, or, up to `most` in all, in proportion.
void plan_blocks(NormArgs &a, int most)
{
    const int each = 256 >> a.head_shift;
    const long long all[2] = {((long long)a.items[0] + each - 1) / each, ((long long)a.items[1] + each - 1) / each};
    for (int s = 0; s < 2; ++s) {
        long long n = all[s];
        if (most > 0 && all[0] + all[1] > most) n = all[s] * most / (all[0] + all[1]);
        a.blocks[s] = (int)(n < 1 ? 1 : n);
    }
}

peqa_status check_norm(int32_t T, int32_t heads, int32_t kv_heads, int32_t head_dim)
{
    if (head_dim != 64 && head_dim != 128 && head_dim != 256) return PEQA_ERR_SHAPE;
    if (T < 1 || heads < 1 || heads > 65536 || kv_heads < 1 || kv_heads > 65536) return PEQA_ERR_SHAPE;
    if (((int64_t)heads + kv_heads) * T * (head_dim / 16) > (int64_t)INT32_MAX - 512) return PEQA_ERR_SHAPE;    // 32-bit numbers of units
    return PEQA_OK;
}

// What forward and backward have in common.
peqa_status norm_args(int32_t T, const int32_t *pos, const float *cos_table, const float *sin_table, int32_t n_pos, int32_t rot,
                      const float *q_weight, const float *k_weight, float eps, int32_t head_dim, int32_t heads, int32_t kv_heads,
                      const uint16_t *q, int64_t q_stride, const uint16_t *k, int64_t k_stride, uint16_t *q_out, int64_t q_out_stride,
                      uint16_t *k_out, int64_t k_out_stride, NormArgs &a)
{
    const peqa_status st = check_norm(T, heads, kv_heads, head_dim);
    if (st != PEQA_OK) return st;
    if (!pos || !q || !k || !q_out || !k_out) return PEQA_ERR_NULL;
    if (rot < 0 || rot > head_dim || rot % 16 || (rot > 0 && n_pos < 1)) return PEQA_ERR_PARAM;
    if (!(eps > 0.f) || eps > 3.402823466e38f) return PEQA_ERR_PARAM;
    if (rot > 0 && (!cos_table || !sin_table)) return PEQA_ERR_NULL;
    const int64_t q_width = (int64_t)heads * head_dim, k_width = (int64_t)kv_heads * head_dim;
    if (q_stride < q_width || q_out_stride < q_width || k_stride < k_width || k_out_stride < k_width) return PEQA_ERR_SHAPE;
    if (!aligned16(q) || !aligned16(k) || !aligned16(q_out) || !aligned16(k_out) || !aligned16(q_weight) || !aligned16(k_weight)) return PEQA_ERR_ALIGN;
    if (q_stride % 8 || k_stride % 8 || q_out_stride % 8 || k_out_stride % 8) return PEQA_ERR_ALIGN;
    if (rot > 0 && (!aligned16(cos_table) || !aligned16(sin_table))) return PEQA_ERR_ALIGN;
    if (reinterpret_cast<uintptr_t>(pos) & 3) return PEQA_ERR_ALIGN;
    a.pos = pos; a.cos_table = cos_table; a.sin_table = sin_table;
    a.weight[0] = q_weight; a.weight[1] = k_weight;
    a.x[0] = q; a.x[1] = k; a.x_stride[0] = q_stride; a.x_stride[1] = k_stride;
    a.y[0] = q_out; a.y[1] = k_out; a.y_stride[0] = q_out_stride; a.y_stride[1] = k_out_stride;
    a.heads[0] = heads; a.heads[1] = kv_heads;
    for (int s = 0; s < 2; ++s) {
        a.items[s] = T * a.heads[s];
        a.inverse_heads[s] = UINT32_MAX / (uint32_t)a.heads[s];
    }
    a.n_pos = n_pos; a.eps = eps;
    a.head_shift = __builtin_ctz((unsigned)(head_dim / 16));
    a.rot_units = rot / 16;
    return PEQA_OK;
}

}  // namespace
}  // namespace peqa

extern "C" {

peqa_status peqa_norm_rope(int32_t T, const int32_t *pos, const float *cos_table, const float *sin_table, int32_t n_pos, int32_t rot,
                           int32_t interleaved, const float *q_weight, const float *k_weight, float eps, int32_t head_dim, int32_t heads,
                           int32_t kv_heads, const uint16_t *q, int64_t q_stride, const uint16_t *k, int64_t k_stride, uint16_t *q_out,
                           int64_t q_out_stride, uint16_t *k_out, int64_t k_out_stride, void *stream)
{
    peqa::NormArgs a{};
    const peqa_status st = peqa::norm_args(T, pos, cos_table, sin_table, n_pos, rot, q_weight, k_weight, eps, head_dim, heads, kv_heads, q, q_stride,
                                           k, k_stride, q_out, q_out_stride, k_out, k_out_stride, a);
    if (st != PEQA_OK) return st;
    peqa::plan_blocks(a, 0);
    hipStream_t s = static_cast<hipStream_t>(stream);
    auto kernel = interleaved ? peqa::norm_rope_kernel<true> : peqa::norm_rope_kernel<false>;
    peqa::trace_before(peqa::KID_NORM_ROPE, s);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.blocks[0] + a.blocks[1])), dim3(256), 0, s, a);
    peqa::trace_after(peqa::KID_NORM_ROPE, s);
    return dev_status(hipGetLastError());
}

size_t peqa_norm_rope_bwd_workspace_bytes(int32_t T, int32_t heads, int32_t kv_heads, int32_t head_dim)
{
    if (peqa::check_norm(T, heads, kv_heads, head_dim) != PEQA_OK) return 0;
    peqa::NormArgs a{};
    a.head_shift = __builtin_ctz((unsigned)(head_dim / 16));
    a.items[0] = T * heads;
    a.items[1] = T * kv_heads;
    peqa::plan_blocks(a, peqa::TRAINED_BLOCKS);
    return round256((size_t)(a.blocks[0] + a.blocks[1]) * (size_t)head_dim * sizeof(float));
}

peqa_status peqa_norm_rope_bwd(int32_t T, const int32_t *pos, const float *cos_table, const float *sin_table, int32_t n_pos, int32_t rot,
                               int32_t interleaved, const float *q_weight, const float *k_weight, float eps, int32_t head_dim, int32_t heads,
                               int32_t kv_heads, const uint16_t *q, int64_t q_stride, const uint16_t *k, int64_t k_stride,
                               const uint16_t *d_q_out, int64_t d_q_out_stride, const uint16_t *d_k_out, int64_t d_k_out_stride,
                               uint16_t *dq, int64_t dq_stride, uint16_t *dk, int64_t dk_stride, float *d_q_weight, float *d_k_weight,
                               void *workspace, size_t workspace_bytes, void *stream)
{
    peqa::NormArgs a{};
    const peqa_status st = peqa::norm_args(T, pos, cos_table, sin_table, n_pos, rot, q_weight, k_weight, eps, head_dim, heads, kv_heads, q, q_stride,
                                           k, k_stride, dq, dq_stride, dk, dk_stride, a);
    if (st != PEQA_OK) return st;
    if (!d_q_out || !d_k_out) return PEQA_ERR_NULL;
    if (d_q_out_stride < (int64_t)heads * head_dim || d_k_out_stride < (int64_t)kv_heads * head_dim) return PEQA_ERR_SHAPE;
    if (!aligned16(d_q_out) || !aligned16(d_k_out) || d_q_out_stride % 8 || d_k_out_stride % 8 || !aligned16(d_q_weight) || !aligned16(d_k_weight))
        return PEQA_ERR_ALIGN;
    a.dy[0] = d_q_out; a.dy[1] = d_k_out;
    a.dy_stride[0] = d_q_out_stride; a.dy_stride[1] = d_k_out_stride;
    const bool trained = d_q_weight || d_k_weight;
    peqa::plan_blocks(a, trained ? peqa::TRAINED_BLOCKS : 0);
    if (trained) {
        if (!workspace || workspace_bytes < peqa_norm_rope_bwd_workspace_bytes(T, heads, kv_heads, head_dim)) return PEQA_ERR_WORKSPACE;
        if (!aligned16(workspace)) return PEQA_ERR_ALIGN;
        float *rows = static_cast<float *>(workspace);
        a.part[0] = d_q_weight ? rows : nullptr;
        a.part[1] = d_k_weight ? rows + (size_t)a.blocks[0] * (size_t)head_dim : nullptr;
        a.dw[0] = d_q_weight; a.dw[1] = d_k_weight;
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    auto kernel = trained ? (interleaved ? peqa::norm_rope_bwd_kernel<true, true> : peqa::norm_rope_bwd_kernel<false, true>)
                          : (interleaved ? peqa::norm_rope_bwd_kernel<true, false> : peqa::norm_rope_bwd_kernel<false, false>);
    peqa::trace_before(peqa::KID_NORM_ROPE_BWD, s);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.blocks[0] + a.blocks[1])), dim3(256), 0, s, a);
    peqa::trace_after(peqa::KID_NORM_ROPE_BWD, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !trained) return dev_status(e);
    peqa::trace_before(peqa::KID_NORM_WEIGHTS, s);
    hipLaunchKernelGGL(peqa::norm_weights_kernel, dim3((unsigned)(2 * head_dim / 32)), dim3(256), 0, s, a);
    peqa::trace_after(peqa::KID_NORM_WEIGHTS, s);
    return dev_status(hipGetLastError());
}

}  // extern "C"
