// Norm of every query and key head, rotary positions, the store of keys and values into the paged cache, and the backward of norm and
// rotation (nq_decoder.h).
//
// With n the head (normalised or not), a rotated element is  y_e = n_e C_e + n_p S_e:  C = magnitude cos, S = -+ magnitude sin, p the
// other element of e's pair; C = 1, S = 0 past rot_dim.  The backward of the rotation is the same with -S.  The angles are formed
// in binary64 (position times frequency, less the nearest multiple of 2 pi), once per token and pair, and shared through LDS by all heads of the
// token: a binary64 angle and an fp32 sine per element would cost more than the element's bytes.
//
// A lane owns eight consecutive elements (16 bytes of a 16-bit type) of one head, 16 lanes a head of 128; the lanes of a head are neighbours, so
// that the sum of squares is a few lane exchanges.  Eight C, S and weights stay in registers while a lane walks the heads of its token.
// The other elements of the pairs are loaded a second time (from the cache that holds them: the head's own lanes have just read
// them) where the layout is halves, and are in the lane already where it is interleaved.  Bound by bytes: each is read and written once.
// 4093 tokens of 96 heads of 128, bf16, interleaved (201 MB): 42 us, 4.8 TB/s, as a large copy; forward and backward with norm of 4096 tokens of 72 heads
// (377 MB): 98 us; one token: 4.7 us.
#include <algorithm>
#include <cmath>

#include "nq_decoder_internal.h"

struct nq_rope_s {
    int q_heads, kv_heads, head_dim, rot_dim, layout, in_dtype, out_dtype, device;
    float eps, weight_offset, magnitude;
    double* inv_freq;        // device, rot_dim / 2
};

namespace nq {

// how the other elements of a lane's eight pairs are had
enum { kPairInLane, kPairInChunk, kPairSingle };      // interleaved; halves, rot_dim / 2 a multiple of 8: the same places of another chunk; halves, else

struct RopeArgs {
    const void *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;
    const float *qw, *kw;
    const int32_t* positions;
    const int64_t* slots;           // with a cache
    const void *dq_out, *dk_out;    // backward
    int64_t dq_out_stride, dk_out_stride;
    void *q_out, *k_out;            // forward: results; backward: gradients
    int64_t q_out_stride, k_out_stride;
    KvDesc kv;
    const double* inv_freq;
    float* partial;                 // backward: [workgroups][2][head_dim], or nullptr
    float eps, weight_offset, magnitude, per_element;      // per_element: 1 / head_dim
    int n_tokens, q_heads, kv_heads, head_dim, rot_dim, pairing;
    int tokens_per_wg, heads_per_wg;   // heads_per_wg: of the token's q, k and v heads, numbered in this order
};

constexpr int kRopeThreads = 256;
constexpr int kRopeAngles = 512;        // pairs whose angles a workgroup holds at a time (4 KiB)

template <int DT>
__device__ __forceinline__ void store8(void* p, int64_t at, const float x[8])
{
    typedef __attribute__((address_space(1))) v4f_any* out_v4f;
    typedef __attribute__((address_space(1))) v4u_any* out_v4u;
    if (DT == NQ_F32) {
        *(out_v4f)((float*)p + at) = v4f{x[0], x[1], x[2], x[3]};
        *(out_v4f)((float*)p + at + 4) = v4f{x[4], x[5], x[6], x[7]};
    } else {
        v4u a;
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = round2<DT>(x[2 * i], x[2 * i + 1]);
        *(out_v4u)((uint16_t*)p + at) = a;
    }
}

// eight neighbouring elements as they are stored: loads under way take half the registers of their values
template <int DT>
struct Eight {
    v4u w[DT == NQ_F32 ? 2 : 1];
    __device__ __forceinline__ void load(const void* p, int64_t at)
    {
        const char* const from = (const char*)p + at * (DT == NQ_F32 ? 4 : 2);
        w[0] = *(gptr_v4u_any)from;
        if (DT == NQ_F32) w[DT == NQ_F32 ? 1 : 0] = *(gptr_v4u_any)(from + 16);
    }
    __device__ __forceinline__ float operator[](int i) const
    {
        const uint32_t bits = w[DT == NQ_F32 ? i >> 2 : 0][DT == NQ_F32 ? i & 3 : i >> 1];       // (a copy: __builtin_bit_cast of a vector's element takes its first)
        if (DT == NQ_F32) return __builtin_bit_cast(float, bits);
        const uint16_t h = (uint16_t)(bits >> (16 * (i & 1)));
        return DT == NQ_F16 ? half_bits_to_float(h) : bf16_bits_to_float(h);
    }
    // element i becomes element i + by, in a ring of eight (16-bit types)
    __device__ __forceinline__ Eight turned(int by) const
    {
        uint32_t x[4], y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = by & 4 ? w[0][(i + 2) & 3] : w[0][i];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = by & 2 ? x[(i + 1) & 3] : x[i];
        Eight t;
#pragma unroll
        for (int i = 0; i < 4; ++i) t.w[0][i] = __builtin_amdgcn_alignbit(y[(i + 1) & 3], y[i], 16 * (by & 1));
        return t;
    }
};

// The elements that form pairs with elements e0 .. e0 + 7 of the head at `at`: o (0 past rot).  fetch() asks for those that lie elsewhere, get() has them.
// Halves that are no whole chunks: 16-bit types read eight elements from e0 + half on and eight from e0 - half on, kept within the head and turned round to their places
// (what they lack lies outside the rotated part); fp32 reads single elements, as turning eight words costs more.  4093 tokens of 96 heads: 66 us, halves of whole chunks 53.
template <int DT, int PAIR>
struct Others {
    static constexpr bool kTurned = PAIR == kPairSingle && DT != NQ_F32, kEach = PAIR == kPairSingle && DT == NQ_F32;
    Eight<DT> raw[kTurned ? 2 : 1];
    __device__ __forceinline__ static int within(int e, int dim) { return min(max(e, 0), dim - 8); }
    __device__ __forceinline__ void fetch(const void* p, int64_t at, int e0, int rot, int dim)
    {
        const int half = rot >> 1;
        if (PAIR == kPairInChunk) raw[0].load(p, at + (e0 < half ? e0 + half : e0 < rot ? e0 - half : e0));
        if (kTurned) {
            raw[0].load(p, at + within(e0 + half, dim));
            raw[kTurned ? 1 : 0].load(p, at + within(e0 - half, dim));
        }
        if (kEach) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int e = e0 + i;
                raw[0].w[kEach ? i >> 2 : 0][i & 3] = ((const uint32_t*)p)[at + (e < half ? e + half : e < rot ? e - half : e)];
            }
        }
    }
    __device__ __forceinline__ void get(int e0, int rot, int dim, const Eight<DT>& own, float o[8]) const
    {
        const int half = rot >> 1;
        if (PAIR == kPairInLane) {
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = e0 + i < rot ? own[i ^ 1] : 0.f;
        } else if (!kTurned) {
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = (kEach ? e0 + i : e0) < rot ? raw[0][i] : 0.f;
        } else {
            const Eight<DT> up = raw[0].turned(e0 + half - within(e0 + half, dim)), down = raw[kTurned ? 1 : 0].turned(e0 - half - within(e0 - half, dim));
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int e = e0 + i;
                o[i] = e < half ? up[i] : e < rot ? down[i] : 0.f;
            }
        }
    }
};

// sum over the `lanes` (a power of two, at most 32) neighbours that share a head, by data-parallel moves up to 16: neighbours in twos, in fours, then the other half
// of eight and of 16 (mirrored: its lanes are alike by then)
__device__ __forceinline__ float head_sum(float v, int lanes)
{
    auto add = [&](auto ctrl) { v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, 0xf, 0xf, false)); };
    if (lanes > 1) add(std::integral_constant<int, 0xb1>());
    if (lanes > 2) add(std::integral_constant<int, 0x4e>());
    if (lanes > 4) add(std::integral_constant<int, 0x141>());
    if (lanes > 8) add(std::integral_constant<int, 0x140>());
    if (lanes > 16) v += __shfl_xor(v, 16);
    return v;
}

// 1 / sqrt(mean of squares + eps), by the instruction (within a unit of its last place) except where that would take a subnormal number for zero
__device__ __forceinline__ float rsqrt_of(float sum, const RopeArgs& a)
{
    const float s = fmaf(sum, a.per_element, a.eps);
    return s >= 1e-30f ? __builtin_amdgcn_rsqf(s) : 1.f / sqrtf(s);
}

// magnitude (cos, sin) of pair i at a position
__device__ __forceinline__ float2 rope_angle(const RopeArgs& a, int token, int i)
{
    const double t = (double)a.positions[token] * a.inv_freq[i];
    const double turns = rint(t * 0.15915494309189535);
    const float r = (float)fma(turns, -2.4492935982947064e-16, fma(turns, -6.283185307179586, t));    // 2 pi in two parts
    float s, c;
    sincosf(r, &s, &c);
    return make_float2(c * a.magnitude, s * a.magnitude);
}

// What a lane keeps of a token: C and S of its elements (1 and 0 past rot_dim), times the weights of the element and of its pair's other
struct LaneCoef {
    float c[8], s[8];
};
template <int PAIR>
__device__ __forceinline__ LaneCoef lane_coef(const RopeArgs& a, const float2* angles, int e0)
{
    LaneCoef l;
    const int half = a.rot_dim >> 1;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int e = e0 + i;
        l.c[i] = 1.f;
        l.s[i] = 0.f;
        if (e < a.rot_dim) {
            const bool first = PAIR == kPairInLane ? !(e & 1) : e < half;
            const float2 cs = angles[PAIR == kPairInLane ? e >> 1 : first ? e : e - half];
            l.c[i] = cs.x;
            l.s[i] = first ? -cs.y : cs.y;
        }
    }
    return l;
}
__device__ __forceinline__ void lane_weights(const float* w, const RopeArgs& a, int e0, float own[8])
{
    Eight<NQ_F32> raw;
    raw.load(w, e0);
#pragma unroll
    for (int i = 0; i < 8; ++i) own[i] = raw[i] + a.weight_offset;
}
template <int PAIR>
__device__ __forceinline__ void weigh(LaneCoef& l, const float* w, const RopeArgs& a, int e0)
{
    Eight<NQ_F32> own;
    Others<NQ_F32, PAIR> there;
    own.load(w, e0);
    there.fetch(w, 0, e0, a.rot_dim, a.head_dim);
    float other[8];
    there.get(e0, a.rot_dim, a.head_dim, own, other);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        l.c[i] *= own[i] + a.weight_offset;
        l.s[i] *= other[i] + a.weight_offset;
    }
}

// The workgroup's tokens, as many at a time as their angles fit; F(token, angles of the token) runs for each.
template <class F>
__device__ __forceinline__ void for_tokens(const RopeArgs& a, F f)
{
    __shared__ float2 angles[kRopeAngles];
    const int half = a.rot_dim >> 1;
    const int t0 = blockIdx.x * a.tokens_per_wg, t1 = min(a.n_tokens, t0 + a.tokens_per_wg);
    const int batch = half > 0 ? kRopeAngles / half : a.tokens_per_wg;             // >= 4: rot_dim <= 256
    for (int b0 = t0; b0 < t1; b0 += batch) {
        const int n = min(batch, t1 - b0);
        if (b0 != t0) __syncthreads();
        for (int i = threadIdx.x; i < n * half; i += kRopeThreads) angles[i] = rope_angle(a, b0 + i / half, i % half);
        __syncthreads();
        for (int i = 0; i < n; ++i) f(b0 + i, angles + i * half);
    }
}

// ---------------------------------------------------------------------------------------------
// Forward.  blockIdx.x: tokens; blockIdx.y: a part of the token's heads.
// ---------------------------------------------------------------------------------------------
template <int IN, int OUT, int PAIR, bool CACHE>
__global__ __launch_bounds__(kRopeThreads) void rope_forward_kernel(RopeArgs a, int lanes)
{
    constexpr int kHeads = 2;
    const int group = threadIdx.x / lanes, groups = kRopeThreads / lanes;
    const bool live = (int)(threadIdx.x % lanes) * 8 < a.head_dim;       // head_dim / 8 is no power of two: idle lanes, which follow the last one
    const int e0 = min((int)(threadIdx.x % lanes) * 8, a.head_dim - 8);
    const int h0 = blockIdx.y * a.heads_per_wg, h1 = h0 + a.heads_per_wg;
    for_tokens(a, [&](int t, const float2* angles) {
        int64_t to = -1;                                     // where the token's head 0 lies in the cache
        if (CACHE) {
            const int64_t slot = a.slots[t];
            if (slot >= 0 && slot < (a.kv.n_pages << a.kv.page_shift))
                to = (slot >> a.kv.page_shift) * a.kv.page_stride + (slot & ((1 << a.kv.page_shift) - 1)) * a.kv.slot_stride;
        }
        // heads of q and of k, kHeads of a group of lanes under way at a time
        auto rotate = [&](int first, int last, const void* x, int64_t base, const float* w, bool to_cache, void* out, int64_t out_base) {
            if (first >= last) return;
            LaneCoef m = lane_coef<PAIR>(a, angles, e0);
            if (w) weigh<PAIR>(m, w, a, e0);
            for (int h = first + group; h - group < last; h += kHeads * groups) {
                Eight<IN> own[kHeads];
                Others<IN, PAIR> there[kHeads];
                auto place = [&](int u) { return base + (int64_t)min(h + u * groups, last - 1) * a.head_dim; };
#pragma unroll
                for (int u = 0; u < kHeads; ++u) {
                    own[u].load(x, place(u) + e0);
                    there[u].fetch(x, place(u), e0, a.rot_dim, a.head_dim);
                }
#pragma unroll
                for (int u = 0; u < kHeads; ++u) {
                    float o[8], rstd = 1.f;
                    there[u].get(e0, a.rot_dim, a.head_dim, own[u], o);
                    if (w) {
                        float sum = 0.f;
#pragma unroll
                        for (int i = 0; i < 8; ++i) sum += own[u][i] * own[u][i];
                        sum = head_sum(live ? sum : 0.f, lanes);
                        rstd = rsqrt_of(sum, a);
                    }
                    if (!live || h + u * groups >= last) continue;
                    float y[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = rstd * own[u][i] * m.c[i] + rstd * o[i] * m.s[i];
                    if (to_cache) {
                        if (to >= 0) store8<OUT>(a.kv.k, to + (h + u * groups) * a.kv.head_stride + e0, y);
                    } else {
                        store8<OUT>(out, out_base + (int64_t)(h + u * groups) * a.head_dim + e0, y);
                    }
                }
            }
        };
        rotate(h0, min(h1, a.q_heads), a.q, t * a.q_stride, a.qw, false, a.q_out, t * a.q_out_stride);
        rotate(max(h0 - a.q_heads, 0), min(h1 - a.q_heads, a.kv_heads), a.k, t * a.k_stride, a.kw, CACHE, a.k_out, t * a.k_out_stride);
        if (CACHE && to >= 0 && live) {
            const int last = min(h1 - a.q_heads - a.kv_heads, a.kv_heads);
            for (int h = max(h0 - a.q_heads - a.kv_heads, 0) + group; h < last; h += kHeads * groups) {
                Eight<IN> v[kHeads];
#pragma unroll
                for (int u = 0; u < kHeads; ++u) v[u].load(a.v, t * a.v_stride + (int64_t)min(h + u * groups, last - 1) * a.head_dim + e0);
#pragma unroll
                for (int u = 0; u < kHeads; ++u) {
                    if (h + u * groups >= last) continue;
                    float y[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = v[u][i];
                    store8<OUT>(a.kv.v, to + (h + u * groups) * a.kv.head_stride + e0, y);
                }
            }
        }
    });
}

// ---------------------------------------------------------------------------------------------
// Backward:  g = R^T dy,  h = g (.) (w + offset),  xhat = rstd x:   dx = rstd (h - xhat mean(h (.) xhat)),  dw = sum g (.) xhat.
// The sums of a workgroup's tokens and heads stay in eight registers of a lane, are added up in LDS and left to rope_weight_grad_kernel:
// no atomics, the same bits every time.
// ---------------------------------------------------------------------------------------------
template <int IN, int OUT, int PAIR>
__global__ __launch_bounds__(kRopeThreads) void rope_backward_kernel(RopeArgs a, int lanes)
{
    constexpr int kHeads = 2;
    const int group = threadIdx.x / lanes, groups = kRopeThreads / lanes;
    const bool live = (int)(threadIdx.x % lanes) * 8 < a.head_dim;
    const int e0 = min((int)(threadIdx.x % lanes) * 8, a.head_dim - 8);
    float dw[2][8] = {};
    for_tokens(a, [&](int t, const float2* angles) {
        const LaneCoef l = lane_coef<PAIR>(a, angles, e0);
        auto turn_back = [&](int heads, const void* x, int64_t base, const void* dy, int64_t dy_base, const float* w, void* dx, int64_t dx_base, float sum_w[8]) {
            float weight[8];
            if (w) lane_weights(w, a, e0, weight);
            for (int h = group; h - group < heads; h += kHeads * groups) {
                Eight<IN> v[kHeads];
                Eight<OUT> own[kHeads];
                Others<OUT, PAIR> there[kHeads];
                auto head = [&](int u) { return (int64_t)min(h + u * groups, heads - 1) * a.head_dim; };
#pragma unroll
                for (int u = 0; u < kHeads; ++u) {
                    own[u].load(dy, dy_base + head(u) + e0);
                    there[u].fetch(dy, dy_base + head(u), e0, a.rot_dim, a.head_dim);
                    if (w) v[u].load(x, base + head(u) + e0);
                }
#pragma unroll
                for (int u = 0; u < kHeads; ++u) {
                    const bool mine = live && h + u * groups < heads;
                    float g[8], sum = 0.f, dot = 0.f;
                    there[u].get(e0, a.rot_dim, a.head_dim, own[u], g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) g[i] = own[u][i] * l.c[i] - g[i] * l.s[i];
                    if (w) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            sum += v[u][i] * v[u][i];
                            dot += g[i] * weight[i] * v[u][i];
                        }
                        sum = head_sum(mine ? sum : 0.f, lanes);
                        dot = head_sum(mine ? dot : 0.f, lanes);
                    }
                    if (!mine) continue;
                    if (w) {
                        const float rstd = rsqrt_of(sum, a);
                        const float back = dot * rstd * rstd * a.per_element;        // mean(h xhat) rstd
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            sum_w[i] += g[i] * (v[u][i] * rstd);
                            g[i] = rstd * (g[i] * weight[i] - v[u][i] * back);
                        }
                    }
                    store8<IN>(dx, dx_base + (int64_t)(h + u * groups) * a.head_dim + e0, g);
                }
            }
        };
        turn_back(a.q_heads, a.q, t * a.q_stride, a.dq_out, t * a.dq_out_stride, a.qw, a.q_out, t * a.q_out_stride, dw[0]);
        turn_back(a.kv_heads, a.k, t * a.k_stride, a.dk_out, t * a.dk_out_stride, a.kw, a.k_out, t * a.k_out_stride, dw[1]);
    });
    if (!a.partial) return;
    // one of the two sums at a time: [lanes' elements][groups], the groups of an element side by side
    __shared__ float sums[kRopeThreads * 8];
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (live) sums[(e0 + i) * groups + group] = dw[which][i];
        __syncthreads();
        for (int e = threadIdx.x; e < a.head_dim; e += kRopeThreads) {
            float s = 0.f;
            for (int g = 0; g < groups; ++g) s += sums[e * groups + g];
            a.partial[((int64_t)blockIdx.x * 2 + which) * a.head_dim + e] = s;
        }
    }
}

// sums of the workgroups' parts: a workgroup for 16 elements of one weight, 64 threads an element
__global__ __launch_bounds__(1024) void rope_weight_grad_kernel(const float* __restrict__ partial, int parts, int head_dim, float* dqw, float* dkw)
{
    __shared__ float sums[64][17];
    float* const out = blockIdx.y ? dkw : dqw;
    if (!out) return;
    const int e = blockIdx.x * 16 + (threadIdx.x & 15), row = threadIdx.x >> 4;
    float s = 0.f;
    if (e < head_dim) {
#pragma unroll 8
        for (int p = row; p < parts; p += 64) s += partial[((int64_t)p * 2 + blockIdx.y) * head_dim + e];
    }
    sums[row][threadIdx.x & 15] = s;
    __syncthreads();
    if (threadIdx.x < 16 && e < head_dim) {
        s = 0.f;
#pragma unroll
        for (int r = 0; r < 64; ++r) s += sums[r][threadIdx.x];
        out[e] = s;
    }
}

__global__ void clear_floats_kernel(float* a, float* b, int n)
{
    if ((int)threadIdx.x < n) {
        if (a) a[threadIdx.x] = 0.f;
        if (b) b[threadIdx.x] = 0.f;
    }
}

static int head_lanes(int head_dim)
{
    int lanes = 1;
    while (lanes * 8 < head_dim) lanes <<= 1;
    return lanes;
}

// workgroups of the backward: four to a CU, as long as a workgroup has a token
static int backward_workgroups(int n_tokens) { return std::max(1, std::min(n_tokens, 4 * device_cu_count())); }

static RopeArgs base_args(nq_rope r, int n_tokens, const float* qw, const float* kw, const int32_t* positions)
{
    RopeArgs a = {};
    a.qw = qw;
    a.kw = kw;
    a.positions = positions;
    a.inv_freq = r->inv_freq;
    a.eps = r->eps;
    a.per_element = 1.f / (float)r->head_dim;
    a.weight_offset = r->weight_offset;
    a.magnitude = r->magnitude;
    a.n_tokens = n_tokens;
    a.q_heads = r->q_heads;
    a.kv_heads = r->kv_heads;
    a.head_dim = r->head_dim;
    a.rot_dim = r->rot_dim;
    a.pairing = r->layout == NQ_ROPE_INTERLEAVED ? kPairInLane : r->rot_dim % 16 == 0 ? kPairInChunk : kPairSingle;
    return a;
}

static int check_tensor(const char* who, const char* name, const void* p, int64_t stride, int64_t width, int dtype)
{
    if (!p) return refuse(NQ_E_NULL, who, "%s is NULL", name);
    if (off_align(p, type_bytes(dtype))) return refuse(NQ_E_ALIGN, who, "%s must have the alignment of its elements", name);
    if (stride < width) return refuse(NQ_E_SHAPE, who, "%s: stride between tokens below a token's length", name);
    if (stride > (INT64_C(1) << 31)) return refuse(NQ_E_SHAPE, who, "%s: stride beyond 2^31", name);
    return NQ_OK;
}

static int check_call(const char* who, nq_rope r, const float* qw, const float* kw, const int32_t* positions, int n_tokens)
{
    if (!r) return refuse(NQ_E_NULL, who, "NULL handle");
    if (n_tokens < 0) return refuse(NQ_E_INVALID_ARG, who, "n_tokens must be >= 0");
    if (n_tokens > 0 && !positions) return refuse(NQ_E_NULL, who, "positions is NULL");
    if (off_align(positions, 4) || off_align(qw, 4) || off_align(kw, 4)) return refuse(NQ_E_ALIGN, who, "positions and weights must be 4-byte aligned");
    int device = -1;
    NQ_HIP(hipGetDevice(&device));
    if (device != r->device) return refuse(NQ_E_INVALID_ARG, who, "the handle lives on another device than the current one");
    return NQ_OK;
}

// dispatch over the types and the pairing: f(integral_constant IN, OUT, PAIR)
template <class F>
static void with_kernel(int in, int out, int pairing, F f)
{
    auto paired = [&](auto i, auto o) {
        if (pairing == kPairInLane) f(i, o, std::integral_constant<int, kPairInLane>());
        else if (pairing == kPairInChunk) f(i, o, std::integral_constant<int, kPairInChunk>());
        else f(i, o, std::integral_constant<int, kPairSingle>());
    };
    auto inner = [&](auto i) {
        if (out == NQ_F32) paired(i, std::integral_constant<int, NQ_F32>());
        else if (out == NQ_F16) paired(i, std::integral_constant<int, NQ_F16>());
        else paired(i, std::integral_constant<int, NQ_BF16>());
    };
    if (in == NQ_F32) inner(std::integral_constant<int, NQ_F32>());
    else if (in == NQ_F16) inner(std::integral_constant<int, NQ_F16>());
    else inner(std::integral_constant<int, NQ_BF16>());
}

// How a forward is cut: one token to a workgroup and its heads dealt out where there are few tokens (a workgroup's pass over as many heads as it
// has groups of lanes is the least), whole tokens where those alone fill the chip.
static dim3 cut_forward(RopeArgs& a, int heads, int lanes)
{
    const int groups = kRopeThreads / lanes, passes = (heads + groups - 1) / groups;
    const int want = 8 * device_cu_count();
    // (four tokens have angles for all threads of a workgroup)
    a.tokens_per_wg = std::max(1, std::min(4, a.n_tokens / (8 * device_cu_count())));
    int parts = std::min(passes, std::max(1, want / std::max(1, a.n_tokens)));
    a.heads_per_wg = (passes + parts - 1) / parts * groups;
    parts = (heads + a.heads_per_wg - 1) / a.heads_per_wg;
    return dim3((a.n_tokens + a.tokens_per_wg - 1) / a.tokens_per_wg, parts);
}

}  // namespace nq

using namespace nq;

extern "C" int nq_rope_freqs(int kind, int rot_dim, double base, double factor, double trained_len, double low, double high, double* inv_freq, double* magnitude)
{
    const char* const who = "nq_rope_freqs";
    if (!inv_freq || !magnitude) return refuse(NQ_E_NULL, who, "inv_freq or magnitude is NULL");
    if (kind < NQ_ROPE_PLAIN || kind > NQ_ROPE_BANDED) return refuse(NQ_E_INVALID_ARG, who, "unknown kind");
    if (rot_dim < 2 || rot_dim % 2 || rot_dim > NQ_MAX_HEAD_DIM) return refuse(NQ_E_SHAPE, who, "rot_dim must be even, 2 to %d", NQ_MAX_HEAD_DIM);
    if (!(base > 1.0) || !std::isfinite(base)) return refuse(NQ_E_INVALID_ARG, who, "base must be above 1");
    if (kind != NQ_ROPE_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return refuse(NQ_E_INVALID_ARG, who, "factor must be at least 1");
    if (kind == NQ_ROPE_BASE && rot_dim == 2) return refuse(NQ_E_SHAPE, who, "rot_dim must be above 2 for NQ_ROPE_BASE");
    if (kind >= NQ_ROPE_YARN && (!(trained_len >= 1.0) || !std::isfinite(trained_len) || !(low > 0.0) || !(high > low) || !std::isfinite(high)))
        return refuse(NQ_E_INVALID_ARG, who, "trained_len must be at least 1 and 0 < low < high");
    const double two_pi = 6.283185307179586;
    if (kind == NQ_ROPE_BASE) base *= std::pow(factor, rot_dim / (rot_dim - 2.0));
    *magnitude = kind == NQ_ROPE_YARN ? 0.1 * std::log(factor) + 1.0 : 1.0;
    // the pair, as a real number, that turns n times over the trained length
    auto pair_of = [&](double n) { return rot_dim * std::log(trained_len / (n * two_pi)) / (2.0 * std::log(base)); };
    double from = 0.0, to = 0.0;
    if (kind == NQ_ROPE_YARN) {
        from = std::max(0.0, std::floor(pair_of(high)));
        to = std::min(rot_dim - 1.0, std::ceil(pair_of(low)));
        if (to <= from) to = from + 0.001;
    }
    for (int i = 0; i < rot_dim / 2; ++i) {
        const double f = std::pow(base, -2.0 * i / rot_dim);
        double g = 1.0;                                       // how much of f is kept as it is
        if (kind == NQ_ROPE_LINEAR) g = 0.0;
        if (kind == NQ_ROPE_YARN) g = 1.0 - std::min(1.0, std::max(0.0, (i - from) / (to - from)));
        if (kind == NQ_ROPE_BANDED) g = std::min(1.0, std::max(0.0, (trained_len * f / two_pi - low) / (high - low)));
        inv_freq[i] = kind == NQ_ROPE_PLAIN || kind == NQ_ROPE_BASE ? f : f * ((1.0 - g) / factor + g);
    }
    return NQ_OK;
}

extern "C" int nq_rope_create(nq_rope* out, int q_heads, int kv_heads, int head_dim, int rot_dim, int layout, const double* inv_freq, double magnitude, double eps,
                              double weight_offset, int in_dtype, int out_dtype)
{
    const char* const who = "nq_rope_create";
    if (!out) return refuse(NQ_E_NULL, who, "out is NULL");
    *out = nullptr;
    if (q_heads < 1 || kv_heads < 1 || q_heads % kv_heads || q_heads > 65535) return refuse(NQ_E_SHAPE, who, "q_heads must be a multiple of kv_heads, at most 65535");
    if (head_dim < 8 || head_dim > NQ_MAX_HEAD_DIM || head_dim % 8) return refuse(NQ_E_SHAPE, who, "head_dim must be a multiple of 8, 8 to %d", NQ_MAX_HEAD_DIM);
    if (rot_dim < 0 || rot_dim > head_dim || rot_dim % 2) return refuse(NQ_E_SHAPE, who, "rot_dim must be even, 0 to head_dim");
    if (layout != NQ_ROPE_HALF && layout != NQ_ROPE_INTERLEAVED) return refuse(NQ_E_INVALID_ARG, who, "unknown layout");
    if (rot_dim > 0 && !inv_freq) return refuse(NQ_E_NULL, who, "inv_freq is NULL");
    for (int i = 0; i < rot_dim / 2; ++i)
        if (!std::isfinite(inv_freq[i])) return refuse(NQ_E_INVALID_ARG, who, "inv_freq holds a value that is not finite");
    if (!std::isfinite((float)magnitude) || !std::isfinite((float)weight_offset)) return refuse(NQ_E_INVALID_ARG, who, "magnitude and weight_offset must be finite in fp32");
    if (!(eps >= 0.0) || !std::isfinite((float)eps)) return refuse(NQ_E_INVALID_ARG, who, "eps must be at least 0 and finite in fp32");
    if (!is_float_type(in_dtype) || !is_float_type(out_dtype)) return refuse(NQ_E_INVALID_ARG, who, "types must be NQ_F32, NQ_F16 or NQ_BF16");
    int device = -1;
    NQ_HIP(hipGetDevice(&device));
    nq_rope r = new (std::nothrow) nq_rope_s{q_heads, kv_heads, head_dim, rot_dim, layout, in_dtype, out_dtype, device, (float)eps, (float)weight_offset, (float)magnitude, nullptr};
    if (!r) return refuse(NQ_E_HIP, who, "out of host memory");
    const size_t bytes = std::max(2, rot_dim) / 2 * sizeof(double);
    hipError_t e = hipMalloc((void**)&r->inv_freq, bytes);
    if (e == hipSuccess && rot_dim > 0) e = hipMemcpy(r->inv_freq, inv_freq, bytes, hipMemcpyHostToDevice);
    if (e != hipSuccess) {
        nq_rope_destroy(r);
        return hip_fail(e, "nq_rope_create", __FILE__, __LINE__);
    }
    *out = r;
    return NQ_OK;
}

extern "C" int nq_rope_destroy(nq_rope r)
{
    if (!r) return NQ_OK;
    const hipError_t e = r->inv_freq ? hipFree(r->inv_freq) : hipSuccess;
    delete r;
    return e == hipSuccess ? NQ_OK : hip_fail(e, "nq_rope_destroy", __FILE__, __LINE__);
}

extern "C" int nq_rope_forward(nq_rope r, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const float* q_weight, const float* k_weight,
                               const int32_t* positions, int n_tokens, void* q_out, int64_t q_out_stride, void* k_out, int64_t k_out_stride, void* stream)
{
    const char* const who = "nq_rope_forward";
    if (const int rc = check_call(who, r, q_weight, k_weight, positions, n_tokens)) return rc;
    if (n_tokens == 0) return NQ_OK;
    const int64_t qw = (int64_t)r->q_heads * r->head_dim, kw = (int64_t)r->kv_heads * r->head_dim;
    if (const int rc = check_tensor(who, "q", q, q_stride, qw, r->in_dtype)) return rc;
    if (const int rc = check_tensor(who, "k", k, k_stride, kw, r->in_dtype)) return rc;
    if (const int rc = check_tensor(who, "q_out", q_out, q_out_stride, qw, r->out_dtype)) return rc;
    if (const int rc = check_tensor(who, "k_out", k_out, k_out_stride, kw, r->out_dtype)) return rc;
    RopeArgs a = base_args(r, n_tokens, q_weight, k_weight, positions);
    a.q = q; a.k = k; a.q_stride = q_stride; a.k_stride = k_stride;
    a.q_out = q_out; a.k_out = k_out; a.q_out_stride = q_out_stride; a.k_out_stride = k_out_stride;
    const int lanes = head_lanes(r->head_dim);
    const dim3 grid = cut_forward(a, r->q_heads + r->kv_heads, lanes);
    with_kernel(r->in_dtype, r->out_dtype, a.pairing, [&](auto in, auto out, auto pair) {
        hipLaunchKernelGGL((rope_forward_kernel<decltype(in)::value, decltype(out)::value, decltype(pair)::value, false>), grid, dim3(kRopeThreads), 0, (hipStream_t)stream, a, lanes);
    });
    return launched(who);
}

extern "C" int nq_rope_cache(nq_rope r, nq_kv kv, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride, const float* q_weight,
                             const float* k_weight, const int32_t* positions, const int64_t* slots, int n_tokens, void* q_out, int64_t q_out_stride, void* stream)
{
    const char* const who = "nq_rope_cache";
    if (!kv) return refuse(NQ_E_NULL, who, "NULL cache");
    if (const int rc = check_call(who, r, q_weight, k_weight, positions, n_tokens)) return rc;
    if (kv->d.heads != r->kv_heads || kv->d.head_dim != r->head_dim) return refuse(NQ_E_SHAPE, who, "the cache's heads are not the handle's");
    if (kv->d.dtype != r->out_dtype) return refuse(NQ_E_INVALID_ARG, who, "the cache's type is not the handle's out_dtype");
    if (n_tokens == 0) return NQ_OK;
    const int64_t qw = (int64_t)r->q_heads * r->head_dim, kw = (int64_t)r->kv_heads * r->head_dim;
    if (const int rc = check_tensor(who, "q", q, q_stride, qw, r->in_dtype)) return rc;
    if (const int rc = check_tensor(who, "k", k, k_stride, kw, r->in_dtype)) return rc;
    if (const int rc = check_tensor(who, "v", v, v_stride, kw, r->in_dtype)) return rc;
    if (const int rc = check_tensor(who, "q_out", q_out, q_out_stride, qw, r->out_dtype)) return rc;
    if (!slots) return refuse(NQ_E_NULL, who, "slots is NULL");
    if (off_align(slots, 8)) return refuse(NQ_E_ALIGN, who, "slots must be 8-byte aligned");
    RopeArgs a = base_args(r, n_tokens, q_weight, k_weight, positions);
    a.q = q; a.k = k; a.v = v; a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride;
    a.slots = slots;
    a.kv = kv->d;
    a.q_out = q_out; a.q_out_stride = q_out_stride;
    const int lanes = head_lanes(r->head_dim);
    const dim3 grid = cut_forward(a, r->q_heads + 2 * r->kv_heads, lanes);
    with_kernel(r->in_dtype, r->out_dtype, a.pairing, [&](auto in, auto out, auto pair) {
        if constexpr (decltype(out)::value != NQ_F32)
            hipLaunchKernelGGL((rope_forward_kernel<decltype(in)::value, decltype(out)::value, decltype(pair)::value, true>), grid, dim3(kRopeThreads), 0, (hipStream_t)stream, a, lanes);
    });
    return launched(who);
}

extern "C" int nq_rope_backward_workspace_bytes(nq_rope r, int n_tokens, size_t* bytes)
{
    const char* const who = "nq_rope_backward_workspace_bytes";
    if (!r || !bytes) return refuse(NQ_E_NULL, who, "NULL handle or pointer");
    if (n_tokens < 0) return refuse(NQ_E_INVALID_ARG, who, "n_tokens must be >= 0");
    *bytes = (size_t)backward_workgroups(n_tokens) * 2 * r->head_dim * sizeof(float);
    return NQ_OK;
}

extern "C" int nq_rope_backward(nq_rope r, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const float* q_weight, const float* k_weight,
                                const int32_t* positions, int n_tokens, const void* dq_out, int64_t dq_out_stride, const void* dk_out, int64_t dk_out_stride, void* dq,
                                int64_t dq_stride, void* dk, int64_t dk_stride, float* dq_weight, float* dk_weight, void* workspace, size_t workspace_bytes, void* stream)
{
    const char* const who = "nq_rope_backward";
    if (const int rc = check_call(who, r, q_weight, k_weight, positions, n_tokens)) return rc;
    if ((dq_weight && !q_weight) || (dk_weight && !k_weight)) return refuse(NQ_E_INVALID_ARG, who, "a gradient is asked for of a weight that is NULL");
    if (off_align(dq_weight, 4) || off_align(dk_weight, 4)) return refuse(NQ_E_ALIGN, who, "dq_weight and dk_weight must be 4-byte aligned");
    if (n_tokens == 0) {
        if (dq_weight || dk_weight) hipLaunchKernelGGL(clear_floats_kernel, dim3(1), dim3(256), 0, (hipStream_t)stream, dq_weight, dk_weight, r->head_dim);
        return launched(who);
    }
    const int64_t qw = (int64_t)r->q_heads * r->head_dim, kw = (int64_t)r->kv_heads * r->head_dim;
    if (const int rc = check_tensor(who, "q", q, q_stride, qw, r->in_dtype)) return rc;
    if (const int rc = check_tensor(who, "k", k, k_stride, kw, r->in_dtype)) return rc;
    if (const int rc = check_tensor(who, "dq_out", dq_out, dq_out_stride, qw, r->out_dtype)) return rc;
    if (const int rc = check_tensor(who, "dk_out", dk_out, dk_out_stride, kw, r->out_dtype)) return rc;
    if (const int rc = check_tensor(who, "dq", dq, dq_stride, qw, r->in_dtype)) return rc;
    if (const int rc = check_tensor(who, "dk", dk, dk_stride, kw, r->in_dtype)) return rc;
    RopeArgs a = base_args(r, n_tokens, q_weight, k_weight, positions);
    const int workgroups = backward_workgroups(n_tokens);
    if (dq_weight || dk_weight) {
        if (!workspace) return refuse(NQ_E_NULL, who, "workspace is NULL");
        if (off_align(workspace, 16)) return refuse(NQ_E_ALIGN, who, "workspace must be 16-byte aligned");
        if (workspace_bytes < (size_t)workgroups * 2 * r->head_dim * sizeof(float)) return refuse(NQ_E_INVALID_ARG, who, "workspace too small");
        a.partial = (float*)workspace;
    }
    a.q = q; a.k = k; a.q_stride = q_stride; a.k_stride = k_stride;
    a.dq_out = dq_out; a.dk_out = dk_out; a.dq_out_stride = dq_out_stride; a.dk_out_stride = dk_out_stride;
    a.q_out = dq; a.k_out = dk; a.q_out_stride = dq_stride; a.k_out_stride = dk_stride;
    a.tokens_per_wg = (n_tokens + workgroups - 1) / workgroups;
    const int lanes = head_lanes(r->head_dim), grid = (n_tokens + a.tokens_per_wg - 1) / a.tokens_per_wg;
    with_kernel(r->in_dtype, r->out_dtype, a.pairing, [&](auto in, auto out, auto pair) {
        hipLaunchKernelGGL((rope_backward_kernel<decltype(in)::value, decltype(out)::value, decltype(pair)::value>), dim3(grid), dim3(kRopeThreads), 0, (hipStream_t)stream, a, lanes);
    });
    if (const int rc = launched(who)) return rc;
    if (a.partial)
        hipLaunchKernelGGL(rope_weight_grad_kernel, dim3((r->head_dim + 15) / 16, 2), dim3(1024), 0, (hipStream_t)stream, a.partial, grid, r->head_dim, dq_weight, dk_weight);
    return launched(who);
}
