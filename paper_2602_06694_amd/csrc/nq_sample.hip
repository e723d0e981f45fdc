// Next tokens from logits: temperature, top-k, top-p and min-p from given uniform numbers (nq_decoder.h).
//
// All three limits keep a prefix of the tokens in falling order of their logits, and so does the draw look for a place in that order: the
// token at which the running sum of weights passes a number.  Each is therefore the same question -- the first place at which the count
// (top-k) or the sum (top-p, the draw) reaches a value -- and none needs the vocabulary sorted: a histogram over the distance from
// the largest logit answers it up to a bin, whose few tokens are then sorted in LDS.  Weights are whole multiples of 2^-31 of the largest, so
// that sums are exact in whatever order atomics add them: the answer is that of a sequential sum, the same bits every time.
//
// Three passes read a row: its largest logit, the histogram, the tokens of the bins in question (one bin range serves all questions as a rule); the
// passes after the first read from the caches.  One workgroup does all of it where there are rows for every CU; with fewer rows the first two passes are launches of
// their own, with several workgroups to a row, whose histograms the third adds up.  The histogram is bound by the vector unit (an exponential and some 25
// other instructions a logit), the rest by latency.  192 rows of 131071 bf16 logits, top-p and min-p: 11.5, 26 and 37 us for the three launches (50 MB: 7.4 at the rate of a
// plain read), 10 of the last for its pass over the row; one row of 32000 fp32 logits, top-k and top-p: 15.8 us in one workgroup.
#include <algorithm>

#include "nq_decoder_internal.h"

namespace nq {

struct SampleArgs {
    const void* logits;
    const float *temperature, *top_p, *min_p, *uniform;
    const int32_t* top_k;
    int32_t* tokens;
    float* logprobs;
    int64_t row_stride;
    int vocab;
    int slices;                             // parts of a row that workgroups of their own take (1: none do)
    struct SamplePart* parts;               // [rows][slices], in the workspace
};

constexpr int kSampleThreads = 1024;
constexpr int kBins = 2048;             // two a thread
constexpr int kListed = 1024;           // tokens that are put in order in LDS, one a thread
constexpr int kRanked = 256;            // as many are ordered by comparing each with all, more by sorting
constexpr int kFew = 512;               // as many asked for by top-k are listed right away, with those that share the last one's bin
// bins per unit of z: weights are 0 below z = -32 ln 2 = -22.18
constexpr float kBinScale = kBins / 22.2f;

constexpr int kMostSlices = 8;

// what a workgroup finds in its part of a row
struct SamplePart {
    uint64_t mass[kBins];
    uint32_t count[kBins];
    uint64_t kept;
    float top;
    int nan;
};

struct TopLds {                                     // of the waves
    float top[kSampleThreads / 64];
    int nan[kSampleThreads / 64];
};
struct SampleLds {
    uint64_t mass[kBins], mass2[kBins];             // running sums over the bins; of the bins a crowded bin is cut into
    uint32_t count[kBins], count2[kBins];           // count: where top-k asks for it exactly, else bounds from above
    uint64_t list[kListed], upto[kListed];          // tokens, in any order, and the sums of their weights up to each in the order
    uint32_t rank[kListed], weight[kListed];
    uint64_t part_mass[16], lo, hi;
    uint32_t part_count[16], n, found;
    TopLds part_top;
};

// x's place in falling order, then the token: ascending numbers are the order of the tokens
__device__ __forceinline__ uint64_t order_of(float x, int token)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.f);       // (-0 is 0)
    const uint32_t rising = u >> 31 ? ~u : u | 0x80000000u;
    return (uint64_t)~rising << 32 | (uint32_t)token;
}
__device__ __forceinline__ float logit_of(uint64_t order)
{
    const uint32_t rising = ~(uint32_t)(order >> 32);
    return __builtin_bit_cast(float, rising >> 31 ? rising & 0x7fffffffu : ~rising);
}

struct Weights {
    float top, inverse;
    // (an infinite temperature makes all logits alike but those of minus infinity)
    __device__ __forceinline__ Weights() = default;
    __device__ __forceinline__ Weights(float top, float temperature) : top(top), inverse(fmaxf(1.f / temperature, 1.17549435e-38f)) {}
    // at most 0; what is not a number (infinity less infinity, zero times infinity) is the largest logit's own
    __device__ __forceinline__ float z(float x) const { return fminf((x - top) * inverse, 0.f); }
    __device__ __forceinline__ float e(float z) const { return expf(z); }
    __device__ __forceinline__ uint32_t w(float e) const { return (uint32_t)rintf(e * 2147483648.f); }
    __device__ __forceinline__ int bin(float z) const { return (int)fminf(-z * kBinScale, (float)(kBins - 1)); }
    // the least weight that a token of bin b can have (rounding of z, of the exponential and of the weight allowed for): bounds how many there are
    __device__ __forceinline__ float least(int b) const { return fmaxf(1.f, expf(-(float)(b + 1) / kBinScale) * (2147483648.f * 0.9999f) - 1.f); }
};

constexpr uint64_t kNone = ~UINT64_C(0);        // no token: behind all in the order, weighs nothing
__device__ __forceinline__ uint64_t weight_of(const Weights& w, uint64_t order) { return order == kNone ? 0 : w.w(w.e(w.z(logit_of(order)))); }

// eight neighbouring logits as they are stored
template <int DT>
struct Eight {
    v4u w[DT == NQ_F32 ? 2 : 1];
    __device__ __forceinline__ void load(const void* row, int c)
    {
        w[0] = *(gptr_v4u_any)((const char*)row + (int64_t)c * (DT == NQ_F32 ? 32 : 16));
        if (DT == NQ_F32) w[DT == NQ_F32 ? 1 : 0] = *(gptr_v4u_any)((const char*)row + (int64_t)c * 32 + 16);
    }
    __device__ __forceinline__ float operator[](int i) const
    {
        const uint32_t bits = w[DT == NQ_F32 ? i >> 2 : 0][DT == NQ_F32 ? i & 3 : i >> 1];       // (a copy: __builtin_bit_cast of a vector's element takes its first)
        if (DT == NQ_F32) return __builtin_bit_cast(float, bits);
        const uint16_t h = (uint16_t)(bits >> (16 * (i & 1)));
        return DT == NQ_F16 ? half_bits_to_float(h) : bf16_bits_to_float(h);
    }
};

// part `part` of `parts` of a row: whole eights of its tokens, the last part those beyond as well
struct Span {
    int e0, e1, tail, vocab;
    __device__ __forceinline__ Span(int vocab, int part, int parts) : vocab(vocab)
    {
        const int eights = vocab >> 3, each = (eights + parts - 1) / parts;
        e0 = min(part * each, eights);
        e1 = min(e0 + each, eights);
        tail = part == parts - 1 ? 8 * eights : vocab;
    }
};

// whole(eight logits, first token) and single(logit, token) for the tokens of a span; a thread has kAtOnce loads of eight under way
template <int DT, int kAtOnce, class W, class S>
__device__ __forceinline__ void for_eights(const void* row, const Span& span, W whole, S single)
{
    for (int c0 = span.e0 + threadIdx.x; c0 < span.e1; c0 += kAtOnce * kSampleThreads) {
        Eight<DT> x[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) x[k].load(row, min(c0 + k * kSampleThreads, span.e1 - 1));
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
            if (c0 + k * kSampleThreads < span.e1) whole(x[k], 8 * (c0 + k * kSampleThreads));
    }
    const int t = span.tail + threadIdx.x;
    if (t < span.vocab) single(load_as_float(row, DT, t), t);
}
template <int DT, class F>
__device__ __forceinline__ void for_row(const void* row, int vocab, F f)
{
    for_eights<DT, DT == NQ_F32 ? 4 : 8>(row, Span(vocab, 0, 1), [&](const Eight<DT>& x, int t) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f(x[i], t + i);
    }, f);
}
// a range of logits
struct Near {
    float middle, half;
    __device__ __forceinline__ float off(float x) const { return fabsf(x - middle); }
    __device__ __forceinline__ bool has(float x) const { return off(x) <= half; }
};
// f(logit, token) for the tokens of a row that are in either range: few, found by the least distances of eight
template <int DT, class F>
__device__ __forceinline__ void for_near(const void* row, int vocab, const Near& p, const Near& q, F f)
{
    for_eights<DT, DT == NQ_F32 ? 4 : 8>(row, Span(vocab, 0, 1), [&](const Eight<DT>& x, int t) {
        float least = p.off(x[0]), least2 = q.off(x[0]);
#pragma unroll
        for (int i = 1; i < 8; ++i) {
            least = fminf(least, p.off(x[i]));
            least2 = fminf(least2, q.off(x[i]));
        }
        if (!(least <= p.half) && !(least2 <= q.half)) return;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (p.has(x[i]) || q.has(x[i])) f(x[i], t + i);
    }, [&](float x, int t) {
        if (p.has(x) || q.has(x)) f(x, t);
    });
}

// The largest logit of a thread's tokens, and whether one is NaN, from the bits: of numbers with a plus sign the largest integer is the largest number, of those with
// a minus sign the smallest unsigned one; NaN has the largest magnitude.  Two 16-bit logits an instruction.
template <int DT>
struct Top {
    static constexpr int kBits = DT == NQ_F32 ? 32 : 16;
    typedef typename std::conditional<DT == NQ_F32, int32_t, int16_t>::type I;
    typedef typename std::conditional<DT == NQ_F32, uint32_t, uint16_t>::type U;
    typedef I VI __attribute__((ext_vector_type(4 / sizeof(I))));
    typedef U VU __attribute__((ext_vector_type(4 / sizeof(U))));
    VI most = (I)((U)1 << (kBits - 1));
    VU least = (U)~(U)0, size = (U)0;
    __device__ __forceinline__ void add(uint32_t w)
    {
        constexpr uint32_t magnitude = DT == NQ_F32 ? 0x7fffffffu : 0x7fff7fffu;
        most = __builtin_elementwise_max(most, __builtin_bit_cast(VI, w));
        least = __builtin_elementwise_min(least, __builtin_bit_cast(VU, w));
        size = __builtin_elementwise_max(size, __builtin_bit_cast(VU, w & magnitude));
    }
    __device__ __forceinline__ void get(float* top, int* nan) const
    {
        constexpr uint32_t infinity = DT == NQ_F32 ? 0x7f800000u : DT == NQ_F16 ? 0x7c00u : 0x7f80u;
        I m = most[0];
        U l = least[0], z = size[0];
        if (DT != NQ_F32) {
            m = max(m, most[DT == NQ_F32 ? 0 : 1]);
            l = min(l, least[DT == NQ_F32 ? 0 : 1]);
            z = max(z, size[DT == NQ_F32 ? 0 : 1]);
        }
        const U bits = m >= 0 ? (U)m : l;
        *top = DT == NQ_F32 ? __builtin_bit_cast(float, (uint32_t)bits) : DT == NQ_F16 ? half_bits_to_float((uint16_t)bits) : bf16_bits_to_float((uint16_t)bits);
        *nan = z > infinity;
    }
};

// running sums over bins in place; both values of two neighbouring bins a thread
__device__ __forceinline__ void scan_bins(SampleLds& s, uint32_t* count, uint64_t* mass)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b = 2 * threadIdx.x;
    uint32_t c0 = count[b], c = c0 + count[b + 1];
    uint64_t m0 = mass[b], m = m0 + mass[b + 1];
    const uint32_t c_own = c - c0;
    const uint64_t m_own = m - m0;
    c = wave_scan(c);
    m = wave_scan(m);
    if (lane == 63) { s.part_count[wave] = c; s.part_mass[wave] = m; }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kSampleThreads / 64 - 1; ++w) {
        c += w < wave ? s.part_count[w] : 0u;
        m += w < wave ? s.part_mass[w] : 0ull;
    }
    count[b + 1] = c;
    count[b] = c - c_own;
    mass[b + 1] = m;
    mass[b] = m - m_own;
    __syncthreads();
}

// What is asked of the order: the first place where the running count, or sum, reaches something
struct Question {
    int kind;             // 0: count >= k; 1: sum >= need (binary64); 2: sum > target
    uint32_t k;
    double need;
    uint64_t target;
    __device__ __forceinline__ bool reached(uint32_t count, uint64_t mass) const
    {
        return kind == 0 ? count >= k : kind == 1 ? (double)mass >= need : mass > target;
    }
};

// the first bin that reaches it (there is one), to all threads
__device__ __forceinline__ int first_bin(SampleLds& s, const uint32_t* count, const uint64_t* mass, const Question& ask, uint32_t before, uint64_t mass_before)
{
    for (int b = threadIdx.x; b < kBins; b += kSampleThreads) {
        const bool earlier = b > 0 && ask.reached(before + count[b - 1], mass_before + mass[b - 1]);
        if (!earlier && ask.reached(before + count[b], mass_before + mass[b])) s.found = b;
    }
    __syncthreads();
    const int b = (int)s.found;
    __syncthreads();
    return b;
}

// the n tokens in s.list, sorted, and the running sums of their weights: a token a thread; steps within a wave need neither LDS nor barrier
__device__ __forceinline__ void sort_list(SampleLds& s, int n, const Weights& w)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint64_t x = (int)threadIdx.x < n ? s.list[threadIdx.x] : kNone;
    int size = 2;
    while (size < n) size <<= 1;
    for (int k = 2; k <= size; k <<= 1)
        for (int j = k >> 1; j > 0; j >>= 1) {
            uint64_t y;
            if (j >= 64) {
                __syncthreads();
                s.list[threadIdx.x] = x;
                __syncthreads();
                y = s.list[threadIdx.x ^ j];
            } else if (64 * wave < size) {
                y = __shfl_xor((unsigned long long)x, j);
            } else {
                continue;                                    // (a wave without places)
            }
            const bool keep_low = ((threadIdx.x & k) == 0) == ((threadIdx.x & j) == 0);
            x = keep_low ? min(x, y) : max(x, y);
        }
    const uint64_t own = weight_of(w, x);
    uint64_t sum = wave_scan(own);
    if (lane == 63) s.part_mass[wave] = sum;
    __syncthreads();
    for (int v = 0; v < wave; ++v) sum += s.part_mass[v];
    s.list[threadIdx.x] = x;
    s.upto[threadIdx.x] = sum;
    s.rank[threadIdx.x] = threadIdx.x;
    __syncthreads();
}

// the same for few tokens: each is compared with all.  A lane has every 64th of them, a wave one part of those that they are compared with, so that a read of LDS
// serves four comparisons of a lane (40 tokens: 1.3 us, 233: 3 us, where the comparisons in 64 bits bound it)
__device__ __forceinline__ void rank_list(SampleLds& s, int n, const Weights& w)
{
    constexpr int kWaves = kSampleThreads / 64, kEach = kRanked / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if ((int)threadIdx.x < kRanked) {
        s.weight[threadIdx.x] = (int)threadIdx.x < n ? (uint32_t)weight_of(w, s.list[threadIdx.x]) : 0u;
        s.upto[threadIdx.x] = 0;
        s.rank[threadIdx.x] = ~0u;                           // (the token itself is counted)
    }
    __syncthreads();
    const int each = (n + kWaves - 1) / kWaves, first = wave * each, last = min(n, first + each);
    if (first < last) {
        uint64_t own[kEach], sum[kEach];
        uint32_t upto[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            own[i] = s.list[lane + 64 * i];
            sum[i] = 0;
            upto[i] = 0;
        }
        for (int j = first; j < last; ++j) {
            const uint64_t other = s.list[j];
            const uint32_t weight = s.weight[j];
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const bool before = other <= own[i];
                sum[i] += before ? weight : 0u;
                upto[i] += before;
            }
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (lane + 64 * i < n) {
                atomicAdd((unsigned long long*)&s.upto[lane + 64 * i], (unsigned long long)sum[i]);
                atomicAdd(&s.rank[lane + 64 * i], upto[i]);
            }
    }
    __syncthreads();
}

struct Row {
    const void* logits;
    int vocab;
    Weights w;
    // what s.list holds: the tokens of these bins (both included), and what precedes them; and those of an earlier bin (-1: none), where the next question is expected to fall
    int first, last, n, lead;
    uint32_t before, lead_before, lead_count;
    uint64_t mass_before, lead_mass_before, lead_mass;
    bool whole;                   // the list holds all that the questions are about
};

struct Answer {
    uint64_t order, mass;         // the token, and the sum of weights up to it
};

// puts the tokens of bins first .. bin with orders from lo to hi in the list, in order, with those of r.lead
template <int DT>
__device__ __forceinline__ void gather(SampleLds& s, Row& r, int first, int bin, uint64_t lo, uint64_t hi)
{
    if (threadIdx.x == 0) s.n = 0;
    __syncthreads();
    // Logits within the bins' edges, a hundredth of a bin more on either side for rounding, are listed as they come; which of them are of the bins, weigh something and are in
    // the order's range is found afterwards, a thread each.
    const float unit = 1.f / (kBinScale * r.w.inverse);             // of a bin
    const bool extreme = r.w.top == INFINITY || !(unit > 0.f) || !(unit < 1e30f);
    auto edges = [&](int b0, int b1) {
        return Near{r.w.top - 0.5f * (float)(b0 + b1 + 1) * unit, (0.5f * (float)(b1 + 1 - b0) + 0.01f) * unit + 4e-7f * (fabsf(r.w.top) + (float)(b1 + 1) * unit)};
    };
    auto among = [&](uint64_t o) {
        const float z = r.w.z(logit_of(o));
        const int b = r.w.bin(z);
        return ((b >= first && b <= bin) || b == r.lead) && r.w.w(r.w.e(z)) != 0 && o >= lo && o <= hi;
    };
    auto list = [&](uint64_t o) {
        const uint32_t at = atomicAdd(&s.n, 1u);
        if (at < kListed) s.list[at] = o;
    };
    if (!extreme) {
        const Near own = edges(first, bin);
        for_near<DT>(r.logits, r.vocab, own, r.lead >= 0 ? edges(r.lead, r.lead) : own, [&](float x, int t) { list(order_of(x, t)); });
    }
    __syncthreads();
    if (extreme || s.n > kListed) {
        // (distances from an infinity, or in bins of no width, say nothing; or the hundredths hold too many, or the bin is crowded)
        __syncthreads();
        if (threadIdx.x == 0) s.n = 0;
        __syncthreads();
        for_row<DT>(r.logits, r.vocab, [&](float x, int t) {
            const uint64_t o = order_of(x, t);
            if (among(o)) list(o);
        });
        __syncthreads();
    }
    r.n = min((int)s.n, kListed);
    if ((int)threadIdx.x < r.n && !among(s.list[threadIdx.x])) s.list[threadIdx.x] = kNone;
    __syncthreads();
    if (r.n <= kRanked) rank_list(s, r.n, r.w);
    else sort_list(s, r.n, r.w);
}

// the sum of weights up to a token of the list (those of the lead come first in it)
__device__ __forceinline__ uint64_t listed_mass(const SampleLds& s, const Row& r, int i)
{
    const uint64_t upto = s.upto[i];
    return r.lead >= 0 && upto <= r.lead_mass ? r.lead_mass_before + upto : r.mass_before - r.lead_mass + upto;
}

// next(sum of the weights up to a bin): the question that follows if the answer is the bin's last token
template <int DT, class Next>
__device__ __forceinline__ Answer locate(SampleLds& s, Row& r, const Question& ask, Next next)
{
    const int bin = r.whole ? 0 : first_bin(s, s.count, s.mass, ask, 0, 0);
    if (!r.whole && (bin < r.first || bin > r.last) && bin != r.lead) {
        // all bins up to this one if they hold few tokens (the next question is likely to fall among them), else this one
        const uint32_t upto = s.count[bin], own = upto - (bin > 0 ? s.count[bin - 1] : 0);
        r.first = upto <= kRanked ? 0 : bin;
        r.last = bin;
        r.before = r.first > 0 ? s.count[r.first - 1] : 0;
        r.mass_before = r.first > 0 ? s.mass[r.first - 1] : 0;
        r.lead = -1;
        r.lead_mass = 0;
        r.lead_count = 0;
        if (ask.kind < 2 && r.first > 0 && own <= kListed) {
            // the next question's bin in the same pass over the row, if both fit the list: a bin is a small part of the weights, so that it is known but for few draws
            const int lead = first_bin(s, s.count, s.mass, next(s.mass[bin]), 0, 0);
            const uint32_t count = s.count[lead] - (lead > 0 ? s.count[lead - 1] : 0);
            if (lead < bin && own + count <= kListed) {
                r.lead = lead;
                r.lead_before = lead > 0 ? s.count[lead - 1] : 0;
                r.lead_mass_before = lead > 0 ? s.mass[lead - 1] : 0;
                r.lead_count = count;
                r.lead_mass = s.mass[lead] - r.lead_mass_before;
            }
        }
        uint64_t lo = 0, hi = ~UINT64_C(0);           // of the order, within the bins
        if (own > kListed) {
            // a crowded bin: cut what its tokens span into bins, as often as it takes until one in question fits the list
            if (threadIdx.x == 0) { s.lo = ~UINT64_C(0); s.hi = 0; }
            __syncthreads();
            uint64_t l = ~UINT64_C(0), h = 0;
            for_row<DT>(r.logits, r.vocab, [&](float x, int t) {
                if (r.w.bin(r.w.z(x)) != bin || r.w.w(r.w.e(r.w.z(x))) == 0) return;
                const uint64_t o = order_of(x, t);
                l = min(l, o);
                h = max(h, o);
            });
            atomicMin((unsigned long long*)&s.lo, (unsigned long long)l);
            atomicMax((unsigned long long*)&s.hi, (unsigned long long)h);
            __syncthreads();
            lo = s.lo;
            hi = s.hi;
            for (uint32_t in = own; in > kListed;) {
                int shift = 0;
                while ((hi - lo) >> shift >= kBins) ++shift;
                for (int b = threadIdx.x; b < kBins; b += kSampleThreads) { s.count2[b] = 0; s.mass2[b] = 0; }
                __syncthreads();
                for_row<DT>(r.logits, r.vocab, [&](float x, int t) {
                    const float z = r.w.z(x);
                    const uint64_t o = order_of(x, t);
                    if (r.w.bin(z) != bin || o < lo || o > hi) return;
                    const uint32_t w = r.w.w(r.w.e(z));
                    if (w == 0) return;
                    atomicAdd(&s.count2[(o - lo) >> shift], 1u);
                    atomicAdd((unsigned long long*)&s.mass2[(o - lo) >> shift], (unsigned long long)w);
                });
                __syncthreads();
                scan_bins(s, s.count2, s.mass2);
                const int b = first_bin(s, s.count2, s.mass2, ask, r.before, r.mass_before);
                in = s.count2[b] - (b > 0 ? s.count2[b - 1] : 0);
                if (b > 0) {
                    r.before += s.count2[b - 1];
                    r.mass_before += s.mass2[b - 1];
                }
                lo += (uint64_t)b << shift;
                hi = min(hi, lo + ((UINT64_C(1) << shift) - 1));
                __syncthreads();
            }
            r.first = kBins;                           // the list is good for this question alone
            r.last = -1;
        }
        gather<DT>(s, r, r.first == kBins ? bin : r.first, bin, lo, hi);
    }
    if ((int)threadIdx.x < r.n && s.list[threadIdx.x] != kNone) {
        const int i = threadIdx.x;
        const bool lead = r.lead >= 0 && s.upto[i] <= r.lead_mass;
        const uint32_t rank = (lead ? r.lead_before : r.before - r.lead_count) + s.rank[i];
        const uint64_t mass = listed_mass(s, r, i), own = weight_of(r.w, s.list[i]);
        const bool earlier = s.rank[i] > 0 && ask.reached(rank, mass - own);
        if (!earlier && ask.reached(rank + 1, mass)) s.found = i;
    }
    __syncthreads();
    const int at = (int)s.found;
    const Answer a = {s.list[at], listed_mass(s, r, at)};
    __syncthreads();
    return a;
}

// the largest logit of a span, and whether one is NaN, to all threads
template <int DT>
__device__ __forceinline__ void span_top(TopLds& s, const void* logits, const Span& span, float* top_out, int* nan_out)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float top;
    int nan;
    Top<DT> best;
    for_eights<DT, 4>(logits, span, [&](const Eight<DT>& x, int) {
#pragma unroll
        for (int k = 0; k < (DT == NQ_F32 ? 2 : 1); ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) best.add(x.w[k][i]);
    }, [&](float, int t) {
        // (a 16-bit logit twice)
        best.add(DT == NQ_F32 ? ((const uint32_t*)logits)[t] : ((const uint16_t*)logits)[t] * 0x10001u);
    });
    best.get(&top, &nan);
    if (nan || top != top) top = -INFINITY;                  // (a thread without tokens has a NaN for its largest)
    for (int m = 1; m < 64; m <<= 1) {
        top = fmaxf(top, __shfl_xor(top, m));
        nan |= __shfl_xor(nan, m);
    }
    if (lane == 0) { s.top[wave] = top; s.nan[wave] = nan; }
    __syncthreads();
    for (int w = 0; w < kSampleThreads / 64; ++w) {
        top = fmaxf(top, s.top[w]);
        nan |= s.nan[w];
    }
    *top_out = top;
    *nan_out = nan;
}
__device__ __forceinline__ void parts_top(const SampleArgs& a, int row, float* top, int* nan)
{
    *top = -INFINITY;
    *nan = 0;
    for (int i = 0; i < a.slices; ++i) {
        *top = fmaxf(*top, a.parts[(int64_t)row * a.slices + i].top);
        *nan |= a.parts[(int64_t)row * a.slices + i].nan;
    }
}

// histogram of a span into the cleared bins of s; returns, to all threads, the weight of the tokens that min-p keeps
template <int DT>
__device__ __forceinline__ uint64_t span_histogram(SampleLds& s, const void* logits, const Span& span, const Weights& w, int k, float min_p)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint64_t kept = 0;
    // N logits side by side; those that weigh nothing are computed as well (no branch) and left out at the end
    auto add = [&](const auto& x, auto count) {
        constexpr int N = decltype(count)::value;
        float e[N];
        uint32_t weight[N];
        int bin[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float z = w.z(x[i]);
            e[i] = w.e(z);
            weight[i] = w.w(e[i]);
            bin[i] = w.bin(z);
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (weight[i] > 0) atomicAdd((unsigned long long*)&s.mass[bin[i]], (unsigned long long)weight[i]);
        if (k > 0) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (weight[i] > 0) atomicAdd(&s.count[bin[i]], 1u);
        }
        if (min_p > 0.f) {
#pragma unroll
            for (int i = 0; i < N; ++i) kept += e[i] >= min_p ? weight[i] : 0u;
        }
    };
    for_eights<DT, DT == NQ_F32 ? 2 : 4>(logits, span, [&](const Eight<DT>& x, int) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float four[4] = {x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]};
            add(four, std::integral_constant<int, 4>());
        }
    }, [&](float x, int) {
        const float one[1] = {x};
        add(one, std::integral_constant<int, 1>());
    });
    for (int m = 1; m < 64; m <<= 1) kept += __shfl_xor((unsigned long long)kept, m);
    if (lane == 0) s.part_mass[wave] = kept;
    __syncthreads();
    kept = 0;
    for (int v = 0; v < kSampleThreads / 64; ++v) kept += s.part_mass[v];
    __syncthreads();
    return kept;
}

// the same with counts alone, which is all that a few tokens asked for by top-k need: no exponentials
template <int DT>
__device__ __forceinline__ void span_counts(SampleLds& s, const void* logits, const Span& span, const Weights& w)
{
    auto add = [&](float x) {
        const float z = w.z(x);
        if (z > -22.2f) atomicAdd(&s.count[w.bin(z)], 1u);
    };
    for_eights<DT, 4>(logits, span, [&](const Eight<DT>& x, int) {
#pragma unroll
        for (int i = 0; i < 8; ++i) add(x[i]);
    }, [&](float x, int) { add(x); });
    __syncthreads();
}

// the first two passes as launches of their own: blockIdx.x a part, blockIdx.y a row
template <int DT>
__global__ __launch_bounds__(kSampleThreads, 8) void sample_top_kernel(SampleArgs a)
{
    __shared__ TopLds s;
    float top;
    int nan;
    span_top<DT>(s, (const char*)a.logits + blockIdx.y * a.row_stride * (DT == NQ_F32 ? 4 : 2), Span(a.vocab, blockIdx.x, a.slices), &top, &nan);
    SamplePart& part = a.parts[(int64_t)blockIdx.y * a.slices + blockIdx.x];
    if (threadIdx.x == 0) { part.top = top; part.nan = nan; }
}
template <int DT>
__global__ __launch_bounds__(kSampleThreads, 8) void sample_bins_kernel(SampleArgs a)
{
    extern __shared__ char lds[];
    SampleLds& s = *(SampleLds*)lds;
    const int row = blockIdx.y;
    float top;
    int nan;
    parts_top(a, row, &top, &nan);
    const float temperature = a.temperature ? a.temperature[row] : 1.f;
    if (nan || top == -INFINITY || !(temperature > 0.f)) return;
    for (int b = threadIdx.x; b < kBins; b += kSampleThreads) { s.count[b] = 0; s.mass[b] = 0; }
    __syncthreads();
    const int k = a.top_k ? a.top_k[row] : 0;
    const void* const logits = (const char*)a.logits + row * a.row_stride * (DT == NQ_F32 ? 4 : 2);
    const Span span(a.vocab, blockIdx.x, a.slices);
    const bool few = k > 0 && k <= kFew;
    uint64_t kept = 0;
    if (few) span_counts<DT>(s, logits, span, Weights(top, temperature));
    else kept = span_histogram<DT>(s, logits, span, Weights(top, temperature), k, a.min_p ? a.min_p[row] : 0.f);
    SamplePart& part = a.parts[(int64_t)row * a.slices + blockIdx.x];
    for (int b = threadIdx.x; b < kBins; b += kSampleThreads) {
        if (!few) part.mass[b] = s.mass[b];
        if (k > 0) part.count[b] = s.count[b];
    }
    if (threadIdx.x == 0) part.kept = kept;
}

template <int DT>
__global__ __launch_bounds__(kSampleThreads) void sample_kernel(SampleArgs a)
{
    extern __shared__ char lds[];
    SampleLds& s = *(SampleLds*)lds;
    const int row = blockIdx.x;
    Row r;
    r.logits = (const char*)a.logits + row * a.row_stride * (DT == NQ_F32 ? 4 : 2);
    r.vocab = a.vocab;
    r.first = kBins;
    r.last = -1;
    r.n = 0;
    r.whole = false;
    r.lead = -1;
    r.lead_mass = 0;
    r.lead_count = 0;

    float top;
    int nan;
    if (a.slices == 1) {
        for (int b = threadIdx.x; b < kBins; b += kSampleThreads) { s.count[b] = 0; s.mass[b] = 0; }       // (before the barrier in span_top)
        span_top<DT>(s.part_top, r.logits, Span(a.vocab, 0, 1), &top, &nan);
    } else {
        parts_top(a, row, &top, &nan);
    }
    const float temperature = a.temperature ? a.temperature[row] : 1.f;
    if (nan || top == -INFINITY || !(temperature > 0.f)) {
        const bool good = !nan && top != -INFINITY && temperature == 0.f;
        if (threadIdx.x == 0) s.found = INT32_MAX;
        __syncthreads();
        if (good) {                                          // the first token of the largest logit
            uint32_t at = INT32_MAX;
            for_row<DT>(r.logits, a.vocab, [&](float x, int t) {
                if (x == top) at = min(at, (uint32_t)t);
            });
            if (at != INT32_MAX) atomicMin(&s.found, at);
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            a.tokens[row] = good ? (int)s.found : -1;
            if (a.logprobs) a.logprobs[row] = good ? 0.f : NAN;
        }
        return;
    }
    r.w = Weights(top, temperature);
    const int k = a.top_k ? a.top_k[row] : 0;
    const float min_p = a.min_p ? a.min_p[row] : 0.f;
    const Span all(a.vocab, 0, 1);
    const bool few = k > 0 && k <= kFew;
    uint64_t kept = 0;
    if (a.slices == 1) {
        if (few) span_counts<DT>(s, r.logits, all, r.w);
        else kept = span_histogram<DT>(s, r.logits, all, r.w, k, min_p);
    } else {
        const SamplePart* const parts = a.parts + (int64_t)row * a.slices;
        typedef uint64_t v2u64 __attribute__((ext_vector_type(2)));
        typedef uint32_t v2u32 __attribute__((ext_vector_type(2)));
        const int b = 2 * threadIdx.x;
        v2u64 m = {0, 0}, each[kMostSlices];
        v2u32 c = {0, 0};
        if (!few) {
#pragma unroll
            for (int i = 0; i < kMostSlices; ++i) each[i] = *(const v2u64*)&parts[min(i, a.slices - 1)].mass[b];
#pragma unroll
            for (int i = 0; i < kMostSlices; ++i)
                if (i < a.slices) m += each[i];
            for (int i = 0; i < a.slices; ++i) kept += parts[i].kept;
        }
        if (k > 0)
            for (int i = 0; i < a.slices; ++i) c += *(const v2u32*)&parts[i].count[b];
        s.mass[b] = m.x;
        s.mass[b + 1] = m.y;
        s.count[b] = c.x;
        s.count[b + 1] = c.y;
        __syncthreads();
    }
    if (few) {
        // the tokens up to the k-th one's bin, if they fit the list; else the row's whole histogram after all
        scan_bins(s, s.count, s.mass);
        const int last = (uint32_t)k < s.count[kBins - 1] ? first_bin(s, s.count, s.mass, Question{0, (uint32_t)k, 0.0, 0}, 0, 0) : kBins - 1;
        if (s.count[last] <= kListed) {
            r.whole = true;
            r.before = 0;
            r.mass_before = 0;
            gather<DT>(s, r, 0, last, 0, ~UINT64_C(0));
            if (threadIdx.x == 0) { s.lo = 0; s.hi = 0; s.n = 0; }
            __syncthreads();
            // how many, all their weights, those that min-p keeps: over a wave, then over the waves that have some
            if (((int)threadIdx.x & ~63) < r.n) {
                const bool is = (int)threadIdx.x < r.n && s.list[threadIdx.x] != kNone;
                const float e = is ? r.w.e(r.w.z(logit_of(s.list[threadIdx.x]))) : 0.f;
                const uint64_t weight = r.w.w(e), all = wave_scan(weight), these = wave_scan(e >= min_p ? weight : UINT64_C(0));
                const uint64_t some = __ballot(is);
                if ((threadIdx.x & 63) == 63) {
                    atomicAdd(&s.n, (uint32_t)__builtin_popcountll(some));
                    atomicAdd((unsigned long long*)&s.lo, (unsigned long long)all);
                    atomicAdd((unsigned long long*)&s.hi, (unsigned long long)these);
                }
            }
            __syncthreads();
            kept = s.hi;
        } else {
            __syncthreads();
            for (int b = threadIdx.x; b < kBins; b += kSampleThreads) { s.count[b] = 0; s.mass[b] = 0; }
            __syncthreads();
            kept = span_histogram<DT>(s, r.logits, all, r.w, k, min_p);
        }
    }
    if (k <= 0) {
        for (int b = threadIdx.x; b < kBins; b += kSampleThreads) s.count[b] = s.mass[b] == 0 ? 0u : (uint32_t)fminf((float)s.mass[b] / r.w.least(b) * 1.0001f + 1.f, (float)NQ_MAX_VOCAB);
        __syncthreads();
    }
    if (!r.whole) scan_bins(s, s.count, s.mass);

    // each limit keeps a prefix of the order: the shortest counts
    const uint64_t one = UINT64_C(1) << 31;                 // the first token's weight
    uint64_t total = r.whole ? s.lo : s.mass[kBins - 1];
    const uint32_t weighty = r.whole ? s.n : s.count[kBins - 1];
    const float top_p = a.top_p ? a.top_p[row] : 1.f;
    Answer drawn = {0, 0};
    auto left = [&](uint64_t among) { return min_p > 0.f ? min(among, max(kept, one)) : among; };
    // where the draw falls among the tokens that the limits leave
    auto draw = [&](uint64_t among) {
        const float u = a.uniform[row];
        const double place = u > 0.f ? (double)u * (double)among : 0.0;
        return Question{2, 0, 0.0, place >= (double)among ? among - 1 : min((uint64_t)place, among - 1)};
    };
    for (int kind = 0; kind < 3; ++kind) {
        Question ask = {kind, (uint32_t)k, (double)top_p * (double)total, 0};
        if (kind == 0 && (k <= 0 || (uint32_t)k >= weighty)) continue;
        if (kind == 1 && !(top_p < 1.f)) continue;
        if (kind == 2) {
            total = left(total);
            ask = draw(total);
        }
        drawn = locate<DT>(s, r, ask, [&](uint64_t among) { return kind == 0 && top_p < 1.f ? Question{1, 0, (double)top_p * (double)among, 0} : draw(left(among)); });
        if (kind < 2) total = drawn.mass;
    }
    if (threadIdx.x == 0) {
        a.tokens[row] = (int32_t)(uint32_t)drawn.order;
        if (a.logprobs) a.logprobs[row] = r.w.z(logit_of(drawn.order)) - logf((float)total * 0x1p-31f);
    }
}

// Parts of a row: three workgroups to a CU in all, at least 16384 tokens each, at most 8 (whose histograms the last launch adds up)
static int sample_slices(int n_rows, int64_t vocab)
{
    const int64_t want = (3 * device_cu_count() + std::max(1, n_rows) - 1) / std::max(1, n_rows);
    return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(want, vocab / 16384), kMostSlices));
}

static size_t part_bytes(int n_rows, int64_t vocab)
{
    const int slices = sample_slices(n_rows, vocab);
    return slices > 1 ? (size_t)n_rows * slices * sizeof(SamplePart) : 0;
}
// Room for so many rows and for fewer, so that one buffer serves whatever batch a program has next: n rows have at most ceil(3 CUs / n) parts each, fewer than 3 CUs + n in all
// (191 rows of 131071 tokens 955, 192 rows 768).
static size_t most_part_bytes(int n_rows, int64_t vocab)
{
    const int64_t fill = 3 * device_cu_count(), each = std::min<int64_t>(vocab / 16384, kMostSlices), rows = std::min<int64_t>(n_rows, fill - 1);
    return each > 1 && rows > 0 ? (size_t)std::min(each * rows, fill + rows - 1) * sizeof(SamplePart) : 0;
}

}  // namespace nq

using namespace nq;

extern "C" int nq_sample_workspace_bytes(int n_rows, int64_t vocab, size_t* bytes)
{
    const char* const who = "nq_sample_workspace_bytes";
    if (!bytes) return refuse(NQ_E_NULL, who, "bytes is NULL");
    if (n_rows < 0) return refuse(NQ_E_INVALID_ARG, who, "n_rows must be >= 0");
    if (vocab < 1 || vocab > NQ_MAX_VOCAB) return refuse(NQ_E_SHAPE, who, "vocab must be 1 to 2^20");
    *bytes = most_part_bytes(n_rows, vocab);
    return NQ_OK;
}

extern "C" int nq_sample(const void* logits, int dtype, int n_rows, int64_t vocab, int64_t row_stride, const float* temperature, const int32_t* top_k, const float* top_p,
                         const float* min_p, const float* uniform, int32_t* tokens, float* logprobs, void* workspace, size_t workspace_bytes, void* stream)
{
    const char* const who = "nq_sample";
    size_t most = 0;
    if (const int rc = nq_sample_workspace_bytes(n_rows, vocab, &most)) return rc;
    const size_t need = part_bytes(n_rows, vocab);
    if (!is_float_type(dtype)) return refuse(NQ_E_INVALID_ARG, who, "dtype must be NQ_F32, NQ_F16 or NQ_BF16");
    if (n_rows == 0) return NQ_OK;
    if (!logits || !uniform || !tokens) return refuse(NQ_E_NULL, who, "logits, uniform or tokens is NULL");
    if (off_align(logits, type_bytes(dtype))) return refuse(NQ_E_ALIGN, who, "logits must have the alignment of its elements");
    if (off_align(temperature, 4) || off_align(top_k, 4) || off_align(top_p, 4) || off_align(min_p, 4) || off_align(uniform, 4) || off_align(tokens, 4) || off_align(logprobs, 4))
        return refuse(NQ_E_ALIGN, who, "arrays must be 4-byte aligned");
    if (row_stride < vocab) return refuse(NQ_E_SHAPE, who, "row_stride below vocab");
    if (row_stride > (INT64_C(1) << 31)) return refuse(NQ_E_SHAPE, who, "row_stride beyond 2^31");
    if (need > 0 && !workspace) return refuse(NQ_E_NULL, who, "workspace is NULL");
    if (off_align(workspace, 16)) return refuse(NQ_E_ALIGN, who, "workspace must be 16-byte aligned");
    if (workspace_bytes < need) return refuse(NQ_E_INVALID_ARG, who, "workspace too small");
    const SampleArgs a = {logits, temperature, top_p, min_p, uniform, top_k, tokens, logprobs, row_stride, (int)vocab, sample_slices(n_rows, vocab), (SamplePart*)workspace};
    auto launch = [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const dim3 block(kSampleThreads);
        if (a.slices > 1) {                                              // (fewer rows than three to a CU)
            NQ_ALLOW_LDS((sample_bins_kernel<DT>), sizeof(SampleLds));
            const dim3 grid(a.slices, n_rows);
            hipLaunchKernelGGL((sample_top_kernel<DT>), grid, block, 0, (hipStream_t)stream, a);
            if (const int rc = launched(who)) return rc;
            hipLaunchKernelGGL((sample_bins_kernel<DT>), grid, block, sizeof(SampleLds), (hipStream_t)stream, a);
            if (const int rc = launched(who)) return rc;
        }
        NQ_ALLOW_LDS((sample_kernel<DT>), sizeof(SampleLds));
        hipLaunchKernelGGL((sample_kernel<DT>), dim3(n_rows), block, sizeof(SampleLds), (hipStream_t)stream, a);
        return launched(who);
    };
    if (dtype == NQ_F32) return launch(std::integral_constant<int, NQ_F32>());
    if (dtype == NQ_F16) return launch(std::integral_constant<int, NQ_F16>());
    return launch(std::integral_constant<int, NQ_BF16>());
}
