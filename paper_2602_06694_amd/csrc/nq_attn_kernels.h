// Attention of new tokens -- one, a tree of drafted ones, a chunk of a prompt -- over a paged cache (nq_decoder.h): one pass over the keys with running maxima and sums,
// out = sum 2^(s - top) v / sum 2^(s - top), split over the keys where there are few rows.
//
// Rows.  The query heads of a key head read the same keys, so the rows of a sequence and key head are (token, head of the group), and a tile of 16, 64 or 128 of them goes
// through the keys together: a single token of a 70B-shaped model is eight rows, eight drafted tokens 64.
//
// Operands.  Scores are computed transposed, S^T = K Q^T (16 keys x 16 rows a matrix instruction), and so is the result, O^T = V^T P^T.  Lane (g, n), g = lane / 16,
// n = lane % 16, then holds for its row n the scores of keys 4g..4g+3 of each 16: as the operand P^T of the second product a lane has to hold eight keys of one row, and since
// the order of the keys in a sum is free those are taken to be 4g..4g+3 of two tiles of 16: the lane's own scores, exponentiated.  Row maxima need two lane exchanges, and
// only where one grows by more than 2^8; rescaling needs none (a lane has one row).
// attn_split_kernel, up to 16 rows: nothing passes through LDS but the join of the four waves at the end.  K is loaded as the operand it is (16 bytes: eight elements of a
// key), V as whole rows too: lane (g, n) loads elements 8n..8n+7 of the same eight keys 4g.., 16+4g.., and one byte permute per two elements turns the 8 x 8 block into eight
// operands, the c-th of elements 8n + c.  The results of a lane are then eight consecutive elements.
// attn_wide_kernel, more rows: the waves share the keys through LDS.
//
// Work.  Every workgroup finds its own item -- a tile of rows and a run of 64-key blocks -- from the lengths in device memory (no host copy, so that a captured graph serves
// any lengths); run_length chooses how tiles are cut into runs for whatever mixture of lengths there is.  Tiles with one run are finished by their workgroup; the others leave
// unnormalised sums and their maxima, which attn_join_kernel adds up.
//
// Bound by the cache's bytes up to some 64 rows (4 to 5.9 TB/s of it at 64 and 8 heads of 128 from 150 MB on, one to 256 sequences, 6.8 is what a plain read reaches), then by
// the matrix and the vector unit together (2048 tokens behind 4095: 323 to 345 us on several cards, 1.0 PFLOP/s; 1.36 is what a large matrix
// product reaches).
#pragma once

#include <algorithm>
#include <cmath>

#include "nq_decoder_internal.h"

namespace nq {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef unsigned int v2u __attribute__((ext_vector_type(2)));
typedef const __attribute__((address_space(1))) v2u* gptr_v2u;
typedef const __attribute__((address_space(4))) int32_t* sptr_i32;      // read through the scalar cache: the same for the whole wave

struct AttnArgs {
    KvDesc kv;
    const void* q;
    const int32_t *begin, *ctx, *table;
    const uint32_t* tree;
    void* out;
    float *lse, *part_o, *part_ml;
    int64_t q_stride, out_stride, table_stride;
    int tree_words, n_seqs, n_tokens, q_heads, group, out_dtype;
    float scale, cap;
    int slots;               // workgroups of a key head that run at a time
    int items;               // most items of a key head (the grid)
    int rows;                // of a tile; 16: attn_split_kernel, 64 and 128: attn_wide_kernel
    bool few;                // rows of a sequence, on average up to 64: bound by bytes
};

// A call, checked, over a cache of this type
int attend_f16(const AttnArgs& a, const char* who, hipStream_t s);
int attend_bf16(const AttnArgs& a, const char* who, hipStream_t s);

constexpr int kBlock = 64;           // keys of a block, the unit in which runs are dealt out
constexpr int kWaves = 4;            // of a workgroup
constexpr int kMinRun = 2;           // blocks of the shortest run: a step of 32 keys to every wave of attn_split_kernel

// over the wave, to all lanes
__device__ __forceinline__ int64_t wave_sum(int64_t v)
{
    const uint64_t all = wave_scan((uint64_t)v);
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(all >> 32), 63) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)all, 63));
}

// A sequence as the device finds it, cut to the call's buffers
struct Seq {
    int first, n, ctx, keys;         // first new token, new tokens, cached tokens, keys in all (at least the cached ones)
};
__device__ __forceinline__ Seq sequence(const AttnArgs& a, int s)
{
    Seq q = {0, 0, 0, 0};
    if (s < a.n_seqs) {
        q.first = min(max(a.begin[s], 0), a.n_tokens);
        q.n = min(max(a.begin[s + 1], q.first), a.n_tokens) - q.first;
        // both within the table: every key below ctx is one
        const int64_t most = min(a.table_stride << a.kv.page_shift, (int64_t)INT32_MAX - 4096);
        q.ctx = (int)min((int64_t)max(a.ctx[s], 0), most);
        q.keys = (int)min((int64_t)q.ctx + q.n, most);
    }
    return q;
}

// how a sequence is cut: tiles of rows, blocks of keys; with runs of at most `run` blocks
__device__ __forceinline__ int tiles_of(const Seq& q, const AttnArgs& a, int rows) { return (q.n * a.group + rows - 1) / rows; }
__device__ __forceinline__ int blocks_of(const Seq& q) { return q.n > 0 ? (q.keys + kBlock - 1) / kBlock : 0; }
__device__ __forceinline__ int runs_of(int blocks, int run) { return (blocks + run - 1) / run; }
// items of a sequence, or one more than the call has room for: where new_begin does not rise, tiles may be more than rows, and any number of items is asked for
__device__ __forceinline__ int items_of(int tiles, int runs, const AttnArgs& a) { return (int)min((int64_t)tiles * runs, (int64_t)a.items + 1); }

// Blocks of a run, or kNoRuns.  The chip holds a.slots workgroups of a key head at a time; each would have `share` blocks if they could be dealt out evenly.  Of three
// ways the one that is expected to end first, in blocks:
// - tiles stay whole: the rounds that they take, or the longest of them;
// - runs that all fit the chip at once: each tile in as many as there are places to a tile, or runs of one length (the last of a tile comes on top of those of full length,
//   hence the tiles taken off);
// - runs of half a share, more than fit at once, which places take as they become free: a quarter of a share is left at the end.
// A run costs what it leaves for the joining, 4 blocks' time where tiles have 64 rows and more and 2 where they have 16, the joining itself 3.  Of 15 calls of 12 to 330 us, each
// timed with all three ways, the one chosen is within 6 % of the best in 13; 512 tokens behind 1023 take 59 us where whole tiles take 44, 16 sequences of 512 17 and 14.  front: the
// lane's sequence of the first 64.
constexpr int kNoRuns = 1 << 25;
__device__ __forceinline__ int run_length(const AttnArgs& a, int rows, int lane, const Seq& front)
{
    int64_t work = (int64_t)tiles_of(front, a, rows) * blocks_of(front), tiles = tiles_of(front, a, rows);
    int longest = blocks_of(front);
    for (int s0 = 64; s0 < a.n_seqs; s0 += 64) {
        const Seq q = sequence(a, s0 + lane);
        work += (int64_t)tiles_of(q, a, rows) * blocks_of(q);
        tiles += tiles_of(q, a, rows);
        longest = max(longest, blocks_of(q));
    }
    work = wave_sum(work);
    tiles = wave_sum(tiles);
    longest = (int)wave_max((uint32_t)longest);
    // quotients, rounded up by less than a block and 2^-22 of it: longer runs are fewer items (exact ones of 64 bits take a microsecond)
    auto over = [](float x, float y) { return (int)min(x * (1.0000002f / y), (float)kNoRuns) + 1; };
    const float blocks = (float)work, slots = (float)a.slots, cost = rows == 16 ? 2.f : 4.f;
    const uint32_t n = max(1u, (uint32_t)tiles), rounds = (n + a.slots - 1) / a.slots, places = (uint32_t)a.slots / n;
    const float whole = max((float)longest, blocks * (float)rounds / (float)n);
    const int fit = places == 0 ? kNoRuns : min((longest + (int)places - 1) / (int)places, places == 1 ? kNoRuns : over(blocks, slots - (float)n));
    const int half = over(blocks, 2.f * slots);
    const float at_once = (float)fit + cost + 3.f, in_turn = 2.5f * (float)half + 2.f * cost + 3.f;
    if (whole <= min(at_once, in_turn)) return kNoRuns;
    return max(kMinRun, at_once <= in_turn ? fit : half);
}

struct Item {
    Seq q;
    int seq, tile, run, runs, per;   // run of `runs` runs of `per` blocks
    int index;                       // of the tile's first run among the key head's items
};

// The item with this number, found by the wave's lanes from 64 sequences at a time; false: there is none
__device__ __forceinline__ bool find_item(const AttnArgs& a, int rows, int number, int lane, Item* it)
{
    const Seq front = sequence(a, lane);
    const int run = run_length(a, rows, lane, front);
    int before = 0;
    for (int s0 = 0; s0 < a.n_seqs; s0 += 64) {
        const Seq q = s0 == 0 ? front : sequence(a, s0 + lane);
        const int tiles = tiles_of(q, a, rows), blocks = blocks_of(q), runs = runs_of(blocks, run), items = items_of(tiles, runs, a);
        const int upto = before + (int)wave_scan((uint32_t)items);
        const uint64_t past = __ballot(upto > number);
        if (past) {
            const int at = __builtin_ctzll(past);
            auto pick = [&](int v) { return __builtin_amdgcn_readlane(v, at); };
            it->q = Seq{pick(q.first), pick(q.n), pick(q.ctx), pick(q.keys)};
            it->seq = s0 + at;
            it->runs = pick(runs);
            const int first = pick(upto - items), mine = number - first;
            // what several runs leave has to have its place, whichever of them this is (only a new_begin that does not rise has more)
            if (it->runs > 1 && first + pick(items) > a.items) return false;
            // the tiles of a run next to one another: they read the same keys; the last first: where rows see what precedes them those have most to do, and a place
            // that is free again early then gets less than one that is free late
            const int n_tiles = pick(tiles);
            it->run = mine / n_tiles;
            it->tile = n_tiles - 1 - (mine - it->run * n_tiles);
            it->per = (pick(blocks) + it->runs - 1) / it->runs;
            it->index = first + it->tile;
            return true;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// keys up to a new token and its own (a length near 2^31 and a token are more than 32 bits hold)
__device__ __forceinline__ int keys_upto(const Seq& q, int token) { return (int)min((int64_t)q.keys, (int64_t)q.ctx + token + 1); }
// keys that some row of a tile may see: all, or up to the tile's last token where the rows see what precedes them
__device__ __forceinline__ int tile_keys(const AttnArgs& a, const Seq& q, int tile, int rows)
{
    if (a.tree) return q.keys;
    return keys_upto(q, (min((tile + 1) * rows, q.n * a.group) - 1) / a.group);
}

template <int DT>
__device__ __forceinline__ v4f mfma16(v4u x, v4u y, v4f c)
{
    if constexpr (DT == NQ_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
}

// the larger of two; NaN is left out (fmaxf would have operands that come from matrix instructions made quiet first; assembly has no place here, as the compiler does not wait
// for matrix instructions before it)
__device__ __forceinline__ float max2(float a, float b) { return __builtin_amdgcn_fmed3f(a, b, INFINITY); }
template <int DT>
__device__ __forceinline__ float widen(uint32_t w, int high)
{
    const uint16_t h = (uint16_t)(high ? w >> 16 : w);
    return DT == NQ_F16 ? half_bits_to_float(h) : bf16_bits_to_float(h);
}
template <int DT>
__device__ __forceinline__ bool half_not_finite(uint32_t h)
{
    constexpr uint32_t e = DT == NQ_F16 ? 0x7c00u : 0x7f80u;
    return (h & e) == e;
}

template <int DT>
constexpr uint32_t kOne = DT == NQ_F16 ? 0x3c00u : 0x3f80u;
// whether 16 bits are NaN (kind 0), infinity (1) or -infinity (2)
template <int DT>
__device__ __forceinline__ bool of_kind(uint32_t h, int kind)
{
    constexpr uint32_t inf = DT == NQ_F16 ? 0x7c00u : 0x7f80u;
    return kind == 0 ? (h & 0x7fffu) > inf : h == (kind == 1 ? inf : inf | 0x8000u);
}

// Values that are not finite must not meet the zero weights of rows that do not see them: they are taken out of the operand, and the rows that do see one are
// found by products of ones with ones.  ones_of(r): operand with 1 where the rows of tile r see a key; sums(r): their accumulators.
template <int DT, int R, class Ones, class Sums>
__device__ __forceinline__ void mend_values(v4u& value, Ones ones_of, Sums sums)
{
#pragma clang loop unroll(disable)
    for (int kind = 0; kind < 3; ++kind) {              // NaN, infinity, -infinity
        v4u ones;
#pragma unroll
        for (int w = 0; w < 4; ++w) ones[w] = (of_kind<DT>(value[w] & 0xffffu, kind) ? kOne<DT> : 0u) | (of_kind<DT>(value[w] >> 16, kind) ? kOne<DT> << 16 : 0u);
        const float special = kind == 0 ? NAN : kind == 1 ? INFINITY : -INFINITY;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const v4f count = mfma16<DT>(ones, ones_of(r), v4f{0.f, 0.f, 0.f, 0.f});
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (count[i] > 0.f) sums(r)[i] += special;
        }
    }
#pragma unroll
    for (int w = 0; w < 4; ++w) value[w] &= (half_not_finite<DT>(value[w]) ? 0u : 0xffffu) | (half_not_finite<DT>(value[w] >> 16) ? 0u : 0xffff0000u);
}

// Which of the keys from + 16t + i (bit 4t + i, i < 4) a new token sees; token -1: no row, none
template <int TILES>
__device__ __forceinline__ uint32_t seen_keys(const AttnArgs& a, const Seq& q, int token, int from)
{
    uint32_t seen = 0;
    if (token < 0) return seen;
    const uint32_t* const row = a.tree + (int64_t)(q.first + token) * a.tree_words;
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int key = from + 16 * t + i, late = key - q.ctx;
            bool yes = key < q.keys;
            if (yes && late >= 0) {
                if (a.tree) yes = (late >> 5) < a.tree_words && (row[late >> 5] >> (late & 31) & 1u);
                else yes = late <= token;
            }
            seen |= (yes ? 1u : 0u) << (4 * t + i);
        }
    return seen;
}
// eight such bits as an operand with ones
template <int DT>
__device__ __forceinline__ v4u seen_ones(uint32_t seen)
{
    v4u x;
#pragma unroll
    for (int w = 0; w < 4; ++w) x[w] = (seen >> (2 * w) & 1u ? kOne<DT> : 0u) | (seen >> (2 * w + 1) & 1u ? kOne<DT> << 16 : 0u);
    return x;
}

// four neighbouring results; the element's alignment is all that is known
__device__ __forceinline__ void store4(void* out, int dtype, int64_t at, v4f x)
{
    typedef v2u v2u_any __attribute__((aligned(2)));
    if (dtype == NQ_F32) *(__attribute__((address_space(1))) v4f_any*)((float*)out + at) = x;
    else if (dtype == NQ_F16) *(__attribute__((address_space(1))) v2u_any*)((uint16_t*)out + at) = v2u{round2<NQ_F16>(x[0], x[1]), round2<NQ_F16>(x[2], x[3])};
    else *(__attribute__((address_space(1))) v2u_any*)((uint16_t*)out + at) = v2u{round2<NQ_BF16>(x[0], x[1]), round2<NQ_BF16>(x[2], x[3])};
}

// over the four lanes that share a row (lane bits 4 and 5)
template <class Op>
__device__ __forceinline__ float over_rows(float v, Op op)
{
    typedef unsigned int v2u_t __attribute__((ext_vector_type(2)));
    uint32_t x = __builtin_bit_cast(uint32_t, v);
    const v2u_t a = __builtin_amdgcn_permlane16_swap(x, x, false, false);       // each lane's own 16, and those beside them
    const uint32_t a0 = a.x, a1 = a.y;
    x = __builtin_bit_cast(uint32_t, op(__builtin_bit_cast(float, a0), __builtin_bit_cast(float, a1)));
    const v2u_t b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    const uint32_t b0 = b.x, b1 = b.y;
    return op(__builtin_bit_cast(float, b0), __builtin_bit_cast(float, b1));
}
__device__ __forceinline__ float row_max(float v) { return over_rows(v, [](float x, float y) { return fmaxf(x, y); }); }
__device__ __forceinline__ float row_sum(float v) { return over_rows(v, [](float x, float y) { return x + y; }); }

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLazy = 8.f;         // a row's maximum is raised only by more than this (in powers of two): until then weights are up to 2^8
// What a row's `top` is below its maximum: weights of fp16 are up to 2^15 then, so that the parts of those that are small next to the largest are no subnormal numbers
template <int DT>
constexpr float kLift = DT == NQ_F16 ? 7.f : 0.f;

// Scores in powers of two: log2(e) times the products, scaled, and capped by cap tanh(x / cap).  The capped ones' error counts in units of cap, so that small ones have to be
// exact relative to themselves: below one half the continued fraction x / (1 + x^2 / (3 + x^2 / (5 + x^2 / 7))) (its error is 4 10^-8 at one half), else
// 1 - 2 / (1 + e^2x).  Where the wave's are all small that is no more than one of the two (an exponential less).
__device__ __forceinline__ v4f scores(v4f dot, float scale, float cap)
{
    if (!(cap > 0.f)) return dot * (scale * kLog2e);
    const v4f x = dot * (scale / cap);
    const bool large = !(fmaxf(fmaxf(fabsf(x[0]), fabsf(x[1])), fmaxf(fabsf(x[2]), fabsf(x[3]))) < 0.5f);
    v4f y;
    auto below = [](float x) {
        const float x2 = x * x;
        return x * fmaf(x2, 10.f, 105.f) * __builtin_amdgcn_rcpf(fmaf(x2, x2 + 45.f, 105.f));
    };
    if (__ballot(large) == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = below(x[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float above = 1.f - 2.f * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x[i] * (2.f * kLog2e)));
            y[i] = fabsf(x[i]) < 0.5f ? below(x[i]) : above;
        }
    }
    return y * (cap * kLog2e);
}

// elements of one key of a step as operands: K two tiles of 16 keys, V eight keys of a lane
template <int DP>
struct KeyStep {
    static constexpr int kParts = DP / 32;              // of a key, 32 elements a matrix instruction
    static constexpr int kHalves = DP > 128 ? 2 : 1;    // of a value, 128 elements (64: four a lane)
    v4u k[2][kParts];
    v4u v[8][kHalves];
};

// ---------------------------------------------------------------------------------------------
// Up to 16 rows: the waves of a workgroup share them and take every fourth step of 32 keys, straight from memory to the operands' registers, the next step's loads
// under way while one is worked on; their sums meet in LDS at the end.  Bound by the bytes of the cache: 32 ragged sequences of up to 8191 tokens in 122 us
// under a kernel trace, 623 MB read for 621 of keys and values.
// DP: head_dim rounded up to 64, 128 or 256; PARTS: parts in which the weights are rounded
// ---------------------------------------------------------------------------------------------
constexpr int split_lds(int dp) { return kWaves * (16 * (dp + 4) + 32) * (int)sizeof(float); }

template <int DT, int DP, int PARTS>
__global__ __launch_bounds__(kWaves * 64, DP == 256 ? 1 : 2) void attn_split_kernel(AttnArgs a)
{
    constexpr int kRows = 16;
    constexpr int kParts = DP / 32, kHalves = KeyStep<DP>::kHalves, kEach = DP == 64 ? 4 : 8;        // kEach: elements of a value that a lane holds, per half
    constexpr int kRowFloats = DP + 4;
    constexpr bool kAhead = DP <= 128;                               // registers for the next step
    extern __shared__ float lds[];
    float* const lds_o = lds;                                       // [waves][16][kRowFloats]
    float* const lds_ml = lds + kWaves * 16 * kRowFloats;           // [waves][16][2]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = lane >> 4, n = lane & 15;
    const int head = blockIdx.x % a.kv.heads, number = blockIdx.x / a.kv.heads;
    Item it;
    if (!find_item(a, kRows, number, lane, &it)) return;
    const int keys = tile_keys(a, it.q, it.tile, kRows);
    const int step0 = it.run * it.per * 2, step1 = min((it.run + 1) * it.per * 2, (keys + 31) / 32);

    // this lane's row: its token and its operands
    const int my_row = it.tile * kRows + n;
    const bool real = my_row < it.q.n * a.group;
    const int token = real ? my_row / a.group : -1;
    v4u q[kParts];
    {
        const int h = head * a.group + (real ? my_row - token * a.group : 0);
        const uint16_t* const at = (const uint16_t*)a.q + (it.q.first + max(token, 0)) * a.q_stride + (int64_t)h * a.kv.head_dim;
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
            const int d = 32 * p + 8 * g;
            q[p] = v4u{0, 0, 0, 0};
            if (real && d < a.kv.head_dim) q[p] = *(gptr_v4u_any)(at + d);
        }
    }
    v4f o[kHalves][kEach];
    float top, sum;                                                 // of the row so far (sum: of this lane's keys), in powers of two

    const sptr_i32 pages = (sptr_i32)(a.table + it.seq * a.table_stride);
    const int page_mask = (1 << a.kv.page_shift) - 1;
    // where 16 keys begin (a page holds whole sixteens); keys past the end are read where the last sixteen is
    auto place = [&](int key) -> int64_t {
        key = min(key, (keys - 1) & ~15);
        const int64_t page = min((uint32_t)pages[key >> a.kv.page_shift], (uint32_t)(a.kv.n_pages - 1));
        return page * a.kv.page_stride + (int64_t)(key & page_mask) * a.kv.slot_stride + head * a.kv.head_stride;
    };
    const uint32_t slot_bytes = (uint32_t)a.kv.slot_stride * 2;
    const int last_d = a.kv.head_dim - 8;                            // elements past head_dim: others are read, for a query's zeros or a result that is not stored
    auto load = [&](int step, KeyStep<DP>& s) {
        const int64_t at[2] = {place(step * 32), place(step * 32 + 16)};
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const char* const k = (const char*)(a.kv.k + at[t]);
#pragma unroll
            for (int p = 0; p < kParts; ++p) s.k[t][p] = *(gptr_v4u)(k + (n * slot_bytes + 2 * min(32 * p + 8 * g, last_d)));
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const char* const v = (const char*)(a.kv.v + at[t]);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int h = 0; h < kHalves; ++h) {
                    if (DP == 64) {
                        const v2u two = *(gptr_v2u)(v + ((4 * g + i) * slot_bytes + 2 * min(4 * n, a.kv.head_dim - 4)));
                        s.v[4 * t + i][h] = v4u{two.x, two.y, 0, 0};
                    } else {
                        s.v[4 * t + i][h] = *(gptr_v4u)(v + ((4 * g + i) * slot_bytes + 2 * min(128 * h + 8 * n, last_d)));
                    }
                }
        }
    };
    // element of the results that accumulator (h, c, i) of this lane is
    auto element = [&](int h, int c, int i) { return 128 * h + kEach * (4 * g + i) + c; };

    // masked: some key of the step is not seen by some row
    auto compute = [&](int step, KeyStep<DP>& s, auto masked_t) {
        constexpr bool masked = decltype(masked_t)::value;
        const int key0 = step * 32;
        bool mend = false;
        if (masked) {
            // values past the sequence's end are memory of any content
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool past = key0 + (j < 4 ? 4 * g + j : 12 + 4 * g + j) >= it.q.keys;
#pragma unroll
                for (int h = 0; h < kHalves; ++h)
#pragma unroll
                    for (int w = 0; w < (DP == 64 ? 2 : 4); ++w) {
                        if (past) s.v[j][h][w] = 0u;
                        mend |= half_not_finite<DT>(s.v[j][h][w]) || half_not_finite<DT>(s.v[j][h][w] >> 16);
                    }
            }
            mend = __ballot(mend) != 0;
        }
        v4f dot[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            dot[t] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int p = 0; p < kParts; ++p) dot[t] = mfma16<DT>(s.k[t][p], q[p], dot[t]);
        }
        uint32_t seen = 0;                                           // bit j: key j of the lane's eight
        if (masked) seen = seen_keys<2>(a, it.q, token, key0 + 4 * g);
        float x[8];
#pragma unroll
        for (int t = 0; t < 2; ++t) dot[t] = scores(dot[t], a.scale, a.cap);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[j] = dot[j >> 2][j & 3];
            if (masked && !(seen >> j & 1u)) x[j] = -INFINITY;
        }
        float most = x[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) most = fmaxf(most, x[j]);
        most -= kLift<DT>;
        if (__ballot(most > top + kLazy)) {
            most = fmaxf(row_max(most), top);
            const float factor = most == top ? 1.f : __builtin_amdgcn_exp2f(top - most);
            top = most;
            sum *= factor;
#pragma unroll
            for (int h = 0; h < kHalves; ++h)
#pragma unroll
                for (int c = 0; c < kEach; ++c) o[h][c] *= factor;
        }
        const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[j] = __builtin_amdgcn_exp2f(x[j] - base);
            sum += x[j];
        }
        v4u weight[PARTS];
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int part = 0; part < PARTS; ++part) {
                weight[part][w] = round2<DT>(x[2 * w], x[2 * w + 1]);
                x[2 * w] -= widen<DT>(weight[part][w], 0);
                x[2 * w + 1] -= widen<DT>(weight[part][w], 1);
            }
#pragma unroll
        for (int h = 0; h < kHalves; ++h)
#pragma unroll
            for (int c = 0; c < kEach; ++c) {
                v4u value;
#pragma unroll
                for (int w = 0; w < 4; ++w) value[w] = __builtin_amdgcn_perm(s.v[2 * w + 1][h][c >> 1], s.v[2 * w][h][c >> 1], (c & 1) ? 0x07060302u : 0x05040100u);
                if (masked && mend) mend_values<DT, 1>(value, [&](int) { return seen_ones<DT>(seen); }, [&](int) -> v4f& { return o[h][c]; });
#pragma unroll
                for (int part = 0; part < PARTS; ++part) o[h][c] = mfma16<DT>(value, weight[part], o[h][c]);
            }
    };

    // An infinite value must not meet weights that are rounded to zero, nor parts of weights of both signs: where a sum is not finite the wave goes through its keys once more and
    // takes such values out of all steps, as where they must not meet the weights of rows that do not see them.  The second pass is code of its own, off the way: as a loop around
    // one, whose end is a jump, it cost a single token 0.7 us of 11.6.
    auto pass = [&](bool careful) __attribute__((always_inline)) {
        top = -INFINITY;
        sum = 0.f;
#pragma unroll
        for (int h = 0; h < kHalves; ++h)
#pragma unroll
            for (int c = 0; c < kEach; ++c) o[h][c] = v4f{0.f, 0.f, 0.f, 0.f};
        // the steps that every row sees whole, the next one's loads under way; then those with new tokens or the end in them
        const int whole1 = careful ? step0 : min(step1, it.q.ctx >> 5);
        int step = step0 + wave;
        KeyStep<DP> one;
        if (step < step1) load(step, one);
        if constexpr (kAhead) {
            KeyStep<DP> two;
            while (step < whole1) {
                if (step + kWaves < step1) load(step + kWaves, two);
                compute(step, one, std::false_type());
                step += kWaves;
                if (step >= whole1) {
                    one = two;
                    break;
                }
                if (step + kWaves < step1) load(step + kWaves, one);
                compute(step, two, std::false_type());
                step += kWaves;
            }
        } else {
            while (step < whole1) {
                compute(step, one, std::false_type());
                step += kWaves;
                if (step < step1) load(step, one);
            }
        }
        while (step < step1) {
            compute(step, one, std::true_type());
            step += kWaves;
            if (step < step1) load(step, one);
        }
    };
    pass(false);
    float zero = 0.f;
#pragma unroll
    for (int h = 0; h < kHalves; ++h)
#pragma unroll
        for (int c = 0; c < kEach; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) zero = fmaf(o[h][c][i], 0.f, zero);
    if (__builtin_expect(__ballot(zero != 0.f) != 0, 0)) pass(true);

    // the waves' results: maxima and sums of all rows first, so that each wave brings its own to the common maximum
    sum = row_sum(sum);
    if (g == 0) {
        lds_ml[(wave * 16 + n) * 2] = top;
        lds_ml[(wave * 16 + n) * 2 + 1] = sum;
    }
    __syncthreads();
    // of a part whose maximum is t: its factor under the maximum `high`
    auto share = [](float t, float high) { return t == -INFINITY ? (t == high ? 1.f : 0.f) : __builtin_amdgcn_exp2f(t - high); };
    {
        float high = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) high = fmaxf(high, lds_ml[(w * 16 + n) * 2]);
        const float factor = share(top, high);
        float* const mine = lds_o + (wave * 16 + n) * kRowFloats;
#pragma unroll
        for (int h = 0; h < kHalves; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int c = 0; c < kEach; c += 4) *(v4f*)(mine + element(h, c, i)) = v4f{o[h][c][i], o[h][c + 1][i], o[h][c + 2][i], o[h][c + 3][i]} * factor;
    }
    __syncthreads();
    constexpr int kAcross = kWaves * 4;                             // threads to a row
    const int r = threadIdx.x / kAcross, part = threadIdx.x % kAcross, row = it.tile * kRows + r;
    if (row >= it.q.n * a.group) return;
    float high = -INFINITY, total = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) high = fmaxf(high, lds_ml[(w * 16 + r) * 2]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) total += lds_ml[(w * 16 + r) * 2 + 1] * share(lds_ml[(w * 16 + r) * 2], high);
    const int t = row / a.group, h = head * a.group + row - t * a.group;
    const int64_t item = (int64_t)(it.index + it.run * tiles_of(it.q, a, kRows)) * a.kv.heads + head;
    const bool whole = it.runs == 1;
    const float scale = total == 0.f ? 0.f : 1.f / total;
    for (int d = part * 4; d < a.kv.head_dim; d += kAcross * 4) {
        v4f x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) x += *(const v4f*)(lds_o + (w * 16 + r) * kRowFloats + d);
        if (whole) store4(a.out, a.out_dtype, (it.q.first + t) * a.out_stride + (int64_t)h * a.kv.head_dim + d, total == 0.f ? v4f{0.f, 0.f, 0.f, 0.f} : x * scale);
        else *(v4f*)(a.part_o + (item * kRows + r) * DP + d) = x;
    }
    if (part == 0) {
        if (!whole) {
            a.part_ml[(item * kRows + r) * 2] = high;
            a.part_ml[(item * kRows + r) * 2 + 1] = total;
        } else if (a.lse) {
            a.lse[(int64_t)(it.q.first + t) * a.q_heads + h] = total == 0.f ? -INFINITY : (high + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
        }
    }
}

// ---------------------------------------------------------------------------------------------
// Many rows: the four waves of a workgroup have rows of their own, 16 R each, and share the keys through LDS.  Loads go to LDS directly, three blocks ahead of
// the one that is worked on (one, for heads of 256); one barrier a block.  Rows of keys lie in LDS with their 16-byte pieces
// exchanged by the key's number (every lane chooses the piece that it loads), so that neither the operands of K (a piece of 16 keys) nor those of V (read transposed: four keys
// of 16 elements by each 16 lanes) meet in the same banks.  Two rows of 16 to a wave where there are more than 64 rows to a sequence: an operand of keys then serves two
// products (2048 tokens behind 4095, 64 and 8 heads of 128: 342 us; with one 440, on the same card).  Four, one wave to a SIMD, do not fit its registers (545 us).
// Six tokens behind 131071: 106 us for 537 MB (562 read, 13 written for the joining); five trees of up to 21 tokens behind up to 12301, capped scores, fp32 results: 52 us for 174 MB (187 read),
// where products, exponentials and bytes take as much each and do not overlap whole.
// ---------------------------------------------------------------------------------------------
constexpr int wide_keys(int dp) { return dp == 64 ? 64 : 32; }             // of a block
constexpr int wide_buffers(int dp) { return dp == 256 ? 2 : 4; }           // a power of two
constexpr int wide_lds(int dp) { return wide_buffers(dp) * 2 * wide_keys(dp) * dp * 2 + kWaves * (int)sizeof(int); }

// 16 bytes of each lane at base + offset -> LDS, one lane's after the other's, from byte `to` on (the same in all lanes)
// (the waits: one instruction between m0's write and its use, five between a scalar register's by the vector unit and its use as an address; m0 is named as written: the compiler
// sets it before uses of its own, but may set it once for several, and warns of any reserved register in such a list)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void lds_load(const void* base, uint32_t offset, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop

// the order of a region with the products of a block's keys and the weights of another: an exponential and what belongs to it to every product
template <int R, int TILES, int PARTS>
__device__ __forceinline__ void interleave()
{
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        __builtin_amdgcn_sched_group_barrier(0x100, PARTS, 0);           // LDS reads
#pragma unroll
        for (int i = 0; i < R * PARTS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);           // matrix
            __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);           // vector
            __builtin_amdgcn_sched_group_barrier(0x400, 1, 0);           // exponentials
        }
    }
}

template <int DT, int DP, int R, int PARTS, bool CAP>
__global__ __launch_bounds__(kWaves * 64, 2) void attn_wide_kernel(AttnArgs a)
{
    constexpr int kRows = 64 * R, kKeys = wide_keys(DP), kAhead = wide_buffers(DP) - 1, kTiles = kKeys / 16, kParts = DP / 32, kCols = DP / 16;
    constexpr int kRowBytes = DP * 2, kPieces = DP / 8, kSide = kKeys * kRowBytes, kLoads = kSide / 1024 / kWaves, kKeysPerLoad = 1024 / kRowBytes;
    constexpr int kSwizzle = kPieces < 16 ? kPieces - 1 : 15;
    typedef __attribute__((address_space(3))) char* lptr;
    typedef const __attribute__((address_space(3))) v4u* lptr_v4u;
    typedef short v4s __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) v4s* lptr_v4s;
    extern __shared__ float lds[];                                  // [kAhead + 1][K, V][kKeys][kRowBytes], then [kWaves]: values that are not finite
    const lptr base = (lptr)(__attribute__((address_space(3))) void*)lds;
    int* const odd = (int*)((char*)lds + (kAhead + 1) * 2 * kSide);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = lane >> 4, n = lane & 15;
    const int head = blockIdx.x % a.kv.heads, number = blockIdx.x / a.kv.heads;
    Item it;
    if (!find_item(a, kRows, number, lane, &it)) return;
    const int keys = tile_keys(a, it.q, it.tile, kRows);
    const int block0 = it.run * it.per * (kBlock / kKeys), block1 = min((it.run + 1) * it.per * (kBlock / kKeys), (keys + kKeys - 1) / kKeys);

    // this lane's rows, one of each 16: their tokens and their operands
    const int row0 = it.tile * kRows + wave * 16 * R, all_rows = it.q.n * a.group;
    int token[R];
    v4u q[R][kParts];
    const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;         // scores are taken with a positive scale
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = row0 + r * 16 + n;
        const bool real = row < all_rows;
        token[r] = real ? row / a.group : -1;
        const int h = head * a.group + (real ? row - token[r] * a.group : 0);
        const uint16_t* const at = (const uint16_t*)a.q + (it.q.first + max(token[r], 0)) * a.q_stride + (int64_t)h * a.kv.head_dim;
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
            const int d = 32 * p + 8 * g;
            q[r][p] = v4u{0, 0, 0, 0};
            if (real && d < a.kv.head_dim) q[r][p] = *(gptr_v4u_any)(at + d);
#pragma unroll
            for (int i = 0; i < 4; ++i) q[r][p][i] ^= flip;
        }
    }
    // keys that every row of the wave sees, and that some row sees
    const int last_row = min(row0 + 16 * R, all_rows) - 1;
    const int whole = row0 >= all_rows ? 0 : a.tree ? min(it.q.keys, it.q.ctx) : keys_upto(it.q, row0 / a.group);
    const int some = row0 >= all_rows ? 0 : a.tree ? it.q.keys : keys_upto(it.q, last_row / a.group);
    const int tile_whole = a.tree ? min(it.q.keys, it.q.ctx) : keys_upto(it.q, it.tile * kRows / a.group);     // that every row of the tile sees

    v4f o[R][kCols];
    float top[R], sum[R];                                           // (sum: of this lane's keys)

    const sptr_i32 pages = (sptr_i32)(a.table + it.seq * a.table_stride);
    const int page_mask = (1 << a.kv.page_shift) - 1;
    const uint32_t slot_bytes = (uint32_t)a.kv.slot_stride * 2;
    // what this lane loads: piece `piece` of key `mine` of each of its wave's loads
    uint32_t from[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int mine = i * kKeysPerLoad + lane / kPieces, key = wave * (kKeys / kWaves) + mine;        // (kPieces lanes to a key)
        const int piece = (lane % kPieces) ^ (key & kSwizzle);
        from[i] = mine * slot_bytes + 2 * min(8 * piece, a.kv.head_dim - 8);
    }
    // The loads of a block, straight to LDS (64 lanes' 16 bytes one after the other).  They are written in assembly because the compiler takes any read of LDS
    // to need all of them; what waits for them is `arrived`, by count.  Past the end the last sixteen keys are loaded again: the count stays the same.
    auto key_of = [&](int block) {
        const int first = block * kKeys + wave * (kKeys / kWaves);
        return min(first & ~15, (keys - 1) & ~15) + (first & 15);
    };
    int next_page = pages[key_of(block0) >> a.kv.page_shift];       // of the block that is fetched next
    auto fetch = [&](int block, int buffer) {
        const int key = key_of(block);
        const int64_t page = min((uint32_t)next_page, (uint32_t)(a.kv.n_pages - 1));
        next_page = pages[key_of(block + 1) >> a.kv.page_shift];
        const int64_t at = page * a.kv.page_stride + (int64_t)(key & page_mask) * a.kv.slot_stride + head * a.kv.head_stride;
        const uint32_t to = (uint32_t)(uintptr_t)base + buffer * 2 * kSide + wave * kLoads * 1024;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) lds_load(a.kv.k + at, from[i], to + i * 1024);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) lds_load(a.kv.v + at, from[i], to + kSide + i * 1024);
    };
    // all of this wave's loads but those of the last `under_way` blocks are in LDS, and so are, after the barrier, the other waves'; nobody reads the blocks before them any more
    auto arrived = [&](auto under_way) { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(decltype(under_way)::value * 2 * kLoads) : "memory"); };
    // Values past the end are memory of any content: zeros.  Whether others are not finite.
    auto look = [&](int block, int buffer) {
        constexpr uint32_t exponent = DT == NQ_F16 ? 0x7c007c00u : 0x7f807f80u, lowest = DT == NQ_F16 ? 0x04000400u : 0x00800080u;
        typedef __attribute__((address_space(3))) v4u* lptr_out;
        const lptr v = base + buffer * 2 * kSide + kSide + wave * kLoads * 1024 + lane * 16;
        uint32_t bad = 0;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            v4u x = *(lptr_v4u)(v + i * 1024);
            if (block * kKeys + wave * (kKeys / kWaves) + i * kKeysPerLoad + lane / kPieces >= keys) *(lptr_out)(v + i * 1024) = x = v4u{0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < 4; ++w) bad |= (x[w] & exponent) + lowest;
        }
        const bool any = __ballot((bad & 0x80008000u) != 0) != 0;
        if (lane == 0) odd[wave] = any;
        __syncthreads();
        return (odd[0] | odd[1] | odd[2] | odd[3]) != 0;
    };
    // where this lane's operands are: K, piece 4p + g of key n; V, half a piece of key 4g + n / 4
    uint32_t at_k[kParts], at_v[kCols];
#pragma unroll
    for (int p = 0; p < kParts; ++p) at_k[p] = n * kRowBytes + (((4 * p + g) ^ (n & kSwizzle)) * 16);
#pragma unroll
    for (int c = 0; c < kCols; ++c) {
        const int key = 4 * g + (n >> 2);
        at_v[c] = kSide + key * kRowBytes + (((2 * c + ((n >> 1) & 1)) ^ (key & kSwizzle)) * 16) + (n & 1) * 8;
    }
    const float scale = fmaxf(fabsf(a.scale) * kLog2e, 1.17549435e-38f);      // of scores in powers of two (above zero: minus infinity stays)

    // the pieces of a block's work: products with the keys, the rows' maxima, weights, products with the values
    auto products = [&](int buffer, v4f (&s)[R][kTiles]) {
        const lptr from = base + buffer * 2 * kSide;
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int p = 0; p < kParts; ++p) {
                const v4u k = *(lptr_v4u)(from + at_k[p] + t * 16 * kRowBytes);
#pragma unroll
                for (int r = 0; r < R; ++r) s[r][t] = mfma16<DT>(k, q[r][p], p == 0 ? v4f{0.f, 0.f, 0.f, 0.f} : s[r][t]);
            }
    };
    const float unit = CAP ? 1.f : scale;
    auto raise = [&](v4f (&s)[R][kTiles]) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float most = s[r][0][0];
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) most = max2(most, s[r][t][i]);
            most = most * unit - kLift<DT>;
            if (__ballot(most > top[r] + kLazy)) {
                most = fmaxf(row_max(most), top[r]);
                const float factor = most == top[r] ? 1.f : __builtin_amdgcn_exp2f(top[r] - most);
                top[r] = most;
                sum[r] *= factor;
#pragma unroll
                for (int c = 0; c < kCols; ++c) o[r][c] *= factor;
            }
        }
    };
    auto cap_scores = [&](v4f (&s)[R][kTiles]) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
                s[r][t] = scores(s[r][t], fabsf(a.scale), a.cap);
    };
    typedef v4u Weights[PARTS][R][kTiles / 2];
    auto weigh = [&](const v4f (&s)[R][kTiles], Weights& weight) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float low = top[r] == -INFINITY ? 0.f : -top[r];
#pragma unroll
            for (int u = 0; u < kTiles / 2; ++u)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    float x = __builtin_amdgcn_exp2f(fmaf(s[r][2 * u + (w >> 1)][2 * (w & 1)], unit, low));
                    float y = __builtin_amdgcn_exp2f(fmaf(s[r][2 * u + (w >> 1)][2 * (w & 1) + 1], unit, low));
                    sum[r] += x + y;
                    weight[0][r][u][w] = round2<DT>(x, y);
#pragma unroll
                    for (int part = 1; part < PARTS; ++part) {
                        x -= widen<DT>(weight[part - 1][r][u][w], 0);
                        y -= widen<DT>(weight[part - 1][r][u][w], 1);
                        weight[part][r][u][w] = round2<DT>(x, y);
                    }
                }
        }
    };
    uint32_t seen[R];                                               // bit 4t + i: key 16t + 4g + i of a block
    auto add_values = [&](int buffer, const Weights& weight, auto mend_t) {
        const lptr from = base + buffer * 2 * kSide;
#pragma unroll
        for (int u = 0; u < kTiles / 2; ++u)
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                const v2u low = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr_v4s)(from + at_v[c] + u * 32 * kRowBytes)));
                const v2u high = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr_v4s)(from + at_v[c] + (u * 32 + 16) * kRowBytes)));
                v4u value = {low.x, low.y, high.x, high.y};
                if (decltype(mend_t)::value) mend_values<DT, R>(value, [&](int r) { return seen_ones<DT>(seen[r] >> (8 * u)); }, [&](int r) -> v4f& { return o[r][c]; });
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int part = 0; part < PARTS; ++part) o[r][c] = mfma16<DT>(value, weight[part][r][u], o[r][c]);
            }
    };
    // a block by itself.  masked: some key of it is not seen by some row of the wave; mend: and it has values that are not finite (a copy of its own, off the way)
    auto compute = [&](int block, int buffer, bool masked, auto mend_t) {
        v4f s[R][kTiles];
        Weights weight;
        products(buffer, s);
        if (CAP) cap_scores(s);
        if (decltype(mend_t)::value || masked) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                seen[r] = seen_keys<kTiles>(a, it.q, token[r], block * kKeys + 4 * g);
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!(seen[r] >> (4 * t + i) & 1u)) s[r][t][i] = -INFINITY;
            }
        }
        raise(s);
        weigh(s, weight);
        add_values(buffer, weight, mend_t);
    };

    // (as in attn_split_kernel: once more, if a sum is not finite; by the whole workgroup)
    auto pass = [&](bool careful) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            top[r] = -INFINITY;
            sum[r] = 0.f;
#pragma unroll
            for (int c = 0; c < kCols; ++c) o[r][c] = v4f{0.f, 0.f, 0.f, 0.f};
        }
        if (block0 < block1) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) fetch(block0 + i, i);
            // blocks that every row of the tile sees, one after the other through the buffers; then the rest
            int block = block0;
            const int upto = careful ? block0 : min(block1, tile_whole / kKeys) - kAhead;
            if constexpr (kAhead == 3) {
                // the products with a block's keys run while the weights of the block before it are formed
                if (block < upto) {
                    v4f s[2][R][kTiles];
                    arrived(std::integral_constant<int, 2>());
                    // (a wave without rows loads its part of the keys and leaves the rest to the other workgroup's)
                    for (; row0 >= all_rows && block < upto; block += 4) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            arrived(std::integral_constant<int, 1>());
                            fetch(block + i + 3, (i + 3) & 3);
                        }
                    }
                    if (block < upto) products(0, s[0]);
                    for (; block < upto; block += 4) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            arrived(std::integral_constant<int, 1>());
                            fetch(block + i + 3, (i + 3) & 3);
                            Weights weight;
                            if (CAP) cap_scores(s[i & 1]);
                            raise(s[i & 1]);
                            __builtin_amdgcn_sched_barrier(0);
                            products((i + 1) & 3, s[(i + 1) & 1]);
                            weigh(s[i & 1], weight);
                            interleave<R, kTiles, kParts>();
                            __builtin_amdgcn_sched_barrier(0);
                            add_values(i, weight, std::false_type());
                        }
                    }
                }
            } else {
                for (; block < upto; block += 2) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        arrived(std::integral_constant<int, 0>());
                        fetch(block + i + 1, (i + 1) & 1);
                        if (row0 < all_rows) compute(block + i, i, false, std::false_type());
                    }
                }
            }
            for (int buffer = 0; block < block1; ++block, buffer = (buffer + 1) & kAhead) {
                arrived(std::integral_constant<int, kAhead - 1>());
                fetch(block + kAhead, (buffer + kAhead) & kAhead);
                bool mend = careful;
                if ((block + 1) * kKeys > tile_whole) mend |= __builtin_amdgcn_readfirstlane(look(block, buffer)) != 0;
                if (block * kKeys >= some) continue;
                if (mend) compute(block, buffer, true, std::true_type());
                else compute(block, buffer, (block + 1) * kKeys > whole, std::false_type());
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");            // the loads past the end: nothing may arrive after the workgroup
        }
    };
    auto once_more = [&]() __attribute__((always_inline)) {
        float zero = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < kCols; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) zero = fmaf(o[r][c][i], 0.f, zero);
        const bool any = __ballot(zero != 0.f) != 0;
        __syncthreads();
        if (lane == 0) odd[wave] = any;
        __syncthreads();
        if (__builtin_expect((odd[0] | odd[1] | odd[2] | odd[3]) == 0, 1)) return false;
        __syncthreads();
        next_page = pages[key_of(block0) >> a.kv.page_shift];
        return true;
    };
    // (tiles of 128 rows: code of its own, 2048 tokens behind 4095 of an fp16 cache 351 us, as a loop 365; of 64: as a loop, five trees without caps 42.2 us, code of its own 43.6)
    constexpr bool kExact = PARTS == 1 && DT == NQ_BF16;               // a single part of bf16 has the range of fp32: no weight is rounded to zero
    if constexpr (R == 2) {
        pass(false);
        if constexpr (!kExact)
            if (once_more()) pass(true);
    } else {
        for (bool careful = false;; careful = true) {
            pass(careful);
            if (kExact || careful || !once_more()) break;
        }
    }

    const int64_t item = (int64_t)(it.index + it.run * tiles_of(it.q, a, kRows)) * a.kv.heads + head;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const float total = row_sum(sum[r]);
        if (token[r] < 0) continue;
        const int row = row0 + r * 16 + n, h = head * a.group + row - token[r] * a.group;
        if (it.runs == 1) {
            const float inverse = total == 0.f ? 0.f : 1.f / total;
            const int64_t to = (it.q.first + token[r]) * a.out_stride + (int64_t)h * a.kv.head_dim;
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                const int d = 16 * c + 4 * g;
                if (d >= a.kv.head_dim) continue;
                const v4f x = total == 0.f ? v4f{0.f, 0.f, 0.f, 0.f} : o[r][c] * inverse;
                store4(a.out, a.out_dtype, to + d, x);
            }
            if (g == 0 && a.lse) a.lse[(int64_t)(it.q.first + token[r]) * a.q_heads + h] = total == 0.f ? -INFINITY : (top[r] + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
        } else {
            const int64_t place = item * kRows + (row - it.tile * kRows);
#pragma unroll
            for (int c = 0; c < kCols; ++c) *(v4f*)(a.part_o + place * DP + 16 * c + 4 * g) = o[r][c];
            if (g == 0) {
                a.part_ml[place * 2] = top[r];
                a.part_ml[place * 2 + 1] = total;
            }
        }
    }
}

// Where the runs of a row are among the items' rows: `used` of them (0: it needs no joining), from `at` on, `step` apart.  number: of a (token, query head); the same in the wave
struct RowRuns {
    int used;
    int64_t at, step;
};
__device__ __forceinline__ RowRuns find_runs(const AttnArgs& a, int rows, int run, int lane, const Seq& front, int64_t number)
{
    const int t = (int)(number / a.q_heads), h = (int)(number - (int64_t)t * a.q_heads);
    int before = 0;
    for (int s0 = 0; s0 < a.n_seqs; s0 += 64) {
        const Seq q = s0 == 0 ? front : sequence(a, s0 + lane);
        const int tiles = tiles_of(q, a, rows), blocks = blocks_of(q), runs = runs_of(blocks, run);
        const int items = items_of(tiles, runs, a), upto = before + (int)wave_scan((uint32_t)items);
        const uint64_t here = __ballot(t >= q.first && t < q.first + q.n);
        if (here) {
            const int s = __builtin_ctzll(here);
            auto pick = [&](int v) { return __builtin_amdgcn_readlane(v, s); };
            const int n_runs = pick(runs), n_tiles = pick(tiles), n_blocks = pick(blocks);
            const int64_t first = pick(upto - items);
            const Seq mine = {pick(q.first), pick(q.n), pick(q.ctx), pick(q.keys)};
            if (n_runs <= 1 || first + pick(items) > a.items) break;                                // (the latter as in find_item)
            const int row = (t - mine.first) * a.group + h % a.group, tile = row / rows;
            const int per = (n_blocks + n_runs - 1) / n_runs;
            const int used = min(n_runs, ((tile_keys(a, mine, tile, rows) + kBlock - 1) / kBlock + per - 1) / per);
            return RowRuns{used, ((first + tile) * a.kv.heads + h / a.group) * rows + (row - tile * rows), (int64_t)n_tiles * a.kv.heads * rows};
        }
        before = min(__builtin_amdgcn_readlane(upto, 63), a.items + 1);
    }
    return RowRuns{0, 0, 0};
}

// Sums under the largest maximum of the runs that were added: four elements of a row, from every stride-th run, four runs' loads at a time
struct Joined {
    v4f x = {0.f, 0.f, 0.f, 0.f};
    float total = 0.f, high = -INFINITY;
    // of a part whose maximum is t (minus infinity: runs that the row sees nothing of, and those of which every score is NaN, whose sum is NaN as well)
    static __device__ __forceinline__ float share(float t, float top) { return t == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(t - top); }
    static __device__ __forceinline__ bool nothing(float t, float total) { return t == -INFINITY && total == 0.f; }
    template <int DP>
    __device__ __forceinline__ void add(const AttnArgs& a, const RowRuns& r, int d, int first, int stride)
    {
        for (int r0 = first; r0 < r.used; r0 += 4 * stride) {
            v4f v[4];
            float top[4], sum[4], most = high;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int64_t p = r.at + min(r0 + k * stride, r.used - 1) * r.step;
                v[k] = d < a.kv.head_dim ? *(const v4f*)(a.part_o + p * DP + d) : v4f{0.f, 0.f, 0.f, 0.f};
                top[k] = r0 + k * stride < r.used ? a.part_ml[p * 2] : -INFINITY;
                sum[k] = r0 + k * stride < r.used ? a.part_ml[p * 2 + 1] : 0.f;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) most = fmaxf(most, top[k]);
            const float f = share(high, most);
            x *= f;
            total *= f;
            high = most;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (nothing(top[k], sum[k])) continue;
                const float g = share(top[k], high);
                x += v[k] * g;
                total += sum[k] * g;
            }
        }
    }
    __device__ __forceinline__ void store(const AttnArgs& a, int64_t number, int d) const
    {
        const int64_t t = number / a.q_heads, h = number - t * a.q_heads;
        if (d < a.kv.head_dim) store4(a.out, a.out_dtype, t * a.out_stride + h * a.kv.head_dim + d, total == 0.f ? v4f{0.f, 0.f, 0.f, 0.f} : x * (1.f / total));
        if (d == 0 && a.lse) a.lse[number] = total == 0.f ? -INFINITY : (high + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
    }
};

// The runs of the rows that have several, in a fixed order.  A row's elements are DP / 4 threads' four; MANY: they go through all its runs, each group of so many threads
// with a row of its own; else a workgroup has one row, and its groups every so manyth run, whose sums meet in LDS.  Bound by the latency of what is looked up and loaded one
// after the other, and with many waves by the looking up itself, hence MANY from two rows to a CU on: 32768 rows of two runs in 20 us (a workgroup to a row: 73), 2048 rows of
// up to four runs in 7 (11).
template <int DP, bool MANY>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a, int rows)
{
    constexpr int kAcross = DP / 4, kAtOnce = 256 / kAcross;
    const int lane = threadIdx.x & 63;
    const Seq front = sequence(a, lane);
    const int run = run_length(a, rows, lane, front);
    if (run == kNoRuns) return;
    const int64_t all = (int64_t)a.n_tokens * a.q_heads;
    const int part = threadIdx.x / kAcross, d = (threadIdx.x % kAcross) * 4;
    if constexpr (MANY) {
        constexpr int kWaveRows = 64 / kAcross;
        const int wave = threadIdx.x >> 6;
        for (int64_t at = ((int64_t)blockIdx.x * 4 + wave) * kWaveRows; at < all; at += (int64_t)gridDim.x * kAtOnce) {
            RowRuns mine = {0, 0, 0};
#pragma unroll
            for (int w = 0; w < kWaveRows; ++w) {
                const RowRuns r = find_runs(a, rows, run, lane, front, min(at + w, all - 1));
                if (lane / kAcross == w && at + w < all) mine = r;
            }
            Joined j;
            j.add<DP>(a, mine, d, 0, 1);
            if (mine.used > 0) j.store(a, at + lane / kAcross, d);
        }
    } else {
        __shared__ float lds_x[kAtOnce][DP], lds_total[kAtOnce], lds_high[kAtOnce];
        for (int64_t at = blockIdx.x; at < all; at += gridDim.x) {
            const RowRuns mine = find_runs(a, rows, run, lane, front, at);
            if (mine.used == 0) continue;
            Joined j;
            j.add<DP>(a, mine, d, part, kAtOnce);
            *(v4f*)&lds_x[part][d] = j.x;
            if (d == 0) {
                lds_total[part] = j.total;
                lds_high[part] = j.high;
            }
            __syncthreads();
            if (threadIdx.x < kAcross) {
                Joined sum;
#pragma unroll
                for (int p = 0; p < kAtOnce; ++p) sum.high = fmaxf(sum.high, lds_high[p]);
#pragma unroll
                for (int p = 0; p < kAtOnce; ++p) {
                    if (Joined::nothing(lds_high[p], lds_total[p])) continue;
                    const float f = Joined::share(lds_high[p], sum.high);
                    sum.x += *(const v4f*)&lds_x[p][d] * f;
                    sum.total += lds_total[p] * f;
                }
                sum.store(a, at, d);
            }
            __syncthreads();
        }
    }
}

static int padded_dim(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; }

// PARTS: parts of the weights where there are many rows.  One part of bf16 is eight bits, an error as large as the results' own rounding: 2.3 10^-3 of the results in the 2-norm,
// where a single rounding of exact ones leaves 1.7 10^-3.  Few rows have two parts in any case: their calls are bound by bytes for the most part (one token behind 1023: 12.5 us with two
// parts, 12.1 with one; 32 sequences of up to 8191 125.5 and 125.2; six tokens behind 131071 110 and 109; five trees with capped scores, fp16 results 55.5 and 49).  Many rows
// are bound by the matrix products, and have one part where the results are of the cache's type or a coarser one: 2048 tokens behind 4095 take 342 us with one part, 447 with two.
template <int DT, int DP, int PARTS>
static int launch_attention(const AttnArgs& a, const char* who, hipStream_t s)
{
    constexpr int kFew = PARTS < 2 ? 2 : PARTS;
    const dim3 grid((unsigned)a.items * a.kv.heads), block(kWaves * 64);
    if (a.rows == 16) {
        constexpr int lds = split_lds(DP);
        NQ_ALLOW_LDS((attn_split_kernel<DT, DP, kFew>), lds);
        hipLaunchKernelGGL((attn_split_kernel<DT, DP, kFew>), grid, block, lds, s, a);
    } else {
        constexpr int lds = wide_lds(DP);
        auto wide = [&](auto r, auto parts, auto capped) {
            constexpr int R = decltype(r)::value, kParts = decltype(parts)::value;
            constexpr bool CAP = decltype(capped)::value;
            NQ_ALLOW_LDS((attn_wide_kernel<DT, DP, R, kParts, CAP>), lds);
            hipLaunchKernelGGL((attn_wide_kernel<DT, DP, R, kParts, CAP>), grid, block, lds, s, a);
            return NQ_OK;
        };
        auto tiles = [&](auto r, auto parts) { return a.cap > 0.f ? wide(r, parts, std::true_type()) : wide(r, parts, std::false_type()); };
        typedef std::integral_constant<int, DP < 256 ? 2 : 1> Many;          // tiles of 16 rows to a wave
        const int rc = a.few ? tiles(std::integral_constant<int, 1>(), std::integral_constant<int, kFew>()) : tiles(Many(), std::integral_constant<int, PARTS>());
        if (rc) return rc;
    }
    if (const int rc = launched(who)) return rc;
    const int64_t all = (int64_t)a.n_tokens * a.q_heads;
    const int cus = device_cu_count(), many = 256 / (DP / 4);
    if (all > 2 * cus) hipLaunchKernelGGL((attn_join_kernel<DP, true>), dim3((unsigned)std::min<int64_t>((all + many - 1) / many, 8 * cus)), dim3(256), 0, s, a, a.rows);
    else hipLaunchKernelGGL((attn_join_kernel<DP, false>), dim3((unsigned)all), dim3(256), 0, s, a, a.rows);
    return launched(who);
}

template <int DT, int PARTS>
static int launch_for_head_dim(const AttnArgs& a, const char* who, hipStream_t s)
{
    const int dp = padded_dim(a.kv.head_dim);
    return dp == 64 ? launch_attention<DT, 64, PARTS>(a, who, s) : dp == 128 ? launch_attention<DT, 128, PARTS>(a, who, s) : launch_attention<DT, 256, PARTS>(a, who, s);
}

}  // namespace nq
