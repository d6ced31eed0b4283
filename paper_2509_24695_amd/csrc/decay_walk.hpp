// Causal linear attention with a decay for each head, over whole sequences.
//
//   S_t = l S_{t-1} + k_t v_t^T          o_t = S_t^T q_t          l = exp(log_decay[h])
//
// In chunks of C tokens (rows i, j = 0..C-1; S the state before the chunk):
//
//   o_i = l^{i+1} S^T q_i + sum_{j <= i} l^{i-j} (q_i . k_j) v_j
//   S  <- l^C S + sum_j l^{C-1-j} k_j v_j^T
//
// All four products run on the matrix cores; every power of l that occurs has an exponent >= 0, so nothing overflows however strong the
// decay is (and a growing head's weights are held to finite ones).  The backward pass is the same walk three times, on other operands (WalkProblem):
//
//   dq   q, k, v = dO, V, K from the transposed state        forwards
//   dv             K, Q, dO from the gradient of the state   backwards in time
//   dk             V, dO, Q from its transpose               backwards in time
//
// Backwards, G_c = l^C G_{c+1} + sum_i l^{i+1} q_i do_i^T is what the tokens behind a chunk hand to it (G at the end: the gradient of
// the final state), so with rows counted from the chunk's last token the state's factor is l^r where it is l^{r+1} forwards, and a row's
// weight in the new state l^{C-r} where it is l^{C-1-r} (`back`).
//
// One workgroup walks one segment of one head's sequence, a wave per 32 value features: the wave keeps its 32 columns of S as fp32
// accumulators over the whole segment.  The chunk's C x C products are the same for all of the workgroup's waves: at bf16 and four waves each
// wave works one of the three 32 x 32 tiles out for all (with scores in one piece: 32 760 tokens of 20 heads of 112 228 us, every wave for itself,
// 24 of its 94 matrix instructions, 243; 7 x 8 heads of up to 1 501 tokens of 128 46 and 51; with two pieces the latter would not fit the registers), at fp32
// each adds up a part of the features (4 680 tokens of 32 heads of 64 73.2 us, every wave for itself 76.6; 8 000 tokens of 20 heads of 112 195
// and 216), at bf16 with fewer waves every wave has its own (4 680 tokens of 32 heads of 64, backward, with scores in one piece: 60 us, shared 72).
//
// Products are arranged so that a product's accumulators are the next one's operands as they lie: the lane of a 32 x 32 accumulator holds rows
// 8 (r / 4) + 4 h + r % 4 of one column, the lane of an operand eight consecutive indices 8 h .. 8 h + 7 of the contraction, so rows are dealt to
// the first operand of a product in the order decay_row, which makes eight accumulators in a row eight consecutive indices.
//
// Roundings (bf16 tokens): S enters o, the weighted scores l^{i-j} (q_i . k_j) enter o, and the weighted values l^{..} v_j enter S, as two bf16
// pieces (together within 2^-16), so that outputs are off by their own rounding, 1.66e-3 in the 2-norm.  (S in one piece: calls 3 to 8 % shorter, outputs
// 2.4e-3 off.  Scores in one: 2.3e-3 off for heads that remember up to some twenty tokens, 1.8e-3 over heads that remember 1 to 1 000; us with two / one:
// 32 760 tokens of 20 heads of 112 243 / 236, 75 600 of 64 heads of 64 644 / 639, backward pass of 4 680 of 32 heads of 64 66.4 / 62.5, 300 tokens of 224
// heads of 64 18.0 / 16.8.)  A state that the caller gets is an fp32 one: what goes into it, in the sums and in the last segment's walk, is in
// three pieces (2.7e-7 off after 32 760 tokens, with two 2.4e-6; with scores in one piece 246 us and 233).  fp32 tokens: fp32 products throughout (32 x 32 x 2 matrix
// instructions).
//
// A call of several segments is three launches: what each segment adds to the state, the scan over a head's segments, the walk.  It reads k and v
// twice, but for what weighs nothing any more: 64 heads of 75 600 tokens of 64 (2.5 GB that must move, 3.2 that do, where memories run from one token to
// a thousand) 640 to 658 us by device, 4.9 to 5.1 TB/s, as much as a copy of that size reaches: the walk is bound by memory, the sums by the heads that
// forget nothing (710 to 717 us where none forgets).  Heads of 112 whose rows lie between others' (32 760 tokens of 20; 0.59 GB, 0.82) take 236 to 248
// us (245 to 251): rows of 224 bytes begin and end inside lines of 128, the walk's reads are 1.13 times its bytes, and the walk alone took 138
// of 150 us without its products, 114 without its memory accesses (scores in one piece).  Calls that give each compute unit one or two
// workgroups are bound by a chunk's own run through LDS and the matrix cores (2.4 us at d = 64, 3.5 at 128; decay_plan.hpp).
// Measured with scores in one piece, and left: LDS rows whose 16-byte pieces change places, so that no read conflicts (of decay_sums' LDS cycles at d = 112 62 % are
// conflicts, the walk's 39 %): 1 to 3 % slower by the addresses' arithmetic, as LDS is busy for a sixth of the time; two chunks' rows on their way
// in decay_sums (the same, +-2 %) or in the walk (one workgroup less on a compute unit: 289 us instead of 252); heads in groups whose k and v fit
// the memory side's cache, one group after the other (702 us instead of 718).
#pragma once

#include "common.hpp"
#include "decay_plan.hpp"

namespace sv {

constexpr int kDecayTableBytes = (96 + 2 * 64 + 4) * 4;     // weights of scores and of the state's share; a word of each wave
constexpr uint32_t kNoRow = 0x80000000u;      // past every resource: the host keeps 64 rows below 2 GiB

// Row m of a 32-row operand serves index decay_row(m): bits 2 and 3 change places.
__host__ __device__ constexpr int decay_row(int m) { return (m & 0x13) | ((m & 4) << 1) | ((m & 8) >> 1); }

// One walk over the sequences (device pointers; strides in elements).
struct WalkProblem {
    const void *q, *k, *v;
    void *o;
    TokStrides sq, sk, sv, so;
    const float *s_begin;      // [BH][d][d]: state before the walk, NULL: zeros
    float *s_end;              // [BH][d][d]: receives the state behind it, or NULL
    float *slots;              // [BH][segments][d][d] partial states: begin of each segment
    float weight_state;        // factor of what comes out of the state,
    float weight_chunk;        //   of what comes out of the chunk itself,
    float weight_update;       //   and of what goes into the state
    int back;                  // 1: tokens from the last to the first, G's weights
    int turned;                // 1: s_begin and slots hold the transpose of this walk's state
    int kept;                  // 1: the state behind the walk is one that a caller may ask for (asked or not: outputs do not depend on it)
};

struct WalkArgs {
    WalkProblem p[3];
    const float *log_decay;    // [H]
    const int32_t *lengths;    // [B] or NULL
    int B, H, N;
    int segments, per_segment;
    int problems;
    int together;              // neighbouring heads that one die takes in a row
};

// ---- operands ------------------------------------------------------------------------------------------------------

// Eight consecutive indices of a contraction over 16 (lane half h: 8 h .. 8 h + 7), and the product over them.
template <typename T> struct Oct;
template <> struct Oct<uint16_t> {
    bf16x8 v;
};
template <> struct Oct<float> {
    float v[8];
};
__device__ __forceinline__ f32x16 oct_product(const Oct<uint16_t> &a, const Oct<uint16_t> &b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 oct_product(const Oct<float> &a, const Oct<float> &b, f32x16 c)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[e], b.v[e], c, 0, 0, 0);
    return c;
}

// Eight fp32 values as an operand: one piece, or (hi + lo) two.
__device__ __forceinline__ void oct_from(const float (&x)[8], Oct<float> &o)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) o.v[e] = x[e];
}
__device__ __forceinline__ void oct_from(const float (&x)[8], Oct<uint16_t> &o)
{
    const u32x4 w = {pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
    o.v = __builtin_bit_cast(bf16x8, w);
}
template <typename T> struct Pieces;
template <> struct Pieces<float> {
    Oct<float> hi;
    __device__ __forceinline__ explicit Pieces(const float (&x)[8]) { oct_from(x, hi); }
    __device__ __forceinline__ f32x16 first(const Oct<float> &b, f32x16 c) const { return oct_product(hi, b, c); }
    __device__ __forceinline__ f32x16 second(const Oct<float> &, f32x16 c) const { return c; }
    __device__ __forceinline__ f32x16 first_right(const Oct<float> &a, f32x16 c) const { return oct_product(a, hi, c); }
    __device__ __forceinline__ f32x16 second_right(const Oct<float> &, f32x16 c) const { return c; }
};
template <> struct Pieces<uint16_t> {
    Oct<uint16_t> hi, lo;
    __device__ __forceinline__ explicit Pieces(const float (&x)[8])
    {
        u32x4 h, l;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const uint32_t w = pack_bf16x2(x[2 * p], x[2 * p + 1]);
            h[p] = w;
            l[p] = pack_bf16x2(x[2 * p] - bf16_lo(w), x[2 * p + 1] - bf16_hi(w));
        }
        hi.v = __builtin_bit_cast(bf16x8, h);
        lo.v = __builtin_bit_cast(bf16x8, l);
    }
    __device__ __forceinline__ f32x16 first(const Oct<uint16_t> &b, f32x16 c) const { return oct_product(hi, b, c); }
    __device__ __forceinline__ f32x16 second(const Oct<uint16_t> &b, f32x16 c) const { return oct_product(lo, b, c); }
    __device__ __forceinline__ f32x16 first_right(const Oct<uint16_t> &a, f32x16 c) const { return oct_product(a, hi, c); }
    __device__ __forceinline__ f32x16 second_right(const Oct<uint16_t> &a, f32x16 c) const { return oct_product(a, lo, c); }
};

// What two pieces leave of the values, as a third.
struct Rest : Oct<uint16_t> {
    __device__ __forceinline__ Rest(const float (&x)[8], const Pieces<uint16_t> &p)
    {
        const u32x4 h = __builtin_bit_cast(u32x4, p.hi.v), l = __builtin_bit_cast(u32x4, p.lo.v);
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2((x[2 * i] - bf16_lo(h[i])) - bf16_lo(l[i]), (x[2 * i + 1] - bf16_hi(h[i])) - bf16_hi(l[i]));
        v = __builtin_bit_cast(bf16x8, w);
    }
};

// Sizes of the walk for element type T and head dimension D (112 is computed as 128: missing features are zeros in LDS).
template <typename T, int D> struct WalkShape {
    static constexpr int kDP = (D + 31) / 32 * 32, kPanels = kDP / 32, kWalkThreads = 64 * kPanels;
    static constexpr int kChunk = sizeof(T) == 2 ? kDecayChunkBf16 : kDecayChunkF32, kTiles = kChunk / 32;
    static constexpr int kVec = 16 / (int)sizeof(T), kRowVecs = kDP / kVec;
    // LDS row: 16 bytes past a multiple of 128 (64 at d = 32, bf16), so that eight rows' 16-byte pieces lie in different banks
    static constexpr int kRowBytes = kDP * (int)sizeof(T) + 16;
    static constexpr int kTileBytes = kChunk * kRowBytes;
    static constexpr int kRowsPerStep = kWalkThreads / kRowVecs, kSteps = kChunk / kRowsPerStep;
    static constexpr int kSubs = D / 16;                     // contractions over features, 16 at a time
    static constexpr int kTokSubs = kChunk / 16;             // and over the chunk's tokens
    static constexpr int kScoreTiles = kTiles == 2 ? 3 : 1;
    // who works the scores out: tile by tile for each other (kShared), each a part of the features (kSplit), or every wave for itself
    static constexpr bool kShared = sizeof(T) == 2 && kPanels == 4, kSplit = sizeof(T) == 4 && kPanels > 1;
    static constexpr int kOwnTiles = kShared ? 1 : kScoreTiles, kScoreBytes = kShared ? kScoreTiles * 2 * 2 * 64 * 8 * (int)sizeof(T) : 0;
    // bf16 pieces of a weighted score.  One would put 2^-8 of a term into the output beside the output's own rounding, which shows where a few terms
    // make up an output: heads that remember up to some twenty tokens, or short sequences (2.3e-3 off instead of 1.66e-3).
    static constexpr int kPieces = sizeof(T) == 2 ? 2 : 1;
    // Tiles in LDS: queries, keys, values and outputs.  With shared scores the waves meet after their last look at the queries, so that the outputs
    // take their place: a fourth tile and two pieces of each score would cost the compute unit its second workgroup (2 000 heads of 128, one
    // token: 83 us instead of 55).  A thread fetches those pieces of the outputs from there that it then overwrites with the next queries.
    static constexpr int kTilesInLds = kShared ? 3 : 4;
    static_assert(kSteps * kRowsPerStep == kChunk && D % 16 == 0, "whole rows");
};

// Eight features of a token row in LDS.
__device__ __forceinline__ void row_operand(const unsigned char *p, Oct<uint16_t> &o)
{
    o.v = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(p));
}
__device__ __forceinline__ void row_operand(const unsigned char *p, Oct<float> &o)
{
    const f32x4 a = *reinterpret_cast<const f32x4 *>(p), b = *reinterpret_cast<const f32x4 *>(p + 16);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        o.v[e] = a[e];
        o.v[4 + e] = b[e];
    }
}

// One feature of eight consecutive tokens: tokens tok0 + 8 h .. of a tile, features f0 .. f0 + 31 over the lanes' 32 rows, in their
// order or in that of decay_row (ROWS).
template <typename W, bool ROWS> __device__ __forceinline__ void token_operand(const unsigned char *tile, int tok0, int f0, int lane, Oct<uint16_t> &o)
{
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    typedef s16x4 __attribute__((address_space(3))) * lds_s16x4_ptr;
    // transposing read: within 16 lanes, lane i names token i / 4, features 4 (i % 4) .. + 3 and receives feature i of the four tokens
    const int i = lane & 15, fb = (lane >> 4) & 1, g = lane >> 5;
    const int quad = ROWS ? ((i & 1) << 1) | ((i & 2) >> 1) : i & 3;
    const unsigned char *p = tile + (tok0 + 8 * g + (i >> 2)) * W::kRowBytes + (f0 + 16 * fb + 4 * quad) * 2;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(p));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(p + 4 * W::kRowBytes));
    const s16x8 both = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    o.v = __builtin_bit_cast(bf16x8, both);
}
template <typename W, bool ROWS> __device__ __forceinline__ void token_operand(const unsigned char *tile, int tok0, int f0, int lane, Oct<float> &o)
{
    const int m = lane & 31, g = lane >> 5;
    const unsigned char *p = tile + (tok0 + 8 * g) * W::kRowBytes + (f0 + (ROWS ? decay_row(m) : m)) * 4;
#pragma unroll
    for (int e = 0; e < 8; ++e) o.v[e] = *reinterpret_cast<const float *>(p + e * W::kRowBytes);
}
__device__ __forceinline__ void oct_to(const Oct<uint16_t> &o, float (&x)[8])
{
    const u32x4 w = __builtin_bit_cast(u32x4, o.v);
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        x[2 * p] = bf16_lo(w[p]);
        x[2 * p + 1] = bf16_hi(w[p]);
    }
}
__device__ __forceinline__ void oct_to(const Oct<float> &o, float (&x)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = o.v[e];
}

// The operand is worked out here: nothing that reads memory later is moved in front of it.  (A scheduling barrier does not do: the compiler
// puts arithmetic next to its use before it schedules, and scores then live on in fp32 through the next product.)
__device__ __forceinline__ void settle(Oct<uint16_t> &o)
{
    u32x4 w = __builtin_bit_cast(u32x4, o.v);
    asm volatile("" : "+v"(w)::"memory");
    o.v = __builtin_bit_cast(bf16x8, w);
}
__device__ __forceinline__ void settle(Oct<float> &o)
{
    asm volatile("" : "+v"(o.v[0]), "+v"(o.v[1]), "+v"(o.v[2]), "+v"(o.v[3]), "+v"(o.v[4]), "+v"(o.v[5]), "+v"(o.v[6]), "+v"(o.v[7])::"memory");
}

// ---- powers of the decay ---------------------------------------------------------------------------------------------

// A weight that meets zeros (rows that are no tokens, a state of nothing) has to stay a number: a growing head's powers, l > 1, end at the largest.
__device__ __forceinline__ float held(float x)
{
    constexpr float kMost = 3.40282347e38f;
    return x > kMost ? kMost : x < -kMost ? -kMost : x;
}

// l^e for e >= 0.  A log decay of minus infinity is a decay of zero: l^0 = 1, all other powers 0.
struct DecayPower {
    float lg;
    __device__ __forceinline__ explicit DecayPower(float log_decay) : lg((log_decay < -1e30f ? -1e30f : log_decay) * 1.44269504088896f) {}
    __device__ __forceinline__ float operator()(int e) const { return held(power(e)); }
    // not held: infinite where it is too large
    __device__ __forceinline__ float power(int e) const { return exp2f(lg * (float)e); }
    __device__ __forceinline__ bool grows() const { return lg > 0.f; }
    // for exponents that are the same in all lanes: kept in scalar registers
    __device__ __forceinline__ float uniform(int e) const { return scalar((*this)(e)); }
    static __device__ __forceinline__ float scalar(float x)
    {
        return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x)));
    }
};

// l^C, by which a segment multiplies its state chunk after chunk.  With a long memory, l^C just below 1, the rounding of one float would add
// up over hundreds of chunks: every eighth factor makes up for the other seven's.
struct ChunkDecay {
    float usual, eighth;
    __device__ __forceinline__ ChunkDecay(int chunk, float log_decay)
    {
        const double x = exp((double)(log_decay < -1e30f ? -1e30f : log_decay) * (double)chunk);
        const float f = held((float)x);
        usual = DecayPower::scalar(f);
        eighth = DecayPower::scalar(x < 1e38 ? (float)(x + 7.0 * (x - (double)f)) : f);
    }
    __device__ __forceinline__ float operator()(int nth) const { return (nth & 7) == 7 ? eighth : usual; }
};

// ---- a chunk's tokens: global memory -> registers -> LDS ------------------------------------------------------------

// Where the rows of the walk's chunk c lie: a buffer resource over the chunk's rows and this lane's offset into it.  BACK: row r of the
// chunk is its r-th token from behind.  The lane takes every kRowsPerStep-th row, in the order in which they lie in memory.
template <typename T, int D, bool BACK> struct ChunkRows {
    using W = WalkShape<T, D>;
    const unsigned char *head;      // token 0 of the (batch, head)
    int64_t row_bytes;
    uint32_t off0;                  // of the lane's first row; past every row for features that do not exist
    int row0;

    __device__ __forceinline__ ChunkRows(const void *p, const TokStrides &st, int b, int h)
        : head(static_cast<const unsigned char *>(p) + (b * st.b + h * st.h) * (int64_t)sizeof(T)), row_bytes(st.n * (int64_t)sizeof(T))
    {
        const int c = threadIdx.x % W::kRowVecs;
        row0 = threadIdx.x / W::kRowVecs;
        off0 = c * W::kVec < D ? (uint32_t)row0 * (uint32_t)row_bytes + (uint32_t)c * 16u : kNoRow;
    }
    // Rows that are no tokens (the lead of the first chunk; all of them unless `live`) read as zeros.  BEGIN: chunk c may be the first.  (Left to the
    // comparison c == 0 the compiler finds out by an addition with carry whether c + 1 is zero, the resource is no longer a scalar one for
    // it, and each load gets a loop of its own over the resources of the lanes.)
    template <bool NT, bool BEGIN> __device__ __forceinline__ void load(int64_t c, bool live, int chunks, int lead, u32x4 (&reg)[W::kSteps]) const
    {
        const int64_t base = BACK ? (int64_t)(chunks - 1 - c) * W::kChunk : c * W::kChunk - lead;
        const rsrc_t r = make_rsrc(head + base * row_bytes, live ? (uint32_t)((W::kChunk - 1) * row_bytes + D * (int)sizeof(T)) : 0u);
        // the steps' offsets are worked out anew for every chunk: kept over the loop they are twelve registers too many
        uint32_t off = off0;
        asm volatile("" : "+v"(off));
        constexpr int kStep = W::kRowsPerStep;
        if constexpr (BEGIN) {
            const int nothing = c == 0 ? lead : 0;                     // rows in front of the first token
#pragma unroll
            for (int i = 0; i < W::kSteps; ++i) {
                const bool is = BACK ? row0 < W::kChunk - nothing - i * kStep : row0 >= nothing - i * kStep;
                reg[i] = load_stream16<NT>(r, is ? off + (uint32_t)(i * kStep) * (uint32_t)row_bytes : kNoRow);
            }
        } else {
#pragma unroll
            for (int i = 0; i < W::kSteps; ++i) reg[i] = load_stream16<NT>(r, off + (uint32_t)(i * kStep) * (uint32_t)row_bytes);
        }
    }
    __device__ __forceinline__ void put(unsigned char *tile, const u32x4 (&reg)[W::kSteps]) const
    {
        unsigned char *p = tile + (BACK ? W::kRowsPerStep - 1 - row0 : row0) * W::kRowBytes + (threadIdx.x % W::kRowVecs) * 16;
#pragma unroll
        for (int i = 0; i < W::kSteps; ++i)
            *reinterpret_cast<u32x4 *>(p + (BACK ? W::kSteps - 1 - i : i) * W::kRowsPerStep * W::kRowBytes) = reg[i];
    }
    // the other way: chunk c's rows from LDS, where they are tokens (none unless `live`)
    __device__ __forceinline__ void store(int64_t c, bool live, int chunks, int lead, const unsigned char *tile) const
    {
        const int64_t base = BACK ? (int64_t)(chunks - 1 - c) * W::kChunk : c * W::kChunk - lead;
        const rsrc_t r = make_rsrc(head + base * row_bytes, live ? (uint32_t)((W::kChunk - 1) * row_bytes + D * (int)sizeof(T)) : 0u);
        const int nothing = c == 0 ? lead : 0;
        const unsigned char *p = tile + (BACK ? W::kRowsPerStep - 1 - row0 : row0) * W::kRowBytes + (threadIdx.x % W::kRowVecs) * 16;
        uint32_t off = off0;
        asm volatile("" : "+v"(off));
#pragma unroll
        for (int i = 0; i < W::kSteps; ++i) {
            constexpr int kStep = W::kRowsPerStep;
            const bool is = BACK ? row0 < W::kChunk - nothing - i * kStep : row0 >= nothing - i * kStep;
            const u32x4 v = *reinterpret_cast<const u32x4 *>(p + (BACK ? W::kSteps - 1 - i : i) * kStep * W::kRowBytes);
            store_stream16<true>(r, is ? off + (uint32_t)(i * kStep) * (uint32_t)row_bytes : kNoRow, v);
        }
    }
};

// ---- the state ---------------------------------------------------------------------------------------------------------

// A wave's 32 columns of S: accumulator kt, register r of lane l is key feature 32 kt + 16 (r / 8) + 8 (l / 32) + r % 8, value feature
// 32 panel + l % 32.
template <int D> struct StatePanel {
    static constexpr int kKeyTiles = (D + 31) / 32;
    f32x16 s[kKeyTiles];

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int kt = 0; kt < kKeyTiles; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[kt][r] = 0.f;
    }
    // features that do not exist (112 is computed as 128) read as zeros and are not stored
    __device__ __forceinline__ void load(const float *src, bool turned, int panel, int lane)
    {
        const int h = lane >> 5, vf = 32 * panel + (lane & 31);
        const rsrc_t r = make_rsrc(src, D * D * 4);
        if (turned) {
            const uint32_t at = vf < D ? (uint32_t)(vf * D + 8 * h) * 4u : kNoRow;
#pragma unroll
            for (int kt = 0; kt < kKeyTiles; ++kt)
#pragma unroll
                for (int q = 0; q < 4; ++q) {                            // 16 features of a row and half: two times four for this lane half
                    const int kf = 32 * kt + 16 * (q >> 1) + 4 * (q & 1);
                    const f32x4 x = kf < D ? load_cached16(r, at + (uint32_t)kf * 4u) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[kt][4 * q + e] = x[e];
                }
        } else {
            const uint32_t at = vf < D ? (uint32_t)(8 * h * D + vf) * 4u : kNoRow;
#pragma unroll
            for (int kt = 0; kt < kKeyTiles; ++kt)
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                    const int kf = 32 * kt + 16 * (q >> 3) + (q & 7);
                    s[kt][q] = kf < D ? __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(r, at + (uint32_t)(kf * D) * 4u, 0, 0)) : 0.f;
                }
        }
    }
    __device__ __forceinline__ void store(float *dst, int panel, int lane) const
    {
        const int h = lane >> 5, vf = 32 * panel + (lane & 31);
        const rsrc_t r = make_rsrc(dst, D * D * 4);
        const uint32_t at = vf < D ? (uint32_t)(8 * h * D + vf) * 4u : kNoRow;
#pragma unroll
        for (int kt = 0; kt < kKeyTiles; ++kt)
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                const int kf = 32 * kt + 16 * (q >> 3) + (q & 7);
                if (kf < D) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(s[kt][q]), r, at + (uint32_t)(kf * D) * 4u, 0, 0);
            }
    }
    __device__ __forceinline__ void scale(float f)
    {
#pragma unroll
        for (int kt = 0; kt < kKeyTiles; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[kt][r] *= f;
    }
    __device__ __forceinline__ void eight(int sub, float (&x)[8]) const
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = s[sub / 2][8 * (sub % 2) + e];
    }
    __device__ __forceinline__ bool finite() const
    {
        float zero[4] = {0.f, 0.f, 0.f, 0.f};                           // zero times a number is zero
#pragma unroll
        for (int kt = 0; kt < kKeyTiles; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) zero[r & 3] = __builtin_fmaf(s[kt][r], 0.f, zero[r & 3]);
        return (zero[0] + zero[1]) + (zero[2] + zero[3]) == 0.f;
    }
};

// A row's weight in the new state, by lane half: l^{C-1-j} for j = 16 sub + 8 h + e.
template <int SUBS> struct UpdateWeights {
    float w[SUBS][8];
    // (a branch for growing heads: holding all of them costs a short call up to 1 us)
    __device__ __forceinline__ UpdateWeights(const DecayPower &pw, int chunk, int back, float factor, int lane)
    {
        const int h = lane >> 5;
        auto fill = [&](auto hold) __attribute__((always_inline)) {
            float near[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) near[e] = DecayPower::scalar(hold(pw.power(7 - e)));
#pragma unroll
            for (int s = 0; s < SUBS; ++s) {
                const float base = hold(factor * hold(pw.power(chunk - 8 - 16 * s - 8 * h + back)));
#pragma unroll
                for (int e = 0; e < 8; ++e) w[s][e] = hold(base * near[e]);
            }
        };
        if (pw.grows()) fill([](float x) { return held(x); });
        else fill([](float x) { return x; });
    }
    __device__ __forceinline__ void scale(float f)
    {
#pragma unroll
        for (int s = 0; s < SUBS; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) w[s][e] *= f;
        if (f > 1.f) {
#pragma unroll
            for (int s = 0; s < SUBS; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) w[s][e] = held(w[s][e]);
        }
    }
};

// S += sum over one sub-chunk of 16 tokens, weighted.  `values` is the wave's 32 value features of these tokens; `kept`: for a state that is kept.
template <typename T, int D>
__device__ __forceinline__ void state_update(StatePanel<D> &S, const unsigned char *tileK, const Oct<T> &values, const float (&w)[8], int sub,
                                             int lane, bool kept)
{
    using W = WalkShape<T, D>;
    float x[8];
    oct_to(values, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= w[e];
    const Pieces<T> v(x);
    Oct<T> k[StatePanel<D>::kKeyTiles];
#pragma unroll
    for (int kt = 0; kt < StatePanel<D>::kKeyTiles; ++kt) {
        token_operand<W, true>(tileK, 16 * sub, 32 * kt, lane, k[kt]);
        S.s[kt] = v.first_right(k[kt], S.s[kt]);
        S.s[kt] = v.second_right(k[kt], S.s[kt]);
    }
    if constexpr (sizeof(T) == 2)
        if (kept) {
            const Rest rest(x, v);
#pragma unroll
            for (int kt = 0; kt < StatePanel<D>::kKeyTiles; ++kt) S.s[kt] = oct_product(k[kt], rest, S.s[kt]);
        }
}

// ---- kernels -----------------------------------------------------------------------------------------------------------

// Which segment of which head a workgroup walks.
struct WalkTask {
    int problem, segment, bh;
    bool any;
    __device__ __forceinline__ WalkTask(int tasks, int BH, int segments, int together)
    {
        const int task = decay_task((int)blockIdx.x, together);
        any = task < tasks;
        bh = task % BH;
        segment = task / BH % segments;
        problem = task / BH / segments;
    }
};

__device__ __forceinline__ int walk_length(const WalkArgs &a, int b)
{
    if (!a.lengths) return a.N;
    const int n = __builtin_amdgcn_readfirstlane(a.lengths[b]);
    return n < 0 ? 0 : n > a.N ? a.N : n;
}

// What each segment but the last adds to the state, starting from zero: into slot segment + 1 of its head.  From the segment's end to its beginning:
// what a chunk loses to the decay until then is taken into its tokens' weights (32 of them, where the state would be 64 numbers of a lane), and
// the walk ends where the weights have come to zero: with a memory of 14 tokens (l = exp(-0.073)) 1 450 tokens back, l^1450 < 2^-150, half the
// smallest fp32 number (75 600 tokens of 64 heads whose memories run from one token to a thousand: 1.16 GB read and 216 us to the end, 0.70 GB and
// 180 so).  Sums of half a segment or less, for shorter walks and more workgroups, take longer (697 us a call instead of 650): less of them weighs
// nothing.
template <typename T, int D, bool BACK> __device__ __forceinline__ void segment_sum(const WalkArgs &a, const WalkProblem &p, const WalkTask &task, unsigned char *lds)
{
    using W = WalkShape<T, D>;
    unsigned char *tileK = lds, *tileV = lds + W::kTileBytes;
    const int b = task.bh / a.H, h = task.bh % a.H, lane = threadIdx.x & 63, panel = threadIdx.x >> 6;
    const float g = a.log_decay[h];
    const DecayWalk walk(walk_length(a, b), W::kChunk);
    const int c0 = task.segment * a.per_segment, c1 = c0 + a.per_segment;
    if (c1 >= walk.chunks) return;                                   // the last segment of this sequence, or one behind it
    // the first tokens are on their way while the powers are worked out
    const ChunkRows<T, D, BACK> rk(p.k, p.sk, b, h), rv(p.v, p.sv, b, h);
    u32x4 nk[W::kSteps], nv[W::kSteps];
    rk.template load<false, true>(c1 - 1, true, walk.chunks, walk.lead, nk);
    rv.template load<false, true>(c1 - 1, true, walk.chunks, walk.lead, nv);
    const DecayPower pw(g);
    UpdateWeights<W::kTokSubs> uw(pw, W::kChunk, BACK, p.weight_update, lane);
    const ChunkDecay decay(W::kChunk, g);
    StatePanel<D> S;
    S.clear();
    float most = p.weight_update;                                    // no weight of a decaying head is larger
    for (int c = c1 - 1;; --c) {
        lds_barrier();
        rk.put(tileK, nk);
        rv.put(tileV, nv);
        lds_barrier();
        rk.template load<false, true>(c - 1, c > c0, walk.chunks, walk.lead, nk);
        rv.template load<false, true>(c - 1, c > c0, walk.chunks, walk.lead, nv);
#pragma unroll
        for (int sub = 0; sub < W::kTokSubs; ++sub) {
            Oct<T> v;
            token_operand<W, false>(tileV, 16 * sub, 32 * panel, lane, v);
            state_update<T, D>(S, tileK, v, uw.w[sub], sub, lane, p.kept != 0);
        }
        if (c == c0) break;
        const float f = decay(c1 - 1 - c);
        uw.scale(f);
        most *= f;
        if (most == 0.f) break;
    }
    S.store(p.slots + ((int64_t)task.bh * a.segments + task.segment + 1) * D * D, panel, lane);
}
template <typename T, int D> __global__ __launch_bounds__((WalkShape<T, D>::kWalkThreads), 2) void decay_sums(WalkArgs a)
{
    __shared__ __align__(16) unsigned char lds[2 * WalkShape<T, D>::kTileBytes];
    const int BH = a.B * a.H;
    const WalkTask task(a.problems * BH * (a.segments - 1), BH, a.segments - 1, a.together);
    if (!task.any) return;
    const WalkProblem &p = a.p[task.problem];
    if (p.back) segment_sum<T, D, true>(a, p, task, lds);
    else segment_sum<T, D, false>(a, p, task, lds);
}

// Slot s of each head: from what segment s - 1 adds to the state before segment s, over all segments.  A thread per four elements, eight segments
// on their way (10 us for 24 MB of states; sixteen, or threads of two elements, the same).
template <typename T, int D> __global__ __launch_bounds__(256) void decay_scan(WalkArgs a)
{
    using W = WalkShape<T, D>;
    constexpr int kQuads = D * D / 4, kAhead = 8;
    const int BH = a.B * a.H, blocks = (kQuads + 255) / 256;
    const int i = (int)(blockIdx.x % blocks) * 256 + (int)threadIdx.x, bh = (int)(blockIdx.x / blocks) % BH;
    if (i >= kQuads) return;
    const WalkProblem &p = a.p[blockIdx.x / blocks / BH];
    const int b = bh / a.H, h = bh % a.H;
    const DecayWalk walk(walk_length(a, b), W::kChunk);
    const int last = (walk.chunks - 1) / a.per_segment;             // last segment with chunks
    if (walk.chunks == 0) return;
    const DecayPower pw(a.log_decay[h]);
    f32x4 *slot = reinterpret_cast<f32x4 *>(p.slots) + (int64_t)bh * a.segments * kQuads + i;
    f32x4 S = {0.f, 0.f, 0.f, 0.f};
    if (p.s_begin) {
        S = reinterpret_cast<const f32x4 *>(p.s_begin)[(int64_t)bh * kQuads + i];
        slot[0] = S;
    }
    const float whole = pw(a.per_segment * W::kChunk), first = pw(a.per_segment * W::kChunk - walk.lead);
    for (int s0 = 1; s0 <= last; s0 += kAhead) {
        f32x4 u[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (s0 + j <= last) u[j] = slot[(int64_t)(s0 + j) * kQuads];
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (s0 + j <= last) {
                const float f = s0 + j == 1 ? first : whole;
#pragma unroll
                for (int e = 0; e < 4; ++e) S[e] = __builtin_fmaf(S[e], f, u[j][e]);
                slot[(int64_t)(s0 + j) * kQuads] = S;
            }
    }
}

// Sixteen value features of a row tile into the tokens' rows in LDS: accumulators 8 x .. 8 x + 7 of lane l are features 16 x + 8 (.. / 4) + 4 h
// + .. of the panel, token l % 32.
template <typename W> __device__ __forceinline__ void put_features(unsigned char *row, const f32x16 &acc, int half, uint16_t)
{
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const uint32_t a0 = pack_bf16x2(acc[8 * x], acc[8 * x + 1]), a1 = pack_bf16x2(acc[8 * x + 2], acc[8 * x + 3]);
        const uint32_t b0 = pack_bf16x2(acc[8 * x + 4], acc[8 * x + 5]), b1 = pack_bf16x2(acc[8 * x + 6], acc[8 * x + 7]);
        // lane half 0 gives its features 8..11 for the other half's 4..7: each lane then holds eight in a row
        const auto p = __builtin_amdgcn_permlane32_swap(a0, b0, false, false), q = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
        *reinterpret_cast<u32x4 *>(row + (16 * x + 8 * half) * 2) = u32x4{p[0], q[0], p[1], q[1]};
    }
}
template <typename W> __device__ __forceinline__ void put_features(unsigned char *row, const f32x16 &acc, int half, float)
{
#pragma unroll
    for (int x = 0; x < 4; ++x) *reinterpret_cast<f32x4 *>(row + (8 * x + 4 * half) * 4) = f32x4{acc[4 * x], acc[4 * x + 1], acc[4 * x + 2], acc[4 * x + 3]};
}

// Where a walk's things lie in LDS.
template <typename T, int D> struct WalkLds {
    using W = WalkShape<T, D>;
    unsigned char *q, *k, *v, *o;       // tiles
    Oct<T> *scores;
    float *table, *from_state;
    int *votes;                         // of each wave
    __device__ __forceinline__ explicit WalkLds(unsigned char *lds)
        : q(lds), k(lds + W::kTileBytes), v(lds + 2 * W::kTileBytes), o(W::kTilesInLds == 4 ? lds + 3 * W::kTileBytes : q),
          scores(reinterpret_cast<Oct<T> *>(lds + W::kTilesInLds * W::kTileBytes)),
          table(reinterpret_cast<float *>(lds + W::kTilesInLds * W::kTileBytes + W::kScoreBytes)), from_state(table + 96),
          votes(reinterpret_cast<int *>(from_state + 128)) {}
};

// The state that a segment begins from, or NULL: zeros.
template <int D> __device__ __forceinline__ const float *begin_of(const WalkArgs &a, const WalkProblem &p, const WalkTask &task, int chunks)
{
    return a.segments > 1 && chunks > 0 && (task.segment > 0 || p.s_begin) ? p.slots + ((int64_t)task.bh * a.segments + task.segment) * D * D
           : p.s_begin                                                     ? p.s_begin + (int64_t)task.bh * D * D
                                                                           : nullptr;
}

// What a value adds to products: itself, or nothing and a mark where it is no number.
template <typename T> __device__ __forceinline__ void part_numbers(const Oct<T> &o, Oct<T> &numbers, Oct<T> &marks)
{
    float x[8], n[8], m[8];
    oct_to(o, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const bool is = __builtin_isfinite(x[e]);
        n[e] = is ? x[e] : 0.f;
        m[e] = is ? 0.f : 1.f;
    }
    oct_from(n, numbers);
    oct_from(m, marks);
}

// The walk of a segment into which a NaN or an infinity has come, once more.  A product over a chunk multiplies what lies ahead of a row by zero,
// and zero times such a value is NaN: in the walk proper it reaches outputs of up to 63 tokens before its own.  Here scores ahead of a row are taken
// out by their place, and values that are no numbers add nothing, but marks, whose products with ones at and behind their tokens tell
// which outputs see one of them.  `table` and `from_state` are as the walk has left them.  Nothing here is for speed; looking for such values
// in the state, once at a segment's end, takes 0.2 to 0.4 us of a call.
template <typename T, int D, bool BACK> __device__ __forceinline__ void walk_again(const WalkArgs &a, const WalkProblem &p, const WalkTask &task, unsigned char *lds)
{
    using W = WalkShape<T, D>;
    const WalkLds<T, D> at(lds);
    const int b = task.bh / a.H, h = task.bh % a.H, lane = threadIdx.x & 63, panel = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int half = lane >> 5, col = lane & 31;
    const float g = a.log_decay[h];
    const DecayWalk walk(walk_length(a, b), W::kChunk);
    const int c0 = task.segment * a.per_segment, c1 = c0 + a.per_segment < walk.chunks ? c0 + a.per_segment : walk.chunks;
    const bool last = c0 + a.per_segment >= walk.chunks;
    const ChunkRows<T, D, BACK> rq(p.q, p.sq, b, h), rk(p.k, p.sk, b, h), rv(p.v, p.sv, b, h), ro(p.o, p.so, b, h);
    const float *begin = begin_of<D>(a, p, task, walk.chunks);
    StatePanel<D> S;
    if (begin) S.load(begin, p.turned, panel, lane);
    else S.clear();
    const DecayPower pw(g);
    const ChunkDecay decay(W::kChunk, g);
    const float first_decay = pw.uniform(W::kChunk - walk.lead);
#pragma unroll 1
    for (int c = c0; c < c1; ++c) {
        u32x4 next[W::kSteps];
        lds_barrier();
        rq.template load<false, true>(c, true, walk.chunks, walk.lead, next);
        rq.put(at.q, next);
        rk.template load<false, true>(c, true, walk.chunks, walk.lead, next);
        rk.put(at.k, next);
        rv.template load<false, true>(c, true, walk.chunks, walk.lead, next);
        rv.put(at.v, next);
        lds_barrier();
#pragma unroll 1
        for (int it = 0; it < W::kTiles; ++it) {
            f32x16 acc, marked;
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[r] = marked[r] = 0.f;
            const unsigned char *rows = at.q + (32 * it + col) * W::kRowBytes + 8 * half * (int)sizeof(T);
#pragma unroll
            for (int sub = 0; sub < W::kSubs; ++sub) {
                Oct<T> q;
                row_operand(rows + 16 * sub * (int)sizeof(T), q);
                float x[8];
                S.eight(sub, x);
                // (taken apart anew for each tile: all of the state's pieces are as many registers as the state)
                asm volatile("" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]), "+v"(x[4]), "+v"(x[5]), "+v"(x[6]), "+v"(x[7]));
                const Pieces<T> s(x);
                acc = s.second(q, s.first(q, acc));
            }
            const float weight = at.from_state[(c == 0 ? 64 : 0) + 32 * it + col];
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[r] *= weight;
#pragma unroll 1
            for (int jt = 0; jt <= it; ++jt) {
                f32x16 P;
#pragma unroll
                for (int r = 0; r < 16; ++r) P[r] = 0.f;
#pragma unroll 1
                for (int sub = 0; sub < W::kSubs; ++sub) {
                    Oct<T> q, k;
                    row_operand(rows + 16 * sub * (int)sizeof(T), q);
                    row_operand(at.k + (32 * jt + decay_row(col)) * W::kRowBytes + (16 * sub + 8 * half) * (int)sizeof(T), k);
                    P = oct_product(k, q, P);
                }
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    float x[8], one[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int distance = 32 * (it - jt) + col - 16 * s - 8 * half - e;
                        x[e] = distance < 0 ? 0.f : P[8 * s + e] * at.table[63 - distance];
                        one[e] = distance < 0 ? 0.f : 1.f;
                    }
                    Oct<T> v, numbers, marks, ones;
                    token_operand<W, false>(at.v, 32 * jt + 16 * s, 32 * panel, lane, v);
                    part_numbers(v, numbers, marks);
                    oct_from(one, ones);
                    const Pieces<T> both(x);
                    acc = both.second_right(numbers, both.first_right(numbers, acc));
                    marked = oct_product(marks, ones, marked);
                }
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[r] = marked[r] > 0.f ? __builtin_nanf("") : acc[r];
            lds_barrier();                                             // rows of this tile are read here only: outputs may take their place
            put_features<W>(at.o + (32 * it + col) * W::kRowBytes + 32 * panel * (int)sizeof(T), acc, half, T{});
        }
        S.scale(c == 0 ? first_decay : decay(c));
#pragma unroll 1
        for (int sub = 0; sub < W::kTokSubs; ++sub) {
            Oct<T> v;
            token_operand<W, false>(at.v, 16 * sub, 32 * panel, lane, v);
            const UpdateWeights<1> uw(pw, W::kChunk - 16 * sub, BACK, p.weight_update, lane);
            state_update<T, D>(S, at.k, v, uw.w[0], sub, lane, last && p.kept);
        }
        lds_barrier();
        ro.store(c, true, walk.chunks, walk.lead, at.o);
    }
    if (last && p.s_end) S.store(p.s_end + (int64_t)task.bh * D * D, panel, lane);
}

template <typename T, int D, bool BACK, bool NT> __device__ __forceinline__ void walk_segment(const WalkArgs &a, const WalkProblem &p, const WalkTask &task, unsigned char *lds)
{
    using W = WalkShape<T, D>;
    const WalkLds<T, D> at(lds);
    unsigned char *const tileQ = at.q, *const tileK = at.k, *const tileV = at.v, *const tileO = at.o;
    Oct<T> *const scores = at.scores;
    float *const table = at.table, *const from_state = at.from_state;
    constexpr int kPieces = W::kPieces;
    const int b = task.bh / a.H, h = task.bh % a.H, own_lane = threadIdx.x & 63, panel = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const float g = a.log_decay[h];
    const DecayWalk walk(walk_length(a, b), W::kChunk);
    const int c0 = task.segment * a.per_segment;
    int c1 = c0 + a.per_segment;
    const bool last = c1 >= walk.chunks;
    if (c1 > walk.chunks) c1 = walk.chunks;
    if (c0 >= c1 && task.segment > 0) return;
    // the first tokens and the state are on their way while the powers are worked out
    const ChunkRows<T, D, BACK> rq(p.q, p.sq, b, h), rk(p.k, p.sk, b, h), rv(p.v, p.sv, b, h), ro(p.o, p.so, b, h);
    u32x4 nq[W::kSteps], nk[W::kSteps], nv[W::kSteps];
    rq.template load<NT, true>(c0, c0 < c1, walk.chunks, walk.lead, nq);
    rk.template load<NT, true>(c0, c0 < c1, walk.chunks, walk.lead, nk);
    rv.template load<NT, true>(c0, c0 < c1, walk.chunks, walk.lead, nv);
    const float *begin = begin_of<D>(a, p, task, walk.chunks);
    StatePanel<D> S;
    if (begin) S.load(begin, p.turned, panel, own_lane);
    else S.clear();
    const bool keep = last && p.s_end, fine = last && p.kept;        // this workgroup's state is the sequence's last

    const DecayPower pw(g);
    const UpdateWeights<W::kTokSubs> uw(pw, W::kChunk, BACK, p.weight_update, own_lane);
    const ChunkDecay decay(W::kChunk, g);
    const float first_decay = pw.uniform(W::kChunk - walk.lead);     // the first chunk of a sequence holds `lead` tokens fewer
    // a row's weight on what comes out of the state, whole chunks and the first one
    for (int i = threadIdx.x; i < W::kChunk; i += W::kWalkThreads) {
        const int e = i + 1 - (int)BACK;
        from_state[i] = held(p.weight_state * pw(e));
        from_state[64 + i] = held(p.weight_state * pw(e < walk.lead ? 0 : e - walk.lead));
    }
    // weights of the scores by distance: table[63 - distance], zeros where the row lies behind.  Row 32 it + col and row 32 jt + 16 s + 8 half
    // + e are 32 (it - jt) + col - 16 s - 8 half - e apart.  In LDS: sixteen registers that every chunk needs for a moment only.
    for (int i = threadIdx.x; i < 96; i += W::kWalkThreads) table[i] = i < 64 ? held(p.weight_chunk * pw(63 - i)) : 0.f;

    for (int c = c0; c < c1; ++c) {
        lds_barrier();
        ro.store(c - 1, c > c0, walk.chunks, walk.lead, tileO);
        rq.put(tileQ, nq);
        rk.put(tileK, nk);
        rv.put(tileV, nv);
        lds_barrier();
        rq.template load<NT, false>(c + 1, c + 1 < c1, walk.chunks, walk.lead, nq);
        rk.template load<NT, false>(c + 1, c + 1 < c1, walk.chunks, walk.lead, nk);
        rv.template load<NT, false>(c + 1, c + 1 < c1, walk.chunks, walk.lead, nv);
        // addresses are worked out anew for every chunk: kept over the loop they take the registers that the products need
        int lane = own_lane;
        asm volatile("" : "+v"(lane));
        const int half = lane >> 5, col = lane & 31;
        const float *distance = table + 31 - col + 8 * half;
        // Scores P[jt, it] (rows jt, in decay_row's order, x rows it), weighted, as operands, and acc[it]: the output of rows it (value features x
        // tokens) from the state.  SHARED: each tile of the scores is one wave's work (another one's with every chunk) for all waves, through LDS,
        // in one run over the features with the products of the state; otherwise every wave has its own, worked out before.
        f32x16 acc[W::kTiles];
        Oct<T> own[W::kOwnTiles][2][kPieces];
        auto weigh = [&](const f32x16 &p, const float *near, Oct<T> (&o)[2][kPieces]) __attribute__((always_inline)) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = p[8 * s + e] * near[16 * s + e];
                if constexpr (kPieces == 2) {
                    const Pieces<T> both(x);
                    o[s][0] = both.hi;
                    o[s][1] = both.lo;
                } else {
                    oct_from(x, o[s][0]);
                }
            }
        };
        f32x16 part;                                                   // kSplit: this wave's sum over its features
        if constexpr (W::kSplit) {
#pragma unroll
            for (int r = 0; r < 16; ++r) part[r] = 0.f;
#pragma unroll
            for (int i = 0; i < (W::kSubs + W::kPanels - 1) / W::kPanels; ++i) {
                const int sub = panel + i * W::kPanels, at = (16 * sub + 8 * half) * (int)sizeof(T);
                if (sub < W::kSubs) {
                    Oct<T> q, k;
                    row_operand(tileQ + col * W::kRowBytes + at, q);
                    row_operand(tileK + decay_row(col) * W::kRowBytes + at, k);
                    part = oct_product(k, q, part);
                }
            }
        } else if constexpr (!W::kShared) {
            f32x16 P[W::kScoreTiles];
#pragma unroll
            for (int t = 0; t < W::kScoreTiles; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) P[t][r] = 0.f;
#pragma unroll
            for (int sub = 0; sub < W::kSubs; ++sub) {
                const int at = (16 * sub + 8 * half) * (int)sizeof(T);
                Oct<T> q[W::kTiles], k[W::kTiles];
#pragma unroll
                for (int t = 0; t < W::kTiles; ++t) {
                    row_operand(tileQ + (32 * t + col) * W::kRowBytes + at, q[t]);
                    row_operand(tileK + (32 * t + decay_row(col)) * W::kRowBytes + at, k[t]);
                }
                P[0] = oct_product(k[0], q[0], P[0]);
                if constexpr (W::kTiles == 2) {
                    P[1] = oct_product(k[0], q[1], P[1]);
                    P[2] = oct_product(k[1], q[1], P[2]);
                }
            }
#pragma unroll
            for (int t = 0; t < W::kScoreTiles; ++t) weigh(P[t], distance + (t == 1 ? 0 : 32), own[t]);
#pragma unroll
            for (int t = 0; t < W::kScoreTiles; ++t)
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int x = 0; x < kPieces; ++x) settle(own[t][s][x]);
        }
        // the tile that is this wave's (SHARED): none from kScoreTiles on, which is worked out all the same to keep the run free of branches
        f32x16 P;
        const int mine = (panel + c) % W::kPanels;
        const int my_j = W::kTiles == 2 && mine >= 2, my_i = W::kTiles == 2 && mine >= 1;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            P[r] = 0.f;
#pragma unroll
            for (int it = 0; it < W::kTiles; ++it) acc[it][r] = 0.f;
        }
#pragma unroll
        for (int sub = 0; sub < W::kSubs; ++sub) {
            const int at = (16 * sub + 8 * half) * (int)sizeof(T);
            Oct<T> q[W::kTiles];
#pragma unroll
            for (int t = 0; t < W::kTiles; ++t) row_operand(tileQ + (32 * t + col) * W::kRowBytes + at, q[t]);
            if constexpr (W::kShared) {
                Oct<T> k, mq;
                row_operand(tileK + (32 * my_j + decay_row(col)) * W::kRowBytes + at, k);
                row_operand(tileQ + (32 * my_i + col) * W::kRowBytes + at, mq);
                P = oct_product(k, mq, P);
            }
            float x[8];
            S.eight(sub, x);
            const Pieces<T> s(x);
#pragma unroll
            for (int t = 0; t < W::kTiles; ++t) acc[t] = s.first(q[t], acc[t]);
#pragma unroll
            for (int t = 0; t < W::kTiles; ++t) acc[t] = s.second(q[t], acc[t]);
        }
        if constexpr (W::kShared) {
            if (mine < W::kScoreTiles) {
                weigh(P, distance + (mine == 1 ? 0 : 32), own[0]);
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int x = 0; x < kPieces; ++x) scores[((2 * mine + s) * kPieces + x) * 64 + lane] = own[0][s][x];
            }
            lds_barrier();
        }
        if constexpr (W::kSplit) {
            // the parts are added up in the panels' order, in the room of the queries, which are done with
            f32x4 *parts = reinterpret_cast<f32x4 *>(tileQ);
            static_assert(W::kPanels * 4096 <= W::kTileBytes, "sixteen floats of each lane");
            lds_barrier();
#pragma unroll
            for (int x = 0; x < 4; ++x) parts[(panel * 4 + x) * 64 + lane] = f32x4{part[4 * x], part[4 * x + 1], part[4 * x + 2], part[4 * x + 3]};
            lds_barrier();
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                f32x4 sum = parts[x * 64 + lane];
#pragma unroll
                for (int w = 1; w < W::kPanels; ++w) sum += parts[(w * 4 + x) * 64 + lane];
#pragma unroll
                for (int e = 0; e < 4; ++e) part[4 * x + e] = sum[e];
            }
            weigh(part, distance + 32, own[0]);
        }
#pragma unroll
        for (int it = 0; it < W::kTiles; ++it) {
            const float weight = from_state[(c == 0 ? 64 : 0) + 32 * it + col];
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[it][r] *= weight;
        }
        // from the chunk itself, and the chunk into the state
        S.scale(c == 0 ? first_decay : decay(c));
#pragma unroll
        for (int sub = 0; sub < W::kTokSubs; ++sub) {
            Oct<T> v;
            token_operand<W, false>(tileV, 16 * sub, 32 * panel, lane, v);
            auto weights = [&](int t, int s, int x) __attribute__((always_inline)) {
                return W::kShared ? scores[((2 * t + s) * kPieces + x) * 64 + lane] : own[W::kShared ? 0 : t][s][x];
            };
#pragma unroll
            for (int x = 0; x < kPieces; ++x) {
                if (sub < 2) acc[0] = oct_product(v, weights(0, sub, x), acc[0]);
                if constexpr (W::kTiles == 2) acc[1] = oct_product(v, weights(1 + sub / 2, sub % 2, x), acc[1]);
            }
            state_update<T, D>(S, tileK, v, uw.w[sub], sub, lane, fine);
        }
        // the output's rows, for whole-row stores once all panels are in
#pragma unroll
        for (int it = 0; it < W::kTiles; ++it) put_features<W>(tileO + (32 * it + col) * W::kRowBytes + 32 * panel * (int)sizeof(T), acc[it], half, T{});
    }
    // a token that is no number leaves its trace in the state
    const bool clean = __all(S.finite());
    if (own_lane == 0) at.votes[panel] = clean;
    lds_barrier();
    if (c0 < c1) ro.store(c1 - 1, true, walk.chunks, walk.lead, tileO);
    int all = 1;
#pragma unroll
    for (int w = 0; w < W::kPanels; ++w) all &= at.votes[w];
    if (__builtin_amdgcn_readfirstlane(all) || c0 >= c1) {
        if (keep) S.store(p.s_end + (int64_t)task.bh * D * D, panel, own_lane);
    } else {
        WalkTask same = task;                                          // nothing of the walk is kept for this
        asm volatile("" : "+s"(same.bh), "+s"(same.segment));
        walk_again<T, D, BACK>(a, p, same, lds);
    }
}
// NT: tokens are read past the caches.
template <typename T, int D, bool NT> __global__ __launch_bounds__((WalkShape<T, D>::kWalkThreads), 2) void decay_walk(WalkArgs a)
{
    using W = WalkShape<T, D>;
    __shared__ __align__(16) unsigned char lds[W::kTilesInLds * W::kTileBytes + W::kScoreBytes + kDecayTableBytes];
    const int BH = a.B * a.H;
    const WalkTask task(a.problems * BH * a.segments, BH, a.segments, a.together);
    if (!task.any) return;
    const WalkProblem &p = a.p[task.problem];
    if (p.back) walk_segment<T, D, true, NT>(a, p, task, lds);
    else walk_segment<T, D, false, NT>(a, p, task, lds);
}

}  // namespace sv
