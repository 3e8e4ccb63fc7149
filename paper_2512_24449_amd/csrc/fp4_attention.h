// Attention over the 4-bit paged cache, one pass with the running maximum and sum of a softmax.
//
// Scores are computed transposed: S^T = K Q^T (rows: tokens, columns: the query heads of a kv-head, of one or several new
// rows), then O^T = V^T P^T.  A lane then holds scores, weights and outputs of one column only, so maximum and sum are the
// lane's own (joined over the four lanes of a column), and the layout in which the matrix cores leave S^T is the one in which
// they take P^T: nothing passes through LDS or other lanes between the two products.  Which 32 tokens a step's rows stand
// for is free as long as both products agree; row 4g + i of the first (second) product of 16 is token 8g + i (8g + 4 + i), so
// that a lane's eight weights are eight consecutive tokens: a word of V.
//
// K and V enter as fp16 (K as bf16 where q is): E2M1 numbers with scales 2^-23 .. 2^13 are exact there.
#pragma once

#include <algorithm>
#include <cfloat>
#include <cmath>

#include "fp4.h"
#include "last_group.h"

namespace packkv {


typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf162_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf168_t __attribute__((ext_vector_type(8)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef uint32_t uint4_t __attribute__((ext_vector_type(4)));

constexpr int FP4_STEP = 32;             // tokens of a step of the streaming kernel: half a page
constexpr int FP4_COLUMNS = 16;          // of a product; of a block of the streaming kernel
constexpr int FP4_TILE_COLUMNS = 128;    // of a block of the tile kernel, whose steps are pages
// Weights are relative to a maximum that follows the scores only when one is P_SLACK (in powers of two) above it: most steps
// scale no sums then.  They are held as 2^P_LIFT times their size, so that the largest is between 2^12 and 2^15, and fp16
// keeps its eleven bits down to 2^-26 of it.
constexpr float P_LIFT = 12.0f, P_SLACK = 3.0f;
// How the maximum m is subtracted: up to |m * scale| of P_FAR in the exponential's argument, one instruction to a score,
// s * scale + (P_LIFT - m * scale), whose bracket is rounded to 2^-13 at most; beyond, where that rounding would come to be whole powers
// of two, from the score: (s - m) * scale + P_LIFT, for the waves that have such a column.
constexpr float P_FAR = 2048.0f;
// The workspace: a counter byte for each of so many (stream, sequence) pairs whose splits are joined by the last workgroup
// of them, and partial results, at most so many rows (of a column in a split) of HD + 4 floats.
constexpr int FP4_COUNTERS = 4096;
constexpr int64_t FP4_PART_ROWS = 65536;
constexpr int FP4_SPLITS_MAX = 256;
// Sequences that share workgroups by their lengths.
constexpr int FP4_FLAT = 64;
// Steps that a split has at least: two to a wave in a call of few workgroups, else three.  Passes with two and with three: one
// head x 1000 tokens 7.8 / 8.5 us, 32 heads x 4100 14.8 / 13.2, a window of 4096 of 8 kv-heads 10.0 / 9.6.
constexpr int FP4_LEAST_STEPS = 8, FP4_MORE_STEPS = 12;
constexpr int64_t FP4_FEW_GROUPS = 128;
constexpr int FP4_LEAST_PAGES = 4;       // the same, of the tile kernel
// Steps of a split that more workgroups than fit at once may have: then its start costs little.
constexpr int FP4_LONG_STEPS = 64;

// sm_scale * log2(e) as the kernels use it.  A negative scale is one of -q: the largest scaled score is then that of the
// largest score.  With 0 all tokens that are seen weigh the same: q is taken as 0 then and the scale as 1 (0 times -infinity, the
// score of a token that is not seen, would be a NaN).
struct Fp4Scale {
    float scale, slack;      // slack: P_SLACK / scale
    uint32_t sign;           // of two fp16 or bf16 values of q
    bool zero;
    static Fp4Scale of(float s) {
        const float size = s == 0.0f ? 1.0f : std::fabs(s);
        return {size, std::fmin(P_SLACK / size, FLT_MAX), s < 0.0f ? 0x80008000u : 0u, s == 0.0f};
    }
    // q as an operand, but for its sign: an infinity as the NaN that it makes of its row (whose scores may all be -infinity, and are
    // then told from those of a row that sees nothing), and what is finite as 0 where the scale is.
    template <bool BF16, int N>
    __device__ inline void settle(uint4_t (&q)[N]) const {
        constexpr uint32_t INFINITE = BF16 ? 0x7F80u : 0x7C00u;
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 4 * N; ++i) m = max16(m, q[i / 4][i % 4] & 0x7FFF7FFFu);
        if (__builtin_expect(!zero && !__any(max(m & 0xFFFFu, m >> 16) >= INFINITE), true)) return;
#pragma unroll
        for (int i = 0; i < 4 * N; ++i) {
            const uint32_t x = q[i / 4][i % 4], finite = zero ? 0u : x;
            q[i / 4][i % 4] = ((x & 0x7FFFu) >= INFINITE ? 0x7FFFu : finite & 0xFFFFu) |
                              (((x >> 16) & 0x7FFFu) >= INFINITE ? 0x7FFF0000u : finite & 0xFFFF0000u);
        }
    }
};

struct Fp4Attention {
    Fp4View v;
    const uint16_t *q;
    int64_t q_stride;
    Fp4Scale scale;
    int window, sinks;
    void *out;
    int out_type;
    float *lse;
    float *part;             // partial results: HD sums, maximum and sum of the weights
    uint8_t *counters;       // not null: the last workgroup of a sequence joins its splits
    int width, blocks;       // columns of a block, blocks; a stream is a block of a kv-head
    int rows;                // columns of a block with partial results: all, or what max_new has
    int least_steps;         // of a split
    int few;                 // splits of all sequences that share, where those have FP4_LONG_STEPS or fewer
    int most_splits;         // of a sequence
    bool flat;               // the workgroups of 64 sequences of a stream go to them by their lengths; else each has as many
    int splits;              // workgroups of those; or of a stream and sequence

    __device__ inline int64_t part_row(uint32_t stream, int b, int first, int column) const {   // of the first split
        const int64_t streams = int64_t(blocks) * v.H, at = flat ? (b / FP4_FLAT * streams + stream) * splits + first : (b * streams + stream) * splits;
        return at * rows + column;
    }
};

// A word of a row of K (eight channels of a token) as an operand.
template <bool BF16>
__device__ inline uint4_t row_operand(uint32_t w, float scale) {
    if constexpr (BF16)
        return uint4_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)),
                       __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
                       __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)),
                       __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3))};
    else
        return uint4_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 0)),
                       __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 1)),
                       __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 2)),
                       __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 3))};
}

template <bool BF16>
__device__ inline float4_t product16(uint4_t a, uint4_t b, float4_t c) {
    if constexpr (BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf168_t, a), __builtin_bit_cast(bf168_t, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
}

// The scales of eight tokens (bytes e + 127) as fp16 pairs.
__device__ inline void scale_pairs(uint2 bytes, half2_t (&out)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t two = (i < 2 ? bytes.x : bytes.y) >> (16 * (i & 1));
        out[i] = __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_pkrtz(__uint_as_float((two & 255u) << 23),
                                                                         __uint_as_float(((two >> 8) & 255u) << 23)));
    }
}

// A word of V (one channel of eight tokens) with the tokens' scales.
__device__ inline uint4_t column_operand(uint32_t w, const half2_t (&scale)[4]) {
    uint4_t r;
    r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 0) * scale[0]);
    r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 1) * scale[1]);
    r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 2) * scale[2]);
    r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 3) * scale[3]);
    return r;
}

// Maximum and sum over the four lanes of a column (lane, lane ^ 16, lane ^ 32, lane ^ 48).
__device__ inline float column_max(float x) {
    uint32_t a = __float_as_uint(x), b = a;
    swap_rows16(a, b);
    x = fmaxf(__uint_as_float(a), __uint_as_float(b));
    a = b = __float_as_uint(x);
    swap_rows32(a, b);
    return fmaxf(__uint_as_float(a), __uint_as_float(b));
}

__device__ inline float column_sum(float x) {
    uint32_t a = __float_as_uint(x), b = a;
    swap_rows16(a, b);
    x = __uint_as_float(a) + __uint_as_float(b);
    a = b = __float_as_uint(x);
    swap_rows32(a, b);
    return __uint_as_float(a) + __uint_as_float(b);
}

// The largest of three, a NaN if one is: one instruction, and the compiler's own, so that it waits for the matrix products whose
// results these are (inline assembly would read them whenever it comes).  fmaxf would quiet signalling NaNs first.
__device__ inline float max3(float a, float b, float c) {
    return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}

// The weight of a maximum a relative to b; -inf relative to -inf: none.
__device__ inline float weight_of(float a, float b, float scale) { return b == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((a - b) * scale); }

// The natural logarithm of a sum of weights l (2^P_LIFT times their size) relative to the maximum m.
__device__ inline float log_sum(float m, float l, float scale) {
    return l > 0.0f || l != l ? (m * scale - P_LIFT + __log2f(l)) * 0.6931471805599453f : -INFINITY;
}

template <int N>
__device__ inline void store_out(void *out, int type, int64_t at, const float (&x)[N]) {
    if (type == KV_TYPE_FP32) {
#pragma unroll
        for (int i = 0; i < N; i += 4)
            *reinterpret_cast<float4 *>(static_cast<float *>(out) + at + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
        return;
    }
    uint32_t w[N / 2];
#pragma unroll
    for (int i = 0; i < N; i += 2)
        w[i / 2] = type == KV_TYPE_BF16 ? __builtin_bit_cast(uint32_t, bf162_t{__bf16(x[i]), __bf16(x[i + 1])})
                                        : __builtin_bit_cast(uint32_t, half2_t{_Float16(x[i]), _Float16(x[i + 1])});
#pragma unroll
    for (int i = 0; i < N / 2; i += 2)
        *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(out) + at + 2 * i) = make_uint2(w[i], w[i + 1]);
}

// The tokens that a block of columns sees, in steps of UNIT (32 or 64): those that hold first tokens, then those from the window's
// start to the last row.
template <int UNIT>
struct Fp4Steps {
    int first_row, last_row;   // new rows of the block
    int end;                   // tokens from here on are seen by none
    int begin;                 // nor are those below, but for the first ones
    int sink_steps, window_step, n;
    __device__ inline Fp4Steps(const Fp4Sequence &seq, int column0, int columns, int G, int window, int sinks) {
        const int pos0 = seq.pos0, rows = seq.n;
        first_row = column0 / G;
        last_row = min((column0 + columns - 1) / G, rows - 1);
        end = min(pos0 + last_row + 1, seq.held);
        begin = window ? max(max(pos0 + first_row, 0) - window + 1, 0) : 0;
        window_step = begin / UNIT;
        sink_steps = min((min(window ? sinks : 0, max(end, 0)) + UNIT - 1) / UNIT, window_step);
        n = end > 0 && first_row < rows ? sink_steps + max((end + UNIT - 1) / UNIT - window_step, 0) : 0;
    }
    __device__ inline int token(int step) const { return UNIT * (step < sink_steps ? step : step - sink_steps + window_step); }
};

// A column of a wave's matrix products: its running softmax and its sums.
template <int HD>
struct Fp4Column {
    static constexpr int OT = HD / 16;
    float4_t o[OT];
    float l;                 // sum of this lane's weights
    // The score that the weights are relative to, and P_LIFT less it times the scale.  Beyond P_FAR, and before the first score, m is
    // -inf, so that every score seen is above it, and `lift` the score.
    float m, lift;
    int hi;                  // last token that the column sees

    __device__ inline void clear() {
#pragma unroll
        for (int i = 0; i < OT; ++i) o[i] = float4_t{0, 0, 0, 0};
        l = 0.0f;
        m = lift = -INFINITY;
    }
    __device__ inline float largest() const { return m == -INFINITY ? lift : m; }
    // Scores of T / 2 times eight tokens, the first from t8 on, the next 32 further: those that the column does not see count
    // nothing.
    template <int T>
    __device__ inline void mask(float4_t (&s)[T], int t8, int end, int window, int sinks) const {
        const int lo = window ? hi - window + 1 : 0;
#pragma unroll
        for (int i = 0; i < 4 * T; ++i) {
            const int t = t8 + 32 * (i >> 3) + (i & 7);
            s[i >> 2][i & 3] = (t <= hi) & (t < end) & ((t >= lo) | (t < sinks)) ? s[i >> 2][i & 3] : -INFINITY;
        }
    }
    // The tokens' weights as operands.
    template <int T>
    __device__ inline void weigh(float4_t (&s)[T], const Fp4Scale &scale, uint4_t (&p)[T / 2]) {
        float top = max3(s[0][0], s[0][1], s[0][2]);
#pragma unroll
        for (int i = 3; i + 1 < 4 * T; i += 2) top = max3(top, s[i >> 2][i & 3], s[(i + 1) >> 2][(i + 1) & 3]);
        top = __builtin_elementwise_maximum(top, s[T - 1][3]);
        float add = lift;
        if (__any(top - m > scale.slack)) {
            top = column_max(top);
            float now = largest();
            if (top - now > scale.slack) {
                const float f = now == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((now - top) * scale.scale);
#pragma unroll
                for (int i = 0; i < OT; ++i) o[i] *= f;
                l *= f;
                now = top;
            }
            m = now, add = lift = fmaf(-now, scale.scale, P_LIFT);
            const bool far = !(fabsf(lift) <= P_FAR);   // (of the column: others of the wave weigh as they would without it)
            if (__builtin_expect(__any(far), false)) {
                const float base = far ? fmaxf(now, -FLT_MAX) : 0.0f;   // (no score so far: nothing to subtract)
#pragma unroll
                for (int i = 0; i < T; ++i) s[i] -= base;
                if (far) m = -INFINITY, lift = now, add = P_LIFT;
            }
        }
#pragma unroll
        for (int i = 0; i < 2 * T; ++i) {
            const float x = __builtin_amdgcn_exp2f(fmaf(s[i >> 1][2 * (i & 1)], scale.scale, add));
            const float y = __builtin_amdgcn_exp2f(fmaf(s[i >> 1][2 * (i & 1) + 1], scale.scale, add));
            l += x + y;
            p[i >> 2][i & 3] = __builtin_bit_cast(uint32_t, half2_t{_Float16(x), _Float16(y)});
        }
    }
};

// Scales (a byte each) of the lane's eight tokens: of one that no row sees, which may be any bits, 0 -- no infinity times a weight
// of 0.
__device__ inline uint2 seen_scales(uint2 bytes, int t8, int begin, int end, int sinks) {
    uint32_t keep[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int t = t8 + i;
        keep[i >> 2] |= (t < end) & ((t >= begin) | (t < sinks)) ? 255u << (8 * (i & 3)) : 0u;
    }
    return make_uint2(bytes.x & keep[0], bytes.y & keep[1]);
}

// Which sequence a workgroup works for, and which of how many splits of its steps.  Flat: the workgroups of 64 sequences of
// a stream are shared out so that none has more steps than some U >= all steps / (workgroups - sequences): the sum of
// ceil(steps / U) is then at most the workgroups, and a long sequence among short ones has more of them.  Every wave finds
// the shares by itself, a sequence to a lane.  Else a sequence has the workgroups to itself, and again takes as many as U says.
template <int UNIT>
struct Fp4Share {
    int b, split, splits;    // splits 0: no work
    int first;               // flat: the sequence's first workgroup among those of the 64

    // U and ceil(steps / U), with quotients in fp32: U is too large rather than too small, the splits are then exact
    static __device__ inline uint32_t steps_of_split(const Fp4Attention &a, float all, int room) {
        const auto over = [&](int n) { return uint32_t(all * __builtin_amdgcn_rcpf(float(n)) * (1.0f + 0x1p-20f)) + 1; };
        return max(max(over(room), min(over(a.few), uint32_t(FP4_LONG_STEPS))), uint32_t(a.least_steps));
    }
    static __device__ inline int splits_of(const Fp4Attention &a, uint32_t steps, uint32_t of_split) {
        // (the quotient is below 2^11, or the splits below are the most: off by one at most)
        uint32_t q = uint32_t(float(steps) * __builtin_amdgcn_rcpf(float(of_split)));
        q = q * of_split < steps ? q + 1 : q;
        return min(int(q * of_split < steps ? q + 1 : q), a.most_splits);
    }

    // For workgroup `group` of sequence (or 64 sequences) `chunk`, or, group -1, for sequence `sequence`.
    __device__ inline Fp4Sequence find(const Fp4Attention &a, int chunk, int group, int sequence, int column0, int lane) {
        const kv_fp4_batch_t &t = a.v.batch;
        if (!a.flat) {
            b = chunk, split = group, first = 0;
            const Fp4Sequence seq(a.v, b);
            const uint32_t steps = column0 < seq.n * a.v.G ? max(Fp4Steps<UNIT>(seq, column0, a.width, a.v.G, a.window, a.sinks).n, 1) : 0;
            splits = splits_of(a, steps, steps_of_split(a, float(steps), a.splits));
            if (group >= splits) splits = 0;
            return seq;
        }
        const int b0 = FP4_FLAT * chunk, here = min(t.batch - b0, FP4_FLAT);
        uint32_t steps = 0;
        int len = 0, rows = 0, row0 = 0;
        if (lane < here) {
            len = t.lens[b0 + lane], rows = Fp4Sequence::raw_rows(a.v, b0 + lane), row0 = Fp4Sequence::raw_first(a.v, b0 + lane);
            const Fp4Sequence seq(a.v, b0 + lane, len, rows, row0);
            // (a row that sees nothing is written, too)
            if (column0 < seq.n * a.v.G) steps = max(Fp4Steps<UNIT>(seq, column0, a.width, a.v.G, a.window, a.sinks).n, 1);
        }
        const float all = float(uint32_t(__builtin_amdgcn_readlane(wave_inclusive_scan(int(steps)), 63)));   // at most 64 * 2^25
        const int mine = splits_of(a, steps, steps_of_split(a, all, a.splits - here)), before = wave_inclusive_scan(mine) - mine;
        int at = sequence - b0;
        if (group >= 0) {
            const uint64_t has = __ballot(before <= group && group < before + mine);
            at = has ? __builtin_ctzll(has) : 0;
        }
        b = b0 + at;
        splits = __builtin_amdgcn_readlane(mine, at);
        first = __builtin_amdgcn_readlane(before, at);
        split = group - first;
        if (group >= 0 && uint32_t(split) >= uint32_t(splits)) splits = 0;
        return Fp4Sequence(a.v, b, __builtin_amdgcn_readlane(len, at), __builtin_amdgcn_readlane(rows, at),
                           __builtin_amdgcn_readlane(row0, at));
    }
};

int launch_fp4_tiles(const Fp4Attention &a, dim3 grid, int head_dim, bool bf16, hipStream_t s);

}  // namespace packkv
