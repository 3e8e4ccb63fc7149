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
#include <algorithm>

#include "fp4.h"
#include "last_group.h"

namespace packkv {

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf162_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf168_t __attribute__((ext_vector_type(8)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef uint32_t uint4_t __attribute__((ext_vector_type(4)));

constexpr int FP4_STEP = 32;             // tokens of a step: half a page
constexpr int FP4_COLUMNS = 16;
// Weights are relative to a maximum that follows the scores only when one is P_SLACK (in powers of two) above it: most steps
// scale no sums then.  They are held as 2^P_LIFT times their size, so that the largest is between 2^12 and 2^15, and fp16
// keeps its eleven bits down to 2^-26 of it.
constexpr float P_LIFT = 12.0f, P_SLACK = 3.0f;
// The workspace: a counter byte for each of so many (stream, sequence) pairs whose splits are joined by the last workgroup
// of them, and partial results, at most so many rows (of a column in a split) of HD + 4 floats.
constexpr int FP4_COUNTERS = 4096;
constexpr int64_t FP4_PART_ROWS = 32768;
constexpr int FP4_SPLITS_MAX = 256;
// Sequences that share workgroups by their lengths.
constexpr int FP4_FLAT = 64;
// Steps that a split has at least: two to a wave in a call of few workgroups, else three.  Passes with two and with three: one
// head x 1000 tokens 7.8 / 8.5 us, 32 heads x 4100 14.8 / 13.2, a window of 4096 of 8 kv-heads 10.0 / 9.6.
constexpr int FP4_LEAST_STEPS = 8, FP4_MORE_STEPS = 12;
constexpr int64_t FP4_FEW_GROUPS = 128;

size_t fp4_workspace_bytes(int head_dim) { return FP4_COUNTERS + size_t(FP4_PART_ROWS) * (head_dim + 4) * sizeof(float); }

struct Fp4Attention {
    Fp4View v;
    const uint16_t *q;
    int64_t q_stride;
    float scale;             // sm_scale * log2(e)
    int window, sinks;
    void *out;
    int out_type;
    float *lse;
    float *part;             // partial results: HD sums, maximum and sum of the weights
    uint8_t *counters;       // not null: the last workgroup of a sequence joins its splits
    int blocks;              // column blocks; a stream is one of them of a kv-head
    int rows;                // columns of a block with partial results: all, or what max_new has
    int least_steps;         // of a split (flat)
    bool flat;               // the workgroups of 64 sequences of a stream go to them by their lengths; else each has as many
    int splits;              // workgroups of those; or of a stream and sequence

    __device__ inline int64_t part_row(uint32_t stream, int b, int first, int column) const {   // of the first split
        const int64_t streams = int64_t(blocks) * v.H, at = flat ? (b / FP4_FLAT * streams + stream) * splits + first : (b * streams + stream) * splits;
        return at * rows + column;
    }
};

// Four words of a row (32 values' codes, HD / 4 of a lane) as operands: value pairs in the order of the channels.
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

__device__ inline float max3(float a, float b, float c) {   // (without the instructions that quiet a signalling NaN first)
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// exp2(a - b) where -inf - -inf means no weight.
__device__ inline float weight_of(float a, float b) { return b == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(a - b); }

// The natural logarithm of a sum of weights l (2^P_LIFT times their size) relative to the maximum m.
__device__ inline float log_sum(float m, float l) {
    return l > 0.0f || l != l ? (m - P_LIFT + __log2f(l)) * 0.6931471805599453f : -INFINITY;
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

// The tokens that a block of columns sees, in steps of 32: those that hold first tokens, then those from the window's
// start to the last row.
struct Fp4Steps {
    int first_row, last_row;   // new rows of the block
    int end;                   // tokens from here on are seen by none
    int begin;                 // nor are those below, but for the first ones
    int sink_steps, window_step, n;
    __device__ inline Fp4Steps(const Fp4Sequence &seq, int column0, int G, int window, int sinks) {
        const int pos0 = seq.pos0, rows = seq.n;
        first_row = column0 / G;
        last_row = min((column0 + FP4_COLUMNS - 1) / G, rows - 1);
        end = min(pos0 + last_row + 1, seq.held);
        begin = window ? max(max(pos0 + first_row, 0) - window + 1, 0) : 0;
        window_step = begin / FP4_STEP;
        sink_steps = min((min(window ? sinks : 0, max(end, 0)) + FP4_STEP - 1) / FP4_STEP, window_step);
        n = end > 0 && first_row < rows ? sink_steps + max((end + FP4_STEP - 1) / FP4_STEP - window_step, 0) : 0;
    }
    __device__ inline int token(int step) const { return FP4_STEP * (step < sink_steps ? step : step - sink_steps + window_step); }
};

// What a wave reads of a step: of K a lane's quarter of two tokens' rows, of V a word (or HD / 64 times four) of eight tokens.
template <int HD>
struct Fp4Stage {
    using P = Fp4Block<HD>;
    static constexpr int KW = HD / 32, VH = HD / 64;
    uint32_t k[2][KW];
    uint4 v[VH];
    uint32_t ks[2];
    uint2 vs[VH];
    int t0, end;             // first token; tokens from `end` on are not there (0: the page is missing)

    // block: the head's in the page; at: the step's first token in it
    __device__ inline void load(const uint8_t *block, int at, int c16, int g) {
        const uint8_t *kp = block + P::K + at * (HD / 2), *sp = block + P::KS + at * (HD / FP4_GROUP);
        const int token = 8 * (c16 >> 2) + (c16 & 3);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            if constexpr (KW == 4) {
                const uint4 x = *reinterpret_cast<const uint4 *>(kp + (token + 4 * t) * (HD / 2) + g * (HD / 8));
                k[t][0] = x.x, k[t][1] = x.y, k[t][2] = x.z, k[t][3] = x.w;
            } else {
                const uint2 x = *reinterpret_cast<const uint2 *>(kp + (token + 4 * t) * (HD / 2) + g * (HD / 8));
                k[t][0] = x.x, k[t][1] = x.y;
            }
            ks[t] = sp[(token + 4 * t) * (HD / FP4_GROUP) + g * (HD / 4) / FP4_GROUP];
        }
        const uint8_t *vp = block + P::V + at * (HD / 2), *wp = block + P::VS + at;
#pragma unroll
        for (int x = 0; x < VH; ++x) {
            // channels 64 x + 4 c16 .. of tokens at + 8g ..
            v[x] = *reinterpret_cast<const uint4 *>(vp + (g * HD + 64 * x + 4 * c16) * 4);
            vs[x] = *reinterpret_cast<const uint2 *>(wp + (2 * x + (c16 >> 3)) * FP4_PAGE + 8 * g);
        }
    }
};

// The columns of a wave's matrix products, its running softmax and its sums.
template <int HD, bool BF16>
struct Fp4Columns {
    static constexpr int KW = HD / 32, VH = HD / 64, OT = HD / 16;
    uint4_t q[KW];
    float4_t o[OT];
    float l, m, bar, lift;   // sum of this lane's weights; what the weights are relative to; score that moves it; P_LIFT - m * scale
    int hi, lo;              // last token that the column sees; first of its window
    float scale, slack;      // slack: P_SLACK / scale
    int sinks, begin;

    __device__ inline void clear() {
#pragma unroll
        for (int i = 0; i < OT; ++i) o[i] = float4_t{0, 0, 0, 0};
        l = 0.0f;
        m = bar = -INFINITY;
        lift = P_LIFT;
    }

    // edge (wave-uniform): there are tokens that not every column sees
    __device__ inline void step(const Fp4Stage<HD> &in, int g, bool edge) {
        float4_t s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = float4_t{0, 0, 0, 0};
            const float ks = __uint_as_float(in.ks[t] << 23);
#pragma unroll
            for (int i = 0; i < KW; ++i) s[t] = product16<BF16>(row_operand<BF16>(in.k[t][i], ks), q[i], s[t]);
        }
        uint2 vs[VH];
#pragma unroll
        for (int x = 0; x < VH; ++x) vs[x] = in.vs[x];
        if (edge) {
            uint32_t keep[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int t = in.t0 + 8 * g + i;
                const bool ok = (t <= hi) & (t < in.end) & ((t >= lo) | (t < sinks));
                s[i >> 2][i & 3] = ok ? s[i >> 2][i & 3] : -INFINITY;
                // a token that no row sees may be any bits: no infinity times a weight of 0
                const bool seen = (t < in.end) & ((t >= begin) | (t < sinks));
                keep[i >> 2] |= seen ? 255u << (8 * (i & 3)) : 0u;
            }
#pragma unroll
            for (int x = 0; x < VH; ++x) vs[x].x &= keep[0], vs[x].y &= keep[1];
        }
        float top = max3(max3(s[0][0], s[0][1], s[0][2]), max3(s[0][3], s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3]));
        if (__any(top > bar)) {
            top = column_max(top);
            if (top > bar) {
                const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - top) * scale);
#pragma unroll
                for (int i = 0; i < OT; ++i) o[i] *= f;
                l *= f;
                m = top;
                bar = top + slack;
                lift = P_LIFT - top * scale;
            }
        }
        half2_t p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = __builtin_amdgcn_exp2f(fmaf(s[i >> 1][2 * (i & 1)], scale, lift));
            const float y = __builtin_amdgcn_exp2f(fmaf(s[i >> 1][2 * (i & 1) + 1], scale, lift));
            l += x + y;
            p[i] = half2_t{_Float16(x), _Float16(y)};
        }
        const uint4_t pw = {__builtin_bit_cast(uint32_t, p[0]), __builtin_bit_cast(uint32_t, p[1]), __builtin_bit_cast(uint32_t, p[2]),
                            __builtin_bit_cast(uint32_t, p[3])};
#pragma unroll
        for (int x = 0; x < VH; ++x) {
            half2_t scales[4];
            scale_pairs(vs[x], scales);
            const uint32_t words[4] = {in.v[x].x, in.v[x].y, in.v[x].z, in.v[x].w};
#pragma unroll
            for (int c = 0; c < 4; ++c) o[4 * x + c] = product16<false>(column_operand(words[c], scales), pw, o[4 * x + c]);
        }
    }
};

// The page numbers of the next 64 steps of a wave, one to a lane: none of its transfers waits for the table.
struct Fp4Pages {
    int page;                // (page numbers fit 31 bits) -1: missing
    __device__ inline void load(const Fp4View &v, const Fp4Sequence &seq, const Fp4Steps &steps, int step, int end, int lane) {
        const int mine = step + 4 * lane;
        page = mine < end ? int(seq.page(v, steps.token(mine) / FP4_PAGE)) : -1;
    }
    __device__ inline int at(int i) const { return __builtin_amdgcn_readlane(page, i); }
};

// Which sequence a workgroup works for, and which of how many splits of its steps.  Flat: the workgroups of 64 sequences of
// a stream are shared out so that none has more steps than some U >= all steps / (workgroups - sequences): the sum of
// ceil(steps / U) is then at most the workgroups, and a long sequence among short ones has more of them.  Every wave finds
// the shares by itself, a sequence to a lane.
struct Fp4Share {
    int b, split, splits;    // splits 0: no work
    int first;               // flat: the sequence's first workgroup among those of the 64
    int b0, mine, before;    // the 64 sequences begin at b0; lane i: splits of sequence b0 + i, of those before it
    int len, rows, row0;     // and what the batch says of it

    __device__ inline void find(const Fp4Attention &a, int chunk, int column0, int lane) {
        const kv_fp4_batch_t &t = a.v.batch;
        b0 = FP4_FLAT * chunk;
        const int here = min(t.batch - b0, FP4_FLAT);
        uint32_t steps = 0;
        len = rows = row0 = 0;
        if (lane < here) {
            len = t.lens[b0 + lane], rows = Fp4Sequence::raw_rows(a.v, b0 + lane), row0 = Fp4Sequence::raw_first(a.v, b0 + lane);
            const Fp4Sequence seq(a.v, b0 + lane, len, rows, row0);
            // (a row that sees nothing is written, too)
            if (column0 < seq.n * a.v.G) steps = max(Fp4Steps(seq, column0, a.v.G, a.window, a.sinks).n, 1);
        }
        const float all = float(uint32_t(__builtin_amdgcn_readlane(wave_inclusive_scan(int(steps)), 63)));   // at most 64 * 2^25
        // quotients in fp32: U is too large rather than too small, the splits are then exact
        const uint32_t most = max(uint32_t(all * __builtin_amdgcn_rcpf(float(a.splits - here)) * (1.0f + 0x1p-20f)) + 1, uint32_t(a.least_steps));
        uint32_t q = uint32_t(float(steps) * __builtin_amdgcn_rcpf(float(most)));      // at most 2^8: off by one at most
        q = q * most < steps ? q + 1 : q;
        mine = int(q * most < steps ? q + 1 : q);
        before = wave_inclusive_scan(mine) - mine;
    }
    __device__ inline void of_sequence(int sequence) {
        b = sequence;
        splits = __builtin_amdgcn_readlane(mine, b - b0);
        first = __builtin_amdgcn_readlane(before, b - b0);
    }
    __device__ inline void of_group(int group) {
        const uint64_t has = __ballot(before <= group && group < before + mine);
        splits = 0;
        if (!has) return;
        of_sequence(b0 + __builtin_ctzll(has));
        split = group - first;
    }
    __device__ inline Fp4Sequence sequence(const Fp4View &v) const {
        return Fp4Sequence(v, b, __builtin_amdgcn_readlane(len, b - b0), __builtin_amdgcn_readlane(rows, b - b0),
                           __builtin_amdgcn_readlane(row0, b - b0));
    }
};

template <int HD, bool BF16>
__global__ __launch_bounds__(256, HD == 128 ? 3 : 5) void fp4_attention_kernel(Fp4Attention a) {
    using P = Fp4Block<HD>;
    constexpr int KW = HD / 32, VH = HD / 64, OT = HD / 16;
    __shared__ float lds_o[4][FP4_COLUMNS][HD + 4];
    __shared__ float lds_m[4][FP4_COLUMNS], lds_l[4][FP4_COLUMNS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c16 = lane & 15, g = lane >> 4;
    const Fp4View &v = a.v;
    __shared__ uint32_t lds_last;
    const int h = blockIdx.x, block = int(blockIdx.y), column0 = block * FP4_COLUMNS;
    const uint32_t stream = uint32_t(block) * v.H + h;
    Fp4Share share;
    // (numbers of workgroups are the slowest axis: those without work come last and leave no compute unit out)
    const int chunk = int(blockIdx.z / uint32_t(a.splits)), group = int(blockIdx.z % uint32_t(a.splits));
    if (a.flat) {
        share.find(a, chunk, column0, lane);
        share.of_group(group);
        if (share.splits == 0) return;
    } else {
        share.b = chunk, share.split = group, share.splits = a.splits, share.first = 0;
    }
    const Fp4Sequence seq = a.flat ? share.sequence(v) : Fp4Sequence(v, share.b);
    const int columns = seq.n * v.G;
    if (column0 >= columns) return;
    const Fp4Steps steps(seq, column0, v.G, a.window, a.sinks);
    const int per_split = (steps.n + share.splits - 1) / share.splits;
    const int step_end = min((share.split + 1) * per_split, steps.n);
    int step = __builtin_amdgcn_readfirstlane(share.split * per_split + wave);

    // this lane's column
    const int column = column0 + c16, row = column / v.G, head = h * v.G + column % v.G;
    const int64_t out_row = seq.first + row;
    const bool real = column < columns && out_row >= 0 && out_row < v.n_rows;
    Fp4Columns<HD, BF16> col;
    col.hi = max(seq.pos0 + row, -1), col.lo = a.window ? col.hi - a.window + 1 : 0;
    col.sinks = a.sinks, col.begin = steps.begin;
    // A negative scale is one of -q: the largest scaled score is then that of the largest score.  Scores are below 2^39, so
    // below 1e-30 all that are seen weigh the same, as with 0 (which would make a NaN of a score that is not seen).
    col.scale = fmaxf(fabsf(a.scale), 1e-30f);
    const uint32_t sign = a.scale < 0.0f ? 0x80008000u : 0u;
#pragma unroll
    for (int i = 0; i < KW; ++i) {
        col.q[i] = uint4_t{0, 0, 0, 0};
        if (real) col.q[i] = *reinterpret_cast<const uint4_t *>(a.q + out_row * a.q_stride + int64_t(head) * HD + g * (HD / 4) + 8 * i) ^ sign;
    }
    col.slack = P_SLACK / col.scale;
    col.clear();
    // a step whose tokens every column of the block sees needs no masks
    const int first_hi = max(seq.pos0 + steps.first_row, -1), last_lo = a.window ? max(seq.pos0 + steps.last_row - a.window + 1, 0) : 0;

    Fp4Stage<HD> in[2];
    Fp4Pages pages;
    auto fetch = [&](Fp4Stage<HD> &to, int at_step) {
        const int i = (at_step - step) >> 2;
        const int page = pages.at(i);
        to.t0 = steps.token(at_step);
        to.end = page < 0 ? 0 : steps.end;
        to.load(v.pages + (int64_t(max(page, 0)) * v.H + h) * size_t(P::BYTES), to.t0 % FP4_PAGE, c16, g);
    };
    auto compute = [&](const Fp4Stage<HD> &from) {
        col.step(from, g, from.t0 + FP4_STEP > min(from.end, first_hi + 1) || from.t0 < last_lo);
    };
    for (; step < step_end; step += 4 * 64) {
        pages.load(v, seq, steps, step, step_end, lane);
        const int last = min(step_end, step + 4 * 64);
        const int most = last - 1 - (last - 1 - step) % 4;      // the wave's last step of these
        // Every fetch is made, behind the last one of that step again: a transfer that is made on some paths only would have
        // the next use of any wait for all of them.
        fetch(in[0], step);
        for (int at = step; at < last; at += 8) {
            fetch(in[1], min(at + 4, most));
            compute(in[0]);
            if (at + 4 >= last) break;
            fetch(in[0], min(at + 8, most));
            compute(in[1]);
        }
    }
    float4_t(&o)[OT] = col.o;
    const float l = column_sum(col.l), m = col.m == -INFINITY ? col.m : col.m * col.scale;

    // The four waves' results: each scaled to their common maximum, then summed.  A lane's o[4x + c][i] is channel
    // 64x + 16g + 4i + c.
    if (g == 0) lds_m[wave][c16] = m, lds_l[wave][c16] = l;
    __syncthreads();
    const float top = fmaxf(fmaxf(lds_m[0][c16], lds_m[1][c16]), fmaxf(lds_m[2][c16], lds_m[3][c16]));
    const float mine = weight_of(m, top);
#pragma unroll
    for (int x = 0; x < VH; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<float4 *>(&lds_o[wave][c16][64 * x + 16 * g + 4 * i]) =
                make_float4(o[4 * x][i] * mine, o[4 * x + 1][i] * mine, o[4 * x + 2][i] * mine, o[4 * x + 3][i] * mine);
    __syncthreads();
    // sixteen threads to a column, four channels at a time
    const int to = threadIdx.x >> 4, part = threadIdx.x & 15;
    const int to_column = column0 + to;
    const float to_m = fmaxf(fmaxf(lds_m[0][to], lds_m[1][to]), fmaxf(lds_m[2][to], lds_m[3][to]));
    float to_l = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) to_l += lds_l[w][to] * weight_of(lds_m[w][to], to_m);
    const auto place = [&](int column, int64_t &index) {   // of a column's output row; false: it has none
        const int64_t out = seq.first + column / v.G;
        index = out * (int64_t(v.H) * v.G) + h * v.G + column % v.G;
        return column < columns && out >= 0 && out < v.n_rows;
    };
    int64_t index;
    if (place(to_column, index)) {
        float *row = a.part + (a.part_row(stream, share.b, share.first, to) + int64_t(share.split) * a.rows) * (HD + 4);
        const float inverse = to_l > 0.0f || to_l != to_l ? 1.0f / to_l : 0.0f;
#pragma unroll
        for (int x = 0; x < VH; ++x) {
            const int channel = 64 * x + 4 * part;
            float r[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                r[i] = (lds_o[0][to][channel + i] + lds_o[1][to][channel + i]) + (lds_o[2][to][channel + i] + lds_o[3][to][channel + i]);
            if (share.splits == 1) {
#pragma unroll
                for (int i = 0; i < 4; ++i) r[i] *= inverse;
                store_out(a.out, a.out_type, index * HD + channel, r);
            } else if (a.counters) {
                store_shared(row + channel, r[0], r[1]);
                store_shared(row + channel + 2, r[2], r[3]);
            } else {
                *reinterpret_cast<float4 *>(row + channel) = make_float4(r[0], r[1], r[2], r[3]);
            }
        }
        if (part == 0) {
            if (share.splits == 1) {
                if (a.lse) a.lse[index] = log_sum(to_m, to_l);
            } else if (a.counters) {
                store_shared(row + HD, to_m, to_l);
            } else {
                row[HD] = to_m, row[HD + 1] = to_l;
            }
        }
    }
    if (!a.counters || share.splits == 1) return;
    if (!last_group(a.counters + stream * v.batch.batch + share.b, share.splits, &lds_last)) return;
    // HD / 4 threads to a row, four channels each; the other threads take other columns, or other splits of the same where
    // there are few columns, four rows at a time
    constexpr int PARTS = 256 / (HD / 4);
    const int here = min(columns - column0, FP4_COLUMNS), four = threadIdx.x % (HD / 4), team = threadIdx.x / (HD / 4);
    const int each = here > PARTS / 2 ? 1 : here > PARTS / 4 ? 2 : here > PARTS / 8 ? 4 : PARTS > 8 && here == 1 ? 16 : 8;   // teams to a column
    const int beside = team % each;
    for (int c0 = 0; c0 < here; c0 += PARTS / each) {
        const int c = c0 + team / each;
        const float *rows = a.part + a.part_row(stream, share.b, share.first, min(c, here - 1)) * (HD + 4);
        const int64_t pitch = int64_t(a.rows) * (HD + 4);
        float m = -INFINITY, l = 0.0f, r[4] = {0, 0, 0, 0};
        for (int s0 = beside; s0 < share.splits; s0 += 4 * each) {
            float2 x[4], y[4], ml[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float *from = rows + min(s0 + i * each, share.splits - 1) * pitch;
                x[i] = load_shared(from + 4 * four), y[i] = load_shared(from + 4 * four + 2), ml[i] = load_shared(from + HD);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (s0 + i * each >= share.splits) break;
                const float now = fmaxf(m, ml[i].x), old = weight_of(m, now), f = weight_of(ml[i].x, now);
                m = now;
                l = l * old + ml[i].y * f;
                r[0] = r[0] * old + x[i].x * f, r[1] = r[1] * old + x[i].y * f;
                r[2] = r[2] * old + y[i].x * f, r[3] = r[3] * old + y[i].y * f;
            }
        }
        if (each > 1) {      // the teams of a column: one after the other through LDS (here fits in one turn then)
            float *mine = &lds_o[0][0][0] + team * (HD + 4);
            *reinterpret_cast<float4 *>(mine + 4 * four) = make_float4(r[0], r[1], r[2], r[3]);
            if (four == 0) mine[HD] = m, mine[HD + 1] = l;
            __syncthreads();
            if (beside) return;
            for (int i = 1; i < each; ++i) {
                const float *from = mine + i * (HD + 4);
                const float4 x = *reinterpret_cast<const float4 *>(from + 4 * four);
                const float now = fmaxf(m, from[HD]), old = weight_of(m, now), f = weight_of(from[HD], now);
                m = now;
                l = l * old + from[HD + 1] * f;
                r[0] = r[0] * old + x.x * f, r[1] = r[1] * old + x.y * f, r[2] = r[2] * old + x.z * f, r[3] = r[3] * old + x.w * f;
            }
        }
        if (c >= here || !place(column0 + c, index)) continue;
        const float inverse = l > 0.0f || l != l ? 1.0f / l : 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] *= inverse;
        store_out(a.out, a.out_type, index * HD + 4 * four, r);
        if (a.lse && four == 0) a.lse[index] = log_sum(m, l);
    }
}

// Joins the splits: a workgroup to a column.  Threads first read a split's maximum each, then sum rows: HD / 4 threads to a
// row, four channels each, eight (sixteen) rows at a time.
template <int HD>
__global__ __launch_bounds__(256) void fp4_join_kernel(Fp4Attention a) {
    constexpr int PARTS = 256 / (HD / 4);
    __shared__ float weight[FP4_SPLITS_MAX], sums[PARTS][HD + 4], shared[4];
    const Fp4View &v = a.v;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int column = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
    Fp4Share share;
    share.splits = a.splits, share.first = 0;
    if (a.flat) {
        share.find(a, b / FP4_FLAT, column / FP4_COLUMNS * FP4_COLUMNS, lane);
        share.of_sequence(b);
    }
    const int splits = share.splits;
    const Fp4Sequence seq = a.flat ? share.sequence(v) : Fp4Sequence(v, b);
    const int64_t out_row = seq.first + column / v.G;
    if (splits <= 1 || column >= seq.n * v.G || out_row < 0 || out_row >= v.n_rows) return;
    const float *rows = a.part + a.part_row(column / FP4_COLUMNS * v.H + h, b, share.first, column % FP4_COLUMNS) * (HD + 4);
    const int64_t pitch = int64_t(a.rows) * (HD + 4);
    const int s = threadIdx.x;
    static_assert(FP4_SPLITS_MAX <= 256, "a thread to a split");
    const float my_m = s < splits ? rows[s * pitch + HD] : -INFINITY, my_l = s < splits ? rows[s * pitch + HD + 1] : 0.0f;
    const int part = threadIdx.x / (HD / 4), four = threadIdx.x % (HD / 4);
    float m = my_m;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    if (lane == 0) shared[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(shared[0], shared[1]), fmaxf(shared[2], shared[3]));
    const float f = weight_of(my_m, m);
    weight[s] = f;
    float l = my_l * f;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) l += __shfl_xor(l, d);
    __syncthreads();
    if (lane == 0) shared[wave] = l;
    float4 acc = make_float4(0, 0, 0, 0);
#pragma unroll 4
    for (int i = part; i < splits; i += PARTS) {
        const float4 x = *reinterpret_cast<const float4 *>(rows + i * pitch + 4 * four);
        const float w = weight[i];
        acc.x = fmaf(w, x.x, acc.x), acc.y = fmaf(w, x.y, acc.y), acc.z = fmaf(w, x.z, acc.z), acc.w = fmaf(w, x.w, acc.w);
    }
    *reinterpret_cast<float4 *>(&sums[part][4 * four]) = acc;
    __syncthreads();
    if (threadIdx.x >= HD) return;
    l = (shared[0] + shared[1]) + (shared[2] + shared[3]);
    float o = 0.0f;
#pragma unroll
    for (int i = 0; i < PARTS; ++i) o += sums[i][threadIdx.x];
    const bool some = l > 0.0f || l != l;
    const int64_t index = out_row * (int64_t(v.H) * v.G) + h * v.G + column % v.G;
    const float r = some ? o / l : 0.0f;
    const int64_t at = index * HD + threadIdx.x;
    if (a.out_type == KV_TYPE_FP32) static_cast<float *>(a.out)[at] = r;
    else if (a.out_type == KV_TYPE_BF16) static_cast<__bf16 *>(a.out)[at] = __bf16(r);
    else static_cast<_Float16 *>(a.out)[at] = _Float16(r);
    if (a.lse && threadIdx.x == 0) a.lse[index] = log_sum(m, l);
}

__global__ __launch_bounds__(64) void fp4_clear_kernel(uint32_t *counters) {
    for (int i = threadIdx.x; i < int(FP4_COUNTERS / sizeof(uint32_t)); i += 64) counters[i] = 0;
}

int launch_fp4_clear(const kv_fp4_cache *c, hipStream_t s) {
    hipLaunchKernelGGL(fp4_clear_kernel, dim3(1), dim3(64), 0, s, reinterpret_cast<uint32_t *>(c->workspace));
    KV_HIP_CHECK(hipGetLastError());
    return KV_OK;
}

// Workgroups that a call is split into at most: not quite two to each of the 256 compute units (a third one on some of them
// would hold up the call).  Four sequences of up to 32788 tokens, 8 kv-heads: 480 workgroups 26.9 us, 512 28.3, 256 27.1, 768 29.
constexpr int64_t FP4_GROUPS = 480;
// The last workgroup of a sequence joins its splits itself up to so many rows of partial results; beyond, a kernel with a
// workgroup to each row of the output does.  Passes joined so / by the kernel: one head x 1000 tokens 7.8 / 8.6 us, a window
// of 4096 of 8 kv-heads in 11 splits 9.6 / 10.6, four sequences of up to 32788 28.3 / 29, 32 heads x 4100 in 11 splits 13.2 /
// 13.0; where no sequence turns out to be split (8 sequences x 52 heads) the kernel would be launched for nothing.
constexpr int64_t FP4_MERGED_ROWS = 256;

int launch_fp4_attention(const kv_fp4_cache *c, const Fp4View &v, const void *q, int64_t q_stride, bool bf16, float sm_scale,
                         int window, int sinks, void *out, int out_type, float *lse, hipStream_t s) {
    const int64_t columns = int64_t(v.batch.max_new) * v.G;
    if (columns > (int64_t(1) << 30)) return KV_ERR_UNSUPPORTED;
    Fp4Attention a;
    a.v = v;
    a.q = static_cast<const uint16_t *>(q);
    a.q_stride = q_stride;
    a.scale = sm_scale * 1.4426950408889634f;
    a.window = window, a.sinks = sinks;
    a.out = out, a.out_type = out_type, a.lse = lse;
    a.blocks = int((columns + FP4_COLUMNS - 1) / FP4_COLUMNS);
    a.rows = int(std::min<int64_t>(columns, FP4_COLUMNS));
    // Steps that a block of columns can have.
    int64_t most = int64_t(v.batch.table_pages) * (FP4_PAGE / FP4_STEP);
    if (window) most = std::min(most, (int64_t(window) + FP4_COLUMNS + sinks) / FP4_STEP + 3);
    const int batch = v.batch.batch;
    const int64_t streams = int64_t(a.blocks) * v.H, room = FP4_PART_ROWS / a.rows / streams;   // workgroups that the workspace takes
    a.least_steps = streams * batch * (most / FP4_LEAST_STEPS) <= FP4_FEW_GROUPS ? FP4_LEAST_STEPS : FP4_MORE_STEPS;
    const int64_t useful = (most + a.least_steps - 1) / a.least_steps;       // splits of a sequence
    const int chunk = std::min(batch, FP4_FLAT), chunks = (batch + FP4_FLAT - 1) / FP4_FLAT;
    int64_t want = FP4_GROUPS / streams;
    a.flat = batch > 1 && useful > 1 && room >= 2 * chunk * chunks;
    if (a.flat)
        a.splits = int(std::min({std::max<int64_t>(want / chunks, 2 * chunk), chunk * (1 + useful), room / chunks, int64_t(FP4_SPLITS_MAX)}));
    else
        a.splits = int(std::max<int64_t>(std::min({want / batch, useful, room / batch, int64_t(FP4_SPLITS_MAX)}), 1));
    const int64_t groups = int64_t(a.flat ? chunks : batch) * a.splits;
    if (a.blocks > 65535 || groups > 65535) return KV_ERR_UNSUPPORTED;
    const bool merged = a.splits > 1 && a.splits <= 64 && streams * batch <= FP4_COUNTERS && a.rows * a.splits <= FP4_MERGED_ROWS;
    a.counters = merged ? reinterpret_cast<uint8_t *>(c->workspace) : nullptr;
    a.part = c->workspace + FP4_COUNTERS / sizeof(float);
    const dim3 grid = dim3(uint32_t(v.H), uint32_t(a.blocks), uint32_t(groups));
#define LAUNCH(HD, BF) hipLaunchKernelGGL((fp4_attention_kernel<HD, BF>), grid, dim3(256), 0, s, a)
    if (c->cfg.head_dim == 128) {
        if (bf16) LAUNCH(128, true); else LAUNCH(128, false);
    } else {
        if (bf16) LAUNCH(64, true); else LAUNCH(64, false);
    }
#undef LAUNCH
    KV_HIP_CHECK(hipGetLastError());
    if (a.splits > 1 && !a.counters) {
        const dim3 grid = dim3(uint32_t(columns), uint32_t(v.H), uint32_t(batch));
        if (c->cfg.head_dim == 128) hipLaunchKernelGGL(fp4_join_kernel<128>, grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL(fp4_join_kernel<64>, grid, dim3(256), 0, s, a);
        KV_HIP_CHECK(hipGetLastError());
    }
    return KV_OK;
}

}  // namespace packkv
