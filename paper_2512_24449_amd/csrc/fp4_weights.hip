// The attention weight that cached tokens get from a call's rows (packkv.h: kv_fp4_weights):
//   mass[t] = past[t] + sum over the rows that see t and the G heads of  exp(sm_scale q . k_t - lse).
// The logarithm of the softmax's sum is the attention call's, so that one pass over K does it: no maximum, no sum to wait for.
//
// Scores are S = Q K^T with the tokens as columns: a lane holds scores of one token, so the sum over rows and heads is its
// own, joined over the four lanes of a token at the end, and K's rows are read as the attention kernels read them.  Row
// 4g + i of a product is column 4i + g of the call's columns (row after row, the heads of the kv-head next to each other): with up
// to four columns a lane has one exponential to a token, not four.
//
// Few columns are bound by HBM: 8 sequences x 52 heads x 32000 tokens, 1.01 GB, in 198 us, 5.1 TB/s (half of every block of a
// page is read, and a tenth of the bytes is weights, read and written: a copy reaches 4.7 to 5.0, a read 5.9 to 6.8).  Many columns by
// exponentials and products, which share the issue: 2048 rows of 32 heads at 12288 (2.2e11 operations) take 225 to 237 us by the card, 945 to
// 990 TFLOP/s, where a large library product reaches 1345 (some 260 us in the first passes after a pause: the clock rises over
// hundreds); per 16 columns and page 68 vector instructions, 16 of them exponentials of four times the cost, beside 16 products: vector
// instructions are issued 72 % of the time, the matrix cores are busy 40 %.
#include "fp4_attention.h"
#include "overlap.h"

namespace packkv {

struct Fp4Weights {
    Fp4View v;
    const uint16_t *q;
    int64_t q_stride;
    const float *lse;
    float scale;             // for powers of two
    int window, sinks;
    const float *past;
    float *mass;
    int64_t pitch;           // values of a (sequence, kv-head) in mass and past
    float *part;             // not null: sums of each split of the columns, [splits][batch][H][table_pages * 64]
    int splits;
};

constexpr int WEIGHTS_HELD = 8;          // blocks of 16 columns that stay in LDS

// What the rows of a block of 16 columns need beside q: register i of a lane's results is column 4i + g.
struct Fp4RowSet {
    float4 less[4];          // [g]: minus the logarithms, in powers of two
    int4 hi[4];              // [g]: last tokens that the rows see
    int first_hi, last_hi;   // of the rows that there are, least and largest
    int pad[2];
};

// A lane's part of 16 columns' operand on its way, and (lanes 0 .. 15) of what their rows need; then 64 columns further on.
// An infinity in q needs no care where its row counts: the row's lse is NaN then.
template <int HD, bool BF16>
struct Fp4Columns {
    static constexpr int KW = HD / 32;
    uint4_t q[KW];
    float lse;
    int of, beside;          // row and head of the column
    int row;                 // of what was loaded
    bool real;
    __device__ inline void start(const Fp4Weights &a, int column0, int lane) {
        const int column = column0 + 4 * (lane & 3) + ((lane & 15) >> 2);
        of = column / a.v.G, beside = column - of * a.v.G;
    }
    // Every lane loads, from somewhere: loads that are made on some paths only would be waited for one by one.
    __device__ inline void load(const Fp4Weights &a, const Fp4Sequence &seq, int h, int lane) {
        const Fp4View &v = a.v;
        const int64_t at = seq.first + of;
        const int head = h * v.G + beside;
        real = of < seq.n && at >= 0 && at < v.n_rows;
        const uint16_t *from = a.q + at * a.q_stride + int64_t(head) * HD + (lane >> 4) * (HD / 4);
        const float *sum = a.lse + (at * (int64_t(v.H) * v.G) + head);
        from = real ? from : reinterpret_cast<const uint16_t *>(v.pages);
        sum = real ? sum : reinterpret_cast<const float *>(v.pages);
#pragma unroll
        for (int i = 0; i < KW; ++i) q[i] = *reinterpret_cast<const uint4_t *>(from + 8 * i);
        lse = *sum;
        row = of;
    }
    __device__ inline void advance(int G, int rows64, int heads64) {     // 64 / G, 64 % G
        of += rows64, beside += heads64;
        if (beside >= G) beside -= G, ++of;
    }
    // 0 for q where there is no row, where its scores do not count and where the scale is 0: minus infinity added to an infinite score, or 0
    // times it, is NaN.
    __device__ inline void settle(const Fp4Weights &a) {
        const bool counts = real && lse != -INFINITY && a.scale != 0.0f;
        if (__all(counts)) return;
#pragma unroll
        for (int i = 0; i < KW; ++i) q[i] = counts ? q[i] : uint4_t{0, 0, 0, 0};
    }
    __device__ inline void store(Fp4RowSet &set, const Fp4Sequence &seq, int lane) const {
        const int hi = max(seq.pos0 + min(row, seq.n - 1), -1);
        // (-infinity: a row that sees nothing)
        if (lane < 16) {
            reinterpret_cast<float *>(set.less)[lane] = real && lse != -INFINITY ? -(lse * FP4_LOG2E) : -INFINITY;
            reinterpret_cast<int *>(set.hi)[lane] = hi;      // (lane 4g + i: column 4i + g)
        }
        if (lane == 0) set.first_hi = hi;
        if (lane == 15) set.last_hi = hi;
    }
};

// The rows of a page on their way: of K a lane's quarter of four tokens' rows.
template <int HD>
struct Fp4KPage {
    using P = Fp4Block<HD>;
    static constexpr int KW = HD / 32;
    uint32_t k[4][KW], ks[4];
    __device__ inline void load(const uint8_t *block, int c16, int g) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int token = 16 * t + c16;
            const uint8_t *from = block + P::K + token * (HD / 2) + g * (HD / 8);
            if constexpr (KW == 4) {
                const uint4_t x = *reinterpret_cast<const uint4_t *>(from);
                k[t][0] = x.x, k[t][1] = x.y, k[t][2] = x.z, k[t][3] = x.w;
            } else {
                const uint2 x = *reinterpret_cast<const uint2 *>(from);
                k[t][0] = x.x, k[t][1] = x.y;
            }
            ks[t] = block[P::KS + token * (HD / FP4_GROUP) + g * (HD / 4) / FP4_GROUP];
        }
    }
    template <bool BF16>
    __device__ inline void operands(uint4_t (&to)[4][KW]) const {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < KW; ++i) to[t][i] = row_operand<BF16>(k[t][i], __uint_as_float(ks[t] << 23));
    }
};

template <int HD, bool BF16>
__device__ inline void scores(const uint4_t (&q)[HD / 32], const uint4_t (&k)[4][HD / 32], float4_t (&s)[4]) {
#pragma unroll
    for (int t = 0; t < 4; ++t) s[t] = float4_t{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < HD / 32; ++i)
#pragma unroll
        for (int t = 0; t < 4; ++t) s[t] = product16<BF16>(q[i], k[t][i], s[t]);
}

// Products and exponentials of the code before in turn: the matrix core works beside the vector instructions then.
template <int KW>
__device__ inline void interleave() {
#pragma unroll
    for (int i = 0; i < 4 * KW; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 12 / KW, 0);
    }
}

// Adds the weights that 16 columns give to the page's tokens, all of which they see.  NI: registers of a result that hold columns.
template <int NI>
__device__ inline void weigh_whole(const Fp4Weights &a, const float4_t (&s)[4], const float4 &less4, float (&sum)[4]) {
    const float less[4] = {less4.x, less4.y, less4.z, less4.w};
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        float p[NI];
#pragma unroll
        for (int i = 0; i < NI; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(s[t][i], a.scale, less[i]));
        if constexpr (NI == 4) sum[t] += (p[0] + p[1]) + (p[2] + p[3]);
        else if constexpr (NI == 2) sum[t] += p[0] + p[1];
        else sum[t] += p[0];
    }
}

// The same where some do not see some.
template <int NI>
__device__ inline void weigh_some(const Fp4Weights &a, const float4_t (&s)[4], const float4 &less4, const int4 &hi4, int t0, int end, int c16,
                                  float (&sum)[4]) {
    const float less[4] = {less4.x, less4.y, less4.z, less4.w};
    const int hi[4] = {hi4.x, hi4.y, hi4.z, hi4.w};
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int token = t0 + 16 * t + c16;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int lo = a.window ? hi[i] - a.window : -1;
            const float p = __builtin_amdgcn_exp2f(fmaf(s[t][i], a.scale, less[i]));
            sum[t] += (token <= hi[i]) & (token < end) & ((token > lo) | (token < a.sinks)) ? p : 0.0f;
        }
    }
}

// Whether rows that see up to first_hi .. last_hi see all tokens of the page at t0.
__device__ inline bool sees_whole(const Fp4Weights &a, int t0, int end, int first_hi, int last_hi) {
    return t0 + FP4_PAGE <= min(end, first_hi + 1) && !(a.window && t0 <= last_hi - a.window);
}

__device__ inline float token_sum(const float (&sum)[4], int g) {     // of token 16g + c16
    float mine = 0.0f;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const float all = column_sum(sum[t]);
        mine = g == t ? all : mine;
    }
    return mine;
}

// Which rows may see a token of the 64 from t0 on; every row of the sequence does see a token before `sinks` that it sees at all.
struct Fp4RowsOf {
    int first, end;
    __device__ inline Fp4RowsOf(const Fp4Weights &a, const Fp4Sequence &seq, int t0) {
        first = max(int(min(int64_t(t0) - seq.pos0, int64_t(seq.n))), 0);
        end = seq.n;
        if (a.window && t0 >= a.sinks) end = int(max(min(int64_t(t0) + FP4_PAGE - 1 + a.window - seq.pos0, int64_t(seq.n)), int64_t(0)));
    }
};

// Few columns (up to 128): their operands stay, in LDS or, of one block, in registers, and pages stream past them, each wave's next one
// on its way while one is weighed.  A workgroup takes 4 * pages_of_wave pages in a row, a wave every fourth.
template <int HD, bool BF16, int NI, bool ONE>
__global__ __launch_bounds__(256) void fp4_weights_kernel(Fp4Weights a, int pages_of_wave, int page_groups) {
    using P = Fp4Block<HD>;
    constexpr int KW = HD / 32, HELD = ONE ? 1 : WEIGHTS_HELD;
    __shared__ uint4_t held[HELD][KW][64];
    __shared__ Fp4RowSet sets[HELD];
    const Fp4View &v = a.v;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c16 = lane & 15, g = lane >> 4;
    const int h = blockIdx.x % uint32_t(v.H), b = blockIdx.y;
    int group = int(blockIdx.x / uint32_t(v.H));
    const Fp4Sequence seq(v, b);
    const int columns = seq.n * v.G, blocks = (columns + 31) / 32 * 2;
    const int table_end = (seq.held + FP4_PAGE - 1) / FP4_PAGE;
    if (4 * pages_of_wave * group >= table_end) return;
    Fp4Columns<HD, BF16> cols;
    for (int n = wave; n < (ONE ? 4 : blocks); n += 4) {
        const int block = ONE ? 0 : n;
        cols.start(a, 16 * block, lane);
        cols.load(a, seq, h, lane);
        cols.settle(a);
        if (!ONE) {
#pragma unroll
            for (int i = 0; i < KW; ++i) held[block][i][lane] = cols.q[i];
        }
        if (!ONE || wave == 0) cols.store(sets[block], seq, lane);
    }
    __syncthreads();
    const float *past = a.past ? a.past + (int64_t(b) * v.H + h) * a.pitch : nullptr;
    float *mass = a.mass + (int64_t(b) * v.H + h) * a.pitch;
    const int past_end = int(min(int64_t(min(seq.held, seq.pos0)), a.pitch)), mass_end = int(min(int64_t(seq.held), a.pitch));
    for (; 4 * pages_of_wave * group < table_end; group += page_groups) {
        // the wave's pages, one to a lane
        const int mine = 4 * (pages_of_wave * group + lane) + wave;
        const bool there = lane < pages_of_wave && mine < table_end;
        int page = -1;
        if (there) {
            const Fp4RowsOf rows(a, seq, mine * FP4_PAGE);
            if (rows.first < rows.end) page = int(seq.page(v, mine));
        }
        uint64_t todo = __ballot(page >= 0), idle = __ballot(there && page < 0);
        while (idle) {       // nothing sees these
            const int j = __builtin_ctzll(idle), token = (4 * (pages_of_wave * group + j) + wave) * FP4_PAGE + lane;
            idle &= idle - 1;
            if (token < mass_end) mass[token] = past && token < past_end ? past[token] : 0.0f;
        }
        if (!todo) continue;
        Fp4KPage<HD> in[2];
        int at[2];           // pages of the sequence
        float old[2];        // what the lane's token had
        const auto fetch = [&](int to, int j) {
            at[to] = 4 * (pages_of_wave * group + j) + wave;
            const int token = at[to] * FP4_PAGE + lane;
            in[to].load(v.pages + (int64_t(__builtin_amdgcn_readlane(page, j)) * v.H + h) * size_t(P::BYTES), c16, g);
            old[to] = *(past && token < past_end ? past + token : reinterpret_cast<const float *>(v.pages));
        };
        const auto compute = [&](int which) {
            uint4_t k[4][KW];
            in[which].template operands<BF16>(k);
            const int t0 = at[which] * FP4_PAGE;
            float sum[4] = {0, 0, 0, 0};
            const bool whole = sees_whole(a, t0, seq.held, max(seq.pos0, -1), max(seq.pos0 + seq.n - 1, -1));   // (wave-uniform)
            if constexpr (ONE) {
                float4_t s[4];
                scores<HD, BF16>(cols.q, k, s);
                if (whole) weigh_whole<NI>(a, s, sets[0].less[g], sum);
                else weigh_some<NI>(a, s, sets[0].less[g], sets[0].hi[g], t0, seq.held, c16, sum);
            } else if (whole) {
                // two blocks in turn: the products of one beside the exponentials of the other
                float4_t s[2][4];
                uint4_t q[2][KW];
                const auto operand = [&](int to, int n) {
#pragma unroll
                    for (int i = 0; i < KW; ++i) q[to][i] = held[n][i][lane];
                };
                operand(0, 0);
                operand(1, 1);
                scores<HD, BF16>(q[0], k, s[0]);
                for (int n = 0; n < blocks; n += 2) {
                    operand(0, min(n + 2, blocks - 1));
                    scores<HD, BF16>(q[1], k, s[1]);
                    weigh_whole<NI>(a, s[0], sets[n].less[g], sum);
                    interleave<KW>();
                    operand(1, min(n + 3, blocks - 1));
                    scores<HD, BF16>(q[0], k, s[0]);         // (behind the last one that one again)
                    weigh_whole<NI>(a, s[1], sets[n + 1].less[g], sum);
                    interleave<KW>();
                }
            } else {
                for (int n = 0; n < blocks; ++n) {
                    uint4_t q[KW];
                    float4_t s[4];
#pragma unroll
                    for (int i = 0; i < KW; ++i) q[i] = held[n][i][lane];
                    scores<HD, BF16>(q, k, s);
                    weigh_some<NI>(a, s, sets[n].less[g], sets[n].hi[g], t0, seq.held, c16, sum);
                }
            }
            const int token = t0 + lane;
            const float all = token_sum(sum, g);
            if (token < mass_end) __builtin_nontemporal_store(past && token < past_end ? old[which] + all : all, mass + token);
        };
        // every fetch is made, behind the last page that one again
        const auto next = [&]() {
            const int j = __builtin_ctzll(todo);
            if (todo & (todo - 1)) todo &= todo - 1;
            return j;
        };
        int left = __popcll(todo);
        fetch(0, next());
        while (true) {
            fetch(1, next());
            compute(0);
            if (--left == 0) break;
            fetch(0, next());
            compute(1);
            if (--left == 0) break;
        }
    }
}

// Many columns: a wave keeps the operands of a page, the columns pass through LDS, 64 at a time, in two buffers in turn.
template <int HD, bool BF16>
__global__ __launch_bounds__(256, 3) void fp4_weights_tile_kernel(Fp4Weights a, int page_groups) {
    using P = Fp4Block<HD>;
    constexpr int KW = HD / 32;
    __shared__ uint4_t staged[2][4][KW][64];
    __shared__ Fp4RowSet sets[2][4];
    const Fp4View &v = a.v;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c16 = lane & 15, g = lane >> 4;
    const int h = blockIdx.x % uint32_t(v.H), b = blockIdx.y, split = blockIdx.z;
    const Fp4Sequence seq(v, b);
    const int table_end = (seq.held + FP4_PAGE - 1) / FP4_PAGE;
    const float *past = a.past ? a.past + (int64_t(b) * v.H + h) * a.pitch : nullptr;
    float *mass = a.mass + (int64_t(b) * v.H + h) * a.pitch;
    const int past_end = int(min(int64_t(min(seq.held, seq.pos0)), a.pitch)), mass_end = int(min(int64_t(seq.held), a.pitch));
    const int rows64 = 64 / v.G, heads64 = 64 % v.G;
    for (int group = int(blockIdx.x / uint32_t(v.H)); 4 * group < table_end; group += page_groups) {
        const int index = 4 * group + wave, t0 = index * FP4_PAGE, token = t0 + lane;
        const Fp4RowsOf lowest(a, seq, 4 * group * FP4_PAGE), highest(a, seq, (4 * group + 3) * FP4_PAGE);
        const int row0 = lowest.first, row_end = max(lowest.end, highest.end);
        // the split's columns, 64 at a time
        const int from = row0 * v.G / 64, stages = (row_end * v.G + 63) / 64 - from, each = (max(stages, 0) + a.splits - 1) / a.splits;
        const int column0 = 64 * (from + min(each * split, max(stages, 0)));
        const int column_end = 64 * (from + min(each * (split + 1), max(stages, 0)));
        const int64_t page = index < table_end ? seq.page(v, index) : -1;
        Fp4KPage<HD> in;
        in.load(v.pages + (max(page, int64_t(0)) * v.H + h) * size_t(P::BYTES), c16, g);
        uint4_t k[4][KW];
        in.template operands<BF16>(k);
        float sum[4] = {0, 0, 0, 0};
        Fp4Columns<HD, BF16> cols;
        const auto store = [&](int to) {
            cols.settle(a);
#pragma unroll
            for (int i = 0; i < KW; ++i) staged[to][wave][i][lane] = cols.q[i];
            cols.store(sets[to][wave], seq, lane);
        };
        if (column0 < column_end) {
            cols.start(a, column0 + 16 * wave, lane);
            cols.load(a, seq, h, lane);
            store(0);
        }
        __syncthreads();
        int now = 0;
        for (int column = column0; column < column_end; column += 64, now ^= 1) {
            cols.advance(v.G, rows64, heads64);              // (behind the last ones some more, which nobody reads)
            cols.load(a, seq, h, lane);
            const int first_hi = __builtin_amdgcn_readfirstlane(sets[now][0].first_hi), last_hi = __builtin_amdgcn_readfirstlane(sets[now][3].last_hi);
            float part[4] = {0, 0, 0, 0};
            const uint4_t(*tile)[KW][64] = staged[now];
            if (page < 0 || last_hi < t0 || (a.window && t0 >= a.sinks && t0 + FP4_PAGE - 1 <= first_hi - a.window)) {
            } else if (sees_whole(a, t0, seq.held, first_hi, last_hi)) {
                uint4_t q[2][KW];
                float4_t s[2][4];
#pragma unroll
                for (int i = 0; i < KW; ++i) q[0][i] = tile[0][i][lane];
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    if (n < 3) {
#pragma unroll
                        for (int i = 0; i < KW; ++i) q[(n + 1) & 1][i] = tile[n + 1][i][lane];
                    }
                    scores<HD, BF16>(q[n & 1], k, s[n & 1]);
                    if (n > 0) {
                        weigh_whole<4>(a, s[(n - 1) & 1], sets[now][n - 1].less[g], part);
                        interleave<KW>();
                    }
                }
                weigh_whole<4>(a, s[1], sets[now][3].less[g], part);
            } else {
                for (int n = 0; n < 4; ++n) {
                    uint4_t q[KW];
                    float4_t s[4];
#pragma unroll
                    for (int i = 0; i < KW; ++i) q[i] = tile[n][i][lane];
                    scores<HD, BF16>(q, k, s);
                    weigh_some<4>(a, s, sets[now][n].less[g], sets[now][n].hi[g], t0, seq.held, c16, part);
                }
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) sum[t] += part[t];
            store(now ^ 1);
            __syncthreads();
        }
        const float all = token_sum(sum, g);
        if (a.part) {
            if (token < mass_end) a.part[((int64_t(split) * v.batch.batch + b) * v.H + h) * (int64_t(v.batch.table_pages) * FP4_PAGE) + token] = all;
        } else {
            if (token < mass_end) mass[token] = past && token < past_end ? past[token] + all : all;
        }
    }
}

// Joins the splits, a thread to a token.
__global__ __launch_bounds__(256) void fp4_weights_join_kernel(Fp4Weights a, int page_groups) {
    const Fp4View &v = a.v;
    const int h = blockIdx.x % uint32_t(v.H), b = blockIdx.y;
    const Fp4Sequence seq(v, b);
    const int past_end = int(min(int64_t(min(seq.held, seq.pos0)), a.pitch)), mass_end = int(min(int64_t(seq.held), a.pitch));
    const int64_t stream = int64_t(b) * v.H + h, room = int64_t(v.batch.table_pages) * FP4_PAGE, pitch = room * v.H * v.batch.batch;
    for (int64_t token = int64_t(blockIdx.x / uint32_t(v.H)) * 256 + threadIdx.x; token < mass_end; token += 256 * int64_t(page_groups)) {
        const float *part = a.part + stream * room + token;
        float sum = a.past && token < past_end ? a.past[stream * a.pitch + token] : 0.0f;
        float all = 0.0f;
        for (int i = 0; i < a.splits; ++i) all += part[i * pitch];
        a.mass[stream * a.pitch + token] = sum + all;
    }
}

// Pages of a wave: one to each of so many waves first (two workgroups to a compute unit).  With more columns than 16 no more
// waves than these, so that each operand is fetched and laid out as seldom as may be; else up to so many pages.  With 1 / 2 / 4 / 6 / 8 / 12 / 16
// pages to a wave 8 x 52 heads x 32000 tokens take 281 / 217 / 200 / 198 / 199 / 202 / 204 us, four sequences of up to 32788 tokens, 8 kv-heads, 18.1 / 15.1 /
// 14.0 / 14.7 / 13.8 / 17.1 / 17.0, 32 rows of 32 heads at 131072 (128 columns) 60 / 47 / 42 / 44 / 40 / 53 / 46.
constexpr int64_t WEIGHTS_ROUND = 2048;
constexpr int WEIGHTS_PAGES = 6;
// Workgroups that many columns are split into; their sums are joined by a kernel.  The chunk of 2048 rows with 1 / 2 / 5 / 10 / 20 splits 299 / 292 / 238 /
// 235 / 243 us.  (128 columns past pages that stay 51 us, pages past columns that stay 43: those take up to WEIGHTS_HELD blocks.)
constexpr int64_t WEIGHTS_GROUPS = 2304;

int launch_fp4_weights(const kv_fp4_cache *c, const Fp4View &v, const void *q, int64_t q_stride, bool bf16, float sm_scale, int window,
                       int sinks, const float *lse, const float *past, float *mass, int64_t mass_tokens, hipStream_t s) {
    Fp4Weights a{v, static_cast<const uint16_t *>(q), q_stride, lse, sm_scale * FP4_LOG2E, window, sinks,
                 past, mass, mass_tokens, nullptr, 1};
    const int64_t columns = int64_t(v.batch.max_new) * v.G, most = int64_t(v.batch.table_pages) * v.H * v.batch.batch;   // pages
    const bool tiles = columns > 16 * WEIGHTS_HELD;
    const int each = tiles ? 1 : int(std::max<int64_t>(columns > 16 ? std::min<int64_t>((most + WEIGHTS_ROUND - 1) / WEIGHTS_ROUND, 64)
                                                                    : std::min<int64_t>(most / WEIGHTS_ROUND, WEIGHTS_PAGES), 1));
    const int64_t groups = std::min({(v.batch.table_pages + int64_t(4) * each - 1) / (4 * each), int64_t(4096), FP4_GROUPS_MOST / v.H});
    if (tiles) {
        const int64_t room = FP4_PART_ROWS * (c->cfg.head_dim + 4) / (most * FP4_PAGE), stages = (columns + 63) / 64;
        a.splits = int(std::max<int64_t>(std::min({WEIGHTS_GROUPS / (groups * v.H * v.batch.batch), room, stages / 4, int64_t(64)}), 1));
        if (a.splits > 1) a.part = c->workspace + FP4_COUNTERS / sizeof(float);
    }
    const dim3 grid = dim3(uint32_t(groups * v.H), uint32_t(v.batch.batch), uint32_t(a.splits));
#define LAUNCH(HD, BF)                                                                                                              \
    do {                                                                                                                            \
        if (tiles) hipLaunchKernelGGL((fp4_weights_tile_kernel<HD, BF>), grid, dim3(256), 0, s, a, int(groups));                    \
        else if (columns > 16) hipLaunchKernelGGL((fp4_weights_kernel<HD, BF, 4, false>), grid, dim3(256), 0, s, a, each, int(groups)); \
        else if (columns > 8) hipLaunchKernelGGL((fp4_weights_kernel<HD, BF, 4, true>), grid, dim3(256), 0, s, a, each, int(groups));   \
        else if (columns > 4) hipLaunchKernelGGL((fp4_weights_kernel<HD, BF, 2, true>), grid, dim3(256), 0, s, a, each, int(groups));   \
        else hipLaunchKernelGGL((fp4_weights_kernel<HD, BF, 1, true>), grid, dim3(256), 0, s, a, each, int(groups));                \
    } while (0)
    if (c->cfg.head_dim == 128) {
        if (bf16) LAUNCH(128, true); else LAUNCH(128, false);
    } else {
        if (bf16) LAUNCH(64, true); else LAUNCH(64, false);
    }
#undef LAUNCH
    KV_HIP_CHECK(hipGetLastError());
    if (a.part) {
        hipLaunchKernelGGL(fp4_weights_join_kernel, dim3(uint32_t(groups * v.H), uint32_t(v.batch.batch)), dim3(256), 0, s, a, int(groups));
        KV_HIP_CHECK(hipGetLastError());
    }
    return KV_OK;
}

}  // namespace packkv

using namespace packkv;

extern "C" int kv_fp4_weights(kv_fp4_cache_t *c, const kv_fp4_batch_t *batch, const void *q, int64_t q_stride, int32_t type,
                              int64_t n_rows, float sm_scale, int32_t window, int32_t sinks, const float *lse, const float *past,
                              float *mass, int64_t mass_tokens, void *hip_stream) {
    const int rc = c ? fp4_check_batch(batch) : KV_ERR_ARG;
    if (rc) return rc;
    if (n_rows < 0 || (type != KV_TYPE_FP16 && type != KV_TYPE_BF16)) return KV_ERR_ARG;
    if (!std::isfinite(sm_scale * FP4_LOG2E) || window < 0 || sinks < 0) return KV_ERR_ARG;
    if (q_stride < int64_t(c->cfg.n_q_heads) * c->cfg.head_dim || q_stride % 8) return KV_ERR_ARG;
    if (mass_tokens < 1 || !fp4_aligned(mass, 4) || (past && !fp4_aligned(past, 4))) return KV_ERR_ARG;
    if (n_rows > 0 && batch->max_new > 0 && (!fp4_aligned(q, 16) || !fp4_aligned(lse, 4))) return KV_ERR_ARG;
    if (int64_t(batch->max_new) * (c->cfg.n_q_heads / c->cfg.n_kv_heads) > (int64_t(1) << 30)) return KV_ERR_UNSUPPORTED;
    const int64_t n = batch->batch, columns = c->cfg.n_q_heads, places = n * c->cfg.n_kv_heads, rows = batch->max_new > 0 ? n_rows : 0;
    const Rows written(mass, Rows::Wide(places) * mass_tokens, 4);
    if (overlap(written, {Rows(mass == past ? nullptr : past, Rows::Wide(places) * mass_tokens, 4), Rows(lse, Rows::Wide(rows) * columns, 4),
                          Rows(q, columns * c->cfg.head_dim * 2, Rows::Wide(q_stride) * 2, rows), Rows(batch->lens, n, 4),
                          Rows(batch->new_rows, n, 4), Rows(batch->first_row, n, 4), Rows(batch->page_table, n * batch->table_pages, 4)}))
        return KV_ERR_ARG;
    return launch_fp4_weights(c, fp4_view(c, batch, n_rows), q, q_stride, type == KV_TYPE_BF16, sm_scale, window, sinks, lse, past, mass,
                              mass_tokens, static_cast<hipStream_t>(hip_stream));
}
