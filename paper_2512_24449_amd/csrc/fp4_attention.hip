// Attention over the 4-bit paged cache for few new rows: a wave streams the cache past 16 columns, 32 tokens a step, the next
// step's rows on their way into registers while one is computed.  Four waves of a workgroup take every fourth step and join
// their sums through LDS.  Long contexts are bound by the rate at which HBM delivers pages (8 sequences x 52 heads x 32000 tokens,
// 1.81 GB, in 313 us: 5.8 TB/s where a plain read reaches 6.8), with heads of 64 by vector instructions as well (130 a step of 2176
// bytes, 180 a step of 4352 with heads of 128; 8 sequences x 12 heads x 111355 tokens, 0.73 GB, 143 us, 5.1 TB/s), short ones by
// a chain of memory latencies -- lengths, page numbers, rows, partial results -- of some 5 us.
#include "fp4_attention.h"

namespace packkv {

size_t fp4_workspace_bytes(int head_dim) { return FP4_COUNTERS + size_t(FP4_PART_ROWS) * (head_dim + 4) * sizeof(float); }

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

// The page numbers of the next 64 steps of a wave, one to a lane: none of its transfers waits for the table.
struct Fp4Pages {
    int page;                // (page numbers fit 31 bits) -1: missing
    __device__ inline void load(const Fp4View &v, const Fp4Sequence &seq, const Fp4Steps<FP4_STEP> &steps, int step, int end, int lane) {
        const int mine = step + 4 * lane;
        page = mine < end ? int(seq.page(v, steps.token(mine) / FP4_PAGE)) : -1;
    }
    __device__ inline int at(int i) const { return __builtin_amdgcn_readlane(page, i); }
};

// (heads of 64: 96 registers, one more would cost the fifth wave of a SIMD)
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
    // (numbers of workgroups are the slowest axis: those without work come last and leave no compute unit out)
    Fp4Share<FP4_STEP> share;
    const Fp4Sequence seq = share.find(a, int(blockIdx.z / uint32_t(a.splits)), int(blockIdx.z % uint32_t(a.splits)), 0, column0, lane);
    if (share.splits == 0) return;
    const int columns = seq.n * v.G;
    const Fp4Steps<FP4_STEP> steps(seq, column0, FP4_COLUMNS, v.G, a.window, a.sinks);
    const int per_split = (steps.n + share.splits - 1) / share.splits;
    const int step_end = min((share.split + 1) * per_split, steps.n);
    int step = __builtin_amdgcn_readfirstlane(share.split * per_split + wave);

    // this lane's column
    const int column = column0 + c16, row = column / v.G, head = h * v.G + column % v.G;
    const int64_t out_row = seq.first + row;
    const bool real = column < columns && out_row >= 0 && out_row < v.n_rows;
    Fp4Column<HD> col;
    col.hi = max(seq.pos0 + row, -1);
    const Fp4Scale &scale = a.scale;
    uint4_t q[KW];
#pragma unroll
    for (int i = 0; i < KW; ++i) {
        q[i] = uint4_t{0, 0, 0, 0};
        if (real) q[i] = *reinterpret_cast<const uint4_t *>(a.q + out_row * a.q_stride + int64_t(head) * HD + g * (HD / 4) + 8 * i) ^ scale.sign;
    }
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
        float4_t s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = float4_t{0, 0, 0, 0};
            const float ks = __uint_as_float(from.ks[t] << 23);
#pragma unroll
            for (int i = 0; i < KW; ++i) s[t] = product16<BF16>(row_operand<BF16>(from.k[t][i], ks), q[i], s[t]);
        }
        uint2 vs[VH];
#pragma unroll
        for (int x = 0; x < VH; ++x) vs[x] = from.vs[x];
        if (from.t0 + FP4_STEP > min(from.end, first_hi + 1) || from.t0 < last_lo) {   // (wave-uniform)
            const int t8 = from.t0 + 8 * g;
            col.mask(s, t8, from.end, a.window, a.sinks);
#pragma unroll
            for (int x = 0; x < VH; ++x) vs[x] = seen_scales(vs[x], t8, steps.begin, from.end, a.sinks);
        }
        uint4_t p[1];
        col.weigh(s, scale, p);
#pragma unroll
        for (int x = 0; x < VH; ++x) {
            half2_t scales[4];
            scale_pairs(vs[x], scales);
            const uint32_t words[4] = {from.v[x].x, from.v[x].y, from.v[x].z, from.v[x].w};
#pragma unroll
            for (int c = 0; c < 4; ++c) col.o[4 * x + c] = product16<false>(column_operand(words[c], scales), p[0], col.o[4 * x + c]);
        }
    };
    for (; step < step_end; step += 4 * 64) {
        pages.load(v, seq, steps, step, step_end, lane);
        const int last = min(step_end, step + 4 * 64);
        const int most = last - 1 - (last - 1 - step) % 4;      // the wave's last step of these
        // Every fetch is made, behind the last one of that step again: a transfer that is made on some paths only would have
        // the next use of any wait for all of them.
        fetch(in[0], step);
        scale.settle<BF16>(q);      // (here, where it waits for nothing that the transfers do not)
        for (int at = step; at < last; at += 8) {
            fetch(in[1], min(at + 4, most));
            compute(in[0]);
            if (at + 4 >= last) break;
            fetch(in[0], min(at + 8, most));
            compute(in[1]);
        }
    }
    float4_t(&o)[OT] = col.o;
    const float l = column_sum(col.l), m = col.largest();

    // The four waves' results: each scaled to their common maximum, then summed.  A lane's o[4x + c][i] is channel
    // 64x + 16g + 4i + c.
    if (g == 0) lds_m[wave][c16] = m, lds_l[wave][c16] = l;
    __syncthreads();
    const float top = fmaxf(fmaxf(lds_m[0][c16], lds_m[1][c16]), fmaxf(lds_m[2][c16], lds_m[3][c16]));
    const float mine = weight_of(m, top, scale.scale);
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
    for (int w = 0; w < 4; ++w) to_l += lds_l[w][to] * weight_of(lds_m[w][to], to_m, scale.scale);
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
                if (a.lse) a.lse[index] = log_sum(to_m, to_l, scale.scale);
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
                const float now = fmaxf(m, ml[i].x), old = weight_of(m, now, scale.scale), f = weight_of(ml[i].x, now, scale.scale);
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
                const float now = fmaxf(m, from[HD]), old = weight_of(m, now, scale.scale), f = weight_of(from[HD], now, scale.scale);
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
        if (a.lse && four == 0) a.lse[index] = log_sum(m, l, scale.scale);
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
    const int chunk = a.flat ? b / FP4_FLAT : b, column0 = column / a.width * a.width;
    int splits, first;
    const auto find = [&](auto share) {
        const Fp4Sequence seq = share.find(a, chunk, -1, b, column0, lane);
        splits = share.splits, first = share.first;
        return seq;
    };
    const Fp4Sequence seq = a.width == FP4_TILE_COLUMNS ? find(Fp4Share<FP4_PAGE>()) : find(Fp4Share<FP4_STEP>());
    const int64_t out_row = seq.first + column / v.G;
    if (splits <= 1 || column >= seq.n * v.G || out_row < 0 || out_row >= v.n_rows) return;
    const float *rows = a.part + a.part_row(column / a.width * v.H + h, b, first, column - column0) * (HD + 4);
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
    const float scale = a.scale.scale, f = weight_of(my_m, m, scale);
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
    if (a.lse && threadIdx.x == 0) a.lse[index] = log_sum(m, l, scale);
}

__global__ __launch_bounds__(64) void fp4_clear_kernel(uint32_t *counters) {
    for (int i = threadIdx.x; i < int(FP4_COUNTERS / sizeof(uint32_t)); i += 64) counters[i] = 0;
}

int launch_fp4_clear(const kv_fp4_cache *c, hipStream_t s) {
    hipLaunchKernelGGL(fp4_clear_kernel, dim3(1), dim3(64), 0, s, reinterpret_cast<uint32_t *>(c->workspace));
    KV_HIP_CHECK(hipGetLastError());
    return KV_OK;
}

// Which kernel: a block of 128 columns takes the tile kernel as long as five to six passes over the cache for 16 columns take
// the streaming kernel, if there are workgroups for all compute units -- blocks enough, or splits of a long context.  Tile /
// streaming kernel, heads of 128 (64): 16 sequences of 2000 tokens, 32 kv-heads, 64 columns each 104 / 79 us (85 / 49), 96 columns
// 81 / 103 (59 / 64), 128 columns 86 / 133 (61 / 83); 64 of 4000 tokens, 8 kv-heads, 96 columns 141 / 188 (102 / 118); one of
// 30000, 8 kv-heads, 256 columns 60 / 70 (43 / 46); one of 2000, 8 kv-heads, 512 columns 31 / 16 (27 / 12).
//
// Workgroups that a call is split into: one to each of the 256 compute units, or, where that leaves more than FP4_LONG_STEPS to
// each, more than fit at once (those end at different times, so that no compute unit is left without).  Passes with 256 /
// 480: 32 heads x 4100 tokens 13.0 / 13.6 us, four sequences of up to 32788 tokens, 8 kv-heads, 27.4 / 27.7, three of 21683, two
// kv-heads, 12.1 / 13.0, one of 103991, 8 kv-heads, 20.7 / 19.9; with 1536 where splits are long: 156 (sequence, head) pairs of up
// to 69824 tokens 217 / 238.
constexpr int64_t FP4_GROUPS = 256, FP4_MORE_GROUPS = 1536;
// The last workgroup of a sequence joins its splits itself where twice its fair share of them makes so many rows of partial
// results at most (it has no more then); beyond, a kernel does, a workgroup to each row of the output.  Passes joined so / by
// the kernel: one head x 1000 tokens 8.0 / 9.5 us, a window of 4096 of 8 kv-heads in 11 splits 9.9 / 11.2, four sequences of up
// to 32788 27.4 / 29.1, 32 heads x 4100 in 8 splits 13.0 / 12.8; where no sequence turns out to be split (8 sequences x 52 heads)
// the kernel would be launched for nothing.
constexpr int64_t FP4_MERGED_ROWS = 256;

int launch_fp4_attention(const kv_fp4_cache *c, const Fp4View &v, const void *q, int64_t q_stride, bool bf16, float sm_scale,
                         int window, int sinks, void *out, int out_type, float *lse, hipStream_t s) {
    const int64_t columns = int64_t(v.batch.max_new) * v.G;
    if (columns > (int64_t(1) << 30)) return KV_ERR_UNSUPPORTED;
    Fp4Attention a;
    a.v = v;
    a.q = static_cast<const uint16_t *>(q);
    a.q_stride = q_stride;
    a.scale = Fp4Scale::of(sm_scale * FP4_LOG2E);
    a.window = window, a.sinks = sinks;
    a.out = out, a.out_type = out_type, a.lse = lse;
    const int batch = v.batch.batch;
    const int64_t tiles = (columns + FP4_TILE_COLUMNS - 1) / FP4_TILE_COLUMNS, passes = (columns + FP4_COLUMNS - 1) / FP4_COLUMNS;
    int64_t pages = v.batch.table_pages;
    if (window) pages = std::min(pages, (int64_t(window) + FP4_TILE_COLUMNS + sinks) / FP4_PAGE + 3);
    const int64_t tile_groups = tiles * v.H * batch;
    a.width = 11 * tiles < 2 * passes && (tile_groups >= 384 || (tile_groups >= 16 && pages >= 256)) ? FP4_TILE_COLUMNS : FP4_COLUMNS;
    a.blocks = int((columns + a.width - 1) / a.width);
    a.rows = int(std::min<int64_t>(columns, a.width));
    // Steps that a block of columns can have.
    const int unit = a.width == FP4_TILE_COLUMNS ? FP4_PAGE : FP4_STEP;
    const int64_t most = pages * (FP4_PAGE / unit);
    const int64_t streams = int64_t(a.blocks) * v.H, room = FP4_PART_ROWS / a.rows / streams;   // workgroups that the workspace takes
    a.least_steps = a.width == FP4_TILE_COLUMNS ? FP4_LEAST_PAGES : streams * batch * (most / FP4_LEAST_STEPS) <= FP4_FEW_GROUPS ? FP4_LEAST_STEPS : FP4_MORE_STEPS;
    const int64_t useful = (most + a.least_steps - 1) / a.least_steps;       // splits of a sequence
    const int chunk = std::min(batch, FP4_FLAT), chunks = (batch + FP4_FLAT - 1) / FP4_FLAT;
    const int64_t want = FP4_GROUPS / streams, more = FP4_MORE_GROUPS / streams;
    a.flat = batch > 1 && useful > 1 && room > 2 * chunk * chunks;   // (the workgroups are below 2^16 then)
    if (a.flat) {
        a.splits = int(std::min({std::max<int64_t>(more / chunks, 2 * chunk), chunk * (1 + useful), room / chunks}));
        a.few = int(std::max<int64_t>(want / chunks - chunk, 1));
    } else {
        a.splits = int(std::max<int64_t>(std::min({more / batch, useful, room / batch, int64_t(FP4_SPLITS_MAX)}), 1));
        a.few = int(std::max<int64_t>(want / batch, 1));
    }
    a.most_splits = FP4_SPLITS_MAX;
    const int64_t groups = int64_t(a.flat ? chunks : batch) * a.splits;
    if (a.blocks > 65535 || groups > 65535) return KV_ERR_UNSUPPORTED;
    a.counters = nullptr;
    const int64_t alone = std::min<int64_t>(64, FP4_MERGED_ROWS / a.rows), fair = std::min(useful, std::max<int64_t>(want / batch, 1));
    if (a.width == FP4_COLUMNS && a.splits > 1 && streams * batch <= FP4_COUNTERS && 2 * fair <= alone) {
        a.counters = reinterpret_cast<uint8_t *>(c->workspace);
        a.most_splits = int(alone);
    }
    a.part = c->workspace + FP4_COUNTERS / sizeof(float);
    const dim3 grid = dim3(uint32_t(v.H), uint32_t(a.blocks), uint32_t(groups));
#define LAUNCH(HD, BF) hipLaunchKernelGGL((fp4_attention_kernel<HD, BF>), grid, dim3(256), 0, s, a)
    if (a.width == FP4_TILE_COLUMNS) {
        const int rc = launch_fp4_tiles(a, grid, c->cfg.head_dim, bf16, s);
        if (rc) return rc;
    } else if (c->cfg.head_dim == 128) {
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
