// Attention over the 4-bit paged cache for many new rows (chunks of a prompt, prompts, long drafts): a workgroup takes 128
// columns, a wave 32 of them.  What a tile (a page, 64 tokens) costs once -- its transfer and its conversion to fp16 -- is shared
// by the four waves through LDS, where it lies as the operands that the products take: every wave reads 16 bytes a lane, a
// kilobyte in a row, without bank conflicts.  Two tiles in turn, one barrier each: while one is multiplied, the next is converted
// and the one after that is on its way.
//
// Bound by the vector instructions of the softmax and by the matrix cores, which share the issue: per 32 columns and page 232
// vector instructions (68 of them the conversion, 32 exponentials) and 64 products of 16 cycles; a product keeps vector instructions out
// for about 8.  2048 rows of 32 heads at 12288 (4.5e11 operations) take 446 us, 1000 TFLOP/s, where a large library product reaches
// 1345 once its clock is up; the matrix cores are busy 39 % of the time, two waves to a SIMD.
#include "fp4_attention.h"

namespace packkv {

// A wave's quarter of a tile on its way: the K of 16 tokens, the V of 32 tokens and half the channels.
template <int HD>
struct Fp4Quarter {
    using P = Fp4Block<HD>;
    static constexpr int KW = HD / 32, OT = HD / 16, VN = OT / 2;   // operands of 16 tokens' K, of 32 tokens' V; of V that a wave makes
    uint32_t k[KW], v[VN];
    uint32_t ks;
    uint2 vs;
    int t0, end;             // as of Fp4Stage

    __device__ inline void load(const uint8_t *block, int wave, int c16, int g) {
        // operand o of K or V is row o % 2 of half o / 2 of the page: tokens 8g + 4 (wave % 2) + .. of the half, its channels
        const int half = 32 * (wave >> 1), token = half + 8 * (c16 >> 2) + (c16 & 3) + 4 * (wave & 1);
        const uint8_t *kp = block + P::K + token * (HD / 2) + g * (HD / 8);
        ks = block[P::KS + token * (HD / FP4_GROUP) + g * (HD / 4) / FP4_GROUP];
        const int x = HD == 128 ? wave & 1 : 0, c = HD == 128 ? 0 : 2 * (wave & 1);   // V: 64 channels, four (two) operands of them
        const uint8_t *vp = block + P::V + half * (HD / 2) + (g * HD + 64 * x + 4 * c16 + c) * 4;
        if constexpr (HD == 128) {
            const uint4 a = *reinterpret_cast<const uint4 *>(kp), b = *reinterpret_cast<const uint4 *>(vp);
            k[0] = a.x, k[1] = a.y, k[2] = a.z, k[3] = a.w, v[0] = b.x, v[1] = b.y, v[2] = b.z, v[3] = b.w;
        } else {
            const uint2 a = *reinterpret_cast<const uint2 *>(kp), b = *reinterpret_cast<const uint2 *>(vp);
            k[0] = a.x, k[1] = a.y, v[0] = b.x, v[1] = b.y;
        }
        vs = *reinterpret_cast<const uint2 *>(block + P::VS + (2 * x + (c16 >> 3)) * FP4_PAGE + half + 8 * g);
    }
    // tile: 4 KW operands of K (64 x 16 bytes each), 2 OT of V
    template <bool BF16>
    __device__ inline void store(uint4_t (*tile)[64], int wave, int lane) const {
        const float scale = __uint_as_float(ks << 23);
#pragma unroll
        for (int i = 0; i < KW; ++i) tile[KW * wave + i][lane] = row_operand<BF16>(k[i], scale);
        half2_t scales[4];
        scale_pairs(vs, scales);
#pragma unroll
        for (int i = 0; i < VN; ++i) tile[4 * KW + VN * wave + i][lane] = column_operand(v[i], scales);
    }
};

// Page numbers of the steps to come, 64 to a register, the register after it loaded 64 steps ahead.
struct Fp4PagesAhead {
    int now, next, base;
    __device__ inline int load(const Fp4View &v, const Fp4Sequence &seq, const Fp4Steps<FP4_PAGE> &steps, int from, int end, int lane) {
        return from + lane < end ? int(seq.page(v, steps.token(from + lane) / FP4_PAGE)) : -1;
    }
    __device__ inline void start(const Fp4View &v, const Fp4Sequence &seq, const Fp4Steps<FP4_PAGE> &steps, int from, int end, int lane) {
        base = from;
        now = load(v, seq, steps, from, end, lane);
        next = load(v, seq, steps, from + 64, end, lane);
    }
    __device__ inline int at(const Fp4View &v, const Fp4Sequence &seq, const Fp4Steps<FP4_PAGE> &steps, int step, int end, int lane) {   // steps in order
        if (step - base >= 64) {
            base += 64;
            now = next;
            next = load(v, seq, steps, base + 64, end, lane);
        }
        return __builtin_amdgcn_readlane(now, step - base);
    }
};

template <int HD, bool BF16>
__global__ __launch_bounds__(256, HD == 128 ? 2 : 3) void fp4_tile_kernel(Fp4Attention a) {
    using P = Fp4Block<HD>;
    constexpr int KW = HD / 32, VH = HD / 64, OT = HD / 16, NB = FP4_TILE_COLUMNS / 64;
    __shared__ uint4_t tiles[2][4 * KW + 2 * OT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c16 = lane & 15, g = lane >> 4;
    const Fp4View &v = a.v;
    const int h = blockIdx.x, block = int(blockIdx.y), column0 = block * FP4_TILE_COLUMNS;
    const uint32_t stream = uint32_t(block) * v.H + h;
    Fp4Share<FP4_PAGE> share;
    const Fp4Sequence seq = share.find(a, int(blockIdx.z / uint32_t(a.splits)), int(blockIdx.z % uint32_t(a.splits)), 0, column0, lane);
    if (share.splits == 0) return;
    const int columns = seq.n * v.G;
    const Fp4Steps<FP4_PAGE> steps(seq, column0, FP4_TILE_COLUMNS, v.G, a.window, a.sinks);
    const int per_split = (steps.n + share.splits - 1) / share.splits;
    const int step0 = share.split * per_split, step_end = min(step0 + per_split, steps.n);

    const Fp4Scale &scale = a.scale;
    Fp4Column<HD> col[NB];
    uint4_t q[NB][KW];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        const int column = column0 + 16 * (NB * wave + n) + c16, row = column / v.G, head = h * v.G + column % v.G;
        const int64_t out_row = seq.first + row;
        const bool real = column < columns && out_row >= 0 && out_row < v.n_rows;
        col[n].hi = max(seq.pos0 + row, -1);
        col[n].clear();
#pragma unroll
        for (int i = 0; i < KW; ++i) {
            q[n][i] = uint4_t{0, 0, 0, 0};
            if (real) q[n][i] = *reinterpret_cast<const uint4_t *>(a.q + out_row * a.q_stride + int64_t(head) * HD + g * (HD / 4) + 8 * i) ^ scale.sign;
        }
    }
    // what the wave's columns see: from the first row's window (or the first tokens) to the last row
    const int wave0 = column0 + 16 * NB * wave, wave_columns = min(columns - wave0, 16 * NB);
    const int first_hi = max(seq.pos0 + wave0 / v.G, -1), last_hi = max(seq.pos0 + (wave0 + wave_columns - 1) / v.G, -1);
    const int first_lo = a.window ? max(first_hi, 0) - a.window + 1 : 0, last_lo = a.window ? last_hi - a.window + 1 : 0;

    Fp4Quarter<HD> in;
    Fp4PagesAhead pages;
    auto fetch = [&](int step) {
        const int page = pages.at(v, seq, steps, step, step_end, lane);
        in.t0 = steps.token(step);
        in.end = page < 0 ? 0 : steps.end;
        in.load(v.pages + (int64_t(max(page, 0)) * v.H + h) * size_t(P::BYTES), wave, c16, g);
    };
    auto convert = [&](int to) {
        if (in.t0 + FP4_PAGE > in.end || in.t0 < steps.begin)
            in.vs = seen_scales(in.vs, in.t0 + 32 * (wave >> 1) + 8 * g, steps.begin, in.end, a.sinks);
        in.template store<BF16>(tiles[to], wave, lane);
    };
    int t0 = 0, end = 0;
    if (step0 < step_end) {
        pages.start(v, seq, steps, step0, step_end, lane);
        fetch(step0);
        convert(0);
        t0 = in.t0, end = in.end;
        fetch(min(step0 + 1, step_end - 1));
#pragma unroll
        for (int n = 0; n < NB; ++n) scale.settle<BF16>(q[n]);
        __syncthreads();
    }
    for (int step = step0; step < step_end; ++step) {
        const int now = (step - step0) & 1;
        convert(now ^ 1);    // (behind the last tile that one again, which nobody reads)
        const int next_t0 = in.t0, next_end = in.end;
        fetch(min(step + 2, step_end - 1));
        if (wave_columns > 0 && t0 <= last_hi && (t0 + FP4_PAGE > first_lo || t0 < a.sinks)) {
            // Operands are read ahead of the products: K's of 32 tokens, the others as those are used, V's of 32 tokens before
            // the softmax.
            const uint4_t(*tile)[64] = tiles[now];
            uint4_t f[2 * KW];
            float4_t s[NB][4];
#pragma unroll
            for (int i = 0; i < 2 * KW; ++i) f[i] = tile[i][lane];
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
#pragma unroll
                for (int n = 0; n < NB; ++n) s[n][2 * u] = s[n][2 * u + 1] = float4_t{0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < KW; ++i)
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        const uint4_t k = f[t * KW + i];
#pragma unroll
                        for (int n = 0; n < NB; ++n) s[n][2 * u + t] = product16<BF16>(k, q[n][i], s[n][2 * u + t]);
                        f[t * KW + i] = tile[(2 * u + 2 + t) * KW + i][lane];   // (behind K: V's first)
                    }
            }
            __builtin_amdgcn_s_setprio(0);
            static_assert(OT == 2 * KW, "as many operands of V for 32 tokens as of K");
            if (t0 + FP4_PAGE > min(end, first_hi + 1) || t0 < last_lo) {
#pragma unroll
                for (int n = 0; n < NB; ++n) col[n].mask(s[n], t0 + 8 * g, end, a.window, a.sinks);
            }
            uint4_t p[NB][2];
#pragma unroll
            for (int n = 0; n < NB; ++n) col[n].weigh(s[n], scale, p[n]);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < OT; ++i) {
                    const uint4_t w = f[i];
                    if (u == 0) f[i] = tile[4 * KW + OT + i][lane];
#pragma unroll
                    for (int n = 0; n < NB; ++n) col[n].o[i] = product16<false>(w, p[n][u], col[n].o[i]);
                }
            __builtin_amdgcn_s_setprio(0);
        }
        t0 = next_t0, end = next_end;
        __syncthreads();
    }

    // a lane's o[4x + c][i] is channel 64x + 16g + 4i + c of its column
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        const int column = column0 + 16 * (NB * wave + n) + c16;
        const float l = column_sum(col[n].l), m = col[n].largest();
        const int64_t out_row = seq.first + column / v.G, index = out_row * (int64_t(v.H) * v.G) + h * v.G + column % v.G;
        if (column >= columns || out_row < 0 || out_row >= v.n_rows) continue;
        float *row = a.part + (a.part_row(stream, share.b, share.first, column - column0) + int64_t(share.split) * a.rows) * (HD + 4);
        const float inverse = share.splits > 1 ? 1.0f : l > 0.0f || l != l ? 1.0f / l : 0.0f;
#pragma unroll
        for (int x = 0; x < VH; ++x) {
            float r[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) r[i] = col[n].o[4 * x + i % 4][i / 4] * inverse;
            if (share.splits > 1) store_out(row, KV_TYPE_FP32, 64 * x + 16 * g, r);
            else store_out(a.out, a.out_type, index * HD + 64 * x + 16 * g, r);
        }
        if (g == 0) {
            if (share.splits > 1) row[HD] = m, row[HD + 1] = l;
            else if (a.lse) a.lse[index] = log_sum(m, l, scale.scale);
        }
    }
}

int launch_fp4_tiles(const Fp4Attention &a, dim3 grid, int head_dim, bool bf16, hipStream_t s) {
#define LAUNCH(HD, BF) hipLaunchKernelGGL((fp4_tile_kernel<HD, BF>), grid, dim3(256), 0, s, a)
    if (head_dim == 128) {
        if (bf16) LAUNCH(128, true); else LAUNCH(128, false);
    } else {
        if (bf16) LAUNCH(64, true); else LAUNCH(64, false);
    }
#undef LAUNCH
    KV_HIP_CHECK(hipGetLastError());
    return KV_OK;
}

}  // namespace packkv
