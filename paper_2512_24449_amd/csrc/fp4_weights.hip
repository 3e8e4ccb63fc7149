// The attention weight that cached tokens get from a call's rows (packkv.h: kv_fp4_weights):
//   mass[t] = past[t] + sum over the rows that see t and the G heads of  exp(sm_scale q . k_t - lse).
// The logarithm of the softmax's sum is the attention call's, so that one pass over K does it: no maximum, no sum to wait for.
//
// Scores are S = Q K^T with the tokens as columns: a lane holds scores of one token, so the sum over rows and heads is its
// own, joined over the four lanes of a token at the end, and K's rows are read as the attention kernels read them.  Row
// 4g + i of a product is column 4i + g of the call's columns (row after row, the heads of the kv-head next to each other): with up
// to four columns a lane has one exponential to a token, not four.
#include "fp4_attention.h"

namespace packkv {

struct Fp4Weights {
    Fp4View v;
    const uint16_t *q;
    int64_t q_stride;
    const float *lse;
    Fp4Scale scale;
    int window, sinks;
    const float *past;
    float *mass;
    int64_t pitch;           // values of a (sequence, kv-head) in mass and past
};

// A wave takes a page of a kv-head past all columns.
template <int HD, bool BF16>
__global__ __launch_bounds__(256) void fp4_weights_kernel(Fp4Weights a, int page_groups) {
    using P = Fp4Block<HD>;
    constexpr int KW = HD / 32;
    const Fp4View &v = a.v;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c16 = lane & 15, g = lane >> 4;
    const int group = int(blockIdx.x / uint32_t(v.H)), h = int(blockIdx.x - uint32_t(group) * v.H), b = blockIdx.y;
    const Fp4Sequence seq(v, b);
    for (int index = 4 * group + wave; int64_t(index) * FP4_PAGE < seq.held; index += 4 * page_groups) {
        const int t0 = index * FP4_PAGE;
        const int64_t page = seq.page(v, index);
        // rows that may see a token of the page
        const int first_row = max(int(min(int64_t(t0) - seq.pos0, int64_t(seq.n))), 0);
        int end_row = seq.n;
        if (a.window && t0 >= a.sinks) end_row = int(max(min(int64_t(t0) + FP4_PAGE - 1 + a.window - seq.pos0, int64_t(seq.n)), int64_t(0)));
        float sum[4] = {0, 0, 0, 0};
        if (page >= 0 && first_row < end_row) {
            const uint8_t *block = v.pages + (page * v.H + h) * size_t(P::BYTES);
            uint4_t k[4][KW];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int token = 16 * t + c16;
                const uint32_t *from = reinterpret_cast<const uint32_t *>(block + P::K + token * (HD / 2) + g * (HD / 8));
                const float scale = __uint_as_float(uint32_t(block[P::KS + token * (HD / FP4_GROUP) + g * (HD / 4) / FP4_GROUP]) << 23);
#pragma unroll
                for (int i = 0; i < KW; ++i) k[t][i] = row_operand<BF16>(from[i], scale);
            }
            const int64_t end_column = int64_t(end_row) * v.G;
            for (int64_t column0 = int64_t(first_row) * v.G; column0 < end_column; column0 += 16) {
                const auto place = [&](int64_t column, int64_t &row, int &head) {   // false: no such row of the call's tensors
                    const int64_t of = column / v.G;
                    row = seq.first + of, head = h * v.G + int(column - of * v.G);
                    return column < end_column && row >= 0 && row < v.n_rows;
                };
                uint4_t q[KW];
                int64_t row;
                int head;
                const bool real = place(column0 + 4 * (c16 & 3) + (c16 >> 2), row, head);
#pragma unroll
                for (int i = 0; i < KW; ++i) {
                    q[i] = uint4_t{0, 0, 0, 0};
                    if (real) q[i] = *reinterpret_cast<const uint4_t *>(a.q + row * a.q_stride + int64_t(head) * HD + g * (HD / 4) + 8 * i) ^ a.scale.sign;
                }
                a.scale.settle<BF16>(q);
                float less[4];
                int hi[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int64_t column = column0 + 4 * i + g;
                    less[i] = -INFINITY, hi[i] = -1;
                    if (place(column, row, head)) {
                        const float lse = a.lse[row * (int64_t(v.H) * v.G) + head];
                        if (lse != -INFINITY) less[i] = -(lse * FP4_LOG2E);   // (-infinity: a row that sees nothing)
                        hi[i] = seq.pos0 + int(column / v.G);
                    }
                }
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    float4_t s = float4_t{0, 0, 0, 0};
#pragma unroll
                    for (int i = 0; i < KW; ++i) s = product16<BF16>(q[i], k[t][i], s);
                    const int token = t0 + 16 * t + c16;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float p = __builtin_amdgcn_exp2f(fmaf(s[i], a.scale.scale, less[i]));
                        const bool seen = (token <= hi[i]) & (token < seq.held) & ((a.window == 0) | (token > hi[i] - a.window) | (token < a.sinks));
                        sum[t] += seen ? p : 0.0f;
                    }
                }
            }
        }
        float mine = 0.0f;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const float all = column_sum(sum[t]);
            if (g == t) mine = all;
        }
        const int token = t0 + lane;     // 16g + c16
        if (token < seq.held && token < a.pitch) {
            const int64_t at = (int64_t(b) * v.H + h) * a.pitch + token;
            a.mass[at] = a.past && token < seq.pos0 ? a.past[at] + mine : mine;
        }
    }
}

int launch_fp4_weights(const kv_fp4_cache *c, const Fp4View &v, const void *q, int64_t q_stride, bool bf16, float sm_scale, int window,
                       int sinks, const float *lse, const float *past, float *mass, int64_t mass_tokens, hipStream_t s) {
    const Fp4Weights a{v, static_cast<const uint16_t *>(q), q_stride, lse, Fp4Scale::of(sm_scale * FP4_LOG2E), window, sinks,
                       past, mass, mass_tokens};
    const int64_t pages = std::min<int64_t>((v.batch.table_pages + 3) / 4, 4096);
    if (pages * v.H > FP4_GROUPS_MOST) return KV_ERR_UNSUPPORTED;
    const dim3 grid = dim3(uint32_t(pages * v.H), uint32_t(v.batch.batch));
#define LAUNCH(HD, BF) hipLaunchKernelGGL((fp4_weights_kernel<HD, BF>), grid, dim3(256), 0, s, a, int(pages))
    if (c->cfg.head_dim == 128) {
        if (bf16) LAUNCH(128, true); else LAUNCH(128, false);
    } else {
        if (bf16) LAUNCH(64, true); else LAUNCH(64, false);
    }
#undef LAUNCH
    KV_HIP_CHECK(hipGetLastError());
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
    return launch_fp4_weights(c, fp4_view(c, batch, n_rows), q, q_stride, type == KV_TYPE_BF16, sm_scale, window, sinks, lse, past, mass,
                              mass_tokens, static_cast<hipStream_t>(hip_stream));
}
