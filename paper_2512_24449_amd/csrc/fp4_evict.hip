// Which tokens of the 4-bit paged cache are kept, and their rows moved together (packkv.h: kv_fp4_select, kv_fp4_compact).
#include <algorithm>

#include "fp4.h"
#include "unpack.h"

namespace packkv {

struct Fp4Select {
    Fp4View v;
    const float *mass;
    int64_t pitch;
    int keep, sinks, recent;
    const int32_t *budgets;
    int32_t *kept, *n_kept;
};

// Ordered like the weights: unsigned numbers, the two zeros equal, a NaN above all.
__device__ inline uint32_t mass_key(float x) {
    if (x != x) return 0xFFFFFFFFu;
    const uint32_t u = __float_as_uint(x + 0.0f);    // -0 + 0 = +0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// A workgroup to a (sequence, kv-head).  The weight below which nothing is kept is found digit by digit (11, 11 and 10 bits) by
// counting keys with the digits found so far; then every wave counts what it has above it and equal to it in a sixteenth of the
// tokens, and writes its positions behind those of the waves before it.
constexpr int SELECT_THREADS = 1024, SELECT_WAVES = SELECT_THREADS / 64;

__global__ __launch_bounds__(SELECT_THREADS) void fp4_select_kernel(Fp4Select a) {
    __shared__ uint32_t bins[2048];
    __shared__ uint32_t found[2], part[SELECT_WAVES], above[SELECT_WAVES], equal[SELECT_WAVES];
    const Fp4View &v = a.v;
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Fp4Sequence seq(v, b);
    const int64_t stream = int64_t(b) * v.H + h;
    const float *mass = a.mass + stream * a.pitch;
    int32_t *kept = a.kept + stream * a.keep;
    const int len = seq.held, budget = min(a.budgets ? max(a.budgets[b], 0) : a.keep, a.keep), n = min(len, budget);
    if (h == 0 && tid == 0) a.n_kept[b] = n;
    for (int i = n + tid; i < a.keep; i += SELECT_THREADS) kept[i] = -1;
    if (len <= budget) {
        for (int i = tid; i < n; i += SELECT_THREADS) kept[i] = i;
        return;
    }
    const int sinks = min(a.sinks, budget), recent = min(a.recent, budget - sinks), begin = sinks, end = len - recent;
    int wanted = budget - sinks - recent;              // of begin .. end - 1
    const auto key = [&](int t) { return mass_key(t < a.pitch ? mass[t] : 0.0f); };
    uint32_t digits = 0, mask = 0;                     // of the key that is looked for, and which are known
    if (wanted > 0) {
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, count = pass == 2 ? 1024 : 2048;
            for (int i = tid; i < 2048; i += SELECT_THREADS) bins[i] = 0;
            __syncthreads();
            for (int t = begin + tid; t < end; t += SELECT_THREADS) {
                const uint32_t x = key(t);
                if (((x ^ digits) & mask) == 0) atomicAdd(&bins[(x >> shift) & (count - 1)], 1u);
            }
            __syncthreads();
            // bins from the top: two to a thread, thread 0 the highest
            const uint32_t hi = bins[2047 - 2 * tid], lo = bins[2046 - 2 * tid];
            const uint32_t upto = uint32_t(wave_inclusive_scan(int(hi + lo)));
            if (lane == 63) part[wave] = upto;
            __syncthreads();
            uint32_t before = upto - hi - lo;
            for (int w = 0; w < wave; ++w) before += part[w];
            if (before < uint32_t(wanted) && uint32_t(wanted) <= before + hi + lo) {
                const bool in_hi = uint32_t(wanted) <= before + hi;
                found[0] = uint32_t(in_hi ? 2047 - 2 * tid : 2046 - 2 * tid);
                found[1] = in_hi ? before : before + hi;
            }
            __syncthreads();
            digits |= found[0] << shift, mask |= uint32_t(count - 1) << shift;
            wanted -= int(found[1]);                   // still wanted of those with these digits
            __syncthreads();
        }
    } else {
        digits = 0xFFFFFFFFu;
        wanted = 0;
    }
    // a wave's tokens: a sixteenth of all, in order
    const bool some = budget - sinks - recent > 0;
    const int each = ((len + SELECT_WAVES - 1) / SELECT_WAVES + 63) & ~63, from = min(wave * each, len), to = min(from + each, len);
    const auto classify = [&](int t, bool &sure, bool &tie) {
        sure = tie = false;
        if (t >= to) return;
        if (t < begin || t >= end) sure = true;
        else if (some) {
            const uint32_t x = key(t);
            sure = x > digits, tie = x == digits;
        }
    };
    uint32_t sures = 0, ties = 0;
    for (int t0 = from; t0 < to; t0 += 64) {
        bool sure, tie;
        classify(t0 + lane, sure, tie);
        sures += uint32_t(__popcll(__ballot(sure))), ties += uint32_t(__popcll(__ballot(tie)));
    }
    if (lane == 0) above[wave] = sures, equal[wave] = ties;
    __syncthreads();
    uint32_t at = 0, tied = 0;                         // kept and tied of the waves before
    for (int w = 0; w < wave; ++w) at += above[w], tied += equal[w];
    at += min(tied, uint32_t(wanted));
    const uint64_t lower = (uint64_t(1) << lane) - 1;
    for (int t0 = from; t0 < to; t0 += 64) {
        bool sure, tie;
        classify(t0 + lane, sure, tie);
        const uint64_t tie_mask = __ballot(tie);
        const bool mine = sure || (tie && tied + uint32_t(__popcll(tie_mask & lower)) < uint32_t(wanted));
        const uint64_t keep_mask = __ballot(mine);
        if (mine) kept[at + uint32_t(__popcll(keep_mask & lower))] = t0 + lane;
        at += uint32_t(__popcll(keep_mask)), tied += uint32_t(__popcll(tie_mask));
    }
}

struct Fp4Compact {
    Fp4View from, to;
    const int32_t *kept, *n_kept;
    int keep;
    const float *mass;
    int64_t pitch;
    float *mass_out;
    int64_t out_pitch;
};

// A wave to eight tokens of a kv-head where they go: a word of V's channels there takes a code from each of eight words, HD / 64
// channels to a lane.  K's rows are 8 (4) bytes to a lane.
template <int HD>
__global__ __launch_bounds__(256) void fp4_compact_kernel(Fp4Compact a, int eights) {
    using P = Fp4Block<HD>;
    constexpr int C = HD / 64, SCALES = HD / FP4_GROUP;
    const int lane = threadIdx.x & 63;
    const Fp4View &v = a.from;
    const uint32_t unit = blockIdx.x * 4 + (threadIdx.x >> 6);
    const int eight = int(unit / uint32_t(v.H)), h = int(unit - uint32_t(eight) * v.H), b = blockIdx.y;
    if (eight >= eights) return;
    const int n = min(max(a.n_kept[b], 0), a.keep), i0 = 8 * eight;
    if (i0 >= n) return;
    const Fp4Sequence to_seq(a.to, b, n, 0, 0);
    const int64_t to_page = i0 / FP4_PAGE < a.to.batch.table_pages ? to_seq.page(a.to, i0 / FP4_PAGE) : -1;
    const Fp4Sequence seq(v, b);
    const int64_t stream = int64_t(b) * v.H + h;
    // where each of the eight comes from, one to a lane (of eight, again and again)
    const int j = lane & 7;
    const int from = i0 + j < n ? a.kept[stream * a.keep + i0 + j] : -1;
    int page = -1;
    if (from >= 0 && from < seq.held) page = int(seq.page(v, from / FP4_PAGE));
    if (a.mass_out && lane < 8 && i0 + j < n && i0 + j < a.out_pitch) {
        const bool has = from >= 0 && from < a.pitch && from < seq.held;
        a.mass_out[stream * a.out_pitch + i0 + j] = has ? a.mass[stream * a.pitch + from] : 0.0f;
    }
    if (to_page < 0) return;
    uint8_t *out = v.pages + (to_page * v.H + h) * size_t(P::BYTES);
    const int at = i0 % FP4_PAGE;
    const uint8_t *mine = v.pages + (int64_t(max(page, 0)) * v.H + h) * size_t(P::BYTES);
    const int slot = from & (FP4_PAGE - 1);
    // scales: of the lane's token, group lane / 8
    if (lane / 8 < SCALES && i0 + j < n) {
        const int s = lane / 8;
        out[P::KS + (at + j) * SCALES + s] = page < 0 ? uint8_t(127) : mine[P::KS + slot * SCALES + s];
        out[P::VS + s * FP4_PAGE + at + j] = page < 0 ? uint8_t(127) : mine[P::VS + s * FP4_PAGE + slot];
    }
    // K: token lane / 8, an eighth of its row
    {
        const int t = lane / 8, part = lane & 7, p = __shfl(page, t), s = __shfl(slot, t);
        const uint8_t *row = v.pages + (int64_t(max(p, 0)) * v.H + h) * size_t(P::BYTES) + P::K + s * (HD / 2) + part * (HD / 16);
        uint8_t *to = out + P::K + (at + t) * (HD / 2) + part * (HD / 16);
        if (i0 + t < n) {
            uint32_t w[C];
#pragma unroll
            for (int c = 0; c < C; ++c) {
                w[c] = p < 0 ? 0u : reinterpret_cast<const uint32_t *>(row)[c];
                reinterpret_cast<uint32_t *>(to)[c] = w[c];
            }
        }
    }
    // V: channels C * lane .. of each of the eight
    uint32_t word[C] = {};
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        const int p = __builtin_amdgcn_readlane(page, t), s = __builtin_amdgcn_readlane(slot, t);
        if (p < 0) continue;
        const uint32_t *row = reinterpret_cast<const uint32_t *>(v.pages + (int64_t(p) * v.H + h) * size_t(P::BYTES) + P::V) + (s / 8) * HD + C * lane;
#pragma unroll
        for (int c = 0; c < C; ++c) word[c] |= ((row[c] >> (4 * (s & 7))) & 15u) << (4 * t);
    }
    uint32_t *to = reinterpret_cast<uint32_t *>(out + P::V) + (at / 8) * HD + C * lane;
#pragma unroll
    for (int c = 0; c < C; ++c) to[c] = word[c];
}

}  // namespace packkv

using namespace packkv;

extern "C" int kv_fp4_select(kv_fp4_cache_t *c, const kv_fp4_batch_t *batch, const float *mass, int64_t mass_tokens, int32_t keep,
                             const int32_t *budgets, int32_t sinks, int32_t recent, int32_t *kept, int32_t *n_kept, void *hip_stream) {
    const int rc = c ? fp4_check_batch(batch) : KV_ERR_ARG;
    if (rc) return rc;
    if (mass_tokens < 1 || keep < 1 || sinks < 0 || recent < 0) return KV_ERR_ARG;
    if (!fp4_aligned(mass, 4) || !fp4_aligned(kept, 4) || !fp4_aligned(n_kept, 4) || (budgets && !fp4_aligned(budgets, 4))) return KV_ERR_ARG;
    const Fp4Select a{fp4_view(c, batch, 0), mass, mass_tokens, keep, sinks, recent, budgets, kept, n_kept};
    hipLaunchKernelGGL(fp4_select_kernel, dim3(uint32_t(c->cfg.n_kv_heads), uint32_t(batch->batch)), dim3(SELECT_THREADS), 0,
                       static_cast<hipStream_t>(hip_stream), a);
    KV_HIP_CHECK(hipGetLastError());
    return KV_OK;
}

extern "C" int kv_fp4_compact(kv_fp4_cache_t *c, const kv_fp4_batch_t *from, const kv_fp4_batch_t *to, const int32_t *kept, int32_t keep,
                              const int32_t *n_kept, const float *mass, int64_t mass_tokens, float *mass_out, int64_t mass_out_tokens,
                              void *hip_stream) {
    int rc = c ? fp4_check_batch(from) : KV_ERR_ARG;
    if (rc == KV_OK) rc = fp4_check_batch(to);
    if (rc) return rc;
    if (from->batch != to->batch || keep < 1 || !fp4_aligned(kept, 4) || !fp4_aligned(n_kept, 4)) return KV_ERR_ARG;
    if (!mass != !mass_out) return KV_ERR_ARG;
    if (mass && (mass_tokens < 1 || mass_out_tokens < 1 || !fp4_aligned(mass, 4) || !fp4_aligned(mass_out, 4))) return KV_ERR_ARG;
    const Fp4Compact a{fp4_view(c, from, 0), fp4_view(c, to, 0), kept, n_kept, keep, mass, mass_tokens, mass_out, mass_out_tokens};
    const int64_t eights = (int64_t(keep) + 7) / 8, groups = (eights * c->cfg.n_kv_heads + 3) / 4;
    if (groups > FP4_GROUPS_MOST) return KV_ERR_UNSUPPORTED;
    const dim3 grid = dim3(uint32_t(groups), uint32_t(from->batch));
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (c->cfg.head_dim == 128) hipLaunchKernelGGL(fp4_compact_kernel<128>, grid, dim3(256), 0, s, a, int(eights));
    else hipLaunchKernelGGL(fp4_compact_kernel<64>, grid, dim3(256), 0, s, a, int(eights));
    KV_HIP_CHECK(hipGetLastError());
    return KV_OK;
}
