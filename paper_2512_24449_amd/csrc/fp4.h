// The 4-bit paged cache (packkv.h has its format): what its kernels share.
//
// Codes are E2M1 numbers with a power-of-two scale per 32 channels because gfx950 converts those in one instruction per two
// values, scale included, in both directions: dequantizing costs half an instruction per element (K; V one, its pairs hold
// two tokens with a scale each), against one and a half for integer codes with a scale and a minimum.  K is held token by token, the
// channels of a token next to each other: a lane's 16 bytes are the channels of one token, which is what it feeds the matrix
// cores as a row of K.  V is held by groups of eight tokens, a word to a channel: a word is what a lane feeds them as
// eight tokens of a column of V.  Neither is moved between lanes.
#pragma once

#include "common.h"

struct kv_fp4_cache {
    kv_fp4_config_t cfg;
    uint8_t *pages;
    float *workspace;
};

namespace packkv {

constexpr int FP4_PAGE = KV_FP4_PAGE_TOKENS, FP4_GROUP = KV_FP4_GROUP;
constexpr float FP4_LOG2E = 1.4426950408889634f;              // scores are scaled for powers of two
constexpr int FP4_E_LEAST = 127 - 23, FP4_E_MOST = 127 + 13;  // as held: e + 127

// Offsets inside a head's block of a page.
template <int HD>
struct Fp4Block {
    static constexpr int K = 0, KS = FP4_PAGE * HD / 2, V = KS + FP4_PAGE * HD / FP4_GROUP, VS = V + FP4_PAGE * HD / 2,
                         BYTES = VS + FP4_PAGE * HD / FP4_GROUP;
};
inline size_t fp4_block_bytes(int head_dim) { return size_t(FP4_PAGE) * (head_dim + head_dim / 16); }

// The larger of each of two unsigned 16-bit numbers.
typedef uint16_t ushort2_t __attribute__((ext_vector_type(2)));
__device__ inline uint32_t max16(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(ushort2_t, a), __builtin_bit_cast(ushort2_t, b)));
}

// What a kernel needs to know of the cache and the batch.
struct Fp4View {
    uint8_t *pages;
    int64_t n_pages;
    int H, G;                // kv-heads, query heads to each
    kv_fp4_batch_t batch;
    int64_t n_rows;          // of the call's tensors
};

// A sequence's part of the batch.
struct Fp4Sequence {
    int len, n;              // tokens, new rows
    int pos0;                // position of new row 0 (negative where there are more new rows than tokens)
    int64_t first;           // first row
    int held;                // tokens that the page table has room for
    const int32_t *table;
    int64_t base;            // number of page 0 where there is no table

    // of lens[b], new_rows[b] and first_row[b] as they stand (or would: see raw_rows and raw_first)
    __device__ inline Fp4Sequence(const Fp4View &v, int b, int raw_len, int raw_rows, int raw_first) {
        const kv_fp4_batch_t &t = v.batch;
        len = max(raw_len, 0);
        n = t.new_rows ? min(max(raw_rows, 0), t.max_new) : t.max_new;
        pos0 = len - n;
        held = int(min(int64_t(len), int64_t(t.table_pages) * FP4_PAGE));
        base = int64_t(b) * t.table_pages;
        table = t.page_table ? t.page_table + base : nullptr;
        first = t.first_row ? int64_t(raw_first) : int64_t(b) * t.max_new;
    }
    __device__ inline Fp4Sequence(const Fp4View &v, int b)
        : Fp4Sequence(v, b, v.batch.lens[b], raw_rows(v, b), raw_first(v, b)) {}
    static __device__ inline int raw_rows(const Fp4View &v, int b) { return v.batch.new_rows ? v.batch.new_rows[b] : 0; }
    static __device__ inline int raw_first(const Fp4View &v, int b) { return v.batch.first_row ? v.batch.first_row[b] : 0; }
    // Number of page i < table_pages, or -1 where it is missing.
    __device__ inline int64_t page(const Fp4View &v, int i) const {
        const int64_t p = table ? int64_t(table[i]) : base + i;
        return p >= 0 && p < v.n_pages ? p : -1;
    }
};

int launch_fp4_append(const kv_fp4_cache *c, const Fp4View &v, const void *k, int64_t k_stride, const void *vv, int64_t v_stride,
                      bool bf16, hipStream_t s);
int launch_fp4_read(const kv_fp4_cache *c, const Fp4View &v, void *k, void *vv, int type, hipStream_t s);
int launch_fp4_attention(const kv_fp4_cache *c, const Fp4View &v, const void *q, int64_t q_stride, bool bf16, float sm_scale,
                         int window, int sinks, void *out, int out_type, float *lse, hipStream_t s);
size_t fp4_workspace_bytes(int head_dim);
int launch_fp4_clear(const kv_fp4_cache *c, hipStream_t s);   // the workspace's counters, once

}  // namespace packkv
