// The 4-bit paged cache: host side of its entry points, and the kernels that write rows into pages and read them back.
// Format and contract are in packkv.h, the reasons for the format in fp4.h.
#include <cmath>
#include <new>

#include "fp4.h"
#include "unpack.h"

namespace packkv {

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf162_t __attribute__((ext_vector_type(2)));
typedef float float2_t __attribute__((ext_vector_type(2)));

// Both kernels move bytes: what bounds them is HBM (and, for a few tokens, three dependent memory latencies: lengths, page
// number, rows).  They give a wave a tile of 8 * 512 / HD tokens (an aligned eight per row of HD / 8 lanes) of one sequence and
// kv-head, a lane eight tokens of eight channels: its loads and stores of rows are 16 bytes, a group of 32 channels is a
// quad of lanes, and the 8 x 8 codes that V's layout turns around are the lane's own.  Neighbouring waves take neighbouring
// heads of the same tokens, which lie next to each other in the rows.  Measured, heads of 128: 8 sequences x
// 52 heads x 32000 tokens written in 1.68 ms (8.6 GB moved, 5.1 TB/s), 25077 bf16 rows of 32 heads written in 124 us
// (4.2 TB/s) and read back in 96 (5.4), 131072 rows of 8 heads read back in 145 us (4.7 TB/s): of the same
// kind as a copy, which reaches 4.7 to 5.0 here, reading and writing as much; reads alone reach 6.8, writes alone 6.9.
template <int HD>
struct Fp4Tile {
    static constexpr int ROW_LANES = HD / 8, TOKENS = 8 * 64 / ROW_LANES;
};

// 8 x 8 nibbles: nibble i of w[j] <-> nibble j of w[i].  Halves, then bytes, then nibbles of pairs of words.
__device__ inline void turn_nibbles(uint32_t (&w)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t a = w[j], b = w[j + 4];
        w[j] = __builtin_amdgcn_perm(b, a, 0x05040100);
        w[j + 4] = __builtin_amdgcn_perm(b, a, 0x07060302);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = (i & 1) | ((i & 2) << 1);
        const uint32_t a = w[j], b = w[j + 2];
        w[j] = __builtin_amdgcn_perm(b, a, 0x06020400);
        w[j + 2] = __builtin_amdgcn_perm(b, a, 0x07030501);
    }
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
        const uint32_t a = w[j], b = w[j + 1], m = 0x0F0F0F0Fu;
        w[j] = (a & m) | ((b & m) << 4);
        w[j + 1] = ((a >> 4) & m) | (b & ~m);
    }
}

// Eight channels of a token (two to a word, fp16 or bf16) -> their codes; the byte of the scale is found over the quad of
// lanes that holds the group.  |x| as bits is ordered like |x|, NaNs above infinity.
template <bool BF16>
__device__ inline uint32_t quantize_fp4(uint32_t (&x)[4], uint32_t *scale_byte) {
    constexpr uint32_t INFINITE = BF16 ? 0x7F80u : 0x7C00u;
    auto largest = [&]() {
        uint32_t m = max16(max16(x[0] & 0x7FFF7FFFu, x[1] & 0x7FFF7FFFu), max16(x[2] & 0x7FFF7FFFu, x[3] & 0x7FFF7FFFu));
        m = max(m & 0xFFFFu, m >> 16);
        m = max(m, uint32_t(__builtin_amdgcn_update_dpp(0, int(m), DPP_QUAD_XOR1, 0xF, 0xF, false)));
        return max(m, uint32_t(__builtin_amdgcn_update_dpp(0, int(m), DPP_QUAD_XOR2, 0xF, 0xF, false)));
    };
    uint32_t m = largest();
    if (__any(m > INFINITE)) {  // a NaN somewhere: held as 0
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if ((x[i] & 0x7FFFu) > INFINITE) x[i] &= 0xFFFF0000u;
            if (((x[i] >> 16) & 0x7FFFu) > INFINITE) x[i] &= 0x0000FFFFu;
        }
        m = largest();
    }
    // least e with |x| <= 7 * 2^e = 1.75 * 2^(e + 2): the exponent less two, one more where the significand is above 1.75
    const uint32_t bits = BF16 ? m << 16 : __float_as_uint(__half2float(__ushort_as_half(uint16_t(m))));
    const int e = min(max(int((bits + 0x1FFFFFu) >> 23) - 2, FP4_E_LEAST), FP4_E_MOST);
    *scale_byte = uint32_t(e);
    const float scale = __uint_as_float(uint32_t(e) << 23);
    // to nearest, ties to the even code, above 6 (infinities too) 6
    uint32_t w = 0;
    if constexpr (BF16) {
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf162_t, x[0]), scale, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf162_t, x[1]), scale, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf162_t, x[2]), scale, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf162_t, x[3]), scale, 3);
    } else {
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(half2_t, x[0]), scale, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(half2_t, x[1]), scale, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(half2_t, x[2]), scale, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(half2_t, x[3]), scale, 3);
    }
    return w;
}

template <int HD, bool BF16>
__global__ __launch_bounds__(256) void fp4_append_kernel(Fp4View v, const uint16_t *__restrict__ k, int64_t k_stride,
                                                         const uint16_t *__restrict__ vv, int64_t v_stride, int tiles) {
    using T = Fp4Tile<HD>;
    using P = Fp4Block<HD>;
    const int lane = threadIdx.x & 63;
    const uint32_t unit = blockIdx.x * 4 + (threadIdx.x >> 6);
    const int tile = int(unit / uint32_t(v.H)), h = int(unit - tile * v.H), b = blockIdx.y;
    if (tile >= tiles) return;
    const Fp4Sequence seq(v, b);
    const int begin = max(seq.pos0, 0);                        // first position of the sequence that is written
    const int64_t start = (int64_t(begin / T::TOKENS) + tile) * T::TOKENS;
    if (start >= seq.held || seq.n == 0) return;               // (wave-uniform)
    const int t0 = int(start);                                 // first position of the tile
    const int64_t page = seq.page(v, t0 / FP4_PAGE);
    if (page < 0) return;
    uint8_t *block = v.pages + (page * v.H + h) * size_t(P::BYTES);
    const int cl = lane % T::ROW_LANES;                        // channels 8 cl ..
    const int t8 = t0 + 8 * (lane / T::ROW_LANES), at8 = t8 % FP4_PAGE;

    uint32_t live = 0;                                         // bit j: token t8 + j is written
    uint4 kr[8], vr[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int t = t8 + j;
        const int64_t row = seq.first + (t - seq.pos0);
        kr[j] = vr[j] = make_uint4(0, 0, 0, 0);
        if (t >= begin && t < seq.held && row >= 0 && row < v.n_rows) {
            live |= 1u << j;
            kr[j] = *reinterpret_cast<const uint4 *>(k + row * k_stride + int64_t(h) * HD + 8 * cl);
            vr[j] = *reinterpret_cast<const uint4 *>(vv + row * v_stride + int64_t(h) * HD + 8 * cl);
        }
    }
    // V: a word to a channel; where some of the eight tokens are not written, they keep their codes (read with the rows, not after)
    uint4 *to = reinterpret_cast<uint4 *>(block + P::V + ((at8 / 8) * HD + 8 * cl) * 4);
    uint4 old0 = make_uint4(0, 0, 0, 0), old1 = old0;
    if (live != 0 && live != 0xFFu) old0 = to[0], old1 = to[1];
    uint32_t word[8], scale[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint32_t x[4] = {kr[j].x, kr[j].y, kr[j].z, kr[j].w};
        const uint32_t w = quantize_fp4<BF16>(x, &scale[0]);
        if ((live >> j) & 1u) {
            *reinterpret_cast<uint32_t *>(block + P::K + (at8 + j) * (HD / 2) + 4 * cl) = w;
            if (cl % 4 == 0) block[P::KS + (at8 + j) * (HD / FP4_GROUP) + cl / 4] = uint8_t(scale[0]);
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint32_t x[4] = {vr[j].x, vr[j].y, vr[j].z, vr[j].w};
        word[j] = quantize_fp4<BF16>(x, &scale[j]);
    }
    if (!live) return;
    turn_nibbles(word);
    uint8_t *scales = block + P::VS + (cl / 4) * FP4_PAGE + at8;
    if (live == 0xFFu) {
        to[0] = make_uint4(word[0], word[1], word[2], word[3]);
        to[1] = make_uint4(word[4], word[5], word[6], word[7]);
        if (cl % 4 == 0)
            *reinterpret_cast<uint2 *>(scales) = make_uint2(scale[0] | scale[1] << 8 | scale[2] << 16 | scale[3] << 24,
                                                            scale[4] | scale[5] << 8 | scale[6] << 16 | scale[7] << 24);
    } else {
        uint32_t mask = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) mask |= ((live >> j) & 1u) ? 0xFu << (4 * j) : 0u;
        auto join = [&](uint32_t old, uint32_t now) { return (old & ~mask) | (now & mask); };
        to[0] = make_uint4(join(old0.x, word[0]), join(old0.y, word[1]), join(old0.z, word[2]), join(old0.w, word[3]));
        to[1] = make_uint4(join(old1.x, word[4]), join(old1.y, word[5]), join(old1.z, word[6]), join(old1.w, word[7]));
        if (cl % 4 == 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if ((live >> j) & 1u) scales[j] = uint8_t(scale[j]);
        }
    }
}

// Eight codes of a token -> eight values of `TYPE` at `to`: one conversion to two values.
template <int TYPE>
__device__ inline void store_values(void *to, uint32_t w, float scale) {
    if constexpr (TYPE == KV_TYPE_FP32) {
        float4 *f = static_cast<float4 *>(to);
        const float2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
        const float2_t c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
        f[0] = make_float4(a.x, a.y, b.x, b.y);
        f[1] = make_float4(c.x, c.y, d.x, d.y);
    } else if constexpr (TYPE == KV_TYPE_BF16) {
        *static_cast<uint4 *>(to) = make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)),
                                               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
                                               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)),
                                               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3)));
    } else {
        *static_cast<uint4 *>(to) = make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 0)),
                                               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 1)),
                                               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 2)),
                                               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 3)));
    }
}

// The tile's rows that are not held (positions below 0 or behind the table, missing pages) come out as zeros: their codes
// are taken as 0.
template <int HD, int TYPE>
__global__ __launch_bounds__(256) void fp4_read_kernel(Fp4View v, uint8_t *__restrict__ k, uint8_t *__restrict__ vv, int tiles) {
    using T = Fp4Tile<HD>;
    using P = Fp4Block<HD>;
    constexpr int SIZE = TYPE == KV_TYPE_FP32 ? 4 : 2;
    const int lane = threadIdx.x & 63;
    const uint32_t unit = blockIdx.x * 4 + (threadIdx.x >> 6);
    const int tile = int(unit / uint32_t(v.H)), h = int(unit - tile * v.H), b = blockIdx.y;
    if (tile >= tiles) return;
    const Fp4Sequence seq(v, b);
    // positions may be negative here: tiles are aligned to multiples of TOKENS below them too
    const int64_t t0 = (seq.pos0 & ~(T::TOKENS - 1)) + int64_t(tile) * T::TOKENS;
    if (t0 >= seq.len) return;
    const int64_t page = t0 >= 0 && t0 < seq.held ? seq.page(v, int(t0 / FP4_PAGE)) : -1;
    const uint8_t *block = v.pages + ((page < 0 ? 0 : page) * v.H + h) * size_t(P::BYTES);
    const int cl = lane % T::ROW_LANES;
    const int64_t t8 = t0 + 8 * (lane / T::ROW_LANES);
    const int at8 = int(t8 & (FP4_PAGE - 1));
    const bool held8 = page >= 0 && t8 < seq.held;             // (held may end inside the eight: only where len does)
    const int64_t row8 = seq.first + (t8 - seq.pos0);
    const int64_t pitch = int64_t(v.H) * HD * SIZE, column = (int64_t(h) * HD + 8 * cl) * SIZE;
    auto asked = [&](int j) { return t8 + j >= seq.pos0 && t8 + j < seq.len && row8 + j >= 0 && row8 + j < v.n_rows; };
    if (k) {
        uint32_t w[8], s[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            w[j] = held8 ? *reinterpret_cast<const uint32_t *>(block + P::K + (at8 + j) * (HD / 2) + 4 * cl) : 0u;
            s[j] = held8 ? block[P::KS + (at8 + j) * (HD / FP4_GROUP) + cl / 4] : 127u;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (asked(j)) store_values<TYPE>(k + (row8 + j) * pitch + column, w[j], __uint_as_float(s[j] << 23));
    }
    if (vv) {
        uint4 a = make_uint4(0, 0, 0, 0), c = a;
        uint2 s = make_uint2(0x7F7F7F7Fu, 0x7F7F7F7Fu);
        if (held8) {
            const uint4 *from = reinterpret_cast<const uint4 *>(block + P::V + ((at8 / 8) * HD + 8 * cl) * 4);
            a = from[0], c = from[1];
            s = *reinterpret_cast<const uint2 *>(block + P::VS + (cl / 4) * FP4_PAGE + at8);
        }
        uint32_t w[8] = {a.x, a.y, a.z, a.w, c.x, c.y, c.z, c.w};
        turn_nibbles(w);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (asked(j))
                store_values<TYPE>(vv + (row8 + j) * pitch + column, w[j],
                                   __uint_as_float((((j < 4 ? s.x : s.y) >> (8 * (j & 3))) & 255u) << 23));
    }
}

// Tiles of `tokens` tokens that a sequence's new rows can touch, wherever they begin.
inline int tiles_touched(int max_new, int tokens) { return int((int64_t(max_new) + tokens - 2) / tokens) + 1; }

int launch_fp4_append(const kv_fp4_cache *c, const Fp4View &v, const void *k, int64_t k_stride, const void *vv, int64_t v_stride,
                      bool bf16, hipStream_t s) {
    const int tiles = tiles_touched(v.batch.max_new, c->cfg.head_dim == 128 ? Fp4Tile<128>::TOKENS : Fp4Tile<64>::TOKENS);
    const int64_t groups = (int64_t(tiles) * v.H + 3) / 4;
    if (groups > FP4_GROUPS_MOST) return KV_ERR_UNSUPPORTED;
    const dim3 grid = dim3(uint32_t(groups), uint32_t(v.batch.batch));
#define LAUNCH(HD, BF)                                                                                                    \
    hipLaunchKernelGGL((fp4_append_kernel<HD, BF>), grid, dim3(256), 0, s, v, static_cast<const uint16_t *>(k), \
                       k_stride, static_cast<const uint16_t *>(vv), v_stride, tiles)
    if (c->cfg.head_dim == 128) {
        if (bf16) LAUNCH(128, true); else LAUNCH(128, false);
    } else {
        if (bf16) LAUNCH(64, true); else LAUNCH(64, false);
    }
#undef LAUNCH
    KV_HIP_CHECK(hipGetLastError());
    return KV_OK;
}

int launch_fp4_read(const kv_fp4_cache *c, const Fp4View &v, void *k, void *vv, int type, hipStream_t s) {
    const int tiles = tiles_touched(v.batch.max_new, c->cfg.head_dim == 128 ? Fp4Tile<128>::TOKENS : Fp4Tile<64>::TOKENS);
    const int64_t groups = (int64_t(tiles) * v.H + 3) / 4;
    if (groups > FP4_GROUPS_MOST) return KV_ERR_UNSUPPORTED;
    const dim3 grid = dim3(uint32_t(groups), uint32_t(v.batch.batch));
#define LAUNCH(HD, TYPE)                                                                                                  \
    hipLaunchKernelGGL((fp4_read_kernel<HD, TYPE>), grid, dim3(256), 0, s, v, static_cast<uint8_t *>(k), \
                       static_cast<uint8_t *>(vv), tiles)
#define LAUNCH_TYPE(HD)                                                     \
    switch (type) {                                                         \
        case KV_TYPE_FP16: LAUNCH(HD, KV_TYPE_FP16); break;                 \
        case KV_TYPE_BF16: LAUNCH(HD, KV_TYPE_BF16); break;                 \
        default: LAUNCH(HD, KV_TYPE_FP32); break;                           \
    }
    if (c->cfg.head_dim == 128) {
        LAUNCH_TYPE(128)
    } else {
        LAUNCH_TYPE(64)
    }
#undef LAUNCH_TYPE
#undef LAUNCH
    KV_HIP_CHECK(hipGetLastError());
    return KV_OK;
}

}  // namespace packkv

using namespace packkv;

namespace {

int check_config(const kv_fp4_config_t *c) {
    if (!c || c->n_kv_heads < 1 || c->n_q_heads < 1 || c->n_pages < 1 || c->n_pages > 0x7FFFFFFF) return KV_ERR_ARG;
    if (c->n_q_heads % c->n_kv_heads) return KV_ERR_ARG;
    if (c->head_dim != 128 && c->head_dim != 64) return KV_ERR_UNSUPPORTED;
    if (c->n_q_heads > 65535) return KV_ERR_UNSUPPORTED;
    return KV_OK;
}

}  // namespace

extern "C" int kv_fp4_query_sizes(const kv_fp4_config_t *cfg, kv_fp4_sizes_t *out) {
    const int rc = check_config(cfg);
    if (rc) return rc;
    if (!out) return KV_ERR_ARG;
    const size_t page = size_t(cfg->n_kv_heads) * fp4_block_bytes(cfg->head_dim);   // below 2^30
    if (size_t(cfg->n_pages) > (size_t(1) << 46) / page) return KV_ERR_UNSUPPORTED;
    out->pages = size_t(cfg->n_pages) * page;
    out->workspace = fp4_workspace_bytes(cfg->head_dim);
    return KV_OK;
}

extern "C" int kv_fp4_cache_create(const kv_fp4_config_t *cfg, void *pages, void *workspace, const kv_fp4_sizes_t *sizes,
                                   kv_fp4_cache_t **out) {
    kv_fp4_sizes_t need;
    const int rc = kv_fp4_query_sizes(cfg, &need);
    if (rc) return rc;
    if (!sizes || !out || !fp4_aligned(pages, 256) || !fp4_aligned(workspace, 256)) return KV_ERR_ARG;
    if (sizes->pages < need.pages || sizes->workspace < need.workspace) return KV_ERR_ARG;
    kv_fp4_cache *c = new (std::nothrow) kv_fp4_cache;
    if (!c) return KV_ERR_ARG;
    c->cfg = *cfg;
    c->pages = static_cast<uint8_t *>(pages);
    c->workspace = static_cast<float *>(workspace);
    int made = launch_fp4_clear(c, nullptr);
    if (made == KV_OK && hipStreamSynchronize(nullptr) != hipSuccess) made = KV_ERR_HIP;
    if (made) {
        delete c;
        return made;
    }
    *out = c;
    return KV_OK;
}

extern "C" int kv_fp4_cache_destroy(kv_fp4_cache_t *cache) {
    if (!cache) return KV_ERR_ARG;
    delete cache;
    return KV_OK;
}

extern "C" int kv_fp4_append(kv_fp4_cache_t *c, const kv_fp4_batch_t *batch, const void *k, int64_t k_stride, const void *v,
                             int64_t v_stride, int32_t type, int64_t n_rows, void *hip_stream) {
    const int rc = c ? fp4_check_batch(batch) : KV_ERR_ARG;
    if (rc) return rc;
    if (n_rows < 0 || (type != KV_TYPE_FP16 && type != KV_TYPE_BF16)) return KV_ERR_ARG;
    const int64_t width = int64_t(c->cfg.n_kv_heads) * c->cfg.head_dim;
    if (k_stride < width || v_stride < width || k_stride % 8 || v_stride % 8) return KV_ERR_ARG;
    if (n_rows == 0 || batch->max_new == 0) return KV_OK;
    if (!fp4_aligned(k, 16) || !fp4_aligned(v, 16)) return KV_ERR_ARG;
    return launch_fp4_append(c, fp4_view(c, batch, n_rows), k, k_stride, v, v_stride, type == KV_TYPE_BF16,
                             static_cast<hipStream_t>(hip_stream));
}

extern "C" int kv_fp4_read(kv_fp4_cache_t *c, const kv_fp4_batch_t *batch, void *k, void *v, int32_t type, int64_t n_rows,
                           void *hip_stream) {
    const int rc = c ? fp4_check_batch(batch) : KV_ERR_ARG;
    if (rc) return rc;
    if (n_rows < 0 || type < KV_TYPE_FP16 || type > KV_TYPE_FP32) return KV_ERR_ARG;
    if (n_rows == 0 || batch->max_new == 0) return KV_OK;
    if ((!k && !v) || (k && !fp4_aligned(k, 16)) || (v && !fp4_aligned(v, 16))) return KV_ERR_ARG;
    return launch_fp4_read(c, fp4_view(c, batch, n_rows), k, v, type, static_cast<hipStream_t>(hip_stream));
}

extern "C" int kv_fp4_attention(kv_fp4_cache_t *c, const kv_fp4_batch_t *batch, const void *q, int64_t q_stride, int32_t type,
                                int64_t n_rows, float sm_scale, int32_t window, int32_t sinks, void *out, int32_t out_type,
                                float *lse, void *hip_stream) {
    const int rc = c ? fp4_check_batch(batch) : KV_ERR_ARG;
    if (rc) return rc;
    if (n_rows < 0 || (type != KV_TYPE_FP16 && type != KV_TYPE_BF16) || out_type < KV_TYPE_FP16 || out_type > KV_TYPE_FP32)
        return KV_ERR_ARG;
    if (!std::isfinite(sm_scale * FP4_LOG2E) || window < 0 || sinks < 0) return KV_ERR_ARG;
    if (q_stride < int64_t(c->cfg.n_q_heads) * c->cfg.head_dim || q_stride % 8) return KV_ERR_ARG;
    if (n_rows == 0 || batch->max_new == 0) return KV_OK;
    if (!fp4_aligned(q, 16) || !fp4_aligned(out, 16) || (lse && !fp4_aligned(lse, 4))) return KV_ERR_ARG;
    return launch_fp4_attention(c, fp4_view(c, batch, n_rows), q, q_stride, type == KV_TYPE_BF16, sm_scale, window, sinks, out,
                                out_type, lse, static_cast<hipStream_t>(hip_stream));
}
