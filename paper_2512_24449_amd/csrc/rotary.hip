// Rotary positions of query and key rows (packkv.h: kv_rotary): pair i of a head's first `dims` channels is turned by position
// times frequency i and multiplied by a constant,
//   (x, y) -> m (x cos a - y sin a, y cos a + x sin a),  a = 2 pi p t_i.
//
// The angle is found in whole numbers: t_i is given in 2^-64 of a turn, the product with the position is taken modulo a turn by
// 64-bit arithmetic that does so by itself, and of its fraction the upper 32 bits are used: so far the angle is off by 2^-32 of a
// turn, and by the position times what t_i is (a product in fp32 is off by a tenth of a radian at a million).  Two bits say the quarter;
// the rest, at most an eighth of a turn, becomes radians in fp32, by three roundings: 3 * 2^-24 * pi / 4 = 1.4e-7 at most, at any position.  Its
// sine and cosine are their power series up to the 9th and 10th power (remainders below 2e-9 and 2e-10).
#include <algorithm>
#include <cmath>

#include "common.h"
#include "overlap.h"

namespace packkv {

typedef uint32_t uint4_t __attribute__((ext_vector_type(4)));

struct Rotary {
    const void *q, *k;
    void *q_out, *k_out;
    int64_t q_stride, k_stride, q_out_stride, k_out_stride;   // of rows, in values
    int q_heads, heads;          // of q; of both
    const int32_t *positions;
    int64_t n_rows;
    const uint64_t *turns;
    int head_dim, dims;
    float magnitude, sign;       // sign: of the angle
    int units, slots;            // vector pairs of a head that are moved; slots of a workgroup
    int splits;                  // slots of a row: slot s takes heads s, s + splits, ..
};

// Sine and cosine of `fraction` * 2^-32 turns.
__device__ inline void sin_cos(uint32_t fraction, float *s, float *c) {
    const uint32_t quarter = (fraction + 0x20000000u) >> 30;
    const float x = float(int32_t(fraction - (quarter << 30))) * 1.4629180792671596e-9f;   // 2 pi 2^-32
    const float z = x * x;
    float a = fmaf(z, 2.7557319e-6f, -1.9841270e-4f), b = fmaf(z, -2.7557319e-7f, 2.4801587e-5f);   // 1/9!, 1/7!; 1/10!, 1/8!
    a = fmaf(z, a, 8.3333333e-3f), b = fmaf(z, b, -1.3888889e-3f);
    a = fmaf(z, a, -1.6666667e-1f), b = fmaf(z, b, 4.1666667e-2f);
    b = fmaf(z, b, -0.5f);
    a = fmaf(x * z, a, x), b = fmaf(z, b, 1.0f);
    const float sine = quarter & 1u ? b : a, cosine = quarter & 1u ? a : b;
    *s = quarter & 2u ? -sine : sine;
    *c = (quarter + 1u) & 2u ? -cosine : cosine;
}

template <typename T, int N>
struct alignas(sizeof(T) * N) Values {
    T x[N];
};

// A slot is `units` threads, each with two vectors of V values: V pairs.  A thread keeps its sines and cosines for all
// heads of its slot.  Vectors behind the turned channels are copied.  STREAMED: outputs that no cache holds are stored past them.
template <typename T, int V, bool INTERLEAVED, bool STREAMED>
__global__ __launch_bounds__(256) void rotary_kernel(Rotary r) {
    const int slot = int(threadIdx.x) / r.units, unit = int(threadIdx.x) - slot * r.units;
    const int64_t at = int64_t(blockIdx.x) * r.slots + slot;
    const int64_t row = at / r.splits;
    const int split = int(at - row * r.splits);
    if (slot >= r.slots || row >= r.n_rows) return;
    const int pairs = V * unit;                          // first pair of the unit
    const bool turned = 2 * pairs < r.dims;
    // where the two vectors are in a head
    const int a = turned && !INTERLEAVED ? pairs : 2 * pairs, b = turned && !INTERLEAVED ? r.dims / 2 + pairs : 2 * pairs + V;
    float s[V], c[V];
    if (turned) {
        const int64_t position = r.positions[row];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            sin_cos(uint32_t((uint64_t(position) * r.turns[pairs + j]) >> 32), &s[j], &c[j]);
            s[j] *= r.magnitude * r.sign, c[j] *= r.magnitude;
        }
    }
    for (int head = split; head < r.heads; head += r.splits) {
        const bool of_k = head >= r.q_heads;
        const int h = of_k ? head - r.q_heads : head;
        const T *from = static_cast<const T *>(of_k ? r.k : r.q) + row * (of_k ? r.k_stride : r.q_stride) + int64_t(h) * r.head_dim;
        T *to = static_cast<T *>(of_k ? r.k_out : r.q_out) + row * (of_k ? r.k_out_stride : r.q_out_stride) + int64_t(h) * r.head_dim;
        Values<T, V> u = *reinterpret_cast<const Values<T, V> *>(from + a), w = *reinterpret_cast<const Values<T, V> *>(from + b);
        if (turned) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                T &first = INTERLEAVED ? (2 * j < V ? u.x[2 * j % V] : w.x[2 * j % V]) : u.x[j];
                T &second = INTERLEAVED ? (2 * j + 1 < V ? u.x[(2 * j + 1) % V] : w.x[(2 * j + 1) % V]) : w.x[j];
                const float x = float(first), y = float(second);
                first = T(fmaf(x, c[j], -(y * s[j])));
                second = T(fmaf(y, c[j], x * s[j]));
            }
        }
        if constexpr (STREAMED) {
            __builtin_nontemporal_store(__builtin_bit_cast(uint4_t, u), reinterpret_cast<uint4_t *>(to + a));
            __builtin_nontemporal_store(__builtin_bit_cast(uint4_t, w), reinterpret_cast<uint4_t *>(to + b));
        } else {
            *reinterpret_cast<Values<T, V> *>(to + a) = u;
            *reinterpret_cast<Values<T, V> *>(to + b) = w;
        }
    }
}

// A row is spread over so many slots (if it has as many heads), and more in a call of few rows: sines are found anew in each, which
// costs less than fewer threads do.  25077 bf16 rows of 40 heads (514 MB moved) with 8 / 20 / 40 slots to a row 98.7 / 93.9 / 93.8 us.
// Outputs of 128 MB or more, half of the last-level cache, are stored past the caches where pairs are halves apart: those rows 88.5 us
// (5.8 TB/s; a copy reaches 4.7 to 5.0) for 93.2, fp32 178.5 for 184.7.  Interleaved pairs are stored by 16 bytes with as many between, which
// the caches join: past them 120.7 us for 99.6, fp32 191.5 for 189.0.
constexpr int64_t ROTARY_SPLITS = 20, ROTARY_SLOTS = 16384, ROTARY_STREAMED = int64_t(1) << 27;

template <typename T, int V>
int launch_rotary(const Rotary &r, bool interleaved, bool streamed, int64_t groups, hipStream_t s) {
    constexpr bool WIDE = sizeof(T) * V == 16;
#define LAUNCH(I, S) hipLaunchKernelGGL((rotary_kernel<T, V, I, S>), dim3(uint32_t(groups)), dim3(256), 0, s, r)
    if (interleaved) LAUNCH(true, false);
    else if (WIDE && streamed) LAUNCH(false, WIDE);
    else LAUNCH(false, false);
#undef LAUNCH
    KV_HIP_CHECK(hipGetLastError());
    return KV_OK;
}

}  // namespace packkv

using namespace packkv;

extern "C" int kv_rotary(const kv_rotary_t *rotary, const int32_t *positions, int64_t n_rows, int32_t type, int32_t inverse,
                         const void *q, int64_t q_stride, int32_t n_q_heads, void *q_out, int64_t q_out_stride, const void *k,
                         int64_t k_stride, int32_t n_k_heads, void *k_out, int64_t k_out_stride, void *hip_stream) {
    if (!rotary || n_rows < 0 || type < KV_TYPE_FP16 || type > KV_TYPE_FP32) return KV_ERR_ARG;
    const int D = rotary->head_dim, dims = rotary->dims;
    if (D < 2 || D % 2 || dims < 2 || dims % 2 || dims > D || !std::isfinite(rotary->magnitude)) return KV_ERR_ARG;
    if (n_q_heads < 0 || n_k_heads < 0 || (n_q_heads == 0 && n_k_heads == 0)) return KV_ERR_ARG;
    if (D > 512 || n_q_heads > 65535 || n_k_heads > 65535) return KV_ERR_UNSUPPORTED;
    const uintptr_t size = type == KV_TYPE_FP32 ? 4 : 2;
    const struct { const void *in; void *out; int64_t in_stride, out_stride; int heads; } both[2] = {
        {q, q_out, q_stride, q_out_stride, n_q_heads}, {k, k_out, k_stride, k_out_stride, n_k_heads}};
    uintptr_t bits = uintptr_t(dims) / 2 | uintptr_t(D - dims) / 2;   // what a vector has to divide, in values
    bool in_place = true;
    for (const auto &t : both)
        if (t.heads && (t.in_stride < int64_t(t.heads) * D || t.out_stride < int64_t(t.heads) * D)) return KV_ERR_ARG;
    if (n_rows == 0) return KV_OK;
    for (const auto &t : both) {
        if (!t.heads) continue;
        const uintptr_t in = reinterpret_cast<uintptr_t>(t.in), out = reinterpret_cast<uintptr_t>(t.out);
        if (!in || !out || in % size || out % size) return KV_ERR_ARG;
        bits |= in / size | out / size | uintptr_t(t.in_stride) | uintptr_t(t.out_stride) | uintptr_t(D);
        in_place = in_place && in == out && t.in_stride == t.out_stride;
    }
    const uintptr_t table = reinterpret_cast<uintptr_t>(rotary->turns), at = reinterpret_cast<uintptr_t>(positions);
    if (!table || table % 8 || !at || at % 4) return KV_ERR_ARG;
    int width = int(16 / size);
    while (width > 1 && bits % uintptr_t(width)) width /= 2;

    Rotary r{q, k, q_out, k_out, q_stride, k_stride, q_out_stride, k_out_stride, n_q_heads, n_q_heads + n_k_heads, positions, n_rows,
             rotary->turns, D, dims, rotary->magnitude, inverse ? -1.0f : 1.0f, 0, 0, 0};
    r.units = (in_place ? dims : D) / (2 * width);
    r.slots = 256 / r.units;
    // A launch takes fewer than 2^32 threads: beyond, fewer slots to a row.
    const int64_t slots = r.slots * ((int64_t(1) << 24) - 1);
    if (n_rows > slots) return KV_ERR_UNSUPPORTED;
    r.splits = int(std::min<int64_t>({r.heads, std::max<int64_t>(ROTARY_SPLITS, ROTARY_SLOTS / n_rows), slots / n_rows}));
    const int64_t groups = (n_rows * r.splits + r.slots - 1) / r.slots;
    const auto rows = [&](const void *p, int64_t stride, int heads) {
        return Rows(p, Rows::Wide(heads) * D * size, Rows::Wide(stride) * size, heads ? n_rows : 0);
    };
    const Rows in[2] = {rows(q, q_stride, n_q_heads), rows(k, k_stride, n_k_heads)};
    const Rows out[2] = {rows(q_out, q_out_stride, n_q_heads), rows(k_out, k_out_stride, n_k_heads)};
    for (int i = 0; i < 2; ++i) {
        const bool own = both[i].in == both[i].out && (n_rows == 1 || both[i].in_stride == both[i].out_stride);
        if ((!own && overlap(out[i], in[i])) || overlap(out[i], {in[1 - i], Rows(positions, n_rows, 4), Rows(rotary->turns, dims / 2, 8)}))
            return KV_ERR_ARG;
    }
    if (overlap(out[0], out[1])) return KV_ERR_ARG;
    const bool streamed = n_rows * r.heads * int64_t(D) * int64_t(size) >= ROTARY_STREAMED;
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const bool i = rotary->interleaved != 0;
#define WIDTHS(T)                                                    \
    switch (width) {                                                 \
        case 1: return launch_rotary<T, 1>(r, i, streamed, groups, s);         \
        case 2: return launch_rotary<T, 2>(r, i, streamed, groups, s);         \
        case 4: return launch_rotary<T, 4>(r, i, streamed, groups, s);         \
        default: break;                                              \
    }
    if (type == KV_TYPE_FP32) {
        WIDTHS(float)
    } else if (type == KV_TYPE_BF16) {
        WIDTHS(__bf16)
        return launch_rotary<__bf16, 8>(r, i, streamed, groups, s);
    } else {
        WIDTHS(_Float16)
        return launch_rotary<_Float16, 8>(r, i, streamed, groups, s);
    }
#undef WIDTHS
    return KV_ERR_ARG;
}
