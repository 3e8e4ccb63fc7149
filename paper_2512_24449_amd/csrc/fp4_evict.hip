// Which tokens of the 4-bit paged cache are kept, and their rows moved together (packkv.h: kv_fp4_select, kv_fp4_compact).
#include <algorithm>
#include <type_traits>

#include "fp4.h"
#include "overlap.h"
#include "unpack.h"

namespace packkv {

struct Fp4Select {
    Fp4View v;
    const float *mass;
    int64_t pitch;
    int keep, sinks, recent;
    const int32_t *budgets;
    int32_t *kept, *n_kept;
    uint32_t *space;         // of sequences in parts
    int parts;
};

// Ordered like the weights: unsigned numbers, the two zeros equal, a NaN above all.
__device__ inline uint32_t mass_key(float x) {
    if (x != x) return 0xFFFFFFFFu;
    const uint32_t u = __float_as_uint(x + 0.0f);    // -0 + 0 = +0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The weight below which nothing is kept is found digit by digit (11, 11 and 10 bits of its key) by counting keys with the digits
// found so far; of the tokens with that weight the first are kept.
constexpr int SELECT_THREADS = 1024, SELECT_WAVES = SELECT_THREADS / 64, SELECT_BINS = 2048;
__device__ constexpr int select_shift(int pass) { return pass == 0 ? 21 : pass == 1 ? 10 : 0; }
__device__ constexpr int select_bins(int pass) { return pass == 2 ? 1024 : 2048; }

// A sequence's part of a call.
struct SelectRange {
    int len, budget, n, begin, end, wanted;   // wanted: of the tokens begin .. end - 1, whose weights decide
    __device__ inline SelectRange(const Fp4Select &a, const Fp4Sequence &seq, int b) {
        len = __builtin_amdgcn_readfirstlane(seq.held);
        budget = __builtin_amdgcn_readfirstlane(min(a.budgets ? max(a.budgets[b], 0) : a.keep, a.keep)), n = min(len, budget);
        const int sinks = min(a.sinks, budget), recent = min(a.recent, budget - sinks);
        begin = sinks, end = len - recent, wanted = budget - sinks - recent;
    }
};

// Counts keys: one in a bin that many lanes share is counted for all of them.
__device__ inline void count_key(uint32_t *bins, uint32_t bin, bool counts) {
    const uint64_t all = __ballot(counts);
    if (!all) return;
    const uint32_t first = __builtin_amdgcn_readlane(bin, __builtin_ctzll(all));
    const uint64_t same = __ballot(counts && bin == first);
    if (counts && bin != first) atomicAdd(&bins[bin], 1u);
    if ((threadIdx.x & 63) == 0) atomicAdd(&bins[first], uint32_t(__popcll(same)));
}

// The bin from the top in which the wanted-th key is, and how many are above it.  The thread has bins 2047 - 2 tid and 2046 - 2 tid;
// all threads call, found and part are LDS.  Contains two barriers.
struct SelectBin {
    uint32_t bin, above;
};
__device__ inline SelectBin find_bin(uint32_t hi, uint32_t lo, uint32_t wanted, uint32_t *part, uint32_t *found) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t upto = uint32_t(wave_inclusive_scan(int(hi + lo)));
    if (lane == 63) part[wave] = upto;
    __syncthreads();
    const uint32_t waves = uint32_t(wave_inclusive_scan(lane < SELECT_WAVES ? int(part[lane]) : 0));
    const uint32_t before = upto - hi - lo + (wave ? __builtin_amdgcn_readlane(waves, (wave - 1) & 63) : 0u);
    if (before < wanted && wanted <= before + hi + lo) {
        const bool in_hi = wanted <= before + hi;
        found[0] = uint32_t(in_hi ? 2047 - 2 * tid : 2046 - 2 * tid);
        found[1] = in_hi ? before : before + hi;
    }
    __syncthreads();
    return {found[0], found[1]};
}

// Writes the positions of what is kept of 64 tokens, in order: those that are sure, and of the tied ones as many as are still wanted.
__device__ inline void write_kept(int32_t *kept, int t, bool sure, bool tie, uint32_t wanted, uint32_t &at, uint32_t &tied, int lane) {
    const uint64_t lower = (uint64_t(1) << lane) - 1, ties = __ballot(tie);
    const bool mine = sure || (tie && tied + uint32_t(__popcll(ties & lower)) < wanted);
    const uint64_t keeps = __ballot(mine);
    if (mine) kept[at + uint32_t(__popcll(keeps & lower))] = t;
    at += uint32_t(__popcll(keeps)), tied += uint32_t(__popcll(ties));
}

// A workgroup to a (sequence, kv-head), a wave to a sixteenth of the tokens, four in a row to a lane, 256 at a time.  Up to KEYS
// keys of a lane are read once and stay in registers; which of them are kept is bits of a word.  The first digit's counting takes
// no branches: what does not count is counted in a place of the lane's own.  The keys with that digit, a few per cent as a rule, go to
// LDS, where the other digits are found.  8 x 52 heads of 32000 tokens take 28 us: a workgroup some 13, of which the weights' way here
// takes 3, counting 4 (9 cycles of LDS to 64 keys), barriers and positions most of the rest, in two rounds (85 registers: one workgroup to a
// compute unit; with 64 some keys are held in scratch memory, 37 to 40 us).  Read again for every digit 36 us.
constexpr uint32_t KEY_OF_0 = 0x80000000u, KEY_OF_NONE = 0;      // (no number has the key 0, or one of its first digit)
constexpr int SELECT_LIST = 4096;
template <int KEYS>
__global__ __launch_bounds__(SELECT_THREADS, 4) void fp4_select_kernel(Fp4Select a) {
    using Bits = std::conditional_t<(KEYS > 32), uint64_t, uint32_t>;
    constexpr int CHUNKS = KEYS / 4;
    __shared__ uint32_t bins[SELECT_BINS + 64], list[SELECT_LIST];
    __shared__ uint32_t found[2], part[SELECT_WAVES], sums[2][SELECT_WAVES], listed;
    const Fp4View &v = a.v;
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Fp4Sequence seq(v, b);
    const SelectRange r(a, seq, b);
    const int64_t stream = int64_t(b) * v.H + h;
    const float *mass = a.mass + stream * a.pitch;
    int32_t *kept = a.kept + stream * a.keep;
    if (h == 0 && tid == 0) a.n_kept[b] = r.n;
    for (int64_t i = r.n + tid; i < a.keep; i += SELECT_THREADS) kept[i] = -1;
    if (r.len <= r.budget) {
        for (int i = tid; i < r.n; i += SELECT_THREADS) kept[i] = i;
        return;
    }
    const int chunks = (r.len + 256 * SELECT_WAVES - 1) / (256 * SELECT_WAVES), from = 256 * chunks * wave, t0 = from + 4 * lane;
    const int upto = int(min(int64_t(r.len), a.pitch));          // (tokens without a place have weight 0)
    typedef float four_t __attribute__((ext_vector_type(4), aligned(4)));
    const float *base = upto < 4 ? reinterpret_cast<const float *>(v.pages) : mass;
    const int last = max(upto - 4, 0);
    uint32_t key[KEYS];
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
        // (the last four there are where there would be fewer; behind the last chunk some again, which do not decide)
        const int t = t0 + 256 * min(i, chunks - 1);
        const uint32_t at = 4u * uint32_t(min(t, last));
        const four_t x = *reinterpret_cast<const four_t *>(reinterpret_cast<const char *>(base) + at);
#pragma unroll
        for (int j = 0; j < 4; ++j) key[4 * i + j] = __float_as_uint(x[j]);
        if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
    }
    if (from + 256 * chunks > upto) {                            // (wave-uniform)
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            const int t = t0 + 256 * i, past = t + 4 - upto;     // the four are `past` places too early
            uint32_t *x = key + 4 * i;
            if (past > 0) {
                x[0] = past == 1 ? x[1] : past == 2 ? x[2] : past == 3 ? x[3] : 0u;
                x[1] = past == 1 ? x[2] : past == 2 ? x[3] : 0u;
                x[2] = past == 1 ? x[3] : 0u;
                x[3] = 0u;
            }
            if (i == 0 && t == 0 && upto < 4) {
#pragma unroll
                for (int j = 0; j < 3; ++j) x[j] = j < upto ? __float_as_uint(mass[min(j, upto - 1)]) : 0u;
            }
        }
    }
    // Weights are hardly ever negative or NaN: a key is then the number's bits with the highest set.
    uint32_t largest = 0;
#pragma unroll
    for (int i = 0; i < KEYS; ++i) largest = max(largest, key[i]);
    if (__any(largest > 0x7F800000u)) {
#pragma unroll
        for (int i = 0; i < KEYS; ++i) key[i] = mass_key(__uint_as_float(key[i]));
    } else {
#pragma unroll
        for (int i = 0; i < KEYS; ++i) key[i] |= KEY_OF_0;
    }
    // Bits of the tokens that there are, and of those that decide; others have no key.
    Bits there = 4 * chunks < int(8 * sizeof(Bits)) ? (Bits(1) << (4 * chunks)) - 1 : ~Bits(0), decides = there;
    if (from < r.begin || from + 256 * chunks > r.end) {           // (wave-uniform)
        there = decides = 0;
        for (int i = 0; i < chunks; ++i) {
            const auto below = [&](int t) { return (1u << min(max(t - (t0 + 256 * i), 0), 4)) - 1; };
            there |= Bits(below(r.len)) << (4 * i), decides |= Bits(below(r.end) & ~below(r.begin)) << (4 * i);
        }
    }
    if (decides != ~Bits(0)) {
#pragma unroll
        for (int i = 0; i < KEYS; ++i) key[i] = (decides >> i) & 1 ? key[i] : KEY_OF_NONE;
    }

    Bits sure = there & ~decides, tie = 0;
    uint32_t wanted = uint32_t(max(r.wanted, 0));
    if (wanted > 0) {                                            // (uniform)
        const auto clear = [&]() {
            bins[tid] = bins[tid + SELECT_THREADS] = 0;
            __syncthreads();
        };
        if (tid == 0) listed = 0;
        clear();
        // weights of 0 are many where a window hides tokens: counted for the wave
        uint32_t zeros = 0;
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            if (i >= 4 * chunks) continue;
            zeros += uint32_t(__popcll(__ballot(key[i] == KEY_OF_0)));
            atomicAdd(&bins[key[i] << 1 ? key[i] >> select_shift(0) : SELECT_BINS + lane], 1u);
            if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // (else places of all keys are found first, in as many registers)
        }
        if (lane == 0 && zeros) atomicAdd(&bins[KEY_OF_0 >> select_shift(0)], zeros);
        __syncthreads();
        SelectBin x = find_bin(bins[2047 - 2 * tid], bins[2046 - 2 * tid], wanted, part, found);
        wanted -= x.above;
        uint32_t digits = x.bin << select_shift(0), mask = 0xFFFFFFFFu << select_shift(0);
        // The keys with the digit, in any order, in LDS if there is room.
        const uint32_t total = bins[x.bin];
        const bool room = total <= SELECT_LIST;
        if (room) {
            Bits in = 0;
#pragma unroll
            for (int i = 0; i < KEYS; ++i) in |= Bits(key[i] - digits < 1u << select_shift(0)) << i;
            const uint32_t own = uint32_t(__popcll(uint64_t(in))), to = uint32_t(wave_inclusive_scan(int(own)));
            uint32_t at = 0;
            if (lane == 63 && to) at = atomicAdd(&listed, to);
            at = uint32_t(__builtin_amdgcn_readlane(int(at), 63)) + to - own;
#pragma unroll
            for (int i = 0; i < KEYS; ++i)
                if ((in >> i) & 1) list[at++] = key[i];
        }
        for (int pass = 1; pass < 3; ++pass) {
            const int shift = select_shift(pass), count = select_bins(pass);
            __syncthreads();                                     // (all have read bins)
            clear();
            if (room) {
                for (uint32_t j = 64 * wave; j < total; j += SELECT_THREADS) {
                    const uint32_t k = j + lane < total ? list[j + lane] : 0u;
                    count_key(bins, (k >> shift) & (count - 1), j + lane < total && ((k ^ digits) & mask) == 0);
                }
            } else {                                             // (read again: seldom)
                for (int i = 0; i < 4 * chunks; ++i) {
                    const int t = from + 64 * i + lane;
                    const uint32_t k = mass_key(t < upto ? mass[t] : 0.0f);
                    count_key(bins, (k >> shift) & (count - 1), t >= r.begin && t < r.end && ((k ^ digits) & mask) == 0);
                }
            }
            __syncthreads();
            x = find_bin(bins[2047 - 2 * tid], bins[2046 - 2 * tid], wanted, part, found);
            digits |= x.bin << shift, mask |= uint32_t(count - 1) << shift;
            wanted -= x.above;
        }
        if (bins[x.bin] == wanted) {                             // all of the tied ones
#pragma unroll
            for (int i = 0; i < KEYS; ++i) sure |= Bits(key[i] >= digits) << i;
        } else {
#pragma unroll
            for (int i = 0; i < KEYS; ++i) sure |= Bits(key[i] > digits) << i, tie |= Bits(key[i] == digits) << i;
        }
    }
    const auto wave_sum = [](uint32_t n) { return uint32_t(__builtin_amdgcn_readlane(wave_inclusive_scan(int(n)), 63)); };
    const uint32_t mine[2] = {wave_sum(uint32_t(__popcll(uint64_t(sure)))), wave_sum(uint32_t(__popcll(uint64_t(tie))))};
    if (lane == 0) sums[0][wave] = mine[0], sums[1][wave] = mine[1];
    __syncthreads();
    uint32_t tied = wave_sum(lane < wave ? sums[1][lane] : 0u);  // in the waves before
    uint32_t at = wave_sum(lane < wave ? sums[0][lane] : 0u) + min(tied, wanted);
    for (int i = 0; i < chunks; ++i) {
        uint32_t keep = uint32_t(sure >> (4 * i)) & 15u, more = uint32_t(tie >> (4 * i)) & 15u;
        if (mine[1]) {       // (wave-uniform) of the tied ones as many as are still wanted, from the front
            const uint32_t own = __popc(more), to = uint32_t(wave_inclusive_scan(int(own))), before = tied + to - own;
            for (uint32_t n = before < wanted ? wanted - before : 0u; n && more; --n) keep |= more & (~more + 1), more &= more - 1;
            tied += __builtin_amdgcn_readlane(to, 63);
        }
        const uint32_t own = __popc(keep), to = uint32_t(wave_inclusive_scan(int(own)));
        uint32_t place = at + to - own;
        for (; keep; keep &= keep - 1) kept[place++] = t0 + 256 * i + __builtin_ctz(keep);
        at += __builtin_amdgcn_readlane(to, 63);
    }
}

// Any length, of any number of heads: the keys are read again for every digit, a wave's sixteenth of the tokens in order.
__global__ __launch_bounds__(SELECT_THREADS) void fp4_select_long_kernel(Fp4Select a) {
    __shared__ uint32_t bins[SELECT_BINS];
    __shared__ uint32_t found[2], part[SELECT_WAVES], above[SELECT_WAVES], equal[SELECT_WAVES];
    const Fp4View &v = a.v;
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Fp4Sequence seq(v, b);
    const SelectRange r(a, seq, b);
    const int64_t stream = int64_t(b) * v.H + h;
    const float *mass = a.mass + stream * a.pitch;
    int32_t *kept = a.kept + stream * a.keep;
    if (h == 0 && tid == 0) a.n_kept[b] = r.n;
    for (int64_t i = r.n + tid; i < a.keep; i += SELECT_THREADS) kept[i] = -1;
    if (r.len <= r.budget) {
        for (int i = tid; i < r.n; i += SELECT_THREADS) kept[i] = i;
        return;
    }
    const int rounds = ((r.len + SELECT_WAVES - 1) / SELECT_WAVES + 63) / 64, from = wave * rounds * 64;
    const int upto = int(min(int64_t(r.end), a.pitch));
    const auto each = [&](auto f) {                              // f(position, key)
        for (int i = 0; i < rounds; ++i) {
            const int t = from + 64 * i + lane;
            f(t, mass_key(t < upto ? mass[t] : 0.0f));
        }
    };
    uint32_t digits = 0, mask = 0, wanted = uint32_t(max(r.wanted, 0));   // of the key that is looked for, and which are known
    const bool some = wanted > 0;
    for (int pass = 0; some && pass < 3; ++pass) {
        for (int i = tid; i < SELECT_BINS; i += SELECT_THREADS) bins[i] = 0;
        __syncthreads();
        const int shift = select_shift(pass), count = select_bins(pass);
        each([&](int t, uint32_t key) { count_key(bins, (key >> shift) & (count - 1), t >= r.begin && t < r.end && ((key ^ digits) & mask) == 0); });
        __syncthreads();
        const SelectBin x = find_bin(bins[2047 - 2 * tid], bins[2046 - 2 * tid], wanted, part, found);
        digits |= x.bin << shift, mask |= uint32_t(count - 1) << shift;
        wanted -= x.above;                                       // still wanted of those with these digits
    }
    const auto sure = [&](int t, uint32_t key) { return t < r.len && (t < r.begin || t >= r.end || (some && key > digits)); };
    const auto tie = [&](int t, uint32_t key) { return some && t >= r.begin && t < r.end && key == digits; };
    uint32_t sures = 0, ties = 0;
    each([&](int t, uint32_t key) { sures += uint32_t(__popcll(__ballot(sure(t, key)))), ties += uint32_t(__popcll(__ballot(tie(t, key)))); });
    if (lane == 0) above[wave] = sures, equal[wave] = ties;
    __syncthreads();
    uint32_t at = 0, tied = 0;                                   // of the waves before
    for (int i = 0; i < wave; ++i) at += above[i], tied += equal[i];
    at += min(tied, wanted);
    each([&](int t, uint32_t key) { write_kept(kept, t, sure(t, key), tie(t, key), wanted, at, tied, lane); });
}

// Long sequences, a workgroup to SELECT_PART tokens, in three launches (8 heads of 131079 tokens 21.5 us, 4 + 8 + 10 in the kernels; a
// workgroup to each, reading again for every digit, 163): counts of the first digit of every part; that
// digit from all parts' counts, and each part's keys with it; the other digits from those keys -- every workgroup for
// itself -- and the positions.  What the parts hand on of a (sequence, kv-head): counts [parts][2048], keys
// [parts][SELECT_PART], tokens above the digit [parts] and keys [parts], the digit and how many are wanted of it.
constexpr int SELECT_ROUNDS = 8, SELECT_PART = SELECT_ROUNDS * SELECT_THREADS, SELECT_LISTED = 12288, SELECT_PARTS = 256;

struct SelectSpace {
    uint32_t *counts, *keys, *above, *listed, *digit;
    static __host__ __device__ inline int64_t words(int parts) { return int64_t(parts) * (SELECT_BINS + SELECT_PART + 2) + 2; }
    __device__ inline SelectSpace(const Fp4Select &a, int64_t stream) {
        counts = a.space + stream * words(a.parts);
        keys = counts + int64_t(a.parts) * SELECT_BINS;
        above = keys + int64_t(a.parts) * SELECT_PART;
        listed = above + a.parts;
        digit = listed + a.parts;
    }
};

// A part's keys, wave by wave in order.
struct SelectPart {
    float held[SELECT_ROUNDS];
    int from;
    __device__ inline void load(const float *mass, int upto, int part, int wave, int lane) {
        from = part * SELECT_PART + wave * (64 * SELECT_ROUNDS) + lane;
#pragma unroll
        for (int i = 0; i < SELECT_ROUNDS; ++i) held[i] = from + 64 * i < upto ? mass[from + 64 * i] : 0.0f;
    }
    template <class F>
    __device__ inline void each(F f) const {
#pragma unroll
        for (int i = 0; i < SELECT_ROUNDS; ++i) f(from + 64 * i, mass_key(held[i]));
    }
};

template <int STEP>
__global__ __launch_bounds__(SELECT_THREADS) void fp4_select_part_kernel(Fp4Select a) {
    __shared__ uint32_t bins[SELECT_BINS];
    __shared__ uint32_t found[2], part_sums[SELECT_WAVES], above[SELECT_WAVES], equal[SELECT_WAVES];
    __shared__ uint32_t list[STEP == 2 ? SELECT_LISTED : 1], starts[STEP == 2 ? SELECT_PARTS + 1 : 1];
    const Fp4View &v = a.v;
    const int h = blockIdx.x % uint32_t(v.H), part = int(blockIdx.x / uint32_t(v.H)), b = blockIdx.y;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Fp4Sequence seq(v, b);
    const SelectRange r(a, seq, b);
    const int64_t stream = int64_t(b) * v.H + h;
    int32_t *kept = a.kept + stream * a.keep;
    if (STEP == 2) {
        if (h == 0 && part == 0 && tid == 0) a.n_kept[b] = r.n;
        for (int64_t i = r.n + int64_t(part) * SELECT_THREADS + tid; i < a.keep; i += int64_t(a.parts) * SELECT_THREADS) kept[i] = -1;
    }
    if (part * SELECT_PART >= r.len) return;
    if (r.len <= r.budget) {
        if (STEP == 2)
            for (int i = part * SELECT_PART + tid; i < min(r.n, (part + 1) * SELECT_PART); i += SELECT_THREADS) kept[i] = i;
        return;
    }
    const SelectSpace space(a, stream);
    const int parts = (r.len + SELECT_PART - 1) / SELECT_PART;   // that there are
    const bool some = r.wanted > 0;
    if (!some && STEP < 2) return;
    SelectPart mine;
    mine.load(a.mass + stream * a.pitch, int(min(int64_t(r.end), a.pitch)), part, wave, lane);
    const auto decides = [&](int t) { return t >= r.begin && t < r.end; };

    if constexpr (STEP == 0) {
        for (int i = tid; i < SELECT_BINS; i += SELECT_THREADS) bins[i] = 0;
        __syncthreads();
        mine.each([&](int t, uint32_t key) { count_key(bins, key >> 21, decides(t)); });
        __syncthreads();
        for (int i = tid; i < SELECT_BINS; i += SELECT_THREADS) space.counts[int64_t(part) * SELECT_BINS + i] = bins[i];
        return;
    }
    if constexpr (STEP == 1) {
        uint32_t hi = 0, lo = 0;
#pragma unroll 8
        for (int i = 0; i < parts; ++i) {
            const uint2 two = *reinterpret_cast<const uint2 *>(space.counts + int64_t(i) * SELECT_BINS + 2046 - 2 * tid);
            lo += two.x, hi += two.y;
        }
        const SelectBin x = find_bin(hi, lo, uint32_t(r.wanted), part_sums, found);
        if (part == 0 && tid == 0) space.digit[0] = x.bin, space.digit[1] = uint32_t(r.wanted) - x.above;
        uint32_t more = 0, same = 0;
        mine.each([&](int t, uint32_t key) {
            more += uint32_t(__popcll(__ballot(t < r.len && (!decides(t) || (key >> 21) > x.bin))));
            same += uint32_t(__popcll(__ballot(decides(t) && (key >> 21) == x.bin)));
        });
        if (lane == 0) above[wave] = more, equal[wave] = same;
        __syncthreads();
        const uint32_t before = uint32_t(wave_inclusive_scan(lane < SELECT_WAVES ? int(equal[lane]) : 0));
        const uint32_t sures = uint32_t(wave_inclusive_scan(lane < SELECT_WAVES ? int(above[lane]) : 0));
        if (tid == 63) space.above[part] = sures, space.listed[part] = before;
        uint32_t at = wave ? __builtin_amdgcn_readlane(before, (wave - 1) & 63) : 0u;
        uint32_t *keys = space.keys + int64_t(part) * SELECT_PART;
        mine.each([&](int t, uint32_t key) {
            const bool in = decides(t) && (key >> 21) == x.bin;
            const uint64_t all = __ballot(in);
            if (in) keys[at + uint32_t(__popcll(all & ((uint64_t(1) << lane) - 1)))] = key;
            at += uint32_t(__popcll(all));
        });
        return;
    }
    if constexpr (STEP == 2) {
        uint32_t digits = 0, wanted = 0, before = 0, tied = 0;   // before, tied: kept for sure and tied in the parts before
        if (some) {
            digits = space.digit[0] << 21, wanted = space.digit[1];
            // where each part's listed keys begin among all, and the keys themselves, in LDS if there is room
            if (wave == 0) {
                uint32_t sum = 0;
                for (int i = 0; i < parts; i += 64) {
                    const uint32_t n = i + lane < parts ? space.listed[i + lane] : 0u, upto = uint32_t(wave_inclusive_scan(int(n)));
                    if (i + lane < parts) starts[i + lane] = sum + upto - n;
                    sum += __builtin_amdgcn_readlane(upto, 63);
                }
                if (lane == 0) starts[parts] = sum;
            }
            __syncthreads();
            const uint32_t total = starts[parts], mine_at = starts[part];
            const bool room = total <= SELECT_LISTED;
            if (room) {
                for (int i = wave; i < parts; i += SELECT_WAVES) {
                    const uint32_t at = starts[i], n = starts[i + 1] - at;
                    for (uint32_t j = lane; j < n; j += 64) list[at + j] = space.keys[int64_t(i) * SELECT_PART + j];
                }
                __syncthreads();
            }
            const auto listed = [&](auto f) {                    // f(number among all, key, whether there is one), whole waves
                if (room) {
                    for (uint32_t j = 64 * wave; j < total; j += SELECT_THREADS) {
                        const bool in = j + lane < total;
                        f(j + lane, in ? list[j + lane] : 0u, in);
                    }
                } else {
                    for (int i = 0; i < parts; ++i) {
                        const uint32_t at = starts[i], n = starts[i + 1] - at;
                        for (uint32_t j = 64 * wave; j < n; j += SELECT_THREADS) {
                            const bool in = j + lane < n;
                            f(at + j + lane, in ? space.keys[int64_t(i) * SELECT_PART + j + lane] : 0u, in);
                        }
                    }
                }
            };
            uint32_t mask = 0xFFFFFFFFu << 21;
            for (int pass = 1; pass < 3; ++pass) {
                for (int i = tid; i < SELECT_BINS; i += SELECT_THREADS) bins[i] = 0;
                __syncthreads();
                const int shift = select_shift(pass), count = select_bins(pass);
                listed([&](uint32_t, uint32_t key, bool in) { count_key(bins, (key >> shift) & (count - 1), in && ((key ^ digits) & mask) == 0); });
                __syncthreads();
                const SelectBin x = find_bin(bins[2047 - 2 * tid], bins[2046 - 2 * tid], wanted, part_sums, found);
                digits |= x.bin << shift, mask |= uint32_t(count - 1) << shift;
                wanted -= x.above;
                __syncthreads();
            }
            uint32_t more = 0, same = 0;
            listed([&](uint32_t i, uint32_t key, bool in) {
                more += uint32_t(__popcll(__ballot(in && i < mine_at && key > digits)));
                same += uint32_t(__popcll(__ballot(in && i < mine_at && key == digits)));
            });
            uint32_t sures = 0;
            for (int i = 64 * wave; i < part; i += SELECT_THREADS) sures += i + lane < part ? space.above[i + lane] : 0u;
            more += __builtin_amdgcn_readlane(uint32_t(wave_inclusive_scan(int(sures))), 63);
            if (lane == 0) above[wave] = more, equal[wave] = same;
            __syncthreads();
            for (int i = 0; i < SELECT_WAVES; ++i) before += above[i], tied += equal[i];
            __syncthreads();
        } else {
            before = uint32_t(min(part * SELECT_PART, r.begin) + max(part * SELECT_PART - r.end, 0));
        }
        const auto sure = [&](int t, uint32_t key) { return t < r.len && (!decides(t) || (some && key > digits)); };
        const auto tie = [&](int t, uint32_t key) { return some && decides(t) && key == digits; };
        uint32_t sures = 0, ties = 0;
        mine.each([&](int t, uint32_t key) { sures += uint32_t(__popcll(__ballot(sure(t, key)))), ties += uint32_t(__popcll(__ballot(tie(t, key)))); });
        if (lane == 0) above[wave] = sures, equal[wave] = ties;
        __syncthreads();
        for (int i = 0; i < wave; ++i) before += above[i], tied += equal[i];
        uint32_t at = before + min(tied, wanted);
        mine.each([&](int t, uint32_t key) { write_kept(kept, t, sure(t, key), tie(t, key), wanted, at, tied, lane); });
    }
}

// Which kernel goes by the table's room.  Keys of up to 40960 tokens fit a workgroup's registers: four sequences of up to 32788 tokens, 8
// heads, selected, moved and read back so / in parts 91 / 100 us.  Beyond, parts, where the workspace holds what they hand on.
int launch_fp4_select(const kv_fp4_cache *c, Fp4Select a, hipStream_t s) {
    const int64_t room = int64_t(a.v.batch.table_pages) * FP4_PAGE, streams = int64_t(a.v.H) * a.v.batch.batch;
    a.parts = int((room + SELECT_PART - 1) / SELECT_PART);
    a.space = reinterpret_cast<uint32_t *>(c->workspace) + FP4_COUNTERS / sizeof(uint32_t);
    const bool in_parts = room > 40 * SELECT_THREADS && a.parts <= SELECT_PARTS && streams * SelectSpace::words(a.parts) <= FP4_PART_ROWS * (c->cfg.head_dim + 4);
    if (in_parts) {
        const dim3 grid = dim3(uint32_t(a.parts * a.v.H), uint32_t(a.v.batch.batch));
        hipLaunchKernelGGL(fp4_select_part_kernel<0>, grid, dim3(SELECT_THREADS), 0, s, a);
        KV_HIP_CHECK(hipGetLastError());
        hipLaunchKernelGGL(fp4_select_part_kernel<1>, grid, dim3(SELECT_THREADS), 0, s, a);
        KV_HIP_CHECK(hipGetLastError());
        hipLaunchKernelGGL(fp4_select_part_kernel<2>, grid, dim3(SELECT_THREADS), 0, s, a);
    } else {
        const dim3 grid = dim3(uint32_t(a.v.H), uint32_t(a.v.batch.batch));
        if (room <= 4 * SELECT_THREADS) hipLaunchKernelGGL(fp4_select_kernel<4>, grid, dim3(SELECT_THREADS), 0, s, a);
        else if (room <= 16 * SELECT_THREADS) hipLaunchKernelGGL(fp4_select_kernel<16>, grid, dim3(SELECT_THREADS), 0, s, a);
        else if (room <= 32 * SELECT_THREADS) hipLaunchKernelGGL(fp4_select_kernel<32>, grid, dim3(SELECT_THREADS), 0, s, a);
        else if (room <= 40 * SELECT_THREADS) hipLaunchKernelGGL(fp4_select_kernel<40>, grid, dim3(SELECT_THREADS), 0, s, a);
        else hipLaunchKernelGGL(fp4_select_long_kernel, grid, dim3(SELECT_THREADS), 0, s, a);
    }
    KV_HIP_CHECK(hipGetLastError());
    return KV_OK;
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

// A wave to some eights of tokens of a kv-head where they go, the next eight on its way while one is written: a word of V's channels there
// takes a code from each of eight words, HD / 64 channels to a lane; K's rows are 8 (4) bytes to a lane.  Where
// the tokens come from -- positions, then page numbers -- is found for all of them at once, a token to a lane.
// Bound by HBM and the chain of latencies before the first row (lengths, positions, page numbers): 4 x 8 heads, 8197 of up to 32788
// tokens each, in 31 us (some 120 MB: a quarter of the tokens touches nearly all of V's groups of eight and half of K's lines).
// Eights to a wave: one to each of so many waves first, then up to eight, a token to a lane.  Selected, moved and read back, that cut
// with 1 / 2 / 4 / 8 eights to a wave 99.4 / 91.9 / 90.3 / 87.4 us, one of 1000 tokens to 200 16.7 / 17.4 / 18.5 / 24.1.
constexpr int COMPACT_EIGHTS = 8;
constexpr int64_t COMPACT_WAVES = 4096;
template <int HD>
struct Fp4Eight {
    using P = Fp4Block<HD>;
    static constexpr int C = HD / 64, SCALES = HD / FP4_GROUP;
    uint32_t k[C], v[8][C];
    uint8_t ks, vs;
    // page, slot: of token (lane) of the wave's
    __device__ inline void load(const Fp4View &view, int h, int page, int slot, int eight, int lane) {
        const auto block = [&](int p) { return view.pages + (int64_t(max(p, 0)) * view.H + h) * size_t(P::BYTES); };
        const int j = 8 * eight + (lane & 7), s = min(lane / 8, SCALES - 1), at = __shfl(slot, j);
        const uint8_t *from = block(__shfl(page, j));
        ks = from[P::KS + at * SCALES + s], vs = from[P::VS + s * FP4_PAGE + at];
        const int t = 8 * eight + lane / 8;
        const uint32_t *row = reinterpret_cast<const uint32_t *>(block(__shfl(page, t)) + P::K + __shfl(slot, t) * (HD / 2) + (lane & 7) * (HD / 16));
#pragma unroll
        for (int c = 0; c < C; ++c) k[c] = row[c];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int p = __builtin_amdgcn_readlane(page, 8 * eight + i), x = __builtin_amdgcn_readlane(slot, 8 * eight + i);
            const uint32_t *words = reinterpret_cast<const uint32_t *>(block(p) + P::V) + (x / 8) * HD + C * lane;
#pragma unroll
            for (int c = 0; c < C; ++c) v[i][c] = words[c];
        }
    }
    // out: the page's block; at: the first of the eight in it.  All eight are written: those without a page, behind the last token too, as zeros.
    __device__ inline void store(uint8_t *out, int at, int page, int slot, int eight, int lane) const {
        const int j = lane & 7, s = lane / 8;
        const bool there = __shfl(page, 8 * eight + j) >= 0;
        if (s < SCALES) {
            out[P::KS + (at + j) * SCALES + s] = there ? ks : uint8_t(127);
            out[P::VS + s * FP4_PAGE + at + j] = there ? vs : uint8_t(127);
        }
        const bool row = __shfl(page, 8 * eight + s) >= 0;
        uint32_t *to = reinterpret_cast<uint32_t *>(out + P::K + (at + s) * (HD / 2) + j * (HD / 16));
#pragma unroll
        for (int c = 0; c < C; ++c) to[c] = row ? k[c] : 0u;
        uint32_t word[C] = {};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int p = __builtin_amdgcn_readlane(page, 8 * eight + i), x = __builtin_amdgcn_readlane(slot, 8 * eight + i);
            const uint32_t keep = p >= 0 ? 15u : 0u;
#pragma unroll
            for (int c = 0; c < C; ++c) word[c] |= ((v[i][c] >> (4 * (x & 7))) & keep) << (4 * i);
        }
        uint32_t *words = reinterpret_cast<uint32_t *>(out + P::V) + (at / 8) * HD + C * lane;
#pragma unroll
        for (int c = 0; c < C; ++c) words[c] = word[c];
    }
};

template <int HD>
__global__ __launch_bounds__(256) void fp4_compact_kernel(Fp4Compact a, int units, int eights_of_wave) {
    using P = Fp4Block<HD>;
    const int lane = threadIdx.x & 63;
    const Fp4View &v = a.from;
    const uint32_t number = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int unit = int(number / uint32_t(v.H)), h = int(number - uint32_t(unit) * v.H), b = blockIdx.y;
    if (unit >= units) return;
    const int n = min(max(a.n_kept[b], 0), a.keep);
    const int64_t first = int64_t(unit) * 8 * eights_of_wave;
    if (first >= n) return;
    const int i0 = int(first), here = min(n - i0, 8 * eights_of_wave), eights = (here + 7) / 8;
    const Fp4Sequence to_seq(a.to, b, n, 0, 0), seq(v, b);
    const int64_t stream = int64_t(b) * v.H + h;
    // token `lane` of the wave's: where it comes from, and the page that it goes to
    const int from = lane < here ? a.kept[stream * a.keep + i0 + lane] : -1;
    const bool held = from >= 0 && from < seq.held;
    const int page = held ? int(seq.page(v, from / FP4_PAGE)) : -1, slot = from & (FP4_PAGE - 1);
    const int to_page = lane < here && (i0 + lane) / FP4_PAGE < a.to.batch.table_pages ? int(to_seq.page(a.to, (i0 + lane) / FP4_PAGE)) : -1;
    if (a.mass_out && lane < here && i0 + lane < a.out_pitch)
        a.mass_out[stream * a.out_pitch + i0 + lane] = held && from < a.pitch ? a.mass[stream * a.pitch + from] : 0.0f;
    const auto store = [&](const Fp4Eight<HD> &x, int e) {
        const int to = __builtin_amdgcn_readlane(to_page, 8 * e);
        if (to < 0) return;
        x.store(v.pages + (int64_t(to) * v.H + h) * size_t(P::BYTES), (i0 + 8 * e) % FP4_PAGE, page, slot, e, lane);
    };
    Fp4Eight<HD> in[2];
    in[0].load(v, h, page, slot, 0, lane);
    for (int e = 0;; e += 2) {           // (behind the last eight that one again)
        in[1].load(v, h, page, slot, min(e + 1, eights - 1), lane);
        store(in[0], e);
        if (e + 1 >= eights) break;
        in[0].load(v, h, page, slot, min(e + 2, eights - 1), lane);
        store(in[1], e + 1);
        if (e + 2 >= eights) break;
    }
}

}  // namespace packkv

using namespace packkv;

extern "C" int kv_fp4_select(kv_fp4_cache_t *c, const kv_fp4_batch_t *batch, const float *mass, int64_t mass_tokens, int32_t keep,
                             const int32_t *budgets, int32_t sinks, int32_t recent, int32_t *kept, int32_t *n_kept, void *hip_stream) {
    const int rc = c ? fp4_check_batch(batch) : KV_ERR_ARG;
    if (rc) return rc;
    if (mass_tokens < 1 || keep < 1 || sinks < 0 || recent < 0) return KV_ERR_ARG;
    if (!fp4_aligned(mass, 4) || !fp4_aligned(kept, 4) || !fp4_aligned(n_kept, 4) || (budgets && !fp4_aligned(budgets, 4))) return KV_ERR_ARG;
    const int64_t streams = int64_t(batch->batch) * c->cfg.n_kv_heads;
    const Rows lens(batch->lens, batch->batch, 4), weights(mass, Rows::Wide(streams) * mass_tokens, 4), most(budgets, batch->batch, 4),
        positions(kept, Rows::Wide(streams) * keep, 4), counts(n_kept, batch->batch, 4);
    if (overlap(positions, {lens, weights, most, counts}) || overlap(counts, {lens, weights, most})) return KV_ERR_ARG;
    return launch_fp4_select(c, Fp4Select{fp4_view(c, batch, 0), mass, mass_tokens, keep, sinks, recent, budgets, kept, n_kept, nullptr, 0},
                             static_cast<hipStream_t>(hip_stream));
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
    const int64_t streams = int64_t(from->batch) * c->cfg.n_kv_heads;
    if (overlap(Rows(mass_out, Rows::Wide(streams) * mass_out_tokens, 4),
                {Rows(mass, Rows::Wide(streams) * mass_tokens, 4), Rows(kept, Rows::Wide(streams) * keep, 4), Rows(n_kept, from->batch, 4),
                 Rows(from->lens, from->batch, 4), Rows(from->page_table, int64_t(from->batch) * from->table_pages, 4),
                 Rows(to->page_table, int64_t(to->batch) * to->table_pages, 4)}))
        return KV_ERR_ARG;
    const Fp4Compact a{fp4_view(c, from, 0), fp4_view(c, to, 0), kept, n_kept, keep, mass, mass_tokens, mass_out, mass_out_tokens};
    const int64_t eights = (int64_t(keep) + 7) / 8;
    const int64_t each = std::max<int64_t>(std::min<int64_t>(eights * c->cfg.n_kv_heads * from->batch / COMPACT_WAVES, COMPACT_EIGHTS), 1);
    const int64_t units = (eights + each - 1) / each, groups = (units * c->cfg.n_kv_heads + 3) / 4;
    if (groups > FP4_GROUPS_MOST) return KV_ERR_UNSUPPORTED;
    const dim3 grid = dim3(uint32_t(groups), uint32_t(from->batch));
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (c->cfg.head_dim == 128) hipLaunchKernelGGL(fp4_compact_kernel<128>, grid, dim3(256), 0, s, a, int(units), int(each));
    else hipLaunchKernelGGL(fp4_compact_kernel<64>, grid, dim3(256), 0, s, a, int(units), int(each));
    KV_HIP_CHECK(hipGetLastError());
    return KV_OK;
}
