// Filtered draws: temperature, top-k, top-p and min-p, and a draw from a given uniform; one workgroup per row.
//
// A row's entries are ordered by (value descending, index ascending): by a 64-bit integer `rank`, an order-preserving
// image of the value above the inverted index, of which no two are alike.  top-k and top-p each keep a head of that
// order: the entries whose rank is at least some C.  To find C without sorting, entries are dealt to bins along the value
// (a histogram of counts, or of masses), the bin in which the head ends is found by a prefix sum, and its few entries are
// ordered among themselves.  Where too many share a bin (equal values, outliers) the digits of the rank take the place
// of the bins.
//
// Masses are integers, w = rint(2^44 2^((z - max z) log2(e) / T)): their sums (at most 2^62) do not depend on their order, so
// neither atomics nor the shape of a launch show in a result, and at 2^-45 of the largest weight an entry they place a
// border or a draw where sums in 64-bit floating point place it.
//
// What bounds it: one row, the chain of its passes and barriers (16384 entries, top-k 2000: 26 thousand cycles, 11.7 us, of which
// the launch is 5; 32 guided rows 16.1); many rows, vector instructions: 60 an entry, the vector pipes busy 72 % (2048 rows of 16384,
// top-p and min-p, logits out: 81 us, 3.3 TB/s of the 5.05 that a copy reaches).
#include <hip/hip_bf16.h>

#include <type_traits>

#include "mulo_internal.h"

namespace mulo {
namespace {

typedef unsigned long long u64;
constexpr float MOST = 3.402823466e38f;   // the largest finite float32
constexpr float NEG = -__builtin_huge_valf();
constexpr int CAND = 512;                 // entries of a bin that are ordered by comparing them all
constexpr int DIGIT = 10;                 // bits of a rank that a histogram of them tells apart
constexpr int LDS_ENTRIES = 32768;        // of a row that is kept in LDS (128 KB)
constexpr int ONE = 44;                   // bits of the largest weight
static_assert(ONE == 44, "Weights::value");

// order-preserving integer of a value (not NaN); -0 and 0 are the same value
__device__ __forceinline__ uint32_t key_of(float z) {
    const uint32_t b = __float_as_uint(z == 0.f ? 0.f : z);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ u64 rank_of(float z, int i) { return (u64)key_of(z) << 32 | (uint32_t)~i; }

// Weights, 2^x with x = (z - max z) log2(e) / T <= 0.  y = STEPS x = n + f, |f| <= 1/2:
//   2^x = 2^(n / STEPS) e^t, t = f ln 2 / STEPS, |t| <= 6.8e-4
// The first factor is a table's, its exponent moved.  e^t - 1 = t + t^2 (1/2 + t / 6), less than t^4 / 24 = 2^-46 of it left
// out; the sum's second part is below 2^-22 and float32 is enough for it.  18 instructions, all of which issue at the same
// rate (a polynomial of 2^x over all of [-1/2, 1/2] takes 10 more).  Relative error: 2^-44.
constexpr int STEPS = 512;
struct Weights {
    double zmax, c;            // the maximum; STEPS log2(e) / temperature
    float least_value, least;  // smallest z with a weight that value(), and integer(), tell from 0
    const double* table;       // 2^(ONE + i / STEPS), in LDS
    __device__ __forceinline__ double part(float z) const {     // 2^(ONE + x), for z of at least least_value
        constexpr double K = 0.6931471805599453 / STEPS, shift = 6755399441055744.0;      // 1.5 2^52: the sum's low word is the nearest integer
        const double d = (double)z - zmax;
        const double ys = __builtin_fma(d, c, shift), f = __builtin_fma(d, c, -(ys - shift));
        const uint32_t n = (uint32_t)__double_as_longlong(ys);
        const u64 tb = (u64)__double_as_longlong(table[n & (STEPS - 1)]);
        const double tw = __longlong_as_double((long long)((u64)((uint32_t)(tb >> 32) + ((n & ~(STEPS - 1u)) << (20 - LOG_STEPS))) << 32 | (uint32_t)tb));
        const float t = (float)f;
        const double r = __builtin_fma(f, K, (double)(t * t * __builtin_fmaf(t, (float)(K * K * K / 6), (float)(K * K / 2))));
        return __builtin_fma(tw, r, tw);
    }
    static constexpr int LOG_STEPS = 9;
    static_assert(STEPS == 1 << LOG_STEPS, "the steps");
    // + 2^52: rounds to an integer.  Of an entry below `least` the result means nothing.
    __device__ __forceinline__ u64 integer(float z) const { return (u64)__double_as_longlong(part(z) + 4503599627370496.0) & 0xFFFFFFFFFFFFFull; }
    // the weights of the entries of four that are in, 0 of the others: side by side, without a branch
    __device__ __forceinline__ void integers(const float z[4], const bool in[4], u64 out[4]) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] = 0;
        if (!__any(in[0] || in[1] || in[2] || in[3])) return;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const u64 t = integer(z[e]);
            out[e] = in[e] && z[e] >= least ? t : 0;
        }
    }
    __device__ __forceinline__ double value(float z) const { return z >= least_value ? part(z) * 0x1p-44 : 0.0; }
};

// Sums and maxima over the lanes of a wavefront by data-parallel moves: shifts by 1, 2, 4, 8 inside a row of 16 lanes, then the
// last lane of a row to the next row, and lane 31 to the upper half.  Lanes without a source take `none`.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t moved(uint32_t none, uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, CTRL, ROWS, 0xf, false);
}
template <class F>
__device__ __forceinline__ void six_moves(F&& f) {
    f(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});
    f(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
    f(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
    f(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
    f(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});
    f(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
}
__device__ __forceinline__ u64 wave_scan(u64 v) {      // inclusive
    six_moves([&](auto c, auto r) {
        const uint32_t lo = moved<decltype(c)::value, decltype(r)::value>(0, (uint32_t)v), hi = moved<decltype(c)::value, decltype(r)::value>(0, (uint32_t)(v >> 32));
        v += (u64)hi << 32 | lo;
    });
    return v;
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
    six_moves([&](auto c, auto r) { v += moved<decltype(c)::value, decltype(r)::value>(0, v); });
    return v;
}
__device__ __forceinline__ u64 lane_of(u64 v, int i) {
    return (u64)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), i) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, i);
}
__device__ __forceinline__ uint32_t lane_of(uint32_t v, int i) { return (uint32_t)__builtin_amdgcn_readlane((int)v, i); }
__device__ __forceinline__ float wave_max(float v) {
    six_moves([&](auto c, auto r) {
        const uint32_t b = __float_as_uint(v);
        v = fmaxf(v, __uint_as_float(moved<decltype(c)::value, decltype(r)::value>(b, b)));
    });
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), 63));
}

// LDS: the row is read from memory once and kept there; else every pass reads it again.  (Kept in registers, a row of 16384
// unrolls every pass 64 times: 70000 instructions, which neither registers nor the instruction cache hold.)
// Wavefront w has the stretch [w seg, (w + 1) seg) of the row, in runs of 256: consecutive lanes, consecutive entries.
// A thread takes the same entries in every pass.
// PER: entries of the list a thread takes.  Where top-k leaves at most PER NT entries they are listed, and everything behind it
// (masses, top-p, the draw's sums, what is written of them) goes by the list: of 16384 entries 2000 cost an eighth (a row of 16384,
// 512 threads, top-p 0.9 alone 19.6 us, behind top-k 200 13.6).  With 512 threads a thread takes one: two would serve top-k up to
// 1024, but a list takes two passes of its own, which only masses win back, and a shorter top-k is slower with two.  2048 rows of 16384, us, one / two: top-k 200 and top-p 0.9, tokens 64.6 / 65.7, logits 72.7 / 73.5; top-k 1000,
// tokens 78.4 / 62.9, logits 55.8 / 77.8; top-k 1000 and top-p 0.9, tokens 115 / 73, logits 88.6 / 83.7.
// KIND: ANY_ROWS, or what the rows are (1: bf16, 2: guided), for the form that reads them in every pass: each pass holds the loads of its
// kind alone (of all kinds the code took 152 KB, more than the instruction cache by far; now 97 to 112.
// 1 row of 33000 28.4 and 25.8 us, 16 of 131072 56 and 53, bf16 59.5 and 55.3, guided 66 and 62.5).
constexpr int ANY_ROWS = -1;
template <int NT, bool LDS, int PER, int KIND>
__global__ __launch_bounds__(NT) void k_sample(const SampleArgs a, int runs) {
    constexpr int NW = NT / 64;
    // Bins of a histogram.  Long rows, which leave LDS free, have more, so that a bin near their middle holds no more than CAND entries:
    // of 150000 normal ones 520 fell into one of 1024 bins, and the digits took over (16 rows 245 us, with 4096 bins 118; 1 row of
    // 131072 103 and 91).
    constexpr int BINS = LDS ? 1024 : 4096;
    extern __shared__ __attribute__((aligned(16))) float4 kept_row[];      // [NW][runs][64]
    __shared__ __align__(16) u64 hist[BINS];       // then the entries of a bin, and their weights
    __shared__ double table[STEPS];
    __shared__ u64 s_wave[NW], s_mass[NW], s_front, s_border;
    __shared__ float s_lo[NW], s_hi[NW];
    __shared__ int s_bin, s_n, s_count[NW];
    constexpr bool OWN_LIST = PER * NT > BINS;     // else the list passes through the histogram's place
    __shared__ u64 own_list[OWN_LIST ? PER * NT : 1];
    u64* const cand = hist;
    u64* const candw = hist + CAND;
    u64* const list = OWN_LIST ? own_list : hist;  // value << 32 | index

    const int64_t r = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), V = a.V;
    const int w_first = wave * runs * 256, w_runs = V - w_first <= 0 ? 0 : (V - w_first + 255) / 256 < runs ? (V - w_first + 255) / 256 : runs;
    const int first = w_first + lane * 4;
    float4* const mine = kept_row + wave * runs * 64 + lane;
    const bool bf16 = KIND == ANY_ROWS ? a.dtype == 1 : KIND & 1, guided = KIND == ANY_ROWS ? a.logits_u != nullptr : KIND & 2;
    const size_t esz = bf16 ? 2 : 4;
    const char* const zc = (const char*)a.logits + r * a.row_stride * esz;
    const char* const zu = (const char*)a.logits_u + (guided ? r * a.row_stride * esz : 0);
    // Four entries an access, wherever the row begins (global memory takes vectors at any alignment of their elements).  Four
    // runs that lie in the row as a whole take one address; else an access that would pass the end moves back to it, and what it
    // then holds too early is shifted out.
    struct __attribute__((packed)) Four { float v[4]; };
    struct __attribute__((packed)) FourShort { uint16_t v[4]; };
    auto wide = [](const FourShort t) {
        auto one = [&](int e) { return __uint_as_float((uint32_t)t.v[e] << 16); };
        return make_float4(one(0), one(1), one(2), one(3));
    };
    auto four_runs = [&](const char* row, int i, float4 v[4]) {      // entries i .. i + 3 and 256, 512 and 768 further on
        if (i - lane * 4 + 1024 <= V) {
            if (bf16) {
                FourShort t[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) t[j] = reinterpret_cast<const FourShort*>(row + (size_t)i * 2)[j * 64];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = wide(t[j]);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const Four t = reinterpret_cast<const Four*>(row + (size_t)i * 4)[j * 64];
                    v[j] = make_float4(t.v[0], t.v[1], t.v[2], t.v[3]);
                }
            }
        } else if (!LDS || V >= 4) {
            int at[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) at[j] = i + j * 256 < V - 4 ? i + j * 256 : V - 4;
            if (bf16) {
                FourShort t[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) t[j] = *reinterpret_cast<const FourShort*>(row + (size_t)at[j] * 2);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = wide(t[j]);
            } else {
                Four t[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) t[j] = *reinterpret_cast<const Four*>(row + (size_t)at[j] * 4);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = make_float4(t[j].v[0], t[j].v[1], t[j].v[2], t[j].v[3]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int past = i + j * 256 - at[j];      // four and more: all of them lie behind the end
                if (past & 1) { v[j].x = v[j].y; v[j].y = v[j].z; v[j].z = v[j].w; }
                if (past & 2) { v[j].x = v[j].z; v[j].y = v[j].w; }
            }
        } else {
            auto one = [&](int k) {
                k = k < V ? k : 0;
                return bf16 ? __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(row)[k] << 16) : reinterpret_cast<const float*>(row)[k];
            };
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = make_float4(one(0), one(1), one(2), one(3));
        }
    };
    // f(index of the first, four entries, number of the run), four runs requested together; guided; NaN, and what lies past the
    // end, is masked.  (+inf becomes the largest finite number: below where the row is kept in LDS.)
    auto from_memory = [&](auto&& f) {
        for (int j0 = 0; j0 < w_runs; j0 += 4) {
            float4 c[4];
            four_runs(zc, first + j0 * 256, c);
            if (guided) {
                float4 u[4];
                four_runs(zu, first + j0 * 256, u);
                auto guide = [&](float x, float y) {
#pragma clang fp contract(off)      // every operation is rounded: a fused one gives another value
                    const float d = x - y, m = a.cfg_scale * d;
                    return y + m;
                };
#pragma unroll
                for (int j = 0; j < 4; ++j) c[j] = make_float4(guide(c[j].x, u[j].x), guide(c[j].y, u[j].y), guide(c[j].z, u[j].z), guide(c[j].w, u[j].w));
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int i = first + (j0 + j) * 256;
                auto clean = [](float z) { z = fmaxf(z, NEG); return LDS ? z : fminf(z, MOST); };      // of a NaN and a number the maximum is the number
                float4 v = make_float4(clean(c[j].x), clean(c[j].y), clean(c[j].z), clean(c[j].w));
                if (i - lane * 4 + 256 > V) v = make_float4(i < V ? v.x : NEG, i + 1 < V ? v.y : NEG, i + 2 < V ? v.z : NEG, i + 3 < V ? v.w : NEG);
                if (j0 + j < w_runs) f(i, v, j0 + j);
            }
        }
    };
    auto each4 = [&](auto&& f) {
        if constexpr (LDS) {
            for (int j = 0; j < w_runs; ++j) f(first + j * 256, mine[j * 64]);
        } else {
            from_memory([&](int i, const float4 z, int) { f(i, z); });
        }
    };
    auto put = [&](float* row, int i, const float4 v) {
        if (i + 4 <= V) {
            *reinterpret_cast<Four*>(row + i) = Four{{v.x, v.y, v.z, v.w}};
        } else {
            if (i < V) row[i] = v.x;
            if (i + 1 < V) row[i + 1] = v.y;
            if (i + 2 < V) row[i + 2] = v.z;
        }
    };
    for (int i = tid; i < BINS; i += NT) hist[i] = 0;
    const bool greedy = a.temperature == 0.0;
    const int top_k = greedy ? 1 : a.top_k;
    // (from memory in every pass, the row has to stay as it is where the filtered logits take its place)
    const bool by_list = top_k > 0 && top_k <= PER * NT && top_k < V && (LDS || (const void*)a.kept != a.logits);
    float* const probs = a.probs ? a.probs + r * V : nullptr;
    float* const kept = a.kept ? a.kept + r * V : nullptr;
    // ---- the largest entry, and the smallest that is not masked (masked ones are left out in a pass of their own)
    float hi = NEG, lo = -NEG;
    auto meet = [&]() {
        hi = wave_max(hi);
        lo = -wave_max(-lo);
        if (lane == 0) { s_hi[wave] = hi; s_lo[wave] = lo; }
        __syncthreads();
        const float h = s_hi[lane & (NW - 1)], l = s_lo[lane & (NW - 1)];
        hi = wave_max(h);
        lo = -wave_max(-l);
    };
    from_memory([&](int i, const float4 z, int j) {
        if constexpr (LDS) mine[j * 64] = z;
        hi = fmaxf(fmaxf(hi, fmaxf(z.x, z.y)), fmaxf(z.z, z.w));
        lo = fminf(fminf(lo, fminf(z.x, z.y)), fminf(z.z, z.w));
        // what the list does not hold; the list's entries are written over it, barriers later
        if (by_list && probs) put(probs, i, make_float4(0.f, 0.f, 0.f, 0.f));
        if (by_list && kept) put(kept, i, make_float4(NEG, NEG, NEG, NEG));
    });
    for (int i = tid; i < STEPS; i += NT) table[i] = exp2((double)ONE + (double)i / STEPS);      // while the row is on its way
    meet();
    if (lo == NEG && hi > NEG) {
        lo = -NEG;
        each4([&](int, const float4 z) {
            auto some = [](float x) { return x > NEG ? x : -NEG; };
            lo = fminf(fminf(lo, fminf(some(z.x), some(z.y))), fminf(some(z.z), some(z.w)));
        });
        __syncthreads();         // the others have read s_hi and s_lo
        meet();
    }
    if (LDS && hi > MOST) {
        for (int j = 0; j < w_runs; ++j) {
            const float4 z = mine[j * 64];
            mine[j * 64] = make_float4(fminf(z.x, MOST), fminf(z.y, MOST), fminf(z.z, MOST), fminf(z.w, MOST));
        }
        hi = MOST;
        lo = fminf(lo, MOST);
    }
    const bool none = hi == NEG;
    const float top = hi;
    const double per_z = a.temperature * 0.6931471805599453;
    // the least float32 that is at most `bits` below the maximum.  (A conversion alone may step below: where a step is hundreds
    // of bits, part() would move the exponent of an entry there by more than there is.)
    auto at_least = [&](double bits) {
        const double limit = fmax((double)top - bits * per_z, -(double)MOST);
        const float z = (float)limit;
        return (double)z < limit ? of_key(key_of(z) + 1) : z;
    };
    const Weights w{(double)top, greedy ? 0.0 : STEPS * 1.4426950408889634 / a.temperature, at_least(900.0), at_least(ONE + 2.0), table};
    // the border, so far: entries above b_z stay, and those at it up to index b_i
    float b_z = NEG;
    int b_i = -1;
    auto inside = [&](int i, float z) -> bool { return (z > b_z) | ((z == b_z) & (i <= b_i)); };
    auto above = [](float z) { return of_key(key_of(z) + 1); };
    // f(index of the first, the four, which of them are inside).  Whether an entry at b_z is inside is the same for a whole run,
    // but for the run that holds b_i: there those that are not are masked first.
    auto each = [&](auto&& f) {
        each4([&](int i, const float4 v) {
            const int r0 = __builtin_amdgcn_readfirstlane(i - lane * 4);
            float z[4] = {v.x, v.y, v.z, v.w};
            if (r0 <= b_i && r0 + 255 > b_i) {
#pragma unroll
                for (int e = 0; e < 4; ++e) z[e] = z[e] == b_z && i + e > b_i ? NEG : z[e];
            }
            const float t = r0 <= b_i ? b_z : above(b_z);
            const bool in[4] = {z[0] >= t, z[1] >= t, z[2] >= t, z[3] >= t};
            f(i, z, in);
        });
    };

    // ---- the head of what is inside that ends with the entry at which the count, or the mass, reaches want(all of it)
    // Bins along the value: linear over the range of the row, or over the first 128 below the maximum (masks of very low values).
    // Float subtraction and multiplication by a positive number are monotone, so a larger value is never in a later bin.
    const float scale = (float)BINS / fmaxf(fminf(top - lo, 128.f), 1e-30f);
    auto bin_of = [&](float z) { return (int)__builtin_amdgcn_fmed3f((top - z) * scale, 0.f, (float)(BINS - 1)); };
    // where the prefix sum of the bins (of counts: their low words) reaches want: s_bin, and the sum in front of it in s_front
    auto cross = [&](auto by_mass, u64 before, auto&& want) -> u64 {
        typedef std::conditional_t<decltype(by_mass)::value, u64, uint32_t> X;
        constexpr int BPT = BINS / NT;
        X v[BPT], sum = 0;
#pragma unroll
        for (int i = 0; i < BPT; ++i) sum += v[i] = (X)hist[tid * BPT + i];
        const X upto = wave_scan(sum);
        if (lane == 63) s_wave[wave] = upto;
        __syncthreads();
        const X waves = wave_scan(lane < NW ? (X)s_wave[lane] : X(0));
        const u64 target = want(before + lane_of(waves, NW - 1));
        u64 front = before + (wave ? lane_of(waves, wave - 1) : X(0)) + (upto - sum);
#pragma unroll
        for (int i = 0; i < BPT; ++i) {
            if (front < target && front + v[i] >= target) {
                s_bin = tid * BPT + i;
                s_front = front;
            }
            front += v[i];
        }
        if (tid == 0) s_n = 0;
        __syncthreads();
        return target;
    };
    // the entry of the bin that was found at which target is reached, in the order of the ranks: s_border
    auto order_bin = [&](auto by_mass, u64 front, u64 target, int n) {
        constexpr bool MASS = decltype(by_mass)::value;
        if (MASS) {
            for (int t = tid; t < n; t += NT) {
                const float z = of_key((uint32_t)(cand[t] >> 32));
                candw[t] = z >= w.least ? w.integer(z) : 0;
            }
            __syncthreads();
        }
        for (int t = tid; t < n; t += NT) {
            const u64 own = cand[t];
            u64 before = front;
#pragma unroll 4
            for (int i = 0; i < n; ++i) {
                const u64 amount = MASS ? candw[i] : 1ull;
                before += cand[i] > own ? amount : 0;
            }
            if (before < target && before + (MASS ? candw[t] : 1ull) >= target) s_border = own;
        }
        __syncthreads();
    };
    auto take_border = [&]() {
        b_z = of_key((uint32_t)(s_border >> 32));
        b_i = (int)~(uint32_t)s_border;
    };
    auto find_border = [&](auto by_mass, auto&& want) {
        constexpr bool MASS = decltype(by_mass)::value;
        // adds the counts, or the weights, of entries to their bins
        auto add = [&](const float z[4], const bool in[4], auto&& bin) {
            if constexpr (MASS) {
                if (!__any(in[0] || in[1] || in[2] || in[3])) return;
                u64 x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = w.integer(z[e]);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (in[e] && z[e] >= w.least) atomicAdd(&hist[bin(e)], x[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) atomicAdd(reinterpret_cast<uint32_t*>(&hist[bin(e)]), in[e] ? 1u : 0u);      // at most 2^18: the low words
            }
        };
        each([&](int, const float z[4], const bool in[4]) { add(z, in, [&](int e) { return bin_of(z[e]); }); });
        __syncthreads();
        const u64 target = cross(by_mass, 0, want);
        const int bin = s_bin;
        u64 front = s_front;
        // the bin's entries lie between zl and zh, which are wider than it by more than the roundings of bin_of
        const float width = 1.0f / scale, slack = (fabsf(top) + (bin + 1) * width) * 4.8e-7f;
        const float zh = bin == 0 ? -NEG : top - bin * width + slack, zl = bin == BINS - 1 ? NEG : top - (bin + 1) * width - slack;
        each4([&](int i, const float4 v) {
            const float z[4] = {v.x, v.y, v.z, v.w};
            bool near[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) near[e] = (z[e] >= zl) & (z[e] <= zh);
            if (near[0] | near[1] | near[2] | near[3]) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (near[e] && bin_of(z[e]) == bin && inside(i + e, z[e])) {
                        const int at = atomicAdd(&s_n, 1);
                        if (at < CAND) cand[at] = rank_of(z[e], i + e);
                    }
            }
        });
        __syncthreads();
        const int n = s_n;
        if (n <= CAND) {
            order_bin(by_mass, front, target, n);
        } else {
            // by the digits of the rank, the largest first: 32 bits of the value, and the 18 of an index that can differ
            auto short_rank = [](float z, int i) { return (u64)key_of(z) << 18 | ((uint32_t)~i & 0x3FFFFu); };
            u64 known = 0;
#pragma unroll 1
            for (int shift = 4 * DIGIT; shift >= 0; shift -= DIGIT) {
                for (int i = tid; i < BINS; i += NT) hist[i] = 0;
                __syncthreads();
                each([&](int i, const float z[4], const bool in[4]) {
                    bool here[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) here[e] = in[e] && bin_of(z[e]) == bin && short_rank(z[e], i + e) >> (shift + DIGIT) == known;
                    add(z, here, [&](int e) { return BINS - 1 - (int)(short_rank(z[e], i + e) >> shift & ((1 << DIGIT) - 1)); });
                });
                __syncthreads();
                cross(by_mass, front, [&](u64) { return target; });
                front = s_front;
                known = known << DIGIT | (BINS - 1 - s_bin);
            }
            if (tid == 0) s_border = known >> 18 << 32 | 0xFFFC0000ull | (known & 0x3FFFFu);
            __syncthreads();
        }
        take_border();
    };
    static_assert(BINS >= 1 << DIGIT && BINS >= 2 * CAND, "a bin for every digit, and room for the entries of one");
    bool cleared = true;
    auto clear_hist = [&]() {
        if (!cleared) {
            for (int i = tid; i < BINS; i += NT) hist[i] = 0;
            __syncthreads();
        }
        cleared = false;
    };
    const bool listed = by_list && !none;
    float lz[PER];
    uint32_t lat[PER];
    if (!none) {
        auto share = [&](u64 all) {
            const u64 t = (u64)__builtin_ceil(a.top_p * (double)all);      // the mass in front of the next entry is below top_p of all
            return t < 1 ? 1ull : t < all ? t : all;
        };
        const bool top_p = !greedy && a.top_p < 1.0;
        if (top_k > 0 && top_k < V) {
            clear_hist();
            find_border(std::false_type{}, [&](u64 all) { return all < (u64)top_k ? all : (u64)top_k; });      // fewer are not masked: all of them
        }
        if (listed) {
            // in the order of the indexes: first how many of every wavefront
            int count = 0;
            each([&](int, const float[4], const bool in[4]) {
#pragma unroll
                for (int e = 0; e < 4; ++e) count += __popcll(__ballot(in[e]));
            });
            if (lane == 0) s_count[wave] = count;
            __syncthreads();
            const uint32_t counts = wave_scan(lane < NW ? (uint32_t)s_count[lane] : 0u);
            int base = (int)lane_of(counts, wave) - count;
            each([&](int i, const float z[4], const bool in[4]) {
                u64 b[4];
                int before = base;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    b[e] = __ballot(in[e]);
                    base += __popcll(b[e]);
                    before = __builtin_amdgcn_mbcnt_hi((uint32_t)(b[e] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)b[e], before));
                }
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (in[e]) {
                        list[before++] = (u64)__float_as_uint(z[e]) << 32 | (uint32_t)(i + e);
                    }
            });
            __syncthreads();
            const int n = (int)lane_of(counts, NW - 1);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int t = tid * PER + i;
                lz[i] = t < n ? __uint_as_float((uint32_t)(list[t] >> 32)) : NEG;
                lat[i] = t < n ? (uint32_t)list[t] : 0;
            }
            if (top_p) {
                __syncthreads();
                clear_hist();
            }
            if (top_p) {
#pragma unroll
                for (int i = 0; i < PER; ++i)
                    if (lz[i] >= w.least) atomicAdd(&hist[bin_of(lz[i])], w.integer(lz[i]));
                __syncthreads();
                const u64 target = cross(std::true_type{}, 0, share);
                const int bin = s_bin;
                const u64 front = s_front;
#pragma unroll
                for (int i = 0; i < PER; ++i)
                    if (lz[i] > NEG && bin_of(lz[i]) == bin) {
                        const int at = atomicAdd(&s_n, 1);
                        if (at < CAND) cand[at] = rank_of(lz[i], (int)lat[i]);
                    }
                __syncthreads();
                if (s_n <= CAND) {
                    order_bin(std::true_type{}, front, target, s_n);
                    take_border();
                } else {
                    for (int i = tid; i < BINS; i += NT) hist[i] = 0;
                    __syncthreads();
                    find_border(std::true_type{}, share);
                }
            }
        } else if (top_p) {
            clear_hist();
            find_border(std::true_type{}, share);
        }
    }
    // min-p: the least value with enough weight.  It is within a few steps of float32 of where its logarithm says: a lane looks at each.
    if (!greedy && a.min_p > 0.0 && !none) {
        const int64_t most = key_of(hi), least = key_of(-MOST), guess = key_of((float)fmax((double)hi + a.min_p_below, -(double)MOST));
        const int64_t at = guess - 32 + lane, k = at < least ? least : at < most ? at : most;
        const float z = of_key((uint32_t)k);
        const u64 enough = __ballot(k == most || w.value(z) >= a.min_p);      // of the last lane on, at the least
        const float least_z = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(z), enough ? __builtin_ctzll(enough) : 63));
        if (least_z > b_z) {
            b_z = least_z;
            b_i = V;
        }
    }

    // ---- the draw: the mass that stays, by wavefronts (in index order), then the run, the lane and the entry
    u64 total = 0;
    if (a.tokens || probs) {
        float u = a.u ? a.u[r] : 0.f;
        u = u > 0.f ? (u < 1.f ? u : 0.99999994f) : 0.f;
        u64 x[PER], sum = 0, upto;
        if (listed) {
#pragma unroll
            for (int i = 0; i < PER; ++i) sum += x[i] = lz[i] >= w.least && inside((int)lat[i], lz[i]) ? w.integer(lz[i]) : 0;
        } else {
            each([&](int, const float z[4], const bool in[4]) {
                u64 x[4];
                w.integers(z, in, x);
                sum += (x[0] + x[1]) + (x[2] + x[3]);
            });
        }
        upto = wave_scan(sum);
        if (lane == 63) s_mass[wave] = upto;
        __syncthreads();
        const u64 waves = wave_scan(lane < NW ? s_mass[lane] : 0);
        total = lane_of(waves, NW - 1);
        const u64 target = (u64)((double)u * (double)total);
        u64 front = wave ? lane_of(waves, wave - 1) : 0;
        if (none && tid == 0 && a.tokens) a.tokens[r] = -1;
        if (a.tokens && front <= target && target < lane_of(waves, wave)) {      // uniform over the wavefront
            if (listed) {
                front += upto - sum;
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    if (front <= target && target < front + x[i]) a.tokens[r] = (int)lat[i];
                    front += x[i];
                }
            } else {
                each([&](int i, const float z[4], const bool in[4]) {
                    u64 x[4];
                    w.integers(z, in, x);
                    const u64 own = (x[0] + x[1]) + (x[2] + x[3]), run = wave_scan(own), c0 = front + run - own;
                    if (target >= c0 && target < c0 + own)
                        a.tokens[r] = target < c0 + x[0] ? i : target < c0 + x[0] + x[1] ? i + 1 : target < c0 + x[0] + x[1] + x[2] ? i + 2 : i + 3;
                    front += lane_of(run, 63);
                });
            }
        }
    }
    // ---- what stays
    if (probs || kept) {
        const double inv = total ? 1.0 / scalbn((double)total, -ONE) : 0.0, inv_t = greedy ? 1.0 : 1.0 / a.temperature;
        auto logit = [&](bool s, float x) { return s ? __builtin_amdgcn_fmed3f((float)((double)x * inv_t), -MOST, MOST) : NEG; };
        auto prob = [&](bool s, float x) { return s ? (float)(w.value(x) * inv) : 0.f; };
        if (listed) {
            __syncthreads();                // what the entries are written over has been written (a barrier waits for that)
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int at = (int)lat[i];
                if (lz[i] > NEG && inside(at, lz[i])) {
                    if (probs) probs[at] = prob(true, lz[i]);
                    if (kept) kept[at] = logit(true, lz[i]);
                }
            }
        } else {
            if (probs) each([&](int i, const float z[4], const bool s[4]) { put(probs, i, make_float4(prob(s[0], z[0]), prob(s[1], z[1]), prob(s[2], z[2]), prob(s[3], z[3]))); });
            if (kept && inv_t == 1.0) each([&](int i, const float z[4], const bool s[4]) { put(kept, i, make_float4(s[0] ? z[0] : NEG, s[1] ? z[1] : NEG, s[2] ? z[2] : NEG, s[3] ? z[3] : NEG)); });
            else if (kept) each([&](int i, const float z[4], const bool s[4]) { put(kept, i, make_float4(logit(s[0], z[0]), logit(s[1], z[1]), logit(s[2], z[2]), logit(s[3], z[3]))); });
        }
    }
}

template <int NT, bool LDS, int PER, int KIND = ANY_ROWS>
void run(const SampleArgs& a, hipStream_t st) {
    const int runs = (a.V + NT * 4 - 1) / (NT * 4);
    const int lds = LDS ? runs * NT * (int)sizeof(float4) : 0;
    auto kern = k_sample<NT, LDS, PER, KIND>;
    if constexpr (LDS) {
        static int attr_state[MAX_DEVICES] = {};
        if (!ensure_dynamic_lds_here(reinterpret_cast<const void*>(kern), LDS_ENTRIES * 4, attr_state)) return;
    }
    hipLaunchKernelGGL(kern, dim3(a.rows), dim3(NT), lds, st, a, runs);
}

}  // namespace

void launch_sample_filtered(const SampleArgs& args, hipStream_t st) {
    SampleArgs a = args;
    a.min_p_below = a.min_p > 0.0 ? a.temperature * log(a.min_p) : 0.0;
    // A row that has a CU to itself ends soonest with 1024 threads, a short one with 256, whose barriers cost less; more rows than CUs
    // share them, by the side of each other while two rows and their bins find room in LDS.  us, threads 256 / 512 / 1024:
    //   1 row of 1000 entries 7.9 / - / 8.2, 4096 11.2 / 9.2 / 9.5, 16384 29 / 19.6 / 16.4, 32768 - / 34 / 27
    //   600 rows of 1000 10.9 / 15.0 / -, 4096 17.2 / 19.6 / 27, 8192 26.5 / 27.6 / 33, 16384 64 / 47 / 53, 32768 - / 110 / 89
    //   2048 rows of 2048 23.5 / 34 / -, 4096 34 / 44 / 68, 8192 64 / 62 / 87, 16384 146 / 108 / 138
    // Kept in LDS / read again in every pass (1024 threads): 1 row of 8192 11.9 / 14.7, of 32768 26.9 / 30.5, 256 of 32768 33.6 / 37.5.
    const bool many = a.rows > cu_count();
    if (a.V <= (many ? 4096 : 2048)) run<256, true, 2>(a, st);
    else if (many && a.V <= LDS_ENTRIES / 2) run<512, true, 1>(a, st);
    else if (a.V <= LDS_ENTRIES) run<1024, true, 2>(a, st);
    else switch ((a.dtype == 1 ? 1 : 0) + (a.logits_u ? 2 : 0)) {
        case 0: run<1024, false, 2, 0>(a, st); break;
        case 1: run<1024, false, 2, 1>(a, st); break;
        case 2: run<1024, false, 2, 2>(a, st); break;
        default: run<1024, false, 2, 3>(a, st);
    }
}

}  // namespace mulo
