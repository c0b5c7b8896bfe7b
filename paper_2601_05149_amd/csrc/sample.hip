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
#include <hip/hip_bf16.h>

#include <type_traits>

#include "mulo_internal.h"

namespace mulo {
namespace {

typedef unsigned long long u64;
constexpr float MOST = 3.402823466e38f;   // the largest finite float32
constexpr float NEG = -__builtin_huge_valf();
constexpr int BINS = 1024, CAND = 512;    // bins of a histogram; entries of a bin that are ordered by comparing them all
constexpr int DIGIT = 10;                 // bits of a rank that a histogram of them tells apart
constexpr int LDS_ENTRIES = 32768;        // of a row that is kept in LDS (128 KB)
constexpr int ONE = 44;                   // bits of the largest weight

// order-preserving integer of a value (not NaN); -0 and 0 are the same value
__device__ __forceinline__ uint32_t key_of(float z) {
    const uint32_t b = __float_as_uint(z == 0.f ? 0.f : z);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ u64 rank_of(float z, int i) { return (u64)key_of(z) << 32 | (uint32_t)~i; }

// Weights, 2^x with x = (z - max z) log2(e) / T <= 0.  y = STEPS x = n + f, |f| <= 1/2:
//   2^x = 2^(n / STEPS) e^t, t = f ln 2 / STEPS, |t| <= 1.4e-3
// The first factor is a table's, its exponent moved.  e^t - 1 = t + t^2 (1/2 + t (1/6 + t / 24)): the sum's second part is below
// 2^-20 and float32 is enough for it, so that 10 operations in 64 bits are left, at 8 cycles each half of the time (a
// polynomial of 2^x over all of [-1/2, 1/2] takes 18).  Relative error: 2^-43.
constexpr int STEPS = 256;
struct Weights {
    double zmax, c;            // the maximum (of infinite ones: the largest finite number); STEPS log2(e) / temperature
    float least_value, least;  // smallest z with a weight that value(), and integer(), tell from 0
    const double* table;       // 2^(i / STEPS), in LDS
    __device__ __forceinline__ double part(float z, int bits) const {     // 2^(x + bits), for z of at least least_value
        const double shift = 6755399441055744.0;      // 1.5 2^52: the sum's low word is the nearest integer
        const double d = (double)fminf(z, MOST) - zmax;
        const double ys = __builtin_fma(d, c, shift), f = __builtin_fma(d, c, -(ys - shift));
        const int n = (int)__double_as_longlong(ys);
        const long long tb = __double_as_longlong(table[n & (STEPS - 1)]) + ((long long)((n >> 8) + bits) << 52);
        const float t = (float)f * (float)(0.6931471805599453 / STEPS);
        const double r = __builtin_fma(f, 0.6931471805599453 / STEPS, (double)(t * t * __builtin_fmaf(t, __builtin_fmaf(t, 1.f / 24.f, 1.f / 6.f), 0.5f)));
        const double tw = __longlong_as_double(tb);
        return __builtin_fma(tw, r, tw);
    }
    __device__ __forceinline__ u64 integer(float z, bool in) const {       // + 2^52: rounds to an integer
        const u64 t = __double_as_longlong(part(z, ONE) + 4503599627370496.0) & 0xFFFFFFFFFFFFFull;
        return (in && z >= least) ? t : 0;
    }
    // of the entries of four that are in: side by side, without a branch
    __device__ __forceinline__ void integers(const float z[4], const bool in[4], u64 out[4]) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] = 0;
        if (!__any(in[0] || in[1] || in[2] || in[3])) return;
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] = integer(z[e], in[e]);
    }
    __device__ __forceinline__ double value(float z) const { return z >= least_value ? part(z, 0) : 0.0; }
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
// (masses, top-p, the draw's sums, what is written of them) goes by the list: of 16384 entries 2000 cost an eighth.
template <int NT, bool LDS, int PER>
__global__ __launch_bounds__(NT) void k_sample(const SampleArgs a, int runs) {
    constexpr int NW = NT / 64;
    extern __shared__ __attribute__((aligned(16))) float4 kept_row[];      // [NW][runs][64]
    __shared__ __align__(16) u64 hist[BINS];       // then the entries of a bin, and their weights
    __shared__ double table[STEPS];
    __shared__ u64 s_wave[NW], s_mass[NW], s_front, s_border;
    __shared__ float s_lo[NW], s_hi[NW];
    __shared__ int s_bin, s_n, s_listed;
    __shared__ float list_z[PER * NT];
    __shared__ uint32_t list_at[PER * NT];         // wavefront << 18 | index
    u64* const cand = hist;
    u64* const candw = hist + CAND;

    const int64_t r = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), V = a.V;
    const int w_first = wave * runs * 256, w_runs = V - w_first <= 0 ? 0 : (V - w_first + 255) / 256 < runs ? (V - w_first + 255) / 256 : runs;
    const int first = w_first + lane * 4;
    float4* const mine = kept_row + wave * runs * 64 + lane;
    const bool bf16 = a.dtype == 1;
    const size_t esz = bf16 ? 2 : 4;
    const char* const zc = (const char*)a.logits + r * a.row_stride * esz;
    const char* const zu = a.logits_u ? (const char*)a.logits_u + r * a.row_stride * esz : nullptr;
    // whole vectors where rows allow it (entries past the end re-read the row's first)
    const bool vectors = (((uintptr_t)zc | (uintptr_t)zu) & (esz * 4 - 1)) == 0 && (V & 3) == 0;
    auto raw4 = [&](const char* p, int i) -> float4 {
        if (vectors) {
            const size_t at = i < V ? i : 0;
            if (!bf16) return *reinterpret_cast<const float4*>(p + at * 4);
            const uint2 t = *reinterpret_cast<const uint2*>(p + at * 2);
            return make_float4(__uint_as_float(t.x << 16), __uint_as_float(t.x & 0xFFFF0000u), __uint_as_float(t.y << 16), __uint_as_float(t.y & 0xFFFF0000u));
        }
        auto one = [&](int k) {
            k = k < V ? k : 0;
            return bf16 ? __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(p)[k] << 16) : reinterpret_cast<const float*>(p)[k];
        };
        return make_float4(one(i), one(i + 1), one(i + 2), one(i + 3));
    };
    auto row4 = [&](int i, float4 c, float4 u) -> float4 {     // guided; NaN (a maximum's other operand), and what lies past the end, is masked
        if (zu) {
            auto guide = [&](float x, float y) { return __fadd_rn(y, __fmul_rn(a.cfg_scale, __fsub_rn(x, y))); };
            c = make_float4(guide(c.x, u.x), guide(c.y, u.y), guide(c.z, u.z), guide(c.w, u.w));
        }
        c = make_float4(fmaxf(c.x, NEG), fmaxf(c.y, NEG), fmaxf(c.z, NEG), fmaxf(c.w, NEG));
        if (i - lane * 4 + 256 > V) c = make_float4(i < V ? c.x : NEG, i + 1 < V ? c.y : NEG, i + 2 < V ? c.z : NEG, i + 3 < V ? c.w : NEG);
        return c;
    };
    // f(index of the first, four entries, number of the run), four runs requested together
    auto from_memory = [&](auto&& f) {
        for (int j0 = 0; j0 < w_runs; j0 += 4) {
            float4 c[4], u[4] = {};
#pragma unroll
            for (int j = 0; j < 4; ++j) c[j] = raw4(zc, first + (j0 + j) * 256);
            if (zu) {
#pragma unroll
                for (int j = 0; j < 4; ++j) u[j] = raw4(zu, first + (j0 + j) * 256);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j0 + j < w_runs) f(first + (j0 + j) * 256, row4(first + (j0 + j) * 256, c[j], u[j]), j0 + j);
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
        if ((V & 3) == 0 && ((uintptr_t)row & 15) == 0) {
            if (i < V) *reinterpret_cast<float4*>(row + i) = v;
        } else {
            if (i < V) row[i] = v.x;
            if (i + 1 < V) row[i + 1] = v.y;
            if (i + 2 < V) row[i + 2] = v.z;
            if (i + 3 < V) row[i + 3] = v.w;
        }
    };
    for (int i = tid; i < BINS; i += NT) hist[i] = 0;
    if (tid < STEPS) table[tid] = exp2((double)tid / STEPS);
    if (tid < NW) s_mass[tid] = 0;
    if (tid == 0) s_listed = 0;
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
    const bool none = hi == NEG;
    // with infinite entries the largest finite number takes the maximum's place
    const float top = fminf(hi, MOST);
    const double per_x = STEPS * 1.4426950408889634, c_w = greedy ? 0.0 : per_x / a.temperature, per_z = a.temperature * 0.6931471805599453;
    auto at_least = [&](double bits) { return (float)fmax((double)top - bits * per_z, -(double)MOST); };
    const Weights w{(double)top, c_w, at_least(900.0), at_least(ONE + 2.0), table};
    // the border, so far: entries above b_z stay, and those at it up to index b_i
    float b_z = NEG;
    int b_i = -1;
    auto inside = [&](int i, float z) -> bool { return (z > b_z) | ((z == b_z) & (i <= b_i)); };
    auto each = [&](auto&& f) {      // f(index of the first, the four, which of them are inside)
        each4([&](int i, const float4 v) {
            const float z[4] = {v.x, v.y, v.z, v.w};
            const bool in[4] = {inside(i, v.x), inside(i + 1, v.y), inside(i + 2, v.z), inside(i + 3, v.w)};
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
            for (int t = tid; t < n; t += NT) candw[t] = w.integer(of_key((uint32_t)(cand[t] >> 32)), true);
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
                u64 x[4];
                w.integers(z, in, x);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (x[e]) atomicAdd(&hist[bin(e)], x[e]);
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
                    add(z, here, [&](int e) { return BINS - 1 - (int)(short_rank(z[e], i + e) >> shift & (BINS - 1)); });
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
    static_assert(BINS == 1 << DIGIT, "a bin for every digit");
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
            each([&](int i, const float z[4], const bool in[4]) {
                u64 b[4];
                int upto[5] = {0};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    b[e] = __ballot(in[e]);
                    upto[e + 1] = upto[e] + __popcll(b[e]);
                }
                if (upto[4] == 0) return;
                int base = 0;
                if (lane == 0) base = atomicAdd(&s_listed, upto[4]);
                base = __builtin_amdgcn_readfirstlane(base);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (in[e]) {
                        const int at = base + upto[e] + __builtin_amdgcn_mbcnt_hi((uint32_t)(b[e] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)b[e], 0));
                        list_z[at] = z[e];
                        list_at[at] = (uint32_t)wave << 18 | (uint32_t)(i + e);
                    }
            });
            clear_hist();
            __syncthreads();
            const int n = s_listed;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int t = tid + i * NT;
                lz[i] = t < n ? list_z[t] : NEG;
                lat[i] = t < n ? list_at[t] : 0;
            }
            if (top_p) {
#pragma unroll
                for (int i = 0; i < PER; ++i)
                    if (lz[i] > NEG) {
                        const u64 x = w.integer(lz[i], true);
                        if (x) atomicAdd(&hist[bin_of(lz[i])], x);
                    }
                __syncthreads();
                const u64 target = cross(std::true_type{}, 0, share);
                const int bin = s_bin;
                const u64 front = s_front;
#pragma unroll
                for (int i = 0; i < PER; ++i)
                    if (lz[i] > NEG && bin_of(lz[i]) == bin) {
                        const int at = atomicAdd(&s_n, 1);
                        if (at < CAND) cand[at] = rank_of(lz[i], (int)(lat[i] & 0x3FFFFu));
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
    // min-p: the least value with enough weight, from where its logarithm says, a step of float32 at a time
    if (!greedy && a.min_p > 0.0 && !none) {
        const uint32_t most = key_of(hi), least = key_of(-MOST);
        auto enough = [&](uint32_t k) { return k >= most || w.value(of_key(k)) >= a.min_p; };
        uint32_t k = key_of((float)fmax((double)hi + log(a.min_p) * a.temperature, -(double)MOST));
        k = k < most ? k : most;
        for (int i = 0; i < 8 && !enough(k); ++i) ++k;
        for (int i = 0; i < 8 && k > least && enough(k - 1); ++i) --k;
        if (of_key(k) > b_z) {
            b_z = of_key(k);
            b_i = V;
        }
    }

    // ---- the draw: the mass that stays, by wavefronts (in index order), then the run, the lane and the entry
    u64 total = 0;
    if (a.tokens || probs) {
        __syncthreads();                    // s_wave of the searches has been read
        if (listed) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const u64 x = lz[i] > NEG && inside((int)(lat[i] & 0x3FFFFu), lz[i]) ? w.integer(lz[i], true) : 0;
                if (x) atomicAdd(&s_mass[lat[i] >> 18], x);
            }
        } else {
            u64 sum = 0;
            each([&](int, const float z[4], const bool in[4]) {
                u64 x[4];
                w.integers(z, in, x);
                sum += (x[0] + x[1]) + (x[2] + x[3]);
            });
            sum = lane_of(wave_scan(sum), 63);
            if (lane == 0) s_mass[wave] = sum;
        }
        __syncthreads();
        const u64 own = lane < NW ? s_mass[lane] : 0, waves = wave_scan(own);
        total = lane_of(waves, NW - 1);
        if (a.tokens) {
            float u = a.u[r];
            u = u > 0.f ? (u < 1.f ? u : 0.99999994f) : 0.f;
            const u64 target = (u64)((double)u * (double)total);
            if (none && tid == 0) a.tokens[r] = -1;
            u64 front = wave ? lane_of(waves, wave - 1) : 0;
            if (front <= target && target < lane_of(waves, wave)) {      // uniform over the wavefront
                each([&](int i, const float z[4], const bool in[4]) {
                    u64 x[4];
                    w.integers(z, in, x);
                    const u64 own = (x[0] + x[1]) + (x[2] + x[3]), upto = wave_scan(own), c0 = front + upto - own;
                    if (target >= c0 && target < c0 + own)
                        a.tokens[r] = target < c0 + x[0] ? i : target < c0 + x[0] + x[1] ? i + 1 : target < c0 + x[0] + x[1] + x[2] ? i + 2 : i + 3;
                    front += lane_of(upto, 63);
                });
            }
        }
    }
    // ---- what stays
    if (probs || kept) {
        const double inv = total ? 1.0 / scalbn((double)total, -ONE) : 0.0, inv_t = greedy ? 1.0 : 1.0 / a.temperature;
        auto logit = [&](bool s, float x) { return s ? fmaxf(-MOST, fminf(MOST, (float)((double)x * inv_t))) : NEG; };
        auto prob = [&](bool s, float x) { return s ? (float)(w.value(x) * inv) : 0.f; };
        if (listed) {
            __syncthreads();                // what the entries are written over has been written (a barrier waits for that)
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int at = (int)(lat[i] & 0x3FFFFu);
                if (lz[i] > NEG && inside(at, lz[i])) {
                    if (probs) probs[at] = prob(true, lz[i]);
                    if (kept) kept[at] = logit(true, lz[i]);
                }
            }
        } else {
            each([&](int i, const float z[4], const bool s[4]) {
                if (probs) put(probs, i, make_float4(prob(s[0], z[0]), prob(s[1], z[1]), prob(s[2], z[2]), prob(s[3], z[3])));
                if (kept) put(kept, i, make_float4(logit(s[0], z[0]), logit(s[1], z[1]), logit(s[2], z[2]), logit(s[3], z[3])));
            });
        }
    }
}

template <int NT, bool LDS, int PER>
void run(const SampleArgs& a, hipStream_t st) {
    const int runs = (a.V + NT * 4 - 1) / (NT * 4);
    const int lds = LDS ? runs * NT * (int)sizeof(float4) : 0;
    auto kern = k_sample<NT, LDS, PER>;
    if constexpr (LDS) {
        static int attr_state = 0;
        if (!ensure_dynamic_lds(reinterpret_cast<const void*>(kern), LDS_ENTRIES * 4, &attr_state)) return;
    }
    hipLaunchKernelGGL(kern, dim3(a.rows), dim3(NT), lds, st, a, runs);
}

}  // namespace

void launch_sample_filtered(const SampleArgs& a, hipStream_t st) {
    if (a.V <= 2048) run<256, true, 2>(a, st);
    else if (a.V <= LDS_ENTRIES) {
        if (a.rows > cu_count()) run<512, true, 1>(a, st);
        else run<1024, true, 2>(a, st);
    }
    else run<1024, false, 2>(a, st);
}

}  // namespace mulo
