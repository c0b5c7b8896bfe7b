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

#include "mulo_internal.h"

namespace mulo {
namespace {

typedef unsigned long long u64;
constexpr float MOST = 3.402823466e38f;   // the largest finite float32
constexpr float NEG = -__builtin_huge_valf();
constexpr int BINS = 2048, CAND = 1024;   // bins of a histogram; entries of a bin that are ordered by comparing them all
constexpr int LDS_ENTRIES = 32768;        // of a row that is kept in LDS (128 KB)
constexpr int ONE = 44;                   // bits of the largest weight

// order-preserving integer of a value (not NaN); -0 and 0 are the same value
__device__ __forceinline__ uint32_t key_of(float z) {
    const uint32_t b = __float_as_uint(z == 0.f ? 0.f : z);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ u64 rank_of(float z, int i) { return (u64)key_of(z) << 32 | (uint32_t)~i; }

// 2^x for x <= 0 as p 2^n: x = n + f, |f| <= 1/2, p = the polynomial that interpolates 2^f in the 11 Chebyshev nodes
// (relative error 2^-51).  About 20 instructions at full rate; a library exp takes some 40.
struct Pow2 { double p; int n; };
__device__ __forceinline__ Pow2 pow2(double x) {
    const double shift = 6755399441055744.0;      // 1.5 2^52: the sum's low word is the nearest integer
    const double xs = x + shift, f = x - (xs - shift);
    double p = 7.072585949269223e-09;
    p = __builtin_fma(p, f, 1.0208690299958306e-07);
    p = __builtin_fma(p, f, 1.321544258792169e-06);
    p = __builtin_fma(p, f, 1.5252657260200837e-05);
    p = __builtin_fma(p, f, 0.0001540353044173605);
    p = __builtin_fma(p, f, 0.0013333558230164974);
    p = __builtin_fma(p, f, 0.009618129107606888);
    p = __builtin_fma(p, f, 0.05550410866444772);
    p = __builtin_fma(p, f, 0.24022650695910097);
    p = __builtin_fma(p, f, 0.69314718055995);
    p = __builtin_fma(p, f, 1.0);
    return Pow2{p, (int)__double_as_longlong(xs)};
}
__device__ __forceinline__ double scaled(const Pow2& w, int bits) {     // w 2^bits, bits + w.n > -1000
    return w.p * __longlong_as_double((long long)(1023 + bits + w.n) << 52);
}
struct Weights {
    float zmax;
    double c;      // log2(e) / temperature
    __device__ __forceinline__ double exponent(float z) const { return z == zmax ? 0.0 : ((double)z - (double)zmax) * c; }
    __device__ __forceinline__ u64 integer(float z) const {
        const double x = exponent(z);
        if (!(x >= -(ONE + 2.0))) return 0;
        return __double_as_longlong(scaled(pow2(x), ONE) + 4503599627370496.0) & 0xFFFFFFFFFFFFFull;      // + 2^52: rounds to an integer
    }
    __device__ __forceinline__ double value(float z) const {
        const double x = exponent(z);
        return x >= -900.0 ? scaled(pow2(x), 0) : 0.0;
    }
};

__device__ __forceinline__ u64 wave_sum(u64 v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
__device__ __forceinline__ u64 wave_scan(u64 v, int lane) {      // inclusive
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const u64 n = __shfl_up(v, o);
        if (lane >= o) v += n;
    }
    return v;
}

// LDS: the row is read from memory once and kept there; else every pass reads it again.  (Kept in registers, a row of 16384
// unrolls every pass 64 times: 70000 instructions, which neither registers nor the instruction cache hold.)
// Wavefront w has the stretch [w seg, (w + 1) seg) of the row, in runs of 256: consecutive lanes, consecutive entries.
// A thread takes the same entries in every pass.
template <int NT, bool LDS>
__global__ __launch_bounds__(NT) void k_sample(const SampleArgs a, int runs) {
    constexpr int NW = NT / 64;
    extern __shared__ __attribute__((aligned(16))) float4 kept_row[];      // [NW][runs][64]
    __shared__ __align__(16) u64 hist[BINS];       // then the entries of a bin, and their weights
    __shared__ u64 s_wave[NW], s_front, s_border;
    __shared__ float s_lo[NW], s_hi[NW];
    __shared__ int s_bin, s_n;
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
    auto row4 = [&](int i, float4 c, float4 u) -> float4 {     // guided; NaN, and what lies past the end, is masked
        auto clean = [&](float x, float y, int k) {
            const float z = zu ? __fadd_rn(y, __fmul_rn(a.cfg_scale, __fsub_rn(x, y))) : x;
            return z == z && k < V ? z : NEG;
        };
        return make_float4(clean(c.x, u.x, i), clean(c.y, u.y, i + 1), clean(c.z, u.z, i + 2), clean(c.w, u.w, i + 3));
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
    auto each = [&](auto&& f) {
        each4([&](int i, const float4 z) { f(i, z.x); f(i + 1, z.y); f(i + 2, z.z); f(i + 3, z.w); });
    };

    for (int i = tid; i < BINS; i += NT) hist[i] = 0;
    // ---- the largest entry, and the smallest that is not masked
    float hi = NEG, lo = -NEG;
    from_memory([&](int, const float4 z, int j) {
        if constexpr (LDS) mine[j * 64] = z;
        hi = fmaxf(fmaxf(hi, fmaxf(z.x, z.y)), fmaxf(z.z, z.w));
        auto floor = [](float x) { return x > NEG ? x : -NEG; };
        lo = fminf(fminf(lo, fminf(floor(z.x), floor(z.y))), fminf(floor(z.z), floor(z.w)));
    });
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        hi = fmaxf(hi, __shfl_xor(hi, o));
        lo = fminf(lo, __shfl_xor(lo, o));
    }
    if (lane == 0) { s_hi[wave] = hi; s_lo[wave] = lo; }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NW; ++i) {
        hi = fmaxf(hi, s_hi[i]);
        lo = fminf(lo, s_lo[i]);
    }
    const bool none = hi == NEG, greedy = a.temperature == 0.0;
    const Weights w{hi, greedy ? 0.0 : 1.4426950408889634 / a.temperature};
    u64 border = 0;       // C: entries with a rank of at least this stay, so far
    auto inside = [&](int i, float z) { return z > NEG && rank_of(z, i) >= border; };

    // ---- the head of what is inside that ends with the entry at which the count, or the mass, reaches want(all of it)
    // Bins along the value: linear over the range of the row, or over the first 128 below the maximum (masks of very low values).
    // Float subtraction and multiplication by a positive number are monotone, so a larger value is never in a later bin.
    const float scale = (float)BINS / fminf(hi - lo, 128.f);
    auto bin_of = [&](float z) {
        const float t = (hi - z) * scale;
        return t >= (float)(BINS - 1) ? BINS - 1 : t > 0.f ? (int)t : 0;      // NaN (no range, infinities): 0
    };
    // where the prefix sum of the bins reaches want: s_bin, and the sum in front of it in s_front; all of it in s_total
    auto cross = [&](u64 before, auto&& want) -> u64 {
        constexpr int PER = BINS / NT;
        u64 v[PER], sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) sum += v[i] = hist[tid * PER + i];
        const u64 upto = wave_scan(sum, lane);
        if (lane == 63) s_wave[wave] = upto;
        __syncthreads();
        u64 front = before + upto - sum, all = before;
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            if (i < wave) front += s_wave[i];
            all += s_wave[i];
        }
        const u64 target = want(all);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (front < target && front + v[i] >= target) {
                s_bin = tid * PER + i;
                s_front = front;
            }
            front += v[i];
        }
        if (tid == 0) s_n = 0;
        __syncthreads();
        return target;
    };
    auto find_border = [&](bool mass, auto&& want) {
        auto amount = [&](float z) -> u64 { return mass ? w.integer(z) : 1ull; };
        each([&](int i, float z) {
            if (inside(i, z)) {
                const u64 x = amount(z);
                if (x) atomicAdd(&hist[bin_of(z)], x);
            }
        });
        __syncthreads();
        const u64 target = cross(0, want);
        const int bin = s_bin;
        u64 front = s_front;
        each([&](int i, float z) {
            if (inside(i, z) && bin_of(z) == bin) {
                const int at = atomicAdd(&s_n, 1);
                if (at < CAND) cand[at] = rank_of(z, i);
            }
        });
        __syncthreads();
        const int n = s_n;
        if (n <= CAND) {
            if (mass) {
                for (int t = tid; t < n; t += NT) candw[t] = w.integer(of_key((uint32_t)(cand[t] >> 32)));
                __syncthreads();
            }
            for (int t = tid; t < n; t += NT) {
                const u64 own = cand[t];
                u64 before = front;
                for (int i = 0; i < n; ++i)
                    if (cand[i] > own) before += mass ? candw[i] : 1ull;
                if (before < target && before + (mass ? candw[t] : 1ull) >= target) s_border = own;
            }
            __syncthreads();
        } else {
            // by the digits of the rank, the largest first: 32 bits of the value, and the 18 of an index that can differ
            u64 known = 0, mask = 0;
            const int shifts[5] = {53, 42, 32, 9, 0};
#pragma unroll 1
            for (int d = 0; d < 5; ++d) {
                const int shift = shifts[d], bits = d < 2 ? 11 : d == 2 ? 10 : 9;
                for (int i = tid; i < BINS; i += NT) hist[i] = 0;
                __syncthreads();
                each([&](int i, float z) {
                    const u64 c = rank_of(z, i);
                    if (inside(i, z) && bin_of(z) == bin && (c & mask) == known) {
                        const u64 x = amount(z);
                        if (x) atomicAdd(&hist[(1 << bits) - 1 - (int)(c >> shift & ((1u << bits) - 1))], x);
                    }
                });
                __syncthreads();
                cross(front, [&](u64) { return target; });
                front = s_front;
                known |= (u64)((1 << bits) - 1 - s_bin) << shift;
                mask |= (u64)((1 << bits) - 1) << shift;
                if (d == 2) { known |= 0xFFFC0000ull; mask |= 0xFFFC0000ull; }      // an index below 2^18, inverted
            }
            if (tid == 0) s_border = known;
            __syncthreads();
        }
        border = s_border;
    };
    bool cleared = true;
    auto clear_hist = [&]() {
        if (!cleared) {
            for (int i = tid; i < BINS; i += NT) hist[i] = 0;
            __syncthreads();
        }
        cleared = false;
    };
    if (!none) {
        const int top_k = greedy ? 1 : a.top_k;
        if (top_k > 0 && top_k < V) {      // all of a row's entries stay where fewer than top_k are not masked
            clear_hist();
            find_border(false, [&](u64 all) { return all < (u64)top_k ? all : (u64)top_k; });
        }
        if (!greedy && a.top_p < 1.0) {
            clear_hist();
            find_border(true, [&](u64 all) {
                const u64 t = (u64)__builtin_ceil(a.top_p * (double)all);      // the mass in front of the next entry is below top_p of all
                return t < 1 ? 1ull : t < all ? t : all;
            });
        }
    }
    // min-p by the value, and by the weight itself next to the border
    float sure = NEG, never = NEG;
    const bool min_p = !greedy && a.min_p > 0.0 && !none;
    if (min_p) {
        const double d = log(a.min_p) * a.temperature, at = (double)hi + d, eps = 1e-6 * (fabs((double)hi) + fabs(d)) + 1e-40;
        sure = (float)(at + eps);
        never = (float)(at - eps);
    }
    auto stays = [&](int i, float z) {
        if (!inside(i, z)) return false;
        if (!min_p || z > sure || z == hi) return true;
        return z >= never && w.value(z) >= a.min_p;
    };

    // ---- the draw: the mass that stays, by wavefronts (in index order), then the run, the lane and the entry
    u64 total = 0;
    if (a.tokens || a.probs) {
        u64 sum = 0;
        each([&](int i, float z) { if (stays(i, z)) sum += w.integer(z); });
        sum = wave_sum(sum);
        __syncthreads();                    // s_wave of the searches has been read
        if (lane == 0) s_wave[wave] = sum;
        __syncthreads();
        u64 front = 0;
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            if (i < wave) front += s_wave[i];
            total += s_wave[i];
        }
        if (a.tokens) {
            float u = a.u[r];
            u = u > 0.f ? (u < 1.f ? u : 0.99999994f) : 0.f;
            const u64 target = (u64)((double)u * (double)total);
            if (none && tid == 0) a.tokens[r] = -1;
            if (front <= target && target < front + sum) {      // uniform over the wavefront
                each4([&](int i, const float4 z) {
                    const u64 w0 = stays(i, z.x) ? w.integer(z.x) : 0, w1 = stays(i + 1, z.y) ? w.integer(z.y) : 0,
                              w2 = stays(i + 2, z.z) ? w.integer(z.z) : 0, w3 = stays(i + 3, z.w) ? w.integer(z.w) : 0;
                    const u64 mine = w0 + w1 + w2 + w3, upto = wave_scan(mine, lane), run = __shfl(upto, 63);
                    const u64 c0 = front + upto - mine;
                    if (target >= c0 && target < c0 + mine)
                        a.tokens[r] = target < c0 + w0 ? i : target < c0 + w0 + w1 ? i + 1 : target < c0 + w0 + w1 + w2 ? i + 2 : i + 3;
                    front += run;
                });
            }
        }
    }
    // ---- what stays
    if (a.probs || a.kept) {
        const double inv = total ? 1.0 / scalbn((double)total, -ONE) : 0.0, inv_t = greedy ? 1.0 : 1.0 / a.temperature;
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
        each4([&](int i, const float4 z) {
            const bool s0 = stays(i, z.x), s1 = stays(i + 1, z.y), s2 = stays(i + 2, z.z), s3 = stays(i + 3, z.w);
            if (a.probs) put(a.probs + r * V, i, make_float4(s0 ? (float)(w.value(z.x) * inv) : 0.f, s1 ? (float)(w.value(z.y) * inv) : 0.f,
                                                             s2 ? (float)(w.value(z.z) * inv) : 0.f, s3 ? (float)(w.value(z.w) * inv) : 0.f));
            if (a.kept) {
                auto t = [&](bool s, float x) { return s ? fmaxf(-MOST, fminf(MOST, (float)((double)x * inv_t))) : NEG; };
                put(a.kept + r * V, i, make_float4(t(s0, z.x), t(s1, z.y), t(s2, z.z), t(s3, z.w)));
            }
        });
    }
}

template <int NT, bool LDS>
void run(const SampleArgs& a, hipStream_t st) {
    const int runs = (a.V + NT * 4 - 1) / (NT * 4);
    const int lds = LDS ? runs * NT * (int)sizeof(float4) : 0;
    auto kern = k_sample<NT, LDS>;
    if constexpr (LDS) {
        static int attr_state = 0;
        if (!ensure_dynamic_lds(reinterpret_cast<const void*>(kern), LDS_ENTRIES * 4, &attr_state)) return;
    }
    hipLaunchKernelGGL(kern, dim3(a.rows), dim3(NT), lds, st, a, runs);
}

}  // namespace

void launch_sample_filtered(const SampleArgs& a, hipStream_t st) {
    if (a.V <= 2048) run<256, true>(a, st);
    else if (a.V <= LDS_ENTRIES) run<1024, true>(a, st);
    else run<1024, false>(a, st);
}

}  // namespace mulo
