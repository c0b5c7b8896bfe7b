// Filtered draws: temperature, top-k, top-p and min-p, and a draw from a given uniform.
//
// A row's entries are ordered by (value descending, index ascending).  Each of top-k and top-p keeps a head of that order,
// which a key of the value and a number of entries with that very value describe: key > K, and the first n with key == K.
// Masses are integers, w = rint(2^44 exp((z - max z) / T)): sums of them (at most 2^62) do not depend on their order.
#include <hip/hip_bf16.h>

#include "mulo_internal.h"

namespace mulo {
namespace {

constexpr int TPB = 256;
typedef unsigned long long u64;
constexpr float MOST = 3.402823466e38f;   // the largest finite float32

struct Row {
    const void *c, *u;
    float s;
    bool bf16;
    __device__ __forceinline__ float load(const void* p, int i) const {
        return bf16 ? __bfloat162float(((const __hip_bfloat16*)p)[i]) : ((const float*)p)[i];
    }
    __device__ __forceinline__ float at(int i) const {
        float z = load(c, i);
        if (u) {
            const float zu = load(u, i);
            z = __fadd_rn(zu, __fmul_rn(s, __fsub_rn(z, zu)));
        }
        return z != z ? -__builtin_huge_valf() : z;
    }
};

// order-preserving integer of a value (not NaN); -0 and 0 are the same value
__device__ __forceinline__ uint32_t key_of(float z) {
    const uint32_t b = __float_as_uint(z == 0.f ? 0.f : z);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ u64 weight(float z, float zmax, double inv_t) {
    if (z == zmax) return 1ull << 44;
    return (u64)__builtin_rint(exp(((double)z - (double)zmax) * inv_t) * 17592186044416.0);
}

__device__ __forceinline__ u64 block_sum(u64 v, u64* red) {
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return red[0] + red[1] + red[2] + red[3];
}
// exclusive prefix over the workgroup, and the sum
__device__ __forceinline__ u64 block_scan(u64 v, u64* red, u64& total) {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    u64 x = v;
    for (int o = 1; o < 64; o <<= 1) {
        const u64 n = __shfl_up(x, o);
        if (lane >= o) x += n;
    }
    __syncthreads();
    if (lane == 63) red[wv] = x;
    __syncthreads();
    u64 before = 0;
    total = 0;
    for (int i = 0; i < 4; ++i) {
        if (i < wv) before += red[i];
        total += red[i];
    }
    return before + x - v;
}

__global__ __launch_bounds__(TPB) void k_sample_rows(const SampleArgs a) {
    __shared__ u64 hist[256], red[4], s_rest;
    __shared__ uint32_t s_key;
    const int64_t r = blockIdx.x;
    const int tid = threadIdx.x, V = a.V;
    const size_t e = a.dtype == 1 ? 2 : 4;
    const Row row{(const char*)a.logits + r * a.row_stride * e, a.logits_u ? (const char*)a.logits_u + r * a.row_stride * e : nullptr,
                  a.cfg_scale, a.dtype == 1};
    const float NEG = -__builtin_huge_valf();
    u64 mk = 0;
    for (int i = tid; i < V; i += TPB) {
        const u64 k = key_of(row.at(i));
        mk = k > mk ? k : mk;
    }
    for (int o = 32; o > 0; o >>= 1) { const u64 n = __shfl_xor(mk, o); mk = n > mk ? n : mk; }
    if ((tid & 63) == 0) red[tid >> 6] = mk;
    __syncthreads();
    for (int i = 0; i < 4; ++i) mk = red[i] > mk ? red[i] : mk;
    const uint32_t kmax = (uint32_t)mk;
    const float zmax = __uint_as_float(kmax & 0x80000000u ? kmax & 0x7fffffffu : ~kmax);
    const bool none = zmax == NEG;
    const double inv_t = a.temperature > 0.0 ? 1.0 / a.temperature : 1.0;
    const int top_k = a.temperature > 0.0 ? a.top_k : 1;
    // the head of the order: key > K, or key == K and fewer than n such entries in front
    uint32_t K = key_of(NEG);
    u64 n = 0;                        // of the entries at -inf none stays
    auto stays = [&](uint32_t k, u64 tie) { return k > K || (k == K && tie < n); };
    // head whose `amount` (a count, or a mass) reaches `want`: radix search from the top byte down
    auto search = [&](u64 want, bool mass, auto&& in_set) {
        uint32_t prefix = 0;
        u64 rest = want;
        for (int shift = 24; shift >= 0; shift -= 8) {
            hist[tid] = 0;
            __syncthreads();
            for (int i = tid; i < V; i += TPB) {
                const float z = row.at(i);
                const uint32_t k = key_of(z);
                if (k > key_of(NEG) && (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) && in_set(k))
                    atomicAdd(&hist[(k >> shift) & 255], mass ? weight(z, zmax, inv_t) : 1ull);
            }
            __syncthreads();
            if (tid == 0) {
                int d = 255;
                while (d > 0 && hist[d] < rest) rest -= hist[d--];
                s_key = prefix | ((uint32_t)d << shift);
                s_rest = rest;
            }
            __syncthreads();
            prefix = s_key;
            rest = s_rest;
        }
        K = prefix;
        return rest;
    };
    u64 count = 0;
    for (int i = tid; i < V; i += TPB) count += row.at(i) > NEG;
    count = block_sum(count, red);
    if (top_k > 0 && (u64)top_k < count) n = search(top_k, false, [](uint32_t) { return true; });
    // all members at K may have to share it with entries that are out already: ties with an index rank
    if (a.temperature > 0.0 && a.top_p < 1.0 && !none) {
        const uint32_t K0 = K;
        const u64 n0 = n;
        u64 mass = 0;
        for (int i = tid; i < V; i += TPB) {
            const float z = row.at(i);
            if (key_of(z) > K0) mass += weight(z, zmax, inv_t);
        }
        mass = block_sum(mass, red);
        const float z0 = __uint_as_float(K0 & 0x80000000u ? K0 & 0x7fffffffu : ~K0);
        const u64 w0 = n0 ? weight(z0, zmax, inv_t) : 0;
        mass += n0 * w0;
        // the head ends with the first entry whose inclusive mass is at least top_p * mass
        const double want = a.top_p * (double)mass;
        const u64 need = (u64)__builtin_ceil(want);
        u64 above = 0;      // mass of entries larger than K0
        above = mass - n0 * w0;
        if (need > above && n0) {       // inside the ties of K0
            u64 t = w0 ? (need - above + w0 - 1) / w0 : n0;
            n = t < n0 ? t : n0;
        } else {
            const u64 rest = search(need > 0 ? need : 1, true, [&](uint32_t k) { return k > K0; });
            const float zk = __uint_as_float(K & 0x80000000u ? K & 0x7fffffffu : ~K);
            const u64 wk = weight(zk, zmax, inv_t);
            n = wk ? (rest + wk - 1) / wk : 1ull << 40;
        }
    }
    // the mass that stays, in index order
    const double min_w = a.min_p;
    u64 total = 0, ties = 0, target = 0;
    int token = -1;
    for (int pass = 0; pass < 2; ++pass) {
        u64 sum = 0;
        ties = 0;
        for (int i0 = 0; i0 < V; i0 += TPB) {
            const int i = i0 + tid;
            const float z = i < V ? row.at(i) : NEG;
            const uint32_t k = key_of(z);
            u64 t_all, w_all;
            const u64 rank = block_scan(z > NEG && k == K, red, t_all) + ties;
            ties += t_all;
            bool in = z > NEG && stays(k, rank);
            if (in && a.temperature > 0.0 && min_w > 0.0) in = z == zmax || exp(((double)z - (double)zmax) * inv_t) >= min_w;
            const u64 w = in ? weight(z, zmax, inv_t) : 0;
            const u64 before = block_scan(w, red, w_all) + sum;
            if (pass == 1) {
                if (i < V) {
                    if (a.probs) a.probs[r * V + i] = total ? (float)((double)w / (double)total) : 0.f;
                    if (a.kept) a.kept[r * V + i] = in ? fmaxf(-MOST, fminf(MOST, (float)(a.temperature > 0.0 ? (double)z / a.temperature : (double)z))) : NEG;
                }
                if (w && before <= target && target < before + w && a.tokens) a.tokens[r] = i;
            }
            sum += w_all;
        }
        if (pass == 0) {
            total = sum;
            float u = a.u ? a.u[r] : 0.f;
            u = u > 0.f ? (u < 1.f ? u : 0.99999994f) : 0.f;
            target = (u64)((double)u * (double)total);
            if (!total && tid == 0 && a.tokens) a.tokens[r] = token;
            __syncthreads();
        }
    }
}

}  // namespace

void launch_sample_filtered(const SampleArgs& a, hipStream_t st) {
    hipLaunchKernelGGL(k_sample_rows, dim3(a.rows), dim3(TPB), 0, st, a);
}

}  // namespace mulo
