// Attention over a prefix that sequences share and the rows each has of its own, with a window and sinks.
#include <hip/hip_bf16.h>

#include "mulo_internal.h"

namespace mulo {
namespace {

constexpr int NTH = 256;

template <class T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__hip_bfloat16>(__hip_bfloat16 v) { return __bfloat162float(v); }
template <class T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __hip_bfloat16 from_f32<__hip_bfloat16>(float v) { return __float2bfloat16(v); }

__device__ __forceinline__ float block_reduce(float v, float* red, bool is_max) {
    for (int o = 32; o > 0; o >>= 1) {
        const float n = __shfl_xor(v, o);
        v = is_max ? fmaxf(v, n) : v + n;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    float r = red[0];
    for (int i = 1; i < NTH / 64; ++i) r = is_max ? fmaxf(r, red[i]) : r + red[i];
    return r;
}

// one workgroup per query, 256 keys at a time, running maximum and sum
template <class T, int DH>
__global__ __launch_bounds__(NTH) void k_context_rows(const ContextAttn a) {
    __shared__ float qs[DH], ps[NTH], red[NTH / 64], os[NTH];
    const int tid = threadIdx.x;
    const int j = blockIdx.x % a.L, h = (blockIdx.x / a.L) % a.nh, b = blockIdx.x / (a.L * a.nh);
    const int kvh = h / (a.nh / a.nkv), g = b / (a.B / a.G);
    int own = (a.P_seq ? a.P_seq[b] : a.P);
    own = own < a.rows - a.L ? own : a.rows - a.L;
    bool absent = own < 0;
    own += j;
    if (a.pos_tab) {
        own = a.pos_tab[(int64_t)b * a.L + j];
        absent = own < 0;
    }
    const T* q = (const T*)a.q + b * a.q_batch + h * a.q_head + j * a.q_row;
    const T* k = (const T*)a.k + b * a.k_batch + kvh * a.k_head;
    const T* v = (const T*)a.v + b * a.v_batch + kvh * a.v_head;
    const T* pk = (const T*)a.pk + g * a.pk_group + kvh * a.pk_head;
    const T* pv = (const T*)a.pv + g * a.pv_group + kvh * a.pv_head;
    if (tid < DH) qs[tid] = to_f32<T>(q[tid]);
    __syncthreads();
    const int p = a.S + own;
    float m = -__builtin_huge_valf(), l = 0.f, o = 0.f;
    const int c = tid % DH, part = tid / DH, parts = NTH / DH;
    for (int t0 = 0; !absent && t0 <= p; t0 += NTH) {
        const int t = t0 + tid;
        bool see = t <= p && (a.window == 0 || t < a.sinks || p - t < a.window);
        if (a.hide && see && t >= a.S && t < p) {
            const int x = t - a.S - a.P0;
            if (x >= 0 && x < a.Lblk && a.hide[(int64_t)b * a.Lblk + x]) see = false;
        }
        float s = -__builtin_huge_valf();
        if (see) {
            const T* kr = t < a.S ? pk + t * a.pk_row : k + (t - a.S) * a.k_row;
            s = 0.f;
            for (int i = 0; i < DH; ++i) s += qs[i] * to_f32<T>(kr[i]);
            s *= a.scale_log2;
        }
        const float mn = fmaxf(m, block_reduce(s, red, true));
        const float ms = mn == -__builtin_huge_valf() ? 0.f : mn;
        const float w = see ? exp2f(s - ms) : 0.f;
        ps[tid] = see ? w : -1.f;
        const float alpha = exp2f(m - ms);
        l = l * alpha + block_reduce(w, red, false);
        m = mn;
        o *= alpha;
        for (int i = part; i < NTH; i += parts) {
            const float w_i = ps[i];
            const int ti = t0 + i;
            if (w_i >= 0.f) o += w_i * to_f32<T>(ti < a.S ? pv[c * a.pv_chan + ti] : v[c * a.v_chan + ti - a.S]);
        }
        __syncthreads();
    }
    os[tid] = o;
    __syncthreads();
    if (tid < DH) {
        float r = 0.f;
        for (int i = 0; i < parts; ++i) r += os[i * DH + tid];
        r = l > 0.f ? r / l : 0.f;
        T* out = (T*)a.out;
        const int row = b * a.L + j;
        out[a.frag ? frag_index(row, h * DH + tid, a.nh * DH) : b * a.out_batch + h * a.out_head + j * a.out_row + tid] = from_f32<T>(r);
    }
}

template <class T>
void launch_rows(const ContextAttn& a, hipStream_t st) {
    const dim3 grid((unsigned)((int64_t)a.B * a.nh * a.L));
    if (a.dh == 128) hipLaunchKernelGGL((k_context_rows<T, 128>), grid, dim3(NTH), 0, st, a);
    else hipLaunchKernelGGL((k_context_rows<T, 64>), grid, dim3(NTH), 0, st, a);
}

}  // namespace

size_t context_attention_floats(const ContextAttn&) { return 0; }

void launch_context_attention(const ContextAttn& a, hipStream_t st) {
    if (a.dtype == 1) launch_rows<__hip_bfloat16>(a, st);
    else launch_rows<float>(a, st);
}

}  // namespace mulo
