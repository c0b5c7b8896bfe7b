// A cache in 4 or 8 bits: rows packed as they are written, and read back.  (The formats and the tiles: include/mulo.h.)
#include <hip/hip_bf16.h>

#include <type_traits>

#include "index_div.h"
#include "mulo_internal.h"
#include "packed_tile.h"

namespace mulo {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) short i16x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

// ---- eight numbers and their codes ---------------------------------------------------------------------------------
// The byte 127 + e of a group whose largest |x| has these bits: e is the smallest integer with |x| <= T 2^e, T = 7 = 1.75 2^2 or
// 464 = 1.8125 2^8.  Infinities and NaN have the largest bits of all: 255.
template <int FMT> __device__ __forceinline__ uint32_t scale_byte(uint32_t bits) {
    constexpr int TE = FMT == FP4 ? 2 : 8, TOP = FMT == FP4 ? 252 : 246;
    constexpr uint32_t TM = FMT == FP4 ? 0x600000u : 0x680000u;
    if (bits >= 0x7F800000u) return 255;
    const int b = (int)(bits >> 23) - TE + ((bits & 0x7FFFFFu) > TM ? 1 : 0);
    return (uint32_t)(b < 10 ? 10 : b > TOP ? TOP : b);
}
template <int FMT> using Codes8 = std::conditional_t<FMT == FP4, uint32_t, uint2>;
__device__ __forceinline__ Codes8<FP4> encode8(std::integral_constant<int, FP4>, const float* x, float s) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
}
// (The conversion to 8 bits takes what lies beyond the grid for NaN.)
__device__ __forceinline__ Codes8<FP8> encode8(std::integral_constant<int, FP8>, const float* x, float s) {
    const float top = 448.f * s;
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __builtin_amdgcn_fmed3f(x[i], -top, top);
    i16x2 a = {0, 0}, b = {0, 0};
    a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(a, y[0], y[1], s, false);
    a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(a, y[2], y[3], s, true);
    b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, y[4], y[5], s, false);
    b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, y[6], y[7], s, true);
    return make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ void decode8(uint32_t w, float s, float* x) {
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1),
                c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 3);
    x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y; x[4] = c.x; x[5] = c.y; x[6] = d.x; x[7] = d.y;
}
__device__ __forceinline__ void decode8(uint2 w, float s, float* x) {
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.x, s, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.x, s, true),
                c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.y, s, false), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.y, s, true);
    x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y; x[4] = c.x; x[5] = c.y; x[6] = d.x; x[7] = d.y;
}
__device__ __forceinline__ void load8(const __bf16* p, float* x) {
    const bf16x8 v = *reinterpret_cast<const bf16x8*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
}
__device__ __forceinline__ void load8(const float* p, float* x) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void store8(__bf16* p, const float* x) {
    bf16x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (__bf16)x[i];      // exact
    __builtin_nontemporal_store(v, reinterpret_cast<bf16x8*>(p));
}
__device__ __forceinline__ void store8(float* p, const float* x) {
    __builtin_nontemporal_store(f32x4{x[0], x[1], x[2], x[3]}, reinterpret_cast<f32x4*>(p));
    __builtin_nontemporal_store(f32x4{x[4], x[5], x[6], x[7]}, reinterpret_cast<f32x4*>(p + 4));
}
template <int X> __device__ __forceinline__ uint32_t quad_swap(uint32_t v) {      // lane ^ 1 or ^ 2
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, X == 1 ? 0xB1 : 0x4E, 0xF, 0xF, true);
}

// ---- rows in, rows out ----------------------------------------------------------------------------------------------
// A thread has eight channels of a row, four threads a group: 16 bytes of bf16 in, 4 or 8 bytes of codes out, or the other way round.
// Values that come as channels of rows go through LDS, 64 rows a workgroup: in pieces of 16 bytes 4 x 1024 rows of 32 heads of 128 pack in
// 18 us (85 MB, 4.7 TB/s; 8 bits 22) and come back in 15 (16.5); float32 32 and 28; number by number the first two took 92 us.
// Bound by the numbers' bytes; 4 x 4224 rows back, 350 MB, in 50 us, 7 TB/s: written past the caches, which hold the codes that are read, against
// 72 us through them (8 bits 70 us; float32 141, 4.4 TB/s, and as rows of channels, whose lines are written in halves, 4 x 1024 rows in 47).  A token's
// rows of 32 sequences take 3 us, a launch's time.
constexpr int ROWS_THREADS = 256;
struct __attribute__((packed, aligned(2))) Piece { u32x4 v; };
struct RowsArgs : PackedRows {
    Div by_L, by_nkv, by_chunks;
    uint32_t k_blocks;      // the first ones of the grid
    int total, chunks;      // rows of the call; workgroups of a (sequence, head) whose values are channels of rows
    bool v_across, v_whole;      // values are channels of rows; in whole pieces of 16 bytes
};
template <int FMT, int DH> __device__ __forceinline__ void put(uint8_t* tile, int r, int t8, bool keys, Codes8<FMT> w, uint32_t byte) {
    using TL = Tile<FMT, DH>;
    constexpr int B8 = sizeof(w);      // bytes of eight channels
    if (keys) {
        *reinterpret_cast<Codes8<FMT>*>(tile + r * TL::ROW + t8 * B8) = w;
    } else if constexpr (DH == 128) {
        *reinterpret_cast<Codes8<FMT>*>(tile + TL::v_code(r, t8)) = w;
    } else if constexpr (FMT == FP4) {
        *reinterpret_cast<uint16_t*>(tile + TL::v_code(r, 2 * t8)) = (uint16_t)w;
        *reinterpret_cast<uint16_t*>(tile + TL::v_code(r, 2 * t8 + 1)) = (uint16_t)(w >> 16);
    } else {
        *reinterpret_cast<uint32_t*>(tile + TL::v_code(r, 2 * t8)) = w.x;
        *reinterpret_cast<uint32_t*>(tile + TL::v_code(r, 2 * t8 + 1)) = w.y;
    }
    if ((t8 & 3) == 0) tile[keys ? TL::k_scale(r, t8 >> 2) : TL::v_scale(r, t8 >> 2)] = (uint8_t)byte;
}
template <int FMT, int DH> __device__ __forceinline__ Codes8<FMT> get(const uint8_t* tile, int r, int t8, bool keys) {
    using TL = Tile<FMT, DH>;
    constexpr int B8 = sizeof(Codes8<FMT>);
    if (keys) return *reinterpret_cast<const Codes8<FMT>*>(tile + r * TL::ROW + t8 * B8);
    if constexpr (DH == 128) return *reinterpret_cast<const Codes8<FMT>*>(tile + TL::v_code(r, t8));
    else if constexpr (FMT == FP4)
        return *reinterpret_cast<const uint16_t*>(tile + TL::v_code(r, 2 * t8)) | (uint32_t)*reinterpret_cast<const uint16_t*>(tile + TL::v_code(r, 2 * t8 + 1)) << 16;
    else return make_uint2(*reinterpret_cast<const uint32_t*>(tile + TL::v_code(r, 2 * t8)), *reinterpret_cast<const uint32_t*>(tile + TL::v_code(r, 2 * t8 + 1)));
}
template <int FMT, int DH> __device__ __forceinline__ void pack8(uint8_t* tile, int r, int t8, bool keys, const float* x) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t a = __float_as_uint(x[i]) & 0x7FFFFFFFu;
        m = a > m ? a : m;
    }
    const uint32_t m1 = quad_swap<1>(m);
    m = m1 > m ? m1 : m;
    const uint32_t m2 = quad_swap<2>(m);
    m = m2 > m ? m2 : m;
    const uint32_t byte = scale_byte<FMT>(m);
    Codes8<FMT> w = encode8(std::integral_constant<int, FMT>{}, x, scale_of(byte));
    if (byte == 255) w = Codes8<FMT>{};
    put<FMT, DH>(tile, r, t8, keys, w, byte);
}
template <int FMT, int DH> __device__ __forceinline__ void unpack8(const uint8_t* tile, int r, int t8, bool keys, float* x) {
    using TL = Tile<FMT, DH>;
    const uint32_t byte = tile[keys ? TL::k_scale(r, t8 >> 2) : TL::v_scale(r, t8 >> 2)];
    decode8(get<FMT, DH>(tile, r, t8, keys), scale_of(byte), x);
    if (byte == 255) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __builtin_nanf("");
    }
}
__device__ __forceinline__ int first_row(const PackedRows& a, int b) {
    if (!a.P_seq) return a.P;
    const int P = a.P_seq[b];
    return P < a.rows - a.L ? P : a.rows - a.L;
}

// Rows of a thread.  us, one / two, rows of 32 heads of 128 in 4 bits: 4 x 4224 packed 77 / 67, read back 61 / 56; float32, 4 x 1024 33.4 / 32.8 and
// 46.6 / 57.4.
constexpr int rows_each(int esz) { return esz == 2 ? 2 : 1; }

template <int FMT, class T, int DH, bool PACK>
__global__ __launch_bounds__(ROWS_THREADS) void k_packed_rows(const RowsArgs a) {
    using TL = Tile<FMT, DH>;
    constexpr int TR = DH / 8, NR = ROWS_THREADS / TR;      // threads of a row, rows at a time
    constexpr int ROWS_EACH = rows_each(sizeof(T));
    const int tid = threadIdx.x, t8 = tid % TR;
    const bool keys = blockIdx.x < a.k_blocks;
    const int id = (int)(blockIdx.x - (keys ? 0 : a.k_blocks));
    uint8_t* const cache = keys ? a.pk : a.pv;
    if (keys || !a.v_across) {
        T* src[ROWS_EACH];
        uint8_t* tile[ROWS_EACH];
        int r[ROWS_EACH];
        bool there[ROWS_EACH];
        float x[ROWS_EACH][8];
#pragma unroll
        for (int y = 0; y < ROWS_EACH; ++y) {
            const int row = (id * ROWS_EACH + y) * NR + tid / TR, bh = a.by_L.of(row), j = row - bh * a.L, b = a.by_nkv.of(bh), h = bh - b * a.nkv;
            const int P = row < a.total ? first_row(a, b) : -1, at = P + j;
            there[y] = P >= 0;
            r[y] = at % PACKED_TILE;
            tile[y] = cache + b * a.batch + h * a.head + (int64_t)(at / PACKED_TILE) * TL::BYTES;
            src[y] = reinterpret_cast<T*>(keys ? a.k : a.v) + (keys ? b * a.k_batch + h * a.k_head + j * a.k_row : b * a.v_batch + h * a.v_head + j * a.v_row) + t8 * 8;
        }
#pragma unroll
        for (int y = 0; y < ROWS_EACH; ++y)
            if (there[y]) {
                if constexpr (PACK) load8(src[y], x[y]);
                else unpack8<FMT, DH>(tile[y], r[y], t8, keys, x[y]);
            }
#pragma unroll
        for (int y = 0; y < ROWS_EACH; ++y)
            if (there[y]) {
                if constexpr (PACK) pack8<FMT, DH>(tile[y], r[y], t8, keys, x[y]);
                else store8(src[y], x[y]);
            }
        return;
    }
    // 64 rows of a (sequence, head), next to each other in memory: 16-byte pieces of E rows of a channel, in LDS at piece ^ (channel / 8), and of
    // two-byte numbers with the upper channels' pairs exchanged, so that neither the pieces nor the eight channels of 16 threads share a bank.
    constexpr int E = 16 / sizeof(T), CH = PACKED_TILE / E, PER = DH * CH / ROWS_THREADS;
    __shared__ __attribute__((aligned(16))) unsigned char lds[DH * PACKED_TILE * sizeof(T)];
    auto piece = [&](int c, int e) { return lds + (sizeof(T) == 2 ? c ^ (c >> 6) : c) * (PACKED_TILE * (int)sizeof(T)) + (e ^ (c >> 3 & (CH - 1))) * 16; };
    auto number = [&](int c, int j) { return reinterpret_cast<T*>(piece(c, j / E)) + j % E; };
    const int bh = a.by_chunks.of(id), j0 = (id - bh * a.chunks) * PACKED_TILE, b = a.by_nkv.of(bh), h = bh - b * a.nkv;
    const int P = first_row(a, b);
    if (P < 0) return;      // the whole workgroup
    const int n = a.L - j0 < PACKED_TILE ? a.L - j0 : PACKED_TILE;
    T* const src = reinterpret_cast<T*>(a.v) + b * a.v_batch + h * a.v_head + j0;
    uint8_t* const head = cache + b * a.batch + h * a.head;
    if constexpr (PACK) {
        Piece x[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = (tid + i * ROWS_THREADS) / CH, e = tid % CH;
            const T* const from = src + c * a.v_chan + e * E;
            if (e * E + E <= n) {
                if (a.v_whole) x[i].v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(from));
                else x[i] = *reinterpret_cast<const Piece*>(from);      // at any alignment of its numbers
            } else {
#pragma unroll
                for (int y = 0; y < E; ++y)
                    if (e * E + y < n) reinterpret_cast<T*>(&x[i])[y] = from[y];
            }
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) *reinterpret_cast<u32x4*>(piece((tid + i * ROWS_THREADS) / CH, tid % CH)) = x[i].v;
        __syncthreads();
    }
    for (int j = tid / TR; j < n; j += NR) {
        const int at = P + j0 + j;
        uint8_t* const tile = head + (int64_t)(at / PACKED_TILE) * TL::BYTES;
        float x[8];
        if constexpr (PACK) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = (float)*number(t8 * 8 + i, j);
            pack8<FMT, DH>(tile, at % PACKED_TILE, t8, false, x);
        } else {
            unpack8<FMT, DH>(tile, at % PACKED_TILE, t8, false, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) *number(t8 * 8 + i, j) = (T)x[i];
        }
    }
    if constexpr (!PACK) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = (tid + i * ROWS_THREADS) / CH, e = tid % CH;
            T* const to = src + c * a.v_chan + e * E;
            Piece x;
            x.v = *reinterpret_cast<const u32x4*>(piece(c, e));
            if (e * E + E <= n) {
                if (a.v_whole) __builtin_nontemporal_store(x.v, reinterpret_cast<u32x4*>(to));
                else *reinterpret_cast<Piece*>(to) = x;
            } else {
#pragma unroll
                for (int y = 0; y < E; ++y)
                    if (e * E + y < n) to[y] = reinterpret_cast<const T*>(&x)[y];
            }
        }
    }
}
template <int FMT, class T, int DH, bool PACK> void run_rows(const PackedRows& p, hipStream_t st) {
    constexpr int NR = ROWS_THREADS / (DH / 8), ROWS_EACH = rows_each(sizeof(T));
    RowsArgs a{};
    static_cast<PackedRows&>(a) = p;
    a.total = p.B * p.nkv * p.L;
    a.chunks = (p.L + PACKED_TILE - 1) / PACKED_TILE;
    a.v_across = p.v_chan != 1;
    constexpr int64_t E = 16 / sizeof(T);
    a.v_whole = ((uintptr_t)p.v & 15) == 0 && p.v_batch % E == 0 && p.v_head % E == 0 && p.v_chan % E == 0;
    a.by_L = Div(p.L); a.by_nkv = Div(p.nkv); a.by_chunks = Div(a.chunks);
    const uint32_t flat = (uint32_t)((a.total + ROWS_EACH * NR - 1) / (ROWS_EACH * NR));
    a.k_blocks = p.k ? flat : 0;
    const uint32_t v_blocks = !p.v ? 0 : a.v_across ? (uint32_t)(p.B * p.nkv * a.chunks) : flat;
    hipLaunchKernelGGL((k_packed_rows<FMT, T, DH, PACK>), dim3(a.k_blocks + v_blocks), dim3(ROWS_THREADS), 0, st, a);
}
template <bool PACK> void rows_launch(const PackedRows& a, hipStream_t st) {
    auto with = [&](auto fmt, auto dh) {
        constexpr int F = decltype(fmt)::value, D = decltype(dh)::value;
        if (a.dtype == 1) run_rows<F, __bf16, D, PACK>(a, st);
        else run_rows<F, float, D, PACK>(a, st);
    };
    auto with_dh = [&](auto fmt) {
        if (a.dh == 128) with(fmt, std::integral_constant<int, 128>{});
        else with(fmt, std::integral_constant<int, 64>{});
    };
    if (a.fmt == FP4) with_dh(std::integral_constant<int, FP4>{});
    else with_dh(std::integral_constant<int, FP8>{});
}

}  // namespace

void launch_pack_rows(const PackedRows& a, hipStream_t st) { rows_launch<true>(a, st); }
void launch_unpack_rows(const PackedRows& a, hipStream_t st) { rows_launch<false>(a, st); }

}  // namespace mulo
