// Attention over the rows of a packed cache.
//
// The running maximum and sum of context_attention.hip: of a tile of keys with scores s (in units of log2), m' = max(m, max s),
// o = o 2^(m - m') + sum 2^(s - m') v, l likewise; out = o / l; partial results join the same way.  A wavefront goes over tiles of 64
// rows with 16 NQ queries, which are rows of all the heads that share a key head.  S^T = K Q^T and O^T = V^T P^T in 16 x 16 blocks: a
// lane (query c = lane % 16, g = lane / 16) has the scores of keys 16 x + 4 g + i, which are the operand that the second product takes
// of it, and channels (4 g + i) u + m of the output, u = d_h / 16.  Nothing of the cache passes through LDS on its way to an instruction
// of the wavefront that loads it: a lane loads the codes that its instructions take, 16 bytes at a time.
//
// bf16: the keys' codes and scales feed the scaled matrix instruction as they lie.  A query enters as two terms of four
// significant bits, q = hi + lo, with a power of two per group of 32 channels each: bf16's eight bits, exactly, but for channels below 2^-13 of
// their group's largest (2^-21 of it).  Heads of 64 have both terms side by side in one instruction.  Against keys made bf16 first the scores
// take no conversions at all: of a tile of 64 rows of heads of 128, 64 of them a lane.  The exponentials are rounded to bf16, at most 2^-8 of
// each, as the weights of context_attention.hip are.
// float32: codes become bf16, exactly, and a query (and an exponential) three bf16 terms, all its 24 bits; the products are exact in float32.
// Values become bf16 with their own scale, two channels of a row an instruction, and pairs of rows are put together by a byte
// permutation: exact, so that only the exponentials' rounding and the sums' are left.
#include <hip/hip_bf16.h>

#include <type_traits>
#include <utility>

#include "index_div.h"
#include "mulo_internal.h"
#include "packed_tile.h"

namespace mulo {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(2))) short i16x2;

template <class F, int... Is>
__device__ __forceinline__ void static_for_impl(F&& f, std::integer_sequence<int, Is...>) {
    (f(std::integral_constant<int, Is>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void static_for(F&& f) {
    static_for_impl(static_cast<F&&>(f), std::make_integer_sequence<int, N>{});
}

constexpr float LAZY_EXP = 8.0f;     // the reference of the exponentials moves once the maximum has outgrown it by 2^8
constexpr float MINUS_INF = -__builtin_huge_valf();
constexpr int NW = 4;                // wavefronts of a workgroup

struct Plan {
    int nq;            // blocks of 16 queries of a wavefront
    int waves;         // k_packed_few: wavefronts of a workgroup; 0: k_packed_block
    int tiles;         // workgroups of the queries of a (sequence, key head)
    int split;         // shares of the keys
};
struct Args : PackedAttn, Plan {
    float* ml;         // [split][B nh L] pairs of maximum and sum, behind the [split][B nh L][dh] outputs in part
    int group, n, shares;      // heads of a key head, queries of a (sequence, key head), workgroups of a share
    int round;
    Div by_nkv, by_L, by_round, by_in_round, by_shares;
};

// two codes times their scale as bf16.  SEL: which pair of the word
template <int FMT, int SEL> __device__ __forceinline__ uint32_t pair(uint32_t w, float s) {
    if constexpr (FMT == FP4) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, SEL));
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, SEL != 0));
}
__device__ __forceinline__ float scale_of(uint32_t word, int i) {      // byte i of the word, as 2^(byte - 127)
    return __uint_as_float(i == 3 ? (word >> 1) & 0x7F800000u : (word << (23 - 8 * i)) & 0x7F800000u);
}
__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ float max_of_groups(float x) {      // over the four lanes of a query
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}

// ---- what a lane holds of a step of 16 NX rows -----------------------------------------------------------------------
constexpr int key_words(int fmt, int esz, int dh) { return esz == 2 ? (fmt == FP8 && dh == 128 ? 8 : 4) : (fmt == FP4 ? dh / 2 : dh) / 16; }
template <int N> __device__ __forceinline__ void load_words(uint32_t* w, const uint8_t* p, int apart) {      // 8 bytes, or 16-byte pieces `apart` bytes apart
    if constexpr (N == 2) {
        const u32x2 x = *reinterpret_cast<const u32x2*>(p);
        w[0] = x.x; w[1] = x.y;
    } else {
#pragma unroll
        for (int e = 0; e < N / 4; ++e) {
            const u32x4 x = *reinterpret_cast<const u32x4*>(p + e * apart);
            w[4 * e] = x.x; w[4 * e + 1] = x.y; w[4 * e + 2] = x.z; w[4 * e + 3] = x.w;
        }
    }
}
// Keys: row 16 x + c of the codes that the lane's quarter of the contraction takes.  bf16: as the scaled instruction has them (of 8 bits,
// 16 g .. and, heads of 128, 64 + 16 g ..; of 4 bits 32 g ..; heads of 64 repeat their channels for the query's second term); float32:
// d_h / 4 channels next to each other.
template <int FMT, class T, int DH, int NX> struct Keys {
    using TL = Tile<FMT, DH>;
    static constexpr bool BF16 = sizeof(T) == 2;
    static constexpr int KW = key_words(FMT, sizeof(T), DH), SUB = 4 / NX;      // words of a row, steps of a tile
    uint32_t w[NX][KW], scale;
    __device__ __forceinline__ void load(const uint8_t* base, int t, int c16, int lg) {
        const uint8_t* const at = base + (int64_t)(t / SUB) * TL::BYTES;
        const int sub = t % SUB;
        const uint32_t off = c16 * TL::ROW + (!BF16 ? lg * (TL::ROW / 4) : FMT == FP4 && DH == 64 ? (lg & 1) * 16 : lg * 16);
#pragma unroll
        for (int x = 0; x < NX; ++x) load_words<KW>(w[x], at + off + (sub * NX + x) * 16 * TL::ROW, BF16 ? 64 : 16);
        const uint32_t s_off = TL::k_scale(0, 0) + (c16 * TL::G + (DH == 128 ? lg : BF16 ? lg & 1 : lg >> 1)) * 4;
        if constexpr (SUB == 1) scale = *reinterpret_cast<const uint32_t*>(at + s_off);
        else scale = *reinterpret_cast<const uint16_t*>(at + s_off + 2 * sub);
    }
};
// Values: of rows 16 x + 4 g .. + 3 the channels c u .. + u - 1 (words r UNIT / 4 .. of row r; UNIT 2: two rows a word), and those rows' scales
template <int FMT, int DH, int NX> struct Values {
    using TL = Tile<FMT, DH>;
    static constexpr int VW = TL::UNIT, SUB = 4 / NX;
    uint32_t w[NX][VW], scale[NX];
    static __device__ __forceinline__ uint32_t offset(int c16, int lg) { return lg * (4 * TL::ROW) + c16 * (4 * TL::UNIT); }
    static __device__ __forceinline__ uint32_t scale_offset(int c16, int lg) { return TL::v_scale(0, 0) + (lg * TL::G + c16 * (DH / 16) / PACKED_GROUP) * 16; }
    __device__ __forceinline__ void load(const uint8_t* base, int t, int c16, int lg) {
        const uint8_t* const at = base + (int64_t)(t / SUB) * TL::BYTES;
        const int sub = t % SUB;
#pragma unroll
        for (int x = 0; x < NX; ++x) load_words<VW>(w[x], at + offset(c16, lg) + (sub * NX + x) * 16 * TL::ROW, 16);
        if constexpr (NX == 4) load_words<4>(scale, at + scale_offset(c16, lg), 16);
        else load_words<2>(scale, at + scale_offset(c16, lg) + 8 * sub, 16);
    }
    __device__ __forceinline__ void load_block(const uint8_t* base, int t, int x, int c16, int lg) {      // NX == 1: block x of tile t
        const uint8_t* const at = base + (int64_t)t * TL::BYTES;
        load_words<VW>(w[0], at + offset(c16, lg) + x * 16 * TL::ROW, 16);
        scale[0] = *reinterpret_cast<const uint32_t*>(at + scale_offset(c16, lg) + 4 * x);
    }
    __device__ __forceinline__ void clear(int x, int r, bool keep) {      // row r of the four becomes zeros
        if constexpr (TL::UNIT == 2) {
            w[x][r >> 1] &= keep ? 0xFFFFFFFFu : (r & 1) ? 0x0000FFFFu : 0xFFFF0000u;
        } else {
#pragma unroll
            for (int e = 0; e < VW / 4; ++e) w[x][r * (VW / 4) + e] = keep ? w[x][r * (VW / 4) + e] : 0u;
        }
        scale[x] = keep ? scale[x] : (scale[x] & ~(0xFFu << (8 * r))) | 0x7Fu << (8 * r);
    }
    // channels 2 PR and 2 PR + 1 of the lane's, of row R of block x
    template <int PR, int R> __device__ __forceinline__ uint32_t two(int x) const {
        const float s = scale_of(scale[x], R);
        if constexpr (FMT == FP4) {
            if constexpr (DH == 128) return pair<FMT, PR>(w[x][R], s);
            else return pair<FMT, 2 * (R & 1) + PR>(w[x][R / 2], s);
        } else {
            if constexpr (DH == 128) return pair<FMT, PR & 1>(w[x][2 * R + PR / 2], s);
            else return pair<FMT, PR>(w[x][R], s);
        }
    }
};
// A query's first term is rounded, and rounded up from the last of float32's numbers it would be 2^128, an infinity: the first term of those is
// the largest there is of its form (15 16 2^120 in four bits, which leaves 15 2^120 of bf16's largest, (2^8 - 1) 2^120 in bf16), and the other
// terms hold the rest as exactly as of all others.
template <class T> __device__ __forceinline__ float within(float x) {
    constexpr float TOP = sizeof(T) == 2 ? 0x1.Ep127f : 0x1.FEp127f;
    return __builtin_amdgcn_fmed3f(x, -TOP, TOP);
}
// 16 queries, one a lane: the terms of its channels
template <class T, int DH> struct Query {
    static constexpr int NC = DH / 32;      // float32: chunks of 8 channels of a lane
    i32x8 hi, lo;                // bf16: the two terms; heads of 64: both in hi
    int scale;                   // bytes 0 and 1: theirs
    bf16x8 term[3][NC];          // float32: three terms
    __device__ __forceinline__ void load(const T* qp, int c16, int lg) {
        if constexpr (sizeof(T) == 2) {
            // a lane's codes are channels 16 g .. + 15, of heads of 128 also 64 + 16 g .. + 15: halves of the groups g / 2 and 2 + g / 2
            constexpr int NP = DH / 64;
            uint32_t most[NP];
            bf16x8 x[NP][2];
#pragma unroll
            for (int y = 0; y < NP; ++y) {
                x[y][0] = *reinterpret_cast<const bf16x8*>(qp + y * 64 + lg * 16);
                x[y][1] = *reinterpret_cast<const bf16x8*>(qp + y * 64 + lg * 16 + 8);
                most[y] = 0;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const uint32_t bits = __float_as_uint((float)x[y][e >> 3][e & 7]) & 0x7FFFFFFFu;
                    most[y] = bits > most[y] ? bits : most[y];
                }
                const uint32_t other = (uint32_t)__shfl_xor((int)most[y], 16);
                most[y] = other > most[y] ? other : most[y];
                // largest / 2^(byte - 127) lies in [128, 256); at least 5, so that the second term's 2^-4 of it is there too
                most[y] = (most[y] >> 23) > 12 ? (most[y] >> 23) - 7 : 5;
            }
            int codes[2][4 * NP];      // of either term
#pragma unroll
            for (int y = 0; y < NP; ++y) {
                const float s_hi = __uint_as_float(most[y] << 23), s_lo = __uint_as_float((most[y] - 4) << 23);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float v[4];
#pragma unroll
                    for (int f = 0; f < 4; ++f) v[f] = (float)x[y][e >> 1][(e & 1) * 4 + f];
                    i16x2 w = {0, 0}, z = {0, 0};
                    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, within<T>(v[0]), within<T>(v[1]), s_hi, false);
                    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, within<T>(v[2]), within<T>(v[3]), s_hi, true);
                    const uint32_t h = __builtin_bit_cast(uint32_t, w);
                    const f32x2 d0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(h, s_hi, false), d1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(h, s_hi, true);
                    z = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(z, v[0] - d0.x, v[1] - d0.y, s_lo, false);
                    z = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(z, v[2] - d1.x, v[3] - d1.y, s_lo, true);
                    codes[0][4 * y + e] = (int)h;
                    codes[1][4 * y + e] = (int)__builtin_bit_cast(uint32_t, z);
                }
            }
            if constexpr (DH == 128) {
#pragma unroll
                for (int e = 0; e < 8; ++e) { hi[e] = codes[0][e]; lo[e] = codes[1][e]; }
                // the instruction takes the scale of group g from the lanes g
                const int s1 = __shfl((int)most[0], c16 + 32), s2 = __shfl((int)most[1], c16);
                const int s = lg == 0 ? (int)most[0] : lg == 1 ? s1 : lg == 2 ? s2 : (int)most[1];
                scale = s | (s - 4) << 8;
            } else {
                // ... which are here those of the two groups' first terms, then of their second ones
#pragma unroll
                for (int e = 0; e < 4; ++e) { hi[e] = codes[0][e]; hi[4 + e] = codes[1][e]; }
                const int s = __shfl((int)most[0], c16 + 32 * (lg & 1));
                scale = lg < 2 ? s : s - 4;
            }
        } else {
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const f32x4 x0 = *reinterpret_cast<const f32x4*>(qp + lg * (DH / 4) + c * 8), x1 = *reinterpret_cast<const f32x4*>(qp + lg * (DH / 4) + c * 8 + 4);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float x = e < 4 ? x0[e & 3] : x1[e & 3];
#pragma unroll
                    for (int y = 0; y < 3; ++y) {
                        term[y][c][e] = (__bf16)(y == 0 ? within<T>(x) : x);
                        x -= (float)term[y][c][e];
                    }
                }
            }
        }
    }
};
// scores of a step: s[x][q][i] of key 16 x + 4 g + i
template <int FMT, class T, int DH, int NX, int NQ>
__device__ __forceinline__ void scores(f32x4 (&s)[NX][NQ], const Keys<FMT, T, DH, NX>& k, const Query<T, DH> (&query)[NQ]) {
    static_for<NX>([&](auto xc) {
        constexpr int x = decltype(xc)::value;
        if constexpr (sizeof(T) == 2) {
            constexpr int KW = Keys<FMT, T, DH, NX>::KW, CODE = FMT == FP4 ? 4 : 0;
            i32x8 kf;
#pragma unroll
            for (int e = 0; e < 8; ++e) kf[e] = (int)k.w[x][e & (KW - 1)];      // (of 4 bits the instruction takes four words)
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
                s[x][q] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kf, query[q].hi, f32x4{0.f, 0.f, 0.f, 0.f}, CODE, 0, x, (int)k.scale, 0, query[q].scale);
                if constexpr (DH == 128) s[x][q] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kf, query[q].lo, s[x][q], CODE, 0, x, (int)k.scale, 1, query[q].scale);
            }
        } else {
            const float sc = scale_of(k.scale, x);
#pragma unroll
            for (int q = 0; q < NQ; ++q) s[x][q] = f32x4{0.f, 0.f, 0.f, 0.f};
            static_for<DH / 32>([&](auto cc) {
                constexpr int c = decltype(cc)::value;
                u32x4 w;
                static_for<4>([&](auto ec) {
                    constexpr int e = decltype(ec)::value;
                    if constexpr (FMT == FP4) w[e] = pair<FMT, e>(k.w[x][c], sc);
                    else w[e] = pair<FMT, e & 1>(k.w[x][2 * c + e / 2], sc);
                });
#pragma unroll
                for (int q = 0; q < NQ; ++q)
#pragma unroll
                    for (int y = 0; y < 3; ++y) s[x][q] = mma(__builtin_bit_cast(bf16x8, w), query[q].term[y][c], s[x][q]);
                __builtin_amdgcn_sched_barrier(0);
            });
        }
    });
}
// The products end here, in front of the loads and the softmax that follow them in the source.  Without this the compiler spreads them
// among those: the same numbers, and 4 x 1024 queries behind 3200 rows take 214 us instead of 203 (the same call over and over).
template <int N, int NQ> __device__ __forceinline__ void stay(f32x4 (&s)[N][NQ]) {
#pragma unroll
    for (int x = 0; x < N; ++x)
#pragma unroll
        for (int q = 0; q < NQ; ++q) asm volatile("" : "+v"(s[x][q]));
}
// key (of a step, as p, before and head are) seen by a query at row p: behind the window's last unseen row, or of the sinks
__device__ __forceinline__ bool sees(int key, int p, int before, int head) { return (key <= p) & ((key > before) | (key < head)); }
// -inf for the keys of a step (first key k0) that a lane's query (at row p) does not see
template <int NX, int NQ> __device__ __forceinline__ void hide(f32x4 (&s)[NX][NQ], const PackedAttn& a, const int (&row)[NQ], int k0, int lg) {
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        const int p = row[q] - k0 - 4 * lg, before = a.window ? p - a.window : -1 - 16 * NX, head = a.sinks - k0 - 4 * lg;
#pragma unroll
        for (int x = 0; x < NX; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[x][q][e] = sees(16 * x + e, p, before, head) ? s[x][q][e] : MINUS_INF;
    }
}
// Moves the reference of the exponentials where some query's maximum has outgrown it, and what has been added up with it
template <int NX, int NQ, int U> __device__ __forceinline__ void refer(const f32x4 (&s)[NX][NQ], float scale_log2, float (&m_run)[NQ], float (&l_run)[NQ], f32x4 (&o)[U][NQ]) {
    float mx[NQ];
    bool up = false;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        mx[q] = s[0][q][0];
#pragma unroll
        for (int x = 0; x < NX; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e) mx[q] = fmaxf(mx[q], s[x][q][e]);
        mx[q] *= scale_log2;
        up |= mx[q] > m_run[q] + LAZY_EXP;
    }
    if (__any(up)) {
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            const float most = max_of_groups(mx[q]), m_new = most > m_run[q] + LAZY_EXP ? most : m_run[q];
            const float alpha = m_new == MINUS_INF ? 1.f : __builtin_amdgcn_exp2f(m_run[q] - m_new);
            m_run[q] = m_new;
            l_run[q] *= alpha;
#pragma unroll
            for (int m = 0; m < U; ++m) o[m][q] *= alpha;
        }
    }
}
// Exponential e of keys 32 half .. + 31 of a lane, as the terms of the second product's operand
template <bool PIN, int NX, int NQ, int NT> __device__ __forceinline__ void exponential(bf16x8 (&pf)[NQ][NT], const f32x4 (&s)[NX][NQ], int half, int e, float scale_log2, const float (&m_run)[NQ], float (&l_run)[NQ]) {
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        const float ref = m_run[q] == MINUS_INF ? 0.f : m_run[q];      // no key seen yet: every exponential is 0
        float x = s[2 * half + (e >> 2)][q][e & 3];
        if (PIN) asm volatile("" : "+v"(x));      // here, among the matrix instructions of its slice
        float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x, scale_log2, -ref));
        l_run[q] += p;
#pragma unroll
        for (int y = 0; y < NT; ++y) {
            pf[q][y][e] = (__bf16)p;
            if (y + 1 < NT) p -= (float)pf[q][y][e];
        }
    }
}
template <int NX, int NQ, int NT> __device__ __forceinline__ void exponentials(bf16x8 (&pf)[NQ][NT], const f32x4 (&s)[NX][NQ], int half, float scale_log2, const float (&m_run)[NQ], float (&l_run)[NQ]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) exponential<false>(pf, s, half, e, scale_log2, m_run, l_run);
}

// ---- where a workgroup is --------------------------------------------------------------------------------------------
struct Place { int split, qt, b, kvh, P; };
// All query tiles of a (sequence, key head) on one XCD, next to each other; long ones first
__device__ __forceinline__ Place place(const Args& a) {
    Place w;
    const int id = blockIdx.x;
    w.split = a.by_shares.of(id);
    const int bid = id - w.split * a.shares, nbh = a.B * a.nkv, by8 = (nbh & 7) == 0, sq = by8 ? bid >> 3 : bid, n_bh = by8 ? nbh >> 3 : nbh;
    const int grp = a.by_round.of(sq), in = sq - grp * (a.round * a.tiles), first = grp * a.round, left = n_bh - first;
    int t, x;
    if (left >= a.round) { t = a.by_in_round.of(in); x = in - t * a.round; } else { t = in / left; x = in - t * left; }
    w.qt = a.tiles - 1 - t;
    const int s_bh = first + x, bh = by8 ? s_bh * 8 + (bid & 7) : s_bh;
    w.b = a.by_nkv.of(bh);
    w.kvh = bh - w.b * a.nkv;
    w.P = a.P;
    if (a.P_seq) {
        const int P = a.P_seq[w.b];
        w.P = P < 0 ? -1 : P < a.rows - a.L ? P : a.rows - a.L;
    }
    return w;
}
// rows of the first and the last of queries r0 .. r0 + n - 1 (within a head they are consecutive)
__device__ __forceinline__ void span(const Args& a, int P, int r0, int n, int& p_min, int& p_max) {
    const int rb = (r0 + n < a.n ? r0 + n : a.n) - 1, ha = a.by_L.of(r0), hb = a.by_L.of(rb);
    p_min = P + (ha == hb ? r0 - ha * a.L : 0);
    p_max = P + (ha == hb ? rb - hb * a.L : a.L - 1);
}
// The steps of ROWS rows that queries at p_min .. p_max see: the head [0, head) of the sinks and from `from` on the window
struct Steps {
    int head, from, begin, end;
    __device__ __forceinline__ int of(int i) const { return i < head ? i : from + i - head; }
};
template <int ROWS> __device__ __forceinline__ Steps steps(const Args& a, int P, int p_min, int p_max) {
    Steps w;
    int lo = 0;
    w.head = 0;
    if (a.window) {
        lo = p_min - a.window + 1 > 0 ? p_min - a.window + 1 : 0;
        w.head = ((a.sinks < lo ? a.sinks : lo) + ROWS - 1) / ROWS;
    }
    w.from = lo / ROWS > w.head ? lo / ROWS : w.head;
    const int more = p_max / ROWS + 1 - w.from;
    w.begin = 0;
    w.end = P < 0 ? 0 : w.head + (more > 0 ? more : 0);
    return w;
}
__device__ __forceinline__ Steps share_of(Steps w, int split, int i) {      // share i of them
    const int n = w.end, per = (n + split - 1) / split;
    w.begin = i * per;
    w.end = w.begin + per < n ? w.begin + per : n;
    return w;
}
// some query at p_min .. p_max does not see some key of k0 .. k0 + n - 1
__device__ __forceinline__ bool cut(const Args& a, int k0, int n, int p_min, int p_max) {
    return k0 + n - 1 > p_min || (a.window && k0 + n > a.sinks && k0 <= p_max - a.window);
}
template <class T> __device__ __forceinline__ void store4(const Args& a, int b, int h, int j, int c, f32x4 w) {      // channels c .. c + 3 of a query
    T* const op = reinterpret_cast<T*>(a.out) + b * a.out_batch + h * a.out_head + j * a.out_row + c;
    if constexpr (sizeof(T) == 2) {
        bf16x4 t;
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] = (__bf16)w[e];
        *reinterpret_cast<bf16x4*>(op) = t;
    } else {
        *reinterpret_cast<f32x4*>(op) = w;
    }
}
// a query's result: 4 channels of it, or of its share, and its share's maximum and sum
struct Result {
    const Args& a;
    int b, h, j, split;
    __device__ __forceinline__ int64_t row() const { return split * ((int64_t)a.B * a.nh * a.L) + ((int64_t)b * a.nh + h) * a.L + j; }
    template <class T, int DH> __device__ __forceinline__ void put(int c, f32x4 w, float inv) const {
        if (a.split > 1) *reinterpret_cast<f32x4*>(a.part + row() * DH + c) = w;
        else store4<T>(a, b, h, j, c, w * inv);
    }
    __device__ __forceinline__ void put_ml(float m, float l) const {
        if (a.split > 1) *reinterpret_cast<float2*>(a.ml + 2 * row()) = make_float2(m, l);
    }
};
// Queries r0 .. r0 + n - 1 see nothing: zeros
template <class T, int DH> __device__ __forceinline__ void zeros(const Args& a, const Place& w, int r0, int n, int tid, int threads) {
    for (int x = tid; x < n * (DH / 4); x += threads) {
        const int r = r0 + x / (DH / 4);
        if (r >= a.n) return;
        const int hg = a.by_L.of(r);
        store4<T>(a, w.b, w.kvh * a.group + hg, r - hg * a.L, x % (DH / 4) * 4, f32x4{0.f, 0.f, 0.f, 0.f});
    }
}
// ... of this share
__device__ __forceinline__ void empty_share(const Args& a, const Place& w, int r0, int n, int tid, int threads) {
    for (int r = r0 + tid; r < r0 + n && r < a.n; r += threads) {
        const int hg = a.by_L.of(r);
        Result{a, w.b, w.kvh * a.group + hg, r - hg * a.L, w.split}.put_ml(MINUS_INF, 0.f);
    }
}

// ---- few queries: the wavefronts of a workgroup have the same ones, and steps in turn; joined in LDS --------------------
// Bound by the cache where there are many sequences (32 of 4224 rows, 32 heads of 128, 4 bits, 588 MB: 104 us, 5.7 TB/s; 16 with a window
// of 2048 rows and 128 sinks in 8 bits, 303 MB of whole tiles: 54 us, 5.6 TB/s), by a wavefront's own chain of a step (1 to 1.5 us: loads,
// scores, maximum, exponentials, products) where there are few: the plan spreads those over wavefronts and shares.  The next step's codes
// are on their way while a step is computed (three wavefronts of a SIMD with 4 bits); a second step on its way gained nothing (28.3 us
// against 29.4, 29.8 against 30.5).
// Against the running maximum of the keys as each step has it, a reference that moves once it is outgrown by 2^8 leaves out the products
// with alpha of nearly every step.
// Blocks of 16 rows that a wavefront goes over at a time: a tile, or half of one where the codes would take more registers than there are
// (8 bits, heads of 128, two blocks of queries).
constexpr int blocks_of_step(int fmt, int esz, int dh, int nq) { return esz == 2 && fmt == FP8 && dh == 128 && nq > 1 ? 2 : 4; }
constexpr int waves_per_simd(int fmt, int esz, int dh, int nq) { return nq == 1 && fmt == FP4 && (esz == 2 || dh == 64) ? 3 : 2; }      // without spills

template <int FMT, class T, int DH, int NQ, int W>
__global__ __launch_bounds__(64 * W, W == 8 ? 2 : waves_per_simd(FMT, sizeof(T), DH, NQ)) void k_packed_few(const Args a) {
    constexpr int U = DH / 16, NT = sizeof(T) == 2 ? 1 : 3;
    constexpr int NX = blocks_of_step(FMT, sizeof(T), DH, NQ), ROWS = 16 * NX;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c16 = lane & 15, lg = lane >> 4;
    const Place w = place(a);
    const int r0 = w.qt * (16 * NQ);
    int p_min, p_max;
    span(a, w.P, r0, 16 * NQ, p_min, p_max);
    const Steps st = share_of(steps<ROWS>(a, w.P, p_min, p_max), a.split, w.split);
    if (st.begin >= st.end) return a.split > 1 ? empty_share(a, w, r0, 16 * NQ, tid, 64 * W) : zeros<T, DH>(a, w, r0, 16 * NQ, tid, 64 * W);

    const uint8_t* const kb = a.k + w.b * a.batch + w.kvh * a.head;
    const uint8_t* const vb = a.v + w.b * a.batch + w.kvh * a.head;
    Keys<FMT, T, DH, NX> keys;
    Values<FMT, DH, NX> values;
    const int i0 = st.begin + wave;
    if (i0 < st.end) {
        keys.load(kb, st.of(i0), c16, lg);
        values.load(vb, st.of(i0), c16, lg);
    }
    Query<T, DH> query[NQ];
    int at[NQ];      // rows of this lane's queries (past the end the last one again: not stored)
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        const int r = r0 + q * 16 + c16, rc = r < a.n ? r : a.n - 1, hg = a.by_L.of(rc), j = rc - hg * a.L;
        at[q] = w.P + j;
        query[q].load(reinterpret_cast<const T*>(a.q) + w.b * a.q_batch + (w.kvh * a.group + hg) * a.q_head + j * a.q_row, c16, lg);
    }
    f32x4 o[U][NQ];
    float m_run[NQ], l_run[NQ];      // l: of this lane's keys
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        m_run[q] = MINUS_INF;
        l_run[q] = 0.f;
#pragma unroll
        for (int m = 0; m < U; ++m) o[m][q] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    for (int i = i0; i < st.end; i += W) {
        const int k0 = st.of(i) * ROWS, t_next = st.of(i + W);
        const bool next = i + W < st.end;
        f32x4 s[NX][NQ];
        scores<FMT, T, DH, NX, NQ>(s, keys, query);
        stay(s);
        if (next) keys.load(kb, t_next, c16, lg);
        if (cut(a, k0, ROWS, p_min, p_max)) {
            hide(s, a, at, k0, lg);
            // Rows that no query of the workgroup sees may hold anything, and 0 * NaN must not reach the sums.
            const int last = p_max - k0 - 4 * lg, first = a.window ? p_min - a.window - k0 - 4 * lg : -1 - ROWS, head = a.sinks - k0 - 4 * lg;
#pragma unroll
            for (int x = 0; x < NX; ++x)
#pragma unroll
                for (int e = 0; e < 4; ++e) values.clear(x, e, sees(16 * x + e, last, first, head));
        }
        refer(s, a.scale_log2, m_run, l_run, o);
        static_for<NX / 2>([&](auto hc) {
            constexpr int half = decltype(hc)::value;
            bf16x8 pf[NQ][NT];
            exponentials(pf, s, half, a.scale_log2, m_run, l_run);
            static_for<U / 2>([&](auto bc) {
                constexpr int pr = decltype(bc)::value;      // channels 2 pr and 2 pr + 1 of the lane's
                u32x4 even, odd;
                static_for<4>([&](auto kc) {
                    constexpr int k2 = decltype(kc)::value, x = 2 * half + k2 / 2, e = 2 * (k2 & 1);      // rows e and e + 1 of block x
                    const uint32_t w0 = values.template two<pr, e>(x), w1 = values.template two<pr, e + 1>(x);
                    even[k2] = __builtin_amdgcn_perm(w1, w0, 0x05040100u);
                    odd[k2] = __builtin_amdgcn_perm(w1, w0, 0x07060302u);
                });
#pragma unroll
                for (int q = 0; q < NQ; ++q)
#pragma unroll
                    for (int y = 0; y < NT; ++y) {
                        o[2 * pr][q] = mma(__builtin_bit_cast(bf16x8, even), pf[q][y], o[2 * pr][q]);
                        o[2 * pr + 1][q] = mma(__builtin_bit_cast(bf16x8, odd), pf[q][y], o[2 * pr + 1][q]);
                    }
                __builtin_amdgcn_sched_barrier(0);
            });
        });
        if (next) values.load(vb, t_next, c16, lg);
    }
    stay(o);
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        l_run[q] += __shfl_xor(l_run[q], 16);
        l_run[q] += __shfl_xor(l_run[q], 32);
    }
    // the wavefronts' results, 16 queries at a time: 16-byte chunk c of row r sits at c ^ r, so that 16 rows' chunks touch every bank once
    __shared__ f32x4 acc[W][16 * (DH / 4)];
    __shared__ float2 stat[W][16];
    for (int q = 0; q < NQ; ++q) {
        if (q) __syncthreads();
#pragma unroll
        for (int y = 0; y < NQ; ++y)
            if (y == q) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int k4 = 0; k4 < U / 4; ++k4)      // channels (4 g + e) u + 4 k4 ..
                        acc[wave][c16 * (DH / 4) + (((4 * lg + e) * (U / 4) + k4) ^ c16)] = f32x4{o[4 * k4][y][e], o[4 * k4 + 1][y][e], o[4 * k4 + 2][y][e], o[4 * k4 + 3][y][e]};
                if (lg == 0) stat[wave][c16] = make_float2(m_run[y], l_run[y]);
            }
        __syncthreads();
        const int row = tid >> 4 & 15, r = r0 + q * 16 + row;
        if (r >= a.n || tid >= 256) continue;
        const int hg = a.by_L.of(r);
        const Result y{a, w.b, w.kvh * a.group + hg, r - hg * a.L, w.split};
        float M = MINUS_INF, f[W], den = 0.f;
#pragma unroll
        for (int x = 0; x < W; ++x) M = fmaxf(M, stat[x][row].x);
#pragma unroll
        for (int x = 0; x < W; ++x) {
            f[x] = stat[x][row].x == MINUS_INF ? 0.f : __builtin_amdgcn_exp2f(stat[x][row].x - M);
            den += f[x] * stat[x][row].y;
        }
        const float inv = den > 0.f ? 1.0f / den : 0.f;
#pragma unroll
        for (int z = 0; z < DH / 64; ++z) {
            const int c4 = (tid & 15) + z * 16;
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int x = 0; x < W; ++x) sum += f[x] * acc[x][row * (DH / 4) + (c4 ^ row)];
            y.put<T, DH>(c4 * 4, sum, inv);
        }
        if ((tid & 15) == 0) y.put_ml(den >= 0.f ? M : den, den);      // a query with NaN or an infinity has no maximum, and its share is not an empty one
    }
}

// ---- many queries: the wavefronts have queries of their own and share a tile's values ------------------------------------
// Every wavefront unpacks a quarter of a tile's values into LDS, where all of them read the second product's operand: with values unpacked by
// every wavefront for itself they were a third of the vector instructions (4 x 1024 queries behind 3200 rows, 32 heads of 128: 278 us in 4
// bits, 388 in 8, against 217 and 268 here).  Two buffers, one barrier a tile.
// Bound by instructions: 249 GFLOP in those 217 us are 1.15 PFLOP/s, a library product in bf16 of 8192^3 reaches 1.21.  Of the cycles the
// matrix instructions are busy for 51 %, the vector ones (exponentials, maxima, unpacking) for 62 %, so that little is left in which
// neither is.  When the kernel took 241 us, unpacking was 32 of them and the barrier 9, eight wavefronts to a tile's values took 254, scores
// of the next tile beside the exponentials 236 to 308 (registers); a third wavefront of a SIMD spills.  float32's three terms take three times
// the products: its blocks stay with k_packed_few.  A query's keys are one workgroup's, so blocks of few workgroups wait for their longest
// (make_plan's comment: 1 x 1024, 4 x 256).
constexpr int BLOCK_NQ = 2;
template <int FMT, int DH>
__global__ __launch_bounds__(64 * NW, 2) void k_packed_block(const Args a) {
    using T = __bf16;
    constexpr int U = DH / 16, NQ = BLOCK_NQ;
    // bf16 operands of either half of a tile: [half][channel of a lane][lane], 8 keys, 4 of each of the half's blocks
    __shared__ u32x2 lds[2][2][U][64][2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c16 = lane & 15, lg = lane >> 4;
    const Place w = place(a);
    const int g0 = w.qt * (NW * 16 * NQ), r0 = g0 + wave * (16 * NQ);
    int g_min, g_max, p_min = 0, p_max = -1;      // of the workgroup, of the wavefront
    span(a, w.P, g0, NW * 16 * NQ, g_min, g_max);
    if (r0 < a.n) span(a, w.P, r0, 16 * NQ, p_min, p_max);
    const Steps st = steps<PACKED_TILE>(a, w.P, g_min, g_max);      // (of a query's keys there is one share)
    if (st.end == 0) return zeros<T, DH>(a, w, g0, NW * 16 * NQ, tid, 64 * NW);

    const uint8_t* const kb = a.k + w.b * a.batch + w.kvh * a.head;
    const uint8_t* const vb = a.v + w.b * a.batch + w.kvh * a.head;
    Keys<FMT, T, DH, 4> keys;
    Values<FMT, DH, 1> values;
    values.load_block(vb, st.of(0), wave, c16, lg);
    keys.load(kb, st.of(0), c16, lg);
    Query<T, DH> query[NQ];
    int at[NQ];
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        const int r = r0 + q * 16 + c16, rc = r < a.n ? r : a.n - 1, hg = a.by_L.of(rc), j = rc - hg * a.L;
        at[q] = w.P + j;
        query[q].load(reinterpret_cast<const T*>(a.q) + w.b * a.q_batch + (w.kvh * a.group + hg) * a.q_head + j * a.q_row, c16, lg);
    }
    auto clear = [&](int i) {      // rows that no query of the workgroup sees may hold anything
        const int k0 = st.of(i) * PACKED_TILE;
        if (cut(a, k0, PACKED_TILE, g_min, g_max)) {
            const int off = k0 + 16 * wave + 4 * lg, last = g_max - off, first = a.window ? g_min - a.window - off : -1 - PACKED_TILE, head = a.sinks - off;
#pragma unroll
            for (int e = 0; e < 4; ++e) values.clear(0, e, sees(e, last, first, head));
        }
    };
    // channels 2 PR and 2 PR + 1 of this wavefront's block of 16 rows, in two steps
    uint32_t two[4];
    auto unpack = [&](auto pc, int i, bool second) {
        constexpr int pr = decltype(pc)::value;
        if (!second) {
#pragma unroll
            for (int x = 0; x < Values<FMT, DH, 1>::VW; ++x) asm volatile("" : "+v"(values.w[0][x]));      // here, not in front of the loop's other steps
            two[0] = values.template two<pr, 0>(0); two[1] = values.template two<pr, 1>(0); two[2] = values.template two<pr, 2>(0); two[3] = values.template two<pr, 3>(0);
        } else {
            u32x2* const to = &lds[i & 1][wave >> 1][2 * pr][lane][wave & 1];
            to[0] = u32x2{__builtin_amdgcn_perm(two[1], two[0], 0x05040100u), __builtin_amdgcn_perm(two[3], two[2], 0x05040100u)};
            to[128] = u32x2{__builtin_amdgcn_perm(two[1], two[0], 0x07060302u), __builtin_amdgcn_perm(two[3], two[2], 0x07060302u)};
        }
    };
    auto unpack_all = [&](int i) {
        static_for<U / 2>([&](auto pc) {
            unpack(pc, i, false);
            unpack(pc, i, true);
        });
    };
    clear(0);
    unpack_all(0);
    if (1 < st.end) values.load_block(vb, st.of(1), wave, c16, lg);
    f32x4 o[U][NQ];
    float m_run[NQ], l_run[NQ];
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        m_run[q] = MINUS_INF;
        l_run[q] = 0.f;
#pragma unroll
        for (int m = 0; m < U; ++m) o[m][q] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    for (int i = 0; i < st.end; ++i) {
        const int k0 = st.of(i) * PACKED_TILE;
        const bool next = i + 1 < st.end;
        // the buffer is full, and everybody has read the other one
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (next) clear(i + 1);
        f32x4 s[4][NQ];
        __builtin_amdgcn_s_setprio(1);
        scores<FMT, T, DH, 4, NQ>(s, keys, query);
        __builtin_amdgcn_s_setprio(0);
        stay(s);
        if (next) keys.load(kb, st.of(i + 1), c16, lg);
        if (r0 < a.n && cut(a, k0, PACKED_TILE, p_min, p_max)) hide(s, a, at, k0, lg);      // (what a wavefront without queries computes is not stored)
        refer(s, a.scale_log2, m_run, l_run, o);
        // The second product, the operand of an instruction requested four channels in front of it; beside the first half's the exponentials
        // of the second, beside the second half's the unpacking of the next tile (behind the last one: the old values once more, which
        // nobody reads).
        constexpr int AHEAD = 2;
        bf16x8 pf[2][NQ][1], vf[AHEAD];
        auto fragment = [&](int half, int m) { return *reinterpret_cast<const bf16x8*>(&lds[i & 1][half][m][lane][0]); };
#pragma unroll
        for (int x = 0; x < AHEAD; ++x) vf[x] = fragment(0, x);
        exponentials(pf[0], s, 0, a.scale_log2, m_run, l_run);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
        static_for<2 * U>([&](auto mc) {
            constexpr int half = decltype(mc)::value / U, m = decltype(mc)::value % U;
            const bf16x8 v = vf[m % AHEAD];
            if constexpr (half == 0 || m + AHEAD < U) vf[m % AHEAD] = m + AHEAD < U ? fragment(half, m + AHEAD) : fragment(1, m + AHEAD - U);
#pragma unroll
            for (int q = 0; q < NQ; ++q) o[m][q] = mma(v, pf[half][q][0], o[m][q]);
            if constexpr (half == 0) {
#pragma unroll
                for (int e = m * 8 / U; e < (m + 1) * 8 / U; ++e) exponential<true>(pf[1], s, 1, e, a.scale_log2, m_run, l_run);
            } else {
                unpack(std::integral_constant<int, m / 2>{}, i + 1, m & 1);
            }
            __builtin_amdgcn_sched_barrier(0);
        });
        __builtin_amdgcn_s_setprio(0);
        if (i + 2 < st.end) values.load_block(vb, st.of(i + 2), wave, c16, lg);
    }
    stay(o);
    int first = r0;
    asm volatile("" : "+s"(first));      // heads and rows of the queries once more: kept over the loop they would take registers
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        l_run[q] += __shfl_xor(l_run[q], 16);
        l_run[q] += __shfl_xor(l_run[q], 32);
        const int r = first + q * 16 + c16, hg = a.by_L.of(r);
        if (r >= a.n) continue;
        const float inv = l_run[q] > 0.f ? 1.0f / l_run[q] : 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int k4 = 0; k4 < U / 4; ++k4) store4<T>(a, w.b, w.kvh * a.group + hg, r - hg * a.L, (4 * lg + e) * U + 4 * k4, inv * f32x4{o[4 * k4][q][e], o[4 * k4 + 1][q][e], o[4 * k4 + 2][q][e], o[4 * k4 + 3][q][e]});
    }
}

int clamp_int(int64_t v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : (int)v; }

// What a call costs in microseconds, fitted to the times in make_plan's comment: a round of workgroups has START; a wavefront's step of
// 64 rows takes LATENCY by itself, and a SIMD gets through one in WORK; the cache comes in at READ bytes a microsecond, into a CU at INTO_CU;
// JOIN, and JOIN_SHARE and their bytes a share, when there are shares.
struct Cost { double start, latency, work; };
constexpr double READ = 5.9e6, INTO_CU = 45e3, JOIN = 4.5, JOIN_SHARE = 0.08, JOIN_BYTES = 5e6;
Cost cost_few(int esz, int dh, int nq) {
    if (esz == 4) return dh == 128 ? Cost{4.5, 2.0, 1.6} : nq == 1 ? Cost{4.5, 1.3, 0.93} : Cost{5.5, 2.2, 1.8};
    return nq == 1 ? (dh == 128 ? Cost{4.5, 1.05, 0.55} : Cost{4.5, 0.8, 0.35}) : (dh == 128 ? Cost{5.5, 1.5, 0.98} : Cost{5.5, 1.1, 0.62});
}
// 64-row tiles that a workgroup with `rows` queries of a (sequence, key head) sees at most, and on average
void tiles_seen(const PackedAttn& a, int64_t n, int64_t rows, double& most, double& mean) {
    const double last = a.P + a.L, first = a.P, span = n < rows ? a.L : rows < a.L ? rows : a.L;      // rows of its queries
    most = last;
    mean = (first + last + span) / 2;
    if (a.window) {
        const double w = (double)a.window + span + (a.sinks ? a.sinks + 32.0 : 0.0);
        most = w < most ? w : most;
        mean = w < mean ? w : mean;
    }
    most = most / PACKED_TILE + (a.window ? 1 : 0.5);
    mean = mean / PACKED_TILE + (a.window ? 1 : 0.5);
}

// Four or eight wavefronts of k_packed_few with 16 queries, four with 32, shares of the keys, or k_packed_block: the one with the least time
// by the estimate.  Measured, in us (bf16, 32 heads of 128, 4 bits where nothing else is said; "4/1" four wavefronts with 16 queries, "x 8" in
// shares; * what the estimate takes):
//   1 x 1 query, 500 rows             4/1 6.4     8/1 7.2 *   4/1 x 2 8.8
//   1 x 1, 4000                       4/1 22      8/1 17.6    4/1 x 8 11.5     8/1 x 8 12.1 *
//   4 x 1, 4000                       4/1 27      8/1 20.4 *  4/1 x 4 19.8
//   12 x 1, 4000                      4/1 41 *    8/1 45      8/1 x 2 47
//   32 x 1, 4223                      4/1 104 *   8/1 101
//   2 x 1, 60000, 8 key heads         8/1 x 16 31 *           4/1 x 37 36
//   16 x 1, 4000, 16 heads of 64      4/1 22.4    8/1 17.1 *
//   16 x 16, 4000, 8 key heads        4/1 32 *    4/2 34.5    8/1 36.5
//   4 x 256, 3000                     4/1 79      4/2 68 *    block 80
//   4 x 256, 832, 16 heads of 64, 8 bits          4/2 13.5 *  block 22.5
//   16 x 64, 0                        4/1 17.6    4/2 18.1    block 11.5 *
//   1 x 1024, 0                       4/2 28 *    block 28
//   4 x 1024, 3200                    4/2 278     block 217 * (8 bits 388, 268 *)
//   8 x 1024, 0                       4/2 188     block 101 *
//   8 x 1024, 0, 16 heads of 64       4/2 52      block 35 *
//   float32, 6 x 5, 800, 16 heads of 64, 8 bits   4/1 9.6     8/1 9.0 *; 4 x 256   4/1 22.3   4/2 20.1 *
// It takes the slower side of four of these rows, by 3 to 12 %.  Over 46 other calls, spread over all sizes, it was 4 % behind the best of up
// to 22 plans in the mean, more than 10 % behind for five of them, 38 % at most (four single float32 queries over 2000 rows: 8/1 11.7, 4/1 x 8
// 8.5): eight wavefronts have the START of four, and float32's shares look dearer than they are.
// part_floats: the scratch there is (packed_attention_floats asks with as much as can be wanted)
Plan make_plan(const PackedAttn& a, int64_t part_floats) {
    const int64_t n = (int64_t)(a.nh / a.nkv) * a.L, pairs = (int64_t)a.B * a.nkv, slot_floats = (int64_t)a.B * a.nh * a.L * (a.dh + 2);
    const int slots = clamp_int(part_floats / slot_floats, 1, MAX_SHARES), esz = a.dtype == 1 ? 2 : 4, cus = cu_count();
    const double tile_bytes = 2.0 * packed_tile_bytes(a.fmt, a.dh);
    Plan best{};
    double best_time = 0;
    auto offer = [&](const Plan& p, double time) {
        if (best.nq && time >= best_time) return;
        best = p;
        best_time = time;
    };
    double most, mean;
    for (int nq = 1; nq <= 2; ++nq) {
        if (nq == 2 && (n <= 16 || (esz == 4 && a.dh == 128))) break;
        const Cost c = cost_few(esz, a.dh, nq);
        const int64_t tiles = (n + 16 * nq - 1) / (16 * nq), base = pairs * tiles;
        tiles_seen(a, n, 16 * nq, most, mean);
        const double bytes = pairs * most * tile_bytes;
        for (int waves = NW; waves <= (nq == 1 ? 2 * NW : NW); waves += NW) {
            const int places = cus * (waves > NW ? 1 : esz == 2 && nq == 1 && a.fmt == FP4 ? 3 : 2);
            auto with = [&](int split) {
                if (split > slots || (split > 1 && split * waves > most + waves)) return;
                const int64_t rounds = (base * split + places - 1) / places;
                const int steps = (int)(most / (split * waves)) + 1;
                const double alone = rounds * steps * c.latency, work = base * split * (mean / split) / (4.0 * cus) * c.work, most_of = alone > work ? alone : work;
                const double into_cu = rounds * (most / split) * tile_bytes / INTO_CU, read = bytes / READ > into_cu ? bytes / READ : into_cu;
                offer({nq, waves, (int)tiles, split}, rounds * c.start + sqrt(most_of * most_of + read * read) + (split > 1 ? JOIN + split * (JOIN_SHARE + slot_floats * 8.0 / JOIN_BYTES) : 0.0));
            };
            for (int split = 1; split <= slots; split += 1 + split / 4) with(split);
            for (int64_t full = 1; full <= 2; ++full)      // as many as fill the chip once and twice
                if (full * places / base > 1) with(clamp_int(full * places / base, 1, MAX_SHARES));
        }
    }
    if (esz == 2) {
        // a tile's time in a workgroup that has its CU to itself, that shares it with another one, with two others (heads of 64); a round's START
        // again; the last round is as long as its longest
        const double alone[3] = {a.dh == 128 ? 1.5 : 1.0, a.dh == 128 ? 2.0 : 1.25, 1.7}, codes = a.fmt == FP8 && a.dh == 128 ? 1.15 : 1.0, start = 6.0;
        const int per_cu = a.dh == 128 ? 2 : 3;
        const int64_t rows = 16 * BLOCK_NQ * NW, tiles = (n + rows - 1) / rows, wgs = pairs * tiles, places = (int64_t)per_cu * cus, rounds = (wgs + places - 1) / places;
        const int64_t beside = (wgs - (rounds - 1) * places + cus - 1) / cus;
        tiles_seen(a, n, rows, most, mean);
        offer({BLOCK_NQ, 0, (int)tiles, 1}, rounds * start + codes * ((rounds - 1) * mean * alone[per_cu - 1] + (rounds > 1 ? mean : most) * alone[beside - 1]));
    }
    return best;
}

template <int FMT, class T, int DH, int NQ, int W>
void run_cfg(Args a, hipStream_t st) {
    a.group = a.nh / a.nkv;
    a.n = a.group * a.L;
    a.shares = a.tiles * a.nkv * a.B;
    a.by_nkv = Div(a.nkv); a.by_L = Div(a.L); a.round = a.tiles < 64 ? 64 / a.tiles : 1; a.by_round = Div(a.round * a.tiles); a.by_in_round = Div(a.round); a.by_shares = Div(a.shares);
    a.ml = a.part ? a.part + (int64_t)a.split * a.B * a.nh * a.L * DH : nullptr;
    if constexpr (W == 0) hipLaunchKernelGGL((k_packed_block<FMT, DH>), dim3((unsigned)((int64_t)a.shares * a.split)), dim3(64 * NW), 0, st, a);
    else hipLaunchKernelGGL((k_packed_few<FMT, T, DH, NQ, W>), dim3((unsigned)((int64_t)a.shares * a.split)), dim3(64 * W), 0, st, a);
}
template <int FMT, class T, int DH>
void run(const PackedAttn& c, hipStream_t st) {
    Args a{};
    static_cast<PackedAttn&>(a) = c;
    static_cast<Plan&>(a) = make_plan(a, c.part ? c.part_floats : 0);
    if (a.waves > NW) {
        run_cfg<FMT, T, DH, 1, 2 * NW>(a, st);
    } else if (a.nq == 1) {
        run_cfg<FMT, T, DH, 1, NW>(a, st);
    } else if constexpr (sizeof(T) == 2) {
        if (a.waves) run_cfg<FMT, T, DH, 2, NW>(a, st);
        else run_cfg<FMT, T, DH, 2, 0>(a, st);
    } else if constexpr (DH == 64) {
        run_cfg<FMT, T, DH, 2, NW>(a, st);
    }
    if (a.split > 1) {
        ContextAttn j{};
        j.dtype = c.dtype; j.B = c.B; j.L = c.L; j.nh = c.nh; j.nkv = c.nkv; j.dh = c.dh;
        j.out = c.out; j.out_batch = c.out_batch; j.out_head = c.out_head; j.out_row = c.out_row;
        j.P_seq = c.P_seq; j.part = c.part;
        launch_join_shares(j, a.split, st);
    }
}

// Windows that reach over all rows are none, so that positions and windows add up within 32 bits.
PackedAttn within_rows(PackedAttn a) {
    if (a.window >= a.rows) a.window = 0;
    if (a.sinks > a.rows) a.sinks = a.rows;
    return a;
}

}  // namespace

size_t packed_attention_floats(const PackedAttn& c) {
    const PackedAttn a = within_rows(c);
    const int64_t slot_floats = (int64_t)a.B * a.nh * a.L * (a.dh + 2);
    const Plan p = make_plan(a, MAX_SHARES * slot_floats);
    return p.split > 1 ? (size_t)(p.split * slot_floats) : 0;
}

void launch_packed_attention(const PackedAttn& c, hipStream_t st) {
    const PackedAttn a = within_rows(c);
    auto with = [&](auto fmt, auto dh) {
        constexpr int F = decltype(fmt)::value, D = decltype(dh)::value;
        if (a.dtype == 1) run<F, __bf16, D>(a, st);
        else run<F, float, D>(a, st);
    };
    auto with_dh = [&](auto fmt) {
        if (a.dh == 128) with(fmt, std::integral_constant<int, 128>{});
        else with(fmt, std::integral_constant<int, 64>{});
    };
    if (a.fmt == FP4) with_dh(std::integral_constant<int, FP4>{});
    else with_dh(std::integral_constant<int, FP8>{});
}

}  // namespace mulo
