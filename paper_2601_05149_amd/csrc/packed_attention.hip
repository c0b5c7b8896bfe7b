// Attention over the rows of a packed cache.
//
// The running maximum and sum of context_attention.hip: of a tile of keys with scores s (in units of log2), m' = max(m, max s),
// o = o 2^(m - m') + sum 2^(s - m') v, l likewise; out = o / l; partial results join the same way.  A wavefront goes over tiles of 64
// rows with 16 NQ queries, which are rows of all the heads that share a key head.  S^T = K Q^T and O^T = V^T P^T in 16 x 16 blocks: a
// lane (query c = lane % 16, g = lane / 16) has the scores of keys 16 x + 4 g + i, which are the operand that the second product takes
// of it, and channels (4 g + i) u + m of the output, u = d_h / 16.  Nothing of the cache passes through LDS: a lane loads the codes that
// its instructions take.
//
// bf16: the keys' codes and scales feed the scaled matrix instruction as they lie.  A query enters as two terms of four
// significant bits, q = hi + lo, with a power of two per group of 32 channels each: bf16's eight bits, exactly, but for channels below 2^-13 of
// their group's largest (2^-21 of it).  Heads of 64 have both terms side by side in one instruction.  float32: codes become
// bf16, exactly, and a query (and an exponential) three bf16 terms.
// Values become bf16 with their own scale, two channels of a row an instruction, and pairs of rows are put together by a byte
// permutation.
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
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
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
    bool shared;       // the wavefronts of a workgroup have the same queries, and tiles of keys in turn; else queries of their own
    int tiles;         // workgroups of the queries of a (sequence, key head)
    int split;         // shares of the keys
};
struct Args : PackedAttn, Plan {
    float* ml;         // [split][B nh L] pairs of maximum and sum, behind the [split][B nh L][dh] outputs in part
    int group, n, shares;      // heads of a key head, queries of a (sequence, key head), workgroups of a share
    Div by_nkv, by_L, by_tiles, by_shares;
};

// 16 codes bytes a lane feeds the instruction; two codes at once as bf16.  SEL: which pair of the word
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

constexpr int waves_per_simd(int fmt, int esz, int dh, int nq) { return esz == 4 && dh == 128 ? (nq == 1 ? 2 : 1) : nq == 1 && fmt == FP4 ? 3 : 2; }

// Blocks of 16 rows that a wavefront goes over at a time: a tile, or half of one where the codes would take more registers than there are.
constexpr int blocks_of_step(int fmt, int esz, int dh, int nq) { return esz == 2 && fmt == FP8 && dh == 128 && nq > 1 ? 2 : 4; }

template <int FMT, class T, int DH, int NQ, bool SHARED>
__global__ __launch_bounds__(64 * NW, waves_per_simd(FMT, sizeof(T), DH, NQ)) void k_packed_attention(const Args a) {
    using TL = Tile<FMT, DH>;
    constexpr bool BF16 = sizeof(T) == 2;
    constexpr int U = DH / 16;                        // channels of the output that a lane's rows of O^T step over, instructions of the second product
    constexpr int VW = TL::UNIT;                      // words of four rows' values of a lane: 4 UNIT bytes
    constexpr int KW = BF16 ? (FMT == FP8 && DH == 128 ? 8 : 4) : TL::ROW / 16;      // words of a key's codes of a lane
    constexpr int NC = DH / 32;                       // float32: chunks of 8 channels of a lane
    constexpr int NX = blocks_of_step(FMT, sizeof(T), DH, NQ), ROWS = 16 * NX;      // blocks of 16 rows, rows of a step
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c16 = lane & 15, lg = lane >> 4;

    // ---- which queries, which share of which keys.  All query tiles of a (sequence, key head) on one XCD, next to each other; long ones first
    const int id = blockIdx.x, split = a.by_shares.of(id), bid = id - split * a.shares;
    const int nbh = a.B * a.nkv, by8 = (nbh & 7) == 0, sq = by8 ? bid >> 3 : bid, s_bh = a.by_tiles.of(sq);
    const int qt = a.tiles - 1 - (sq - s_bh * a.tiles), bh = by8 ? s_bh * 8 + (bid & 7) : s_bh;
    const int b = a.by_nkv.of(bh), kvh = bh - b * a.nkv;
    const int r0 = (SHARED ? qt : qt * NW + wave) * (16 * NQ), n = a.n;
    if (!SHARED && r0 >= n) return;
    int P = a.P;
    if (a.P_seq) {
        P = a.P_seq[b];
        P = P < a.rows - a.L ? P : a.rows - a.L;
    }
    int row_h[NQ], row_j[NQ];      // of this lane's queries (past the end the last one again: not stored)
    bool live[NQ];
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        const int r = r0 + q * 16 + c16, rc = r < n ? r : n - 1, h = a.by_L.of(rc);
        live[q] = r < n;
        row_h[q] = kvh * a.group + h;
        row_j[q] = rc - h * a.L;
    }
    const int64_t all_rows = (int64_t)a.B * a.nh * a.L;
    const bool partial = a.split > 1;
    auto out_row = [&](int h, int j) { return ((int64_t)b * a.nh + h) * a.L + j; };
    auto store4 = [&](int h, int j, int c, f32x4 w) {      // channels c .. c + 3 of a query
        T* const op = reinterpret_cast<T*>(a.out) + b * a.out_batch + h * a.out_head + j * a.out_row + c;
        if constexpr (BF16) {
            bf16x4 t;
#pragma unroll
            for (int e = 0; e < 4; ++e) t[e] = (__bf16)w[e];
            *reinterpret_cast<bf16x4*>(op) = t;
        } else {
            *reinterpret_cast<f32x4*>(op) = w;
        }
    };

    // ---- which steps: the head [0, n1) of the sinks and from t2 on the window
    int p_min, p_max;
    {
        const int rb = (r0 + 16 * NQ < n ? r0 + 16 * NQ : n) - 1, ha = a.by_L.of(r0), hb = a.by_L.of(rb);      // within a head the queries are consecutive
        p_min = P + (ha == hb ? r0 - ha * a.L : 0);
        p_max = P + (ha == hb ? rb - hb * a.L : a.L - 1);
    }
    int lo = 0, n1 = 0;
    if (a.window) {
        lo = p_min - a.window + 1 > 0 ? p_min - a.window + 1 : 0;
        n1 = ((a.sinks < lo ? a.sinks : lo) + ROWS - 1) / ROWS;
    }
    const int t2 = lo / ROWS > n1 ? lo / ROWS : n1, more = p_max / ROWS + 1 - t2;
    const int n_steps = P < 0 ? 0 : n1 + (more > 0 ? more : 0);
    const int per = (n_steps + a.split - 1) / a.split, t_begin = split * per, t_end = t_begin + per < n_steps ? t_begin + per : n_steps;
    if (t_begin >= t_end) {      // the whole workgroup (SHARED) or wavefront: nothing to see
        if (!SHARED || wave == 0) {
#pragma unroll
            for (int q = 0; q < NQ; ++q)
                if (live[q]) {
                    if (partial) {
                        if (lg == 0) *reinterpret_cast<float2*>(a.ml + 2 * (split * all_rows + out_row(row_h[q], row_j[q]))) = make_float2(MINUS_INF, 0.f);
                    } else {
#pragma unroll
                        for (int c = 0; c < DH / 4; c += 4) store4(row_h[q], row_j[q], lg * (DH / 4) + c, f32x4{0.f, 0.f, 0.f, 0.f});
                    }
                }
        }
        return;
    }
    auto step_of = [&](int i) { return i < n1 ? i : t2 + i - n1; };

    // ---- loads of a step
    const uint8_t* const kb = a.k + b * a.batch + kvh * a.head;
    const uint8_t* const vb = a.v + b * a.batch + kvh * a.head;
    const uint32_t k_off = c16 * TL::ROW + (!BF16 ? lg * (TL::ROW / 4) : FMT == FP4 && DH == 64 ? (lg & 1) * 16 : lg * 16);
    const uint32_t ks_off = TL::k_scale(0, 0) + (c16 * TL::G + (DH == 128 ? lg : BF16 ? lg & 1 : lg >> 1)) * 4;
    const uint32_t v_off = lg * (4 * TL::ROW) + c16 * (4 * TL::UNIT);
    const uint32_t vs_off = TL::v_scale(0, 0) + (lg * TL::G + c16 * U / PACKED_GROUP) * 16;
    uint32_t kw[NX][KW], vw[NX][VW], ks, vs[NX];
    constexpr int SUB = 4 / NX;      // steps of a tile
    auto load_k = [&](int t) {
        const uint8_t* const at = kb + (int64_t)(t / SUB) * TL::BYTES;
        const int sub = t % SUB;
#pragma unroll
        for (int x = 0; x < NX; ++x) {
            const uint8_t* const p = at + k_off + (sub * NX + x) * 16 * TL::ROW;
            if constexpr (KW == 2) {
                const u32x2 w = *reinterpret_cast<const u32x2*>(p);
                kw[x][0] = w.x; kw[x][1] = w.y;
            } else {
#pragma unroll
                for (int e = 0; e < KW / 4; ++e) {
                    const u32x4 w = *reinterpret_cast<const u32x4*>(p + e * (BF16 ? 64 : 16));
                    kw[x][4 * e] = w.x; kw[x][4 * e + 1] = w.y; kw[x][4 * e + 2] = w.z; kw[x][4 * e + 3] = w.w;
                }
            }
        }
        if constexpr (SUB == 1) ks = *reinterpret_cast<const uint32_t*>(at + ks_off);
        else ks = *reinterpret_cast<const uint16_t*>(at + ks_off + 2 * sub);
    };
    auto load_v = [&](int t) {
        const uint8_t* const at = vb + (int64_t)(t / SUB) * TL::BYTES;
        const int sub = t % SUB;
#pragma unroll
        for (int x = 0; x < NX; ++x) {
            const uint8_t* const p = at + v_off + (sub * NX + x) * 16 * TL::ROW;
            if constexpr (VW == 2) {
                const u32x2 w = *reinterpret_cast<const u32x2*>(p);
                vw[x][0] = w.x; vw[x][1] = w.y;
            } else {
#pragma unroll
                for (int e = 0; e < VW / 4; ++e) {
                    const u32x4 w = *reinterpret_cast<const u32x4*>(p + e * 16);
                    vw[x][4 * e] = w.x; vw[x][4 * e + 1] = w.y; vw[x][4 * e + 2] = w.z; vw[x][4 * e + 3] = w.w;
                }
            }
        }
        if constexpr (NX == 4) {
            const u32x4 w = *reinterpret_cast<const u32x4*>(at + vs_off);
            vs[0] = w.x; vs[1] = w.y; vs[2] = w.z; vs[3] = w.w;
        } else {
            const u32x2 w = *reinterpret_cast<const u32x2*>(at + vs_off + 8 * sub);
            vs[0] = w.x; vs[1] = w.y;
        }
    };
    const int step = SHARED ? NW : 1, i0 = t_begin + (SHARED ? wave : 0);
    if (i0 < t_end) {
        load_k(step_of(i0));
        load_v(step_of(i0));
    }

    // ---- the queries
    i32x8 qh[NQ], ql[NQ];         // bf16: the two terms; heads of 64: both in qh
    int qs[NQ];                   // their scales, bytes 0 and 1
    bf16x8 q3[NQ][3][NC];         // float32: three terms
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        const T* const qp = reinterpret_cast<const T*>(a.q) + b * a.q_batch + row_h[q] * a.q_head + row_j[q] * a.q_row;
        if constexpr (BF16) {
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
                    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, v[0], v[1], s_hi, false);
                    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, v[2], v[3], s_hi, true);
                    const uint32_t hi = __builtin_bit_cast(uint32_t, w);
                    const f32x2 d0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hi, s_hi, false), d1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hi, s_hi, true);
                    z = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(z, v[0] - d0.x, v[1] - d0.y, s_lo, false);
                    z = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(z, v[2] - d1.x, v[3] - d1.y, s_lo, true);
                    codes[0][4 * y + e] = (int)hi;
                    codes[1][4 * y + e] = (int)__builtin_bit_cast(uint32_t, z);
                }
            }
            if constexpr (DH == 128) {
#pragma unroll
                for (int e = 0; e < 8; ++e) { qh[q][e] = codes[0][e]; ql[q][e] = codes[1][e]; }
                // the instruction takes the scale of group g from the lanes g
                const int s1 = __shfl((int)most[0], c16 + 32), s2 = __shfl((int)most[1], c16);
                const int s = lg == 0 ? (int)most[0] : lg == 1 ? s1 : lg == 2 ? s2 : (int)most[1];
                qs[q] = s | (s - 4) << 8;
            } else {
                // ... which are here those of the two groups' first terms, then of their second ones
#pragma unroll
                for (int e = 0; e < 4; ++e) { qh[q][e] = codes[0][e]; qh[q][4 + e] = codes[1][e]; }
                const int s = __shfl((int)most[0], c16 + 32 * (lg & 1));
                qs[q] = lg < 2 ? s : s - 4;
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
                        q3[q][y][c][e] = (__bf16)x;
                        x -= (float)q3[q][y][c][e];
                    }
                }
            }
        }
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

    for (int i = i0; i < t_end; i += step) {
        const int t = step_of(i), k0 = t * ROWS;
        const bool next = i + step < t_end;
        const int t_next = step_of(i + step);
        // ---- scores
        f32x4 s[NX][NQ];
        static_for<NX>([&](auto xc) {
            constexpr int x = decltype(xc)::value;
            if constexpr (BF16) {
                i32x8 kf;
#pragma unroll
                for (int e = 0; e < 8; ++e) kf[e] = (int)kw[x][FMT == FP4 ? e & 3 : DH == 64 ? e & 3 : e & (KW - 1)];
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    s[x][q] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kf, qh[q], f32x4{0.f, 0.f, 0.f, 0.f}, FMT == FP4 ? 4 : 0, 0, x, (int)ks, 0, qs[q]);
                    if constexpr (DH == 128)
                        s[x][q] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kf, ql[q], s[x][q], FMT == FP4 ? 4 : 0, 0, x, (int)ks, 1, qs[q]);
                }
            } else {
                const float sc = scale_of(ks, x);
#pragma unroll
                for (int q = 0; q < NQ; ++q) s[x][q] = f32x4{0.f, 0.f, 0.f, 0.f};
                static_for<NC>([&](auto cc) {
                    constexpr int c = decltype(cc)::value;
                    u32x4 w;
                    static_for<4>([&](auto ec) {
                        constexpr int e = decltype(ec)::value;
                        if constexpr (FMT == FP4) w[e] = pair<FMT, e>(kw[x][c], sc);
                        else w[e] = pair<FMT, e & 1>(kw[x][2 * c + e / 2], sc);
                    });
                    const bf16x8 kf = __builtin_bit_cast(bf16x8, w);
#pragma unroll
                    for (int q = 0; q < NQ; ++q)
#pragma unroll
                        for (int y = 0; y < 3; ++y) s[x][q] = mma(kf, q3[q][y][c], s[x][q]);
                    __builtin_amdgcn_sched_barrier(0);
                });
            }
            __builtin_amdgcn_sched_barrier(0);
        });
        // The compiler may move these instructions to where their results are used, also behind a branch that not all lanes take;
        // all lanes' operands are needed.
#pragma unroll
        for (int x = 0; x < NX; ++x)
#pragma unroll
            for (int q = 0; q < NQ; ++q) asm volatile("" : "+v"(s[x][q]));
        if (next) load_k(t_next);
        // ---- rows that some query does not see
        const bool cut = k0 + ROWS - 1 > p_min || (a.window && k0 + ROWS > a.sinks && k0 <= p_max - a.window);
        if (cut) {
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
                const int p = P + row_j[q] - k0 - 4 * lg, before = a.window ? p - a.window : -1 - ROWS, head = a.sinks - k0 - 4 * lg;
#pragma unroll
                for (int x = 0; x < NX; ++x)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = 16 * x + e;
                        s[x][q][e] = (key <= p) & ((key > before) | (key < head)) ? s[x][q][e] : MINUS_INF;
                    }
            }
            // Rows that no query of the wavefront sees may hold anything, and 0 * NaN must not reach the sums: their codes become zeros.
            const int last = p_max - k0, first = a.window ? p_min - a.window - k0 : -1 - ROWS, head = a.sinks - k0;
#pragma unroll
            for (int x = 0; x < NX; ++x)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int key = 16 * x + 4 * lg + e;
                    const bool seen = (key <= last) & ((key > first) | (key < head));
                    if constexpr (TL::UNIT == 2) {
                        vw[x][e >> 1] &= seen ? 0xFFFFFFFFu : (e & 1) ? 0x0000FFFFu : 0xFFFF0000u;
                    } else {
#pragma unroll
                        for (int w = 0; w < VW / 4; ++w) vw[x][e * (VW / 4) + w] = seen ? vw[x][e * (VW / 4) + w] : 0u;
                    }
                    vs[x] = seen ? vs[x] : (vs[x] & ~(0xFFu << (8 * e))) | 0x7Fu << (8 * e);
                }
        }
        // ---- the reference of the exponentials
        float mx[NQ];
        bool up = false;
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            mx[q] = s[0][q][0];
#pragma unroll
            for (int x = 0; x < NX; ++x)
#pragma unroll
                for (int e = 0; e < 4; ++e) mx[q] = fmaxf(mx[q], s[x][q][e]);
            mx[q] *= a.scale_log2;
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
        // ---- exponentials and the second product, 32 keys at a time
        static_for<NX / 2>([&](auto hc) {
            constexpr int half = decltype(hc)::value;
            constexpr int NT = BF16 ? 1 : 3;
            bf16x8 pf[NQ][NT];
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
                const float ref = m_run[q] == MINUS_INF ? 0.f : m_run[q];      // no key seen yet: every exponential is 0
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * half + (e >> 2)][q][e & 3], a.scale_log2, -ref));
                    l_run[q] += p;
#pragma unroll
                    for (int y = 0; y < NT; ++y) {
                        pf[q][y][e] = (__bf16)p;
                        if (y + 1 < NT) p -= (float)pf[q][y][e];
                    }
                }
            }
            static_for<U / 2>([&](auto bc) {
                constexpr int pr = decltype(bc)::value;      // channels 2 pr and 2 pr + 1 of the lane's
                u32x4 even, odd;
                static_for<4>([&](auto kc) {
                    constexpr int k2 = decltype(kc)::value, x = 2 * half + k2 / 2, e = 2 * (k2 & 1);      // rows e and e + 1 of block x
                    auto value = [&](auto rc) {
                        constexpr int r = decltype(rc)::value;
                        const float sc = scale_of(vs[x], r);
                        if constexpr (FMT == FP4) {
                            if constexpr (DH == 128) return pair<FMT, pr>(vw[x][r], sc);
                            else return pair<FMT, 2 * (r & 1) + pr>(vw[x][r / 2], sc);
                        } else {
                            if constexpr (DH == 128) return pair<FMT, pr & 1>(vw[x][2 * r + pr / 2], sc);
                            else return pair<FMT, pr>(vw[x][r], sc);
                        }
                    };
                    const uint32_t w0 = value(std::integral_constant<int, e>{}), w1 = value(std::integral_constant<int, e + 1>{});
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
        if (next) load_v(t_next);
    }
#pragma unroll
    for (int m = 0; m < U; ++m)
#pragma unroll
        for (int q = 0; q < NQ; ++q) asm volatile("" : "+v"(o[m][q]));

#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        l_run[q] += __shfl_xor(l_run[q], 16);
        l_run[q] += __shfl_xor(l_run[q], 32);
    }
    auto mine = [&](int q, int e, int k4) { return f32x4{o[4 * k4][q][e], o[4 * k4 + 1][q][e], o[4 * k4 + 2][q][e], o[4 * k4 + 3][q][e]}; };      // channels (4 g + e) U + 4 k4 ..
    auto leave = [&](int h, int j, int c, f32x4 w, float inv) {
        if (partial) *reinterpret_cast<f32x4*>(a.part + (split * all_rows + out_row(h, j)) * DH + c) = w;
        else store4(h, j, c, w * inv);
    };
    if constexpr (!SHARED) {
        int first = r0;
        asm volatile("" : "+s"(first));      // heads and rows of the queries once more: kept over the loop they would take registers
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            const int r = first + q * 16 + c16, hg = a.by_L.of(r), h = kvh * a.group + hg, j = r - hg * a.L;
            if (r >= n) continue;
            const float inv = l_run[q] > 0.f ? 1.0f / l_run[q] : 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int k4 = 0; k4 < U / 4; ++k4) leave(h, j, (4 * lg + e) * U + 4 * k4, mine(q, e, k4), inv);
            if (partial && lg == 0) *reinterpret_cast<float2*>(a.ml + 2 * (split * all_rows + out_row(h, j))) = make_float2(m_run[q], l_run[q]);
        }
    } else {
        // the wavefronts' results, 16 queries at a time: 16-byte chunk c of row r sits at c ^ r, so that 16 rows' chunks touch every bank once
        __shared__ f32x4 acc[NW][16 * (DH / 4)];
        __shared__ float2 stat[NW][16];
        for (int q = 0; q < NQ; ++q) {
            if (q) __syncthreads();
#pragma unroll
            for (int y = 0; y < NQ; ++y)
                if (y == q) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int k4 = 0; k4 < U / 4; ++k4) acc[wave][c16 * (DH / 4) + ((((4 * lg + e) * U) / 4 + k4) ^ c16)] = mine(y, e, k4);
                    if (lg == 0) stat[wave][c16] = make_float2(m_run[y], l_run[y]);
                }
            __syncthreads();
            const int row = tid >> 4, r = r0 + q * 16 + row;
            if (r < n) {
                const int hg = a.by_L.of(r), h = kvh * a.group + hg, j = r - hg * a.L;
                float M = MINUS_INF, f[NW], den = 0.f;
#pragma unroll
                for (int w = 0; w < NW; ++w) M = fmaxf(M, stat[w][row].x);
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    f[w] = stat[w][row].x == MINUS_INF ? 0.f : __builtin_amdgcn_exp2f(stat[w][row].x - M);
                    den += f[w] * stat[w][row].y;
                }
                const float inv = den > 0.f ? 1.0f / den : 0.f;
#pragma unroll
                for (int x = 0; x < DH / 64; ++x) {
                    const int c4 = (tid & 15) + x * 16;
                    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int w = 0; w < NW; ++w) sum += f[w] * acc[w][row * (DH / 4) + (c4 ^ row)];
                    leave(h, j, c4 * 4, sum, inv);
                }
                if (partial && (tid & 15) == 0) *reinterpret_cast<float2*>(a.ml + 2 * (split * all_rows + out_row(h, j))) = make_float2(M, den);
            }
        }
    }
}

int clamp_int(int64_t v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : (int)v; }

// part_floats: the scratch there is (packed_attention_floats asks with as much as can be wanted)
Plan make_plan(const PackedAttn& a, int64_t part_floats) {
    Plan p{};
    const int64_t n = (int64_t)(a.nh / a.nkv) * a.L, slot_floats = (int64_t)a.B * a.nh * a.L * (a.dh + 2);
    const int slots = clamp_int(part_floats / slot_floats, 0, MAX_SHARES);
    p.shared = n <= 32;
    p.nq = n <= 16 ? 1 : 2;
    const int rows = 16 * p.nq * (p.shared ? 1 : NW);
    p.tiles = (int)((n + rows - 1) / rows);
    // tiles of keys that a workgroup sees at most
    const int64_t end = (int64_t)a.P + a.L;
    int64_t seen = (end + PACKED_TILE - 1) / PACKED_TILE;
    if (a.window) {
        const int64_t w = ((int64_t)a.window + (p.shared || n < rows ? a.L : rows) + PACKED_TILE - 1) / PACKED_TILE + 1 + ((int64_t)a.sinks + PACKED_TILE - 1) / PACKED_TILE;
        seen = w < seen ? w : seen;
    }
    const int64_t base = (int64_t)a.B * a.nkv * p.tiles, places = 3 * cu_count();
    p.split = clamp_int(places / base, 1, clamp_int(seen / (p.shared ? 8 : 4), 1, slots > 1 ? slots : 1));
    return p;
}

template <int FMT, class T, int DH, int NQ, bool SHARED>
void run_cfg(Args a, hipStream_t st) {
    a.group = a.nh / a.nkv;
    a.n = a.group * a.L;
    a.shares = a.tiles * a.nkv * a.B;
    a.by_nkv = Div(a.nkv); a.by_L = Div(a.L); a.by_tiles = Div(a.tiles); a.by_shares = Div(a.shares);
    a.ml = a.part ? a.part + (int64_t)a.split * a.B * a.nh * a.L * DH : nullptr;
    hipLaunchKernelGGL((k_packed_attention<FMT, T, DH, NQ, SHARED>), dim3((unsigned)((int64_t)a.shares * a.split)), dim3(64 * NW), 0, st, a);
}
template <int FMT, class T, int DH>
void run(const PackedAttn& c, hipStream_t st) {
    Args a{};
    static_cast<PackedAttn&>(a) = c;
    static_cast<Plan&>(a) = make_plan(a, c.part ? c.part_floats : 0);
    if (!a.shared) run_cfg<FMT, T, DH, 2, false>(a, st);
    else if (a.nq == 2) run_cfg<FMT, T, DH, 2, true>(a, st);
    else run_cfg<FMT, T, DH, 1, true>(a, st);
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
