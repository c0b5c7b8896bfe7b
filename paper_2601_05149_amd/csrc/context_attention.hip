// Attention over a prefix that the sequences of a group share and the rows that each sequence has of its own, with an
// optional window and sinks: the query at position p sees t <= p with t < sinks or p - t < window.
//
// One pass over the keys with a running maximum m and sum l per query: of a tile of keys with scores s (in units of
// log2), m' = max(m, max s), o = o 2^(m - m') + sum 2^(s - m') v, l = l 2^(m - m') + sum 2^(s - m'); out = o / l.  Partial
// results (o, m, l) over disjoint sets of keys join as sum o_i 2^(m_i - M) / sum l_i 2^(m_i - M), M = max m_i.
//
// A wavefront owns 32 queries and computes S^T = K Q^T and O^T = V^T P^T with 32x32 matrix instructions, so that a
// lane owns ONE query: the reductions of the softmax stay inside the lane (and its twin 32 lanes on), and the exponentials
// are already laid out as the second operand of the second product.  Tiles of K and V^T go from memory to LDS directly,
// double buffered, and are shared by the wavefronts of a workgroup.
//
// What a workgroup's queries are (make_plan chooses, with both sides measured):
//   few     32 queries over few keys, all wavefronts with the same queries and tiles of keys of their own, joined in LDS: one launch
//   stacked few queries per sequence behind a shared prefix: the rows of all sequences of a group go over the prefix
//           together (prefix workgroups), each sequence's over its own rows (own workgroups, the same launch), and
//           k_context_join joins the partial results.  The prefix is read once per 128 stacked rows.
//   whole   128 or 256 queries of one sequence; its tiles are those of its prefix that it sees, then its own.  Keys of few
//           queries are dealt to several workgroups, whose shares k_context_join joins.
//
// bf16: the exponentials are rounded for the second product, whose matrix instruction takes bf16 (half a step of 2^-8 each, of either
// sign, of positive terms; their sum l is taken of what was not rounded); scores, m, l, o and every partial result are float32.
//
// What bounds it, heads of 128, 32 of them, on a card that reads 6.2 TB/s, copies 5.05 and multiplies 8192^3 bf16 at 1.25 PFLOP/s:
//   single tokens over thousands of rows: memory.  64 tokens, two prefixes of 2048 rows and 900 own rows 199 us, 5.1 TB/s; 32 through a
//   window of 2048 with 128 sinks 196 us, 5.8 TB/s
//   long blocks: the matrix instruction and the softmax's vector instructions one after the other at a clock that falls under the load
//   (4 x 1024 queries, 1024 shared and 2048 own rows 247 to 256 us, 940 to 975 TFLOP/s, matrix pipes busy 45 %; through a window of
//   1024 with 128 sinks 106 to 113 us, 700 TFLOP/s, 38 %: a query sees nine tiles' worth of keys, a wavefront computes ten and its
//   workgroup goes through eleven, and each of the two rounds has a prologue and an epilogue that nothing overlaps)
//   16 x 16 queries, 330 own and 4224 shared rows 52.6 us, 364 TFLOP/s: 42 in k_context, where the own rows' workgroups have one
//   wavefront of four at work, and 21 MB of partial results each way
//   everything smaller: launches and one chain of latencies (a tile some 1.2 us; one launch 5 to 9 us, two 9 to 14)
#include <hip/hip_bf16.h>

#include <utility>

#include "index_div.h"
#include "mulo_internal.h"

namespace mulo {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void glb_void;

template <class F, int... Is>
__device__ __forceinline__ void static_for_impl(F&& f, std::integer_sequence<int, Is...>) {
    (f(std::integral_constant<int, Is>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void static_for(F&& f) {
    static_for_impl(static_cast<F&&>(f), std::make_integer_sequence<int, N>{});
}

// 16 bytes of an operand per lane: 8 bf16 feed one 32x32x16 instruction, 4 float32 four 32x32x2 ones (which of the
// contraction's indexes a lane's elements are is the same for both operands, so it does not matter)
template <class T> struct Chunk;
template <> struct Chunk<__bf16> {
    typedef bf16x8 type;
    static __device__ __forceinline__ f32x16 mma(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Chunk<float> {
    typedef f32x4 type;
    static __device__ __forceinline__ f32x16 mma(f32x4 a, f32x4 b, f32x16 c) {
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x, b.x, c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.y, b.y, c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.z, b.z, c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_32x32x2f32(a.w, b.w, c, 0, 0, 0);
    }
};

constexpr float LAZY_EXP = 8.0f;     // the reference of the exponentials moves once the maximum has outgrown it by 2^8 (see attention.hip)
constexpr int MAX_SLOTS = MAX_SHARES;      // shares of a query that k_context_join joins: a lane each

// How a launch is laid out (host).
struct Plan {
    bool few;          // a workgroup per 32 queries, wavefronts with tiles of keys of their own
    bool stacked;      // prefix and own workgroups
    bool by_kv;        // the queries of a workgroup are those of all heads of a key head (else of one head)
    int heads;         // heads, or key heads
    int n;             // queries of a (sequence, head)
    int tiles;         // of them: workgroups
    int prefix_tiles;  // stacked: tiles of the stacked rows of a (group, key head)
    int split;         // shares of the keys (stacked: of the own rows)
    int prefix_split;  // stacked: shares of the prefix
    int prefix_wgs;    // workgroups of the prefix (the first ones of the grid)
};
struct Args : ContextAttn, Plan {
    float* ml;         // [slots][B nh L] pairs: maximum and sum, behind the [slots][B nh L][dh] outputs in part
    int group, in_group, shares;      // heads of a key head, sequences of a prefix, workgroups of a share of the keys (not of the prefix)
    Div by_group, by_in_group, by_L, by_n, by_heads, by_tiles, by_shares, by_gk, by_nkv, by_prefix_tiles;
};

// FEW (few keys): every wavefront has all of the workgroup's 32 queries and tiles of keys of its own, in a buffer of its own, so that
// nobody waits for anybody in front of the end, where the wavefronts' results are joined in LDS.  (Otherwise one of four
// wavefronts works and a second launch joins.)
template <class T, int DH, int BQ, int BKV, int NTH, bool FEW>
__global__ __launch_bounds__(NTH, !FEW && DH * BKV * (int)sizeof(T) <= 16384 ? 2 : 1) void k_context(const Args a) {
    typedef typename Chunk<T>::type chunk;
    constexpr bool BF16 = sizeof(T) == 2;
    constexpr int E = 16 / sizeof(T);      // elements of a chunk
    constexpr int NKK = DH / (2 * E);      // pairs of chunks along a row of K
    constexpr int NDB = DH / 32;           // 32-row blocks of O^T
    constexpr int NKB = BKV / 32;          // 32-key blocks of S^T
    constexpr int NKS = BKV / (2 * E);     // pairs of chunks along a row of V^T
    constexpr int NW = NTH / 64;
    constexpr int KRB = DH * sizeof(T), VRB = BKV * sizeof(T);            // bytes of a row of the K tile, of the V^T tile
    constexpr int KT = BKV * KRB, BUF = KT + DH * VRB;
    constexpr int TW = FEW ? 1 : NW;                                      // wavefronts that share a tile
    constexpr int LK = KT / 1024 / TW, LV = DH * VRB / 1024 / TW;         // loads of a wavefront per tile, a KB of whole rows each
    constexpr int RK = 1024 / KRB, RV = 1024 / VRB;                       // rows of a load
    static_assert(LK * TW * 1024 == KT && LV * TW * 1024 == DH * VRB, "whole loads per wavefront");
    static_assert(!FEW || BQ == 32, "the queries of a wavefront");

    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];  // [2][BUF]; FEW: [NW][BUF]

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, lh = lane >> 5;
    const int tw = FEW ? 0 : wave;      // among those that share a tile
    // A line of arguments that is not in the scalar cache is a microsecond's way off: one of each is asked for here, together, not
    // one after the other where they are used.
    asm volatile("" ::"s"(a.dtype), "s"(a.k), "s"(a.rows), "s"(a.G), "s"(a.window), "s"(a.n), "s"(a.group), "s"(a.by_L.m), "s"(a.by_heads.m), "s"(a.by_gk.m), "s"(a.by_prefix_tiles.m));
    const int group = a.group, in_group = a.in_group;
    // ---- which queries, which share of which keys
    const bool stacked = !FEW && a.stacked, of_prefix = stacked && (int)blockIdx.x < a.prefix_wgs;
    int b = 0, hd, qt, split, nsplit, slot, n, g;
    if (of_prefix) {      // consecutive ids: consecutive (group, head)s, one XCD each; the row tiles of one lie on one XCD
        const int gk = a.G * a.nkv, bid = blockIdx.x;
        const int rest = a.by_gk.of(bid), in = bid - rest * gk;
        g = a.by_nkv.of(in); hd = in - g * a.nkv;
        split = slot = a.by_prefix_tiles.of(rest);
        qt = rest - split * a.prefix_tiles;
        nsplit = a.prefix_split;
        n = in_group * a.n;
    } else {              // all query tiles of a (sequence, head) on one XCD, next to each other; long tiles first
        const int nbh = a.B * a.heads, id = (int)blockIdx.x - (stacked ? a.prefix_wgs : 0);
        split = FEW ? 0 : a.by_shares.of(id);
        const int bid = id - split * a.shares, by8 = (nbh & 7) == 0, s = by8 ? bid >> 3 : bid, s_bh = a.by_tiles.of(s);
        qt = a.tiles - 1 - (s - s_bh * a.tiles);
        const int bh = by8 ? s_bh * 8 + (bid & 7) : s_bh;
        b = a.by_heads.of(bh);
        hd = bh - b * a.heads;
        g = a.by_in_group.of(b);
        slot = split + (stacked ? a.prefix_split : 0);
        nsplit = FEW ? 1 : a.split;
        n = a.n;
    }
    const int kvh = a.by_kv ? hd : a.by_group.of(hd);
    const bool scattered = !FEW && a.pos_tab != nullptr;
    // ---- this lane's query (the last one again past the end; such lanes do not store)
    const int r0 = qt * BQ + tw * 32, r_raw = r0 + l32, r = r_raw < n ? r_raw : n - 1;
    const int r_seq = of_prefix ? a.by_n.of(r) : 0, lb = of_prefix ? g * in_group + r_seq : b, in_seq = r - r_seq * a.n;
    const int r_hd = a.by_kv ? a.by_L.of(in_seq) : 0, lhd = a.by_kv ? hd * group + r_hd : hd, lj = in_seq - r_hd * a.L;
    const bool wave_live = r0 < n;
    int P = a.P;
    if (a.P_seq && !of_prefix) {
        P = a.P_seq[b];
        P = P < a.rows - a.L ? P : a.rows - a.L;
    }
    const bool absent = !of_prefix && P < 0;     // uniform over the workgroup
    int pos = P + lj;                            // own row; of the prefix's workgroups only with a window (then P is everyone's)
    bool active = true;
    if (scattered) {
        const int row = a.pos_tab[(int64_t)lb * a.L + lj];
        active = row >= 0;
        pos = active ? row : a.P0;
    }
    // own rows of the queries: of this wavefront, of the workgroup (bounds)
    auto first_last = [&](int ra, int rb, int& lo, int& hi) {
        rb = rb < n ? rb : n - 1;
        const int ha = a.by_kv ? a.by_L.of(ra) : 0, hb = a.by_kv ? a.by_L.of(rb) : 0;      // within a head the queries are consecutive
        lo = P + (ha == hb ? ra - ha * a.L : 0);
        hi = P + (ha == hb ? rb - hb * a.L : a.L - 1);
        if (scattered) { lo = a.P0; hi = a.P0 + a.Lblk - 1; }
    };
    int w_min, w_max, p_min, p_max;
    first_last(r0, r0 + 31, w_min, w_max);
    first_last(qt * BQ, qt * BQ + BQ - 1, p_min, p_max);

    // ---- which tiles: of either source the head [0, a) of the sinks and [lo, end) of the window
    const int S = a.S, window = a.window;
    int pre_a = 0, pre_lo = 0, own_a = 0, own_lo = 0, np1 = 0, np = 0, tp2 = 0, no1 = 0, no = 0, to2 = 0;
    const int own_end = p_max + 1;
    if (S > 0 && (of_prefix || !stacked)) {
        if (window) {
            const int lo = S + p_min - window + 1;       // S + p_min < 2^25
            pre_lo = lo < 0 ? 0 : lo < S ? lo : S;
            pre_a = a.sinks < pre_lo ? a.sinks : pre_lo;
        }
        np1 = (pre_a + BKV - 1) / BKV;
        tp2 = pre_lo / BKV > np1 ? pre_lo / BKV : np1;
        const int more = pre_lo < S ? (S + BKV - 1) / BKV - tp2 : 0;
        np = np1 + (more > 0 ? more : 0);
    }
    if (!of_prefix) {
        if (window) {
            const int lo = p_min - window + 1, s = a.sinks - S;
            own_lo = lo < 0 ? 0 : lo;
            own_a = s < 0 ? 0 : s < own_lo ? s : own_lo;
        }
        no1 = (own_a + BKV - 1) / BKV;
        to2 = own_lo / BKV > no1 ? own_lo / BKV : no1;
        const int more = (own_end + BKV - 1) / BKV - to2;
        no = no1 + (more > 0 ? more : 0);
    }
    const int n_tiles = absent ? 0 : np + no;
    const int per = (n_tiles + nsplit - 1) / nsplit;
    const int t_begin = split * per, t_end = t_begin + per < n_tiles ? t_begin + per : n_tiles;
    const int64_t all_rows = (int64_t)a.B * a.nh * a.L;
    const bool partial = !FEW && (stacked || a.split > 1);
    const int64_t out_row = ((int64_t)lb * a.nh + lhd) * a.L + lj;
    auto store4 = [&](int b, int h, int j, int c, f32x4 w) {       // channels c .. c + 3, 4 | c, of a query
        T* const op = reinterpret_cast<T*>(a.out) + (a.frag ? frag_index(b * a.L + j, h * DH + c, a.nh * DH)      // inside a run of 8
                                                            : b * a.out_batch + h * a.out_head + j * a.out_row + c);
        if constexpr (BF16) {
            bf16x4 t;
#pragma unroll
            for (int e = 0; e < 4; ++e) t[e] = (__bf16)w[e];
            *reinterpret_cast<bf16x4*>(op) = t;
        } else {
            *reinterpret_cast<f32x4*>(op) = w;
        }
    };
    auto store_out = [&](int i, int g4, f32x4 w) { store4(lb, lhd, lj, i * 32 + g4 * 8 + lh * 4, w); };      // of this lane's query
    if (t_begin >= t_end) {    // uniform over the workgroup, before any barrier: nothing to see
        if (r_raw < n && (!FEW || wave == 0)) {
            if (partial) {
                if (lh == 0) *reinterpret_cast<float2*>(a.ml + 2 * (slot * all_rows + out_row)) = make_float2(-__builtin_huge_valf(), 0.f);
            } else {
#pragma unroll
                for (int i = 0; i < NDB; ++i)
#pragma unroll
                    for (int g4 = 0; g4 < 4; ++g4) store_out(i, g4, f32x4{0.f, 0.f, 0.f, 0.f});
            }
        }
        return;
    }

    chunk qf[NKK];
    {
        const T* qp = reinterpret_cast<const T*>(a.q) + lb * a.q_batch + lhd * a.q_head + lj * a.q_row + lh * E;
#pragma unroll
        for (int kk = 0; kk < NKK; ++kk) qf[kk] = *reinterpret_cast<const chunk*>(qp + kk * 2 * E);
    }

    // Tiles go from memory to LDS directly.  16-byte chunk c of row r sits at chunk position c ^ key(r): 16 lanes that read
    // the same chunk of 16 rows touch every bank once.
    auto key_of = [](int r, int row_bytes) { return row_bytes >= 256 ? r & 15 : row_bytes == 128 ? (r >> 1) & 7 : (r >> 2) & 3; };
    const int krow = tw * RK + lane / (64 / RK), vrow = tw * RV + lane / (64 / RV);
    // this lane's chunk of a row of V^T in load x: the same in all where the rows of a load repeat the key, else one in the even and one in the odd
    constexpr int VKEYS = TW * RV % 16 == 0 ? 1 : 2;
    static_assert(VKEYS * TW * RV % 16 == 0, "the keys of a lane's rows of V^T");
    int vchunk[VKEYS];
#pragma unroll
    for (int y = 0; y < VKEYS; ++y) vchunk[y] = lane % (64 / RV) ^ key_of(vrow + y * TW * RV, VRB);
    const unsigned char* const pk = reinterpret_cast<const unsigned char*>(reinterpret_cast<const T*>(a.pk) + g * a.pk_group + kvh * a.pk_head);
    const unsigned char* const pv = reinterpret_cast<const unsigned char*>(reinterpret_cast<const T*>(a.pv) + g * a.pv_group + kvh * a.pv_head + (int64_t)tw * RV * a.pv_chan);
    const unsigned char* const ok = reinterpret_cast<const unsigned char*>(reinterpret_cast<const T*>(a.k) + b * a.k_batch + kvh * a.k_head);
    const unsigned char* const ov = reinterpret_cast<const unsigned char*>(reinterpret_cast<const T*>(a.v) + b * a.v_batch + kvh * a.v_head + (int64_t)tw * RV * a.v_chan);
    auto to_lds = [](const unsigned char* base, uint32_t off, unsigned char* lds) {
        __builtin_amdgcn_global_load_lds((glb_void*)(base + off), (lds_void*)lds, 16, 0, 0);
    };
    auto tile_of = [&](int i) { return i < np ? (i < np1 ? i : tp2 + i - np1) : (i - np < no1 ? i - np : to2 + (i - np) - no1); };
    // A tile that runs past the end of its cache takes the last row and columns again: nothing sees those keys.
    auto buffer = [&](int i) { return smem + (FEW ? wave : i & 1) * BUF; };
    auto load = [&](int i, bool of_k, bool of_v) {
        const bool pre = i < np;
        const int t = tile_of(i);
        unsigned char* const lds = buffer(i) + tw * 1024;
        const int left = (pre ? a.srows : a.rows) - t * BKV;
        if (of_k) {
            const uint32_t k_row = (uint32_t)(pre ? a.pk_row : a.k_row) * sizeof(T);
            const unsigned char* const kt = (pre ? pk : ok) + (int64_t)t * BKV * k_row;
#pragma unroll
            for (int x = 0; x < LK; ++x) {
                const int row = krow + x * TW * RK;
                to_lds(kt, (uint32_t)(row < left ? row : left - 1) * k_row + ((lane % (64 / RK)) ^ key_of(row, KRB)) * 16, lds + x * TW * 1024);
            }
        }
        if (of_v) {
            const int64_t v_chan = (pre ? a.pv_chan : a.v_chan) * (int64_t)sizeof(T);
            const unsigned char* const vt = (pre ? pv : ov) + (int64_t)t * VRB;
#pragma unroll
            for (int y = 0; y < VKEYS; ++y) {
                const int c = vchunk[y] * E;
                const uint32_t vo = (uint32_t)(lane / (64 / RV)) * (uint32_t)v_chan + (uint32_t)(c < left - E ? c : left - E) * (uint32_t)sizeof(T);
#pragma unroll
                for (int x = y; x < LV; x += VKEYS) to_lds(vt + x * (TW * RV) * v_chan, vo, lds + KT + x * TW * 1024);
            }
        }
    };
    auto load_kv = [&](int i) { load(i, true, true); };
    auto meet = [&]() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
    // Columns of V^T that no query of the workgroup sees may hold anything: their probabilities are 0, and 0 * NaN must not reach
    // the accumulators.  Between the landing of a tile and the barrier that shows it to the others, every lane clears
    // those of the bytes it has loaded itself.
    auto clear_unseen = [&](int i) {
        const bool pre = i < np;
        const int k0 = tile_of(i) * BKV, end = pre ? S : own_end, lo = pre ? pre_lo : own_lo, head = pre ? pre_a : own_a;
        if (k0 + BKV > end || (k0 < lo && k0 + BKV > head)) {
            if (!FEW) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // FEW: the caller has waited
#pragma unroll
            for (int y = 0; y < VKEYS; ++y) {
                const int key = k0 + vchunk[y] * E;
                auto seen = [&](int e) { return key + e < end && (key + e < head || key + e >= lo); };
                auto keep = [&](int w) -> uint32_t {
                    if constexpr (BF16) return (seen(2 * w) ? 0xFFFFu : 0u) | (seen(2 * w + 1) ? 0xFFFF0000u : 0u);
                    else return seen(w) ? 0xFFFFFFFFu : 0u;
                };
                const u32x4 mask = {keep(0), keep(1), keep(2), keep(3)};
#pragma unroll
                for (int x = y; x < LV; x += VKEYS) {
                    u32x4* const at = reinterpret_cast<u32x4*>(buffer(i) + KT + (x * TW + tw) * 1024 + lane * 16);
                    *at = *at & mask;
                }
            }
        }
    };

    f32x16 o[NDB];
#pragma unroll
    for (int i = 0; i < NDB; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
    float m_run = -__builtin_huge_valf(), l_run = 0.f;

    // bf16: row rho of a K block is fed key rho with bits 2 and 3 swapped, so that a lane's accumulators cover 8 consecutive keys
    const int kperm = BF16 ? (l32 & 0x13) | ((l32 & 4) << 1) | ((l32 & 8) >> 1) : l32;
    // accumulator e of block kb holds key key_at(kb, e) + lane_key of the tile.  (Kept apart: the sums are the same in every
    // tile, and 64 registers would hold them.)
    auto key_at = [](int kb, int e) { return BF16 ? kb * 32 + 16 * (e >> 3) + (e & 7) : kb * 32 + 8 * (e >> 2) + (e & 3); };
    const int lane_key = (BF16 ? 8 : 4) * lh;
    const int kfrag = kperm * KRB + (lh ^ key_of(kperm, KRB)) * 16, vfrag = l32 * VRB + (lh ^ key_of(l32, VRB)) * 16;
    f32x16 s[NKB];               // the scores of a tile, then
    float m_safe = 0.f, alpha = 1.f;   // the reference of its exponentials and the factor of what has been added up before it
    auto score = [&](int i) {
        const bool pre = i < np;
        const int kv0 = tile_of(i) * BKV;
        const unsigned char* const kt = buffer(i);
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[kb][e] = 0.f;
        // NKB independent chains, the fragments of a step requested during the step before it
        chunk kf[2][NKB];
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb) kf[0][kb] = *reinterpret_cast<const chunk*>(kt + kfrag + kb * 32 * KRB);
        static_for<NKK>([&](auto kc) {
            constexpr int kk = decltype(kc)::value;
            static_for<NKB>([&](auto bc) {
                constexpr int kb = decltype(bc)::value;
                if constexpr (kk + 1 < NKK) kf[(kk + 1) & 1][kb] = *reinterpret_cast<const chunk*>(kt + (kfrag ^ ((kk + 1) << 5)) + kb * 32 * KRB);
                s[kb] = Chunk<T>::mma(kf[kk & 1][kb], qf[kk], s[kb]);
                __builtin_amdgcn_sched_barrier(0);
            });
        });
        // at most 4 comparisons at once: more than that need more scalars than there are
        auto mask = [&](auto&& seen) {
#pragma unroll
            for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    s[kb][e] = seen(key_at(kb, e)) ? s[kb][e] : -__builtin_huge_valf();
                    if ((e & 3) == 3) __builtin_amdgcn_sched_barrier(0);
                }
        };
        const int last = pre ? S - 1 : w_min;                            // key up to which all queries of the wavefront see
        if (kv0 + BKV - 1 > last) {
            const int lim = (pre ? S - 1 : pos) - kv0 - lane_key;
            mask([&](int key) { return key <= lim; });
        }
        if (window) {
            const int shift = (pre ? S : 0) - window, sinks = a.sinks - (pre ? 0 : S);
            if (kv0 + BKV > sinks && kv0 <= w_max + shift) {             // some key may lie between the sinks and a window
                // the last key in front of this query's window; all below head are sinks.  (One loop for tiles with and without
                // sinks: as two branches their 64 results each take more registers than there are.)
                const int before = pos + shift - kv0 - lane_key, head = sinks - kv0 - lane_key;
                mask([&](int key) -> bool { return (key < head) | (key > before); });
            }
        }
        if constexpr (BF16 && BKV == 64) {
            if (a.hide && !pre) {      // scattered queries: rows of positions that are not settled yet, the query's own excepted
                const int t = kv0 + lane - a.P0;
                const unsigned long long hidden = __ballot(t >= 0 && t < a.Lblk && a.hide[(int64_t)b * a.Lblk + t] != 0);
                if (hidden != 0) {
#pragma unroll
                    for (int kb = 0; kb < NKB; ++kb) {
                        const uint32_t mine = (uint32_t)(hidden >> (kb * 32)) >> (8 * lh);
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            if (((mine >> (16 * (e >> 3) + (e & 7))) & 1u) && kv0 + lane_key + key_at(kb, e) < pos) s[kb][e] = -__builtin_huge_valf();
                            if ((e & 3) == 3) __builtin_amdgcn_sched_barrier(0);
                        }
                    }
                }
            }
        }
        float mx = -__builtin_huge_valf();
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
            for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[kb][e]);
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float mxs = mx * a.scale_log2;
        const float m_new = mxs > m_run + LAZY_EXP ? mxs : m_run;
        // a query that has seen no key yet keeps -inf as its maximum: exponents are then taken against 0, and every
        // term is exp2(-inf) = 0 instead of NaN
        m_safe = m_new == -__builtin_huge_valf() ? 0.f : m_new;
        alpha = __builtin_amdgcn_exp2f(m_run - m_safe);
        m_run = m_new;
    };
    auto output = [&](int i) {
        const unsigned char* const vt = buffer(i) + KT;
        float ps = 0.f;
        auto rescale = [&]() {     // only when some query of the wavefront raised its maximum
            if (!__all(alpha == 1.0f)) {
#pragma unroll
                for (int d = 0; d < NDB; ++d)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[d][e] *= alpha;
            }
        };
        if constexpr (BF16) {
            // keys kv0 + 16 ks .. + 15 per step ks; the exponentials of step ks + 1 and its V^T fragments go between the
            // matrix instructions of step ks, in three stages a slot apart
            chunk pf[2], vf[2][NDB];
            float x[2][2], p[2][2];
            auto arg = [&](auto gc) {
                constexpr int g = decltype(gc)::value, ks = g / 4, e = 2 * (g % 4);
                if constexpr (g < BKV / 4) {
#pragma unroll
                    for (int q = 0; q < 2; ++q) x[g & 1][q] = __builtin_fmaf(s[ks >> 1][(ks & 1) * 8 + e + q], a.scale_log2, -m_safe);
                }
            };
            auto expo = [&](auto gc) {
                constexpr int g = decltype(gc)::value;
                if constexpr (g < BKV / 4) {
#pragma unroll
                    for (int q = 0; q < 2; ++q) p[g & 1][q] = __builtin_amdgcn_exp2f(x[g & 1][q]);
                }
            };
            auto take = [&](auto gc) {
                constexpr int g = decltype(gc)::value, ks = g / 4, e = 2 * (g % 4);
                if constexpr (g < BKV / 4) {
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        ps += p[g & 1][q];
                        pf[ks & 1][e + q] = (__bf16)p[g & 1][q];
                    }
                }
            };
#pragma unroll
            for (int d = 0; d < NDB; ++d) vf[0][d] = *reinterpret_cast<const chunk*>(vt + vfrag + d * 32 * VRB);
            static_for<4>([&](auto gc) { arg(gc); expo(gc); take(gc); });
            arg(std::integral_constant<int, 4>{});
            expo(std::integral_constant<int, 4>{});
            arg(std::integral_constant<int, 5>{});
            rescale();
            static_for<NKS>([&](auto kc) {
                constexpr int ks = decltype(kc)::value, nxt = ks + 1 < NKS ? ks + 1 : ks;
                static_for<NDB>([&](auto ic) {
                    constexpr int d = decltype(ic)::value, m = 4 / NDB;   // pairs per slot
                    if constexpr (nxt > ks) vf[nxt & 1][d] = *reinterpret_cast<const chunk*>(vt + (vfrag ^ (nxt << 5)) + d * 32 * VRB);
                    static_for<m>([&](auto qc) {
                        constexpr int g = 4 * ks + d * m + decltype(qc)::value + 4;
                        take(std::integral_constant<int, g>{});
                        expo(std::integral_constant<int, g + 1>{});
                        arg(std::integral_constant<int, g + 2>{});
                    });
                    o[d] = Chunk<T>::mma(vf[ks & 1][d], pf[ks & 1], o[d]);
                    __builtin_amdgcn_sched_barrier(0);
                });
            });
        } else {
            rescale();
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks) {
                chunk p;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[ks / (16 / E)][ks % (16 / E) * E + e], a.scale_log2, -m_safe));
                    ps += p[e];
                }
#pragma unroll
                for (int d = 0; d < NDB; ++d) o[d] = Chunk<T>::mma(*reinterpret_cast<const chunk*>(vt + (vfrag ^ (ks << 5)) + d * 32 * VRB), p, o[d]);
            }
        }
        l_run = l_run * alpha + ps;
    };
    // does some query of the wavefront see some key of the tile?
    auto in_sight = [&](int i) {
        const bool pre = i < np;
        const int kv0 = tile_of(i) * BKV;
        if (!pre && kv0 > w_max) return false;
        return !window || kv0 < a.sinks - (pre ? 0 : S) || kv0 + BKV - 1 > w_min + (pre ? S : 0) - window;
    };
    if constexpr (FEW) {
        // K of the next tile goes out once this one's scores are read, V^T once its products are
        const int i0 = t_begin + wave;
        if (i0 < t_end) load_kv(i0);
        for (int i = i0; i < t_end; i += NW) {
            const int next = i + NW;
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LV) : "memory");       // K has landed (and the queries)
            score(i);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (next < t_end) {
                load(next, true, false);
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LK) : "memory");
            } else {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            }
            clear_unseen(i);
            asm volatile("" ::: "memory");
            output(i);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (next < t_end) load(next, false, true);
        }
        // the join: every wavefront leaves its output, unnormalised, in its buffer, 16-byte chunk c of row r at c ^ (r mod DH / 4)
        __shared__ float2 stat[NW][32];
        l_run += __shfl_xor(l_run, 32);
        static_assert(32 * DH * 4 <= BUF, "an output in a buffer");
        f32x4* const mine = reinterpret_cast<f32x4*>(buffer(0)) + l32 * (DH / 4);
#pragma unroll
        for (int d = 0; d < NDB; ++d)
#pragma unroll
            for (int g4 = 0; g4 < 4; ++g4)
                mine[(d * 8 + g4 * 2 + lh) ^ (l32 & (DH / 4 - 1))] = f32x4{o[d][g4 * 4], o[d][g4 * 4 + 1], o[d][g4 * 4 + 2], o[d][g4 * 4 + 3]};
        if (lh == 0) stat[wave][l32] = make_float2(m_run, l_run);
        __syncthreads();
        const int live = n - qt * 32 < 32 ? n - qt * 32 : 32;
        for (int x = tid; x < live * (DH / 4); x += NTH) {
            const int row = x / (DH / 4), c4 = x % (DH / 4);
            float M = -__builtin_huge_valf();
#pragma unroll
            for (int w = 0; w < NW; ++w) M = fmaxf(M, stat[w][row].x);
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
            float den = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float2 st = stat[w][row];
                const float f = st.x == -__builtin_huge_valf() ? 0.f : __builtin_amdgcn_exp2f(st.x - M);
                sum += f * reinterpret_cast<const f32x4*>(smem + w * BUF)[row * (DH / 4) + (c4 ^ (row & (DH / 4 - 1)))];
                den += f * st.y;
            }
            const int rr = qt * 32 + row, in_head = a.by_L.of(rr);      // of the heads of a key head
            store4(b, hd * group + in_head, rr - in_head * a.L, c4 * 4, sum * (den > 0.f ? 1.0f / den : 0.f));
        }
        return;
    }
    load_kv(t_begin);
    clear_unseen(t_begin);
#pragma unroll
    for (int kk = 0; kk < NKK; ++kk) asm volatile("" : "+v"(qf[kk]));   // wait for the queries here: among the tiles' loads that wait is for those as well
    meet();
    for (int t = t_begin; t < t_end; ++t) {
        if (t + 1 < t_end) load_kv(t + 1);   // everybody has read the buffer: the barrier at the end of the tile before
        if (wave_live && in_sight(t)) {
            score(t);
            output(t);
        }
        if (t + 1 < t_end) {
            clear_unseen(t + 1);
            meet();
        }
    }

    l_run += __shfl_xor(l_run, 32);
    if (r_raw >= n) return;
    if (partial) {
        float* const pq = a.part + (slot * all_rows + out_row) * DH;
#pragma unroll
        for (int i = 0; i < NDB; ++i)
#pragma unroll
            for (int g4 = 0; g4 < 4; ++g4)
                *reinterpret_cast<f32x4*>(pq + i * 32 + g4 * 8 + lh * 4) = f32x4{o[i][g4 * 4], o[i][g4 * 4 + 1], o[i][g4 * 4 + 2], o[i][g4 * 4 + 3]};
        if (lh == 0) *reinterpret_cast<float2*>(a.ml + 2 * (slot * all_rows + out_row)) = make_float2(m_run, l_run);
        return;
    }
    const float inv = l_run > 0.f ? 1.0f / l_run : 0.f;
    auto done = [&](float x) { return active ? x * inv : 0.f; };      // an unused slot's query may hold anything
#pragma unroll
    for (int i = 0; i < NDB; ++i)
#pragma unroll
        for (int g4 = 0; g4 < 4; ++g4)
            store_out(i, g4, f32x4{done(o[i][g4 * 4]), done(o[i][g4 * 4 + 1]), done(o[i][g4 * 4 + 2]), done(o[i][g4 * 4 + 3])});
}

// A wavefront joins the shares of a query: lane s takes the weight of share s, then every lane DH / 64 channels of all of them.
// One memory round trip: the outputs of NS shares (those there are not re-read the first) are requested together with the weights.
// Rows of absent sequences and unused slots are zeros, whatever the shares hold: workgroups of the prefix have gone over their
// queries as well, which may be infinite or NaN.
constexpr int JOIN_WAVES = 4;
template <class T, int DH, int NS>
__global__ __launch_bounds__(64 * JOIN_WAVES) void k_context_join(const Args a, int slots) {
    constexpr int C = DH / 64;
    const uint32_t all_rows = (uint32_t)(a.B * a.nh * a.L), row = blockIdx.x * JOIN_WAVES + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (row >= all_rows) return;
    const float* const src = a.part + (int64_t)row * DH + lane * C;
    float v[NS][C];
    auto request = [&](int s0) {
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            const float* p = src + (int64_t)(s0 + i < slots ? s0 + i : 0) * all_rows * DH;
#pragma unroll
            for (int c = 0; c < C; ++c) v[i][c] = p[c];
        }
    };
    request(0);
    const float2 ml = lane < slots ? *reinterpret_cast<const float2*>(a.ml + 2 * ((int64_t)lane * all_rows + row)) : make_float2(-__builtin_huge_valf(), 0.f);
    const uint32_t j = row % (uint32_t)a.L, bh = row / (uint32_t)a.L, h = bh % (uint32_t)a.nh, b = bh / (uint32_t)a.nh;
    const bool absent = (a.P_seq && a.P_seq[b] < 0) || (a.pos_tab && a.pos_tab[b * a.L + j] < 0);
    float M = ml.x;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
    const float w = ml.x == -__builtin_huge_valf() ? 0.f : __builtin_amdgcn_exp2f(ml.x - M);
    float den = ml.y * w;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) den += __shfl_xor(den, o);
    float acc[C] = {};
    for (int s0 = 0;;) {
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            const float ws = s0 + i < slots ? __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(w), s0 + i)) : 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c) acc[c] = ws != 0.f ? __builtin_fmaf(v[i][c], ws, acc[c]) : acc[c];      // an empty share has left nothing behind
        }
        s0 += NS;
        if (s0 >= slots) break;
        request(s0);
    }
    const float inv = den > 0.f ? 1.0f / den : 0.f;
    T* const op = reinterpret_cast<T*>(a.out) + (a.frag ? frag_index(b * a.L + j, h * DH + lane * C, a.nh * DH)
                                                        : (int64_t)b * a.out_batch + h * a.out_head + j * a.out_row + lane * C);
#pragma unroll
    for (int c = 0; c < C; ++c) op[c] = (T)(absent ? 0.f : acc[c] * inv);
}
template <class T, int DH>
void join(const Args& a, int slots, hipStream_t st) {
    const dim3 grid((unsigned)(((int64_t)a.B * a.nh * a.L + JOIN_WAVES - 1) / JOIN_WAVES)), block(64 * JOIN_WAVES);
    if (slots <= 4) hipLaunchKernelGGL((k_context_join<T, DH, 4>), grid, block, 0, st, a, slots);
    else if (slots <= 8) hipLaunchKernelGGL((k_context_join<T, DH, 8>), grid, block, 0, st, a, slots);
    else hipLaunchKernelGGL((k_context_join<T, DH, 16>), grid, block, 0, st, a, slots);
}

// Keys per tile where queries are few: at most 64 KB of LDS, two workgroups per CU.  float32 is bound by its matrix instruction (2 us a
// tile of 32 keys and wavefront): smaller tiles deal its keys to more workgroups (heads of 64, 64 / 32 keys, us: 1 x 150 queries,
// 500 rows 22.5 / 17.9, 16 tokens of 8 heads, 1000 shared and 1000 own rows 50 / 34, 2 x 8 16.5 / 13; 4 tokens of 16 heads, 2000 rows 47 / 51).
constexpr int small_tile(int esz) { return esz == 2 ? 64 : 32; }
// Wavefronts of the one-launch kernel: 8, or as many as have room for a tile of 32 keys each in 128 KB.
constexpr int few_waves(int esz, int dh) { return esz * dh > 256 ? 4 : 8; }

// Key tiles that the queries see at most (host; P rows in front of the block)
int own_tiles(const ContextAttn& a, int bkv) {
    const int64_t end = a.pos_tab ? (int64_t)a.P0 + a.Lblk : (int64_t)a.P + a.L;
    if (!a.window) return (int)((end + bkv - 1) / bkv);
    const int64_t first = a.pos_tab ? a.P0 : a.P, lo = first - a.window + 1 > 0 ? first - a.window + 1 : 0;
    int64_t head = (int64_t)a.sinks - a.S;
    head = head < 0 ? 0 : head < lo ? head : lo;
    return (int)((end - lo + bkv - 1) / bkv + 1 + (head + bkv - 1) / bkv);
}
int prefix_tiles(const ContextAttn& a, int bkv) {
    if (!a.S) return 0;
    if (!a.window) return (a.S + bkv - 1) / bkv;
    const int64_t first = a.pos_tab ? a.P0 : a.P;
    int64_t lo = a.S + first - a.window + 1;
    lo = lo < 0 ? 0 : lo < a.S ? lo : a.S;
    const int64_t head = a.sinks < lo ? a.sinks : lo;
    return (int)((a.S - lo + bkv - 1) / bkv + (head + bkv - 1) / bkv);
}

int clamp_int(int64_t v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : (int)v; }

// What a tile costs a workgroup, in halves of what it costs one with 32 queries: float32 wavefronts get in each other's way (16 x 5 of
// 16 heads of 128, 100 own rows, 300 and 600 shared: as 3 halves 33.5 and 35 us, as 2 42.5 and 43; bf16 8 x 16 of 32 heads, 200 and
// 1000 rows, 27.7 and 23.8).
int tile_cost(int esz, int64_t queries) { return esz == 4 && queries > 32 ? 3 : 2; }
// When the last of a launch's workgroups ends, where `places` run at a time: first `prefix` ones of `prefix_time` each, behind them `own` ones.
int64_t makespan(int64_t prefix, int64_t prefix_time, int64_t own, int64_t own_time, int64_t places) {
    const int64_t t = prefix / places * prefix_time, busy = prefix % places;
    if (!busy) return t + (own + places - 1) / places * own_time;
    if (own <= places - busy) return t + (prefix_time > own_time ? prefix_time : own_time);
    const int64_t left = own - (places - busy) * (prefix_time / own_time);      // once the last prefix workgroup has ended
    return t + prefix_time + (left > 0 ? (left + places - 1) / places * own_time : 0);
}

// part_floats: the scratch there is (context_attention_floats asks with as much as can be wanted)
Plan make_plan(const ContextAttn& a, int esz, int64_t part_floats) {
    Plan p{};
    const int group = a.nh / a.nkv, bkv = small_tile(esz);
    const int64_t slot_floats = (int64_t)a.B * a.nh * a.L * (a.dh + 2);
    const int slots = clamp_int(part_floats / slot_floats, 0, MAX_SLOTS);
    p.by_kv = (int64_t)group * a.L <= 128;
    p.heads = p.by_kv ? a.nkv : a.nh;
    p.n = p.by_kv ? group * a.L : a.L;
    p.tiles = (p.n + 127) / 128;
    p.split = 1;
    // Workgroups that run at a time, two per CU, and to how many keys are dealt.  us, 256 / 512 / 1024, heads of 128: 8 tokens, 100 own and
    // 1000 shared rows 15.8 / 14.9 / 19.4, 16 x 16 of 330 and 4224 74 / 58 / 70, 1 token of 4000 rows 23.3 / 20.7 / 25.5, 1 x 64 of
    // 4000 27.4 / 29.9 / 38; 8 tokens of 16 heads of 64, 100 and 4000 15.5 / 13.9 / 15.0; float32 6 x 5 of 300 and 333 16.4 / 14.3 / 14.4.
    const int TARGET = 512;
    const int64_t base = (int64_t)a.B * p.heads * p.tiles;
    const int n_own = own_tiles(a, bkv), n_pre = prefix_tiles(a, bkv);
    // One launch instead of two, as long as every (sequence, key head) has its place on a CU (128 KB of LDS; heads of 64 half) and
    // streams its keys there about as fast as more CUs would and the join adds.  Tokens of 32 heads of 128, us, two launches / one:
    // 1 sequence of 60, 250, 500, 700, 1000 rows 6.2 / 5.2, 9.3 / 7.0, 10.2 / 9.3, 11.3 / 10.6, 11.9 / 13.3; 4 of 250, 700, 1000
    // 11.3 / 8.1, 15.8 / 14.5, 20.7 / 23.4; 8 (256 workgroups) of 500, 1000, 1500 21 / 17, 32 / 28, 44 / 40; 16 of 60, 500 8.8 / 10.7,
    // 29 / 31; 8 behind a prefix of 250, 500, 1000, 60 own rows 11 / 8, 12.2 / 10, 13.8 / 14.  16 heads of 64: 4, 16, 32
    // sequences of 1000 rows 11.5 / 9.2, 22 / 16, 30 / 28.  Blocks, a workgroup per 32 queries, up to two rounds of them: 1 x 150 queries
    // of 32 heads of 128, 500 rows in front 22.6 / 12.4, 1 x 300 (320 workgroups) 26 / 21.5, 1 x 403 through a window of 35 22 / 13,
    // four rounds: 4 x 256 18 / 30, 2 x 502 through one of 27 26.7 / 30; 16 heads of 64: 1 x 500 12 / 7, 1 x 250 through one of 300 18 / 7.
    // float32 is bound by its matrix instruction: only where every wavefront has one tile.  8 heads of 64 and 8 key heads, us: 1 token,
    // 40 rows 8.9 / 6.3, 16 behind a prefix of 100 11.7 / 7.4, 1 x 100 queries 10.0 / 6.6, three tiles a wavefront: 1 of 500 rows
    // 9.3 / 13.3, 1 x 60 queries behind 200 rows 10.3 / 12.0; 8 heads of 128: 4 tokens of 50 rows 11.0 / 9.6, 1 x 100 13.9 / 10.2.
    const int per_cu = 128 / a.dh, places = cu_count() * per_cu;
    const int64_t few = ((int64_t)group * a.L + 31) / 32 * a.B * a.nkv;
    int few_keys = n_own + n_pre;      // tiles that 32 queries see
    if (a.window) few_keys = clamp_int(((int64_t)a.window + 32) / bkv + 2 + ((int64_t)a.sinks + bkv - 1) / bkv, 1, few_keys);
    const bool fits = esz == 2 ? few <= (group * a.L > 32 ? 2 : 1) * (int64_t)places && n_pre <= 12 * per_cu && few_keys <= (4 * few >= 3 * places ? 24 : 12) * per_cu
                               : few <= cu_count() && few_keys <= few_waves(4, a.dh);
    if (!a.pos_tab && fits) {
        p.few = true;
        p.by_kv = true;
        p.heads = a.nkv;
        p.n = group * a.L;
        return p;
    }
    const int n = n_own + n_pre;
    const int whole_split = a.L <= 128 ? clamp_int(TARGET / base, 1, MAX_SLOTS < n ? MAX_SLOTS : n) : 1;
    // Stacked or whole: the tiles that follow one another on a place, at some 1.2 us a tile (float32, bound by its matrix instruction: 2.6
    // and 5.1 us with heads of 64 and 128), against the partial results that stacking writes and reads more of (5 TB/s), and the join's launch
    // where there would be none.  How finely the keys are dealt is that of the shortest makespan: a few workgroups more than have a
    // place cost as much as a second round of them (4 tokens of 32 heads of 128, 2000 own and shared rows: 640 workgroups 47.7 us, 448
    // 37.7).  us, whole / stacked, 32 heads of 128, rows own + shared: 4 tokens 100 + 2000 23.2 / 15.7, 8 of 1000 + 1000 42.4 / 43.3,
    // 2000 + 500 61 / 68, 32 of 200 + 4000 225 / 47; 16 x 4 200 + 500 29.4 / 27.3; 8 x 64 500 + 2000 63 / 53; 8 key heads: 16 x 4
    // 100 + 1000 16.8 / 18.6 and 100 + 4000 35.7 / 25; 64 x 16 100 + 300 24 / 39.  float32, 8 heads of 64: 16 tokens 100 + 400
    // 22.4 / 13.9, 6 x 5 300 + 333 17.3 / 14.1; 16 of 128: 16 x 5 100 + 600 61 / 35, 800 + 300 94 / 130.
    if (p.by_kv && n_pre > 0 && !(a.P_seq && a.window) && slots >= 2) {
        p.prefix_tiles = (int)(((int64_t)(a.B / a.G) * p.n + 127) / 128);
        const int64_t pbase = (int64_t)a.G * a.nkv * p.prefix_tiles;
        const int own_cost = tile_cost(esz, p.n), prefix_cost = tile_cost(esz, (int64_t)(a.B / a.G) * p.n);
        int64_t best = INT64_MAX;
        for (int64_t per = (base * n_own + pbase * n_pre + TARGET - 1) / TARGET;; per += 1 + per / 16) {      // tiles of a workgroup
            const int s = clamp_int((n_own + per - 1) / per, 1, MAX_SLOTS / 2), ps = clamp_int((n_pre + per - 1) / per, 1, MAX_SLOTS - s);
            const int64_t t = makespan(pbase * ps, (n_pre + ps - 1) / ps * prefix_cost, base * s, (n_own + s - 1) / s * own_cost, TARGET);
            if (t <= best) best = t, p.split = s, p.prefix_split = ps;
            if ((s == 1 && ps == 1) || per > best) break;      // some workgroup has more than half of `per` tiles, 2 each: no shorter one follows
        }
        const int64_t whole = (base * whole_split + TARGET - 1) / TARGET * ((n + whole_split - 1) / whole_split) * own_cost;
        const int more = p.split + p.prefix_split - (whole_split > 1 ? whole_split : 0);
        const double gain = (double)(whole - best) / 2 * (esz == 2 ? 1.2 : a.dh * 0.04);
        const double cost = (more > 0 ? more : 0) * (double)slot_floats * 8 / 5e6 + (whole_split > 1 ? 0 : 3);
        p.stacked = gain > cost;
    }
    if (p.stacked) {
        if (p.split + p.prefix_split > slots) {      // less scratch than this runs fastest with
            const int half = slots / 2;
            if (p.split <= half) p.prefix_split = slots - p.split;
            else if (p.prefix_split <= half) p.split = slots - p.prefix_split;
            else p.split = half, p.prefix_split = slots - half;
        }
        p.prefix_wgs = (int)((int64_t)a.G * a.nkv * p.prefix_tiles * p.prefix_split);
        return p;
    }
    p.split = whole_split < slots ? whole_split : slots < 1 ? 1 : slots;
    // Long blocks that do not find a CU each: shares of at least 4 tiles (float32, whose matrix instruction takes 16 times as long: 2) of
    // what a query sees on average, bf16 from 12 of them on.  1 x 300 queries, 1000 rows in front, us, whole / in shares: bf16
    // 32 heads of 128 37 / 27, 16 of 64 24 / 16, float32 8 of 64 101 / 25; 1 x 1024, nothing in front (8 tiles): 16 of 64 19 / 22;
    // 2 x 600 through a window of 545 (10) 20 / 23, float32 8 of 64 64 / 34.
    if (slots >= 2 && a.L > 128 && base < cu_count()) {
        ContextAttn half = a;
        half.L = a.L / 2;
        int seen = n_pre + own_tiles(half, bkv);
        if (a.window) seen = clamp_int(((int64_t)a.window + a.sinks + 128) / bkv + 1, 1, seen);      // of a workgroup's 128
        const int most = seen / (esz == 2 ? 4 : 2);
        if (esz == 4 || seen >= 12) p.split = clamp_int(TARGET / base, 1, most < 1 ? 1 : most < slots ? most : slots);
    }
    return p;
}

template <class T, int DH, int BQ, int BKV, int NTH, bool FEW = false>
void run_cfg(Args a, hipStream_t st) {
    auto kern = k_context<T, DH, BQ, BKV, NTH, FEW>;
    const int lds = (FEW ? NTH / 64 : 2) * 2 * BKV * DH * (int)sizeof(T);
    static int attr_state[MAX_DEVICES] = {};
    if (!ensure_dynamic_lds_here(reinterpret_cast<const void*>(kern), lds, attr_state)) return;
    a.tiles = (a.n + BQ - 1) / BQ;
    a.group = a.nh / a.nkv;
    a.in_group = a.B / a.G;
    a.shares = a.tiles * a.heads * a.B;
    a.by_group = Div(a.group); a.by_in_group = Div(a.in_group); a.by_L = Div(a.L); a.by_n = Div(a.n); a.by_heads = Div(a.heads);
    a.by_tiles = Div(a.tiles); a.by_shares = Div(a.shares); a.by_gk = Div(a.G * a.nkv); a.by_nkv = Div(a.nkv);
    a.by_prefix_tiles = Div(a.stacked ? a.prefix_tiles : 1);
    const int64_t all_rows = (int64_t)a.B * a.nh * a.L;
    const int slots = a.split + (a.stacked ? a.prefix_split : 0);
    a.ml = a.part ? a.part + slots * all_rows * DH : nullptr;
    hipLaunchKernelGGL(kern, dim3((unsigned)((int64_t)a.tiles * a.heads * a.B * a.split + a.prefix_wgs)), dim3(NTH), lds, st, a);
    if (slots > 1) join<T, DH>(a, slots, st);
}

template <class T, int DH>
void run(const ContextAttn& c, hipStream_t st) {
    Args a{};
    static_cast<ContextAttn&>(a) = c;
    static_cast<Plan&>(a) = make_plan(c, sizeof(T), c.part ? c.part_floats : 0);
    constexpr int SMALL = small_tile(sizeof(T));
    if (a.few) return run_cfg<T, DH, 32, 32, 64 * few_waves(sizeof(T), DH), true>(a, st);
    if constexpr (sizeof(T) == 2) {
        // long blocks that go over their keys as a whole: tiles of 128 keys, and 256 queries where 128 would not find a CU each (heads of 128), as in attention.hip
        if (c.L > 128 && !c.pos_tab && a.split == 1) {
            if (DH == 128 && (int64_t)c.B * c.nh * ((c.L + 127) / 128) > cu_count()) return run_cfg<T, DH, DH == 128 ? 256 : 128, 128, DH == 128 ? 512 : 256>(a, st);
            return run_cfg<T, DH, 128, 128, 256>(a, st);
        }
    }
    run_cfg<T, DH, 128, SMALL, 256>(a, st);
}

}  // namespace

size_t context_attention_floats(const ContextAttn& a) {
    const int64_t slot_floats = (int64_t)a.B * a.nh * a.L * (a.dh + 2);
    const Plan p = make_plan(a, a.dtype == 1 ? 2 : 4, MAX_SLOTS * slot_floats);
    const int slots = p.split + (p.stacked ? p.prefix_split : 0);
    return slots > 1 ? (size_t)(slots * slot_floats) : 0;
}

void launch_join_shares(const ContextAttn& c, int shares, hipStream_t st) {
    Args a{};
    static_cast<ContextAttn&>(a) = c;
    a.ml = c.part + (int64_t)shares * c.B * c.nh * c.L * c.dh;
    if (c.dtype == 1) {
        if (c.dh == 128) join<__bf16, 128>(a, shares, st);
        else join<__bf16, 64>(a, shares, st);
    } else {
        if (c.dh == 128) join<float, 128>(a, shares, st);
        else join<float, 64>(a, shares, st);
    }
}

void launch_context_attention(const ContextAttn& a, hipStream_t st) {
    if (a.dtype == 1) {
        if (a.dh == 128) run<__bf16, 128>(a, st);
        else run<__bf16, 64>(a, st);
    } else {
        if (a.dh == 128) run<float, 128>(a, st);
        else run<float, 64>(a, st);
    }
}

}  // namespace mulo
