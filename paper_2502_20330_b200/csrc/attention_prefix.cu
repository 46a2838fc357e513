// Verify attention of a batch whose sequences share a long prefix (Algorithm 1's LogitsOf pass for several
// requests, or several drafts, over one document).
//
//   out[b,i,h,:] = sum_j softmax_j(scale q[b,i,h,:] . k_j) v_j     over the P prefix keys (seen by every row)
//                                                                  and the keys j <= L_b - R + i of sequence b
//
// The prefix's K/V are stored once and are read once for all rows of the batch: the B*R*G query rows of a
// KV head are packed into tiles of 128 rows (the M axis of the MMAs) whatever sequence they belong to,
// and a CTA takes two such row tiles through the same K/V tiles.  Each sequence's own keys are work of
// the same kernel, as further units; the merge kernel joins what the units left by their log-sum-exp.
//
// Segments.  A CTA works through segments: a run of 128-key tiles of one unit.  Two streams (groups of four softmax
// warps, each with S and O accumulators and an MMA issuer of its own) take every tile in blocks of 64 keys:
//   dual-row segment  prefix of one KV head, two row tiles: stream s takes row tile s through both blocks;
//   dual-key segment  one row tile (the last prefix tile of an odd count, or the R*G rows of one sequence over
//                     its own keys): stream s takes block s, and leaves a partial of its own.
//
//   S_s[128 x 64] = Q_s K_block^T   A = Q tile, B = 64 rows of the K tile, both K-major in shared memory
//   O_s[128 x D] += P_s V_block     A = P (bf16, over the first half of the S block's columns), B = V rows, MN-major
//
// S has room for two blocks: while the softmax warps are at one, the PV and the next QK^T of the other run (with
// one S of 128 keys a stream's softmax and products alternate: 190 us for the 60K-key batch of 1,120 rows).
//
// Work split (worked out by every CTA for itself: no plan kernel, no plan to go stale).  Cost is counted in
// half tiles of a stream's work: 2 for a dual-row tile, 1 for a dual-key tile, kPad for changing to another unit.
// With np pairs of row tiles the prefix is cut into equal ranges of key tiles, each for a team of np CTAs, one
// pair each: a team reads the same K/V tiles at the same time, so they leave HBM once.  The sequences'
// own tiles fill up every CTA to the same level (CTAs outside the teams first, then those with a single
// row tile, then all).
//
// Bound: up to 256 rows per KV head (one pair) a K/V tile of 64 KB is read for every 256 x 128 scores, and HBM
// is the limit; from two pairs on the tensor cores and the exponentials are.  Measured (two kernels, calls in a row in
// a graph, D = 128, bf16):
//     8 requests of 1 row over 32K + up to 1,000 keys, 32 heads over 8       37 us   4.0 TB/s of the keys read once
//     7 requests of 9 rows over 128K + up to 2,048, 32 over 8               146 us   4.0 TB/s and 0.94 PFLOP/s
//    32 requests of 5 rows over 60K + up to 4,000, 28 over 4          156 - 172 us   0.91 - 0.83 PFLOP/s, by process
//    48 requests of 1 row over 8K + up to 1,500, paged in 64, 32 over 8      54 us   3.5 TB/s
//    16 requests of 9 rows over 32K + up to 3,000, paged in 256, 64 over 8  169 us   0.96 PFLOP/s
// and up to a quarter more for the large ones while they run for seconds (the clock falls to 1.5 - 1.6 GHz under the
// power cap).  In those the tensor core is at work 68 - 69 % of the time: a QK^T of N = 64 takes one and a half times
// its products, because it reads its 128 x 16 A operand from shared memory for 64 columns only.  N = 128 would not,
// but leaves no second S (above).  The exponentials take 36 % of the special-function unit, issue slots 49 %.
//
// Waits are bounded as everywhere in this library; see mbar_wait_bounded.  A parity wait tells a phase from its
// neighbours only, so every barrier here is one that at a wait is in the phase waited for or just past it.
// Per stream there are two of each block barrier, for even and for odd blocks: scores of block j in hand
// mean that the PV of block j - 2 has completed, but say nothing of j - 1.
#include <math.h>

#include <atomic>

#include "common.cuh"
#include "prefix_kv8.cuh"
#include "tcgen05.cuh"

namespace rapid {

namespace {

constexpr int kKeys = 128;             // keys per tile
constexpr int kThreads = 384;          // two softmax groups of 128; the producer, the walk, an MMA warp for each stream
constexpr int kBlock = 64;             // keys of a block: what a stream takes at a time
constexpr int kHalfBytes = kKeys * 128;  // one 64-column half of a tile of 128 rows
constexpr int kPad = 3;                // single-stream tiles that a change of unit costs
constexpr int kPoly = 3;               // of 8 pairs of exponentials, those that the FMA pipe takes from the special-function unit
constexpr int kMaxPrefixCtas = 256;
constexpr float kJump = 16.f;          // a score this far (log2) above a row's reference moves it: probabilities stay below 2^16 as
                                       // in the kernels without a prefix, and O below 2^16 |V| a key (at 40 a |V| of 3e26 overflowed)

__host__ __device__ constexpr int k_slots(int D) { return D == 128 ? 2 : 4; }
__host__ __device__ constexpr int v_slots(int D) { return D == 128 ? 3 : 6; }
__host__ __device__ constexpr int tile_bytes(int D) { return (D / 64) * kHalfBytes; }
__host__ __device__ constexpr int smem_bytes(int D) { return (2 + k_slots(D) + v_slots(D)) * tile_bytes(D) + 1024; }

// Partial results: a slot holds `rows` rows of unnormalised O as [D/4][rows][4] floats (so that a warp whose
// lanes are rows writes and reads whole lines), then the rows' references (log2), then their sums.
__host__ __device__ constexpr long long slot_floats(int rows, int D) { return ((long long)rows * (D + 2) + 3) / 4 * 4; }

struct PrefixArgs {
    const int32_t* ctx_lens;
    const int32_t* prefix_len;
    const int32_t* block_table;  // paged cache, or NULL
    float* part_prefix;          // [(team + KV head) * 2 np + 2 pair + stream]
    float* part_own;             // [(worker + unit) * 2 + stream]
    int2* prefix_range;          // per KV head: first and last team with tiles of it
    int2* own_range;             // per (sequence, KV head): first and last worker
    int32_t* status;
    int32_t* plan_sig;           // first word of a verify plan's signature, see ws_layout
    int B, R, G, Hq, Hkv, GR;
    int Pmax, Lmax;              // capacities in keys (paged: both the capacity of a table row)
    int block_size, block_log2, num_blocks, max_blocks, box_rows;
    int rows_tile;               // (sequence, row) pairs in a row tile: 128 / G
    int nrt, np;                 // row tiles, pairs of row tiles
    int team_ctas, max_teams;    // CTAs of a team (np, at most the grid) and teams that the grid holds
    int rounds, row_cost;        // passes over the prefix where np exceeds the grid; cost of a prefix tile to a CTA
    int num_ctas;
    float scale_log2;
    long long wait_limit;
};

// Lengths as the device finds them, brought into range.
__device__ __forceinline__ int clamp_prefix(const PrefixArgs& a, int P) {
    P = max(0, min(P, a.Pmax));
    if (a.block_table) P = min(P, a.Lmax - a.R) & ~(a.block_size - 1);  // whole blocks that leave room for the rows' own
    return P;
}
// A sequence's own keys (those behind the prefix) from its entry of ctx_lens.
__device__ __forceinline__ int clamp_own(const PrefixArgs& a, int L, int P) {
    const int before = a.block_table ? P : 0;  // keys that the entry counts too
    return min(max(L, a.R + before), a.Lmax) - before;
}
__device__ __forceinline__ int tiles_of(int keys) { return (keys + kKeys - 1) / kKeys; }

// What a CTA does.  The prefix part follows from the prefix's length alone and is worked out before anything
// else; the own part needs every sequence's length and is worked out while the CTA is at its prefix tiles.
struct Plan {
    int P, nt, pad, span;   // prefix keys and tiles; virtual tiles in front of every KV head's, and those with the real ones
    int teams, team, pair;  // teams, the CTA's team (-1: none) and its first pair of row tiles
    int h, o, len;          // its run of the prefix's padded tile list: KV head, offset in its span, length
    int worker;             // its rank among the CTAs that hold own tiles
    int own_b, own_h, own_o, own_len;  // its run of the own tiles' padded list
};

// Where share i of n of `total` >= n begins; r = total / n, correctly rounded.  Never decreasing, and no share is
// empty: r is 1, or at least 1 + 1/kMaxPrefixCtas, which the rounding of i * r cannot use up.
__device__ __forceinline__ int share_start(int total, int n, float r, int i) {
    return i >= n ? total : min(total, (int)((float)i * r));
}
// x / d for 0 <= x < 2^31 and a quotient below 2^16 (a KV head, a team): the approximate quotient, off by less than
// 2^16 * 2^-21, is cut to within one of the true one.
__device__ __forceinline__ int small_div(int x, int d) {
    int q = (int)__fdividef((float)x, (float)d);
    if (q * d > x) --q;
    if (x - q * d >= d) ++q;
    return q;
}

// (In both functions the length of the code matters as much as anything: a launch fetches it anew, at several
// cycles an instruction.)
__device__ __forceinline__ void plan_prefix(const PrefixArgs& a, int cta, Plan& p) {
    p.P = clamp_prefix(a, *a.prefix_len);
    p.nt = tiles_of(p.P);
    // Teams: one tile each while that leaves half of the grid's teams idle, then eight tiles each up to all teams
    // (a team's partials cost a write and a read of 128 KB per pair and KV head, a tile about 1.5 us).
    const int NP = a.Hkv * p.nt;
    p.teams = min(a.max_teams, max(min(NP, (a.max_teams + 1) >> 1), NP >> 3));
    p.pad = NP >= 4 * p.teams ? kPad : 0;
    p.span = p.nt + p.pad;
    p.team = small_div(cta, a.team_ctas);
    p.pair = cta - p.team * a.team_ctas;
    p.h = p.o = p.len = 0;
    if (p.team < p.teams) {
        const int total = a.Hkv * p.span;
        const float r = __fdiv_rn((float)total, (float)p.teams);
        const int v0 = share_start(total, p.teams, r, p.team);
        p.len = share_start(total, p.teams, r, p.team + 1) - v0;
        p.h = small_div(v0, p.span);
        p.o = v0 - p.h * p.span;
    } else {
        p.team = -1;
        p.pair = a.np;
    }
}

// The own part.  w = cost of a team's range for a CTA with a full pair of row tiles, wh for one with a single row
// tile (class H: the last CTA of every team if the number of row tiles is odd; A: the teams' others; B: the CTAs
// in no team).  All are filled up to one level X: nB X + nH (X - wh)+ + nA (X - w)+ = S, whose solution is the
// smallest of the three that leave out no, one or both of the upper classes.
__device__ __noinline__ void plan_own(const PrefixArgs& a, int cta, Plan& p) {
    const int lane = threadIdx.x & 31;
    const int first_len = lane < a.B ? a.ctx_lens[lane] : 0;
    const int P = p.P;
    int S = 0;
    bool bad = false;  // lengths out of range: only the device can see them, the first CTA says so
#pragma unroll 1
    for (int b = lane; b < a.B; b += 32) {
        const int L = b < 32 ? first_len : a.ctx_lens[b];
        const int own = clamp_own(a, L, P);
        S += a.Hkv * (tiles_of(own) + kPad);
        bad |= L != own + (a.block_table ? P : 0);
    }
    S = __reduce_add_sync(0xffffffffu, S);
    if (cta == 0) {
        const int given = *a.prefix_len;
        bad |= given != P && !(a.block_table && (given & ~(a.block_size - 1)) == P);
        if (__any_sync(0xffffffffu, bad) && lane == 0) atomicOr(a.status, RAPID_STATUS_BAD_CTX_LEN);
    }
    const int in_teams = p.teams * a.team_ctas;
    const bool half = (a.nrt & 1) && a.np > 1 && a.rounds == 1;
    const int nH = half ? p.teams : 0, nA = in_teams - nH, nB = a.num_ctas - in_teams;
    const float w = p.teams > 0 ? ceilf(__fdividef((float)(a.Hkv * p.span) * a.row_cost, (float)p.teams)) : 0.f;
    const float wh = half ? 0.5f * w : w;
    const float fS = (float)S;
    const float X1 = nB > 0 ? __fdividef(fS, (float)nB) : INFINITY;
    const float X2 = nB + nH > 0 ? __fdividef(fS + nH * wh, (float)(nB + nH)) : INFINITY;
    const float X3 = __fdividef(fS + nH * wh + nA * w, (float)a.num_ctas);
    const float X = fminf(X1, fminf(X2, X3));
    // class totals: whole tiles, what is left over goes to the last class that has CTAs and a share
    int SB = min(S, (int)(X * nB)), SH = min(S - SB, (int)(fmaxf(X - wh, 0.f) * nH)), SA = S - SB - SH;
    if (nA == 0 || X <= w) {
        if (nH > 0 && (nB == 0 || X > wh)) SH += SA, SA = 0;
        else if (nB > 0) SB += SA, SA = 0;
    }
    // workers: the CTAs of class B, then H, then A, those without a share left out
    int n = nA, total = SA, off = SB + SH, off_w = min(nB, SB) + min(nH, SH);
    int rank = half ? p.team * (a.team_ctas - 1) + p.pair : cta;
    if (p.team < 0) n = nB, total = SB, off = 0, off_w = 0, rank = cta - in_teams;
    else if (half && p.pair == a.np - 1) n = nH, total = SH, off = SB, off_w = min(nB, SB), rank = p.team;
    n = min(n, total);  // (fewer tiles than CTAs: one each)
    const float r = __fdiv_rn((float)total, (float)max(n, 1));
    const int s0 = off + share_start(total, n, r, rank);
    const int len = off + share_start(total, n, r, rank + 1) - s0;  // 0 from rank n on
    // the unit s0 lies in
    int base = 0, ub = 0, uh = 0, uo = 0;
#pragma unroll 1
    for (int b0 = 0; b0 < a.B && len > 0; b0 += 32) {
        const int b = b0 + lane;
        int one = 0;
        if (b < a.B) one = tiles_of(clamp_own(a, b0 ? a.ctx_lens[b] : first_len, P)) + kPad;
        int incl = a.Hkv * one;
#pragma unroll 1
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += x;
        }
        const unsigned past = __ballot_sync(0xffffffffu, base + incl > s0);
        if (past) {
            const int src = __ffs(past) - 1;
            const int x = s0 - base - __shfl_sync(0xffffffffu, incl - a.Hkv * one, src);
            const int d = __shfl_sync(0xffffffffu, one, src);
            ub = b0 + src;
            uh = small_div(x, d);
            uo = x - uh * d;
            break;
        }
        base += __shfl_sync(0xffffffffu, incl, 31);
    }
    if (lane == 0) {
        p.worker = off_w + rank;
        p.own_b = ub;
        p.own_h = uh;
        p.own_o = uo;
        p.own_len = len;
    }
}

// One lane of a converged warp.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred P;\n\telect.sync _|P, 0xffffffff;\n\tselp.u32 %0, 1, 0, P;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, const WaitCtx& wc) {
    return __all_sync(0xffffffffu, mbar_wait_bounded(bar, parity, wc));
}

// A CTA's segments: one warp walks through its plan and hands them to the other roles through a ring in shared
// memory (the walk inlined in every role was 700 to 2,900 cycles a segment in each, most of it instruction fetch).
struct __align__(16) Segment {
    int tiles;          // run of tiles inside the unit; 0 = the end
    int flags;          // kOwn, kDualRow
    int keys, tile0;    // keys of the unit (own keys or prefix keys), first tile
    int b, kvh, pair;   // sequence (own) or pair of row tiles (prefix)
    int reserved;
};
constexpr int kOwn = 1, kDualRow = 2;
constexpr int kRing = 8;       // segments in the ring
constexpr int kRingUsers = 11;  // arrivals that free one: 8 softmax warps, the producer, two MMA threads

struct Ring {
    Segment seg[kRing];
    uint64_t full[kRing], empty[kRing];
};
// Puts segment number i into the ring (a whole warp; lane 0 writes).
__device__ __forceinline__ bool ring_put(Ring& r, int i, const Segment& g, const WaitCtx& wc) {
    const int s = i & (kRing - 1);
    if (i >= kRing && !warp_wait(&r.empty[s], (i / kRing - 1) & 1, wc)) return false;
    if ((threadIdx.x & 31) == 0) {
        r.seg[s] = g;
        mbar_arrive(&r.full[s]);
    }
    __syncwarp();
    return true;
}

__device__ __forceinline__ void walk(const PrefixArgs& a, const Plan& p, Ring& ring, int cta, Plan& out, const WaitCtx& wc) {
    int n = 0;
    Segment g = {};
    // the prefix part: every pair of the CTA's over the same run of tiles
    for (int pair = p.pair; pair < a.np; pair += a.team_ctas) {
        int h = p.h, o = p.o, left = p.len;
        while (left > 0) {
            const int e = min(p.span, o + left);
            g.flags = 2 * pair + 1 < a.nrt ? kDualRow : 0;
            g.keys = p.P;
            g.kvh = h;
            g.pair = pair;
            g.tile0 = max(0, o - p.pad);
            g.tiles = max(0, e - p.pad) - g.tile0;
            left -= e - o;
            o = 0;
            ++h;
            if (g.tiles > 0 && !ring_put(ring, n++, g, wc)) return;
        }
    }
    // the own part
    plan_own(a, cta, out);
    __syncwarp();
    int b = p.own_b, h = p.own_h, o = p.own_o, left = p.own_len, keys = 0;
    if (left > 0) keys = clamp_own(a, a.ctx_lens[b], p.P);
    g.flags = kOwn;
    g.pair = 0;
    while (left > 0) {
        const int span = tiles_of(keys) + kPad;
        const int e = min(span, o + left);
        g.keys = keys;
        g.b = b;
        g.kvh = h;
        g.tile0 = max(0, o - kPad);
        g.tiles = max(0, e - kPad) - g.tile0;
        left -= e - o;
        o = 0;
        if (left > 0 && ++h == a.Hkv) {
            h = 0;
            ++b;
            keys = clamp_own(a, a.ctx_lens[b], p.P);
        }
        if (g.tiles > 0 && !ring_put(ring, n++, g, wc)) return;
    }
    g.tiles = 0;
    ring_put(ring, n, g, wc);
}

// Two fp32 values in one 64-bit register: the FMA and the addition of both in one instruction.
__device__ __forceinline__ uint64_t f32x2(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void f32x2_split(uint64_t v, float& lo, float& hi) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t f32x2_fma(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t f32x2_add(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// The largest of three; NaN if any is (a NaN score has to reach the row's reference and so its output).
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// 2^y0 and 2^y1, y at most 126, without the special-function unit: adding 1.5 * 2^23 leaves n, the whole number
// next to y, in the low bits of the sum; f = y - n in [-1/2, 1/2] goes through the polynomial of degree 4 that is 1 at
// f = 0 and has the least largest relative error to 2^f besides (2.9e-6 with fp32 coefficients; 2.7e-6 without the
// condition), and n is added to the exponent.  The condition makes the end of the range exact: at y = -127 and below the
// sum of both exponents is the word 0, so that a score of -inf, of a masked key too, weighs nothing.  From -126 down to there
// the word is a denormal that is off by at most 2^-127.
__device__ __forceinline__ void exp2_poly(float& y0, float& y1) {
    constexpr float kMagic = 12582912.f;
    const uint64_t y = f32x2(fmaxf(y0, -127.f), fmaxf(y1, -127.f));
    const uint64_t t = f32x2_add(y, f32x2(kMagic, kMagic));
    const uint64_t f = f32x2_fma(f32x2_add(t, f32x2(-kMagic, -kMagic)), f32x2(-1.f, -1.f), y);
    uint64_t p = f32x2_fma(f, f32x2(0.009582852944731712f, 0.009582852944731712f), f32x2(0.055906426161527634f, 0.055906426161527634f));
    p = f32x2_fma(p, f, f32x2(0.24024099111557007f, 0.24024099111557007f));
    p = f32x2_fma(p, f, f32x2(0.6931241750717163f, 0.6931241750717163f));
    p = f32x2_fma(p, f, f32x2(1.f, 1.f));
    float t0, t1;
    f32x2_split(t, t0, t1);
    f32x2_split(p, y0, y1);
    y0 = __int_as_float(__float_as_int(y0) + (__float_as_int(t0) << 23));
    y1 = __int_as_float(__float_as_int(y1) + (__float_as_int(t1) << 23));
}

// Scales a row's O accumulators when its reference moves.  Rare: kept out of the way.
template <int D>
__device__ __noinline__ void scale_o(uint32_t tO, float factor) {
#pragma unroll 1
    for (int i = 0; i < D / 16; ++i) {
        uint32_t o[16];
        tmem_ld_x16(tO + 16 * i, o);
        tmem_wait_ld();
#pragma unroll
        for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * factor);
        tmem_st_x16(tO + 16 * i, o);
    }
    tmem_wait_st();
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
prefix_attn_split_kernel(const __grid_constant__ CUtensorMap tmKp, const __grid_constant__ CUtensorMap tmVp,
                         const __grid_constant__ CUtensorMap tmKo, const __grid_constant__ CUtensorMap tmVo,
                         const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ PrefixArgs a) {
    constexpr int NH = D / 64;
    constexpr int NK = k_slots(D), NV = v_slots(D);
    constexpr uint32_t TILE = tile_bytes(D);
    constexpr uint32_t OFF_Q = 0, OFF_K = 2 * TILE, OFF_V = OFF_K + NK * TILE;
    constexpr uint32_t TMEM_COLS = 512, COL_S = 0, COL_O = 256;  // stream s: S at COL_S + 128 s, O at COL_O + 128 s

    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t k_full[NK], k_empty[NK], v_full[NV], v_empty[NV];
    __shared__ uint64_t q_full[2], q_empty[2], s_full[2][2], p_full[2][2], o_rest[2][2], drain_bar[2];
    __shared__ uint32_t tmem_slot;
    __shared__ Ring ring;
    __shared__ int s_abort;
    __shared__ Plan plan;

    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem = smem_raw + (smem_base - smem_u32(smem_raw));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cta = blockIdx.x;

    if (threadIdx.x == 0) {
        for (int i = 0; i < NK; ++i) mbar_init(&k_full[i], 1), mbar_init(&k_empty[i], 2);
        for (int i = 0; i < NV; ++i) mbar_init(&v_full[i], 1), mbar_init(&v_empty[i], 2);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&q_full[i], 1);
            mbar_init(&q_empty[i], 2);
            for (int b = 0; b < 2; ++b) mbar_init(&s_full[i][b], 1), mbar_init(&p_full[i][b], 4), mbar_init(&o_rest[i][b], 1);
            mbar_init(&drain_bar[i], 1);
        }
        for (int i = 0; i < kRing; ++i) mbar_init(&ring.full[i], 1), mbar_init(&ring.empty[i], kRingUsers);
        fence_mbar_init();
        s_abort = 0;
    }
    if (warp == 8 && lane == 0) {
        prefetch_tensormap(&tmKp);
        prefetch_tensormap(&tmVp);
        prefetch_tensormap(&tmKo);
        prefetch_tensormap(&tmVo);
        prefetch_tensormap(&tmQ);
    }
    if (warp == 10) tmem_alloc(&tmem_slot, TMEM_COLS);  // the same warp frees it
    griddep_wait();  // lengths are read from here on
    griddep_launch_dependents();
    if (cta == 0 && threadIdx.x == 32) *a.plan_sig = 0;
    if (threadIdx.x == 0) plan_prefix(a, cta, plan);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = tmem_slot;
    const WaitCtx wc = {&s_abort, a.wait_limit};

    int r = 0;  // segments taken from the ring; a role that comes to the end marker stops
    // (a wait that runs out ends a role's work as well)
#define RAPID_SEG(i) ring.seg[(i) & (kRing - 1)]
    if (warp == 8) {
        // ---------------- producer: Q tiles (a ring of two) and K/V tiles ----------------
        int n_q = 0, n_k = 0, n_v = 0;  // tiles whose copies were issued
        bool ok = true;
        const int parts = kKeys / a.box_rows;
        const uint32_t part_bytes = kHalfBytes / parts;
        while (ok) {
            ok = warp_wait(&ring.full[r & (kRing - 1)], (r / kRing) & 1, wc);
            const Segment g = RAPID_SEG(r);
            if (!ok || g.tiles == 0) break;
            const bool own = g.flags & kOwn;
            const CUtensorMap* mk = own ? &tmKo : &tmKp;
            const CUtensorMap* mv = own ? &tmVo : &tmVp;
            const int row_tiles = g.flags & kDualRow ? 2 : 1;
            for (int i = 0; i < row_tiles; ++i) {
                const int s = n_q & 1;
                if (n_q >= 2) ok = warp_wait(&q_empty[s], (n_q / 2 - 1) & 1, wc);
                if (!ok) break;
                const int row0 = own ? g.b * a.R : (2 * g.pair + i) * a.rows_tile;
                if (elect_one()) {
                    mbar_arrive_expect_tx(&q_full[s], (uint32_t)a.rows_tile * a.G * D * 2);
#pragma unroll
                    for (int h = 0; h < NH; ++h)
                        tma_load_4d(smem + OFF_Q + s * TILE + h * kHalfBytes, &tmQ, &q_full[s], h * 64, g.kvh * a.G,
                                    row0, 0);
                }
                __syncwarp();
                ++n_q;
            }
            for (int t = 0; t < g.tiles && ok; ++t) {
                const int key0 = (g.tile0 + t) * kKeys;
                int c1[2] = {key0, 0}, c3[2] = {g.b, g.b};
                if (a.block_table) {
                    for (int q = 0; q < parts; ++q) {
                        const int in_unit = key0 + q * a.box_rows;
                        const int pos = in_unit + (own ? plan.P : 0);
                        c1[q] = pos & (a.block_size - 1);
                        if (in_unit >= g.keys) {
                            c3[q] = a.num_blocks;  // past the keys: zeros, no table entry is read
                            continue;
                        }
                        c3[q] = __ldg(a.block_table + (size_t)g.b * a.max_blocks + (pos >> a.block_log2));
                        if ((unsigned)c3[q] >= (unsigned)a.num_blocks) {
                            if (lane == 0) atomicOr(a.status, RAPID_STATUS_BAD_BLOCK_TABLE);
                            c3[q] = a.num_blocks;  // outside the pool: the copy reads zeros
                        }
                    }
                }
                const int ks = n_k % NK, vs = n_v % NV;
                if (n_k >= NK) ok = warp_wait(&k_empty[ks], (n_k / NK - 1) & 1, wc);
                if (!ok) break;
                if (elect_one()) {
                    mbar_arrive_expect_tx(&k_full[ks], TILE);
                    for (int q = 0; q < parts; ++q)
#pragma unroll
                        for (int h = 0; h < NH; ++h)
                            tma_load_4d(smem + OFF_K + ks * TILE + h * kHalfBytes + q * part_bytes, mk, &k_full[ks],
                                        h * 64, c1[q], g.kvh, c3[q]);
                }
                __syncwarp();
                ++n_k;
                if (n_v >= NV) ok = warp_wait(&v_empty[vs], (n_v / NV - 1) & 1, wc);
                if (!ok) break;
                if (elect_one()) {
                    mbar_arrive_expect_tx(&v_full[vs], TILE);
                    for (int q = 0; q < parts; ++q)
#pragma unroll
                        for (int h = 0; h < NH; ++h)
                            tma_load_4d(smem + OFF_V + vs * TILE + h * kHalfBytes + q * part_bytes, mv, &v_full[vs],
                                        h * 64, c1[q], g.kvh, c3[q]);
                }
                __syncwarp();
                ++n_v;
            }
            if (lane == 0) mbar_arrive(&ring.empty[r & (kRing - 1)]);
            __syncwarp();
            ++r;
        }
        // every copy lands before the CTA gives up its shared memory, whoever may have given up waiting for it
        for (int s = 0; s < 2 && s < n_q; ++s) mbar_wait_drain(&q_full[s], ((n_q - 1 - s) / 2) & 1);
        for (int s = 0; s < NK && s < n_k; ++s) mbar_wait_drain(&k_full[s], ((n_k - 1 - s) / NK) & 1);
        for (int s = 0; s < NV && s < n_v; ++s) mbar_wait_drain(&v_full[s], ((n_v - 1 - s) / NV) & 1);
    } else if (warp == 9) {
        // ---------------- the walk ----------------
        walk(a, plan, ring, cta, plan, wc);
    } else if (warp >= 10) {
        // ---------------- MMA issuers: a thread for each stream ----------------
        // It issues both products of its stream, because the tensor core works off a thread's instructions in
        // order: the QK^T that refills one half of S goes out behind the PV that reads P from it, with no wait
        // in between.  It runs up to two blocks ahead of PV.  One thread of the warp is here alone: what is called in this
        // branch is inlined, no function is.
        if (elect_one()) {
            constexpr uint32_t idesc_qk = umma_idesc_bf16(128, kBlock, 0, 0);
            constexpr uint32_t idesc_pv = umma_idesc_bf16(128, D, 0, 1);
            constexpr uint32_t BLOCK16 = kBlock * 128 >> 4;  // from a tile's first block of keys to its second, in descriptor units
            const int st = warp - 10;
            const uint32_t tS = tmem + COL_S + 128u * st, tO = tmem + COL_O + 128u * st;
            const uint64_t q_desc = umma_smem_desc(smem_base + OFF_Q, 16, 1024);
            const uint64_t k_desc = umma_smem_desc(smem_base + OFF_K, 16, 1024);
            const uint64_t v_desc = umma_smem_desc(smem_base + OFF_V, kHalfBytes, 1024);
            // QK^T side: segments begun, tiles left of the last and whether it is dual-row, block of the tile, block number, K slot
            int rq = 0, left_q = 0, dual_q = 0, h_q = 0, j_q = 0, ks = 0, k_par = 0;
            int n_q = 0, took_q = 0;  // Q tiles before the segment, and of it
            // PV side
            int left = 0, dual = 0, h = 0, j = 0, vs = 0, v_par = 0;
            uint64_t qd = 0;
            bool ended = false, fresh = true;
            while (true) {
                if (j_q < j + 2 && !ended) {
                    // (the next segment may not be there yet: wait for it only when nothing else is left to do)
                    if (left_q == 0 && (j == j_q || mbar_try_wait(&ring.full[rq & (kRing - 1)], (rq / kRing) & 1))) {
                        if (!mbar_wait_bounded(&ring.full[rq & (kRing - 1)], (rq / kRing) & 1, wc)) break;
                        left_q = RAPID_SEG(rq).tiles;
                        ended = left_q == 0;
                        if (!ended) {
                            dual_q = RAPID_SEG(rq).flags & kDualRow ? 1 : 0;
                            ++rq;
                            n_q += took_q;
                            took_q = 1 + dual_q;
                            const int n = n_q + (dual_q & st);
                            if (!mbar_wait_bounded(&q_full[n & 1], (n >> 1) & 1, wc)) break;
                            qd = q_desc + (uint32_t)(n & 1) * (TILE >> 4);
                        }
                    }
                    if (left_q > 0) {
                        if (h_q == 0 && !mbar_wait_bounded(&k_full[ks], k_par, wc)) break;
                        tc_fence_after_sync();
                        const uint64_t kd = k_desc + (uint32_t)ks * (TILE >> 4) + (uint32_t)(dual_q ? h_q : st) * BLOCK16;
                        const uint32_t d = tS + kBlock * (j_q & 1);
#pragma unroll
                        for (int kk = 0; kk < D / 16; ++kk) {
                            const uint32_t off = (kk >> 2) * (kHalfBytes >> 4) + (kk & 3) * 2;
                            umma_bf16_ss(d, qd + off, kd + off, idesc_qk, kk > 0);
                        }
                        umma_commit(&s_full[st][j_q & 1]);
                        ++j_q;
                        if (h_q == dual_q) {
                            umma_commit(&k_empty[ks]);
                            h_q = 0;
                            if (++ks == NK) ks = 0, k_par ^= 1;
                            if (--left_q == 0) {
                                umma_commit(&q_empty[(n_q + (dual_q & st)) & 1]);
                                if (dual_q) {  // the other stream's row tile: given up for this stream too, once it is there
                                    const int n = n_q + 1 - st;
                                    if (!mbar_wait_bounded(&q_full[n & 1], (n >> 1) & 1, wc)) break;
                                    mbar_arrive(&q_empty[n & 1]);
                                }
                            }
                        } else {
                            h_q = 1;
                        }
                        if (j_q < j + 2) continue;
                    }
                }
                if (j == j_q) {
                    if (ended) break;
                    continue;
                }
                if (left == 0) {  // (the segment is there: its first QK^T went out)
                    left = RAPID_SEG(r).tiles;
                    dual = RAPID_SEG(r).flags & kDualRow ? 1 : 0;
                    fresh = true;
                }
                if (h == 0 && !mbar_wait_bounded(&v_full[vs], v_par, wc)) break;
                if (!mbar_wait_bounded(&p_full[st][j & 1], (j >> 1) & 1, wc)) break;
                tc_fence_after_sync();
                const uint64_t vd = v_desc + (uint32_t)vs * (TILE >> 4) + (uint32_t)(dual ? h : st) * BLOCK16;
                const uint32_t pm = tS + kBlock * (j & 1);
#pragma unroll
                for (int kk = 0; kk < kBlock / 16; ++kk)
                    umma_bf16_ts(tO, pm + 8 * kk, vd + kk * (2048 >> 4), idesc_pv, (!fresh || kk > 0) ? 1u : 0u);
                fresh = false;
                umma_commit(&o_rest[st][j & 1]);
                ++j;
                if (h == dual) {
                    umma_commit(&v_empty[vs]);
                    h = 0;
                    if (++vs == NV) vs = 0, v_par ^= 1;
                    if (--left == 0) mbar_arrive(&ring.empty[r++ & (kRing - 1)]);
                } else {
                    h = 1;
                }
            }
            // every MMA issued here has completed before tensor memory is freed
            umma_commit(&drain_bar[st]);
            const long long t0 = clock64();
            while (!mbar_try_wait(&drain_bar[st], 0) && clock64() - t0 < kWaitCycleLimit) {}
        }
        __syncwarp();
    } else {
        // ---------------- softmax warps: stream = warp / 4, row of the tile = 32 (warp % 4) + lane ----------------
        const int stream = warp >> 2;
        const int row = (warp & 3) * 32 + lane;
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tO = tmem + lane_base + COL_O + 128u * stream;
        const float c = a.scale_log2;
        int n = 0, j = 0;  // tiles of the CTA before the segment, blocks of this stream so far
        bool ok = true;
        while (true) {
            ok = warp_wait(&ring.full[r & (kRing - 1)], (r / kRing) & 1, wc);
            const Segment g = RAPID_SEG(r);
            if (!ok || g.tiles == 0) break;
            const bool own = g.flags & kOwn;
            const int dual = g.flags & kDualRow ? 1 : 0, blocks = g.tiles << dual;
            // the tile's rows: (sequence, row, head in group) of the batch, or (row, head) of one sequence
            const int tile_row0 = (2 * g.pair + (dual ? stream : 0)) * a.rows_tile;
            const int rows = own ? a.GR : min(a.rows_tile, a.B * a.R - tile_row0) * a.G;
            const bool row_valid = row < rows;
            const bool warp_active = (warp & 3) * 32 < rows;
            // keys a row sees: all of the prefix; its own sequence's up to itself
            const int lim = own ? g.keys - a.R + row / a.G : g.keys - 1;
            const int all_see = own ? g.keys - a.R : g.keys - 1;
            float m_ref = -INFINITY, l_run = 0.f;
            for (int u = 0; u < blocks; ++u, ++j) {
                const int t = u >> dual, kb = dual ? u & 1 : stream;  // the block's tile, and which half of its keys
                const uint32_t tS = tmem + lane_base + COL_S + 128u * stream + kBlock * (j & 1);
                ok = warp_wait(&s_full[stream][j & 1], (j >> 1) & 1, wc);
                if (!ok) break;
                const int key0 = (g.tile0 + t) * kKeys + kBlock * kb;
                if (warp_active) {
                    tc_fence_after_sync();
                    uint32_t x[kBlock];
                    tmem_ld_x32(tS, reinterpret_cast<uint32_t(&)[32]>(x[0]));
                    tmem_ld_x32(tS + 32, reinterpret_cast<uint32_t(&)[32]>(x[32]));
                    tmem_wait_ld();
                    if (key0 + kBlock - 1 > all_see) {
#pragma unroll
                        for (int k = 0; k < kBlock; ++k)
                            if (key0 + k > lim) x[k] = __float_as_uint(-INFINITY);
                    }
                    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int k = 0; k < kBlock; k += 2)
                        mx[(k >> 1) & 3] = max3(mx[(k >> 1) & 3], __uint_as_float(x[k]), __uint_as_float(x[k + 1]));
                    const float top = ceilf(max3(max3(mx[0], mx[1], mx[2]), mx[3], mx[3]) * c);
                    // no reference yet, or scores that outgrow it
                    const bool move = row_valid && !(top <= m_ref + kJump) && top != -INFINITY;
                    if (__any_sync(0xffffffffu, move)) {
                        const float factor = move ? fast_exp2(m_ref - top) : 1.f;  // 0 when there was no reference
                        if (move) {
                            l_run *= factor;
                            m_ref = top;
                        }
                        if (u > 0) {  // O at rest: the PV of the stream's latest block has completed
                            ok = warp_wait(&o_rest[stream][(j - 1) & 1], ((j - 1) >> 1) & 1, wc);
                            if (!ok) break;
                            tc_fence_after_sync();
                            scale_o<D>(tO, factor);
                        }
                    }
                    const float m_use = m_ref == -INFINITY ? 0.f : m_ref;
                    const uint64_t c2 = f32x2(c, c), m2 = f32x2(-m_use, -m_use);
                    uint64_t acc[2] = {0, 0};
                    uint32_t pk[kBlock / 2];
#pragma unroll
                    for (int k = 0; k < kBlock; k += 2) {
                        float p0, p1;
                        f32x2_split(f32x2_fma(f32x2(__uint_as_float(x[k]), __uint_as_float(x[k + 1])), c2, m2), p0, p1);
                        if ((k >> 1) % 8 < kPoly) {
                            exp2_poly(p0, p1);
                        } else {
                            p0 = fast_exp2(p0);
                            p1 = fast_exp2(p1);
                        }
                        acc[(k >> 1) & 1] = f32x2_add(acc[(k >> 1) & 1], f32x2(p0, p1));
                        pk[k >> 1] = pack_bf16x2(p0, p1);
                    }
                    tmem_st_x32(tS, pk);
                    float s0, s1;
                    f32x2_split(f32x2_add(acc[0], acc[1]), s0, s1);
                    l_run += s0 + s1;
                }
                if (key0 + kBlock > g.keys) {
                    // V rows past the keys may hold any bits: zero them so that 0 * row = 0
                    const int vs = (n + t) % NV;
                    ok = warp_wait(&v_full[vs], ((n + t) / NV) & 1, wc);
                    if (!ok) break;
                    const int bad = max(0, g.keys - key0);
                    const int chunks = (kBlock - bad) * 8;
#pragma unroll
                    for (int h = 0; h < NH; ++h)
                        for (int ch = row; ch < chunks; ch += 128)
                            *reinterpret_cast<uint4*>(smem + OFF_V + vs * TILE + h * kHalfBytes + (kBlock * kb + bad) * 128 + ch * 16) =
                                make_uint4(0, 0, 0, 0);
                    fence_proxy_async_smem();
                }
                tmem_wait_st();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_full[stream][j & 1]);
            }
            if (!ok) break;

            // ---- end of the segment: the partial of this stream ----
            const int unit = g.b * a.Hkv + g.kvh;
            const int slot_rows = own ? a.GR : 128;
            float* slot = own ? a.part_own + (size_t)((plan.worker + unit) * 2 + stream) * slot_floats(a.GR, D)
                                : a.part_prefix + (size_t)((plan.team + g.kvh) * 2 * a.np + 2 * g.pair + stream) * slot_floats(128, D);
            ok = warp_wait(&o_rest[stream][(j - 1) & 1], ((j - 1) >> 1) & 1, wc);
            if (!ok) break;
            if (warp_active) {
                tc_fence_after_sync();
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    uint32_t o[32];
                    tmem_ld_x32(tO + 32 * i, o);
                    tmem_wait_ld();
                    if (row_valid) {
#pragma unroll
                        for (int k = 0; k < 32; k += 4)
                            *reinterpret_cast<uint4*>(slot + ((size_t)(8 * i + k / 4) * slot_rows + row) * 4) =
                                make_uint4(o[k], o[k + 1], o[k + 2], o[k + 3]);
                    }
                }
                tc_fence_before_sync();
                if (row_valid) {
                    slot[(size_t)slot_rows * D + row] = m_ref;
                    slot[(size_t)slot_rows * (D + 1) + row] = l_run;
                }
            }
            // which workers hold tiles of a unit, for the merge
            if (threadIdx.x == 0) {
                int2* range = own ? a.own_range + unit : a.prefix_range + g.kvh;
                const int who = own ? plan.worker : plan.team;
                if (own || g.pair == 0) {
                    if (g.tile0 == 0) range->x = who;
                    if (g.tile0 + g.tiles == tiles_of(g.keys)) range->y = who;
                }
            }
            n += g.tiles;
            __syncwarp();
            if (lane == 0) mbar_arrive(&ring.empty[r & (kRing - 1)]);
            ++r;
        }
    }

#undef RAPID_SEG

    tc_fence_before_sync();
    __syncthreads();
    if (warp == 10) {
        tc_fence_after_sync();
        tmem_dealloc(tmem, TMEM_COLS);
    }
    if (threadIdx.x == 0 && s_abort) atomicOr(a.status, RAPID_STATUS_PIPELINE_TIMEOUT);
}

// Merge: out = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s over the partials of a row: those of the prefix
// (one per team whose range touches the KV head) and those of the row's own sequence.  A block takes 32
// rows of a KV head (lane = row: slots are stored so that this reads whole lines) and 16 columns; its warps
// take the slots w, w + W, ... each, all loads of four slots in flight at once, and meet in shared memory.
// Latency is what counts here (the call's partials are up to some 20 MB, in L2): one round trip for the ranges, one or
// two for the slots (6 - 18 us with events around it; the launch and its first reads overlap the split kernel's end).
// The order of the sums is fixed: results do not depend on timing.
template <int D, int W>
__global__ void __launch_bounds__(32 * W)
prefix_attn_merge_kernel(const __grid_constant__ PrefixArgs a, __nv_bfloat16* out, float* lse_out, float* out_f32) {
    constexpr int UN = 4;
    __shared__ float4 sh_acc[W][4][32];
    __shared__ float sh_m[W][32], sh_l[W][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int kvh = blockIdx.y;
    const int total_rows = a.B * a.R * a.G;
    const int row0 = blockIdx.x * 32;
    const int flat = min(row0 + lane, total_rows - 1);  // past the end: the last row again, not written
    const int f = flat / a.G, gh = flat - f * a.G;      // (sequence, row), head in group
    const int b = f / a.R, i = f - b * a.R;
    const int rt = f / a.rows_tile;
    const int prow = (f - rt * a.rows_tile) * a.G + gh;
    const int pair = rt >> 1;
    const bool dual = 2 * pair + 1 < a.nrt;
    const int orow = i * a.G + gh;
    const int unit = b * a.Hkv + kvh;
    const int sp = (int)slot_floats(128, D), so = (int)slot_floats(a.GR, D);

    griddep_wait();
    griddep_launch_dependents();
    const int given = *a.prefix_len;
    int2 pr = __ldcg(a.prefix_range + kvh), orr = __ldcg(a.own_range + unit);
    // (a split kernel whose waits ran out may not have written them: whatever they hold, stay inside the slots)
    if (clamp_prefix(a, given) == 0 || pr.x < 0 || pr.y >= a.max_teams) pr = make_int2(0, -1);
    if (orr.x < 0 || orr.y >= a.num_ctas) orr = make_int2(0, -1);
    // The row's slots as one list: the first n_p in the prefix part (one per team, or two where a single row tile's
    // keys went to both streams), the rest in the own part (two per worker).
    const int n_p = max(0, pr.y - pr.x + 1) << (dual ? 0 : 1), n_all = n_p + max(0, orr.y - orr.x + 1) * 2;
    const float* pbase = a.part_prefix + (size_t)((pr.x + kvh) * 2 * a.np + (dual ? rt : 2 * pair)) * sp;
    const float* obase = a.part_own + (size_t)(orr.x + unit) * 2 * so;
    const int d4 = blockIdx.z * 4;

    float m = -INFINITY, l = 0.f;
    float4 acc[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int x0 = warp; x0 < n_all; x0 += W * UN) {
        float ms[UN], ls[UN];
        float4 o[UN][4];
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            const int x = x0 + W * u;
            ms[u] = -INFINITY;
            if (x < n_all) {
                const bool pre = x < n_p;
                const int rows = pre ? 128 : a.GR, r = pre ? prow : orow;
                const float* s = pre ? (dual ? pbase + (size_t)x * 2 * a.np * sp : pbase + ((size_t)(x >> 1) * 2 * a.np + (x & 1)) * sp)
                                     : obase + (size_t)(x - n_p) * so;
                ms[u] = __ldcg(s + rows * D + r);
                ls[u] = __ldcg(s + rows * (D + 1) + r);
#pragma unroll
                for (int j = 0; j < 4; ++j) o[u][j] = __ldcg(reinterpret_cast<const float4*>(s) + (d4 + j) * rows + r);
            }
        }
        float top = m;
#pragma unroll
        for (int u = 0; u < UN; ++u) top = max3(top, ms[u], ms[u]);
        const float keep = m == -INFINITY ? 0.f : exp2f(m - top);
        m = top;
        l *= keep;
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j].x *= keep, acc[j].y *= keep, acc[j].z *= keep, acc[j].w *= keep;
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            if (ms[u] == -INFINITY) continue;  // an untouched slot holds neither a sum nor an O row: its bits are not used
            const float wgt = exp2f(ms[u] - top);
            l += wgt * ls[u];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                acc[j].x += wgt * o[u][j].x;
                acc[j].y += wgt * o[u][j].y;
                acc[j].z += wgt * o[u][j].z;
                acc[j].w += wgt * o[u][j].w;
            }
        }
    }
    sh_m[warp][lane] = m;
    sh_l[warp][lane] = l;
#pragma unroll
    for (int j = 0; j < 4; ++j) sh_acc[warp][j][lane] = acc[j];
    __syncthreads();
    // four neighbouring threads write the 16 columns of a row
    for (int t = threadIdx.x; t < 128; t += 32 * W) {
        const int row = t >> 2, j = t & 3;
        if (row0 + row >= total_rows) return;
        float M = -INFINITY, L = 0.f;
#pragma unroll
        for (int k = 0; k < W; ++k) M = max3(M, sh_m[k][row], sh_m[k][row]);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < W; ++k) {
            if (sh_m[k][row] == -INFINITY) continue;
            const float wgt = exp2f(sh_m[k][row] - M);
            const float4 o = sh_acc[k][j][row];
            L += wgt * sh_l[k][row];
            v.x += wgt * o.x;
            v.y += wgt * o.y;
            v.z += wgt * o.z;
            v.w += wgt * o.w;
        }
        const int fo = (row0 + row) / a.G, go = row0 + row - fo * a.G;
        const size_t at = (size_t)fo * a.Hq + (size_t)kvh * a.G + go;
        const float inv = 1.f / L;
        v = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
        *reinterpret_cast<uint2*>(out + at * D + (d4 + j) * 4) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
        if (out_f32) *reinterpret_cast<float4*>(out_f32 + at * D + (d4 + j) * 4) = v;
        if (lse_out && d4 + j == 0) lse_out[at] = (M + log2f(L)) * 0.69314718055994530942f;
    }
}

// ---- host side ----------------------------------------------------------------------------

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
    static const EncodeTiledFn fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<EncodeTiledFn>(p);
    }();
    return fn;
}

// 4-D bf16 map of 64-column boxes: dims (D, d1, d2, d3), element strides s1..s3, a box of (64, b1, b2, 1).
int make_map(CUtensorMap* map, const void* base, int D, int64_t d1, int64_t d2, int64_t d3, int64_t s1, int64_t s2,
             int64_t s3, int b1, int b2) {
    const EncodeTiledFn enc = encode_fn();
    if (!enc) {
        set_error("cuTensorMapEncodeTiled is not available from the CUDA driver");
        return RAPID_ERR_CUDA;
    }
    const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)d1, (cuuint64_t)d2, (cuuint64_t)d3};
    const cuuint64_t strides[3] = {(cuuint64_t)s1 * 2, (cuuint64_t)s2 * 2, (cuuint64_t)s3 * 2};
    const cuuint32_t box[4] = {64, (cuuint32_t)b1, (cuuint32_t)b2, 1}, estr[4] = {1, 1, 1, 1};
    const CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, estr,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        set_error("cuTensorMapEncodeTiled failed with CUresult %d", (int)r);
        return RAPID_ERR_CUDA;
    }
    return RAPID_OK;
}

// Scratch.  A caller may use the same workspace for rapid_attention_plan and the calls that follow that plan, whose CTAs and
// slots are then addressed by what lies behind the signature at the start of it; what is written here would be taken for
// them.  So the signature's place is kept free of scratch, and every call takes the plan back by its first word (a batch
// size, never 0): a call that still names the plan finds it stale.
struct WsLayout {
    size_t plan_sig, prefix_range, own_range, part_prefix, part_own, total;
};
WsLayout ws_layout(int B, int Hkv, int GR, int np, int D) {
    WsLayout l;
    size_t off = kWorkspaceHeaderBytes;
    l.plan_sig = off;
    off += 256;
    l.prefix_range = off;
    off += align_up((size_t)Hkv * sizeof(int2), 256);
    l.own_range = off;
    off += align_up((size_t)B * Hkv * sizeof(int2), 256);
    l.part_prefix = off;
    // (team + KV head) * 2 np + ...: teams * np is at most the grid, or np where one team has several rounds
    const size_t team_slots = 2 * ((size_t)(np > kMaxPrefixCtas ? np : kMaxPrefixCtas) + (size_t)Hkv * np);
    off += align_up(team_slots * slot_floats(128, D) * sizeof(float), 256);
    l.part_own = off;
    off += (size_t)2 * (kMaxPrefixCtas + (size_t)B * Hkv) * slot_floats(GR, D) * sizeof(float);
    l.total = off;
    return l;
}

bool shape_ok(const rapid_attn_shape* s, int gamma) {
    return s && s->B > 0 && s->Hq > 0 && s->Hkv > 0 && gamma >= 0 && s->Hq % s->Hkv == 0 &&
           (s->D == 64 || s->D == 128) && (int64_t)(s->Hq / s->Hkv) * (gamma + 1) <= 128 &&
           (int64_t)s->B * s->Hkv <= 65535 && (int64_t)s->B * (gamma + 1) <= (1 << 24);
}

template <int D>
int launch(const CUtensorMap (&tm)[5], const PrefixArgs& a, __nv_bfloat16* out, float* lse, float* out_f32,
           void* split_done, cudaStream_t stream) {
    constexpr int smem = smem_bytes(D);
    static_assert(smem <= 232448 - 1024, "shared memory (dynamic + static)");
    int dev = 0;
    RAPID_CUDA_CHECK(cudaGetDevice(&dev));
    static std::atomic<bool> configured[64];  // (first calls may come from several threads at once; all set the same)
    if (dev >= 64 || !configured[dev]) {
        RAPID_CUDA_CHECK(cudaFuncSetAttribute(prefix_attn_split_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        if (dev < 64) configured[dev] = true;
    }
    RAPID_CUDA_CHECK(launch_dependent(prefix_attn_split_kernel<D>, dim3(a.num_ctas), dim3(kThreads), (size_t)smem, stream,
                                      tm[0], tm[1], tm[2], tm[3], tm[4], a));
    if (split_done) RAPID_CUDA_CHECK(cudaEventRecord(static_cast<cudaEvent_t>(split_done), stream));
    const int rows = a.B * a.R * a.G;
    // Few blocks have eight warps, so that a row's slots are all in flight at once; many have two, so that those of more rows
    // are (a row has two to ten slots then).  Whole calls with 8 / 4 / 2 warps, us: 192 blocks 69.4 / 72.2 / 73.1,
    // 320 blocks 16.4 / 15.2 / 16.4, 512 148.5 / 147.7 / 149.0, 1,152 90.4 / 87.2 / 85.1, 1,264 27.2 / 23.7 / 22.2,
    // 2,304 175.1 / 170.3 / 169.2, 4,864 85.8 / 69.4 / 61.6.
    int sms = 0;
    RAPID_CUDA_CHECK(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    const dim3 grid((rows + 31) / 32, a.Hkv, D / 16);
    const int64_t blocks = (int64_t)grid.x * grid.y * grid.z;
    if (2 * blocks <= 3 * sms)
        RAPID_CUDA_CHECK(launch_dependent(prefix_attn_merge_kernel<D, 8>, grid, dim3(256), 0, stream, a, out, lse, out_f32));
    else if (blocks <= 8 * sms)
        RAPID_CUDA_CHECK(launch_dependent(prefix_attn_merge_kernel<D, 4>, grid, dim3(128), 0, stream, a, out, lse, out_f32));
    else
        RAPID_CUDA_CHECK(launch_dependent(prefix_attn_merge_kernel<D, 2>, grid, dim3(64), 0, stream, a, out, lse, out_f32));
    count_launch(2);
    return RAPID_OK;
}

}  // namespace

size_t prefix_attention_workspace_bytes(const rapid_attn_shape* s, int gamma) {
    if (!shape_ok(s, gamma)) return 0;
    const int G = s->Hq / s->Hkv, R = gamma + 1;
    const int rows_tile = 128 / G;
    const int nrt = (s->B * R + rows_tile - 1) / rows_tile;
    return ws_layout(s->B, s->Hkv, G * R, (nrt + 1) / 2, s->D).total;
}

int launch_verify_attention_prefix(const void* q, const void* k_prefix, const void* v_prefix,
                                   const rapid_prefix_kv* prefix, const int32_t* prefix_len, const void* k_cache,
                                   const void* v_cache, const rapid_paged_kv* paged, const int32_t* block_table,
                                   const int32_t* ctx_lens, int gamma, void* out, const rapid_attn_shape* shape,
                                   const rapid_attn_params* params, void* workspace, size_t workspace_bytes,
                                   cudaStream_t stream) {
    const char* who = paged ? "rapid_verify_attention_prefix_paged" : "rapid_verify_attention_prefix";
    if (!q || !k_cache || !v_cache || !prefix_len || !ctx_lens || !out || !shape || (paged && !block_table) ||
        (!paged && (!k_prefix || !v_prefix || !prefix))) {
        set_error("%s: NULL argument", who);
        return RAPID_ERR_INVALID_ARG;
    }
    const rapid_attn_shape& s = *shape;
    if (s.B <= 0 || s.Hq <= 0 || s.Hkv <= 0 || s.Lmax <= 0 || gamma < 0 || s.Hq % s.Hkv) {
        set_error("%s: invalid shape (B=%d Hq=%d Hkv=%d Lmax=%lld gamma=%d)", who, s.B, s.Hq, s.Hkv, (long long)s.Lmax,
                  gamma);
        return RAPID_ERR_INVALID_ARG;
    }
    if (!shape_ok(shape, gamma)) {
        set_error("%s: head_dim must be 64 or 128, (Hq/Hkv) * (gamma+1) at most 128, B * Hkv at most 65535 and "
                  "B * (gamma+1) at most 2^24", who);
        return RAPID_ERR_UNSUPPORTED;
    }
    const int R = gamma + 1, G = s.Hq / s.Hkv;
    if (params && (params->all_keys_visible || params->kernel || params->sink_keys || params->window_keys ||
                   params->plan || params->kv_fp8 || params->kv_settled)) {
        set_error("%s: of params only scale, num_ctas, lse_out, out_f32, split_done_event and wait_cycle_limit apply", who);
        return RAPID_ERR_UNSUPPORTED;
    }
    int64_t sl, sh, sb, keys, outer, psl = 0, psh = 0, pmax;
    int block_log2 = 0;
    if (paged) {
        const int64_t bs = paged->block_size;
        if (bs < 64 || (bs & (bs - 1)) || paged->num_blocks <= 0 || paged->max_blocks_per_seq <= 0) {
            set_error("%s: block_size must be a power of two >= 64, num_blocks and max_blocks_per_seq positive", who);
            return RAPID_ERR_UNSUPPORTED;
        }
        if (s.Lmax != (int64_t)paged->max_blocks_per_seq * bs) {
            set_error("%s: shape->Lmax must equal max_blocks_per_seq * block_size", who);
            return RAPID_ERR_INVALID_ARG;
        }
        while ((1LL << block_log2) < bs) ++block_log2;
        sl = paged->stride_l ? paged->stride_l : s.D;
        sh = paged->stride_h ? paged->stride_h : bs * sl;
        sb = paged->stride_block ? paged->stride_block : s.Hkv * sh;
        keys = bs;
        outer = paged->num_blocks;
        pmax = s.Lmax;
    } else {
        sl = s.kv_stride_l ? s.kv_stride_l : s.D;
        sh = s.kv_stride_h ? s.kv_stride_h : s.Lmax * sl;
        sb = s.kv_stride_b ? s.kv_stride_b : s.Hkv * sh;
        keys = s.Lmax;
        outer = s.B;
        pmax = prefix->Pmax;
        psl = prefix->stride_l ? prefix->stride_l : s.D;
        psh = prefix->stride_h ? prefix->stride_h : prefix->Pmax * psl;
        if (pmax <= 0 || pmax > 0x7fffffffLL - 256) {
            set_error("%s: Pmax %lld out of range", who, (long long)pmax);
            return RAPID_ERR_INVALID_ARG;
        }
        if (psl < s.D || psl % 8 || psh % 8 || psh <= 0) {
            set_error("%s: prefix strides must be positive multiples of 8 elements", who);
            return RAPID_ERR_UNSUPPORTED;
        }
    }
    if (s.Lmax < R || s.Lmax > 0x7fffffffLL - 256) {
        set_error("%s: Lmax %lld out of range", who, (long long)s.Lmax);
        return RAPID_ERR_INVALID_ARG;
    }
    // the padded tile lists are counted in 32 bits, a prefix tile once for every row tile
    const int rows_tile = 128 / G;
    const int64_t nrt = ((int64_t)s.B * R + rows_tile - 1) / rows_tile;
    if ((int64_t)s.B * s.Hkv * (s.Lmax / kKeys + 1 + kPad) > 0x3fffffffLL ||
        (int64_t)s.Hkv * (pmax / kKeys + 1 + kPad) * (nrt + 1) > 0x3fffffffLL) {
        set_error("%s: too many key tiles in one call", who);
        return RAPID_ERR_UNSUPPORTED;
    }
    if (sl < s.D || sl % 8 || sh % 8 || sb % 8 || sh <= 0 || sb <= 0) {
        set_error("%s: K/V strides must be positive multiples of 8 elements", who);
        return RAPID_ERR_UNSUPPORTED;
    }
    if (((uintptr_t)k_cache | (uintptr_t)v_cache | (uintptr_t)q | (uintptr_t)out |
         (paged ? 0 : (uintptr_t)k_prefix | (uintptr_t)v_prefix)) & 15) {
        set_error("%s: q, out and the caches must be 16-byte aligned", who);
        return RAPID_ERR_UNSUPPORTED;
    }
    if (params && params->out_f32 && ((uintptr_t)params->out_f32 & 15)) {
        set_error("%s: out_f32 must be 16-byte aligned", who);
        return RAPID_ERR_UNSUPPORTED;
    }
    const int np = (int)((nrt + 1) / 2);
    const WsLayout lay = ws_layout(s.B, s.Hkv, G * R, np, s.D);
    if (!workspace || workspace_bytes < lay.total || ((uintptr_t)workspace & 255)) {
        set_error("%s: workspace of %zu bytes needed (256-byte aligned), got %zu", who, lay.total, workspace_bytes);
        return RAPID_ERR_WORKSPACE;
    }
    int num_ctas = params ? params->num_ctas : 0;
    if (num_ctas < 0 || num_ctas > kMaxPrefixCtas) {
        set_error("%s: num_ctas %d outside [0, %d]", who, num_ctas, kMaxPrefixCtas);
        return RAPID_ERR_INVALID_ARG;
    }
    if (!num_ctas) {
        int dev = 0;
        RAPID_CUDA_CHECK(cudaGetDevice(&dev));
        RAPID_CUDA_CHECK(cudaDeviceGetAttribute(&num_ctas, cudaDevAttrMultiProcessorCount, dev));
        if (num_ctas > kMaxPrefixCtas) num_ctas = kMaxPrefixCtas;
    }
    const float scale = params && params->scale != 0.f ? params->scale : 1.0f / sqrtf((float)s.D);
    if (!(scale > 0.f) || !isfinite(scale)) {
        set_error("%s: scale must be positive and finite", who);
        return RAPID_ERR_INVALID_ARG;
    }
    const long long wait_limit = params && params->wait_cycle_limit ? params->wait_cycle_limit : kWaitCycleLimit;
    if (wait_limit < 0) {
        set_error("%s: wait_cycle_limit must not be negative", who);
        return RAPID_ERR_INVALID_ARG;
    }

    uint8_t* ws = static_cast<uint8_t*>(workspace);
    PrefixArgs a = {};
    a.ctx_lens = ctx_lens;
    a.prefix_len = prefix_len;
    a.block_table = paged ? block_table : nullptr;
    a.part_prefix = reinterpret_cast<float*>(ws + lay.part_prefix);
    a.part_own = reinterpret_cast<float*>(ws + lay.part_own);
    a.prefix_range = reinterpret_cast<int2*>(ws + lay.prefix_range);
    a.own_range = reinterpret_cast<int2*>(ws + lay.own_range);
    a.status = reinterpret_cast<int32_t*>(ws);
    a.plan_sig = reinterpret_cast<int32_t*>(ws + lay.plan_sig);
    a.B = s.B;
    a.R = R;
    a.G = G;
    a.Hq = s.Hq;
    a.Hkv = s.Hkv;
    a.GR = G * R;
    a.Pmax = (int)pmax;
    a.Lmax = (int)s.Lmax;
    a.block_size = paged ? paged->block_size : 0;
    a.block_log2 = block_log2;
    a.num_blocks = paged ? paged->num_blocks : 0;
    a.max_blocks = paged ? paged->max_blocks_per_seq : 0;
    a.box_rows = paged && paged->block_size < kKeys ? 64 : kKeys;
    a.rows_tile = rows_tile;
    a.nrt = (int)nrt;
    a.np = np;
    a.num_ctas = num_ctas;
    a.team_ctas = np < num_ctas ? np : num_ctas;
    a.max_teams = num_ctas / a.team_ctas;
    a.rounds = (np + num_ctas - 1) / num_ctas;
    a.row_cost = (nrt > 1 ? 2 : 1) * a.rounds;
    a.scale_log2 = scale * 1.4426950408889634f;
    a.wait_limit = wait_limit;

    CUtensorMap tm[5];
    int rc;
    if ((rc = make_map(&tm[2], k_cache, s.D, keys, s.Hkv, outer, sl, sh, sb, a.box_rows, 1)) != RAPID_OK) return rc;
    if ((rc = make_map(&tm[3], v_cache, s.D, keys, s.Hkv, outer, sl, sh, sb, a.box_rows, 1)) != RAPID_OK) return rc;
    if (paged) {  // the prefix lies in the same pools
        tm[0] = tm[2];
        tm[1] = tm[3];
    } else {
        const int64_t psb = psh * s.Hkv;  // (one prefix: its outermost coordinate is always 0)
        if ((rc = make_map(&tm[0], k_prefix, s.D, pmax, s.Hkv, 1, psl, psh, psb, kKeys, 1)) != RAPID_OK) return rc;
        if ((rc = make_map(&tm[1], v_prefix, s.D, pmax, s.Hkv, 1, psl, psh, psb, kKeys, 1)) != RAPID_OK) return rc;
    }
    // q [B, R, Hq, D] as [B*R, Hq, D]: a box of (64 columns, G heads, rows_tile rows) is a row tile, row index r*G + g
    if ((rc = make_map(&tm[4], q, s.D, s.Hq, (int64_t)s.B * R, 1, s.D, (int64_t)s.Hq * s.D, (int64_t)s.B * R * s.Hq * s.D, G,
                       rows_tile)) != RAPID_OK)
        return rc;
    __nv_bfloat16* o = static_cast<__nv_bfloat16*>(out);
    float* lse = params ? params->lse_out : nullptr;
    float* o32 = params ? params->out_f32 : nullptr;
    void* ev = params ? params->split_done_event : nullptr;
    return s.D == 128 ? launch<128>(tm, a, o, lse, o32, ev, stream) : launch<64>(tm, a, o, lse, o32, ev, stream);
}

}  // namespace rapid
