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
// Segments.  A CTA works through segments: a run of 128-key tiles of one unit.
//   dual-row segment  prefix of one KV head, two row tiles: stream s (one of two groups of four softmax warps,
//                     with its own S and O accumulators) takes row tile s through every key tile;
//   dual-key segment  one row tile (the last prefix tile of an odd count, or the R*G rows of one sequence over
//                     its own keys): the streams take alternate key tiles of the CTA, each with a partial
//                     of its own, so that segments of a single tile alternate between them as well.
//
//   S_s[128 x 128] = Q_s K^T      A = Q tile, B = K tile, both K-major in shared memory
//   O_s[128 x D]  += P_s V        A = P (bf16, over the first half of S_s's columns), B = V tile, MN-major
//
// Work split (make_plan, one warp of every CTA: no plan kernel, no plan to go stale).  Cost is counted in
// single-stream tiles: 2 for a dual-row tile, 1 for a dual-key tile, kPad for changing to another unit.
// With np pairs of row tiles the prefix is cut into T equal ranges of key tiles, each for a team of np CTAs,
// one pair each: a team reads the same K/V tiles at the same time, so they leave HBM once.  T is the
// share of the machine that the prefix is of the whole work; the sequences' own tiles fill up every CTA
// to the same level (CTAs outside the teams first, then those with a single row tile, then all).
//
// Bound: up to 256 rows per KV head (one pair) a K/V tile of 64 KB is read for every 256 x 128 scores, and HBM
// is the limit; from two pairs on the tensor cores and the exponentials are.
//
// Waits are bounded as everywhere in this library; see mbar_wait_bounded.  Every mbarrier here is one
// whose next phase cannot complete before all its waiters have passed the current one.
#include <math.h>

#include "common.cuh"
#include "tcgen05.cuh"

namespace rapid {

namespace {

constexpr int kKeys = 128;             // keys per tile
constexpr int kThreads = 384;          // two softmax groups of 128, then K/V producer, Q producer, QK^T, PV warps
constexpr int kHalfBytes = kKeys * 128;  // one 64-column half of a tile of 128 rows
constexpr int kPad = 3;                // single-stream tiles that a change of unit costs
constexpr int kMaxPrefixCtas = 256;
constexpr float kJump = 8.f;           // a maximum this far (log2) above a row's reference moves the reference

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
    int B, R, G, Hq, Hkv, GR;
    int Pmax, Lmax;              // capacities in keys (paged: both the capacity of a table row)
    int block_size, block_log2, num_blocks, max_blocks, box_rows;
    int rows_tile;               // (sequence, row) pairs in a row tile: 128 / G
    int nrt, np;                 // row tiles, pairs of row tiles
    int num_ctas;
    float scale_log2;
    long long wait_limit;
};

__device__ __forceinline__ int prefix_keys(const PrefixArgs& a) {
    int P = *a.prefix_len;
    P = max(0, min(P, a.Pmax));
    if (a.block_table) P = min(P, a.Lmax - a.R) & ~(a.block_size - 1);  // whole blocks that leave room for the rows' own
    return P;
}
// A sequence's own keys (behind the prefix), brought into [R, capacity].
__device__ __forceinline__ int own_keys(const PrefixArgs& a, int b, int P) {
    int L = a.ctx_lens[b];
    if (a.block_table) L -= P;
    return max(a.R, min(L, a.block_table ? a.Lmax - P : a.Lmax));
}
__device__ __forceinline__ int tiles_of(int keys) { return (keys + kKeys - 1) / kKeys; }

// What a CTA does, worked out by its first warp.
struct Plan {
    int P, nt, pad;         // prefix keys, tiles, and the virtual tiles in front of every KV head's
    int team, pair, pairs;  // the CTA's team, its first pair, the step to its next (pairs < np only on a small grid)
    int v0, v1;             // its range in the prefix's padded tile list; empty if it is in no team
    int worker, s0, s1;     // its rank among the CTAs that hold own tiles, and its range in that padded list
    int b, vb;              // the sequence s0 lies in, and where that sequence's tiles begin
};

// Share i of n equal shares of `total`, the first total % n of them one larger.
__device__ __forceinline__ int share_start(int total, int n, int i) {
    const int base = total / n, more = total - base * n;
    return i * base + min(i, more);
}

__device__ __noinline__ void make_plan(const PrefixArgs& a, int cta, Plan& out) {
    const int lane = threadIdx.x & 31;
    Plan p;
    p.P = prefix_keys(a);
    p.nt = tiles_of(p.P);
    int S = 0;
    bool bad = false;  // lengths out of range: only the device can see them, the first CTA says so
    for (int b = lane; b < a.B; b += 32) {
        const int own = own_keys(a, b, p.P);
        S += a.Hkv * (tiles_of(own) + kPad);
        bad |= a.ctx_lens[b] != own + (a.block_table ? p.P : 0);
    }
    if (cta == 0) {
        const int given = *a.prefix_len;
        bad |= given != p.P && !(a.block_table && (given & ~(a.block_size - 1)) == p.P);
        if (__any_sync(0xffffffffu, bad) && lane == 0) atomicOr(a.status, RAPID_STATUS_BAD_CTX_LEN);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) S += __shfl_xor_sync(0xffffffffu, S, o);

    const int C = a.num_ctas;
    const int npc = min(a.np, C);
    const int rounds = (a.np + npc - 1) / npc;
    // teams: the prefix's share of all work, at most what the grid holds, at least one
    int T = 0, w = 0, wh = 0;  // w, wh: cost of a team's range for a full pair and for a single row tile
    const int NP = a.Hkv * p.nt;
    p.pad = 0;
    if (NP > 0) {
        const long long all = (long long)NP * a.nrt + S;
        const int level = (int)max(1LL, min(all / C, 0x3fffffffLL));
        T = max(1, min(min(C / npc, NP), (int)(((long long)NP * (a.nrt > 1 ? 2 : 1) * rounds + level - 1) / level)));
        if (NP >= 4 * T) p.pad = kPad;
        const int range = (a.Hkv * (p.nt + p.pad) + T - 1) / T;
        w = (a.nrt > 1 ? 2 : 1) * range * rounds;
        wh = w;
    }
    const int NPv = a.Hkv * (p.nt + p.pad);
    const int n_team = T * npc;
    const bool half_class = T > 0 && (a.nrt & 1) && a.np > 1 && rounds == 1;  // each team has one CTA with a single row tile
    const int nH = half_class ? T : 0, nA = n_team - nH, nB = C - n_team;
    if (half_class) wh = w / 2;
    p.team = -1;
    p.pair = 0;
    p.pairs = npc;
    p.v0 = p.v1 = 0;
    if (cta < n_team) {
        p.team = cta / npc;
        p.pair = cta - p.team * npc;
        p.v0 = share_start(NPv, T, p.team);
        p.v1 = share_start(NPv, T, p.team + 1);
    }
    // own tiles: fill the classes (no prefix work; a single row tile; a full pair) up to one level
    int SB = 0, SH = 0, SA = 0;
    int left = S;
    const int l1 = (int)min((long long)left, (long long)nB * (half_class ? wh : w));
    SB = l1;
    left -= l1;
    if (left > 0 && nH > 0) {
        const int l2 = (int)min((long long)left, (long long)(nB + nH) * (w - wh));
        const int forH = (int)((long long)l2 * nH / (nB + nH));
        SH += forH;
        SB += l2 - forH;
        left -= l2;
    }
    if (left > 0) {
        const int each = left / C;
        SB += each * nB;
        SH += each * nH;
        SA = left - each * (nB + nH);
    }
    if (nB == 0 && SB > 0) {  // (nothing to give to an empty class)
        SA += SB;
        SB = 0;
    }
    if (nA == 0 && SA > 0) {  // no CTA carries a full pair
        if (nB) SB += SA; else SH += SA;
        SA = 0;
    }
    // workers: the CTAs of class B, then H, then A, those without a share left out
    int cls_n, cls_total, cls_rank, off_w, off_s;
    const int usedB = min(nB, SB), usedH = min(nH, SH);
    if (cta >= n_team) {
        cls_n = nB, cls_total = SB, cls_rank = cta - n_team, off_w = 0, off_s = 0;
    } else if (half_class && p.pair == a.np - 1) {
        cls_n = nH, cls_total = SH, cls_rank = p.team, off_w = usedB, off_s = SB;
    } else {
        cls_n = nA, cls_total = SA, off_w = usedB + usedH, off_s = SB + SH;
        cls_rank = half_class ? p.team * (npc - 1) + p.pair : cta;
    }
    p.worker = off_w + cls_rank;
    p.s0 = off_s + share_start(cls_total, cls_n, cls_rank);
    p.s1 = off_s + share_start(cls_total, cls_n, cls_rank + 1);
    // the sequence s0 lies in
    p.b = 0;
    p.vb = 0;
    if (p.s1 > p.s0) {
        int base = 0;
        for (int b0 = 0; b0 < a.B; b0 += 32) {
            const int b = b0 + lane;
            const int span = b < a.B ? a.Hkv * (tiles_of(own_keys(a, b, p.P)) + kPad) : 0;
            int incl = span;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += x;
            }
            const unsigned past = __ballot_sync(0xffffffffu, base + incl > p.s0 && b < a.B);
            if (past) {
                const int src = __ffs(past) - 1;
                p.b = b0 + src;
                p.vb = base + __shfl_sync(0xffffffffu, incl - span, src);
                break;
            }
            base += __shfl_sync(0xffffffffu, incl, 31);
        }
    }
    if (lane == 0) out = p;
}

// One CTA's way through its segments; every role walks it for itself.
struct Segment {
    bool own, dual_row;
    int b, kvh, pair;   // sequence (own) or pair of row tiles (prefix)
    int tile0, tiles;   // run of tiles inside the unit
    int keys;           // keys of the unit: own keys or prefix keys
    int unit_tiles;
};
struct Walk {
    int pair, v, s, b, vb;
};
__device__ __forceinline__ void walk_begin(const Plan& p, Walk& w) {
    w.pair = p.pair;
    w.v = p.v0;
    w.s = p.s0;
    w.b = p.b;
    w.vb = p.vb;
}
__device__ __forceinline__ bool walk_next(const PrefixArgs& a, const Plan& p, Walk& w, Segment& g) {
    while (w.pair < a.np && p.v1 > p.v0) {  // prefix ranges: one pass per pair
        if (w.v >= p.v1) {
            w.v = p.v0;
            w.pair += p.pairs;
            continue;
        }
        const int span = p.nt + p.pad;
        const int h = w.v / span, o = w.v - h * span;
        const int e = min(span, o + p.v1 - w.v);
        w.v += e - o;
        const int t0 = max(0, o - p.pad), t1 = max(0, e - p.pad);
        if (t1 <= t0) continue;
        g.own = false;
        g.dual_row = 2 * w.pair + 1 < a.nrt;
        g.b = 0;
        g.kvh = h;
        g.pair = w.pair;
        g.tile0 = t0;
        g.tiles = t1 - t0;
        g.keys = p.P;
        g.unit_tiles = p.nt;
        return true;
    }
    while (w.s < p.s1 && w.b < a.B) {
        const int keys = own_keys(a, w.b, p.P);
        const int nt = tiles_of(keys), span = nt + kPad;
        const int x = w.s - w.vb;
        const int h = x / span, o = x - h * span;
        if (h >= a.Hkv) {
            w.vb += a.Hkv * span;
            ++w.b;
            continue;
        }
        const int e = min(span, o + p.s1 - w.s);
        w.s += e - o;
        const int t0 = max(0, o - kPad), t1 = max(0, e - kPad);
        if (t1 <= t0) continue;
        g.own = true;
        g.dual_row = false;
        g.b = w.b;
        g.kvh = h;
        g.pair = 0;
        g.tile0 = t0;
        g.tiles = t1 - t0;
        g.keys = keys;
        g.unit_tiles = nt;
        return true;
    }
    return false;
}

__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, const WaitCtx& wc) {
    return __all_sync(0xffffffffu, mbar_wait_bounded(bar, parity, wc));
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
    __shared__ uint64_t q_full[2], q_empty[2], s_full[2], p_full[2], pv_done[2], drain_bar[2];
    __shared__ uint32_t tmem_slot;
    __shared__ int s_abort;
    __shared__ Plan plan;

    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem = smem_raw + (smem_base - smem_u32(smem_raw));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cta = blockIdx.x;

    if (threadIdx.x == 0) {
        for (int i = 0; i < NK; ++i) mbar_init(&k_full[i], 1), mbar_init(&k_empty[i], 1);
        for (int i = 0; i < NV; ++i) mbar_init(&v_full[i], 1), mbar_init(&v_empty[i], 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&q_full[i], 1);
            mbar_init(&q_empty[i], 1);
            mbar_init(&s_full[i], 1);
            mbar_init(&p_full[i], 4);
            mbar_init(&pv_done[i], 1);
            mbar_init(&drain_bar[i], 1);
        }
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
    if (warp == 0) make_plan(a, cta, plan);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = tmem_slot;
    const WaitCtx wc = {&s_abort, a.wait_limit};

    Walk w;
    walk_begin(plan, w);
    Segment g;
    if (warp == 8) {
        // ---------------- K/V producer ----------------
        if (lane == 0) {
            int n_k = 0, n_v = 0;  // K and V tiles whose copies were issued
            bool ok = true;
            while (ok && walk_next(a, plan, w, g)) {
                const CUtensorMap* mk = g.own ? &tmKo : &tmKp;
                const CUtensorMap* mv = g.own ? &tmVo : &tmVp;
                const int parts = kKeys / a.box_rows;
                const uint32_t part_bytes = kHalfBytes / parts;
                for (int t = 0; t < g.tiles; ++t) {
                    const int key0 = (g.tile0 + t) * kKeys;
                    int c1[2] = {key0, 0}, c3[2] = {g.b, g.b};
                    if (a.block_table) {
                        for (int q = 0; q < parts; ++q) {
                            const int in_unit = key0 + q * a.box_rows;
                            const int pos = in_unit + (g.own ? plan.P : 0);
                            c1[q] = pos & (a.block_size - 1);
                            if (in_unit >= g.keys) {
                                c3[q] = a.num_blocks;  // past the keys: zeros, no table entry is read
                                continue;
                            }
                            c3[q] = __ldg(a.block_table + (size_t)g.b * a.max_blocks + (pos >> a.block_log2));
                            if ((unsigned)c3[q] >= (unsigned)a.num_blocks) {
                                atomicOr(a.status, RAPID_STATUS_BAD_BLOCK_TABLE);
                                c3[q] = a.num_blocks;  // outside the pool: the copy reads zeros
                            }
                        }
                    }
                    const int ks = n_k % NK, vs = n_v % NV;
                    if (n_k >= NK) ok = mbar_wait_bounded_relaxed(&k_empty[ks], (n_k / NK - 1) & 1, wc);
                    if (!ok) break;
                    mbar_arrive_expect_tx(&k_full[ks], TILE);
                    for (int q = 0; q < parts; ++q)
#pragma unroll
                        for (int h = 0; h < NH; ++h)
                            tma_load_4d(smem + OFF_K + ks * TILE + h * kHalfBytes + q * part_bytes, mk, &k_full[ks],
                                        h * 64, c1[q], g.kvh, c3[q]);
                    ++n_k;
                    if (n_v >= NV) ok = mbar_wait_bounded_relaxed(&v_empty[vs], (n_v / NV - 1) & 1, wc);
                    if (!ok) break;
                    mbar_arrive_expect_tx(&v_full[vs], TILE);
                    for (int q = 0; q < parts; ++q)
#pragma unroll
                        for (int h = 0; h < NH; ++h)
                            tma_load_4d(smem + OFF_V + vs * TILE + h * kHalfBytes + q * part_bytes, mv, &v_full[vs],
                                        h * 64, c1[q], g.kvh, c3[q]);
                    ++n_v;
                }
            }
            // every copy lands before the CTA gives up its shared memory, whoever may have given up waiting for it
            for (int s = 0; s < NK && s < n_k; ++s) mbar_wait_drain(&k_full[s], ((n_k - 1 - s) / NK) & 1);
            for (int s = 0; s < NV && s < n_v; ++s) mbar_wait_drain(&v_full[s], ((n_v - 1 - s) / NV) & 1);
        }
    } else if (warp == 9) {
        // ---------------- Q producer: a ring of two row tiles ----------------
        if (lane == 0) {
            int n = 0;
            bool ok = true;
            while (ok && walk_next(a, plan, w, g)) {
                const int cnt = g.dual_row ? 2 : 1;
                for (int i = 0; i < cnt; ++i, ++n) {
                    const int s = n & 1;
                    if (n >= 2) ok = mbar_wait_bounded_relaxed(&q_empty[s], (n / 2 - 1) & 1, wc);
                    if (!ok) break;
                    const int row0 = g.own ? g.b * a.R : (2 * g.pair + i) * a.rows_tile;
                    mbar_arrive_expect_tx(&q_full[s], (uint32_t)a.rows_tile * a.G * D * 2);
#pragma unroll
                    for (int h = 0; h < NH; ++h)
                        tma_load_4d(smem + OFF_Q + s * TILE + h * kHalfBytes, &tmQ, &q_full[s], h * 64, g.kvh * a.G,
                                    row0, 0);
                }
            }
            for (int s = 0; s < 2 && s < n; ++s) mbar_wait_drain(&q_full[s], ((n - 1 - s) / 2) & 1);
        }
    } else if (warp == 10) {
        // ---------------- QK^T issuer ----------------
        if (lane == 0) {
            constexpr uint32_t idesc = umma_idesc_bf16(128, kKeys, 0, 0);
            const uint64_t q_desc = umma_smem_desc(smem_base + OFF_Q, 16, 1024);
            const uint64_t k_desc = umma_smem_desc(smem_base + OFF_K, 16, 1024);
            int n = 0, qn = 0, par = 0, done[2] = {0, 0};
            bool ok = true;
            while (ok && walk_next(a, plan, w, g)) {
                const int cnt = g.dual_row ? 2 : 1;
                for (int i = 0; i < cnt && ok; ++i) ok = mbar_wait_bounded(&q_full[(qn + i) & 1], ((qn + i) >> 1) & 1, wc);
                for (int t = 0; t < g.tiles && ok; ++t, ++n) {
                    const int ks = n % NK;
                    ok = mbar_wait_bounded(&k_full[ks], (n / NK) & 1, wc);
                    for (int i = 0; i < cnt && ok; ++i) {
                        const int s = g.dual_row ? i : par & 1;
                        // the stream's S columns are free once the PV of its previous tile has read P from them
                        const int c = s ? done[1]++ : done[0]++;
                        if (c > 0) ok = mbar_wait_bounded(&pv_done[s], (c - 1) & 1, wc);
                        if (!ok) break;
                        tc_fence_after_sync();
                        const uint64_t qd = q_desc + (uint64_t)(((qn + i) & 1) * (TILE >> 4));
                        const uint64_t kd = k_desc + (uint64_t)(ks * (TILE >> 4));
                        const uint32_t d = tmem + COL_S + 128u * s;
#pragma unroll
                        for (int kk = 0; kk < D / 16; ++kk) {
                            const uint32_t off = (kk >> 2) * (kHalfBytes >> 4) + (kk & 3) * 2;
                            umma_bf16_ss(d, qd + off, kd + off, idesc, kk > 0);
                        }
                        umma_commit(&s_full[s]);
                    }
                    if (!ok) break;
                    umma_commit(&k_empty[ks]);
                    if (!g.dual_row) ++par;
                }
                if (ok)
                    for (int i = 0; i < cnt; ++i) umma_commit(&q_empty[(qn + i) & 1]);
                qn += cnt;
            }
            if (!ok) {  // every MMA issued here has completed before tensor memory is freed
                umma_commit(&drain_bar[0]);
                mbar_wait_drain(&drain_bar[0], 0);
            }
        }
    } else if (warp == 11) {
        // ---------------- PV issuer ----------------
        if (lane == 0) {
            constexpr uint32_t idesc = umma_idesc_bf16(128, D, 0, 1);
            const uint64_t v_desc = umma_smem_desc(smem_base + OFF_V, kHalfBytes, 1024);
            int n = 0, par = 0, done[2] = {0, 0};
            bool ok = true;
            while (ok && walk_next(a, plan, w, g)) {
                const int cnt = g.dual_row ? 2 : 1;
                for (int t = 0; t < g.tiles && ok; ++t, ++n) {
                    const int vs = n % NV;
                    ok = mbar_wait_bounded(&v_full[vs], (n / NV) & 1, wc);
                    for (int i = 0; i < cnt && ok; ++i) {
                        const int s = g.dual_row ? i : par & 1;
                        const bool fresh = g.dual_row ? t == 0 : t < 2;  // the stream's first tile of the segment
                        const int c = s ? done[1]++ : done[0]++;
                        ok = mbar_wait_bounded(&p_full[s], c & 1, wc);
                        if (!ok) break;
                        tc_fence_after_sync();
                        const uint64_t vd = v_desc + (uint64_t)(vs * (TILE >> 4));
                        const uint32_t d = tmem + COL_O + 128u * s, p = tmem + COL_S + 128u * s;
#pragma unroll
                        for (int kk = 0; kk < kKeys / 16; ++kk)
                            umma_bf16_ts(d, p + 8 * kk, vd + kk * (2048 >> 4), idesc, (!fresh || kk > 0) ? 1u : 0u);
                        umma_commit(&pv_done[s]);
                    }
                    if (!ok) break;
                    umma_commit(&v_empty[vs]);
                    if (!g.dual_row) ++par;
                }
            }
            if (!ok) {
                umma_commit(&drain_bar[1]);
                mbar_wait_drain(&drain_bar[1], 0);
            }
        }
    } else {
        // ---------------- softmax warps: stream = warp / 4, row of the tile = 32 (warp % 4) + lane ----------------
        const int stream = warp >> 2;
        const int row = (warp & 3) * 32 + lane;
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + lane_base + COL_S + 128u * stream;
        const uint32_t tO = tmem + lane_base + COL_O + 128u * stream;
        const float c = a.scale_log2;
        int n = 0, par = 0, cnt = 0;  // CTA-wide tile index, dual-key tiles met, tiles of this stream
        bool ok = true;
        while (ok && walk_next(a, plan, w, g)) {
            // the tile's rows: (sequence, row, head in group) of the batch, or (row, head) of one sequence
            const int tile_row0 = (2 * g.pair + (g.dual_row ? stream : 0)) * a.rows_tile;
            const int rows = g.own ? a.GR : min(a.rows_tile, a.B * a.R - tile_row0) * a.G;
            const bool row_valid = row < rows;
            const bool warp_active = (warp & 3) * 32 < rows;
            // keys a row sees: all of the prefix; its own sequence's up to itself
            const int lim = g.own ? g.keys - a.R + row / a.G : g.keys - 1;
            const int all_see = g.own ? g.keys - a.R : g.keys - 1;
            float m_ref = -INFINITY, l_run = 0.f;
            bool first = true;
            const int step = g.dual_row ? 1 : 2;
            for (int t = g.dual_row ? 0 : (stream ^ par) & 1; t < g.tiles && ok; t += step) {
                ok = warp_wait(&s_full[stream], cnt & 1, wc);
                if (!ok) break;
                const int key0 = (g.tile0 + t) * kKeys;
                if (warp_active) {
                    tc_fence_after_sync();
                    uint32_t sr[4][32];
#pragma unroll
                    for (int i = 0; i < 4; ++i) tmem_ld_x32(tS + 32 * i, sr[i]);
                    tmem_wait_ld();
                    if (key0 + kKeys - 1 > all_see) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int k = 0; k < 32; ++k)
                                if (key0 + 32 * i + k > lim) sr[i][k] = __float_as_uint(-INFINITY);
                    }
                    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int k = 0; k < 32; ++k) mx[k & 3] = fmaxf(mx[k & 3], __uint_as_float(sr[i][k]));
                    const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * c;
                    const bool move = row_valid && top > m_ref + kJump;
                    if (__any_sync(0xffffffffu, move)) {
                        const float factor = move ? fast_exp2(m_ref - top) : 1.f;  // 0 when there was no reference
                        if (move) {
                            l_run *= factor;
                            m_ref = top;
                        }
                        if (!first) {
                            // O at rest: the stream's previous PV has completed
                            ok = warp_wait(&pv_done[stream], (cnt - 1) & 1, wc);
                            if (!ok) break;
                            tc_fence_after_sync();
#pragma unroll
                            for (int i = 0; i < D / 16; ++i) {
                                uint32_t o[16];
                                tmem_ld_x16(tO + 16 * i, o);
                                tmem_wait_ld();
#pragma unroll
                                for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * factor);
                                tmem_st_x16(tO + 16 * i, o);
                            }
                        }
                    }
                    const float m_use = m_ref == -INFINITY ? 0.f : m_ref;
                    float s0 = 0.f, s1 = 0.f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t pk[16];
#pragma unroll
                        for (int k = 0; k < 32; k += 2) {
                            const float p0 = fast_exp2(fmaf(__uint_as_float(sr[i][k]), c, -m_use));
                            const float p1 = fast_exp2(fmaf(__uint_as_float(sr[i][k + 1]), c, -m_use));
                            s0 += p0;
                            s1 += p1;
                            pk[k >> 1] = pack_bf16x2(p0, p1);
                        }
                        tmem_st_x16(tS + 16 * i, pk);
                    }
                    l_run += s0 + s1;
                    first = false;
                }
                if (key0 + kKeys > g.keys) {
                    // V rows past the keys may hold any bits: zero them so that 0 * row = 0
                    const int vs = (n + t) % NV;
                    ok = warp_wait(&v_full[vs], ((n + t) / NV) & 1, wc);
                    if (!ok) break;
                    const int first_bad = g.keys - key0;
                    const int chunks = (kKeys - first_bad) * 8;
#pragma unroll
                    for (int h = 0; h < NH; ++h)
                        for (int ch = row; ch < chunks; ch += 128)
                            *reinterpret_cast<uint4*>(smem + OFF_V + vs * TILE + h * kHalfBytes + first_bad * 128 + ch * 16) =
                                make_uint4(0, 0, 0, 0);
                    fence_proxy_async_smem();
                }
                tmem_wait_st();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_full[stream]);
                ++cnt;
            }
            if (!ok) break;

            // ---- end of the segment: the partial of this stream ----
            const int unit = g.b * a.Hkv + g.kvh;
            const int slot_rows = g.own ? a.GR : 128;
            float* slot = g.own ? a.part_own + (size_t)((plan.worker + unit) * 2 + stream) * slot_floats(a.GR, D)
                                : a.part_prefix + (size_t)((plan.team + g.kvh) * 2 * a.np + 2 * g.pair + stream) * slot_floats(128, D);
            if (!first) {
                ok = warp_wait(&pv_done[stream], (cnt - 1) & 1, wc);
                if (!ok) break;
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
            }
            if (row_valid) {
                slot[(size_t)slot_rows * D + row] = m_ref;
                slot[(size_t)slot_rows * (D + 1) + row] = l_run;
            }
            // which workers hold tiles of a unit, for the merge
            if (threadIdx.x == 0) {
                int2* range = g.own ? a.own_range + unit : a.prefix_range + g.kvh;
                const int who = g.own ? plan.worker : plan.team;
                if (g.own || g.pair == 0) {
                    if (g.tile0 == 0) range->x = who;
                    if (g.tile0 + g.tiles == g.unit_tiles) range->y = who;
                }
            }
            n += g.tiles;
            if (!g.dual_row) par += g.tiles;
        }
    }

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
// rows of a KV head (lane = row: slots are stored so that this reads whole lines) and 32 columns, four
// to a warp.  The order of the sums is fixed: results do not depend on timing.
template <int D>
__global__ void __launch_bounds__(256)
prefix_attn_merge_kernel(const __grid_constant__ PrefixArgs a, __nv_bfloat16* out, float* lse_out, float* out_f32) {
    __shared__ float sh_m[8][32], sh_l[8][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int kvh = blockIdx.y;
    const int total_rows = a.B * a.R * a.G;
    const int flat = blockIdx.x * 32 + lane;
    const bool valid = flat < total_rows;
    const int f = (valid ? flat : total_rows - 1) / a.G, gh = (valid ? flat : total_rows - 1) - f * a.G;  // (sequence, row), head in group
    const int b = f / a.R, i = f - b * a.R;
    const int rt = f / a.rows_tile;
    const int prow = (f - rt * a.rows_tile) * a.G + gh;
    const int pair = rt >> 1;
    const bool dual = 2 * pair + 1 < a.nrt;
    const int orow = i * a.G + gh;
    const int unit = b * a.Hkv + kvh;
    const long long sp = slot_floats(128, D), so = slot_floats(a.GR, D);

    griddep_wait();
    griddep_launch_dependents();
    const int P = prefix_keys(a);
    int2 pr = P > 0 ? __ldcg(a.prefix_range + kvh) : make_int2(0, -1);
    int2 orr = __ldcg(a.own_range + unit);
    // (a split kernel whose waits ran out may not have written them: whatever they hold, stay inside the slots)
    const int teams = max(1, a.num_ctas / a.np);
    if (pr.x < 0 || pr.y >= teams) pr = make_int2(0, -1);
    if (orr.x < 0 || orr.y >= a.num_ctas) orr = make_int2(0, -1);
    // The row's slots as one list: index x < np_slots is in the prefix part (one slot per team, or two where a
    // single row tile's keys went to both streams), the rest in the own part (two per worker).
    const int per = dual ? 1 : 2;
    const int n_p = max(0, pr.y - pr.x + 1) * per, n_all = n_p + max(0, orr.y - orr.x + 1) * 2;
    const float* pbase = a.part_prefix + (size_t)((pr.x + kvh) * 2 * a.np + 2 * pair + (dual ? rt & 1 : 0)) * sp;
    const long long pstep = (long long)2 * a.np * sp;
    const float* obase = a.part_own + (size_t)(orr.x + unit) * 2 * so;
    auto slot_of = [&](int x) -> const float* {
        if (x < n_p) return dual ? pbase + x * pstep : pbase + (x >> 1) * pstep + (x & 1) * sp;
        return obase + (x - n_p) * so;
    };
    float m = -INFINITY, l = 0.f;
    for (int x = warp; x < n_all; x += 8) {
        const float* s = slot_of(x);
        const bool pre = x < n_p;
        const float ms = s[(pre ? 128LL : a.GR) * D + (pre ? prow : orow)];
        const float ls = s[(pre ? 128LL : a.GR) * (D + 1) + (pre ? prow : orow)];
        if (ms == -INFINITY) continue;  // (its sum is 0)
        if (ms > m) {
            l = l * exp2f(m - ms) + ls;
            m = ms;
        } else {
            l += ls * exp2f(ms - m);
        }
    }
    sh_m[warp][lane] = m;
    sh_l[warp][lane] = l;
    __syncthreads();
    float M = -INFINITY;
#pragma unroll
    for (int k = 0; k < 8; ++k) M = fmaxf(M, sh_m[k][lane]);
    float Lsum = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (sh_m[k][lane] != -INFINITY) Lsum += sh_l[k][lane] * exp2f(sh_m[k][lane] - M);

    const int d4 = blockIdx.z * 8 + warp;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int x = 0; x < n_all; ++x) {
        const float* s = slot_of(x);
        const bool pre = x < n_p;
        const int rows = pre ? 128 : a.GR, r = pre ? prow : orow;
        const float ms = s[(long long)rows * D + r];
        const float4 o = *reinterpret_cast<const float4*>(s + ((long long)d4 * rows + r) * 4);
        if (ms != -INFINITY) {  // an untouched slot holds no O: its bits are not used
            const float wgt = exp2f(ms - M);
            acc.x += wgt * o.x;
            acc.y += wgt * o.y;
            acc.z += wgt * o.z;
            acc.w += wgt * o.w;
        }
    }
    if (!valid) return;
    const size_t orow_g = ((size_t)f * a.Hq + (size_t)kvh * a.G + gh);
    const float4 v = make_float4(acc.x / Lsum, acc.y / Lsum, acc.z / Lsum, acc.w / Lsum);
    *reinterpret_cast<uint2*>(out + orow_g * D + d4 * 4) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
    if (out_f32) *reinterpret_cast<float4*>(out_f32 + orow_g * D + d4 * 4) = v;
    if (lse_out && d4 == 0) lse_out[orow_g] = (M + log2f(Lsum)) * 0.69314718055994530942f;
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

struct WsLayout {
    size_t prefix_range, own_range, part_prefix, part_own, total;
};
WsLayout ws_layout(int B, int Hkv, int GR, int np, int D) {
    WsLayout l;
    size_t off = kWorkspaceHeaderBytes;
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
    static bool configured[64] = {};
    if (dev >= 64 || !configured[dev]) {
        RAPID_CUDA_CHECK(cudaFuncSetAttribute(prefix_attn_split_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        if (dev < 64) configured[dev] = true;
    }
    RAPID_CUDA_CHECK(launch_dependent(prefix_attn_split_kernel<D>, dim3(a.num_ctas), dim3(kThreads), (size_t)smem, stream,
                                      tm[0], tm[1], tm[2], tm[3], tm[4], a));
    if (split_done) RAPID_CUDA_CHECK(cudaEventRecord(static_cast<cudaEvent_t>(split_done), stream));
    const int rows = a.B * a.R * a.G;
    RAPID_CUDA_CHECK(launch_dependent(prefix_attn_merge_kernel<D>, dim3((rows + 31) / 32, a.Hkv, D / 32), dim3(256), 0,
                                      stream, a, out, lse, out_f32));
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
