// Attention of many new rows of every sequence over its cache: a prompt, the next piece of one, a drafter's retrieved context.
//
//   out[b,i,h,:] = sum_j softmax_j(scale q[b,i,h,:] . k_j) v_j   over the keys j that row i sees: those up to its own position
//   p = L_b - n_b + i; with a window, of them the `window` newest and the first `sink`; or all L_b.
//
// The G query heads of a KV head share its keys, so a row tile (the M axis of the MMAs, 128 rows) is 128 / G neighbouring
// rows of all G heads.  A unit is one KV head of one sequence and two row tiles, which go through the same K/V tiles of 128 keys:
// stream s (eight softmax warps, S and O accumulators) has row tile s.
//
//   S_s[128 x 128] = Q_s K^T   A = Q tile, B = K tile, both K-major in shared memory
//   O_s[128 x D]  += P_s V     A = P (bf16, over the first half of S_s's columns), B = V tile, MN-major
//
// P is rounded to bf16 because both operands of a product have one type and V is bf16: a probability is off by at most 2^-8 of itself, an
// output by 2^-8 of the weighted mean of |v| (2.0 - 2.4e-3 of an output's norm for 1.4 - 1.7e-3 with fp32 probabilities).  The row sums add
// the fp32 probabilities.
//
// One thread issues all products, in the order PV_0 QK_0 PV_1 QK_1: while the tensor core is at one stream's, the softmax warps of
// the other are at theirs.  It works them off in that order, so the QK^T that overwrites S_s goes out right behind the PV that reads P
// from it, and scores in hand mean that the PV before them has completed.
//
// Softmax.  Four warps have a quarter of a stream's rows and half of a tile's keys each, four the other half: with one warp for both
// halves a tile took a sixth longer (646 us for 554 at 8,192 rows), two warps to a scheduler being too few to hide tensor memory's
// latency.  The two warps of a quarter meet once a tile.  A row's reference moves only when a score is 2^16 above it, so the
// exponentials of a tile need not wait for its maximum: they go by the reference in place, the maximum is found on the way, and a tile that
// moves a reference (the first of a unit, hardly any other) is done over; nothing of it was stored.  The reference is a score itself,
// so that the largest probability of a row's first tile is exactly 1 in bf16 too: rows of few keys lose nothing to its rounding.
//
// Work split.  A plan kernel lists the pieces of work: whole units, and of the last units (one to two for every CTA) runs of their
// tiles, so that the CTAs end together and few rows over many keys keep all of them busy.  CTAs take pieces in order from a
// counter: neighbouring units, which read the same keys, run at the same time, the long ones of a causal sequence first.  A
// whole unit writes its output; runs leave partials, which the merge kernel joins by their log-sum-exp in a fixed order.
//
// Bound: power, then the chain of a stream.  Two row tiles and a K/V tile are 2,048 cycles of the tensor core and 2,048 of the
// special-function unit, and take 3,600: a stream's softmax (2,000 cycles) and its products (1,024, and 400 until they are seen) follow
// one another, and the other stream's fill the gaps only in part.  While it runs for long the 1 kW cap holds the clock at 1.6 - 1.75 GHz.
// Measured (three kernels, D = 128, calls in a row in a graph):
//     8,192 rows, 32 heads over 8, causal                            468 us  1.17 PFLOP/s (547 while it runs for long)
//    32,768 rows, causal                                           7,928 us  1.11
//    32,768 rows, 4 sinks and a window of 4,092                    2,088 us  0.99
//       500 rows over 130,000 keys before them, paged in 64        1,067 us  1.00
//     8 prompts of up to 4,001 rows, 28 over 4, paged in 256       1,127 us  0.99
//     2 prompts of up to 100 rows, 8 over 2 of 64                   15.6 us  plan, first tiles, last outputs and merge, one after another
//       500 rows, all of 65,000 keys visible                         502 us  1.06
// (boxes differ by up to 4 %).  At D = 64 the special-function unit has as much to do for half of the products: 16,384 rows of 8 heads 454 us,
// 0.61 PFLOP/s; tensor memory has 128 columns to spare there, which are not used.
// Exponentials as polynomials on the FMA pipe (1 to 4 pairs of 8) gained nothing at D = 128 (8,192 rows 554 us with none, 563 - 599 with some);
// at D = 64 they were not tried.  19 warps leave a thread 96 registers; 40 to 52 bytes a thread are spilled.
//
// Waits are bounded as everywhere in this library; see mbar_wait_bounded.
#include <math.h>

#include <atomic>

#include "attention_rows.cuh"
#include "common.cuh"
#include "prefill.cuh"
#include "tcgen05.cuh"

namespace rapid {

namespace {

constexpr int kKeys = 128;               // keys per tile
constexpr int kSoftmaxWarps = 16;        // of each stream eight: four quarters of the rows by two halves of the keys
constexpr int kThreads = 32 * (kSoftmaxWarps + 3);  // and the producer, the walk, the MMA issuer
constexpr int kHalfBytes = kKeys * 128;  // one 64-column half of a tile of 128 rows
constexpr float kJump = 16.f;            // a score this far (log2) above a row's reference moves it
constexpr int kMaxPrefillCtas = 256;
constexpr int kPlanThreads = 512;        // at least the units of the tail: fewer than two for every CTA
constexpr int kMaxTail = 640;            // pieces the tail is cut into at most
constexpr int kSeqInSmem = 1024;
constexpr float kPieceCost = 2.5f;       // tiles that a piece costs beside its own
constexpr float kSlotCost = 0.03f;       // tiles that a partial costs the whole call, written and read
constexpr float kMergeCost = 2.f;        // tiles that it takes to join any
constexpr int kMaxUnits = 1 << 24;
constexpr int64_t kMaxKeys = 0x7fffffff - 256;

__host__ __device__ constexpr int k_slots(int D) { return D == 128 ? 2 : 4; }
__host__ __device__ constexpr int v_slots(int D) { return D == 128 ? 3 : 6; }
__host__ __device__ constexpr int tile_bytes(int D) { return (D / 64) * kHalfBytes; }
// A piece of work: `tiles` tiles of a unit from the first-th of its list on (-1 tiles: the end).  slot < 0: the whole unit, whose
// output is written; else a partial goes into that slot.
struct __align__(16) Piece {
    int b, kvh, row0, n;  // sequence, KV head, first row of the unit, rows of the sequence
    int L, first, tiles, slot;
};
// A unit of the tail that was cut.
struct __align__(16) Cut {
    int b, kvh, row0, n;
    int slot, parts, reserved0, reserved1;
};
constexpr int kFewParts = 8, kSomeFew = 1, kSomeMany = 2;
struct Control {
    int next, pieces, cuts, shapes;  // shapes: whether there are cuts of few parts, and of many
};

struct PrefillArgs {
    const int32_t* ctx_lens;
    const int32_t* n_tokens;     // or NULL: T each
    const int32_t* block_table;  // paged cache, or NULL
    Control* control;
    int32_t* seq_start;          // [B + 1]: first unit of every sequence
    Piece* pieces;
    Cut* cuts;
    float* slots;
    int32_t* status;
    int32_t* plan_sig;           // first word of a verify plan's signature: taken back, its walks are overwritten
    __nv_bfloat16* out;
    float *out_f32, *lse_out;    // or NULL
    int B, T, G, Hq, Hkv;
    int Lmax;
    int block_size, block_log2, num_blocks, max_blocks, box_rows;
    int rows_tile;               // rows of a sequence in a row tile: 128 / G
    int slot_rows;               // 128, or 256 where a unit has two row tiles
    int max_slots;
    int num_ctas;
    int sink, window, all_visible;
    float scale_log2;
    long long wait_limit;
};

// Partials: a slot holds slot_rows rows of unnormalised O as [D/4][rows][4] floats (a warp whose lanes are rows writes and reads
// whole lines), then the rows' references (log2), then their sums.
__host__ __device__ constexpr size_t slot_floats(int rows, int D) { return (size_t)rows * (D + 2); }

// A sequence's rows and keys as the device finds them; false if they are out of range (the sequence is then left out).
__device__ __forceinline__ bool lengths(const PrefillArgs& a, int b, int& n, int& L) {
    n = a.n_tokens ? a.n_tokens[b] : a.T;
    L = a.ctx_lens[b];
    return n >= 0 && n <= a.T && L >= (a.all_visible ? 0 : n) && L <= a.Lmax;
}

// The tiles that some row of a unit sees: tiles 0 .. sinks - 1, then lo .. end - 1.
struct Span {
    int sinks, lo, end;
};
__device__ __forceinline__ Span span_of(const PrefillArgs& a, int row0, int n, int L) {
    Span s = {0, 0, 0};
    const int p0 = L - n + row0;
    const int keys = a.all_visible ? L : L - n + min(n, row0 + 2 * a.rows_tile);
    s.end = (keys + kKeys - 1) / kKeys;
    if (a.window) {
        s.lo = max(0, p0 - a.window + 1) / kKeys;
        s.sinks = min(s.lo, (int)(((long long)a.sink + kKeys - 1) / kKeys));
    }
    return s;
}

// Inclusive sum over the block; *total receives the block's.
__device__ __forceinline__ int block_scan(int v, int* sh, int* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 31) sh[warp] = x;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kPlanThreads / 32; ++w) {
        if (w < warp) before += sh[w];
        all += sh[w];
    }
    *total = all;
    return x + before;
}

// The list of pieces.  One block; latency is what counts.
__global__ void __launch_bounds__(kPlanThreads) prefill_plan_kernel(const __grid_constant__ PrefillArgs a) {
    __shared__ int sh_start[kSeqInSmem + 1], sh_scan[kPlanThreads / 32], sizes[kPlanThreads];
    __shared__ float sh_est[kPlanThreads / 32];
    __shared__ int sh_len[kPlanThreads / 32], sh_shapes;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    griddep_wait();
    griddep_launch_dependents();
    if (tid == 0) *a.plan_sig = 0, sh_shapes = 0;
    const bool in_smem = a.B <= kSeqInSmem;
    int units = 0;
    for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
        const int b = b0 + tid;
        int mine = 0;
        if (b < a.B) {
            int n, L;
            if (lengths(a, b, n, L)) mine = a.Hkv * ((n + 2 * a.rows_tile - 1) / (2 * a.rows_tile));
            else atomicOr(a.status, RAPID_STATUS_BAD_CTX_LEN);
        }
        int total;
        const int upto = block_scan(mine, sh_scan, &total);
        if (b < a.B) {
            a.seq_start[b] = units + upto - mine;
            if (in_smem) sh_start[b] = units + upto - mine;
        }
        units += total;
    }
    if (tid == 0) {
        a.seq_start[a.B] = units;
        if (in_smem) sh_start[a.B] = units;
    }
    __syncthreads();
    const int* start = in_smem ? sh_start : a.seq_start;

    // unit number u: the sequence, its KV heads one after the other, of each the last rows (the most keys) first
    auto unit = [&](int u, Piece& p) {
        int lo = 0, hi = a.B;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (start[mid] <= u) lo = mid;
            else hi = mid;
        }
        const int of_seq = start[lo + 1] - start[lo], pairs = of_seq / a.Hkv;
        const int r = u - start[lo];
        p.b = lo;
        p.kvh = r / pairs;
        p.row0 = (pairs - 1 - (r - p.kvh * pairs)) * 2 * a.rows_tile;
        lengths(a, lo, p.n, p.L);
        const Span s = span_of(a, p.row0, p.n, p.L);
        p.first = 0;
        p.tiles = s.sinks + s.end - s.lo;
        p.slot = -1;
    };
    const int tail = units < 2 * a.num_ctas ? units : a.num_ctas + units % a.num_ctas;
    const int whole = units - tail;
    for (int u = tid; u < whole; u += kPlanThreads) {
        Piece p;
        unit(u, p);
        a.pieces[u] = p;
    }
    Piece mine = {};
    if (tid < tail) unit(whole + tid, mine);
    sizes[tid] = tid < tail ? mine.tiles : 0;
    __syncthreads();
    // The length of a piece: every warp weighs one.  With `waves` pieces for every CTA a unit is cut into waves * CTAs / units
    // parts; the estimate is whole rounds of pieces of the mean cost (or, behind whole units, an even share and a quarter of a piece),
    // and what the partials cost.
    {
        int most = 0;
        for (int i = lane; i < tail; i += 32) most = max(most, sizes[i]);
        most = __reduce_max_sync(0xffffffffu, most);
        if (most > 2) {  // (to cut one or two tiles never pays)
            const int parts = max(1, (int)((long long)(warp + 1) * a.num_ctas / max(tail, 1)));
            const int len = max(1, (most + parts - 1) / parts);
            int count = 0, cut = 0;
            long long sum = 0;
            for (int i = lane; i < tail; i += 32) {
                const int c = max(1, (sizes[i] + len - 1) / len);
                count += c;
                cut += c > 1 ? c : 0;
                sum += sizes[i];
            }
            count = __reduce_add_sync(0xffffffffu, count);
            cut = __reduce_add_sync(0xffffffffu, cut);
            float all = (float)sum;
#pragma unroll
            for (int o = 16; o; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
            if (lane == 0) {
                const float mean = (all + kPieceCost * count) / max(count, 1), top = len + kPieceCost;
                float est = whole ? mean * count / a.num_ctas + 0.25f * top
                                  : mean * ((count + a.num_ctas - 1) / a.num_ctas) + top - mean;
                if (cut) est += kMergeCost + kSlotCost * cut;
                if (cut > a.max_slots || count > kMaxTail) est = INFINITY;
                sh_est[warp] = est;
                sh_len[warp] = len;
            }
        } else if (lane == 0) {
            sh_est[warp] = INFINITY;
        }
        __syncthreads();
    }
    int len = 0;
    float best = INFINITY;  // (every unit whole, if nothing else is allowed)
#pragma unroll
    for (int w = 0; w < kPlanThreads / 32; ++w)
        if (sh_est[w] < best) best = sh_est[w], len = sh_len[w];
    const int parts = tid >= tail ? 0 : best == INFINITY ? 1 : max(1, (mine.tiles + len - 1) / len);
    // pieces, partials and cut units before this thread's, in one sum: each is at most 640, ten bits
    static_assert(kMaxTail < 1024 && kPlanThreads <= 512, "fields of ten bits");
    if (parts > 1) atomicOr(&sh_shapes, parts <= kFewParts ? kSomeFew : kSomeMany);
    const int one = parts | (parts > 1 ? parts << 10 | 1 << 20 : 0);
    int sums;
    const int before = block_scan(one, sh_scan, &sums) - one;
    const int piece0 = before & 1023, slot0 = before >> 10 & 1023, cut0 = before >> 20;
    const int pieces = sums & 1023, cuts = sums >> 20;
    if (tid < tail) {
        const int tiles = mine.tiles;
        for (int i = 0; i < parts; ++i) {
            Piece p = mine;
            p.first = (int)((long long)tiles * i / parts);
            p.tiles = (int)((long long)tiles * (i + 1) / parts) - p.first;
            p.slot = parts > 1 ? slot0 + i : -1;
            a.pieces[whole + piece0 + i] = p;
        }
        if (parts > 1) a.cuts[cut0] = {mine.b, mine.kvh, mine.row0, mine.n, slot0, parts, 0, 0};
    }
    // (a CTA's first piece is the one of its own number: where there are fewer, an end marker)
    for (int i = whole + pieces + tid; i < a.num_ctas; i += kPlanThreads) a.pieces[i].tiles = -1;
    if (tid == 0) *a.control = {a.num_ctas, whole + pieces, cuts, sh_shapes};
}

constexpr int kRing = 2;                          // pieces a CTA has in hand: the one at work and the next
constexpr int kRingUsers = kSoftmaxWarps + 2;     // arrivals that free one: the softmax warps, the producer, the MMA issuer

// What the roles share, behind the tiles in shared memory.
template <int D>
struct Shared {
    Piece piece[kRing];
    Span span[kRing];
    uint64_t ring_full[kRing], ring_empty[kRing];
    uint64_t taken;  // the producer has all copies of a piece under way: time to look for the next
    uint64_t k_full[k_slots(D)], k_empty[k_slots(D)], v_full[v_slots(D)], v_empty[v_slots(D)];
    uint64_t q_full, q_empty, s_full[2], p_full[2], o_full[2], drain;
    uint64_t pair[2][4];              // the two warps that share a quarter of a stream's rows
    uint32_t flag[2][2][2][4];        // [turn][stream][half][quarter]: a score outgrew its row's reference
    float sum[2][2][128];             // [stream][half][row]
    uint32_t tmem;
    int abort;
};
template <int D>
constexpr int smem_bytes() {
    return (2 + k_slots(D) + v_slots(D)) * tile_bytes(D) + (int)sizeof(Shared<D>);
}

// A whole warp's wait.  What happens when the barrier is not there yet is kept out of line, or a dozen copies of it crowd the
// loops out of the instruction cache.
__device__ __noinline__ bool wait_longer(uint64_t* bar, uint32_t parity, volatile int* abort, long long limit) {
    return __all_sync(0xffffffffu, mbar_wait_bounded(bar, parity, WaitCtx{abort, limit}));
}
__device__ __forceinline__ bool role_wait(uint64_t* bar, uint32_t parity, const WaitCtx& wc) {
    return __all_sync(0xffffffffu, mbar_try_wait(bar, parity)) || wait_longer(bar, parity, wc.abort, wc.limit);
}

__device__ __forceinline__ void tmem_wait_ld_of(uint32_t (&r)[32]) {  // (ties the registers to the wait)
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                   "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]),
                   "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]),
                   "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
                 :
                 : "memory");
}

// Bits lo .. hi (of 0 .. 31) of a word; lo and hi may lie outside.
__device__ __forceinline__ uint32_t bits(int lo, int hi) {
    const int from = max(lo, 0), n = max(hi - from + 1, 0);
    uint32_t r;
    asm("bmsk.clamp.b32 %0, %1, %2;" : "=r"(r) : "r"(from), "r"(n));
    return r;
}

// A V row that no row of a unit sees may hold any bits, and 0 * NaN is NaN.  A stream's softmax warps zero those of a tile: past the keys
// and, in the last tile of the sinks and the first one of the window, between the two.  Few tiles have any: kept out of the loop's way
// (32,768 rows through a window 2,131 us, 2,153 in line; 2,102 without the rows between).
template <int D>
__device__ __noinline__ bool zero_hidden(uint8_t* v, Shared<D>& sh, const PrefillArgs& a, int ring, int key0, int tile, WaitCtx wc) {
    const Piece& g = sh.piece[ring];
    const int end = min(g.L - key0, kKeys), from = max(a.sink - key0, 0);
    const int to = min(max(g.L - g.n + g.row0 - a.window + 1, 0) - key0, kKeys);
    const int between = max(to - from, 0), chunks = (between + kKeys - end) * 8;
    if (chunks == 0) return true;
    const int slot = tile % v_slots(D);
    if (!role_wait(&sh.v_full[slot], (tile / v_slots(D)) & 1, wc)) return false;
    for (int ch = threadIdx.x & 255; ch < chunks; ch += 256) {
        const int r = ch >> 3, at = (r < between ? from + r : end + r - between) * 128 + (ch & 7) * 16;
#pragma unroll
        for (int h = 0; h < D / 64; ++h) *reinterpret_cast<uint4*>(v + slot * tile_bytes(D) + h * kHalfBytes + at) = make_uint4(0, 0, 0, 0);
    }
    fence_proxy_async_smem();
    return true;
}

// WINDOW: the call has window_keys.  A kernel of its own for it: with one for both, calls without a window took longer for the code that
// finds hidden V rows (32 rows over 32,000 keys, batch of one: 44.6 us without, 46.0 with, 44.8 apart).
template <int D, bool WINDOW>
__global__ void __launch_bounds__(kThreads, 1)
prefill_attn_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                    const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ PrefillArgs a) {
    constexpr int NH = D / 64;
    constexpr int NK = k_slots(D), NV = v_slots(D);
    constexpr uint32_t TILE = tile_bytes(D);
    constexpr uint32_t OFF_Q = 0, OFF_K = 2 * TILE, OFF_V = OFF_K + NK * TILE, OFF_SHARED = OFF_V + NV * TILE;
    constexpr uint32_t TMEM_COLS = 512, COL_S = 0, COL_O = 256;  // stream s: S at COL_S + 128 s, O at COL_O + 128 s
    constexpr int kProducer = kSoftmaxWarps, kWalk = kProducer + 1, kIssuer = kProducer + 2;

    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t smem_base = smem_u32(smem);
    Shared<D>& sh = *reinterpret_cast<Shared<D>*>(smem + OFF_SHARED);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (smem_base & 1023) {  // (the swizzled tiles need it; the declaration asks for it)
        if (threadIdx.x == 0) atomicOr(a.status, RAPID_STATUS_PIPELINE_TIMEOUT);
        return;
    }

    if (threadIdx.x == 0) {
        for (int i = 0; i < NK; ++i) mbar_init(&sh.k_full[i], 1), mbar_init(&sh.k_empty[i], 1);
        for (int i = 0; i < NV; ++i) mbar_init(&sh.v_full[i], 1), mbar_init(&sh.v_empty[i], 1);
        mbar_init(&sh.q_full, 1);
        mbar_init(&sh.q_empty, 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.s_full[i], 1);
            mbar_init(&sh.p_full[i], kSoftmaxWarps / 2);
            mbar_init(&sh.o_full[i], 1);
            for (int q = 0; q < 4; ++q) mbar_init(&sh.pair[i][q], 2);
        }
        mbar_init(&sh.drain, 1);
        for (int i = 0; i < kRing; ++i) mbar_init(&sh.ring_full[i], 1), mbar_init(&sh.ring_empty[i], kRingUsers);
        mbar_init(&sh.taken, 1);
        fence_mbar_init();
        sh.abort = 0;
    }
    if (warp == kProducer && lane == 0) {
        prefetch_tensormap(&tmK);
        prefetch_tensormap(&tmV);
        prefetch_tensormap(&tmQ);
    }
    if (warp == kIssuer) tmem_alloc(&sh.tmem, TMEM_COLS);  // the same warp frees it
    griddep_wait();
    griddep_launch_dependents();
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = sh.tmem;
    const WaitCtx wc = {&sh.abort, a.wait_limit};

    int r = 0;  // pieces taken from the ring; a role that comes to the end marker, or whose wait runs out, stops
    if (warp == kProducer) {
        // ---------------- producer: the unit's Q tiles and its K/V tiles ----------------
        int n_q = 0, n_k = 0, n_v = 0;  // copies issued
        const int parts = kKeys / a.box_rows;
        const uint32_t part_bytes = kHalfBytes / parts;
        bool ok = true;
        while (ok) {
            ok = role_wait(&sh.ring_full[r % kRing], (r / kRing) & 1, wc);
            const Piece g = sh.piece[r % kRing];
            const Span sp = sh.span[r % kRing];
            if (!ok || g.tiles < 0) break;
            const int oldest = WINDOW ? g.L - g.n + g.row0 - a.window + 1 : 0;  // key of the unit's windows
#pragma unroll 1
            for (int t = 0; t < g.tiles && ok; ++t) {
                const int u = g.first + t;
                const int key0 = (u < sp.sinks ? u : sp.lo + u - sp.sinks) * kKeys;
                int c1[2] = {key0, 0}, c3[2] = {g.b, g.b};
                if (a.block_table) {
#pragma unroll 1
                    for (int q = 0; q < parts; ++q) {
                        const int pos = key0 + q * a.box_rows;
                        c1[q] = pos & (a.block_size - 1);
                        if (pos >= g.L || (WINDOW && pos >= a.sink && pos + a.box_rows <= oldest)) {
                            c3[q] = a.num_blocks;  // past the keys, or hidden from the unit: zeros, no table entry is read
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
                if (n_k >= NK) ok = role_wait(&sh.k_empty[ks], (n_k / NK - 1) & 1, wc);
                if (!ok) break;
                if (elect_one()) {
                    mbar_arrive_expect_tx(&sh.k_full[ks], TILE);
#pragma unroll 1
                    for (int q = 0; q < parts; ++q)
#pragma unroll 1
                        for (int h = 0; h < NH; ++h)
                            tma_load_4d(smem + OFF_K + ks * TILE + h * kHalfBytes + q * part_bytes, &tmK, &sh.k_full[ks],
                                        h * 64, c1[q], g.kvh, c3[q]);
                }
                __syncwarp();
                ++n_k;
                if (t == 0) {  // (behind the first K tile, which need not wait for the unit before)
                    if (n_q > 0) ok = role_wait(&sh.q_empty, (n_q - 1) & 1, wc);
                    if (!ok) break;
                    const int streams = g.n - g.row0 > a.rows_tile ? 2 : 1;
                    if (elect_one()) {
                        mbar_arrive_expect_tx(&sh.q_full, (uint32_t)(streams * a.rows_tile * a.G * D * 2));
#pragma unroll 1
                        for (int s = 0; s < streams; ++s)
#pragma unroll 1
                            for (int h = 0; h < NH; ++h)
                                tma_load_4d(smem + OFF_Q + s * TILE + h * kHalfBytes, &tmQ, &sh.q_full, h * 64, g.kvh * a.G,
                                            g.row0 + s * a.rows_tile, g.b);
                    }
                    __syncwarp();
                    ++n_q;
                }
                if (n_v >= NV) ok = role_wait(&sh.v_empty[vs], (n_v / NV - 1) & 1, wc);
                if (!ok) break;
                if (elect_one()) {
                    mbar_arrive_expect_tx(&sh.v_full[vs], TILE);
#pragma unroll 1
                    for (int q = 0; q < parts; ++q)
#pragma unroll 1
                        for (int h = 0; h < NH; ++h)
                            tma_load_4d(smem + OFF_V + vs * TILE + h * kHalfBytes + q * part_bytes, &tmV, &sh.v_full[vs],
                                        h * 64, c1[q], g.kvh, c3[q]);
                }
                __syncwarp();
                ++n_v;
            }
            if (lane == 0) {
                mbar_arrive(&sh.ring_empty[r % kRing]);
                mbar_arrive(&sh.taken);
            }
            __syncwarp();
            ++r;
        }
        // every copy lands before the CTA gives up its shared memory, whoever may have given up waiting for it
        if (n_q > 0) mbar_wait_drain(&sh.q_full, (n_q - 1) & 1);
#pragma unroll 1
        for (int s = 0; s < NK && s < n_k; ++s) mbar_wait_drain(&sh.k_full[(n_k - 1 - s) % NK], ((n_k - 1 - s) / NK) & 1);
#pragma unroll 1
        for (int s = 0; s < NV && s < n_v; ++s) mbar_wait_drain(&sh.v_full[(n_v - 1 - s) % NV], ((n_v - 1 - s) / NV) & 1);
    } else if (warp == kWalk) {
        // ---------------- the walk: pieces from the list into the ring ----------------
        int i = blockIdx.x, pieces = i + 1;  // (how many there are is asked for beside the first)
        for (int k = 0;; ++k) {
            const int s = k % kRing;
            if (k >= kRing && !role_wait(&sh.ring_empty[s], (k / kRing - 1) & 1, wc)) break;
            if (k > 0) {
                if (!role_wait(&sh.taken, (k - 1) & 1, wc)) break;
                if (lane == 0) i = atomicAdd(&a.control->next, 1);
                i = __shfl_sync(0xffffffffu, i, 0);
            }
            const int known = pieces;
            if (k == 0) pieces = a.control->pieces;
            if (lane == 0) {
                if (i < known) {
                    const Piece g = a.pieces[i];
                    sh.piece[s] = g;
                    sh.span[s] = span_of(a, g.row0, g.n, g.L);
                } else {
                    sh.piece[s].tiles = -1;
                }
                mbar_arrive(&sh.ring_full[s]);
            }
            __syncwarp();
            if (i >= pieces) break;
        }
    } else if (warp == kIssuer) {
        // ---------------- MMA issuer: a warp in step, of which one lane issues ----------------
        constexpr uint32_t idesc_qk = umma_idesc_bf16(128, kKeys, 0, 0);
        constexpr uint32_t idesc_pv = umma_idesc_bf16(128, D, 0, 1);
        const bool leader = elect_one();
        const uint64_t q_desc = umma_smem_desc(smem_base + OFF_Q, 16, 1024);
        const uint64_t k_desc = umma_smem_desc(smem_base + OFF_K, 16, 1024);
        const uint64_t v_desc = umma_smem_desc(smem_base + OFF_V, kHalfBytes, 1024);
        int n_q = 0, n_k = 0, n_v = 0;  // units and tiles so far
        int p_par[2] = {0, 0};
        bool ok = true;
        while (ok) {
            ok = warp_wait(&sh.ring_full[r % kRing], (r / kRing) & 1, wc);
            const int tiles = __shfl_sync(0xffffffffu, sh.piece[r % kRing].tiles, 0);
            const int streams = __shfl_sync(0xffffffffu, sh.piece[r % kRing].n - sh.piece[r % kRing].row0, 0) > a.rows_tile ? 2 : 1;
            if (!ok || tiles < 0) break;
            if (tiles > 0) {
                ok = warp_wait(&sh.q_full, n_q & 1, wc);
                ++n_q;
            }
#pragma unroll 1
            for (int t = 0; t <= tiles && tiles > 0 && ok; ++t) {
                const int ks = n_k % NK, vs = n_v % NV;
                if (t > 0) ok = warp_wait(&sh.v_full[vs], (n_v / NV) & 1, wc);
                if (t < tiles) ok = ok && warp_wait(&sh.k_full[ks], (n_k / NK) & 1, wc);
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    if (s >= streams) continue;
                    const uint32_t tS = tmem + COL_S + 128u * s, tO = tmem + COL_O + 128u * s;
                    if (t > 0) {
                        ok = ok && warp_wait(&sh.p_full[s], p_par[s], wc);
                        p_par[s] ^= 1;
                        tc_fence_after_sync();
                        if (ok && leader) {
                            const uint64_t vd = v_desc + (uint32_t)vs * (TILE >> 4);
#pragma unroll
                            for (int kk = 0; kk < kKeys / 16; ++kk)
                                umma_bf16_ts(tO, tS + 8 * kk, vd + kk * (2048 >> 4), idesc_pv, (t > 1 || kk > 0) ? 1u : 0u);
                            if (t == tiles) umma_commit(&sh.o_full[s]);
                        }
                        __syncwarp();
                    }
                    if (t < tiles) {
                        tc_fence_after_sync();
                        if (ok && leader) {
                            const uint64_t qd = q_desc + (uint32_t)s * (TILE >> 4), kd = k_desc + (uint32_t)ks * (TILE >> 4);
#pragma unroll
                            for (int kk = 0; kk < D / 16; ++kk) {
                                const uint32_t off = (kk >> 2) * (kHalfBytes >> 4) + (kk & 3) * 2;
                                umma_bf16_ss(tS, qd + off, kd + off, idesc_qk, kk > 0);
                            }
                            umma_commit(&sh.s_full[s]);
                        }
                        __syncwarp();
                    }
                }
                if (ok && leader) {
                    if (t < tiles) umma_commit(&sh.k_empty[ks]);
                    if (t == tiles - 1) umma_commit(&sh.q_empty);
                    if (t > 0) umma_commit(&sh.v_empty[vs]);
                }
                __syncwarp();
                n_k += t < tiles;
                n_v += t > 0;
            }
            if (!ok) break;
            if (lane == 0) mbar_arrive(&sh.ring_empty[r % kRing]);
            __syncwarp();
            ++r;
        }
        // every MMA issued here has completed before tensor memory is freed
        if (leader) {
            umma_commit(&sh.drain);
            const long long t0 = clock64();
            while (!mbar_try_wait(&sh.drain, 0) && clock64() - t0 < kWaitCycleLimit) {}
        }
        __syncwarp();
    } else {
        // ---------------- softmax warps: stream, half of a tile's keys, quarter of its rows ----------------
        const int stream = warp >> 3, half = warp >> 2 & 1, quarter = warp & 3;
        const int row = quarter * 32 + lane;
        const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
        const uint32_t tS = tmem + lane_base + COL_S + 128u * stream, tO = tmem + lane_base + COL_O + 128u * stream + half * (D / 2);
        uint64_t* pair = &sh.pair[stream][quarter];
        const float c = a.scale_log2;
        const int row_t = row / a.G, row_h = row - row_t * a.G;  // row of the sequence within the tile, head in the group
        int j = 0, n_tiles = 0, done = 0;  // tiles of this stream, tiles of the CTA before the piece, pieces of this stream
        int met = 0;                       // times that the two warps of a quarter have met
        bool ok = true;
        while (ok) {
            ok = role_wait(&sh.ring_full[r % kRing], (r / kRing) & 1, wc);
            const Piece g = sh.piece[r % kRing];
            const Span sp = sh.span[r % kRing];
            if (!ok || g.tiles < 0) break;
            const int i0 = g.row0 + stream * a.rows_tile;  // the tile's first row of the sequence
            if (i0 < g.n) {
                const bool row_valid = row_t < a.rows_tile && i0 + row_t < g.n;
                const bool warp_valid = __any_sync(0xffffffffu, row_valid);
                // the keys j of a row: wlo <= j <= lim, or j < sink; and those that all rows of the tile see
                const int p0 = g.L - g.n + i0;
                const int lim = a.all_visible ? g.L - 1 : p0 + row_t;
                const int wlo = WINDOW ? lim - a.window + 1 : 0;
                const int all_lim = a.all_visible ? g.L - 1 : p0;
                const int all_lo = WINDOW ? p0 + a.rows_tile - 1 - a.window + 1 : 0;
                float m_ref = -INFINITY, l_run = 0.f;
#pragma unroll 1
                for (int t = 0; t < g.tiles; ++t, ++j) {
                    ok = role_wait(&sh.s_full[stream], j & 1, wc);
                    if (!ok) break;
                    const int u = g.first + t;
                    const int key0 = (u < sp.sinks ? u : sp.lo + u - sp.sinks) * kKeys;
                    tc_fence_after_sync();
                    if (warp_valid) {
                        const bool masked = key0 + kKeys - 1 > all_lim || (key0 < all_lo && key0 + kKeys > a.sink);
                        uint32_t x[32], pk[32];
                        float mx[2];
                        uint64_t acc[2];
                        auto load = [&](int q) {  // the scores of keys 32 q .. 32 q + 31 of the tile, those out of sight -inf
                            tmem_ld_x32(tS + 32 * q, x);
                            tmem_wait_ld_of(x);
                            if (masked) {
                                const int k0 = key0 + 32 * q;
                                const uint32_t seen = bits(wlo - k0, lim - k0) | bits(0, min(a.sink - 1, lim) - k0);
#pragma unroll
                                for (int k = 0; k < 32; ++k)
                                    if (!(seen >> k & 1)) x[k] = __float_as_uint(-INFINITY);
                            }
                        };
                        auto largest = [&] {
#pragma unroll
                            for (int k = 0; k < 32; k += 2) mx[(k >> 1) & 1] = max3(mx[(k >> 1) & 1], __uint_as_float(x[k]), __uint_as_float(x[k + 1]));
                        };
                        auto weigh = [&](int at) {  // by the reference in place
                            const float m_use = m_ref == -INFINITY ? 0.f : m_ref;
                            const uint64_t c2 = f32x2(c, c), m2 = f32x2(-m_use, -m_use);
#pragma unroll
                            for (int k = 0; k < 32; k += 2) {
                                float p0, p1;
                                f32x2_split(f32x2_fma(f32x2(__uint_as_float(x[k]), __uint_as_float(x[k + 1])), c2, m2), p0, p1);
                                p0 = fast_exp2(p0);
                                p1 = fast_exp2(p1);
                                acc[(k >> 1) & 1] = f32x2_add(acc[(k >> 1) & 1], f32x2(p0, p1));
                                pk[at + (k >> 1)] = pack_bf16x2(p0, p1);
                            }
                        };
                        bool again = t == 0;  // no references yet
                        if (!again) {
                            acc[0] = acc[1] = 0;
                            mx[0] = mx[1] = -INFINITY;
                            auto tell = [&] {  // the other half of the keys; and neither warp writes over scores that the other has not read
                                const float top = max3(mx[0], mx[1], mx[1]) * c;
                                again = __any_sync(0xffffffffu, row_valid && !(top <= m_ref + kJump) && top != -INFINITY);
                                tc_fence_before_sync();
                                if (lane == 0) {
                                    sh.flag[met & 1][stream][half][quarter] = again;
                                    mbar_arrive(pair);
                                }
                            };
                            if (masked) {
                                load(2 * half);
                                largest();
                                weigh(0);
                                load(2 * half + 1);
                                largest();
                                tell();
                                weigh(16);
                            } else {  // straight through, with no test for masked keys between the halves
                                tmem_ld_x32(tS + 64 * half, x);
                                tmem_wait_ld_of(x);
                                largest();
                                weigh(0);
                                tmem_ld_x32(tS + 64 * half + 32, x);
                                tmem_wait_ld_of(x);
                                largest();
                                tell();
                                weigh(16);
                            }
                            ok = role_wait(pair, met & 1, wc);
                            if (!ok) break;
                            tc_fence_after_sync();
                            again |= *(volatile uint32_t*)&sh.flag[met & 1][stream][half ^ 1][quarter] != 0;
                            ++met;
                        }
                        if (again) {  // the references first, by the whole row, then the probabilities once more
                            mx[0] = mx[1] = -INFINITY;
#pragma unroll 1
                            for (int q = 0; q < kKeys / 32; ++q) {
                                const int k0 = key0 + 32 * q;  // (nothing to find where no row of the warp sees any key)
                                if (masked && !__any_sync(0xffffffffu, (bits(wlo - k0, lim - k0) | bits(0, min(a.sink - 1, lim) - k0)) != 0)) continue;
                                load(q);
                                largest();
                            }
                            const float top = max3(mx[0], mx[1], mx[1]) * c;
                            const bool move = row_valid && !(top <= m_ref + kJump) && top != -INFINITY;
                            const float factor = move ? fast_exp2(m_ref - top) : 1.f;  // 0 when there was no reference
                            if (move) {
                                l_run *= factor;
                                m_ref = top;
                            }
                            if (t > 0 && __any_sync(0xffffffffu, move)) scale_o<D / 2>(tO, factor);
                            acc[0] = acc[1] = 0;
                            load(2 * half);
                            weigh(0);
                            load(2 * half + 1);
                            weigh(16);
                            tc_fence_before_sync();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(pair);
                            ok = role_wait(pair, met & 1, wc);
                            if (!ok) break;
                            tc_fence_after_sync();
                            ++met;
                        }
                        tmem_st_x32(tS + 32 * half, pk);
                        float s0, s1;
                        f32x2_split(f32x2_add(acc[0], acc[1]), s0, s1);
                        l_run += s0 + s1;
                    }
                    if (WINDOW && (key0 + kKeys > g.L || u <= sp.sinks)) {
                        ok = zero_hidden<D>(smem + OFF_V, sh, a, r % kRing, key0, n_tiles + t, wc);
                        if (!ok) break;
                    } else if (key0 + kKeys > g.L) {  // V rows past the keys alone: the same in line
                        const int vt = n_tiles + t, vs = vt % NV;
                        ok = role_wait(&sh.v_full[vs], (vt / NV) & 1, wc);
                        if (!ok) break;
                        const int bad = g.L - key0;
                        const int chunks = (kKeys - bad) * 8;
#pragma unroll
                        for (int h = 0; h < NH; ++h)
                            for (int ch = half * 128 + row; ch < chunks; ch += 256)
                                *reinterpret_cast<uint4*>(smem + OFF_V + vs * TILE + h * kHalfBytes + bad * 128 + ch * 16) =
                                    make_uint4(0, 0, 0, 0);
                        fence_proxy_async_smem();
                    }
                    tmem_wait_st();
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.p_full[stream]);
                }
                if (!ok) break;
                // ---- the end of the piece: each warp has half of the columns ----
                if (g.tiles > 0) {
                    ok = role_wait(&sh.o_full[stream], done & 1, wc);
                    if (!ok) break;
                    ++done;
                    tc_fence_after_sync();
                    if (warp_valid) {
                        sh.sum[stream][half][row] = l_run;
                        __syncwarp();
                        if (lane == 0) mbar_arrive(pair);
                        ok = role_wait(pair, met & 1, wc);
                        if (!ok) break;
                        ++met;
                        l_run = sh.sum[stream][0][row] + sh.sum[stream][1][row];
                    }
                }
                const bool empty = m_ref == -INFINITY;  // the row saw no key
                const float inv = empty ? 0.f : 1.f / l_run;
                const size_t at = ((size_t)g.b * a.T + i0 + row_t) * a.Hq + (size_t)g.kvh * a.G + row_h;
                float* slot = a.slots + (size_t)max(g.slot, 0) * slot_floats(a.slot_rows, D);
                const int srow = stream * 128 + row;
#pragma unroll 1
                for (int q = 0; q < D / 64; ++q) {
                    uint32_t o[32] = {};
                    const int d0 = half * (D / 2) + 32 * q;
                    if (g.tiles > 0) {
                        tmem_ld_x32(tO + 32 * q, o);
                        tmem_wait_ld_of(o);
                    }
                    if (g.slot >= 0) {
                        if (row_valid) {
#pragma unroll
                            for (int k = 0; k < 32; k += 4)
                                *reinterpret_cast<uint4*>(slot + ((size_t)((d0 + k) / 4) * a.slot_rows + srow) * 4) =
                                    make_uint4(o[k], o[k + 1], o[k + 2], o[k + 3]);
                        }
                        __syncwarp();
                        continue;
                    }
#pragma unroll
                    for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * inv);
                    if (__any_sync(0xffffffffu, empty)) {
#pragma unroll
                        for (int k = 0; k < 32; ++k) o[k] = empty ? 0u : o[k];
                    }
                    if (row_valid) {
                        uint4* to = reinterpret_cast<uint4*>(a.out + at * D + d0);
#pragma unroll
                        for (int k = 0; k < 32; k += 8)
                            to[k / 8] = make_uint4(pack_bf16x2(__uint_as_float(o[k]), __uint_as_float(o[k + 1])),
                                                   pack_bf16x2(__uint_as_float(o[k + 2]), __uint_as_float(o[k + 3])),
                                                   pack_bf16x2(__uint_as_float(o[k + 4]), __uint_as_float(o[k + 5])),
                                                   pack_bf16x2(__uint_as_float(o[k + 6]), __uint_as_float(o[k + 7])));
                        if (a.out_f32) {
#pragma unroll
                            for (int k = 0; k < 32; k += 4)
                                *reinterpret_cast<uint4*>(a.out_f32 + at * D + d0 + k) = make_uint4(o[k], o[k + 1], o[k + 2], o[k + 3]);
                        }
                    }
                    __syncwarp();
                }
                tc_fence_before_sync();
                if (row_valid && half == 0) {
                    if (g.slot >= 0) {
                        slot[(size_t)a.slot_rows * D + srow] = m_ref;
                        slot[(size_t)a.slot_rows * (D + 1) + srow] = l_run;
                    } else if (a.lse_out) {
                        a.lse_out[at] = empty ? -INFINITY : (m_ref + log2f(l_run)) * 0.69314718055994530942f;
                    }
                }
            }
            n_tiles += g.tiles;
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.ring_empty[r % kRing]);
            ++r;
        }
    }

    tc_fence_before_sync();
    __syncthreads();
    if (warp == kIssuer) {
        tc_fence_after_sync();
        tmem_dealloc(tmem, TMEM_COLS);
    }
    if (threadIdx.x == 0 && sh.abort) atomicOr(a.status, RAPID_STATUS_PIPELINE_TIMEOUT);
}

// Merge of the units that were cut: out = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s over a row's partials.  An item is
// 32 rows (lane = row) and 16 columns.  Where a unit has few parts, a block's warps take an item each (one round trip, nothing to
// join); where it has many, they split an item's parts.  The order of the sums is fixed either way.
struct MergeSum {
    float m, l;
    float4 acc[4];
};
// The parts first, first + step, ... of the item at rows srow, columns 4 d4 .. 4 d4 + 15; four of them in flight at a time.
__device__ __forceinline__ MergeSum merge_parts(const PrefillArgs& a, const float* base, size_t per, int D, int srow, int d4, bool valid,
                                                int first, int step, int parts) {
    constexpr int UN = 4;
    MergeSum r;
    r.m = -INFINITY;
    r.l = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) r.acc[j] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int x0 = first; x0 < parts; x0 += step * UN) {
        float ms[UN], ls[UN];
        float4 o[UN][4];
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            const int x = x0 + step * u;
            ms[u] = -INFINITY;
            if (x < parts && valid) {
                const float* s = base + (size_t)x * per;
                ms[u] = __ldcg(s + (size_t)a.slot_rows * D + srow);
                ls[u] = __ldcg(s + (size_t)a.slot_rows * (D + 1) + srow);
#pragma unroll
                for (int j = 0; j < 4; ++j) o[u][j] = __ldcg(reinterpret_cast<const float4*>(s) + (size_t)(d4 + j) * a.slot_rows + srow);
            }
        }
        float top = r.m;
#pragma unroll
        for (int u = 0; u < UN; ++u) top = max3(top, ms[u], ms[u]);
        const float keep = r.m == -INFINITY ? 0.f : exp2f(r.m - top);
        r.m = top;
        r.l *= keep;
#pragma unroll
        for (int j = 0; j < 4; ++j) r.acc[j].x *= keep, r.acc[j].y *= keep, r.acc[j].z *= keep, r.acc[j].w *= keep;
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            if (ms[u] == -INFINITY) continue;  // a part in which the row saw no key
            const float wgt = exp2f(ms[u] - top);
            r.l += wgt * ls[u];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                r.acc[j].x += wgt * o[u][j].x;
                r.acc[j].y += wgt * o[u][j].y;
                r.acc[j].z += wgt * o[u][j].z;
                r.acc[j].w += wgt * o[u][j].w;
            }
        }
    }
    return r;
}
// Four columns of row `sr` of a cut unit.
__device__ __forceinline__ void merge_write(const PrefillArgs& a, const Cut& g, int D, int sr, int d4, float M, float L, float4 v) {
    const int rt = (sr & 127) / a.G, rh = (sr & 127) - rt * a.G, i = g.row0 + (sr >> 7) * a.rows_tile + rt;
    if (rt >= a.rows_tile || i >= g.n) return;
    const size_t at = ((size_t)g.b * a.T + i) * a.Hq + (size_t)g.kvh * a.G + rh;
    const float inv = M == -INFINITY ? 0.f : 1.f / L;
    v = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
    *reinterpret_cast<uint2*>(a.out + at * D + d4 * 4) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
    if (a.out_f32) *reinterpret_cast<float4*>(a.out_f32 + at * D + d4 * 4) = v;
    if (a.lse_out && d4 == 0) a.lse_out[at] = M == -INFINITY ? -INFINITY : (M + log2f(L)) * 0.69314718055994530942f;
}
template <int D>
__global__ void __launch_bounds__(128) prefill_merge_kernel(const __grid_constant__ PrefillArgs a) {
    constexpr int W = 4, PER_ROWS = D / 64;  // 32 rows are 4 * PER_ROWS items
    __shared__ float4 sh_acc[W][4][32];
    __shared__ float sh_m[W][32], sh_l[W][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    griddep_wait();
    griddep_launch_dependents();
    const int groups = a.slot_rows / 32;
    const Control ctl = *a.control;
    const size_t per = slot_floats(a.slot_rows, D);
    if (ctl.shapes & kSomeFew) {
        for (int quad = blockIdx.x; quad < ctl.cuts * groups * PER_ROWS; quad += gridDim.x) {
            const Cut g = a.cuts[quad / (groups * PER_ROWS)];
            if (g.parts > kFewParts) continue;
            const int rest = quad % (groups * PER_ROWS);
            const int srow = rest / PER_ROWS * 32 + lane, d4 = (rest % PER_ROWS * 4 + warp) * 4, rt = (srow & 127) / a.G;
            const bool valid = rt < a.rows_tile && g.row0 + (srow >> 7) * a.rows_tile + rt < g.n;
            const MergeSum r = merge_parts(a, a.slots + (size_t)g.slot * per, per, D, srow, d4, valid, 0, 1, g.parts);
#pragma unroll
            for (int j = 0; j < 4; ++j) merge_write(a, g, D, srow, d4 + j, r.m, r.l, r.acc[j]);
        }
    }
    if (!(ctl.shapes & kSomeMany)) return;
    for (int item = blockIdx.x; item < ctl.cuts * groups * PER_ROWS * 4; item += gridDim.x) {
        const Cut g = a.cuts[item / (groups * PER_ROWS * 4)];
        if (g.parts <= kFewParts) continue;
        const int rest = item % (groups * PER_ROWS * 4);
        const int srow0 = rest / (PER_ROWS * 4) * 32, d4 = rest % (PER_ROWS * 4) * 4;
        const int srow = srow0 + lane, rt = (srow & 127) / a.G;
        const bool valid = rt < a.rows_tile && g.row0 + (srow >> 7) * a.rows_tile + rt < g.n;
        const MergeSum r = merge_parts(a, a.slots + (size_t)g.slot * per, per, D, srow, d4, valid, warp, W, g.parts);
        __syncthreads();  // (the item before has been read)
        sh_m[warp][lane] = r.m;
        sh_l[warp][lane] = r.l;
#pragma unroll
        for (int j = 0; j < 4; ++j) sh_acc[warp][j][lane] = r.acc[j];
        __syncthreads();
        // four neighbouring threads write the 16 columns of a row
        const int row = threadIdx.x >> 2, j = threadIdx.x & 3;
        float M = -INFINITY, L = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) M = max3(M, sh_m[w][row], sh_m[w][row]);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < W; ++w) {
            if (sh_m[w][row] == -INFINITY) continue;
            const float wgt = exp2f(sh_m[w][row] - M);
            const float4 o = sh_acc[w][j][row];
            L += wgt * sh_l[w][row];
            v.x += wgt * o.x;
            v.y += wgt * o.y;
            v.z += wgt * o.z;
            v.w += wgt * o.w;
        }
        merge_write(a, g, D, srow0 + row, d4 + j, M, L, v);
    }
}

// ---- host side ----------------------------------------------------------------------------

// Scratch.  The place of a verify plan's signature is kept free, and every call takes such a plan back by its first word: what is
// written here overwrites its walks.
struct WsLayout {
    size_t plan_sig, control, seq_start, pieces, cuts, slots, total;
    int max_slots, slot_rows;
};
bool shape_ok(const rapid_attn_shape* s, int T) {
    return s && s->B > 0 && s->Hq > 0 && s->Hkv > 0 && s->Lmax >= 0 && s->Lmax <= kMaxKeys && T > 0 && s->Hq % s->Hkv == 0 && (s->D == 64 || s->D == 128) &&
           s->Hq / s->Hkv <= 128 && s->B <= 65535 && s->Hkv <= 65535 && T <= (1 << 30);
}
int64_t units_of(const rapid_attn_shape* s, int T) {
    const int64_t rows = 2 * (128 / (s->Hq / s->Hkv));
    return (int64_t)s->B * s->Hkv * ((T + rows - 1) / rows);
}
WsLayout ws_layout(const rapid_attn_shape* s, int T) {
    WsLayout l;
    size_t off = kWorkspaceHeaderBytes;
    l.plan_sig = off;
    off += 256;
    l.control = off;
    off += 256;
    l.seq_start = off;
    off += align_up((size_t)(s->B + 1) * sizeof(int32_t), 256);
    l.pieces = off;
    off += align_up((size_t)(units_of(s, T) + kMaxTail) * sizeof(Piece), 256);
    l.cuts = off;
    off += kPlanThreads * sizeof(Cut);
    l.slots = off;
    l.slot_rows = T > 128 / (s->Hq / s->Hkv) ? 256 : 128;
    // partials: no unit of the tail is cut into more than its tiles, and none of one or two tiles is cut
    const int64_t tiles = ((s->Lmax ? s->Lmax : kMaxKeys) + kKeys - 1) / kKeys, tail = units_of(s, T) < kPlanThreads ? units_of(s, T) : kPlanThreads;
    l.max_slots = tiles <= 2 ? 0 : tail * tiles < kMaxTail ? (int)(tail * tiles) : kMaxTail;
    off += l.max_slots * slot_floats(l.slot_rows, s->D) * sizeof(float);
    l.total = off;
    return l;
}

template <int D, bool WINDOW>
int launch(const CUtensorMap (&tm)[3], const PrefillArgs& a, int sms, void* split_done, cudaStream_t stream) {
    constexpr int smem = smem_bytes<D>();
    static_assert(smem <= 232448, "shared memory");
    int dev = 0;
    RAPID_CUDA_CHECK(cudaGetDevice(&dev));
    static std::atomic<bool> configured[64];  // (first calls may come from several threads at once; all set the same)
    if (dev >= 64 || !configured[dev]) {
        RAPID_CUDA_CHECK(cudaFuncSetAttribute(prefill_attn_kernel<D, WINDOW>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        if (dev < 64) configured[dev] = true;
    }
    RAPID_CUDA_CHECK(launch_dependent(prefill_plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, a));
    RAPID_CUDA_CHECK(launch_dependent(prefill_attn_kernel<D, WINDOW>, dim3(a.num_ctas), dim3(kThreads), (size_t)smem, stream, tm[0], tm[1],
                                      tm[2], a));
    if (split_done) RAPID_CUDA_CHECK(cudaEventRecord(static_cast<cudaEvent_t>(split_done), stream));
    RAPID_CUDA_CHECK(launch_dependent(prefill_merge_kernel<D>, dim3(8 * sms), dim3(128), 0, stream, a));
    count_launch(3);
    return RAPID_OK;
}

}  // namespace

size_t prefill_attention_workspace_bytes(const rapid_attn_shape* s, int T) {
    return shape_ok(s, T) && units_of(s, T) <= kMaxUnits ? ws_layout(s, T).total : 0;
}

int launch_prefill_attention(const void* q, const rapid_kv_rows* q_rows, int T, const int32_t* n_tokens, const void* k_cache,
                             const void* v_cache, const rapid_paged_kv* paged, const int32_t* block_table,
                             const int32_t* ctx_lens, void* out, const rapid_attn_shape* shape,
                             const rapid_attn_params* params, void* workspace, size_t workspace_bytes, cudaStream_t stream) {
    const char* who = paged ? "rapid_prefill_attention_paged" : "rapid_prefill_attention";
    if (!q || !k_cache || !v_cache || !ctx_lens || !out || !shape) {
        set_error("%s: NULL argument", who);
        return RAPID_ERR_INVALID_ARG;
    }
    const rapid_attn_shape& s = *shape;
    if (s.B <= 0 || s.Hq <= 0 || s.Hkv <= 0 || s.Lmax <= 0 || T <= 0 || s.Hq % s.Hkv || s.Lmax > kMaxKeys) {
        set_error("%s: invalid shape (B=%d Hq=%d Hkv=%d Lmax=%lld T=%d)", who, s.B, s.Hq, s.Hkv, (long long)s.Lmax, T);
        return RAPID_ERR_INVALID_ARG;
    }
    if (!shape_ok(shape, T) || units_of(shape, T) > kMaxUnits) {
        set_error("%s: head_dim must be 64 or 128, Hq/Hkv at most 128, B and Hkv at most 65535, and B * Hkv * T / (2 * (128 / (Hq/Hkv))) "
                  "at most 2^24", who);
        return RAPID_ERR_UNSUPPORTED;
    }
    if (params && (params->kernel || params->plan || params->kv_fp8 || params->kv_settled)) {
        set_error("%s: of params only scale, num_ctas, lse_out, out_f32, split_done_event, all_keys_visible, sink_keys, window_keys and "
                  "wait_cycle_limit apply", who);
        return RAPID_ERR_UNSUPPORTED;
    }
    const bool all_visible = params && params->all_keys_visible;
    int sink = params ? params->sink_keys : 0, window = params ? params->window_keys : 0;
    if (sink < 0 || window < 0 || (sink > 0 && window == 0) || (window > 0 && all_visible)) {
        set_error("%s: sink_keys and window_keys must not be negative, sink_keys needs a window, and a window cannot be combined with "
                  "all_keys_visible", who);
        return RAPID_ERR_INVALID_ARG;
    }
    // (a window as long as the cache hides nothing; below that the differences of keys and windows stay within 32 bits)
    if (window >= s.Lmax) sink = window = 0;
    const int G = s.Hq / s.Hkv;
    int64_t sl, sh, sb, keys, outer;
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
    } else {
        sl = s.kv_stride_l ? s.kv_stride_l : s.D;
        sh = s.kv_stride_h ? s.kv_stride_h : s.Lmax * sl;
        sb = s.kv_stride_b ? s.kv_stride_b : s.Hkv * sh;
        keys = s.Lmax;
        outer = s.B;
    }
    const int64_t qh = q_rows && q_rows->stride_h ? q_rows->stride_h : s.D;
    const int64_t qt = q_rows && q_rows->stride_t ? q_rows->stride_t : (int64_t)s.Hq * s.D;
    const int64_t qb = q_rows && q_rows->stride_b ? q_rows->stride_b : (int64_t)T * s.Hq * s.D;
    if (sl < s.D || sl % 8 || sh % 8 || sb % 8 || sh <= 0 || sb <= 0 || qh % 8 || qt % 8 || qb % 8 || qh <= 0 || qt <= 0 || qb <= 0) {
        set_error("%s: strides must be positive multiples of 8 elements", who);
        return RAPID_ERR_UNSUPPORTED;
    }
    float* lse = params ? params->lse_out : nullptr;
    float* o32 = params ? params->out_f32 : nullptr;
    if (((uintptr_t)k_cache | (uintptr_t)v_cache | (uintptr_t)q | (uintptr_t)out | (uintptr_t)o32) & 15) {
        set_error("%s: q, out, out_f32 and the caches must be 16-byte aligned", who);
        return RAPID_ERR_UNSUPPORTED;
    }
    const WsLayout lay = ws_layout(shape, T);
    if (!workspace || workspace_bytes < lay.total || ((uintptr_t)workspace & 255)) {
        set_error("%s: workspace of %zu bytes needed (256-byte aligned), got %zu", who, lay.total, workspace_bytes);
        return RAPID_ERR_WORKSPACE;
    }
    int num_ctas = params ? params->num_ctas : 0;
    if (num_ctas < 0 || num_ctas > kMaxPrefillCtas) {
        set_error("%s: num_ctas %d outside [0, %d]", who, num_ctas, kMaxPrefillCtas);
        return RAPID_ERR_INVALID_ARG;
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
    int dev = 0, sms = 0;
    RAPID_CUDA_CHECK(cudaGetDevice(&dev));
    RAPID_CUDA_CHECK(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    if (!num_ctas) num_ctas = sms < kMaxPrefillCtas ? sms : kMaxPrefillCtas;

    uint8_t* ws = static_cast<uint8_t*>(workspace);
    PrefillArgs a = {};
    a.ctx_lens = ctx_lens;
    a.n_tokens = n_tokens;
    a.block_table = paged ? block_table : nullptr;
    a.control = reinterpret_cast<Control*>(ws + lay.control);
    a.seq_start = reinterpret_cast<int32_t*>(ws + lay.seq_start);
    a.pieces = reinterpret_cast<Piece*>(ws + lay.pieces);
    a.cuts = reinterpret_cast<Cut*>(ws + lay.cuts);
    a.slots = reinterpret_cast<float*>(ws + lay.slots);
    a.status = reinterpret_cast<int32_t*>(ws);
    a.plan_sig = reinterpret_cast<int32_t*>(ws + lay.plan_sig);
    a.out = static_cast<__nv_bfloat16*>(out);
    a.out_f32 = o32;
    a.lse_out = lse;
    a.B = s.B;
    a.T = T;
    a.G = G;
    a.Hq = s.Hq;
    a.Hkv = s.Hkv;
    a.Lmax = (int)s.Lmax;
    a.block_size = paged ? paged->block_size : 0;
    a.block_log2 = block_log2;
    a.num_blocks = paged ? paged->num_blocks : 0;
    a.max_blocks = paged ? paged->max_blocks_per_seq : 0;
    a.box_rows = paged && paged->block_size < kKeys ? 64 : kKeys;
    a.rows_tile = 128 / G;
    a.slot_rows = lay.slot_rows;
    a.max_slots = lay.max_slots;
    a.num_ctas = num_ctas;
    a.sink = sink;
    a.window = window;
    a.all_visible = all_visible;
    a.scale_log2 = scale * 1.4426950408889634f;
    a.wait_limit = wait_limit;

    CUtensorMap tm[3];
    int rc;
    if ((rc = make_map(&tm[0], k_cache, s.D, keys, s.Hkv, outer, sl, sh, sb, a.box_rows, 1)) != RAPID_OK) return rc;
    if ((rc = make_map(&tm[1], v_cache, s.D, keys, s.Hkv, outer, sl, sh, sb, a.box_rows, 1)) != RAPID_OK) return rc;
    // q as [B, T, Hq, D]: a box of (64 columns, G heads, rows_tile rows) is a row tile, row index t * G + g
    if ((rc = make_map(&tm[2], q, s.D, s.Hq, T, s.B, qh, qt, qb, G, a.rows_tile)) != RAPID_OK) return rc;
    void* ev = params ? params->split_done_event : nullptr;
    if (window) return s.D == 128 ? launch<128, true>(tm, a, sms, ev, stream) : launch<64, true>(tm, a, sms, ev, stream);
    return s.D == 128 ? launch<128, false>(tm, a, sms, ev, stream) : launch<64, false>(tm, a, sms, ev, stream);
}

}  // namespace rapid
