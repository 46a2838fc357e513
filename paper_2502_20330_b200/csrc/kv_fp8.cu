// The FP8 KV cache around the verify step: quantising rows as they are written (a prompt's, a step's) and reading
// chunks of it back in bf16.  The cache is the one rapid_verify_attention_fp8 reads: E4M3 codes
// [B, Hkv, Lmax, D] and one fp32 scale per (sequence, KV head) for K and one for V; x = scale * decode(code).
//
//   fill     scale = 2^headroom * the smallest power of two with amax <= 448 * scale, over the prompt's rows of the
//            (sequence, KV head); code = E4M3(x / scale), to nearest even.  With a power of two the division is exact
//            (one rounding, the code's own) and so is the read-back (a code has 4 significant bits, bf16 8); codes
//            being floating-point it costs no precision, only up to one binade at the small end of the range.
//   append   code = E4M3(clamp(x / scale, +-448)) with the scales in place
//   read     bf16(scale * decode(code)), the product in fp32
//
// All are bound by memory (2 + 1 bytes an element) or, for a step's few rows, by latency.
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <math.h>

#include <atomic>

#include "common.cuh"
#include "prefix_kv8.cuh"

namespace rapid {

namespace {

constexpr float kE4m3Max = 448.f;

struct RowsIn {  // rows to be written: [B, T, Hkv, D] bf16 by element strides, D contiguous
    const __nv_bfloat16* k;
    const __nv_bfloat16* v;
    long long sb, st, sh;
};
struct Cache8 {
    uint8_t* k;
    uint8_t* v;
    long long sb, sh, sl, Lmax;
};

// 8 bf16 of a row -> 8 codes.  What lies beyond the largest code saturates, infinities included; NaN stays NaN.
__device__ __forceinline__ uint2 quantise8(const uint4& v, float scale, bool& clipped) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float lo = __fdiv_rn(__uint_as_float(w[i] << 16), scale), hi = __fdiv_rn(__uint_as_float(w[i] & 0xffff0000u), scale);
        clipped |= fabsf(lo) > kE4m3Max || fabsf(hi) > kE4m3Max;
        c[i] = __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
    }
    return make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
}
// The same for a scale that is a power of two, `inv` its reciprocal (twice in 64 bits): two products an instruction.
__device__ __forceinline__ uint2 quantise8_pow2(const uint4& v, uint64_t inv) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint64_t x;
        float2 y;
        asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "r"(w[i] << 16), "r"(w[i] & 0xffff0000u));
        asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(x) : "l"(inv));
        asm("mov.b64 {%0, %1}, %2;" : "=f"(y.x), "=f"(y.y) : "l"(x));
        c[i] = __nv_cvt_float2_to_fp8x2(y, __NV_SATFINITE, __NV_E4M3);
    }
    return make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
}

// ---- append -----------------------------------------------------------------------------------------------------
// A step's R rows.  Thread = 8 elements; the length, the scale and the rows are requested together, so that a call
// of a few rows is one round trip.  ctx_out (if any) is another array than ctx here; a caller's in-place update is
// a second kernel, because every block has to have read the length first.
__global__ void __launch_bounds__(128) kv_append_fp8_kernel(RowsIn in, Cache8 c, const float* __restrict__ k_scale,
                                                            const float* __restrict__ v_scale, const int32_t* ctx,
                                                            int32_t* ctx_out, int R, int Hkv, int D, int32_t* status) {
    const int b = blockIdx.y;
    const bool is_v = blockIdx.z;
    const int per_row = D / 8, per_tok = Hkv * per_row;
    const int n = R * per_tok;
    const int i = blockIdx.x * 128 + threadIdx.x, at = min(i, n - 1);
    const int t = at / per_tok, rem = at - t * per_tok;
    const int h = rem / per_row, d = (rem - h * per_row) * 8;
    griddep_wait();
    griddep_launch_dependents();
    const uint4 x = __ldg(reinterpret_cast<const uint4*>((is_v ? in.v : in.k) + b * in.sb + t * in.st + h * in.sh + d));
    const float scale = (is_v ? v_scale : k_scale)[b * Hkv + h];
    const long long L = ctx[b];
    const bool fits = L >= 0 && L + R <= c.Lmax;
    if (i == 0 && !is_v) {
        if (!fits) atomicOr(status, RAPID_STATUS_BAD_CTX_LEN);
        if (ctx_out) ctx_out[b] = (int32_t)(fits ? L + R : L);
    }
    if (!fits || i >= n) return;
    bool clipped = false;
    const uint2 code = quantise8(x, scale, clipped);
    *reinterpret_cast<uint2*>((is_v ? c.v : c.k) + b * c.sb + h * c.sh + (L + t) * c.sl + d) = code;
    if (clipped) atomicOr(status, RAPID_STATUS_FP8_SATURATED);
}

__global__ void kv_append_fp8_lens_kernel(int32_t* ctx, int B, int R, long long Lmax) {
    griddep_wait();
    griddep_launch_dependents();
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b >= B) return;
    const long long L = ctx[b];
    if (L >= 0 && L + R <= Lmax) ctx[b] = (int32_t)(L + R);
}

// ---- fill -------------------------------------------------------------------------------------------------------

// Exponent of the scale for a largest magnitude given as bf16 bits (7 fraction bits): 448 = 1.75 * 2^8.
// An infinity counts as the largest finite value; the scale stays a normal number with a normal reciprocal.
__device__ __forceinline__ int scale_exponent(uint32_t amax_bits, int headroom) {
    const uint32_t a = min(amax_bits, 0x7f7fu);
    if (a == 0) return 0;
    const int e = (int)(a >> 7) - 127 - 8 + ((a & 0x7f) > 0x60 ? 1 : 0) + headroom;
    return max(-126, min(126, e));
}
__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }
__device__ __forceinline__ uint64_t pow2_twice(int e) { return (uint64_t)((uint32_t)(e + 127) << 23) * 0x100000001ull; }

// Running maximum of |x| over pairs of bf16 (a NaN takes no part).
__device__ __forceinline__ __nv_bfloat162 absmax(__nv_bfloat162 m, const uint4& v) {
    const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) m = __hmax2(m, __habs2(p[i]));
    return m;
}
__device__ __forceinline__ uint32_t absmax_bits(__nv_bfloat162 m) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(&m);
    return max(w & 0x7fffu, (w >> 16) & 0x7fffu);
}

struct FillArgs {
    RowsIn in;
    Cache8 c;
    const int32_t* n_tokens;  // [B], or NULL: T each
    float* k_scale;
    float* v_scale;
    int32_t* ctx_out;
    int32_t* status;
    int B, Hkv, D, T, headroom;
};

// Rows of sequence b, or -1 if it cannot be written.
__device__ __forceinline__ int fill_rows(const FillArgs& a, int b) {
    const int n = a.n_tokens ? a.n_tokens[b] : a.T;
    return n < 0 || n > a.T || n > a.c.Lmax ? -1 : n;
}
// What one block per (sequence, K or V, KV head) writes besides the codes.
// (With such a scale nothing but an infinity saturates.)
__device__ __forceinline__ void fill_scalars(const FillArgs& a, int b, bool is_v, int h, int n, uint32_t amax, float scale) {
    if (n >= 0) (is_v ? a.v_scale : a.k_scale)[b * a.Hkv + h] = scale;
    if (amax > 0x7f7fu) atomicOr(a.status, RAPID_STATUS_FP8_SATURATED);
    if (!is_v && h == 0) {
        if (n < 0) atomicOr(a.status, RAPID_STATUS_BAD_CTX_LEN);
        else if (a.ctx_out) a.ctx_out[b] = n;
    }
}

// Short prompts: one cluster per (sequence, K or V, KV head), of up to eight CTAs, holds all of its rows in
// registers, so they are read once: loads, the largest magnitude over block and cluster (a word of each CTA's shared memory that its peers
// push to), codes.  A thread goes down one column of chunks of 8 elements (see kv_fill_kernel), N rows `down` apart;
// CTA r of the cluster takes rows r * down * N .. .
constexpr int kFillThreads = 256;
constexpr int kFillCluster = 8;   // CTAs of a cluster, at most; 16 where kv_fill_sixteen() says so
constexpr int kFillResident = 4;  // blocks of the two-pass kernel on an SM
constexpr int kFillLag = 1;       // its groups between maxima and codes

template <int N, int THREADS>
__global__ void __launch_bounds__(THREADS) kv_fill_cluster_kernel(const FillArgs a) {
    __shared__ uint32_t peers[16];
    __shared__ uint32_t warps[THREADS / 32];
    const int rank = blockIdx.x, size = gridDim.x, unit = blockIdx.y;  // (grid x = cluster)
    const int h = unit % a.Hkv, rest = unit / a.Hkv;
    const bool is_v = rest & 1;
    const int b = rest >> 1;
    const int per_row = a.D / 8, down = THREADS / per_row, my = threadIdx.x / per_row;
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");  // (a peer's shared memory is written to once it runs)
    griddep_wait();
    griddep_launch_dependents();
    const int n = fill_rows(a, b);
    const int row0 = my < down ? rank * down * N + my : a.T, col = (threadIdx.x - my * per_row) * 8;
    const __nv_bfloat16* src = (is_v ? a.in.v : a.in.k) + b * a.in.sb + h * a.in.sh + row0 * a.in.st + col;
    uint4 x[N];
    __nv_bfloat162 m = __float2bfloat162_rn(0.f);
#pragma unroll
    for (int i = 0; i < N; ++i)
        x[i] = row0 + i * down < n ? __ldg(reinterpret_cast<const uint4*>(src + i * (down * a.in.st))) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < N; ++i) m = absmax(m, x[i]);
    uint32_t top = __reduce_max_sync(0xffffffffu, absmax_bits(m));
    if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = top;
    __syncthreads();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (threadIdx.x < size) {  // thread p pushes the block's value to CTA p of the cluster
#pragma unroll
        for (int w = 0; w < THREADS / 32; ++w) top = max(top, warps[w]);
        uint32_t there;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(smem_u32(&peers[rank])), "r"((int)threadIdx.x));
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(there), "r"(top) : "memory");
    }
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    top = 0;
    for (int p = 0; p < size; ++p) top = max(top, peers[p]);
    const int e = scale_exponent(top, a.headroom);
    if (rank == 0 && threadIdx.x == 0) fill_scalars(a, b, is_v, h, n, top, pow2(e));
    const uint64_t inv = pow2_twice(-e);
    uint8_t* dst = (is_v ? a.c.v : a.c.k) + b * a.c.sb + h * a.c.sh + row0 * a.c.sl + col;
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (row0 + i * down < n) *reinterpret_cast<uint2*>(dst + i * (down * a.c.sl)) = quantise8_pow2(x[i], inv);
}

// Long prompts: the rows do not fit on chip, so they are read twice, the second time out of L2.  The units
// (sequence, K or V, KV head) are worked off in groups that L2 holds; work items are handed out by a ticket counter:
// in step s the maxima of group s and the codes of group s - 1, alternating.  An item that writes codes waits until
// the maxima of its group are in: those items were all handed out before it, each to a block that had finished all
// it held, so the wait ends whatever the number of blocks that run at a time (and it is bounded).  That is also why
// no ticket is taken ahead: a block that holds a maximum while it waits for others stalls them (285 us for 8 heads
// of 131,072 rows of 128, K and V; 229 without).
//   The rest of the way from there to 172: four 16-byte loads a thread in flight with 32 warps an SM rather than
// eight with fewer (212), a lag of one group; a thread that goes down one column, so that a load costs one
// addition, and products in pairs (178); as many items as make one step one wave of the grid, rather than items of
// 128 KB.  The same block for both passes over an item gained nothing.  DRAM carries each row once; what
// is left over the 123 us that takes is the second pass's share of L2 and the waves' ends.
struct FillPlan {
    int group_units, groups;   // units of a group, groups in all
    int item_rows, items;      // rows of an item, items of a group (item = row chunk * group_units + unit)
    uint32_t* words;           // ticket, then per group the count of finished maxima items, then per unit the maximum
};
__device__ __forceinline__ uint32_t ld_acquire(const uint32_t* p) {
    uint32_t v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}

__global__ void kv_fill_clear_kernel(uint32_t* words, int n) {
    griddep_wait();
    griddep_launch_dependents();
    for (int i = threadIdx.x; i < n; i += blockDim.x) words[i] = 0;
}

template <int UN>
__global__ void __launch_bounds__(kFillThreads, kFillResident) kv_fill_kernel(const FillArgs a, const FillPlan p) {
    __shared__ uint32_t warps[kFillThreads / 32];
    __shared__ uint32_t sh_ticket, sh_amax;
    uint32_t* ticket = p.words;
    uint32_t* done = p.words + 1;
    uint32_t* amax = done + p.groups;
    // A thread goes down a column of chunks of 8 elements, `down` rows at a step; threads that make no whole row are
    // idle (they begin behind the last row), and rows wider than the block have several columns for each.
    const int per_row = a.D / 8;
    const int down = max(1, kFillThreads / per_row), my = threadIdx.x / per_row;
    const int my_col = threadIdx.x - my * per_row, my_row = my < down ? my : p.item_rows;
    const long long in_step = down * a.in.st, out_step = down * a.c.sl;
    const uint32_t total = (uint32_t)(p.groups + kFillLag) * 2u * p.items;
    griddep_wait();
    griddep_launch_dependents();
    for (;;) {
        if (threadIdx.x == 0) sh_ticket = atomicAdd(ticket, 1u);
        __syncthreads();
        const uint32_t tk = sh_ticket;
        if (tk >= total) break;
        const uint32_t step = tk / (2u * p.items), r = tk - step * 2u * p.items;
        const bool codes = r & 1;
        const int group = (int)step - (codes ? kFillLag : 0), item = (int)(r >> 1);
        const int chunk = item / p.group_units, unit = group * p.group_units + item - chunk * p.group_units;
        const bool work = group >= 0 && unit < 2 * a.B * a.Hkv;
        const int rest = work ? unit / a.Hkv : 0, h = work ? unit - rest * a.Hkv : 0;
        const bool is_v = rest & 1;
        const int b = rest >> 1;
        const int n = work ? fill_rows(a, b) : -1;
        const int row0 = chunk * p.item_rows, rows = min(p.item_rows, max(n, 0) - row0);
        const __nv_bfloat16* src = (is_v ? a.in.v : a.in.k) + b * a.in.sb + h * a.in.sh;
        if (!codes) {
            if (rows > 0) {
                __nv_bfloat162 m = __float2bfloat162_rn(0.f);
                for (int col = my_col; col < per_row; col += kFillThreads) {
                    const __nv_bfloat16* at = src + (long long)(row0 + my_row) * a.in.st + col * 8;
                    for (int r = my_row; r < rows; r += down * UN, at += UN * in_step) {
                        uint4 x[UN];
#pragma unroll
                        for (int u = 0; u < UN; ++u)
                            x[u] = r + u * down < rows ? __ldg(reinterpret_cast<const uint4*>(at + u * in_step)) : make_uint4(0, 0, 0, 0);
#pragma unroll
                        for (int u = 0; u < UN; ++u) m = absmax(m, x[u]);
                    }
                }
                const uint32_t top = __reduce_max_sync(0xffffffffu, absmax_bits(m));
                if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = top;
            }
            __syncthreads();
            if (threadIdx.x == 0 && group >= 0 && group < p.groups) {
                if (rows > 0) {
                    uint32_t top = 0;
#pragma unroll
                    for (int w = 0; w < kFillThreads / 32; ++w) top = max(top, warps[w]);
                    atomicMax(amax + unit, top);
                    __threadfence();
                }
                atomicAdd(done + group, 1u);
            }
        } else {
            if (threadIdx.x == 0 && work) {
                const long long t0 = clock64();
                bool ready = true;
                while (ld_acquire(done + group) < (uint32_t)p.items) {
                    if (clock64() - t0 > kWaitCycleLimit) {
                        ready = false;
                        atomicOr(a.status, RAPID_STATUS_PIPELINE_TIMEOUT);
                        break;
                    }
                    __nanosleep(100);
                }
                sh_amax = ready ? ld_acquire(amax + unit) : 0x10000u;
            }
            __syncthreads();
            if (work && sh_amax <= 0xffffu) {
                const int e = scale_exponent(sh_amax, a.headroom);
                if (chunk == 0 && threadIdx.x == 0) fill_scalars(a, b, is_v, h, n, sh_amax, pow2(e));
                const uint64_t inv = pow2_twice(-e);
                uint8_t* dst = (is_v ? a.c.v : a.c.k) + b * a.c.sb + h * a.c.sh;
                for (int col = my_col; col < per_row; col += kFillThreads) {
                    const __nv_bfloat16* at = src + (long long)(row0 + my_row) * a.in.st + col * 8;
                    uint8_t* to = dst + (long long)(row0 + my_row) * a.c.sl + col * 8;
                    for (int r = my_row; r < rows; r += down * UN, at += UN * in_step, to += UN * out_step) {
                        uint4 x[UN];
#pragma unroll
                        for (int u = 0; u < UN; ++u)
                            if (r + u * down < rows) x[u] = __ldcs(reinterpret_cast<const uint4*>(at + u * in_step));
#pragma unroll
                        for (int u = 0; u < UN; ++u)
                            if (r + u * down < rows) __stcs(reinterpret_cast<uint2*>(to + u * out_step), quantise8_pow2(x[u], inv));
                    }
                }
            }
        }
        __syncthreads();  // (warps, sh_amax and sh_ticket are free again)
    }
}

// ---- read back --------------------------------------------------------------------------------------------------
// Chunks of the cache into a bf16 cache, one behind the other.  A block takes 8 KB of codes of one (sequence, K or
// V, KV head, chunk); where its rows go depends on the chunks before (a partial one is shorter, -1 is none), which
// the block adds up while its codes are on their way.  Bound by HBM: 131,072 rows of 8 heads of 128, K and V, in 104 us,
// ten chunks of 512 in 7.1 (119 and 8.7 with 16 codes a thread, whose two stores fill a sector by halves; 106 and
// 7.2 with blocks of 256 threads).
struct ReadArgs {
    Cache8 c;
    const float* k_scale;
    const float* v_scale;
    const int32_t* ctx;
    const int32_t* idx;  // [B, n_chunks], or NULL: 0, 1, 2, ...
    __nv_bfloat16* k_out;
    __nv_bfloat16* v_out;
    int32_t* out_lens;
    int32_t* status;
    long long ob, oh, ol, Lout;  // strides of the output, its capacity
    int B, Hkv, D, n_chunks, chunk;
    int wide;  // blocks that share a row: 1, or more where it is wider than one
};
constexpr int kReadThreads = 128;
constexpr int kReadUnroll = 8;  // 8-byte loads in flight per thread

// Rows that chunk number i of sequence b holds.
__device__ __forceinline__ int chunk_rows(const ReadArgs& a, int ctx, int i) {
    if (i < 0) return 0;
    const long long from = (long long)i * a.chunk;
    return (int)max(0LL, min((long long)a.chunk, ctx - from));
}

__global__ void __launch_bounds__(kReadThreads) kv_read_fp8_kernel(const ReadArgs a) {
    __shared__ int warps[kReadThreads / 32];
    const int j = blockIdx.y;  // which of the chunks
    const int h = blockIdx.z % a.Hkv, rest = blockIdx.z / a.Hkv;
    const bool is_v = rest & 1;
    const int b = rest >> 1;
    // A thread goes down one column of 8 codes, so that a warp's stores of 16 bytes a lane lie side by side.
    const int per_row = a.D / 8, down = max(1, kReadThreads / per_row), my = threadIdx.x / per_row;
    const int block = blockIdx.x / a.wide, part = blockIdx.x - block * a.wide;
    const int my_col = (part * kReadThreads + threadIdx.x - my * per_row) * 8, row0 = block * (down * kReadUnroll) + my;
    griddep_wait();
    griddep_launch_dependents();
    const int given = a.ctx[b];
    const int ctx = (int)max(0LL, min((long long)given, a.c.Lmax));
    const int number = a.idx ? a.idx[(size_t)b * a.n_chunks + j] : j;
    const int rows = chunk_rows(a, ctx, number);
    const long long from = rows > 0 ? (long long)number * a.chunk : 0;
    const int end = my < down && my_col < a.D ? rows : 0;  // (threads that make no whole row are idle)
    const uint8_t* src = (is_v ? a.c.v : a.c.k) + b * a.c.sb + h * a.c.sh + (from + row0) * a.c.sl + my_col;
    uint2 x[kReadUnroll];
#pragma unroll
    for (int u = 0; u < kReadUnroll; ++u)
        if (row0 + u * down < end) x[u] = __ldcs(reinterpret_cast<const uint2*>(src + u * (down * a.c.sl)));
    const float scale = (is_v ? a.v_scale : a.k_scale)[b * a.Hkv + h];
    // the rows before this chunk's
    long long before = 0;
    const bool teller = blockIdx.x == 0 && h == 0 && !is_v && j == a.n_chunks - 1;
    if (a.idx) {
        int s = 0;
        for (int i = threadIdx.x; i < j; i += kReadThreads) s += chunk_rows(a, ctx, a.idx[(size_t)b * a.n_chunks + i]);
        s = __reduce_add_sync(0xffffffffu, s);
        if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = s;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kReadThreads / 32; ++w) before += warps[w];
    } else {
        before = min((long long)ctx, (long long)j * a.chunk);
    }
    if (threadIdx.x == 0) {
        if (teller) {
            a.out_lens[b] = (int32_t)min(before + rows, a.Lout);
            if (given != ctx) atomicOr(a.status, RAPID_STATUS_BAD_CTX_LEN);
        }
        if (blockIdx.x == 0 && h == 0 && !is_v && (number < -1 || (number >= 0 && rows == 0 && a.idx) || before + rows > a.Lout))
            atomicOr(a.status, RAPID_STATUS_BAD_CTX_LEN);
    }
    __nv_bfloat16* dst = (is_v ? a.v_out : a.k_out) + b * a.ob + h * a.oh + (before + row0) * a.ol + my_col;
#pragma unroll
    for (int u = 0; u < kReadUnroll; ++u) {
        if (row0 + u * down >= end || before + row0 + u * down >= a.Lout) continue;
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)((i & 2 ? x[u].y : x[u].x) >> (16 * (i & 1))), __NV_E4M3);
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&r));
            o[i] = pack_bf16x2(f.x * scale, f.y * scale);
        }
        __stcs(reinterpret_cast<uint4*>(dst + u * (down * a.ol)), make_uint4(o[0], o[1], o[2], o[3]));
    }
}

// ---- host side --------------------------------------------------------------------------------------------------

bool cache8_of(const char* who, const rapid_attn_shape* s, void* k, void* v, Cache8& c) {
    if (s->B <= 0 || s->Hkv <= 0 || s->Lmax <= 0 || s->D <= 0 || s->Lmax > 0x7fffffffLL) {
        set_error("%s: invalid shape", who);
        return false;
    }
    c.k = static_cast<uint8_t*>(k);
    c.v = static_cast<uint8_t*>(v);
    c.sl = s->kv_stride_l ? s->kv_stride_l : s->D;
    c.sh = s->kv_stride_h ? s->kv_stride_h : s->Lmax * c.sl;
    c.sb = s->kv_stride_b ? s->kv_stride_b : s->Hkv * c.sh;
    c.Lmax = s->Lmax;
    return true;
}
// Whether strides and pointers allow 16-byte accesses of codes and of bf16 rows.
bool cache8_aligned(const char* who, int D, const Cache8& c) {
    if (D % 16 || c.sl < D || c.sl % 16 || c.sh % 16 || c.sb % 16 || c.sh <= 0 || c.sb <= 0 || (((uintptr_t)c.k | (uintptr_t)c.v) & 15)) {
        set_error("%s: head_dim and the cache's strides must be positive multiples of 16, its pointers 16-byte aligned", who);
        return false;
    }
    return true;
}
bool rows_of(const char* who, const rapid_kv_rows* r, int T, int Hkv, int D, const void* k, const void* v, RowsIn& in) {
    in.k = static_cast<const __nv_bfloat16*>(k);
    in.v = static_cast<const __nv_bfloat16*>(v);
    in.sh = r && r->stride_h ? r->stride_h : D;
    in.st = r && r->stride_t ? r->stride_t : (long long)Hkv * D;
    in.sb = r && r->stride_b ? r->stride_b : (long long)T * Hkv * D;
    if (in.sh % 8 || in.st % 8 || in.sb % 8 || in.sh <= 0 || in.st <= 0 || in.sb <= 0 || (((uintptr_t)k | (uintptr_t)v) & 15)) {
        set_error("%s: the rows' strides must be positive multiples of 8 elements, their pointers 16-byte aligned", who);
        return false;
    }
    return true;
}

}  // namespace

int launch_kv_append_fp8(const void* k_new, const void* v_new, const rapid_kv_rows* rows, void* k_cache, void* v_cache,
                         const float* k_scale, const float* v_scale, const int32_t* ctx_lens, int32_t* ctx_lens_out,
                         int gamma, const rapid_attn_shape* shape, int32_t* status_word, cudaStream_t stream) {
    const char* who = "rapid_kv_append_fp8";
    if (!k_new || !v_new || !k_cache || !v_cache || !k_scale || !v_scale || !ctx_lens || !shape || !status_word) {
        set_error("%s: NULL argument", who);
        return RAPID_ERR_INVALID_ARG;
    }
    Cache8 c;
    if (!cache8_of(who, shape, k_cache, v_cache, c)) return RAPID_ERR_INVALID_ARG;
    const rapid_attn_shape& s = *shape;
    if (gamma < 0 || s.B > 65535 || ((int64_t)gamma + 1) * s.Hkv * s.D > 0x7fffffffLL - 1024) {
        set_error("%s: gamma must not be negative, B at most 65535 and a sequence's new rows below 2^31 elements", who);
        return RAPID_ERR_INVALID_ARG;
    }
    const int R = gamma + 1;
    RowsIn in;
    if (!cache8_aligned(who, s.D, c) || !rows_of(who, rows, R, s.Hkv, s.D, k_new, v_new, in)) return RAPID_ERR_UNSUPPORTED;
    const bool in_place = ctx_lens_out == ctx_lens;
    const int chunks = R * s.Hkv * (s.D / 8);
    RAPID_CUDA_CHECK(launch_dependent(kv_append_fp8_kernel, dim3((chunks + 127) / 128, s.B, 2), dim3(128), 0, stream, in, c, k_scale,
                                      v_scale, ctx_lens, in_place ? nullptr : ctx_lens_out, R, s.Hkv, s.D, status_word));
    count_launch(1);
    if (in_place) {
        RAPID_CUDA_CHECK(launch_dependent(kv_append_fp8_lens_kernel, dim3((s.B + 127) / 128), dim3(128), 0, stream, ctx_lens_out,
                                          s.B, R, (long long)s.Lmax));
        count_launch(1);
    }
    return RAPID_OK;
}

// Words of scratch of a fill: ticket, a count per group (at most one group per unit), a maximum per unit.
size_t kv_fill_workspace_bytes(int B, int Hkv) {
    if (B <= 0 || Hkv <= 0) return 0;
    return kWorkspaceHeaderBytes + align_up((1 + 2 * (size_t)2 * B * Hkv) * sizeof(uint32_t), 256);
}

// Whether the current device runs clusters of 16 (beyond what every one does); asked once for each.
static int kv_fill_sixteen(int dev, bool& yes) {
    static std::atomic<int> known[64];  // 1 + answer (first calls may come from several threads at once)
    if (const int told = dev < 64 ? known[dev].load() : 0) {
        yes = told == 2;
        return RAPID_OK;
    }
    int least = 16;
    for (auto* f : {kv_fill_cluster_kernel<6, 512>, kv_fill_cluster_kernel<8, 512>}) {
        RAPID_CUDA_CHECK(cudaFuncSetAttribute(f, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(16);
        cfg.blockDim = dim3(512);
        int n = 0;
        RAPID_CUDA_CHECK(cudaOccupancyMaxPotentialClusterSize(&n, f, &cfg));
        if (n < least) least = n;
    }
    yes = least >= 16;
    if (dev < 64) known[dev] = yes ? 2 : 1;
    return RAPID_OK;
}

int launch_kv_fill_fp8(const void* k_new, const void* v_new, const rapid_kv_rows* rows, int T, const int32_t* n_tokens,
                       void* k_cache, void* v_cache, float* k_scale, float* v_scale, int32_t* ctx_lens_out, int headroom,
                       const rapid_attn_shape* shape, void* workspace, size_t workspace_bytes, cudaStream_t stream) {
    const char* who = "rapid_kv_fill_fp8";
    if (!k_new || !v_new || !k_cache || !v_cache || !k_scale || !v_scale || !shape) {
        set_error("%s: NULL argument", who);
        return RAPID_ERR_INVALID_ARG;
    }
    FillArgs a = {};
    if (!cache8_of(who, shape, k_cache, v_cache, a.c)) return RAPID_ERR_INVALID_ARG;
    const rapid_attn_shape& s = *shape;
    if (T <= 0 || headroom < 0 || headroom > 8) {
        set_error("%s: T must be positive and headroom in [0, 8]", who);
        return RAPID_ERR_INVALID_ARG;
    }
    const int64_t units = 2 * (int64_t)s.B * s.Hkv;
    if (units > 65535 || (int64_t)T * s.D > 0x7fffffffLL - 65536) {
        set_error("%s: 2 * B * Hkv at most 65535, T * D below 2^31", who);
        return RAPID_ERR_UNSUPPORTED;
    }
    if (!cache8_aligned(who, s.D, a.c) || !rows_of(who, rows, T, s.Hkv, s.D, k_new, v_new, a.in)) return RAPID_ERR_UNSUPPORTED;
    if (!workspace || workspace_bytes < kv_fill_workspace_bytes(s.B, s.Hkv) || ((uintptr_t)workspace & 255)) {
        set_error("%s: workspace of %zu bytes needed (256-byte aligned), got %zu", who, kv_fill_workspace_bytes(s.B, s.Hkv),
                  workspace_bytes);
        return RAPID_ERR_WORKSPACE;
    }
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    a.n_tokens = n_tokens;
    a.k_scale = k_scale;
    a.v_scale = v_scale;
    a.ctx_out = ctx_lens_out;
    a.status = reinterpret_cast<int32_t*>(ws);
    a.B = s.B;
    a.Hkv = s.Hkv;
    a.D = s.D;
    a.T = T;
    a.headroom = headroom;
    int dev = 0, sms = 0;
    RAPID_CUDA_CHECK(cudaGetDevice(&dev));
    RAPID_CUDA_CHECK(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    // Rows that a CTA holds with one a thread.  Eight a thread in clusters of eight CTAs of 512, 2,048 rows of 128, are
    // the most that is (for any number of units) faster than two passes (8 heads: 5.5 us for 8.7, and 49.7 for 53.8 at 16 sequences; with 16 a
    // thread 14.4 for 12.7 at 4,096 rows).  Six a thread rather than eight where they do: 4.0 us for 4.8 at 1,100 rows.
    const int per_row = s.D / 8, rows_256 = 256 / per_row, rows_512 = 512 / per_row;
    // Sixteen CTAs hold twice as much, which pays while there are few units (8 heads: 4,000 rows 10.2 us for 12.5, 2,100
    // 6.5 for 9.0; four sequences of 4,000 31.1 for 30.8, sixteen 110 for 90).
    bool sixteen = false;
    if (T > 8 * kFillCluster * rows_512 && T <= 8 * 16 * rows_512 && units * 16 <= 4 * sms) {
        const int rc = kv_fill_sixteen(dev, sixteen);
        if (rc != RAPID_OK) return rc;
    }
    if (sixteen || T <= 8 * kFillCluster * rows_512) {
        // Few units take all eight CTAs and few rows a thread; where that would be more than two CTAs an SM, as few CTAs as
        // hold the rows, eight a thread (8 heads: 256 prompts of 64 rows 22 us for 85, 128 of 200 36 for 62, 8 of 500 6.9
        // for 7.8).
        int size = sixteen ? 16 : kFillCluster;
        if (!sixteen && units * kFillCluster > 2 * sms)
            while (size > 1 && T <= 8 * (size / 2) * rows_256) size /= 2;
        const int64_t one_256 = (int64_t)size * rows_256, one_512 = (int64_t)size * rows_512;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(size, (unsigned)units);
        cfg.blockDim = dim3(T <= 8 * one_256 ? 256 : 512);
        cfg.stream = stream;
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = size;
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 2;
        if (T <= one_256) RAPID_CUDA_CHECK(cudaLaunchKernelEx(&cfg, kv_fill_cluster_kernel<1, 256>, a));
        else if (T <= 2 * one_256) RAPID_CUDA_CHECK(cudaLaunchKernelEx(&cfg, kv_fill_cluster_kernel<2, 256>, a));
        else if (T <= 4 * one_256) RAPID_CUDA_CHECK(cudaLaunchKernelEx(&cfg, kv_fill_cluster_kernel<4, 256>, a));
        else if (T <= 8 * one_256) RAPID_CUDA_CHECK(cudaLaunchKernelEx(&cfg, kv_fill_cluster_kernel<8, 256>, a));
        else if (T <= 6 * one_512) RAPID_CUDA_CHECK(cudaLaunchKernelEx(&cfg, kv_fill_cluster_kernel<6, 512>, a));
        else RAPID_CUDA_CHECK(cudaLaunchKernelEx(&cfg, kv_fill_cluster_kernel<8, 512>, a));
        count_launch(1);
        return RAPID_OK;
    }
    const int grid = sms * kFillResident;
    // Groups of equal size of at most 32 MB (or one unit): with the group before it, half of L2.  A step's items,
    // the maxima of a group and the codes of another, are one wave of the grid.
    constexpr int64_t kGroupBytes = 32 << 20;
    FillPlan p;
    const int64_t unit_bytes = (int64_t)T * s.D * 2;
    const int64_t most = kGroupBytes / unit_bytes < 1 ? 1 : kGroupBytes / unit_bytes;
    p.groups = (int)((units + most - 1) / most);
    p.group_units = (int)((units + p.groups - 1) / p.groups);
    p.groups = (int)((units + p.group_units - 1) / p.group_units);
    const int chunks_of_unit = grid / 2 / p.group_units > 1 ? grid / 2 / p.group_units : 1;
    p.item_rows = (T + chunks_of_unit - 1) / chunks_of_unit;
    p.items = (T + p.item_rows - 1) / p.item_rows * p.group_units;
    if (((int64_t)p.groups + kFillLag) * 2 * p.items > 0x7fffffffLL) {
        set_error("%s: too many rows in one call", who);
        return RAPID_ERR_UNSUPPORTED;
    }
    p.words = reinterpret_cast<uint32_t*>(ws + kWorkspaceHeaderBytes);
    RAPID_CUDA_CHECK(launch_dependent(kv_fill_clear_kernel, dim3(1), dim3(256), 0, stream, p.words, (int)(1 + p.groups + units)));
    RAPID_CUDA_CHECK(launch_dependent(kv_fill_kernel<4>, dim3(grid), dim3(kFillThreads), 0, stream, a, p));
    count_launch(2);
    return RAPID_OK;
}

int launch_kv_read_fp8(const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale,
                       const int32_t* ctx_lens, const rapid_attn_shape* shape, const int32_t* chunk_idx, int n_chunks,
                       int chunk_tokens, void* k_out, void* v_out, const rapid_attn_shape* out_shape, int32_t* out_lens,
                       int32_t* status_word, cudaStream_t stream) {
    const char* who = "rapid_kv_read_fp8";
    if (!k_cache || !v_cache || !k_scale || !v_scale || !ctx_lens || !shape || !k_out || !v_out || !out_shape || !out_lens || !status_word) {
        set_error("%s: NULL argument", who);
        return RAPID_ERR_INVALID_ARG;
    }
    ReadArgs a = {};
    Cache8 o;  // (the output's geometry goes through the same defaults)
    if (!cache8_of(who, shape, const_cast<void*>(k_cache), const_cast<void*>(v_cache), a.c) || !cache8_of(who, out_shape, k_out, v_out, o))
        return RAPID_ERR_INVALID_ARG;
    const rapid_attn_shape& s = *shape;
    if (n_chunks <= 0 || chunk_tokens <= 0 || out_shape->B != s.B || out_shape->Hkv != s.Hkv || out_shape->D != s.D) {
        set_error("%s: n_chunks and chunk_tokens must be positive and the output of the cache's B, Hkv and D", who);
        return RAPID_ERR_INVALID_ARG;
    }
    if (!cache8_aligned(who, s.D, a.c)) return RAPID_ERR_UNSUPPORTED;
    if (o.sl < s.D || o.sl % 8 || o.sh % 8 || o.sb % 8 || o.sh <= 0 || o.sb <= 0 || (((uintptr_t)k_out | (uintptr_t)v_out) & 15)) {
        set_error("%s: the output's strides must be positive multiples of 8 elements, its pointers 16-byte aligned", who);
        return RAPID_ERR_UNSUPPORTED;
    }
    const int64_t units = 2 * (int64_t)s.B * s.Hkv;
    if (units > 65535 || n_chunks > 65535 || (int64_t)chunk_tokens * s.D > 0x7fffffffLL - 65536) {
        set_error("%s: 2 * B * Hkv and n_chunks at most 65535, chunk_tokens * D below 2^31", who);
        return RAPID_ERR_UNSUPPORTED;
    }
    if (out_lens == ctx_lens) {
        set_error("%s: out_lens must not be ctx_lens, which blocks still read when it is written", who);
        return RAPID_ERR_INVALID_ARG;
    }
    // no chunk is longer than the cache; the rows of the chunks named are added up in 32 bits
    const int64_t longest = chunk_tokens < s.Lmax ? chunk_tokens : s.Lmax;
    if (chunk_idx && longest * n_chunks > 0x7fffffffLL) {
        set_error("%s: the chunks named must hold less than 2^31 tokens", who);
        return RAPID_ERR_UNSUPPORTED;
    }
    a.k_scale = k_scale;
    a.v_scale = v_scale;
    a.ctx = ctx_lens;
    a.idx = chunk_idx;
    a.k_out = static_cast<__nv_bfloat16*>(k_out);
    a.v_out = static_cast<__nv_bfloat16*>(v_out);
    a.out_lens = out_lens;
    a.status = status_word;
    a.ob = o.sb;
    a.oh = o.sh;
    a.ol = o.sl;
    a.Lout = o.Lmax;
    a.B = s.B;
    a.Hkv = s.Hkv;
    a.D = s.D;
    a.n_chunks = n_chunks;
    a.chunk = chunk_tokens;
    a.wide = (s.D / 8 + kReadThreads - 1) / kReadThreads;
    const int64_t rows_of_block = kReadUnroll * (a.wide > 1 ? 1 : kReadThreads / (s.D / 8));
    const int64_t blocks = (longest + rows_of_block - 1) / rows_of_block * a.wide;
    RAPID_CUDA_CHECK(launch_dependent(kv_read_fp8_kernel, dim3((unsigned)blocks, n_chunks, (unsigned)units), dim3(kReadThreads), 0,
                                      stream, a));
    count_launch(1);
    return RAPID_OK;
}

}  // namespace rapid
