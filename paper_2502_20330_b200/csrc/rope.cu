// Position rotation of queries and keys, alone and on the way into a cache.
//
// Pair i of a head's first rd columns, (x_i, x_{i + rd/2}) or (x_{2i}, x_{2i+1}), is turned by the angle a = p f_i, where p is the
// row's position on the pair's axis and f_i the pair's frequency:
//   y1 = s (x1 cos a - x2 sin a)      y2 = s (x1 sin a + x2 cos a)
// A position of 100,000 times a frequency near 1 leaves an fp32 angle with an error of 2^-8, so p f_i / 2 pi is formed in 64 bits, its
// whole turns are taken off there, and what is left, at most half a turn, goes to 32 bits (2^-25 of a turn).  The angles are worked out
// once a token and serve all its heads.
//
// Bound: HBM.  Every element is read and written once, 4 bytes; an SM's four blocks of 256 threads have up to 128 KB of reads under way.
// Four items of 32 bytes a thread at 64 registers: 100 us for two videos of 20,011 tokens at 28/4 heads of 128 (6.5 TB/s), 191 us for
// prompts of up to 24,000 tokens at 32/8 heads with their append (6.0 TB/s); three items 120 and 224, six 141 and 233, two at six blocks an
// SM 106 and 187.  Calls of few tokens are a launch and dependent accesses: the rotation 2.6 us (positions and rows, then the stores), an
// append 3.3 us (lengths, then rows and table entries, then the stores).
#include <math.h>

#include "common.cuh"
#include "prefill.cuh"

namespace rapid {

namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeItems = 4;       // items of 32 bytes that a thread has in flight
constexpr int kRopeBlocks = 4;      // blocks an SM holds: 64 registers a thread
constexpr int kRopeMaxD = 256;
constexpr int kRopeMaxTokens = 16;  // tokens of a block

struct RopeTensor {  // [B, T, H, D] bf16 by element strides
    __nv_bfloat16* p;
    long long sb, st, sh;
};

struct RopeArgs {
    RopeTensor q, k, v, qo, ko;  // v and the cache are used by the appends alone; ko by the rotation alone
    __nv_bfloat16 *k_cache, *v_cache;
    long long cb, ch, cl;        // strides of the cache between sequences (blocks of a pool) / KV heads / tokens
    long long Lmax;
    const int32_t* block_table;  // paged cache, or NULL
    int block_size, num_blocks, max_blocks;
    const int32_t* n_tokens;     // or NULL: T each
    const int32_t* ctx;          // NULL: the rotation alone
    int32_t* ctx_out;            // or NULL
    const int32_t* positions;    // [axes, B, T], or NULL: ctx + row
    int32_t* status;
    const float* inv_freq;
    uint32_t axis_bits[kRopeMaxD / 2 / 16];  // two bits a pair
    int B, T, Hq, Hkv, D, rd, tokens;
    float scale, sin_sign;
};

__device__ __forceinline__ float2 unpack_bf16x2(uint32_t v) {
    return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&v));
}

// One item is 16 elements of a row, two 16-byte words: eight pairs, or 16 elements that are not turned.
template <bool INTER>
__global__ void __launch_bounds__(kRopeThreads, kRopeBlocks) rope_kernel(const __grid_constant__ RopeArgs a) {
    // cos and sin of the block's tokens: two pairs to a word, the words of an item spread so that the
    // threads of a row read neighbouring ones
    __shared__ float4 turn[kRopeMaxTokens * kRopeMaxD / 4];
    __shared__ long long place[kRopeMaxTokens];  // a token's row in the cache, in elements; -1: not written
    const int b = blockIdx.y;
    const int t0 = blockIdx.x * a.tokens;
    const int per_row = a.D >> 4, turned = a.rd >> 4, half = a.rd >> 1;

    griddep_wait();
    griddep_launch_dependents();
    int n = a.T;
    long long L = 0;
    if (a.ctx) {
        if (a.n_tokens) n = a.n_tokens[b];
        L = a.ctx[b];
        const bool bad = n < 0 || n > a.T || L < 0 || L + n > a.Lmax;
        if (t0 == 0 && threadIdx.x == 0) {
            if (bad) atomicOr(a.status, RAPID_STATUS_BAD_CTX_LEN);
            if (a.ctx_out) a.ctx_out[b] = (int32_t)(bad ? L : L + n);
        }
        if (bad) return;
    }
    const int tokens = min(a.tokens, n - t0);
    if (tokens <= 0) return;
    const int rows_token = a.Hq + (a.ctx ? 2 : 1) * a.Hkv;
    const float inv_rows = 1.f / (float)rows_token;
    const int rows = tokens * rows_token;
    const int lanes = kRopeThreads / per_row;  // rows that the block takes at a time
    const int lane = threadIdx.x / per_row, c = threadIdx.x - lane * per_row;
    // where an item's two words lie in its row
    const int at0 = c < turned ? (INTER ? 16 * c : 8 * c) : 16 * c;
    const int at1 = c < turned && !INTER ? half + 8 * c : at0 + 8;

    auto source = [&](int r, int& tok, int& h) -> const __nv_bfloat16* {
        tok = (int)(((float)r + 0.5f) * inv_rows);
        h = r - tok * rows_token;
        const RopeTensor& x = h < a.Hq ? a.q : h < a.Hq + a.Hkv ? a.k : a.v;
        const int hh = h < a.Hq ? h : h < a.Hq + a.Hkv ? h - a.Hq : h - a.Hq - a.Hkv;
        return x.p + b * x.sb + (t0 + tok) * x.st + hh * x.sh;
    };

    uint4 x[kRopeItems][2];
    auto fetch = [&](int r0) {
#pragma unroll
        for (int u = 0; u < kRopeItems; ++u) {
            const int r = r0 + u * lanes;
            if (r < rows && lane < lanes) {
                int tok, h;
                const __nv_bfloat16* p = source(r, tok, h);
                x[u][0] = *reinterpret_cast<const uint4*>(p + at0);
                x[u][1] = *reinterpret_cast<const uint4*>(p + at1);
            }
        }
    };
    fetch(lane);

    for (int i = threadIdx.x; i < tokens * half; i += kRopeThreads) {
        const int tok = i / half, pair = i - tok * half;
        const int axis = a.axis_bits[pair >> 4] >> (2 * (pair & 15)) & 3;
        const int32_t p = a.positions ? a.positions[((size_t)axis * a.B + b) * a.T + t0 + tok] : (int32_t)(L + t0 + tok);
        double turns = (double)p * (double)a.inv_freq[pair] * 0.15915494309189533577;  // 1 / (2 pi)
        turns -= rint(turns);
        float s, co;
        sincospif(2.f * (float)turns, &s, &co);
        reinterpret_cast<float2*>(turn)[((tok * 4 + (pair & 7) / 2) * turned + (pair >> 3)) * 2 + (pair & 1)] =
            make_float2(co * a.scale, s * a.sin_sign);
    }
    if (a.ctx && threadIdx.x < tokens) {
        const long long pos = L + t0 + threadIdx.x;
        long long at = -1;
        if (a.block_table) {
            const int blk = a.block_table[(size_t)b * a.max_blocks + pos / a.block_size];
            if (blk < 0 || blk >= a.num_blocks) atomicOr(a.status, RAPID_STATUS_BAD_BLOCK_TABLE);
            else at = blk * a.cb + pos % a.block_size * a.cl;
        } else {
            at = b * a.cb + pos * a.cl;
        }
        place[threadIdx.x] = at;
    }
    __syncthreads();

    for (int r0 = lane; r0 < rows && lane < lanes; r0 += kRopeItems * lanes) {
        if (r0 != lane) fetch(r0);
#pragma unroll
        for (int u = 0; u < kRopeItems; ++u) {
            const int r = r0 + u * lanes;
            if (r >= rows) break;
            int tok, h;
            source(r, tok, h);
            uint4 y0 = x[u][0], y1 = x[u][1];
            if (c < turned && h < a.Hq + a.Hkv) {
                const float4* cs = turn + tok * 4 * turned + c;
                uint32_t* p0 = reinterpret_cast<uint32_t*>(&y0);
                uint32_t* p1 = reinterpret_cast<uint32_t*>(&y1);
#pragma unroll
                for (int j = 0; j < 4; ++j) {  // pairs 2j and 2j + 1 of the item
                    const float4 f = cs[j * turned];
                    if constexpr (INTER) {
                        uint32_t& w0 = j < 2 ? p0[2 * j] : p1[2 * j - 4];
                        uint32_t& w1 = j < 2 ? p0[2 * j + 1] : p1[2 * j - 3];
                        const float2 e = unpack_bf16x2(w0), g = unpack_bf16x2(w1);
                        w0 = pack_bf16x2(e.x * f.x - e.y * f.y, e.x * f.y + e.y * f.x);
                        w1 = pack_bf16x2(g.x * f.z - g.y * f.w, g.x * f.w + g.y * f.z);
                    } else {
                        const float2 e = unpack_bf16x2(p0[j]), g = unpack_bf16x2(p1[j]);
                        p0[j] = pack_bf16x2(e.x * f.x - g.x * f.y, e.y * f.z - g.y * f.w);
                        p1[j] = pack_bf16x2(e.x * f.y + g.x * f.x, e.y * f.w + g.y * f.z);
                    }
                }
            }
            __nv_bfloat16* to;
            if (h < a.Hq) {
                to = a.qo.p + b * a.qo.sb + (t0 + tok) * a.qo.st + h * a.qo.sh;
            } else if (!a.ctx) {
                to = a.ko.p + b * a.ko.sb + (t0 + tok) * a.ko.st + (h - a.Hq) * a.ko.sh;
            } else {
                if (place[tok] < 0) continue;
                to = h < a.Hq + a.Hkv ? a.k_cache + place[tok] + (h - a.Hq) * a.ch : a.v_cache + place[tok] + (h - a.Hq - a.Hkv) * a.ch;
            }
            *reinterpret_cast<uint4*>(to + at0) = y0;
            *reinterpret_cast<uint4*>(to + at1) = y1;
        }
    }
}

// Lengths that are counted in place go up behind the rows, whose blocks all read them.
__global__ void rope_lens_kernel(int32_t* ctx, const int32_t* n_tokens, int B, int T, long long Lmax) {
    griddep_wait();
    griddep_launch_dependents();
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b >= B) return;
    const int n = n_tokens ? n_tokens[b] : T;
    const long long L = ctx[b];
    if (n >= 0 && n <= T && L >= 0 && L + n <= Lmax) ctx[b] = (int32_t)(L + n);
}

// ---- host side --------------------------------------------------------------------------------------------------

bool tensor_of(const char* who, const rapid_kv_rows* r, const void* p, int T, int H, int D, RopeTensor& x) {
    x.p = static_cast<__nv_bfloat16*>(const_cast<void*>(p));
    x.sh = r && r->stride_h ? r->stride_h : D;
    x.st = r && r->stride_t ? r->stride_t : (long long)H * D;
    x.sb = r && r->stride_b ? r->stride_b : (long long)T * H * D;
    if (x.sh % 8 || x.st % 8 || x.sb % 8 || x.sh <= 0 || x.st <= 0 || x.sb <= 0 || ((uintptr_t)p & 15)) {
        set_error("%s: the rows' strides must be positive multiples of 8 elements, their pointers 16-byte aligned", who);
        return false;
    }
    return true;
}

// An output has room for its rows, and where it is its input it is so with the same strides.
bool output_of(const char* who, const rapid_kv_rows* r, void* p, int T, int H, int D, const RopeTensor& in, RopeTensor& x) {
    if (!tensor_of(who, r, p, T, H, D, x)) return false;
    if (x.sh < D || x.st < D || x.sb < D || (x.p == in.p && (x.sh != in.sh || x.st != in.st || x.sb != in.sb))) {
        set_error("%s: an output's strides must be at least head_dim, and its input's where it is written in place", who);
        return false;
    }
    return true;
}

int rope_of(const char* who, const rapid_rope* rope, RopeArgs& a) {
    if (a.B <= 0 || a.T <= 0 || a.D <= 0 || a.Hq < 0 || a.Hkv < 0 || a.B > 65535 || a.Hq > 65535 || a.Hkv > 65535 ||
        a.T > 0x7fffffff - 64) {
        set_error("%s: invalid shape (B=%d T=%d Hq=%d Hkv=%d D=%d)", who, a.B, a.T, a.Hq, a.Hkv, a.D);
        return RAPID_ERR_INVALID_ARG;
    }
    if (!rope || !rope->inv_freq) {
        set_error("%s: NULL rope or inv_freq", who);
        return RAPID_ERR_INVALID_ARG;
    }
    a.rd = rope->rotary_dim ? rope->rotary_dim : a.D;
    if (a.D % 16 || a.D > kRopeMaxD || a.rd < 16 || a.rd % 16 || a.rd > a.D) {
        set_error("%s: head_dim must be a multiple of 16 and at most %d, rotary_dim a multiple of 16 and at most head_dim", who, kRopeMaxD);
        return RAPID_ERR_UNSUPPORTED;
    }
    const int axes = rope->n_axes ? rope->n_axes : 1;
    if (axes < 1 || axes > 4) {
        set_error("%s: n_axes must be 1 to 4", who);
        return RAPID_ERR_INVALID_ARG;
    }
    if (!a.positions && axes > 1) {
        set_error("%s: several axes need positions", who);
        return RAPID_ERR_INVALID_ARG;
    }
    if (rope->pair_axis)
        for (int i = 0; i < a.rd / 2; ++i) {
            if (rope->pair_axis[i] >= axes) {
                set_error("%s: pair_axis[%d] is %d of %d axes", who, i, rope->pair_axis[i], axes);
                return RAPID_ERR_INVALID_ARG;
            }
            a.axis_bits[i / 16] |= (uint32_t)rope->pair_axis[i] << (2 * (i % 16));
        }
    a.inv_freq = rope->inv_freq;
    a.scale = rope->scale != 0.f ? rope->scale : 1.f;
    if (!isfinite(a.scale)) {
        set_error("%s: scale must be finite", who);
        return RAPID_ERR_INVALID_ARG;
    }
    a.sin_sign = a.scale;
    return RAPID_OK;
}

int launch(RopeArgs& a, int interleaved, cudaStream_t stream) {
    // As many tokens a block as give its threads four to six items each, fewer while that leaves SMs without four blocks.  (Two videos
    // at 32 heads of 128, four tokens: 100 us, two 136, eight 111; a prompt at 10 heads of 64, sixteen tokens: 7.4 us, four 9.2.)
    int dev = 0, sms = 0;
    RAPID_CUDA_CHECK(cudaGetDevice(&dev));
    RAPID_CUDA_CHECK(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    const int64_t items = (int64_t)(a.Hq + (a.ctx ? 2 : 1) * a.Hkv) * (a.D / 16);
    a.tokens = kRopeMaxTokens;
    while (a.tokens > 1 && (a.tokens * items > 6 * kRopeThreads || (int64_t)a.B * a.T < (int64_t)4 * a.tokens * sms)) a.tokens /= 2;
    const dim3 grid((a.T + a.tokens - 1) / a.tokens, a.B);
    RAPID_CUDA_CHECK(launch_dependent(interleaved ? rope_kernel<true> : rope_kernel<false>, grid, dim3(kRopeThreads), 0, stream, a));
    count_launch(1);
    return RAPID_OK;
}

}  // namespace

int launch_rope_apply(const void* q, const rapid_kv_rows* q_rows, void* q_out, const rapid_kv_rows* q_out_rows, const void* k,
                      const rapid_kv_rows* k_rows, void* k_out, const rapid_kv_rows* k_out_rows, int B, int T, int Hq, int Hkv,
                      int D, const int32_t* positions, const rapid_rope* rope, int inverse, cudaStream_t stream) {
    const char* who = "rapid_rope_apply";
    if (!positions || (!q && !k) || !q != !q_out || !k != !k_out || (q && Hq <= 0) || (k && Hkv <= 0)) {
        set_error("%s: NULL argument or no heads", who);
        return RAPID_ERR_INVALID_ARG;
    }
    RopeArgs a = {};
    a.B = B;
    a.T = T;
    a.Hq = q ? Hq : 0;
    a.Hkv = k ? Hkv : 0;
    a.D = D;
    a.positions = positions;
    const int rc = rope_of(who, rope, a);
    if (rc != RAPID_OK) return rc;
    if (inverse) a.sin_sign = -a.scale;
    if ((q && (!tensor_of(who, q_rows, q, T, Hq, D, a.q) || !output_of(who, q_out_rows, q_out, T, Hq, D, a.q, a.qo))) ||
        (k && (!tensor_of(who, k_rows, k, T, Hkv, D, a.k) || !output_of(who, k_out_rows, k_out, T, Hkv, D, a.k, a.ko))))
        return RAPID_ERR_UNSUPPORTED;
    return launch(a, rope->interleaved, stream);
}

int launch_kv_append_rope(const void* q, const rapid_kv_rows* q_rows, const void* k_new, const void* v_new,
                          const rapid_kv_rows* rows, int T, const int32_t* n_tokens, void* q_out, void* k_cache, void* v_cache,
                          const rapid_paged_kv* paged, const int32_t* block_table, const int32_t* ctx_lens,
                          int32_t* ctx_lens_out, const rapid_rope* rope, const int32_t* positions,
                          const rapid_attn_shape* shape, int32_t* status_word, cudaStream_t stream) {
    const char* who = paged ? "rapid_kv_append_rope_paged" : "rapid_kv_append_rope";
    if (!k_new || !v_new || !k_cache || !v_cache || !ctx_lens || !shape || !status_word || !q != !q_out) {
        set_error("%s: NULL argument", who);
        return RAPID_ERR_INVALID_ARG;
    }
    const rapid_attn_shape& s = *shape;
    RopeArgs a = {};
    a.B = s.B;
    a.T = T;
    a.Hq = q ? s.Hq : 0;
    a.Hkv = s.Hkv;
    a.D = s.D;
    a.positions = positions;
    if (s.Hkv <= 0 || (q && s.Hq <= 0) || s.Lmax <= 0 || s.Lmax > 0x7fffffffLL) {
        set_error("%s: invalid shape (Hq=%d Hkv=%d Lmax=%lld)", who, s.Hq, s.Hkv, (long long)s.Lmax);
        return RAPID_ERR_INVALID_ARG;
    }
    const int rc = rope_of(who, rope, a);
    if (rc != RAPID_OK) return rc;
    if (paged) {
        if (paged->block_size <= 0 || paged->num_blocks <= 0 || paged->max_blocks_per_seq <= 0 ||
            s.Lmax != (int64_t)paged->max_blocks_per_seq * paged->block_size) {
            set_error("%s: block_size, num_blocks and max_blocks_per_seq must be positive and shape->Lmax their capacity", who);
            return RAPID_ERR_INVALID_ARG;
        }
        a.cl = paged->stride_l ? paged->stride_l : s.D;
        a.ch = paged->stride_h ? paged->stride_h : paged->block_size * a.cl;
        a.cb = paged->stride_block ? paged->stride_block : s.Hkv * a.ch;
        a.block_table = block_table;
        a.block_size = paged->block_size;
        a.num_blocks = paged->num_blocks;
        a.max_blocks = paged->max_blocks_per_seq;
    } else {
        a.cl = s.kv_stride_l ? s.kv_stride_l : s.D;
        a.ch = s.kv_stride_h ? s.kv_stride_h : s.Lmax * a.cl;
        a.cb = s.kv_stride_b ? s.kv_stride_b : s.Hkv * a.ch;
    }
    if (a.cl < s.D || a.cl % 8 || a.ch % 8 || a.cb % 8 || a.ch <= 0 || a.cb <= 0 || (((uintptr_t)k_cache | (uintptr_t)v_cache) & 15)) {
        set_error("%s: the cache's strides must be positive multiples of 8 elements, its pointers 16-byte aligned", who);
        return RAPID_ERR_UNSUPPORTED;
    }
    if ((q && (!tensor_of(who, q_rows, q, T, s.Hq, s.D, a.q) || !output_of(who, nullptr, q_out, T, s.Hq, s.D, a.q, a.qo))) ||
        !tensor_of(who, rows, k_new, T, s.Hkv, s.D, a.k) || !tensor_of(who, rows, v_new, T, s.Hkv, s.D, a.v))
        return RAPID_ERR_UNSUPPORTED;
    a.k_cache = static_cast<__nv_bfloat16*>(k_cache);
    a.v_cache = static_cast<__nv_bfloat16*>(v_cache);
    a.Lmax = s.Lmax;
    a.n_tokens = n_tokens;
    a.ctx = ctx_lens;
    a.status = status_word;
    const bool in_place = ctx_lens_out == ctx_lens;
    a.ctx_out = in_place ? nullptr : ctx_lens_out;
    const int rc2 = launch(a, rope->interleaved, stream);
    if (rc2 != RAPID_OK || !in_place) return rc2;
    RAPID_CUDA_CHECK(launch_dependent(rope_lens_kernel, dim3((s.B + 127) / 128), dim3(128), 0, stream, ctx_lens_out, n_tokens, s.B, T,
                                      (long long)s.Lmax));
    count_launch(1);
    return RAPID_OK;
}

}  // namespace rapid
