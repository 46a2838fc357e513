// What the attention kernels with rows on the M axis share: one lane and whole-warp waits, packed fp32 arithmetic, exponentials off the
// special-function unit, the rescaling of an accumulator in tensor memory; on the host, tensor maps of 64-column boxes.
#pragma once

#include "common.cuh"
#include "tcgen05.cuh"

namespace rapid {

namespace {

// One lane of a converged warp.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred P;\n\telect.sync _|P, 0xffffffff;\n\tselp.u32 %0, 1, 0, P;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, const WaitCtx& wc) {
    return __all_sync(0xffffffffu, mbar_wait_bounded(bar, parity, wc));
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

}  // namespace

}  // namespace rapid
