// Operands of the attention kernels over cached rows (snapkv_decode.hip, snapkv_paged.hip): the 16x16x32 products of both
// two-byte types, the split of a probability into two of them, and the 0/1 operand that transposes a value tile by product.
#ifndef SNAPKV_ATTN_H_
#define SNAPKV_ATTN_H_

#include <hip/hip_runtime.h>

namespace snapkv {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 dbf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 df16x8;
typedef __attribute__((ext_vector_type(4))) float dfx4;
typedef __attribute__((ext_vector_type(2))) _Float16 df16x2;

struct dec_bf16 {};
struct dec_f16 {};

__device__ __forceinline__ dfx4 mma(dec_bf16, uint4 a, uint4 b, dfx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(dbf16x8, a), __builtin_bit_cast(dbf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ dfx4 mma(dec_f16, uint4 a, uint4 b, dfx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(df16x8, a), __builtin_bit_cast(df16x8, b), c, 0, 0, 0);
}

// Two fp32 values that are exactly representable in the storage type, packed (first in the low half).
__device__ __forceinline__ unsigned pack_exact(dec_bf16, float a, float b) {
    return (__float_as_uint(a) >> 16) | (__float_as_uint(b) & 0xFFFF0000u);
}
__device__ __forceinline__ unsigned pack_exact(dec_f16, float a, float b) {
    const df16x2 h = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(unsigned, h);
}

// p >= 0 split into hi + lo of the storage type, both by truncation: bf16 less than 2^-14 of p lost, fp16 less than 2^-20 as long
// as lo is a normal number.
__device__ __forceinline__ void split2(dec_bf16, float a, float b, unsigned& hi, unsigned& lo) {
    const unsigned ua = __float_as_uint(a) & 0xFFFF0000u, ub = __float_as_uint(b) & 0xFFFF0000u;
    hi = (ua >> 16) | ub;
    const float ra = a - __uint_as_float(ua), rb = b - __uint_as_float(ub);
    lo = (__float_as_uint(ra) >> 16) | (__float_as_uint(rb) & 0xFFFF0000u);
}
__device__ __forceinline__ void split2(dec_f16, float a, float b, unsigned& hi, unsigned& lo) {
    const df16x2 h = __builtin_bit_cast(df16x2, __builtin_amdgcn_cvt_pkrtz(a, b));
    hi = __builtin_bit_cast(unsigned, h);
    const float ra = a - (float)h.x, rb = b - (float)h.y;
    lo = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_pkrtz(ra, rb));
}

template <typename T> __device__ __forceinline__ unsigned one_bits();
template <> __device__ __forceinline__ unsigned one_bits<dec_bf16>() { return 0x3F80u; }
template <> __device__ __forceinline__ unsigned one_bits<dec_f16>() { return 0x3C00u; }

// Selection operand: column n = l%16 of the 32 x 16 matrix that copies contraction element
// 16*half + n.  A lane's slice covers elements 8*(l/16) .. +7.
template <typename T> __device__ __forceinline__ uint4 selector(int lane, int half) {
    const int n = lane & 15, kg = lane >> 4;
    const int e = 16 * half + n - 8 * kg;   // which of this lane's eight elements, if any
    unsigned w[4] = {0u, 0u, 0u, 0u};
    if (e >= 0 && e < 8) w[e >> 1] = one_bits<T>() << (16 * (e & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

}  // namespace
}  // namespace snapkv
#endif
