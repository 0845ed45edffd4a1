// Shared by the two kernels of the 4-bit LM head: the problem, the expansion of codes to bf16, the store of a logit.
#pragma once

#include <cuda_bf16.h>

#include "polyspec_kernels.cuh"

namespace polyspec {

struct W4Problem {
    const void* hidden;             // [rows, d] bf16
    const uint32_t* codes;          // [V, d / 8]
    const void* scales;             // [V, d / group] bf16
    const unsigned char* zeros;     // [V, d / group] or nullptr
    int rows, V, d, group;
    void* out;                      // [rows, V]
};

// The tensor-core kernel (w4_tensor.cu): any number of rows.
cudaError_t launch_w4_tensor(const W4Problem& q, polyspec_dtype dt, int32_t* device_status, cudaStream_t stream);

namespace w4 {

// The eight weights of a word as four bf16 pairs (0,1) (2,3) (4,5) (6,7), the zero point subtracted.
// `magic` holds 128 + z twice; 128 + q, 128 + z and q - z are all exact in bf16.  `exponent` is kExponent, which callers pass
// from a kernel parameter: a value the compiler cannot see stays in a register, so that mask and exponent are one three-input
// instruction; as two immediates they are two.
constexpr uint32_t kExponent = 0x43004300u;
__device__ __forceinline__ void expand(uint32_t word, uint32_t magic, uint32_t exponent, uint32_t (&pairs)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t x = ((word >> (4 * i)) & 0x000f000fu) | exponent;
        asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(pairs[i]) : "r"(x), "r"(magic));
    }
}

template <int DT>
__device__ __forceinline__ void store_logit(void* out, size_t at, float x)
{
    if (DT == POLYSPEC_F32) static_cast<float*>(out)[at] = x;
    else static_cast<__nv_bfloat16*>(out)[at] = __float2bfloat16_rn(x);         // rounded once, from the fp32 sum
}

}  // namespace w4
}  // namespace polyspec
