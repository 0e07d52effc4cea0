// Products of 8-bit codes (include/tsvd_int8.h) for any number of tokens: y = (Q W^T) s t + bias on v_mfma_i32_16x16x64_i8, sums exact in int32.
#include "tsvd_int8.h"

#include <algorithm>

#include "tsvd_epilogue.h"

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// The four results of a lane in a 16 x 16 block: token `token`, rows row0 .. row0 + 3.
__device__ __forceinline__ void store_block(void* y, long long ldy, int token_major, int out_bf16, const float* t, const float* s, const float* bias, long long M, long long B,
                                            long long token, long long row0, i32x4 acc) {
    if (token >= B) return;
    const float sb = s[token];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const long long row = row0 + v;
        if (row >= M) return;
        const float f = int8_result(acc[v], t[row], sb, bias ? bias[row] : 0.f);
        tsvd_store_y(y, token_major ? (size_t)token * ldy + row : (size_t)row * ldy + token, f, out_bf16);
    }
}

// A wavefront multiplies 64 rows by 64 tokens, operands straight from memory; four of them share a workgroup, 128 x 128.
__global__ void __launch_bounds__(256)
int8_gemm_kernel(const uint8_t* __restrict__ tiles, int nkt, long long strips, const uint8_t* __restrict__ q, long long ldq, const float* __restrict__ t, const float* __restrict__ s,
                 const float* __restrict__ bias, void* __restrict__ y, long long ldy, long long M, long long B, int token_major, int out_bf16) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
    const long long strip0 = (long long)blockIdx.x * 8 + (wave & 1) * 4, b0 = (long long)blockIdx.y * 128 + (wave >> 1) * 64;
    const uint8_t *w[4], *x[4];
#pragma unroll
    for (int a = 0; a < 4; ++a) {
        w[a] = tiles + min(strip0 + a, strips - 1) * nkt * 1024 + lane * 16;       // (rows and tokens beyond the last: that one's again, not stored)
        x[a] = q + min(b0 + 16 * a + i, B - 1) * ldq;
    }
    i32x4 acc[4][4] = {};
    for (int T = 0; T < nkt; ++T) {
        const long long k = min((long long)T * 64 + 16 * g, ldq - 16);             // (beyond the row: the weights' codes are zero there)
        i32x4 wa[4], xb[4];
#pragma unroll
        for (int a = 0; a < 4; ++a) wa[a] = *reinterpret_cast<const i32x4*>(w[a] + (size_t)T * 1024), xb[a] = *reinterpret_cast<const i32x4*>(x[a] + k);
#pragma unroll
        for (int a = 0; a < 4; ++a)
#pragma unroll
            for (int b = 0; b < 4; ++b) acc[a][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wa[a], xb[b], acc[a][b], 0, 0, 0);
    }
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int b = 0; b < 4; ++b) store_block(y, ldy, token_major, out_bf16, t, s, bias, M, B, b0 + 16 * b + i, (strip0 + a) * 16 + 4 * g, acc[a][b]);
}

}  // namespace

hipError_t tsvd_int8_gemm(const tsvd_int8_problem& p, hipStream_t stream) {
    const tsvd_int8_handle& h = *p.h;
    for (long long b0 = 0; b0 < p.B; b0 += 65535LL * 128) {        // (grid.y)
        const long long B = std::min<long long>(p.B - b0, 65535LL * 128);
        uint8_t* y = static_cast<uint8_t*>(p.y) + (size_t)(p.token_major ? b0 * p.ldy : b0) * (p.out_bf16 ? 2 : 4);
        hipLaunchKernelGGL(int8_gemm_kernel, dim3((unsigned)((h.M + 127) / 128), (unsigned)((B + 127) / 128)), dim3(256), 0, stream, h.tiles(), h.nkt, h.strips,
                           reinterpret_cast<const uint8_t*>(p.codes) + b0 * p.ldq, p.ldq, h.scales(), p.scales + b0, p.bias, y, p.ldy, h.M, B, p.token_major, p.out_bf16);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
