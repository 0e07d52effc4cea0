// Internal: layers in 8-bit integers (include/tsvd_int8.h): the packed weights, the launches, and what every kernel does alike.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/tsvd_int8.h"
#include "tsvd_wave.h"

// Packed weights: scales [strips * 16] fp32 (rounded up to 256 bytes), then tiles of 16 rows x 64 columns of codes, 1 KiB each: lane l of a
// wavefront finds row l % 16, columns 16 (l / 16) ... + 15, the operand of v_mfma_i32_16x16x64_i8.  A strip's tiles are contiguous along the
// contraction, an even number of them; rows beyond M and columns beyond N hold zeros, so whatever the activations' codes hold
// beyond N adds nothing.
#define TSVD_INT8_MAX_N ((1 << 17) - 1)
#define TSVD_INT8_MAX_M (1 << 24)
#define TSVD_INT8_MAX_B (1 << 24)
#define TSVD_INT8_MAX_PITCH (1 << 22)                // of codes that a product reads: 256 rows within 32-bit places
#define TSVD_INT8_FLOOR 7.888609052210118e-31f       // 2^-100: the largest magnitude that a token is scaled by at least

struct tsvd_int8_handle {
    int device, cu_count;
    long long M, N, strips;
    int nkt;                  // tiles of a strip
    uint8_t* blob;
    bool owns_blob;
    const float* scales() const { return reinterpret_cast<const float*>(blob); }
    const uint8_t* tiles() const { return blob + (((size_t)strips * 64 + 255) & ~(size_t)255); }
};

struct tsvd_int8_problem {
    const tsvd_int8_handle* h;
    const int8_t* codes;
    long long ldq;
    const float* scales;
    long long B;
    const float* bias;
    void* y;
    int out_bf16, token_major;
    long long ldy;
};
hipError_t tsvd_int8_gemm(const tsvd_int8_problem& p, hipStream_t stream);       // tsvd_int8_gemm.hip: any number of tokens
hipError_t tsvd_int8_gemm_init();                                                // once for each device, as the next
hipError_t tsvd_int8_stream_init();
// tsvd_int8_stream.hip: few tokens; and from x, where it makes the codes itself (p.codes and p.scales are not used then).  rows: x is [B][ldx], else [N][ldx]
bool tsvd_int8_stream_serves(const tsvd_int8_handle& h, long long B);
hipError_t tsvd_int8_stream(const tsvd_int8_problem& p, hipStream_t stream);
bool tsvd_int8_stream_makes(const tsvd_int8_handle& h, long long B);
hipError_t tsvd_int8_stream_from(const tsvd_int8_problem& p, const void* x, bool x_bf16, bool rows, long long ldx, hipStream_t stream);

namespace {

// The scale of a token and the factor of its codes, from the bits of its largest magnitude (an infinity or NaN: NaN, which every output of the token shows).
__device__ __forceinline__ void int8_factors(uint32_t top_bits, float* scale, float* factor) {
    const float a = fmaxf(__uint_as_float(top_bits), TSVD_INT8_FLOOR);
    const bool finite = top_bits < 0x7F800000u;
    *scale = finite ? __fdiv_rn(a, 127.f) : __uint_as_float(0x7FC00000u);
    *factor = finite ? __fdiv_rn(127.f, a) : 0.f;
}
// The code of x in the low byte: adding 1.5 2^23 rounds the exact product to the nearest whole number, ties to even.
__device__ __forceinline__ uint32_t int8_code(float x, float factor) { return __float_as_uint(fmaf(x, factor, 12582912.f)); }
__device__ __forceinline__ uint32_t int8_pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}
// An output from the exact sum: the same three roundings in every kernel.
__device__ __forceinline__ float int8_result(int sum, float row_scale, float token_scale, float bias) {
    return fmaf(__fmul_rn((float)sum, row_scale), token_scale, bias);
}

// Eight consecutive activations, at any element alignment.
template <typename X>
struct int8_eight;
template <>
struct int8_eight<uint16_t> {
    typedef uint32_t vec __attribute__((ext_vector_type(4)));
    typedef vec vec_at __attribute__((aligned(2)));
    vec v;
    __device__ __forceinline__ void zero() { v = vec{0, 0, 0, 0}; }
    __device__ __forceinline__ void load(const uint16_t* p) { v = *reinterpret_cast<const vec_at*>(p); }
    __device__ __forceinline__ void set(int e, uint16_t x) { v[e >> 1] |= (uint32_t)x << (16 * (e & 1)); }
    __device__ __forceinline__ float get(int e) const { return __uint_as_float(e & 1 ? v[e >> 1] & 0xFFFF0000u : v[e >> 1] << 16); }
    // the values from number `by` on, zeros behind them (0 <= by <= 8)
    __device__ __forceinline__ void shift(int by) {
        typedef unsigned __int128 u128;
        v = by < 8 ? __builtin_bit_cast(vec, __builtin_bit_cast(u128, v) >> (16 * by)) : vec{0, 0, 0, 0};
    }
};
template <>
struct int8_eight<float> {
    typedef float vec __attribute__((ext_vector_type(4)));
    typedef vec vec_at __attribute__((aligned(4)));
    vec a, b;
    __device__ __forceinline__ void zero() { a = b = vec{0.f, 0.f, 0.f, 0.f}; }
    __device__ __forceinline__ void load(const float* p) {
        a = *reinterpret_cast<const vec_at*>(p);
        b = *reinterpret_cast<const vec_at*>(p + 4);
    }
    __device__ __forceinline__ void set(int e, float x) { if (e < 4) a[e] = x; else b[e - 4] = x; }
    __device__ __forceinline__ float get(int e) const { return e < 4 ? a[e] : b[e - 4]; }
    __device__ __forceinline__ void shift(int by) {
        float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
#pragma unroll
        for (int s = 1; s <= 8; s *= 2)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = by & s ? (e + s < 8 ? x[e + s] : 0.f) : x[e];
        a = vec{x[0], x[1], x[2], x[3]};
        b = vec{x[4], x[5], x[6], x[7]};
    }
};
// Values at .. at + 7 of a row of n, zeros behind its end.  The last ones are read to end at its end and shifted: one load as elsewhere, where a value at a time would be
// seven, one behind the other.
template <typename X>
__device__ __forceinline__ int8_eight<X> int8_load8(const X* row, int at, int n) {
    int8_eight<X> r;
    if (n >= 8) {                                                // (the same for all lanes of a call's launch, nearly always)
        const int from = min(at, n - 8);
        r.load(row + from);
        if (at > from) r.shift(min(at - from, 8));
    } else {
        r.zero();
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (at + e < n) r.set(e, row[at + e]);
    }
    return r;
}
// The same of several rows (row(k)), at one place: the loads go out together, no branch between them.
template <int N, typename X, typename F>
__device__ __forceinline__ void int8_loads8(int8_eight<X> (&r)[N], F&& row, int at, int n) {
    if (n >= 8) {
        const int from = min(at, n - 8);
#pragma unroll
        for (int k = 0; k < N; ++k) r[k].load(row(k) + from);
        if (at > from)
#pragma unroll
            for (int k = 0; k < N; ++k) r[k].shift(min(at - from, 8));
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) r[k] = int8_load8(row(k), at, n);
    }
}
template <typename X>
__device__ __forceinline__ uint32_t int8_top8(const int8_eight<X>& r, uint32_t top) {
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(r.get(e)) & 0x7FFFFFFFu);
    return top;
}
template <typename X>
__device__ __forceinline__ uint2 int8_codes8(const int8_eight<X>& r, float factor) {
    uint32_t c[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = int8_code(r.get(e), factor);
    return uint2{int8_pack4(c[0], c[1], c[2], c[3]), int8_pack4(c[4], c[5], c[6], c[7])};
}
// The largest over T neighbouring lanes, in all of them.
template <int T>
__device__ __forceinline__ uint32_t int8_lanes_top(uint32_t v) {
    if constexpr (T > 32) v = max(v, lane_xor32<32>(v));
    if constexpr (T > 16) v = max(v, lane_xor32<16>(v));
    if constexpr (T > 8) v = max(v, lane_xor32<8>(v));
    if constexpr (T > 4) v = max(v, lane_xor32<4>(v));
    if constexpr (T > 2) v = max(v, lane_xor32<2>(v));
    return max(v, lane_xor32<1>(v));
}


typedef int i32x4 __attribute__((ext_vector_type(4)));

// 16 bytes a lane from a buffer to LDS, lane l's at lds + 16 l.  The compiler does not see what it moves: every use waits for vmcnt by hand.
__device__ __forceinline__ void load_to_lds(i32x4 rsrc, uint32_t lds, int voff, int soff) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" :: "s"(lds), "v"(voff), "s"(rsrc), "s"(soff) : "memory");
}
__device__ __forceinline__ i32x4 buffer_of(const void* base, uint32_t bytes) {
    const uint64_t a = reinterpret_cast<uintptr_t>(base);
    return i32x4{(int)__builtin_amdgcn_readfirstlane((uint32_t)a), (int)__builtin_amdgcn_readfirstlane((uint32_t)(a >> 32) & 0xFFFF), (int)__builtin_amdgcn_readfirstlane(bytes), 0x00020000};
}
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
    static_assert(N >= 0 && N <= 63, "vmcnt has six bits");
    asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory");
}

}  // namespace
