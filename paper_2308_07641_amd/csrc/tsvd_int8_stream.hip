// Products of 8-bit codes (include/tsvd_int8.h) for few tokens: the weights pass once through the matrix unit, straight from memory into operand registers
// (v_mfma_i32_16x16x64_i8, 16 rows x 16 tokens), and that stream bounds the call.
//
// A workgroup owns a run of strips of 16 rows.  Its wavefronts split the contraction (and, where it is short, the strips): a wavefront holds the codes of its part in
// registers, KT tiles of 64 indices by NB blocks of 16 tokens, and goes through the strips with the tiles of the next two on their way.  The parts meet in LDS
// as integers, by additions whose order does not matter.  Nothing stands between the launch and the stream but the codes.
//
// MAKE: the codes are made here, by every workgroup for itself: each lane reads the activations of its operand places, in either layout, the largest magnitudes of the tokens
// meet in LDS (the one barrier before the end), and the codes are there in operand order, without a launch of their own or a way through memory.  HOLD: they stay in registers in
// between; else (contractions longer than the wavefronts hold at once) they are read a second time, from the caches.
#include "tsvd_int8.h"

#include <algorithm>
#include <type_traits>

#include "tsvd_epilogue.h"

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// A 16 x 16 block of sums in LDS: rows of 20, so that the four rows that a cycle adds to stand in different banks.
constexpr int BLOCK_PITCH = 20, BLOCK = 16 * BLOCK_PITCH;

struct stream_args {
    const uint8_t* tiles;
    const uint8_t* q;             // codes, or (MAKE) activations
    long long ldq;                // ... bytes of codes, elements of activations
    const float *t, *s, *bias;
    void* y;
    long long ldy;
    long long M;
    int nkt, strips, N, B;
    int strips_wg, kw, kw_log2, sw;      // strips of a workgroup; wavefronts along the contraction (a power of two), along the strips
    int token_major, out_bf16;
};

__device__ __forceinline__ i32x4 codes16(uint2 a, uint2 b) { return i32x4{(int)a.x, (int)a.y, (int)b.x, (int)b.y}; }

// Sixteen activations of a token from index `at` on.  ROWS: side by side (zeros beyond N); else `ld` elements apart (beyond N the last one again: the weights' codes
// are zero there).
template <bool ROWS, typename X>
__device__ __forceinline__ void load16(int8_eight<X> (&v)[2], const X* x, long long ld, int at, int N) {
    if constexpr (ROWS) {
        v[0] = int8_load8(x, at, N);
        v[1] = int8_load8(x, at + 8, N);
    } else {
        X e[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) e[k] = x[(long long)min(at + k, N - 1) * ld];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            v[h].zero();
#pragma unroll
            for (int k = 0; k < 8; ++k) v[h].set(k, e[8 * h + k]);
        }
    }
}

template <int KT, int NB, typename MAKE, bool ROWS, bool HOLD>
__global__ void __launch_bounds__(1024)
int8_stream_kernel(stream_args p) {
    constexpr bool make = !std::is_same<MAKE, void>::value;
    extern __shared__ __align__(16) int smem[];
    __shared__ uint32_t tops[16 * 16];
    __shared__ float token_scale[16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
    const int ks = wave & (p.kw - 1), sg = wave >> p.kw_log2;
    const int strip0 = blockIdx.x * p.strips_wg, strips = min(p.strips_wg, p.strips - strip0);
    const uint32_t bytes = (uint32_t)strips * p.nkt * 1024;
    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p.tiles + (size_t)strip0 * p.nkt * 1024), 0, bytes, 0x00020000);
    const int chunk_tiles = p.kw * KT;
    i32x4 w[2][KT];
    // (a strip or tile beyond the last: outside of the buffer, nothing is read)
    auto load = [&](int set, int strip, int k0) {
#pragma unroll
        for (int k = 0; k < KT; ++k) {
            const bool there = strip < strips && k0 + k < p.nkt;
            const uint32_t at = there ? (uint32_t)(strip * p.nkt + k0 + k) * 1024u : bytes;
            w[set][k] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, lane * 16, (int)at, 0));
        }
    };
    i32x4 x[NB][KT];
    float factor = 0.f;
    // (MAKE) the values of this lane's places: token i (beyond the last: that one's again), indices 16 g ... of its tiles
    typedef typename std::conditional<make, MAKE, float>::type value;
    const value* row = reinterpret_cast<const value*>(p.q) + (make ? (long long)min(i, p.B - 1) * (ROWS ? p.ldq : 1) : 0);
    auto load_x = [&](int8_eight<value> (&v)[KT][2], int k0) {
#pragma unroll
        for (int k = 0; k < KT; ++k) load16<ROWS>(v[k], row, p.ldq, (k0 + k) * 64 + 16 * g, p.N);
    };
    auto codes = [&](const int8_eight<value> (&v)[KT][2]) {
#pragma unroll
        for (int k = 0; k < KT; ++k) x[0][k] = codes16(int8_codes8(v[k][0], factor), int8_codes8(v[k][1], factor));
    };
    if constexpr (make) {
        int8_eight<value> v[KT][2];
        uint32_t top = 0;
        auto raise = [&] {
#pragma unroll
            for (int k = 0; k < KT; ++k) top = int8_top8(v[k][1], int8_top8(v[k][0], top));
        };
        load_x(v, ks * KT);
        if constexpr (HOLD) {
            load(0, sg, ks * KT);
            load(1, sg + p.sw, ks * KT);
        }
        for (int n = threadIdx.x; n < strips * NB * BLOCK; n += blockDim.x) smem[n] = 0;
        raise();
        if constexpr (!HOLD)
            for (int c0 = chunk_tiles; c0 < p.nkt; c0 += chunk_tiles) {
                load_x(v, c0 + ks * KT);
                raise();
            }
        top = max(top, lane_xor32<16>(top));
        top = max(top, lane_xor32<32>(top));
        if (lane < 16) tops[wave * 16 + lane] = top;
        __syncthreads();
        top = 0;
        for (int n = 0; n < p.kw; ++n) top = max(top, tops[n * 16 + i]);
        float scale;
        int8_factors(top, &scale, &factor);
        if (threadIdx.x < 16) token_scale[threadIdx.x] = scale;
        if constexpr (HOLD) codes(v);
    } else {
        for (int n = threadIdx.x; n < strips * NB * BLOCK; n += blockDim.x) smem[n] = 0;
        __syncthreads();
    }
    for (int c0 = 0; c0 < p.nkt; c0 += chunk_tiles) {
        const int k0 = c0 + ks * KT;
        if constexpr (!make) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int k = 0; k < KT; ++k) {
                    // (beyond the row's end or the last tile: any codes do, the weights' are zero)
                    const long long at = min((long long)(k0 + k) * 64 + 16 * g, p.ldq - 16);
                    x[b][k] = *reinterpret_cast<const i32x4*>(p.q + (long long)min(16 * b + i, p.B - 1) * p.ldq + at);
                }
            load(0, sg, k0);
            load(1, sg + p.sw, k0);
        } else if constexpr (!HOLD) {
            int8_eight<value> v[KT][2];
            load_x(v, k0);
            load(0, sg, k0);
            load(1, sg + p.sw, k0);
            codes(v);
        }
        auto strip = [&](int set, int at) {
            i32x4 acc[NB] = {};
#pragma unroll
            for (int k = 0; k < KT; ++k)
#pragma unroll
                for (int b = 0; b < NB; ++b) acc[b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[set][k], x[b][k], acc[b], 0, 0, 0);
            load(set, at + 2 * p.sw, k0);
            if (at < strips) {
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int v = 0; v < 4; ++v) atomicAdd(&smem[(at * NB + b) * BLOCK + (4 * g + v) * BLOCK_PITCH + i], acc[b][v]);
            }
        };
        for (int at = sg; at < strips; at += 2 * p.sw) {
            strip(0, at);
            strip(1, at + p.sw);
        }
    }
    __syncthreads();
    // lanes along the rows of a token (token-major y, and single tokens), else along the tokens of a row
    const int rows = (int)min((long long)strips * 16, p.M - (long long)strip0 * 16), along_rows = p.token_major || p.B == 1;
    const int inner = along_rows ? rows : p.B, total = rows * p.B;
    for (int n = threadIdx.x; n < total; n += blockDim.x) {
        const int o = n / inner, e = n - o * inner, row = along_rows ? e : o, token = along_rows ? o : e;
        const long long m = (long long)strip0 * 16 + row;
        const int sum = smem[((row >> 4) * NB + (token >> 4)) * BLOCK + (row & 15) * BLOCK_PITCH + (token & 15)];
        const float f = int8_result(sum, p.t[m], make ? token_scale[token] : p.s[token], p.bias ? p.bias[m] : 0.f);
        tsvd_store_y(p.y, p.token_major ? (size_t)token * p.ldy + m : (size_t)m * p.ldy + token, f, p.out_bf16);
    }
}

constexpr int MAX_BLOCKS = 48;      // 60 KiB of sums

// How a launch is laid out: strips of a workgroup (all workgroups at once on the compute units, sums within 64 KiB of LDS), wavefronts and tiles of each.
struct stream_plan {
    int strips_wg, kw, sw, kt, nb;
};
stream_plan plan_of(long long strips, int nkt, long long B, int cus, int most) {
    stream_plan s;
    s.nb = B <= 16 ? 1 : B <= 32 ? 2 : 4;
    s.strips_wg = (int)std::max<long long>(1, std::min<long long>((strips + cus - 1) / cus, MAX_BLOCKS / s.nb));
    s.kt = std::min(most, s.nb == 1 ? 8 : 4);
    s.kw = 1;
    while (s.kw < 16 && s.kw * s.kt < nkt) s.kw *= 2;
    s.sw = 1;
    while (s.sw * 2 * s.kw <= 16 && s.sw * 2 <= s.strips_wg) s.sw *= 2;
    // wavefronts that have no strip of their own split the contraction further
    while (s.kt > 1 && s.kw * s.sw * 2 <= 16) s.kw *= 2, s.kt /= 2;
    while (s.kt > 1 && s.kw * (s.kt / 2) >= nkt) s.kt /= 2;
    return s;
}

template <int KT, int NB, typename MAKE, bool ROWS, bool HOLD>
hipError_t launch(const stream_args& a, int grid, hipStream_t stream) {
    // (sums within the 64 KiB that need no permission: plan_of)
    hipLaunchKernelGGL((int8_stream_kernel<KT, NB, MAKE, ROWS, HOLD>), dim3(grid), dim3(64 * a.kw * a.sw), (size_t)a.strips_wg * NB * BLOCK * 4, stream, a);
    return hipGetLastError();
}
template <int NB>
hipError_t launch_codes(int kt, const stream_args& a, int grid, hipStream_t stream) {
    if (kt == 1) return launch<1, NB, void, true, true>(a, grid, stream);
    if (kt == 2) return launch<2, NB, void, true, true>(a, grid, stream);
    if (kt == 4) return launch<4, NB, void, true, true>(a, grid, stream);
    if constexpr (NB == 1) return launch<8, NB, void, true, true>(a, grid, stream);
    return hipErrorInvalidValue;
}
template <typename X, bool ROWS>
hipError_t launch_make(int kt, const stream_args& a, int grid, hipStream_t stream) {
    if (a.nkt > a.kw * kt) return launch<4, 1, X, ROWS, false>(a, grid, stream);       // (kt is 4 then)
    if (kt == 1) return launch<1, 1, X, ROWS, true>(a, grid, stream);
    if (kt == 2) return launch<2, 1, X, ROWS, true>(a, grid, stream);
    return launch<4, 1, X, ROWS, true>(a, grid, stream);
}
stream_args args_of(const tsvd_int8_problem& p, const stream_plan& s) {
    const tsvd_int8_handle& h = *p.h;
    stream_args a = {};
    a.tiles = h.tiles(), a.nkt = h.nkt, a.strips = (int)h.strips, a.N = (int)h.N, a.t = h.scales(), a.M = h.M;
    a.s = p.scales, a.B = (int)p.B, a.bias = p.bias, a.y = p.y, a.ldy = p.ldy, a.token_major = p.token_major, a.out_bf16 = p.out_bf16;
    a.strips_wg = s.strips_wg, a.kw = s.kw, a.sw = s.sw;
    while (1 << a.kw_log2 < s.kw) ++a.kw_log2;
    return a;
}

constexpr int MAKE_TILES = 4;       // tiles whose activations, codes and next weights fit the 128 registers of a lane

}  // namespace

bool tsvd_int8_stream_serves(const tsvd_int8_handle&, long long B) { return B <= 64; }

hipError_t tsvd_int8_stream(const tsvd_int8_problem& p, hipStream_t stream) {
    const stream_plan s = plan_of(p.h->strips, p.h->nkt, p.B, p.h->cu_count, 8);
    stream_args a = args_of(p, s);
    a.q = reinterpret_cast<const uint8_t*>(p.codes), a.ldq = p.ldq;
    const int grid = (a.strips + s.strips_wg - 1) / s.strips_wg;
    return s.nb == 1 ? launch_codes<1>(s.kt, a, grid, stream) : s.nb == 2 ? launch_codes<2>(s.kt, a, grid, stream) : launch_codes<4>(s.kt, a, grid, stream);
}

// Whether the codes of B tokens are made in the launch of the product: up to 2^16 activations, which every workgroup reads (and, beyond 4096 features, reads twice).
bool tsvd_int8_stream_makes(const tsvd_int8_handle& h, long long B) { return B <= 16 && B * h.N <= 1 << 16; }

hipError_t tsvd_int8_stream_from(const tsvd_int8_problem& p, const void* x, bool x_bf16, bool rows, long long ldx, hipStream_t stream) {
    const stream_plan s = plan_of(p.h->strips, p.h->nkt, p.B, p.h->cu_count, MAKE_TILES);
    stream_args a = args_of(p, s);
    a.q = static_cast<const uint8_t*>(x), a.ldq = ldx;
    const int grid = (a.strips + s.strips_wg - 1) / s.strips_wg;
    if (rows) return x_bf16 ? launch_make<uint16_t, true>(s.kt, a, grid, stream) : launch_make<float, true>(s.kt, a, grid, stream);
    return x_bf16 ? launch_make<uint16_t, false>(s.kt, a, grid, stream) : launch_make<float, false>(s.kt, a, grid, stream);
}
