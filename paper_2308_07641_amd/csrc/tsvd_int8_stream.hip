// Products of 8-bit codes (include/tsvd_int8.h) for few tokens: the weights pass once through the matrix unit, straight from memory into operand registers
// (v_mfma_i32_16x16x64_i8, 16 rows x 16 tokens), and that stream bounds the call.
//
// A workgroup owns a run of strips of 16 rows and up to 64 tokens.  Its wavefronts split the contraction (and, where it is short, the strips): a wavefront holds the codes of its part in
// registers, KT tiles of 64 indices by NB blocks of 16 tokens, and goes through the strips, and on into the next part, with the tiles of the next two on their way.  The parts
// meet in LDS as integers, by additions whose order does not matter.  Nothing stands between the launch and the stream but the codes.
//
// Codes come by way of LDS, each wavefront's own, in pieces of 16 tokens by up to 256 bytes, the next two pieces on their way: an operand's 16 lanes in turn have 16 tokens, and
// read from memory like that take a request a lane (16 bytes a cycle and compute unit: 64 tokens of 16384 features 37 us, however few the rows).
//
// MAKE: the codes are made here, by every workgroup for itself: each lane reads a part of the activations (ROWS: token-major, eight side by side; else those of its operand
// places), the largest magnitudes of the tokens meet in LDS (the one barrier before the end), and the codes are there without a launch of their own.
//
// Measured, 16384 rows of 4096 features (64 MiB of weights, which stay in the memory-side cache): one token 11.8 us from its activations (5.7 TB/s), 16 tokens 11.9 us from codes and 13.5 from
// activations, 64 tokens 15.1 us.  Twelve such layers in turn, all weights from memory: one token 14.5 us (4.6 TB/s), 16 tokens 15.4 us.
#include "tsvd_int8.h"

#include <algorithm>
#include <type_traits>

#include "tsvd_epilogue.h"
#include "tsvd_kernels.h"

namespace {

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
    int nkt, strips, N;
    long long B;
    int strip_groups;                    // workgroups of a group of tokens (16 NB at most)
    int strips_wg, kw, kw_log2, sw;      // strips of a workgroup; wavefronts along the contraction (a power of two), along the strips
    int token_major, out_bf16;
};

__device__ __forceinline__ i32x4 codes16(uint2 a, uint2 b) { return i32x4{(int)a.x, (int)a.y, (int)b.x, (int)b.y}; }

// Pieces of codes in LDS: rows of 64 KT bytes, their 16 bytes exchanged so that 16 rows' stand in different banks.
template <int KT>
__device__ __forceinline__ int place(int row, int chunk) { return row * 64 * KT + ((chunk ^ (row / (4 / KT) % (4 * KT))) * 16); }

template <int KT, typename MAKE, bool ROWS>
constexpr int wave_bytes() { return std::is_same<MAKE, void>::value ? 2048 * KT : ROWS ? 1024 * KT : 0; }

template <int KT, int NB, typename MAKE, bool ROWS>
__global__ void __launch_bounds__(1024)
int8_stream_kernel(stream_args p) {
    constexpr bool make = !std::is_same<MAKE, void>::value;
    extern __shared__ __align__(16) int smem[];
    __shared__ uint32_t tops[16 * 16];
    __shared__ float token_scale[16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
    const int ks = wave & (p.kw - 1), sg = wave >> p.kw_log2;
    const int token_group = blockIdx.x / (unsigned)p.strip_groups, strip0 = (blockIdx.x - token_group * p.strip_groups) * p.strips_wg, strips = min(p.strips_wg, p.strips - strip0);
    const long long token0 = (long long)token_group * 16 * NB;
    const int B = (int)min(p.B - token0, 16ll * NB);
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
    // pieces: block u of chunk c, n = c NB + u
    uint8_t* stage = reinterpret_cast<uint8_t*>(smem + p.strips_wg * NB * BLOCK) + wave * wave_bytes<KT, MAKE, ROWS>();
    auto take = [&](int u, int set) {
#pragma unroll
        for (int k = 0; k < KT; ++k) x[u][k] = *reinterpret_cast<const i32x4*>(stage + set * 1024 * KT + place<KT>(i, 4 * k + g));
    };
    const uint32_t stage_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)stage;
    const uint32_t codes_bytes = make ? 0 : (uint32_t)((B - 1) * p.ldq) + (uint32_t)((p.N + 15) & ~15);
    const i32x4 qbuf = buffer_of(p.q + token0 * p.ldq, codes_bytes);
    // (tokens and indices beyond the last: zeros, or any codes, where the weights' are zero)
    int voff[KT];
#pragma unroll
    for (int j = 0; j < KT; ++j) {
        const int row = j * (16 / KT) + lane / (4 * KT);
        voff[j] = row * (int)p.ldq + place<KT>(row, lane % (4 * KT)) - row * 64 * KT;
    }
    auto request = [&](int n) {
        const int c = n / NB, u = n % NB;
        const uint32_t soff = min(16u * u * (uint32_t)p.ldq + (c * chunk_tiles + ks * KT) * 64u, codes_bytes);       // (what it leaves bounds voff)
#pragma unroll
        for (int j = 0; j < KT; ++j)
            load_to_lds(qbuf, __builtin_amdgcn_readfirstlane(stage_at) + ((n & 1) * KT + j) * 1024, voff[j], __builtin_amdgcn_readfirstlane(soff));
    };
    if constexpr (make) {
        typedef typename std::conditional<make, MAKE, float>::type value;
        const value* from = reinterpret_cast<const value*>(p.q);
        // ROWS: eight values of a token a lane, 64 / LT tokens at a time; else sixteen of token i for each tile (beyond the last token: that one's again), at the lane's operand places
        constexpr int LT = 8 * KT, STEP = 64 / LT;
        int8_eight<value> v[2 * KT];
        const int own = lane / LT, at = lane % LT;
#pragma unroll
        for (int k = 0; k < 2 * KT; ++k) {
            v[k].zero();
            if constexpr (ROWS) {
                if (k * STEP + own < B) v[k] = int8_load8(from + (long long)(k * STEP + own) * p.ldq, ks * KT * 64 + 8 * at, p.N);
            } else {
                value e[8];
#pragma unroll
                for (int n = 0; n < 8; ++n) e[n] = from[min(i, B - 1) + (long long)min((ks * KT + k / 2) * 64 + 16 * g + k % 2 * 8 + n, p.N - 1) * p.ldq];
#pragma unroll
                for (int n = 0; n < 8; ++n) v[k].set(n, e[n]);
            }
        }
        load(0, sg, ks * KT);
        load(1, sg + p.sw, ks * KT);
        for (int n = threadIdx.x; n < strips * NB * BLOCK; n += blockDim.x) smem[n] = 0;
        if constexpr (ROWS) {
#pragma unroll
            for (int k = 0; k < 2 * KT; ++k) {
                const uint32_t top = int8_lanes_top<LT>(int8_top8(v[k], 0));
                if (at == 0) tops[wave * 16 + k * STEP + own] = top;
            }
        } else {
            uint32_t top = 0;
#pragma unroll
            for (int k = 0; k < 2 * KT; ++k) top = int8_top8(v[k], top);
            top = max(top, lane_xor32<16>(top));
            top = max(top, lane_xor32<32>(top));
            if (lane < 16) tops[wave * 16 + lane] = top;
        }
        __syncthreads();
        uint32_t top = 0;
        for (int n = 0; n < p.kw; ++n) top = max(top, tops[n * 16 + i]);
        float scale, factor;
        int8_factors(top, &scale, &factor);
        if (threadIdx.x < 16) token_scale[threadIdx.x] = scale;
        if constexpr (ROWS) {
#pragma unroll
            for (int k = 0; k < 2 * KT; ++k) {
                const int token = k * STEP + own;
                *reinterpret_cast<uint2*>(stage + place<KT>(token, at / 2) + at % 2 * 8) = int8_codes8(v[k], __shfl(factor, token));
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (a wavefront's own)
            take(0, 0);
        } else {
#pragma unroll
            for (int k = 0; k < KT; ++k) x[0][k] = codes16(int8_codes8(v[2 * k], factor), int8_codes8(v[2 * k + 1], factor));
        }
    } else {
        request(0);
        if (NB > 1 || chunk_tiles < p.nkt) request(1);
        load(0, sg, ks * KT);
        load(1, sg + p.sw, ks * KT);
        for (int n = threadIdx.x; n < strips * NB * BLOCK; n += blockDim.x) smem[n] = 0;
        __syncthreads();
    }
    for (int c0 = 0, n = 0; c0 < p.nkt; c0 += chunk_tiles, n += NB) {
        const int k0 = c0 + ks * KT;
        if constexpr (!make) {
            // The pieces of a chunk, and requests for those two further on (LAST: none of the next chunk's).  Behind piece u there are requested for sure the piece after it, and,
            // for the first two, the weights of two strips.
            auto pieces = [&](auto last) {
                constexpr bool LAST = decltype(last)::value;
#pragma unroll
                for (int u = 0; u < NB; ++u) {
                    if (u < 2 && !(LAST && u + 1 == NB)) wait_vmcnt<3 * KT>();
                    else if (u < 2) wait_vmcnt<2 * KT>();
                    else if (!(LAST && u + 1 == NB)) wait_vmcnt<KT>();
                    else wait_vmcnt<0>();
                    take(u, NB == 1 ? n & 1 : u & 1);
                    if (LAST && u + 2 >= NB) continue;
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the piece is read: another may come in its place
                    request(n + u + 2);
                }
            };
            if (c0 + chunk_tiles < p.nkt) pieces(std::false_type());
            else pieces(std::true_type());
        }
        auto strip = [&](int set, int at, int next, int next_k0) {
            i32x4 acc[NB] = {};
#pragma unroll
            for (int k = 0; k < KT; ++k)
#pragma unroll
                for (int b = 0; b < NB; ++b) acc[b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[set][k], x[b][k], acc[b], 0, 0, 0);
            load(set, next, next_k0);
            if (at < strips) {
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int v = 0; v < 4; ++v) atomicAdd(&smem[(at * NB + b) * BLOCK + (4 * g + v) * BLOCK_PITCH + i], acc[b][v]);
            }
        };
        // (wavefronts without a strip go through it once too: the counts above)
        int at = sg;
        do {
            const bool last = at + 2 * p.sw >= strips;
            const int next = last ? sg : at + 2 * p.sw, next_k0 = last ? k0 + chunk_tiles : k0;
            strip(0, at, next, next_k0);
            strip(1, at + p.sw, next + p.sw, next_k0);
            at += 2 * p.sw;
        } while (at < strips);
    }
    if constexpr (!make) wait_vmcnt<0>();                            // (nothing may come to LDS after the end)
    __syncthreads();
    // lanes along the rows of a token (token-major y, and single tokens), else along the tokens of a row
    const int rows = (int)min((long long)strips * 16, p.M - (long long)strip0 * 16), along_rows = p.token_major || B == 1;
    const int inner = along_rows ? rows : B, total = rows * B;
    for (int n = threadIdx.x; n < total; n += blockDim.x) {
        const int o = n / inner, e = n - o * inner, row = along_rows ? e : o, token = along_rows ? o : e;
        const long long m = (long long)strip0 * 16 + row, t = token0 + token;
        const int sum = smem[((row >> 4) * NB + (token >> 4)) * BLOCK + (row & 15) * BLOCK_PITCH + (token & 15)];
        const float f = int8_result(sum, p.t[m], make ? token_scale[token] : p.s[t], p.bias ? p.bias[m] : 0.f);
        tsvd_store_y(p.y, p.token_major ? (size_t)t * p.ldy + m : (size_t)m * p.ldy + t, f, p.out_bf16);
    }
}

constexpr int MAX_BLOCKS = 48;      // 60 KiB of sums beside 64 KiB of codes

// How a launch is laid out: strips of a workgroup (all workgroups at once on the compute units where their sums allow it), wavefronts and tiles of each.
struct stream_plan {
    int strips_wg, kw, sw, kt, nb;
};
stream_plan plan_of(long long strips, int nkt, long long B, int cus, int most) {
    stream_plan s;
    s.nb = B <= 16 ? 1 : B <= 32 ? 2 : 4;
    const long long groups = (B + 16 * s.nb - 1) / (16 * s.nb);
    s.strips_wg = (int)std::max<long long>(1, std::min<long long>((strips * groups + cus - 1) / cus, MAX_BLOCKS / s.nb));
    s.kt = most;
    s.kw = 1;
    while (s.kw < 16 && s.kw * s.kt < nkt) s.kw *= 2;
    s.sw = 1;
    while (s.sw * 2 * s.kw <= 16 && s.sw * 2 <= s.strips_wg) s.sw *= 2;
    // wavefronts that have no strip of their own split the contraction further
    while (s.kt > 1 && s.kw * s.sw * 2 <= 16) s.kw *= 2, s.kt /= 2;
    while (s.kt > 1 && s.kw * (s.kt / 2) >= nkt) s.kt /= 2;
    return s;
}

template <int KT, int NB, typename MAKE, bool ROWS>
hipError_t launch(const stream_args& a, int grid, hipStream_t stream) {
    const size_t lds = (size_t)a.strips_wg * NB * BLOCK * 4 + (size_t)a.kw * a.sw * wave_bytes<KT, MAKE, ROWS>();
    hipLaunchKernelGGL((int8_stream_kernel<KT, NB, MAKE, ROWS>), dim3(grid), dim3(64 * a.kw * a.sw), lds, stream, a);
    return hipGetLastError();
}
template <int KT, int NB, typename MAKE>
hipError_t allow() {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(int8_stream_kernel<KT, NB, MAKE, true>), hipFuncAttributeMaxDynamicSharedMemorySize,
                               MAX_BLOCKS * BLOCK * 4 + 16 * wave_bytes<KT, MAKE, true>());
}
template <int NB>
hipError_t launch_codes(int kt, const stream_args& a, int grid, hipStream_t stream) {
    return kt == 1 ? launch<1, NB, void, true>(a, grid, stream) : launch<2, NB, void, true>(a, grid, stream);
}
template <typename X, bool ROWS>
hipError_t launch_make(int kt, const stream_args& a, int grid, hipStream_t stream) {
    if (kt == 1) return launch<1, 1, X, ROWS>(a, grid, stream);
    if (kt == 2) return launch<2, 1, X, ROWS>(a, grid, stream);
    return launch<4, 1, X, ROWS>(a, grid, stream);
}
stream_args args_of(const tsvd_int8_problem& p, const stream_plan& s) {
    const tsvd_int8_handle& h = *p.h;
    stream_args a = {};
    a.tiles = h.tiles(), a.nkt = h.nkt, a.strips = (int)h.strips, a.N = (int)h.N, a.t = h.scales(), a.M = h.M;
    a.s = p.scales, a.B = p.B, a.bias = p.bias, a.y = p.y, a.ldy = p.ldy, a.token_major = p.token_major, a.out_bf16 = p.out_bf16;
    a.strips_wg = s.strips_wg, a.strip_groups = (a.strips + s.strips_wg - 1) / s.strips_wg, a.kw = s.kw, a.sw = s.sw;
    while (1 << a.kw_log2 < s.kw) ++a.kw_log2;
    return a;
}

constexpr int CODES_TILES = 2;      // (four: 9216 features, 2048 rows 7.8 us, with two 6.5; 16384 rows of 4096 the same)
constexpr int MAKE_TILES = 4;       // tiles whose activations, codes and next weights fit the 128 registers of a lane

}  // namespace

hipError_t tsvd_int8_stream_init() {
    for (hipError_t e : {allow<1, 1, void>(), allow<2, 1, void>(), allow<1, 2, void>(), allow<2, 2, void>(), allow<1, 4, void>(), allow<2, 4, void>(), allow<1, 1, float>(),
                         allow<2, 1, float>(), allow<4, 1, float>(), allow<1, 1, uint16_t>(), allow<2, 1, uint16_t>(), allow<4, 1, uint16_t>()})
        if (e != hipSuccess) return e;
    return hipSuccess;
}

// Up to 64 tokens; and more, 64 a workgroup, where tiles of rows and tokens would leave most compute units idle over a long contraction: up to two strips for each compute unit.
// 46 rows of 14336 features, 256 tokens 13.8 us (tiles 23.3), 2048 rows of 4096 8.2 (9.1); of 640 features 5.4 (3.8), four strips each, 4096 rows of 4096, 11.8 (10.0).
bool tsvd_int8_stream_serves(const tsvd_int8_handle& h, long long B) {
    if (B <= 64) return true;
    const long long strips = (h.strips * ((B + 63) / 64) + h.cu_count - 1) / h.cu_count;
    return strips <= 2 && h.nkt / 2 >= 10 * strips && tsvd_tune("TSVD_INT8_TILE", 0) == 0;
}

hipError_t tsvd_int8_stream(const tsvd_int8_problem& p, hipStream_t stream) {
    const stream_plan s = plan_of(p.h->strips, p.h->nkt, p.B, p.h->cu_count, CODES_TILES);
    stream_args a = args_of(p, s);
    a.q = reinterpret_cast<const uint8_t*>(p.codes), a.ldq = p.ldq;
    const int grid = (int)(a.strip_groups * ((p.B + 16 * s.nb - 1) / (16 * s.nb)));
    return s.nb == 1 ? launch_codes<1>(s.kt, a, grid, stream) : s.nb == 2 ? launch_codes<2>(s.kt, a, grid, stream) : launch_codes<4>(s.kt, a, grid, stream);
}

// Whether the codes of B tokens are made in the launch of the product: where its wavefronts hold the contraction (4096 features, 16 wavefronts of 4 tiles of 64).  Against a launch
// of their own, 16 tokens: 4096 rows of 2048 features, token-major bf16 4.9 us and 6.6, feature-major 5.7 and 11.5; 16384 rows of 4096 13.0 and 14.7, 13.2 and 20.1; 4096 rows of
// 4096 7.7 and 7.8 (fp32 8.4 and 7.8, the one that loses), one token 6.9 and 7.2.
bool tsvd_int8_stream_makes(const tsvd_int8_handle& h, long long B) { return B <= 16 && h.nkt <= 16 * MAKE_TILES; }

hipError_t tsvd_int8_stream_from(const tsvd_int8_problem& p, const void* x, bool x_bf16, bool rows, long long ldx, hipStream_t stream) {
    const stream_plan s = plan_of(p.h->strips, p.h->nkt, p.B, p.h->cu_count, MAKE_TILES);
    stream_args a = args_of(p, s);
    a.q = static_cast<const uint8_t*>(x), a.ldq = ldx;
    const int grid = a.strip_groups;
    if (rows) return x_bf16 ? launch_make<uint16_t, true>(s.kt, a, grid, stream) : launch_make<float, true>(s.kt, a, grid, stream);
    return x_bf16 ? launch_make<uint16_t, false>(s.kt, a, grid, stream) : launch_make<float, false>(s.kt, a, grid, stream);
}
