// Layers in 8-bit integers (include/tsvd_int8.h): the codes of activations, the packed weights, the entry points.
//
// Codes: q = rne(x 127 / a), a the largest magnitude of the token.  Bound by memory: x once, a byte for each value back; five
// operations a value (unpacking, the magnitude's two, one fma that multiplies and rounds, its share of the byte permutes).
// Measured, bf16: 2048 tokens of 9216 features 16 us token-major (3.5 TB/s), 21 us feature-major in slices; 12544 of 512 feature-major, held in registers, 8.3 us; 256 of 4096 4.8 us.
#include "tsvd_int8.h"

#include <algorithm>
#include <new>
#include <type_traits>

#include "../../include/tsvd_tuning.h"
#include "tsvd_scratch.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

size_t round256(size_t v) { return (v + 255) & ~(size_t)255; }
long long round_up(long long v, long long m) { return (v + m - 1) / m * m; }

// Workgroups go round the XCDs: each XCD gets a run of the numbers, so that neighbours, which share lines of x, meet in one L2.
__device__ __forceinline__ unsigned xcd_run() {
    const unsigned each = gridDim.x >> 3, more = gridDim.x & 7, xcd = blockIdx.x & 7;
    return xcd * each + min(xcd, more) + (blockIdx.x >> 3);
}

// The largest over T threads: some lanes of a wavefront, or a workgroup's wavefronts.
template <int T>
__device__ __forceinline__ uint32_t group_top(uint32_t top, uint32_t* lds) {
    if constexpr (T <= 64) {
        return int8_lanes_top<T>(top);
    } else {
        const int wave = threadIdx.x >> 6;
        top = int8_lanes_top<64>(top);
        if ((threadIdx.x & 63) == 0) lds[wave] = top;
        __syncthreads();
        top = 0;
#pragma unroll
        for (int w = 0; w < T / 64; ++w) top = max(top, lds[w]);
        __syncthreads();
        return top;
    }
}

// Token-major x.  T threads for a token (T < 256: several tokens a workgroup), NV vectors of eight values each, which stay in registers between the largest magnitude
// and the codes; NV = 0: a loop, x read twice (the second time from the caches).
template <typename X, int T, int NV>
__global__ void __launch_bounds__(T < 256 ? 256 : T)
int8_quantize_rows_kernel(const X* __restrict__ x, long long ldx, long long B, int N, uint8_t* __restrict__ q, long long ldq, float* __restrict__ s) {
    __shared__ uint32_t lds[T < 64 ? 1 : T / 64];
    constexpr int TOKENS = T < 256 ? 256 / T : 1;
    const int t = threadIdx.x % T, nvec = (N + 7) / 8;
    for (long long b = (long long)blockIdx.x * TOKENS + threadIdx.x / T; b < B; b += (long long)gridDim.x * TOKENS) {
        const X* row = x + b * ldx;
        uint8_t* out = q + b * ldq;
        uint32_t top = 0;
        float scale, factor;
        if constexpr (NV > 0) {
            int8_eight<X> r[NV];
#pragma unroll
            for (int k = 0; k < NV; ++k) r[k] = int8_load8(row, (t + k * T) * 8, N);
#pragma unroll
            for (int k = 0; k < NV; ++k) top = int8_top8(r[k], top);
            int8_factors(group_top<T>(top, lds), &scale, &factor);
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (t + k * T < nvec) *reinterpret_cast<uint2*>(out + (size_t)(t + k * T) * 8) = int8_codes8(r[k], factor);
        } else {
            for (int v = t; v < nvec; v += T) top = int8_top8(int8_load8(row, v * 8, N), top);
            int8_factors(group_top<T>(top, lds), &scale, &factor);
            for (int v = t; v < nvec; v += T) *reinterpret_cast<uint2*>(out + (size_t)v * 8) = int8_codes8(int8_load8(row, v * 8, N), factor);
        }
        if (t == 0) s[b] = scale;
    }
}

// Feature-major x [N][B]: a workgroup of T threads takes 8 TV tokens.  A thread loads eight tokens of a row of x at a time, four rows in a pass; the largest magnitudes of the tokens meet in
// LDS; then the codes of a pass go through LDS, so that a token's bytes leave side by side.  PASSES: x stays in registers in between (N <= PASSES 4 T / TV); 0: it is read again (from the
// caches).
template <typename X, int T, int TV, int PASSES>
__global__ void __launch_bounds__(T, T == 1024 && PASSES <= 2 && TV > 1 && sizeof(X) == 2 ? 8 : 1)
int8_quantize_columns_kernel(const X* __restrict__ x, long long ldx, long long B, int N, uint8_t* __restrict__ q, long long ldq, float* __restrict__ s) {
    constexpr int ROWS = T / TV, STEP = 4 * ROWS, PITCH = STEP + 16, TOKENS = 8 * TV;        // rows of threads; features a pass
    __shared__ uint32_t tops[TOKENS];
    __shared__ __align__(16) uint8_t tile[TOKENS * PITCH];
    const int v = threadIdx.x % TV, r = threadIdx.x / TV;
    const long long b0 = (long long)xcd_run() * TOKENS;
    const int tokens = (int)min((long long)TOKENS, B - b0);
    if (threadIdx.x < TOKENS) tops[threadIdx.x] = 0;
    const X* mine = x + b0;
    const int at = min(8 * v, tokens - 1);                       // (beyond the last token: that one's again, not stored)
    auto load = [&](int8_eight<X> (&u)[4], int n) {
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = int8_load8(mine + (size_t)min(n + j, N - 1) * ldx, at, tokens);
    };
    uint32_t top[8] = {};
    auto raise = [&](const int8_eight<X> (&u)[4]) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < 8; ++k) top[k] = max(top[k], __float_as_uint(u[j].get(k)) & 0x7FFFFFFFu);
    };
    int8_eight<X> held[PASSES ? PASSES : 1][4];
    if constexpr (PASSES > 0) {
#pragma unroll
        for (int i = 0; i < PASSES; ++i)
            if (i * STEP < N) load(held[i], i * STEP + 4 * r);
#pragma unroll
        for (int i = 0; i < PASSES; ++i)
            if (i * STEP < N) raise(held[i]);
    } else {
        for (int n = 4 * r; n < N; n += STEP) {
            load(held[0], n);
            raise(held[0]);
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        // (first among the lanes that hold the same tokens)
        for (int m = TV; m < 64; m *= 2) top[k] = max(top[k], (uint32_t)__shfl_xor((int)top[k], m));
        if ((threadIdx.x & 63) < TV) atomicMax(&tops[8 * v + k], top[k]);
    }
    __syncthreads();
    float factor[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        float scale;
        int8_factors(tops[8 * v + k], &scale, &factor[k]);
        if (r == 0 && 8 * v + k < tokens) s[b0 + 8 * v + k] = scale;
    }
    auto pass = [&](const int8_eight<X> (&u)[4], int n0) {
        uint32_t c[4][8];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < 8; ++k) c[j][k] = int8_code(u[j].get(k), factor[k]);
#pragma unroll
        for (int k = 0; k < 8; ++k) *reinterpret_cast<uint32_t*>(&tile[(8 * v + k) * PITCH + 4 * r]) = int8_pack4(c[0][k], c[1][k], c[2][k], c[3][k]);
        __syncthreads();
        const int pieces = min(STEP, (N - n0 + 15) / 16 * 16) / 16;
        for (int i = threadIdx.x; i < TOKENS * (STEP / 16); i += T) {
            const int b = i / (STEP / 16), piece = i % (STEP / 16);
            if (b < tokens && piece < pieces) *reinterpret_cast<u32x4*>(q + (b0 + b) * ldq + n0 + 16 * piece) = *reinterpret_cast<const u32x4*>(&tile[b * PITCH + 16 * piece]);
        }
        __syncthreads();
    };
    if constexpr (PASSES > 0) {
#pragma unroll
        for (int i = 0; i < PASSES; ++i)
            if (i * STEP < N) pass(held[i], i * STEP);
    } else {
        for (int n0 = 0; n0 < N; n0 += STEP) {
            load(held[0], n0 + 4 * r);
            pass(held[0], n0);
        }
    }
}

// Feature-major x that a workgroup does not hold, or of so few tokens that few workgroups would have it: two launches, the features cut into slices.  The first leaves the largest
// magnitudes of a slice's tokens, the second takes the largest over the slices and makes the slice's codes, as above.
template <typename X, int TV>
__global__ void __launch_bounds__(256)
int8_column_tops_kernel(const X* __restrict__ x, long long ldx, long long B, int N, int rows, unsigned slices, uint32_t* __restrict__ tops_of) {
    constexpr int ROWS = 256 / TV, TOKENS = 8 * TV;
    __shared__ uint32_t tops[TOKENS];
    const int v = threadIdx.x % TV, r = threadIdx.x / TV;
    const unsigned blocks = gridDim.x / slices, at = xcd_run(), slice = at / blocks, block = at - slice * blocks;
    const long long b0 = (long long)block * TOKENS;
    const int tokens = (int)min((long long)TOKENS, B - b0), first = (int)slice * rows, end = min(first + rows, N);
    if (threadIdx.x < TOKENS) tops[threadIdx.x] = 0;
    const X* mine = x + b0;
    uint32_t top[8] = {};
    for (int n = first + r; n < end; n += 8 * ROWS) {
        int8_eight<X> u[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) u[j] = int8_load8(mine + (size_t)min(n + j * ROWS, end - 1) * ldx, min(8 * v, tokens - 1), tokens);
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int k = 0; k < 8; ++k) top[k] = max(top[k], __float_as_uint(u[j].get(k)) & 0x7FFFFFFFu);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        for (int m = TV; m < 64; m *= 2) top[k] = max(top[k], (uint32_t)__shfl_xor((int)top[k], m));
        if ((threadIdx.x & 63) < TV) atomicMax(&tops[8 * v + k], top[k]);
    }
    __syncthreads();
    if ((int)threadIdx.x < tokens) tops_of[(size_t)slice * B + b0 + threadIdx.x] = tops[threadIdx.x];
}
template <typename X, int TV>
__global__ void __launch_bounds__(256)
int8_column_codes_kernel(const X* __restrict__ x, long long ldx, long long B, int N, int rows, unsigned slices, const uint32_t* __restrict__ tops_of, uint8_t* __restrict__ q,
                         long long ldq, float* __restrict__ s) {
    constexpr int ROWS = 256 / TV, STEP = 4 * ROWS, PITCH = STEP + 16, TOKENS = 8 * TV;
    __shared__ uint32_t tops[TOKENS];
    __shared__ __align__(16) uint8_t tile[TOKENS * PITCH];
    const int v = threadIdx.x % TV, r = threadIdx.x / TV;
    const unsigned blocks = gridDim.x / slices, at = xcd_run(), slice = at / blocks, block = at - slice * blocks;
    const long long b0 = (long long)block * TOKENS;
    const int tokens = (int)min((long long)TOKENS, B - b0), first = (int)slice * rows, end = min(first + rows, N);
    if (threadIdx.x < TOKENS) tops[threadIdx.x] = 0;
    const X* mine = x + b0;
    int8_eight<X> u[4];
    auto load = [&](int n) {
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = int8_load8(mine + (size_t)min(n + j, N - 1) * ldx, min(8 * v, tokens - 1), tokens);
    };
    load(first + 4 * r);
    __syncthreads();
    {
        const int b = threadIdx.x % TOKENS;
        uint32_t top = 0;
        for (unsigned i = threadIdx.x / TOKENS; i < slices; i += 256 / TOKENS) top = max(top, tops_of[(size_t)i * B + min(b0 + b, B - 1)]);
        atomicMax(&tops[b], top);
    }
    __syncthreads();
    float factor[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        float scale;
        int8_factors(tops[8 * v + k], &scale, &factor[k]);
        if (slice == 0 && r == 0 && 8 * v + k < tokens) s[b0 + 8 * v + k] = scale;
    }
    for (int n0 = first; n0 < end; n0 += STEP) {
        uint32_t c[4][8];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < 8; ++k) c[j][k] = int8_code(u[j].get(k), factor[k]);
        if (n0 + STEP < end) load(n0 + STEP + 4 * r);
#pragma unroll
        for (int k = 0; k < 8; ++k) *reinterpret_cast<uint32_t*>(&tile[(8 * v + k) * PITCH + 4 * r]) = int8_pack4(c[0][k], c[1][k], c[2][k], c[3][k]);
        __syncthreads();
        const int pieces = min(STEP, (end - n0 + 15) / 16 * 16) / 16;
        for (int i = threadIdx.x; i < TOKENS * (STEP / 16); i += 256) {
            const int b = i / (STEP / 16), piece = i % (STEP / 16);
            if (b < tokens && piece < pieces) *reinterpret_cast<u32x4*>(q + (b0 + b) * ldq + n0 + 16 * piece) = *reinterpret_cast<const u32x4*>(&tile[b * PITCH + 16 * piece]);
        }
        __syncthreads();
    }
}

// Codes [M][ldw] -> tiles (tsvd_int8.h): a thread makes the 16 bytes of one lane.
__global__ void __launch_bounds__(256)
int8_pack_kernel(const uint8_t* __restrict__ w, long long ldw, long long M, int N, int nkt, long long pieces, uint8_t* __restrict__ tiles) {
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < pieces; i += (long long)gridDim.x * 256) {
        const long long tile = i >> 6, strip = tile / nkt;
        const int l = (int)i & 63, k = (int)(tile - strip * nkt) * 64 + (l >> 4) * 16;
        const long long row = strip * 16 + (l & 15);
        uint32_t d[4] = {};
        if (row < M) {
            const uint8_t* src = w + row * ldw;
            if (k + 16 <= N) {
                typedef u32x4 u32x4_at __attribute__((aligned(1)));
                const u32x4 v = *reinterpret_cast<const u32x4_at*>(src + k);
                d[0] = v[0], d[1] = v[1], d[2] = v[2], d[3] = v[3];
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (k + e < N) d[e >> 2] |= (uint32_t)src[k + e] << (8 * (e & 3));
            }
        }
        *reinterpret_cast<u32x4*>(tiles + i * 16) = u32x4{d[0], d[1], d[2], d[3]};
    }
}
__global__ void __launch_bounds__(256)
int8_pack_scales_kernel(const float* __restrict__ t, long long M, long long rows, float* __restrict__ out) {
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < rows; i += (long long)gridDim.x * 256) out[i] = i < M ? t[i] : 0.f;
}

unsigned grid_of(long long blocks) { return (unsigned)std::min<long long>(blocks, 1 << 20); }

// How feature-major x is cut: vectors of eight tokens side by side, slices of the features (1: one launch), rows of a slice.
struct columns_plan {
    int tv, slices, rows;
};
columns_plan plan_columns(long long B, int N) {
    columns_plan c;
    c.tv = B >= 512 ? 8 : B > 16 ? 2 : 1;
    const long long blocks = (B + 8 * c.tv - 1) / (8 * c.tv), step = 1024 / c.tv;
    // one launch where a workgroup's registers hold all features, or where there is next to nothing to do; slices elsewhere, about 512 workgroups of them (2048 tokens of 9216 features
    // 21 us, 38 in one launch that reads x twice; 64 of 16384 8 us and 28), and for few tokens whose rows do not stand on 16 bytes (4096 features: 197 tokens 11.5 us, in one launch 14.5;
    // 256 tokens 7.7 and 7.6, 3000 tokens 21.2 and 16.9)
    const bool held = N <= 2048 || (N <= 4096 && (B <= 64 || B >= 1024 || B % 8 == 0));
    const long long slices = std::min<long long>((N + step - 1) / step, std::max<long long>(1, (512 + blocks - 1) / blocks));
    c.slices = held || slices < 2 || B * N <= 8192 ? 1 : (int)slices;
    c.rows = (int)(((N + c.slices - 1) / c.slices + step - 1) / step * step);
    c.slices = (N + c.rows - 1) / c.rows;
    return c;
}

// One launch for feature-major x: threads of a workgroup, vectors of eight tokens side by side, passes held in registers (0: a loop), and the features that those hold.
template <int T_, int TV_, int PASSES_>
struct columns_form {
    static constexpr int T = T_, TV = TV_, PASSES = PASSES_, FEATURES = PASSES * 4 * T / TV;
};
// 64 bytes of a row (bf16) for each workgroup where that leaves one for most compute units, else fewer tokens (3000 tokens, 2048 features: 32 bytes 9.5 us, 16 bytes 10.9; 3000 of
// 4096, which only sixteen bytes' worth fits registers of: 16.9).  Beyond 4096 features nothing holds x: the loop (32768 tokens of 9216 features 324 us,
// 4.7 TB/s with both readings).
template <typename X, typename F>
auto with_columns_form(long long B, int N, F&& f) {
    constexpr int WIDEST = sizeof(X) == 2 ? 4 : 0;               // (fp32 values of four passes are 128 registers of a lane, all that 1024 lanes have)
    if (B >= 4096) {
        if (N <= 512) return f(columns_form<256, 4, 2>());
        if (N <= 2048) return f(columns_form<1024, 4, 2>());
        if (N <= 4096) return f(columns_form<1024, 4, WIDEST>());
        return f(columns_form<1024, 4, 0>());
    }
    if (B >= 1024 && N <= 1024) return f(columns_form<256, 2, 2>());
    if (B >= 1024 && N <= 2048) return f(columns_form<1024, 2, 2>());
    if (N <= 512) return f(columns_form<128, 1, 1>());
    if (N <= 1024) return f(columns_form<256, 1, 1>());
    if (N <= 2048) return f(columns_form<512, 1, 1>());
    if (N <= 4096) return f(columns_form<512, 1, 2>());
    return f(columns_form<1024, 1, 0>());
}

template <typename X>
hipError_t quantize(const X* x, bool token_major, long long B, int N, long long ldx, uint8_t* q, long long ldq, float* s, uint32_t* tops, hipStream_t stream) {
    if (token_major) {
        auto rows = [&](auto kernel, int threads, int tokens) {      // tokens: of a workgroup
            hipLaunchKernelGGL(kernel, dim3(grid_of((B + tokens - 1) / tokens)), dim3(threads), 0, stream, x, ldx, B, N, q, ldq, s);
        };
        if (N <= 64) rows(int8_quantize_rows_kernel<X, 8, 1>, 256, 32);
        else if (N <= 128) rows(int8_quantize_rows_kernel<X, 16, 1>, 256, 16);
        else if (N <= 256) rows(int8_quantize_rows_kernel<X, 32, 1>, 256, 8);
        else if (N <= 512) rows(int8_quantize_rows_kernel<X, 64, 1>, 256, 4);
        else if (N <= 1024) rows(int8_quantize_rows_kernel<X, 64, 2>, 256, 4);
        else if (N <= 2048) rows(int8_quantize_rows_kernel<X, 64, 4>, 256, 4);
        else if (N <= 4096) rows(int8_quantize_rows_kernel<X, 256, 2>, 256, 1);
        else if (N <= 8192) rows(int8_quantize_rows_kernel<X, 256, 4>, 256, 1);
        else if (N <= 16384) rows(int8_quantize_rows_kernel<X, 256, 8>, 256, 1);
        else rows(int8_quantize_rows_kernel<X, 1024, 0>, 1024, 1);
    } else {
        const columns_plan c = plan_columns(B, N);
        if (c.slices > 1) {
            auto sliced = [&](auto tv) {
                constexpr int TV = decltype(tv)::value;
                const dim3 grid((unsigned)((B + 8 * TV - 1) / (8 * TV) * c.slices));
                hipLaunchKernelGGL((int8_column_tops_kernel<X, TV>), grid, dim3(256), 0, stream, x, ldx, B, N, c.rows, (unsigned)c.slices, tops);
                const hipError_t e = hipGetLastError();
                if (e != hipSuccess) return e;
                hipLaunchKernelGGL((int8_column_codes_kernel<X, TV>), grid, dim3(256), 0, stream, x, ldx, B, N, c.rows, (unsigned)c.slices, tops, q, ldq, s);
                return hipGetLastError();
            };
            return c.tv == 8 ? sliced(std::integral_constant<int, 8>()) : c.tv == 2 ? sliced(std::integral_constant<int, 2>()) : sliced(std::integral_constant<int, 1>());
        }
        return with_columns_form<X>(B, N, [&](auto form) {
            typedef decltype(form) F;
            if (F::PASSES && N > F::FEATURES) return hipErrorInvalidValue;      // (a rule that is wrong: nothing is launched)
            hipLaunchKernelGGL((int8_quantize_columns_kernel<X, F::T, F::TV, F::PASSES>), dim3((unsigned)((B + 8 * F::TV - 1) / (8 * F::TV))), dim3(F::T), 0, stream, x, ldx, B, N, q, ldq, s);
            return hipGetLastError();
        });
    }
    return hipGetLastError();
}
hipError_t quantize(const void* x, tsvd_dtype x_dtype, bool token_major, long long B, int N, long long ldx, int8_t* codes, long long ldq, float* s, void* workspace, hipStream_t stream) {
    uint8_t* q = reinterpret_cast<uint8_t*>(codes);
    uint32_t* tops = static_cast<uint32_t*>(workspace);
    return x_dtype == TSVD_BF16 ? quantize(static_cast<const uint16_t*>(x), token_major, B, N, ldx, q, ldq, s, tops, stream)
                                : quantize(static_cast<const float*>(x), token_major, B, N, ldx, q, ldq, s, tops, stream);
}

bool bad_codes(const void* codes, int64_t ldq, int64_t N) { return !codes || (reinterpret_cast<uintptr_t>(codes) & 15u) || ldq < N || ldq % 16 != 0; }
bool bad_workspace(const void* ws, size_t bytes, size_t need) { return ws ? bytes < need || (reinterpret_cast<uintptr_t>(ws) & 255u) : need != 0 || bytes != 0; }
bool bad_dtype(int t) { return t != TSVD_F32 && t != TSVD_BF16; }
bool bad_layout(int l) { return l != TSVD_FEATURE_MAJOR && l != TSVD_TOKEN_MAJOR; }

// One token is a contiguous vector in either layout, whatever its stride means: as one row.
bool one_row(tsvd_layout layout, int64_t B, int64_t ldx) { return layout == TSVD_TOKEN_MAJOR || (B == 1 && ldx == 1); }

// The weights are where the launch will be.
bool on_its_device(const tsvd_int8_handle* h) {
    int device = -1;
    return hipGetDevice(&device) == hipSuccess && device == h->device;
}

size_t codes_bytes(const tsvd_int8_handle* h, int64_t B) { return round256((size_t)B * tsvd_int8_row_bytes(h->N)); }

}  // namespace

extern "C" size_t tsvd_int8_row_bytes(int64_t N) { return N <= 0 || N > TSVD_INT8_MAX_N ? 0 : (size_t)round_up(N, 128); }

extern "C" size_t tsvd_int8_quantize_workspace_bytes(int64_t B, int64_t N, tsvd_layout x_layout) {
    if (x_layout != TSVD_FEATURE_MAJOR || B < 1 || N < 1 || B > TSVD_INT8_MAX_B || N > TSVD_INT8_MAX_N) return 0;
    const columns_plan c = plan_columns(B, (int)N);
    return c.slices > 1 ? round256((size_t)c.slices * B * 4) : 0;
}

extern "C" int tsvd_tuning_int8_columns(int64_t B, int64_t N, tsvd_dtype x_dtype) {
    if (B < 1 || N < 1 || B > TSVD_INT8_MAX_B || N > TSVD_INT8_MAX_N || bad_dtype(x_dtype) || plan_columns(B, (int)N).slices > 1) return -1;
    auto features = [](auto form) { return decltype(form)::FEATURES; };
    return x_dtype == TSVD_BF16 ? with_columns_form<uint16_t>(B, (int)N, features) : with_columns_form<float>(B, (int)N, features);
}

extern "C" tsvd_status tsvd_int8_quantize(const void* x_dev, tsvd_dtype x_dtype, tsvd_layout x_layout, int64_t B, int64_t N, int64_t ldx,
                                          int8_t* codes_dev, int64_t ldq, float* scales_dev, void* workspace, size_t workspace_bytes, void* stream) {
    if (!x_dev || !scales_dev || B < 1 || N < 1 || bad_dtype(x_dtype) || bad_layout(x_layout)) return TSVD_EINVAL;
    if (ldx < (x_layout == TSVD_TOKEN_MAJOR ? N : B) || bad_codes(codes_dev, ldq, N)) return TSVD_EINVAL;
    if (N > TSVD_INT8_MAX_N || B > TSVD_INT8_MAX_B) return TSVD_EUNSUPPORTED;
    if (bad_workspace(workspace, workspace_bytes, tsvd_int8_quantize_workspace_bytes(B, N, x_layout))) return TSVD_EINVAL;
    const bool rows = one_row(x_layout, B, ldx);
    return quantize(x_dev, x_dtype, rows, B, (int)N, x_layout == TSVD_TOKEN_MAJOR ? ldx : rows ? N : ldx, codes_dev, ldq, scales_dev, workspace,
                    static_cast<hipStream_t>(stream)) == hipSuccess ? TSVD_OK : TSVD_EDEVICE;
}

extern "C" size_t tsvd_int8_packed_bytes(int64_t M, int64_t N) {
    if (M < 1 || N < 1 || N > TSVD_INT8_MAX_N || M > TSVD_INT8_MAX_M) return 0;
    const size_t strips = (size_t)(M + 15) / 16;
    return round256(strips * 64) + strips * (size_t)(round_up(N, 128) / 64) * 1024;
}

extern "C" tsvd_status tsvd_int8_pack(const int8_t* w_dev, int64_t ldw, const float* t_dev, int64_t M, int64_t N, void* dev_buf, size_t dev_buf_bytes,
                                      void* stream, tsvd_int8_handle** out) {
    if (!w_dev || !t_dev || !out || M < 1 || N < 1 || ldw < N) return TSVD_EINVAL;
    if (N > TSVD_INT8_MAX_N || M > TSVD_INT8_MAX_M) return TSVD_EUNSUPPORTED;
    const size_t bytes = tsvd_int8_packed_bytes(M, N);
    if (dev_buf ? dev_buf_bytes < bytes || (reinterpret_cast<uintptr_t>(dev_buf) & 255u) : dev_buf_bytes != 0) return TSVD_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    int device = 0, cus = 0;
    if (hipStreamIsCapturing(s, &capture) != hipSuccess || capture != hipStreamCaptureStatusNone || hipGetDevice(&device) != hipSuccess ||
        hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess) {
        (void)hipGetLastError();
        return TSVD_EDEVICE;
    }
    if (tsvd_int8_gemm_init() != hipSuccess || tsvd_int8_stream_init() != hipSuccess) {
        (void)hipGetLastError();
        return TSVD_EDEVICE;
    }
    tsvd_int8_handle* h = new (std::nothrow) tsvd_int8_handle();
    if (!h) return TSVD_ENOMEM;
    h->device = device;
    h->cu_count = cus;
    h->M = M, h->N = N, h->strips = (M + 15) / 16;
    h->nkt = (int)(round_up(N, 128) / 64);
    h->blob = static_cast<uint8_t*>(dev_buf);
    if (!dev_buf) {
        void* p = nullptr;
        if (tsvd_device_malloc(&p, bytes) != hipSuccess) {
            (void)hipGetLastError();
            delete h;
            return TSVD_EDEVICE;
        }
        h->blob = static_cast<uint8_t*>(p);
        h->owns_blob = true;
    }
    const long long pieces = h->strips * h->nkt * 64;
    hipLaunchKernelGGL(int8_pack_scales_kernel, dim3(grid_of((h->strips * 16 + 255) / 256)), dim3(256), 0, s, t_dev, (long long)M, h->strips * 16, reinterpret_cast<float*>(h->blob));
    hipLaunchKernelGGL(int8_pack_kernel, dim3(grid_of((pieces + 255) / 256)), dim3(256), 0, s, reinterpret_cast<const uint8_t*>(w_dev), (long long)ldw, (long long)M, (int)N,
                       h->nkt, pieces, const_cast<uint8_t*>(h->tiles()));
    if (hipGetLastError() != hipSuccess || hipStreamSynchronize(s) != hipSuccess) {
        (void)hipGetLastError();
        tsvd_int8_free(h);
        return TSVD_EDEVICE;
    }
    *out = h;
    return TSVD_OK;
}

extern "C" tsvd_status tsvd_int8_info(const tsvd_int8_handle* h, int64_t* M, int64_t* N) {
    if (!h) return TSVD_EINVAL;
    if (M) *M = h->M;
    if (N) *N = h->N;
    return TSVD_OK;
}

extern "C" void tsvd_int8_free(tsvd_int8_handle* h) {
    if (!h) return;
    if (h->owns_blob && h->blob) (void)hipFree(h->blob);
    delete h;
}

extern "C" tsvd_status tsvd_int8_product(const tsvd_int8_handle* h, const int8_t* codes_dev, int64_t ldq, const float* scales_dev, int64_t B,
                                         const float* bias_dev, void* y_dev, tsvd_dtype y_dtype, tsvd_layout y_layout, int64_t ldy, void* stream) {
    if (!h || !scales_dev || !y_dev || B < 1 || bad_dtype(y_dtype) || bad_layout(y_layout)) return TSVD_EINVAL;
    if (bad_codes(codes_dev, ldq, h->N) || ldy < (y_layout == TSVD_TOKEN_MAJOR ? h->M : B)) return TSVD_EINVAL;
    if (B > TSVD_INT8_MAX_B || ldq > TSVD_INT8_MAX_PITCH) return TSVD_EUNSUPPORTED;
    if (!on_its_device(h)) return TSVD_EINVAL;
    const tsvd_int8_problem p = {h, codes_dev, ldq, scales_dev, B, bias_dev, y_dev, y_dtype == TSVD_BF16, y_layout == TSVD_TOKEN_MAJOR, ldy};
    const hipError_t e = tsvd_int8_stream_serves(*h, B) ? tsvd_int8_stream(p, static_cast<hipStream_t>(stream)) : tsvd_int8_gemm(p, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? TSVD_OK : e == hipErrorNotSupported ? TSVD_EUNSUPPORTED : TSVD_EDEVICE;
}

namespace {
// Whether a call makes the codes in the launch of the product, and where x is a contiguous vector.
bool made_in_launch(const tsvd_int8_handle* h, int64_t B) { return tsvd_int8_stream_serves(*h, B) && tsvd_int8_stream_makes(*h, B); }
}  // namespace

extern "C" size_t tsvd_int8_workspace_bytes(const tsvd_int8_handle* h, int64_t B, tsvd_dtype x_dtype, tsvd_layout x_layout) {
    if (!h || B < 1 || B > TSVD_INT8_MAX_B || bad_dtype(x_dtype) || bad_layout(x_layout)) return 0;
    if (made_in_launch(h, B)) return 0;
    return codes_bytes(h, B) + round256((size_t)B * 4) + tsvd_int8_quantize_workspace_bytes(B, h->N, x_layout);
}

extern "C" tsvd_status tsvd_int8_forward(const tsvd_int8_handle* h, const void* x_dev, tsvd_dtype x_dtype, tsvd_layout x_layout, int64_t B, int64_t ldx,
                                         const float* bias_dev, void* y_dev, tsvd_dtype y_dtype, tsvd_layout y_layout, int64_t ldy, void* workspace,
                                         size_t workspace_bytes, void* stream) {
    if (!h || !x_dev || !y_dev || B < 1 || bad_dtype(x_dtype) || bad_layout(x_layout) || bad_dtype(y_dtype) || bad_layout(y_layout)) return TSVD_EINVAL;
    if (ldx < (x_layout == TSVD_TOKEN_MAJOR ? h->N : B) || ldy < (y_layout == TSVD_TOKEN_MAJOR ? h->M : B)) return TSVD_EINVAL;
    if (B > TSVD_INT8_MAX_B) return TSVD_EUNSUPPORTED;
    if (bad_workspace(workspace, workspace_bytes, tsvd_int8_workspace_bytes(h, B, x_dtype, x_layout)) || !on_its_device(h)) return TSVD_EINVAL;
    if (made_in_launch(h, B)) {
        const tsvd_int8_problem p = {h, nullptr, 0, nullptr, B, bias_dev, y_dev, y_dtype == TSVD_BF16, y_layout == TSVD_TOKEN_MAJOR, ldy};
        return tsvd_int8_stream_from(p, x_dev, x_dtype == TSVD_BF16, one_row(x_layout, B, ldx), ldx, static_cast<hipStream_t>(stream)) == hipSuccess ? TSVD_OK : TSVD_EDEVICE;
    }
    int8_t* codes = static_cast<int8_t*>(workspace);
    uint8_t* behind = static_cast<uint8_t*>(workspace) + codes_bytes(h, B);
    float* scales = reinterpret_cast<float*>(behind);
    const int64_t ldq = (int64_t)tsvd_int8_row_bytes(h->N);
    const size_t more = tsvd_int8_quantize_workspace_bytes(B, h->N, x_layout);
    const tsvd_status st = tsvd_int8_quantize(x_dev, x_dtype, x_layout, B, h->N, ldx, codes, ldq, scales, more ? behind + round256((size_t)B * 4) : nullptr, more, stream);
    return st != TSVD_OK ? st : tsvd_int8_product(h, codes, ldq, scales, B, bias_dev, y_dev, y_dtype, y_layout, ldy, stream);
}
