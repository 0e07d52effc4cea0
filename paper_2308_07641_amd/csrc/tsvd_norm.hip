// Group norm with an activation, channels last (include/tsvd_norm.h).
//
// Bound by memory: x once for the statistics, once more for y where an image does not stay on the chip, y once.  Statistics: a workgroup holds a
// piece of one image and of whole groups in registers, takes the sum of each of its groups, then the squares of the deviations from the piece's own mean, so that
// nothing cancels; pieces are joined by n (mean - common mean)^2.  Every sum has a fixed order.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "../../include/tsvd_norm.h"
#include "tsvd_epilogue.h"
#include "tsvd_int8.h"

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

struct norm_args {
    const void* x;
    long long ldx;
    long long images, P;
    int C, G, cg;                 // channels, groups, channels of a group
    const float *gamma, *beta;
    float eps;
    int act;
    void* y;
    long long ldy;
    int out_bf16;
    float* scales;                // int8 output
    float4* parts;                // [images][G][chunks]: mean, sum of squared deviations, values
    float2* stats;                // [images][G]: mean, 1 / sqrt(v + eps)
    long long chunks;             // pieces of an image along its positions (one group a workgroup: along its vectors)
    int gpb, nblk;                // groups of a workgroup, workgroups side by side along the channels
    int rows;                     // positions of a piece, where a workgroup holds several groups
};

__device__ __forceinline__ float norm_act(float h, int act) {
    if (act == TSVD_ACT_RELU) return h > 0.f ? h : h != h ? h : 0.f;
    if (act == TSVD_ACT_SILU) return h / (1.f + __expf(-h));
    if (act == TSVD_ACT_GELU) return 0.5f * h * (1.f + erff(h * 0.70710678118654752f));
    return h;
}

// ---- statistics ------------------------------------------------------------------------------------
// T threads, NV vectors of eight channels each.  Several groups in a workgroup: a thread keeps one vector of the block's channels and takes every T / (vectors)-th position;
// ONE group: vectors of the piece in order, whatever position they belong to.
template <typename X, int T, int NV, bool ONE>
__global__ void __launch_bounds__(T)
norm_stats_kernel(norm_args p) {
    __shared__ float part[ONE ? 64 : T * 9];
    __shared__ float channel[ONE ? 1 : T * 8];
    __shared__ float mean_of[ONE ? 1 : T * 8];
    const int tid = threadIdx.x;
    const long long items = p.images * p.nblk * p.chunks;
    for (long long item = blockIdx.x; item < items; item += gridDim.x) {
        const long long chunk = item % p.chunks, rest = item / p.chunks, image = rest / p.nblk;
        const int blk = (int)(rest % p.nblk);
        const X* x = static_cast<const X*>(p.x) + image * p.P * p.ldx;
        int8_eight<X> v[NV];
        if constexpr (ONE) {
            const int c0 = blk * p.cg, cvec = (p.cg + 7) / 8;
            const long long first = chunk * (T * NV) + tid, total = p.P * cvec;
            long long pos = first / cvec;
            int at = (int)(first - pos * cvec);
            const int step_p = T / cvec, step_v = T % cvec;
            int n[NV];
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                n[k] = pos < p.P ? min(8, p.cg - 8 * at) : 0;
                v[k].zero();
                if (n[k]) v[k] = int8_load8(x + pos * p.ldx + c0, 8 * at, p.cg);
                at += step_v, pos += step_p;
                if (at >= cvec) at -= cvec, ++pos;
            }
            (void)total;
            float sum = 0.f;
            int count = 0;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                count += n[k];
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += v[k].get(e);          // (zeros behind the end)
            }
            auto reduce = [&](float a) {
                for (int m = 32; m > 0; m >>= 1) a += __shfl_xor(a, m);
                __syncthreads();
                if ((tid & 63) == 0) part[tid >> 6] = a;
                __syncthreads();
                a = 0.f;
#pragma unroll
                for (int w = 0; w < T / 64; ++w) a += part[w];
                return a;
            };
            const float cnt = reduce((float)count), mean = reduce(sum) / cnt;
            float m2 = 0.f;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float d = e < n[k] ? v[k].get(e) - mean : 0.f;
                    m2 = fmaf(d, d, m2);
                }
            m2 = reduce(m2);
            if (tid == 0) p.parts[(image * p.G + blk) * p.chunks + chunk] = float4{mean, m2, cnt, 0.f};
        } else {
            const int g0 = blk * p.gpb, ng = min(p.gpb, p.G - g0), c0 = g0 * p.cg, nch = ng * p.cg, cvec = (nch + 7) / 8;
            const int R = T / cvec, at = tid % cvec, r = tid / cvec;
            const long long p0 = chunk * p.rows;
            const int rows = (int)min((long long)p.rows, p.P - p0);
            const bool active = r < R;
            float sum[8] = {};
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                v[k].zero();
                const int pos = r + k * R;
                if (active && pos < rows) v[k] = int8_load8(x + (p0 + pos) * p.ldx + c0, 8 * at, nch);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += v[k].get(e);
            }
            // the sums of the threads of a channel, then of the channels of a group (L lanes for each)
            int L = 64;
            while (L * ng > T && L > 1) L >>= 1;
            auto by_group = [&](const float (&a)[8], float* out) {
                __syncthreads();
                if (active)
#pragma unroll
                    for (int e = 0; e < 8; ++e) part[tid * 9 + e] = a[e];
                __syncthreads();
                for (int c = tid; c < nch; c += T) {
                    float s = 0.f;
                    for (int j = 0; j < R; ++j) s += part[(j * cvec + (c >> 3)) * 9 + (c & 7)];
                    channel[c] = s;
                }
                __syncthreads();
                for (int g = tid / L; g < ng; g += T / L) {
                    float s = 0.f;
                    for (int c = tid % L; c < p.cg; c += L) s += channel[g * p.cg + c];
                    for (int m = L / 2; m > 0; m >>= 1) s += __shfl_xor(s, m);
                    if (tid % L == 0) out[g] = s;
                }
                __syncthreads();
            };
            const float cnt = (float)rows * (float)p.cg;
            by_group(sum, mean_of);
            float mean[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) mean[e] = mean_of[min(8 * at + e, nch - 1) / p.cg] / cnt;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = 0.f;
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (r + k * R < rows)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float d = v[k].get(e) - mean[e];
                        sum[e] = fmaf(d, d, sum[e]);
                    }
            const float keep = tid < ng ? mean_of[tid] / cnt : 0.f;
            by_group(sum, mean_of);
            if (tid < ng) p.parts[(image * p.G + g0 + tid) * p.chunks + chunk] = float4{keep, mean_of[tid], cnt, 0.f};
            __syncthreads();
        }
    }
}

// The pieces of a group joined: a wavefront for each group of an image.
__global__ void __launch_bounds__(256)
norm_join_kernel(const float4* __restrict__ parts, long long groups, long long chunks, float eps, float2* __restrict__ stats) {
    const int lane = threadIdx.x & 63;
    for (long long g = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); g < groups; g += (long long)gridDim.x * 4) {
        const float4* a = parts + g * chunks;
        double n = 0, s = 0;
        for (long long c = lane; c < chunks; c += 64) n += a[c].z, s += (double)a[c].z * a[c].x;
        for (int m = 32; m > 0; m >>= 1) n += __shfl_xor(n, m), s += __shfl_xor(s, m);
        const double mean = s / n;
        double m2 = 0;
        for (long long c = lane; c < chunks; c += 64) {
            const double d = a[c].x - mean;
            m2 += a[c].y + a[c].z * d * d;
        }
        for (int m = 32; m > 0; m >>= 1) m2 += __shfl_xor(m2, m);
        if (lane == 0) stats[g] = float2{(float)mean, (float)(1.0 / sqrt(m2 / n + (double)eps))};
    }
}

// ---- y ---------------------------------------------------------------------------------------------
// Token-major: a thread takes eight channels of a position.
template <typename X>
__global__ void __launch_bounds__(256)
norm_rows_kernel(norm_args p) {
    const int cvec = (p.C + 7) / 8;
    const long long total = p.images * p.P * cvec;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long long)gridDim.x * 256) {
        const long long row = i / cvec, image = row / p.P;
        const int c0 = (int)(i - row * cvec) * 8, n = min(8, p.C - c0);
        const int8_eight<X> v = int8_load8(static_cast<const X*>(p.x) + row * p.ldx, c0, p.C);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) {
                const float2 st = p.stats[image * p.G + (c0 + e) / p.cg];
                const float h = (v.get(e) - st.x) * (st.y * (p.gamma ? p.gamma[c0 + e] : 1.f)) + (p.beta ? p.beta[c0 + e] : 0.f);
                tsvd_store_y(p.y, (size_t)row * p.ldy + c0 + e, norm_act(h, p.act), p.out_bf16);
            }
    }
}

// Feature-major: lanes along the positions, so that a channel's values leave side by side; a thread takes eight channels of a position.
template <typename X>
__global__ void __launch_bounds__(256)
norm_columns_kernel(norm_args p) {
    const int cvec = (p.C + 7) / 8;
    const long long rows = p.images * p.P, blocks = (rows + 255) / 256, items = blocks * cvec;
    for (long long item = blockIdx.x; item < items; item += gridDim.x) {
        const long long row = item / cvec * 256 + threadIdx.x;
        const int c0 = (int)(item % cvec) * 8, n = min(8, p.C - c0);
        if (row >= rows) continue;
        const long long image = row / p.P;
        const int8_eight<X> v = int8_load8(static_cast<const X*>(p.x) + row * p.ldx, c0, p.C);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) {
                const float2 st = p.stats[image * p.G + (c0 + e) / p.cg];
                const float h = (v.get(e) - st.x) * (st.y * (p.gamma ? p.gamma[c0 + e] : 1.f)) + (p.beta ? p.beta[c0 + e] : 0.f);
                tsvd_store_y(p.y, (size_t)(c0 + e) * p.ldy + row, norm_act(h, p.act), p.out_bf16);
            }
    }
}

// Codes: a workgroup for each position, its values computed twice (for the largest magnitude, then for the codes).
template <typename X>
__global__ void __launch_bounds__(256)
norm_int8_kernel(norm_args p) {
    __shared__ uint32_t lds[4];
    const int cvec = (p.C + 7) / 8, tid = threadIdx.x;
    const long long rows = p.images * p.P;
    for (long long row = blockIdx.x; row < rows; row += gridDim.x) {
        const X* x = static_cast<const X*>(p.x) + row * p.ldx;
        const float2* stats = p.stats + row / p.P * p.G;
        auto values = [&](int c0, float (&f)[8]) {
            const int8_eight<X> v = int8_load8(x, c0, p.C);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                f[e] = 0.f;
                if (c0 + e < p.C) {
                    const float2 st = stats[(c0 + e) / p.cg];
                    f[e] = norm_act((v.get(e) - st.x) * (st.y * (p.gamma ? p.gamma[c0 + e] : 1.f)) + (p.beta ? p.beta[c0 + e] : 0.f), p.act);
                }
            }
        };
        uint32_t top = 0;
        for (int i = tid; i < cvec; i += 256) {
            float f[8];
            values(8 * i, f);
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(f[e]) & 0x7FFFFFFFu);
        }
        top = int8_wave_top(top);
        __syncthreads();
        if ((tid & 63) == 0) lds[tid >> 6] = top;
        __syncthreads();
        top = max(max(lds[0], lds[1]), max(lds[2], lds[3]));
        float scale, factor;
        int8_factors(top, &scale, &factor);
        if (tid == 0) p.scales[row] = scale;
        for (int i = tid; i < cvec; i += 256) {
            float f[8];
            values(8 * i, f);
            uint32_t c[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) c[e] = int8_code(f[e], factor);
            *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.y) + (size_t)row * p.ldy + 8 * i) = uint2{int8_pack4(c[0], c[1], c[2], c[3]), int8_pack4(c[4], c[5], c[6], c[7])};
        }
    }
}

// ---- the calls -------------------------------------------------------------------------------------
size_t round256(size_t v) { return (v + 255) & ~(size_t)255; }
unsigned grid_of(long long blocks) { return (unsigned)std::min<long long>(blocks, 1 << 20); }

constexpr int STATS_T = 256, STATS_NV = 8;

// How the channels and positions of an image are cut for the statistics: about 64 channels (128 bytes of bf16, a line) of whole groups a workgroup, one group where it has more.
void cut(long long P, int C, int G, norm_args* a) {
    a->C = C, a->G = G, a->cg = C / G, a->P = P;
    a->gpb = std::max(1, std::min(G, 64 / a->cg));
    a->nblk = (G + a->gpb - 1) / a->gpb;
    if (a->gpb == 1) {
        a->rows = 0;
        a->chunks = (P * ((a->cg + 7) / 8) + STATS_T * STATS_NV - 1) / (STATS_T * STATS_NV);
    } else {
        const int cvec = (a->gpb * a->cg + 7) / 8;
        a->rows = STATS_T / cvec * STATS_NV;
        a->chunks = (P + a->rows - 1) / a->rows;
    }
}
size_t stats_bytes(long long images, int G) { return round256((size_t)images * G * sizeof(float2)); }

template <typename X>
hipError_t statistics(const norm_args& a, hipStream_t stream) {
    const dim3 grid(grid_of(a.images * a.nblk * a.chunks));
    if (a.gpb == 1) hipLaunchKernelGGL((norm_stats_kernel<X, STATS_T, STATS_NV, true>), grid, dim3(STATS_T), 0, stream, a);
    else hipLaunchKernelGGL((norm_stats_kernel<X, STATS_T, STATS_NV, false>), grid, dim3(STATS_T), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const long long groups = a.images * a.G;
    hipLaunchKernelGGL(norm_join_kernel, dim3(grid_of((groups + 3) / 4)), dim3(256), 0, stream, a.parts, groups, a.chunks, a.eps, a.stats);
    return hipGetLastError();
}

bool bad_dtype(int t) { return t != TSVD_F32 && t != TSVD_BF16; }

tsvd_status common(const void* x, tsvd_dtype x_dtype, int64_t images, int64_t P, int64_t C, int64_t ldx, int64_t groups, const float* gamma, const float* beta, float eps,
                   tsvd_activation act, void* workspace, size_t workspace_bytes, norm_args* a) {
    if (!x || images < 1 || P < 1 || C < 1 || groups < 1 || bad_dtype(x_dtype) || ldx < C || !(eps > 0.f) || !std::isfinite(eps) || act < TSVD_ACT_NONE || act > TSVD_ACT_GELU)
        return TSVD_EINVAL;
    if (C % groups != 0) return TSVD_EINVAL;
    if (C > (1 << 20) || images > INT32_MAX / P) return TSVD_EUNSUPPORTED;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < tsvd_group_norm_workspace_bytes(images, P, C, groups)) return TSVD_EINVAL;
    a->x = x, a->ldx = ldx, a->images = images;
    a->gamma = gamma, a->beta = beta, a->eps = eps, a->act = act;
    cut(P, (int)C, (int)groups, a);
    a->stats = static_cast<float2*>(workspace);
    a->parts = reinterpret_cast<float4*>(static_cast<uint8_t*>(workspace) + stats_bytes(images, (int)groups));
    return TSVD_OK;
}

}  // namespace

extern "C" size_t tsvd_group_norm_workspace_bytes(int64_t images, int64_t positions, int64_t C, int64_t groups) {
    if (images < 1 || positions < 1 || C < 1 || groups < 1 || C % groups != 0 || C > (1 << 20) || images > INT32_MAX / positions) return 0;
    norm_args a = {};
    cut(positions, (int)C, (int)groups, &a);
    return stats_bytes(images, (int)groups) + round256((size_t)images * groups * a.chunks * sizeof(float4));
}

extern "C" tsvd_status tsvd_group_norm(const void* x_dev, tsvd_dtype x_dtype, int64_t images, int64_t positions, int64_t C, int64_t ldx, int64_t groups,
                                       const float* gamma_dev, const float* beta_dev, float eps, tsvd_activation act, void* y_dev, tsvd_dtype y_dtype,
                                       tsvd_layout y_layout, int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
    norm_args a = {};
    if (!y_dev || bad_dtype(y_dtype) || (y_layout != TSVD_FEATURE_MAJOR && y_layout != TSVD_TOKEN_MAJOR)) return TSVD_EINVAL;
    const tsvd_status st = common(x_dev, x_dtype, images, positions, C, ldx, groups, gamma_dev, beta_dev, eps, act, workspace, workspace_bytes, &a);
    if (st != TSVD_OK) return st;
    if (ldy < (y_layout == TSVD_TOKEN_MAJOR ? C : images * positions)) return TSVD_EINVAL;
    a.y = y_dev, a.ldy = ldy, a.out_bf16 = y_dtype == TSVD_BF16;
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = x_dtype == TSVD_BF16 ? statistics<uint16_t>(a, s) : statistics<float>(a, s);
    if (e != hipSuccess) return TSVD_EDEVICE;
    const long long rows = a.images * a.P, cvec = (C + 7) / 8;
    if (y_layout == TSVD_TOKEN_MAJOR) {
        const dim3 grid(grid_of((rows * cvec + 255) / 256));
        if (x_dtype == TSVD_BF16) hipLaunchKernelGGL(norm_rows_kernel<uint16_t>, grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL(norm_rows_kernel<float>, grid, dim3(256), 0, s, a);
    } else {
        const dim3 grid(grid_of((rows + 255) / 256 * cvec));
        if (x_dtype == TSVD_BF16) hipLaunchKernelGGL(norm_columns_kernel<uint16_t>, grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL(norm_columns_kernel<float>, grid, dim3(256), 0, s, a);
    }
    return hipGetLastError() == hipSuccess ? TSVD_OK : TSVD_EDEVICE;
}

extern "C" tsvd_status tsvd_group_norm_int8(const void* x_dev, tsvd_dtype x_dtype, int64_t images, int64_t positions, int64_t C, int64_t ldx, int64_t groups,
                                            const float* gamma_dev, const float* beta_dev, float eps, tsvd_activation act, int8_t* codes_dev, int64_t ldq,
                                            float* scales_dev, void* workspace, size_t workspace_bytes, void* stream) {
    norm_args a = {};
    if (!codes_dev || !scales_dev || (reinterpret_cast<uintptr_t>(codes_dev) & 15u) || ldq % 16 != 0) return TSVD_EINVAL;
    const tsvd_status st = common(x_dev, x_dtype, images, positions, C, ldx, groups, gamma_dev, beta_dev, eps, act, workspace, workspace_bytes, &a);
    if (st != TSVD_OK) return st;
    if (ldq < C) return TSVD_EINVAL;
    if (C > TSVD_INT8_MAX_N) return TSVD_EUNSUPPORTED;
    a.y = codes_dev, a.ldy = ldq, a.scales = scales_dev;
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e = x_dtype == TSVD_BF16 ? statistics<uint16_t>(a, s) : statistics<float>(a, s);
    if (e != hipSuccess) return TSVD_EDEVICE;
    const dim3 grid(grid_of(a.images * a.P));
    if (x_dtype == TSVD_BF16) hipLaunchKernelGGL(norm_int8_kernel<uint16_t>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(norm_int8_kernel<float>, grid, dim3(256), 0, s, a);
    return hipGetLastError() == hipSuccess ? TSVD_OK : TSVD_EDEVICE;
}
