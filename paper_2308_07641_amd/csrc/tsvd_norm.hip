// Group norm with an activation, channels last (include/tsvd_norm.h).
//
// Bound by memory: x once and y once where a workgroup can hold what it normalises, else x twice.  A thread keeps eight neighbouring channels and walks along the
// positions: sums of x - k and (x - k)^2 for each channel, k being the first value that it meets.  As k is one of the values, the deviations that cancel are
// part of the result: the sum of squares about the thread's own mean is right to the number of its values times 2^-24, whatever the values are.  Threads, and pieces of an
// image, are then joined in fp64 the same way, as counts, sums and sums of squares about the mean of the first of them.  Every sum has a fixed order.  What is left of a large mean is the
// rounding of the pieces' means to fp32.
//
// Forms: rows (one position and one group: a row in registers, its sums about its first value), one launch (a workgroup has all positions of an image for some groups, or whole images: codes), and two launches
// (statistics of pieces; y or codes, every workgroup joining the pieces that it needs; x comes a second time, from the memory-side cache where it fits).
//
// Measured: 16 images of 16384 positions, 256 channels in 32 groups, bf16: statistics 40 us (3.3 TB/s), y 47 us (5.6 TB/s both ways); 8 of 1024 x 640 in one launch 11.9 us; one of
// 64 x 320 5.0 us; 2048 rows of 4096 into codes 9.1 us (2.8 TB/s; 7.9 back to back).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "../../include/tsvd_norm.h"
#include "tsvd_epilogue.h"
#include "tsvd_int8.h"

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Rows of one thread at most in the statistics, and with the eight channels of a vector the values behind one k: what their error grows with.
constexpr int MAX_ROWS = 64;

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
    int out_bf16, token_major;
    float* scales;                // int8 output
    float4* parts;                // [images][G][chunks]: mean, sum of squared deviations, values
    long long chunks;             // pieces of an image along its positions (single groups: along its vectors)
    int gpb, nblk;                // statistics: groups of a workgroup, workgroups side by side along the channels
    int rows;                     // positions of a piece
    int vecs, vblk;               // y: vectors of a workgroup, workgroups side by side
    long long y_rows, y_chunks;   // y: positions of a workgroup, workgroups one behind the other
};

template <int J>
__device__ __forceinline__ float norm_xor(float v) { return __uint_as_float(lane_xor32<J>(__float_as_uint(v))); }
template <int J>
__device__ __forceinline__ double norm_xor(double v) { return lane_xor<J>(v); }

__device__ __forceinline__ float value_of(float x) { return x; }
__device__ __forceinline__ float value_of(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

// a / b for 0 <= a < 2^20, b >= 1: (a + 1/2) / b is 1 / (2 b) away from a whole number at least, more than the two roundings.  (A division of integers takes some forty
// instructions, one of 64 bits hundreds, and everything here waits for them.)
__device__ __forceinline__ int quotient(int a, int b) { return (int)(((float)a + 0.5f) * __builtin_amdgcn_rcpf((float)b)); }

// erfc(a) for a >= 0 to 1.5e-7 (Abramowitz and Stegun, 7.1.26).
__device__ __forceinline__ float norm_erfc(float a) {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, a, 1.f));
    const float poly = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
    return poly * __expf(-a * a);
}
// act of eight values (act is the same for the whole launch: one branch for all of them)
__device__ __forceinline__ void norm_act(float (&f)[8], int act) {
    if (act == TSVD_ACT_SILU) {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] *= __builtin_amdgcn_rcpf(1.f + __expf(-f[e]));
    } else if (act == TSVD_ACT_GELU) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float c = norm_erfc(fabsf(f[e]) * 0.70710678118654752f);
            f[e] *= f[e] > 0.f ? fmaf(-0.5f, c, 1.f) : 0.5f * c;
        }
    } else if (act == TSVD_ACT_RELU) {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = f[e] < 0.f ? 0.f : f[e];          // (NaN stays)
    }
}

// What a thread multiplies and adds for its eight channels: gamma and beta first (they do not wait for the statistics), then the groups' mean and 1 / sqrt(v + eps).
struct norm_channels {
    float mean[8], factor[8], beta[8];
    __device__ __forceinline__ void load(const norm_args& p, int c0, int n) {
        int8_eight<float> g, b;
        b.zero();
        if (p.beta) b = int8_load8(p.beta + c0, 0, n);
#pragma unroll
        for (int e = 0; e < 8; ++e) beta[e] = b.get(e), factor[e] = 1.f;
        if (p.gamma) {
            g = int8_load8(p.gamma + c0, 0, n);
#pragma unroll
            for (int e = 0; e < 8; ++e) factor[e] = g.get(e);
        }
    }
    // n channels from c0 on; of groups from g0 on
    __device__ __forceinline__ void set(int cg, int c0, int n, int g0, const float* mean_of, const float* rstd_of) {
        const int first = quotient(c0, cg);
        int g = first - g0, left = cg - (c0 - first * cg);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int at = e < n ? g : 0;
            mean[e] = mean_of[at];
            factor[e] *= rstd_of[at];
            if (--left == 0) ++g, left = cg;
        }
    }
    __device__ __forceinline__ void set(float m, float rstd) {
#pragma unroll
        for (int e = 0; e < 8; ++e) mean[e] = m, factor[e] *= rstd;
    }
    template <typename X>
    __device__ __forceinline__ void apply(const int8_eight<X>& v, int act, float (&f)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = fmaf(v.get(e) - mean[e], factor[e], beta[e]);
        norm_act(f, act);
    }
};

// N rows of a vector, from `pos` on in steps: loads that all go out together.  WHOLE: all eight channels exist; no branch stands between the loads then, and
// rows at or behind the end are the last one again (not used).
template <bool WHOLE, int N, typename X>
__device__ __forceinline__ void load_rows(int8_eight<X> (&u)[N], const X* x, long long ldx, int at, int valid, int pos, int step, int end) {
    auto row = [&](int k) { return x + (long long)min(pos + k * step, end - 1) * ldx; };
    if constexpr (WHOLE) {
#pragma unroll
        for (int k = 0; k < N; ++k) u[k].load(row(k) + at);
    } else int8_loads8(u, row, at, valid);
}
// The same where the rows are within 2^31 bytes of x (end * ldx * sizeof(X)): the places in 32 bits.
template <bool WHOLE, int N, typename X>
__device__ __forceinline__ void load_near_rows(int8_eight<X> (&u)[N], const X* x, uint32_t ldx, int at, int valid, int pos, int step, int end) {
    uint32_t from = (uint32_t)min(pos, end - 1) * ldx;
    const uint32_t last = (uint32_t)(end - 1) * ldx, by = (uint32_t)step * ldx;
    if constexpr (WHOLE) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            u[k].load(reinterpret_cast<const X*>(reinterpret_cast<const char*>(x) + (from + (uint32_t)at) * (uint32_t)sizeof(X)));
            from = min(from + by, last);
        }
    } else int8_loads8(u, [&](int) {
        const X* row = x + from;
        from = min(from + by, last);
        return row;
    }, at, valid);
}
template <typename F>
__device__ __forceinline__ void whole_or_not(int channels, F&& body) {
    if (channels % 8 == 0) body(std::true_type());
    else body(std::false_type());
}

// n values side by side (token-major y)
__device__ __forceinline__ void store8(void* y, size_t at, const float (&f)[8], int n, int out_bf16) {
    if (n >= 8) {
        if (out_bf16) {
            typedef u32x4 u32x4_at __attribute__((aligned(2)));
            *reinterpret_cast<u32x4_at*>(static_cast<uint16_t*>(y) + at) = u32x4{tsvd_pack_bf16(f[0], f[1]), tsvd_pack_bf16(f[2], f[3]), tsvd_pack_bf16(f[4], f[5]), tsvd_pack_bf16(f[6], f[7])};
        } else {
            typedef f32x4 f32x4_at __attribute__((aligned(4)));
            *reinterpret_cast<f32x4_at*>(static_cast<float*>(y) + at) = f32x4{f[0], f[1], f[2], f[3]};
            *reinterpret_cast<f32x4_at*>(static_cast<float*>(y) + at + 4) = f32x4{f[4], f[5], f[6], f[7]};
        }
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) tsvd_store_y(y, at + e, f[e], out_bf16);
    }
}
// ... and in rows of their own (feature-major y)
__device__ __forceinline__ void store8_apart(void* y, int c0, long long ldy, long long row, const float (&f)[8], int n, int out_bf16) {
    size_t at = (size_t)c0 * ldy + row;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (e < n) tsvd_store_y(y, at, f[e], out_bf16);
        at += ldy;
        asm("" : "+v"(at));                              // (eight places held over a loop of rows are registers that the rows need)
    }
}

__device__ __forceinline__ uint2 codes_of(const float (&f)[8], float factor) {
    uint32_t c[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = int8_code(f[e], factor);
    return uint2{int8_pack4(c[0], c[1], c[2], c[3]), int8_pack4(c[4], c[5], c[6], c[7])};
}

// ---- sums ------------------------------------------------------------------------------------------
// Of one channel and thread: values about the first of them.
struct norm_sums {
    float k[8], s1[8], s2[8];
    int n;
    __device__ __forceinline__ void clear() {
        n = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) k[e] = s1[e] = s2[e] = 0.f;
    }
    template <typename X>
    __device__ __forceinline__ void add(const int8_eight<X>& v) {
        if (n++ == 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) k[e] = v.get(e);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float d = v.get(e) - k[e];
            s1[e] += d;
            s2[e] = fmaf(d, d, s2[e]);
        }
    }
};

// What the threads of a workgroup know of its groups, in LDS: a thread (row r of R, vector `at` of cvec) leaves mean, sum of squares and number of its values of every
// group g that its eight channels belong to.  Going along a row either the vector or the group is the next one, so at + g is a place of its own.
struct norm_piece {
    float mean, m2, n;
};
struct norm_lds {
    norm_piece* piece;            // [R][cvec + ng]
    float *mean, *m2;             // [ng]: of the groups
    __device__ __forceinline__ norm_lds(float* base, int ng, int R, int cvec) : piece(reinterpret_cast<norm_piece*>(base + 2 * ng)), mean(base), m2(base + ng) {}
    static size_t bytes(int ng, int R, int cvec) { return 8 * (size_t)ng + sizeof(norm_piece) * (size_t)R * (cvec + ng); }
};
// Lanes that join one of ng groups, T threads in all: a power of two up to 64.
__device__ __forceinline__ int lanes_log2(int ng, int T) {
    int log = 6;
    while (log > 0 && (ng << log) > T) --log;
    return log;
}
// Sums over groups of 2^log lanes, in all of them (log is the same for all).
template <typename T>
__device__ __forceinline__ T lanes_sum(T v, int log) {
    if (log > 0) v += norm_xor<1>(v);
    if (log > 1) v += norm_xor<2>(v);
    if (log > 2) v += norm_xor<4>(v);
    if (log > 3) v += norm_xor<8>(v);
    if (log > 4) v += norm_xor<16>(v);
    if (log > 5) v += norm_xor<32>(v);
    return v;
}
// Pieces of one group, about the mean k of the first of them (which has values): their number, sum, and sum of squares.
struct norm_join {
    double k, n = 0, sum = 0, sq = 0;
    __device__ __forceinline__ explicit norm_join(float first) : k(first) {}
    __device__ __forceinline__ void add(float mean, float m2, float count) {
        const double d = mean - k, nd = count * d;
        n += count, sum += nd, sq += m2 + nd * d;
    }
};
// Those of 2^log lanes -> mean, and the sum of squared deviations or 1 / sqrt(v + eps).
template <bool FINAL>
__device__ __forceinline__ void store_joined(const norm_join& of, int log, float eps, bool mine, float* mean, float* m2) {
    const double n = lanes_sum(of.n, log), sum = lanes_sum(of.sum, log), sq = lanes_sum(of.sq, log);
    if (!mine) return;
    // (n is a whole number: its reciprocal in fp32, corrected once, is right to 2^-45, of a mean that is as large as the deviations)
    const double r0 = __builtin_amdgcn_rcpf((float)n), inv = r0 * (2.0 - n * r0), off = sum * inv, dev = sq - sum * off;
    *mean = (float)(of.k + off);
    if constexpr (FINAL) {
        const float v = (float)(dev * inv);
        *m2 = __builtin_amdgcn_rsqf((v < 0.f ? 0.f : v) + eps);       // (a variance that is no number stays none)
    } else {
        *m2 = (float)dev;
    }
}
// Means and sums of squared deviations of the workgroup's groups from its threads' sums.
// (FINAL: 1 / sqrt(v + eps) in the place of the sum of squares)
template <int T, bool FINAL>
__device__ __forceinline__ void join_threads(const norm_lds& l, const norm_sums& s, int at, int r, int cvec, int R, int nch, int ng, int cg, float eps) {
    const int tid = threadIdx.x;
    if (r < R) {
        const float n = (float)s.n, inv = s.n ? __builtin_amdgcn_rcpf(n) : 0.f;
        const int valid = min(8, nch - 8 * at);
        norm_piece* to = l.piece + r * (cvec + ng) + at;
        int g = quotient(8 * at, cg), left = cg - (8 * at - g * cg);
        // channels from .. to - 1 of the vector as one piece: their means about the first of them
        auto piece = [&](int from, int end) {
            float first = 0.f, sum = 0.f, m2 = 0.f;
#pragma unroll
            for (int e = 7; e >= 0; --e) first = e == from ? fmaf(s.s1[e], inv, s.k[e]) : first;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool in = e >= from && e < end;
                const float d = in ? fmaf(s.s1[e], inv, s.k[e]) - first : 0.f;
                sum += d;
                m2 += in ? fmaf(n * d, d, fmaf(-s.s1[e] * inv, s.s1[e], s.s2[e])) : 0.f;
            }
            const float count = (float)(end - from), off = sum * __builtin_amdgcn_rcpf(count);
            to[g++] = norm_piece{first + off, fmaf(-n * sum, off, m2), n * count};
        };
        int from = 0, end = min(left, valid);
        piece(from, end);
        while (end < valid) {
            from = end, end = min(end + cg, valid);
            piece(from, end);
        }
    }
    __syncthreads();
    const int log = lanes_log2(ng, T), L = 1 << log, lane = tid & (L - 1);
    for (int g = tid >> log; g < ((ng + (T >> log) - 1) & -(T >> log)); g += T >> log) {       // (whole wavefronts)
        norm_join join(0.f);
        if (g < ng) {
            const int a0 = (g * cg) >> 3, nv = ((g * cg + cg - 1) >> 3) - a0 + 1, step_r = quotient(L, nv), step_k = L - step_r * nv;
            int row = quotient(lane, nv), k = lane - row * nv;
            const norm_piece* from = l.piece + a0 + g;
            // (the mean of the first piece is read behind the lane's own first one: one wait for both)
            norm_piece q = from[min(row, R - 1) * (cvec + ng) + k];
            join = norm_join(from->mean);
            while (row < R) {
                join.add(q.mean, q.m2, q.n);
                row += step_r, k += step_k;
                if (k >= nv) k -= nv, ++row;
                q = from[min(row, R - 1) * (cvec + ng) + k];
            }
        }
        store_joined<FINAL>(join, log, eps, g < ng && lane == 0, l.mean + g, l.m2 + g);
    }
    __syncthreads();
}

// ---- one launch: a workgroup has the groups blk gpb ... of an image, all positions ----------------------------
// NV: rows of a thread at most, held in registers.
template <typename X, int T, int NV>
__global__ void __launch_bounds__(T)
norm_one_kernel(norm_args p) {
    extern __shared__ __align__(16) float smem[];
    const int tid = threadIdx.x;
    const uint32_t items = (uint32_t)(p.images * p.nblk), each = items >> 3, more = items & 7;
    for (uint32_t id = blockIdx.x; id < items; id += gridDim.x) {
        // workgroups go round the XCDs: each gets a run of the items, so that the groups of an image, which share lines of x and y, meet in one L2
        const uint32_t item = (id & 7) * each + min(id & 7, more) + (id >> 3), image = item / (uint32_t)p.nblk;
        const int blk = (int)(item - image * p.nblk), g0 = blk * p.gpb, ng = min(p.gpb, p.G - g0), c0 = g0 * p.cg, nch = ng * p.cg, cvec = (nch + 7) / 8;
        const int R = quotient(T, cvec), r = quotient(tid, cvec), at = tid - r * cvec, P = (int)p.P;
        // (a last vector that is not whole is read and written as the last eight channels, some of them twice; the sums leave those out)
        const int n = min(8, nch), c = max(0, min(8 * at, nch - 8)), twice = 8 * at - c;
        const bool active = r < R;
        const X* x = static_cast<const X*>(p.x) + (long long)image * p.P * p.ldx + c0;
        const norm_lds l(smem, ng, R, cvec);
        whole_or_not(nch, [&](auto whole) {
        norm_sums s;
        s.clear();
        norm_channels ch;
        int8_eight<X> v[NV];
        load_near_rows<decltype(whole)::value>(v, x, (uint32_t)p.ldx, c, nch, r, R, P);
        if (active) ch.load(p, c0 + c, n);
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (active && r + k * R < P) {
                if constexpr (decltype(whole)::value) s.add(v[k]);
                else {
                    int8_eight<X> own = v[k];
                    own.shift(twice);
                    s.add(own);
                }
            }
        join_threads<T, true>(l, s, at, r, cvec, R, nch, ng, p.cg, p.eps);
        if (active) {
            ch.set(p.cg, c0 + c, n, g0, l.mean, l.m2);
            const long long row0 = (long long)image * p.P;
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (r + k * R < P) {
                    const long long row = row0 + r + k * R;
                    float f[8];
                    ch.apply(v[k], p.act, f);
                    if (p.token_major) store8(p.y, (size_t)row * p.ldy + c0 + c, f, n, p.out_bf16);
                    else store8_apart(p.y, c0 + c, p.ldy, row, f, n, p.out_bf16);
                }
        }
        });
        __syncthreads();
    }
}

// Codes in one launch: a workgroup has a whole image, all channels of all its positions, in registers.  The largest magnitudes of the vectors of a position meet in LDS.
template <typename X, int T, int NV>
__global__ void __launch_bounds__(T)
norm_one_int8_kernel(norm_args p) {
    extern __shared__ __align__(16) float smem[];
    const int tid = threadIdx.x, C = p.C, ng = p.G, cvec = (C + 7) / 8, P = (int)p.P;
    const int R = quotient(T, cvec), r = quotient(tid, cvec), at = tid - r * cvec, n = min(8, C - 8 * at);
    const bool active = r < R;
    const norm_lds l(smem, ng, R, cvec);
    uint32_t* tops = reinterpret_cast<uint32_t*>(smem + 2 * ng);         // [NV][T], where the pieces were
    float* factors = smem + 2 * ng + NV * T;                             // [P]
    for (uint32_t image = blockIdx.x; image < (uint32_t)p.images; image += gridDim.x) {
        const X* x = static_cast<const X*>(p.x) + (long long)image * P * p.ldx;
        whole_or_not(C, [&](auto whole) {
            norm_sums s;
            s.clear();
            norm_channels ch;
            int8_eight<X> v[NV];
            load_near_rows<decltype(whole)::value>(v, x, (uint32_t)p.ldx, 8 * at, C, r, R, P);
            if (active) ch.load(p, 8 * at, n);
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (active && r + k * R < P) s.add(v[k]);
            join_threads<T, true>(l, s, at, r, cvec, R, C, ng, p.cg, p.eps);
            float f[NV][8];
            if (active) {
                ch.set(p.cg, 8 * at, n, 0, l.mean, l.m2);
#pragma unroll
                for (int k = 0; k < NV; ++k)
                    if (r + k * R < P) {
                        ch.apply(v[k], p.act, f[k]);
                        uint32_t top = 0;
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (e < n) top = max(top, __float_as_uint(f[k][e]) & 0x7FFFFFFFu);
                        tops[k * T + tid] = top;
                    }
            }
            __syncthreads();
            const int log = lanes_log2(P, T), lane = tid & ((1 << log) - 1);
            for (int pos = tid >> log; pos < P; pos += T >> log) {
                const int k = quotient(pos, R);
                const uint32_t* row = tops + k * T + (pos - k * R) * cvec;
                uint32_t top = 0;
                for (int i = lane; i < cvec; i += 1 << log) top = max(top, row[i]);
                for (int m = 1 << log >> 1; m > 0; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
                float scale, factor;
                int8_factors(top, &scale, &factor);
                if (lane == 0) factors[pos] = factor, p.scales[(long long)image * P + pos] = scale;
            }
            __syncthreads();
            if (active)
#pragma unroll
                for (int k = 0; k < NV; ++k)
                    if (r + k * R < P) *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.y) + ((long long)image * P + r + k * R) * p.ldy + 8 * at) = codes_of(f[k], factors[r + k * R]);
        });
        __syncthreads();
    }
}

// ---- statistics of pieces --------------------------------------------------------------------------------
// Several groups a workgroup, `rows` positions of them.
template <typename X>
__global__ void __launch_bounds__(256)
norm_stats_kernel(norm_args p) {
    constexpr int T = 256;
    extern __shared__ __align__(16) float smem[];
    const int tid = threadIdx.x;
    const uint32_t chunks = (uint32_t)p.chunks, items = (uint32_t)(p.images * p.nblk) * chunks;
    for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
        const uint32_t rest = item / chunks, chunk = item - rest * chunks, image = rest / (uint32_t)p.nblk;
        const int blk = (int)(rest - image * p.nblk), g0 = blk * p.gpb, ng = min(p.gpb, p.G - g0), c0 = g0 * p.cg, nch = ng * p.cg, cvec = (nch + 7) / 8;
        const int R = quotient(T, cvec), r = quotient(tid, cvec), at = tid - r * cvec;
        const long long p0 = (long long)chunk * p.rows;
        const int rows = (int)min((long long)p.rows, p.P - p0);
        const bool active = r < R;
        const X* x = static_cast<const X*>(p.x) + ((long long)image * p.P + p0) * p.ldx + c0;
        const norm_lds l(smem, ng, R, cvec);
        norm_sums s;
        s.clear();
        if (active) whole_or_not(nch, [&](auto whole) {
            constexpr int AHEAD = sizeof(X) == 2 ? 8 : 4;
            for (int pos = r; pos < rows; pos += AHEAD * R) {
                int8_eight<X> u[AHEAD];
                load_rows<decltype(whole)::value>(u, x, p.ldx, 8 * at, nch, pos, R, rows);
#pragma unroll
                for (int k = 0; k < AHEAD; ++k)
                    if (pos + k * R < rows) s.add(u[k]);
            }
        });
        join_threads<T, false>(l, s, at, r, cvec, R, nch, ng, p.cg, 0.f);
        for (int g = tid; g < ng; g += T) p.parts[((long long)image * p.G + g0 + g) * p.chunks + chunk] = float4{l.mean[g], l.m2[g], (float)rows * (float)p.cg, 0.f};
        __syncthreads();
    }
}
// One group of many channels: `rows` vectors a thread, of the group's vectors in order, whatever position they belong to.
template <typename X>
__global__ void __launch_bounds__(256)
norm_stats_wide_kernel(norm_args p) {
    constexpr int T = 256;
    __shared__ double part[T / 64];
    const int tid = threadIdx.x, cvec = (p.cg + 7) / 8, step_p = T / cvec, step_v = T % cvec;
    auto reduce = [&](double a) {
        a = wave_sum(a);
        __syncthreads();
        if ((tid & 63) == 0) part[tid >> 6] = a;
        __syncthreads();
        a = 0;
#pragma unroll
        for (int w = 0; w < T / 64; ++w) a += part[w];
        return a;
    };
    const uint32_t chunks = (uint32_t)p.chunks, items = (uint32_t)(p.images * p.G) * chunks;
    for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
        const uint32_t group_at = item / chunks, image_at = group_at / (uint32_t)p.G;
        const long long group = group_at, image = image_at, chunk = item - group_at * chunks;
        const X* x = static_cast<const X*>(p.x) + image * p.P * p.ldx + (group - image * p.G) * p.cg;
        const long long first = chunk * T * p.rows + tid;
        long long pos = first / cvec;
        int at = (int)(first - pos * cvec), n = 0;
        float k = 0.f, s1 = 0.f, s2 = 0.f;
        int8_eight<X> v[MAX_ROWS / 8];
        int here[MAX_ROWS / 8];
#pragma unroll
        for (int i = 0; i < MAX_ROWS / 8; ++i) {
            here[i] = 0;
            v[i].zero();
            if (i >= p.rows) continue;                           // (the same for all)
            if (pos < p.P) here[i] = min(8, p.cg - 8 * at);
            if (here[i] == 8) v[i].load(x + pos * p.ldx + 8 * at);
            else if (here[i]) v[i] = int8_load8(x + pos * p.ldx, 8 * at, p.cg);
            at += step_v, pos += step_p;
            if (at >= cvec) at -= cvec, ++pos;
        }
#pragma unroll
        for (int i = 0; i < MAX_ROWS / 8; ++i) {
            if (i >= p.rows) continue;
            if (i == 0) k = v[0].get(0);
            n += here[i];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = e < here[i] ? v[i].get(e) - k : 0.f;
                s1 += d;
                s2 = fmaf(d, d, s2);
            }
        }
        const double N = reduce(n), mean = reduce(n ? (double)n * k + s1 : 0.0) / N;
        double m2 = 0;
        if (n) {
            const double d = k + (double)s1 / n - mean;
            m2 = (double)s2 - (double)s1 * s1 / n + n * d * d;
        }
        m2 = reduce(m2);
        if (tid == 0) p.parts[group * p.chunks + chunk] = float4{(float)mean, (float)m2, (float)N, 0.f};
    }
}

// The pieces of groups g0 ... g0 + ng - 1 of an image joined, as above: mean and 1 / sqrt(v + eps).
template <int T>
__device__ __forceinline__ void join_parts(const norm_args& p, long long image, int g0, int ng, float* mean, float* rstd) {
    const int tid = threadIdx.x, chunks = (int)p.chunks, log = lanes_log2(ng, T), L = 1 << log, lane = tid & (L - 1);
    for (int g = tid >> log; g < ((ng + (T >> log) - 1) & -(T >> log)); g += T >> log) {
        const float4* a = p.parts + (image * p.G + g0 + min(g, ng - 1)) * p.chunks;
        // (the mean of the first piece is asked for behind the lane's own first ones: one wait for all of them)
        float4 q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i == 0 || i * L < chunks) q[i] = a[min(lane + i * L, chunks - 1)];
        norm_join join(a[0].x);
        for (int c = lane;;) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (c + i * L < chunks) join.add(q[i].x, q[i].y, q[i].z);
            c += 4 * L;
            if (c >= chunks) break;
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = a[min(c + i * L, chunks - 1)];
        }
        store_joined<true>(join, log, p.eps, g < ng && lane == 0, mean + g, rstd + g);
    }
    __syncthreads();
}

// ---- y ---------------------------------------------------------------------------------------------
// A workgroup has `vecs` vectors of channels and `y_rows` positions of an image.  Token-major: as in the statistics.  Feature-major: eight vectors of channels, through LDS, so
// that a channel's positions leave side by side.  (Lanes along the positions instead, 16 bytes of 64 rows a load: 50 images of 1599 positions, 768 channels, 171 us.)
template <typename X, bool TOKENS>
__global__ void __launch_bounds__(256)
norm_apply_kernel(norm_args p) {
    constexpr int T = 256;
    extern __shared__ __align__(16) float smem[];
    const int tid = threadIdx.x;
    const uint32_t chunks = (uint32_t)p.y_chunks, items = (uint32_t)(p.images * p.vblk) * chunks;
    for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
        // the pieces read last come first: they are in the caches
        const uint32_t back = items - 1 - item, rest = back / (uint32_t)p.vblk, blk = back - rest * p.vblk, image_at = rest / chunks;
        const long long image = image_at, chunk = rest - image_at * chunks;
        const int c0 = (int)blk * p.vecs * 8, nch = min(p.vecs * 8, p.C - c0), cvec = (nch + 7) / 8, g0 = quotient(c0, p.cg), ng = quotient(c0 + nch - 1, p.cg) - g0 + 1;
        const long long row0 = image * p.P + chunk * p.y_rows;
        const int rows = (int)min(p.y_rows, p.P - chunk * p.y_rows);
        const X* x = static_cast<const X*>(p.x) + row0 * p.ldx + c0;
        if constexpr (TOKENS) {
            const int R = quotient(T, cvec), r = quotient(tid, cvec), at = tid - r * cvec, n = min(8, nch), c = max(0, min(8 * at, nch - 8));     // (a last vector that is not whole: the last eight channels, some twice)
            // (the first rows, gamma and beta are on their way while the statistics are joined)
            whole_or_not(nch, [&](auto whole) {
                constexpr int AHEAD = sizeof(X) == 2 ? 8 : 4;
                norm_channels ch;
                int8_eight<X> u[AHEAD];
                load_rows<decltype(whole)::value>(u, x, p.ldx, c, nch, r, R, rows);
                ch.load(p, c0 + c, n);
                join_parts<T>(p, image, g0, ng, smem, smem + ng);
                if (r >= R) return;
                ch.set(p.cg, c0 + c, n, g0, smem, smem + ng);
                const size_t to = (size_t)row0 * p.ldy + c0 + c;
                for (int pos = r; pos < rows; pos += AHEAD * R) {
                    if (pos != r) load_rows<decltype(whole)::value>(u, x, p.ldx, c, nch, pos, R, rows);
#pragma unroll
                    for (int k = 0; k < AHEAD; ++k)
                        if (pos + k * R < rows) {
                            float f[8];
                            ch.apply(u[k], p.act, f);
                            store8(p.y, to + (size_t)(pos + k * R) * p.ldy, f, n, p.out_bf16);
                        }
                }
            });
        } else {
            // 64 positions at a time: eight lanes (of eight channels each) a position, 128 bytes of bf16, through LDS to 16 bytes of a channel's positions a lane
            constexpr int POS = 64, E = 4;
            float* tile = smem + 2 * ng + (2 * ng & 2);              // [64 channels][POS], a vector's rows turned by 8 times its number (64 banks a write)
            const int lane8 = tid & 7, place = tid >> 3, n = min(8, nch - 8 * lane8);
            norm_channels ch;
            if (n > 0) ch.load(p, c0 + 8 * lane8, n);
            join_parts<T>(p, image, g0, ng, smem, smem + ng);
            if (n > 0) ch.set(p.cg, c0 + 8 * lane8, n, g0, smem, smem + ng);
            for (int first = 0; first < rows; first += POS) {
                const int here = min(POS, rows - first);
                int8_eight<X> u[2];
                int8_loads8(u, [&](int k) { return x + (long long)(first + min(place + 32 * k, here - 1)) * p.ldx; }, 8 * lane8, nch);
                if (n > 0)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        float f[8];
                        ch.apply(u[k], p.act, f);
#pragma unroll
                        for (int e = 0; e < 8; ++e) tile[(8 * lane8 + e) * POS + ((place + 32 * k + 8 * lane8) & (POS - 1))] = f[e];
                    }
                __syncthreads();
                for (int i = tid; i < nch * (POS / E); i += T) {
                    const int c = i / (POS / E), pos = i % (POS / E) * E;
                    const f32x4 f = *reinterpret_cast<const f32x4*>(tile + c * POS + ((pos + (c & 56)) & (POS - 1)));
                    const size_t to = (size_t)(c0 + c) * p.ldy + row0 + first + pos;
                    if (pos + E <= here) {
                        if (p.out_bf16) {
                            typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
                            typedef u32x2 u32x2_at __attribute__((aligned(2)));
                            *reinterpret_cast<u32x2_at*>(static_cast<uint16_t*>(p.y) + to) = u32x2{tsvd_pack_bf16(f[0], f[1]), tsvd_pack_bf16(f[2], f[3])};
                        } else {
                            typedef f32x4 f32x4_at __attribute__((aligned(4)));
                            *reinterpret_cast<f32x4_at*>(static_cast<float*>(p.y) + to) = f;
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < E - 1; ++e)
                            if (pos + e < here) tsvd_store_y(p.y, to + e, f[e], p.out_bf16);
                    }
                }
                __syncthreads();
            }
        }
        __syncthreads();
    }
}

// ---- codes -----------------------------------------------------------------------------------------
// L lanes for each position, NV vectors of channels a lane with their factors in registers, `y_rows` positions of an image a workgroup, AHEAD of each lane's at a time.
template <typename X, int L, int NV>
__global__ void __launch_bounds__(256)
norm_int8_kernel(norm_args p) {
    constexpr int AHEAD = NV == 1 ? 4 : 2, SLOTS = 256 / L;
    extern __shared__ __align__(16) float smem[];
    __shared__ uint32_t tops[2][AHEAD][4];
    const int lane = threadIdx.x % L, slot = threadIdx.x / L, cvec = (p.C + 7) / 8;
    const uint32_t chunks = (uint32_t)p.y_chunks, items = (uint32_t)p.images * chunks;
    for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
        const uint32_t back = items - 1 - item, image_at = back / chunks;
        const long long image = image_at, first = (back - image_at * chunks) * p.y_rows;
        const long long row0 = image * p.P + first;
        const int rows = (int)min(p.y_rows, p.P - first);
        join_parts<256>(p, image, 0, p.G, smem, smem + p.G);
        norm_channels ch[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c0 = 8 * (lane + L * k);
            const int n = max(0, min(8, p.C - c0));
            ch[k].load(p, min(c0, p.C - 1), n);
            ch[k].set(p.cg, min(c0, p.C - 1), n, 0, smem, smem + p.G);
        }
        int turn = 0;
        for (int pos = 0; pos < rows; pos += AHEAD * SLOTS, turn ^= 1) {
            int8_eight<X> v[NV][AHEAD];
#pragma unroll
            for (int k = 0; k < NV; ++k)
                int8_loads8(v[k], [&](int a) { return static_cast<const X*>(p.x) + (row0 + min(pos + a * SLOTS + slot, rows - 1)) * p.ldx; }, 8 * (lane + L * k), p.C);
            float f[AHEAD][NV][8];
            uint32_t top[AHEAD];
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                top[a] = 0;
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    ch[k].apply(v[k][a], p.act, f[a][k]);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (8 * (lane + L * k) + e < p.C) top[a] = max(top[a], __float_as_uint(f[a][k][e]) & 0x7FFFFFFFu);
                }
                top[a] = int8_lanes_top<L < 64 ? L : 64>(top[a]);
                if (L > 64 && lane % 64 == 0) tops[turn][a][lane / 64] = top[a];
            }
            if constexpr (L > 64) __syncthreads();                   // (two sets of tops: the next turn's need not wait for this one's readers)
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                if constexpr (L > 64) top[a] = max(max(tops[turn][a][0], tops[turn][a][1]), max(tops[turn][a][2], tops[turn][a][3]));
                const int at = pos + a * SLOTS + slot;
                if (at >= rows) continue;
                float scale, factor;
                int8_factors(top[a], &scale, &factor);
                if (lane == 0) p.scales[row0 + at] = scale;
#pragma unroll
                for (int k = 0; k < NV; ++k)
                    if (lane + L * k < cvec) *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.y) + (size_t)(row0 + at) * p.ldy + 8 * (lane + L * k)) = codes_of(f[a][k], factor);
            }
        }
        __syncthreads();
    }
}
// Rows of more channels: a workgroup for each position, the values computed twice (for the largest magnitude, then for the codes).
template <typename X>
__global__ void __launch_bounds__(256)
norm_int8_wide_kernel(norm_args p) {
    extern __shared__ __align__(16) float smem[];
    __shared__ uint32_t tops[4];
    const int tid = threadIdx.x, cvec = (p.C + 7) / 8;
    const uint32_t chunks = (uint32_t)p.y_chunks, items = (uint32_t)p.images * chunks;
    for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
        const uint32_t image_at = item / chunks;
        const long long image = image_at, first = (item - image_at * chunks) * p.y_rows;
        join_parts<256>(p, image, 0, p.G, smem, smem + p.G);
        for (long long row = image * p.P + first, end = image * p.P + min(p.P, first + p.y_rows); row < end; ++row) {
            const X* x = static_cast<const X*>(p.x) + row * p.ldx;
            auto values = [&](int at, float (&f)[8]) {
                norm_channels ch;
                ch.load(p, 8 * at, min(8, p.C - 8 * at));
                ch.set(p.cg, 8 * at, min(8, p.C - 8 * at), 0, smem, smem + p.G);
                ch.apply(int8_load8(x, 8 * at, p.C), p.act, f);
            };
            uint32_t top = 0;
            for (int at = tid; at < cvec; at += 256) {
                float f[8];
                values(at, f);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (8 * at + e < p.C) top = max(top, __float_as_uint(f[e]) & 0x7FFFFFFFu);
            }
            top = int8_lanes_top<64>(top);
            if ((tid & 63) == 0) tops[tid >> 6] = top;
            __syncthreads();
            float scale, factor;
            int8_factors(max(max(tops[0], tops[1]), max(tops[2], tops[3])), &scale, &factor);
            if (tid == 0) p.scales[row] = scale;
            for (int at = tid; at < cvec; at += 256) {
                float f[8];
                values(at, f);
                *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.y) + (size_t)row * p.ldy + 8 * at) = codes_of(f, factor);
            }
            __syncthreads();
        }
        __syncthreads();
    }
}

// ---- rows: one position, one group --------------------------------------------------------------------
// T threads for a row (64 and fewer: several rows a workgroup and no barrier), NV vectors of eight channels each, in registers.
template <typename X, int T, int NV, bool CODES>
__global__ void __launch_bounds__(T < 256 ? 256 : T)
norm_rows_kernel(norm_args p) {
    constexpr int WAVES = T < 64 ? 1 : T / 64, ROWS = T < 256 ? 256 / T : 1, LOG = T >= 64 ? 6 : T == 32 ? 5 : 4;
    __shared__ float sums[2][WAVES];
    __shared__ uint32_t tops[WAVES];
    const int t = threadIdx.x % T, wave = t >> 6, C = p.C;
    auto reduce = [&](float a, int which) {
        a = lanes_sum(a, LOG);
        if constexpr (T > 64) {
            if ((t & 63) == 0) sums[which][wave] = a;
            __syncthreads();
            a = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) a += sums[which][w];
        }
        return a;
    };
    whole_or_not(C, [&](auto whole) {
        // (whole: a vector's channels exist all or none)
        constexpr bool WHOLE = decltype(whole)::value;
        // gamma and beta stay for all rows of the workgroup
        norm_channels ch[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) ch[k].load(p, WHOLE ? 8 * min(t + k * T, C / 8 - 1) : min(8 * (t + k * T), C - 1), WHOLE ? 8 : max(1, min(8, C - 8 * (t + k * T))));
        const long long step = (long long)gridDim.x * ROWS;
        long long row = (long long)blockIdx.x * ROWS + threadIdx.x / T;
        auto load = [&](int8_eight<X> (&v)[NV], X& first, long long at) {
            const X* x = static_cast<const X*>(p.x) + min(at, p.images - 1) * p.ldx;
            first = x[0];
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                if constexpr (WHOLE) v[k].load(x + 8 * min(t + k * T, C / 8 - 1));
                else v[k] = int8_load8(x, 8 * (t + k * T), C);
            }
        };
        int8_eight<X> v[NV];
        X first;
        load(v, first, row);
        for (; row < p.images; row += step) {
            // values from the row's first one on: rows without deviation give beta, and a large mean costs nothing
            float f[NV][8], sum = 0.f;
            const float from = value_of(first);
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) f[k][e] = v[k].get(e) - from;
            load(v, first, row + step);
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int n = C - 8 * (t + k * T);
                if (!WHOLE || n > 0)
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum += WHOLE || e < n ? f[k][e] : 0.f;
            }
            const float mean = reduce(sum, 0) / (float)C;
            float m2 = 0.f;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int n = C - 8 * (t + k * T);
                if (n > 0)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        f[k][e] -= mean;
                        const float d = WHOLE || e < n ? f[k][e] : 0.f;
                        m2 = fmaf(d, d, m2);
                    }
            }
            const float rstd = 1.f / sqrtf(reduce(m2, 1) / (float)C + p.eps);
            uint32_t top = 0;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int c0 = 8 * (t + k * T), n = C - c0;
                if (n > 0) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[k][e] = fmaf(f[k][e], rstd * ch[k].factor[e], ch[k].beta[e]);
                    norm_act(f[k], p.act);
                    if constexpr (CODES) {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (WHOLE || e < n) top = max(top, __float_as_uint(f[k][e]) & 0x7FFFFFFFu);
                    } else {
                        if (p.token_major) store8(p.y, (size_t)row * p.ldy + c0, f[k], n, p.out_bf16);
                        else store8_apart(p.y, c0, p.ldy, row, f[k], n, p.out_bf16);
                    }
                }
            }
            if constexpr (CODES) {
                top = int8_lanes_top<(T < 64 ? T : 64)>(top);
                if constexpr (T > 64) {
                    if ((t & 63) == 0) tops[wave] = top;
                    __syncthreads();
#pragma unroll
                    for (int w = 0; w < WAVES; ++w) top = max(top, tops[w]);
                }
                float scale, factor;
                int8_factors(top, &scale, &factor);
                if (t == 0) p.scales[row] = scale;
#pragma unroll
                for (int k = 0; k < NV; ++k)
                    if (8 * (t + k * T) < C) *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.y) + (size_t)row * p.ldy + 8 * (t + k * T)) = codes_of(f[k], factor);
            }
            // (sums[0] is written again behind the barriers of sums[1] and of what follows; a workgroup without codes needs one more)
            if constexpr (T > 64 && !CODES) __syncthreads();
        }
    });
}

// ---- the calls -------------------------------------------------------------------------------------
size_t round256(size_t v) { return (v + 255) & ~(size_t)255; }
unsigned grid_of(long long blocks) { return (unsigned)std::min<long long>(blocks, 1 << 20); }
long long up(long long v, long long m) { return (v + m - 1) / m; }

// (CUS: of a whole card, which the figures of the rules below were measured on.  Results do not depend on it.)
constexpr int CUS = 256, VECS = 20, MAX_GROUPS = 4096;

// Groups whose channels are whole vectors, where that takes 128 channels at most.
int whole_groups(int cg) {
    int unit = 1;
    while (unit < 8 && unit * cg % 8 != 0) unit *= 2;
    return unit * cg % 8 == 0 && unit * cg <= 128 ? unit : 1;
}
// Statistics by pieces: whole groups of about 160 channels side by side (whole lines of x; each workgroup that makes y reads all pieces of its groups, so few groups and few
// pieces: 32 groups by 64 pieces took as long as the rows themselves), pieces of up to 64 positions a thread, about 512 workgroups in all where x is small.
void cut(long long images, long long P, int C, int G, norm_args* a) {
    a->images = images, a->P = P, a->C = C, a->G = G, a->cg = C / G;
    a->gpb = std::min(G, VECS * 8 / a->cg);
    if (a->gpb <= 1 && a->cg > 64) {
        a->gpb = 0;                                          // one group, by its vectors (16384 positions of 128 channels: 1024 pieces, 13.8 us where x and y alone take 2.5)
        a->nblk = G;
        const long long vecs = P * up(a->cg, 8);
        a->rows = (int)std::max<long long>(1, std::min<long long>(MAX_ROWS / 8, up(vecs * images * G, 1024 * 256)));
        a->chunks = up(vecs, 256 * a->rows);
        return;
    }
    a->nblk = (int)up(G, a->gpb);
    const int unit = whole_groups(a->cg);
    a->gpb = (int)(up(up(G, a->nblk), unit) * unit);
    a->nblk = (int)up(G, a->gpb);
    const int R = 256 / (int)up(a->gpb * a->cg, 8);
    // up to 64 positions of a thread: about 512 workgroups, and about 2048 pieces (of all groups) of an image, which workgroups of the next launch join.  Larger images have more, as 64
    // positions are the most: one of 1048576 positions, 128 channels in 32 groups has 1024 pieces for each group, which every workgroup reads for its own: 211 us, 161 without them
    const long long per = std::max<long long>(1, std::min<long long>(MAX_ROWS, std::max(up(images * a->nblk * P, 512 * R), up(P * G, 2048 * R))));
    a->rows = (int)std::min<long long>(per * R, P);
    a->chunks = up(P, a->rows);
}
// y: vectors and positions of a workgroup: up to 16 positions a thread, about 1024 workgroups in all where x is small.
void cut_y(norm_args* a, bool token_major) {
    const int cvec = (int)up(a->C, 8);
    if (token_major) {
        a->vblk = (int)up(cvec, VECS);
        a->vecs = (int)up(cvec, a->vblk);
        const int R = 256 / a->vecs;
        a->y_rows = std::min<long long>(a->P, R * std::max<long long>(1, std::min<long long>(16, up(a->images * a->vblk * a->P, 1024 * R))));
    } else {
        a->vecs = std::min(cvec, 8);
        a->vblk = (int)up(cvec, a->vecs);
        a->y_rows = std::min<long long>(a->P, 64 * std::max<long long>(1, std::min<long long>(8, up(a->images * a->vblk * a->P, 1024 * 64))));
    }
    a->y_chunks = up(a->P, a->y_rows);
}

// One launch: the groups of a workgroup, 0 where it would hold too much.  As few as give every compute unit a workgroup, down to 16 bytes of a row (8 images of 1024 positions, 640
// channels in 32 groups, bf16: single groups, 40 bytes, 12.3 us, pairs on half of the compute units 13.8; fp32, whose rows a compute unit holds half as many of: down to 64 bytes
// in whole vectors, 15.7 us, single groups 17.6), and as few as the registers hold, down to 64 bytes.  Not where a thread would have many positions of less, or few workgroups
// many (4 images of 4096 positions, 320 channels: 19.8 us, by pieces 17.0; one of 714 positions, 4 groups of 73 channels: 16.1, by pieces 10.3).
template <typename X>
int one_launch(const norm_args& a, int T, int rows_of_thread) {
    int gpb = std::min(a.G, T * 8 / a.cg);
    if (gpb < 1 || a.P * a.ldx > INT32_MAX / 4) return 0;       // (places of an image in 32 bits)
    // whole vectors side by side where groups allow it
    const int unit = sizeof(X) == 4 && whole_groups(a.cg) <= gpb ? whole_groups(a.cg) : 1;
    auto rows_with = [&](int groups) { return up(a.P, T / up((long long)groups * a.cg, 8)); };
    auto run = [&](int groups) { return (long long)groups * a.cg * (int)sizeof(X); };
    while (gpb > unit) {
        const int fewer = std::max(unit, gpb / 2 / unit * unit);
        if (!(run(fewer) >= (sizeof(X) == 2 ? 16 : 64) && a.images * up(a.G, gpb) < CUS) && !(run(fewer) >= 64 && rows_with(gpb) > rows_of_thread)) break;
        gpb = fewer;
    }
    const long long rows = rows_with(gpb);
    return rows > rows_of_thread || (rows > 8 && (run(gpb) < 64 || a.images * up(a.G, gpb) < 32)) ? 0 : gpb;
}

template <typename K>
hipError_t launch(K kernel, long long items, int T, size_t lds, hipStream_t stream, const norm_args& a) {
    if (items > INT32_MAX) return hipErrorNotSupported;      // (kernels count in 32 bits)
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, dim3(grid_of(items)), dim3(T), lds, stream, a);
    return hipGetLastError();
}

template <typename X, bool CODES>
hipError_t rows_form(const norm_args& a, hipStream_t stream) {
    // (as many workgroups as the compute units hold at once, each with rows of its own)
    auto rows = [&](auto kernel, int T, long long workgroups, int at_once) { return launch(kernel, std::min<long long>(workgroups, at_once * CUS), T, 0, stream, a); };
    if (a.C <= 128) return rows(norm_rows_kernel<X, 16, 1, CODES>, 256, up(a.images, 16), 6);
    if (a.C <= 256) return rows(norm_rows_kernel<X, 32, 1, CODES>, 256, up(a.images, 8), 6);
    if (a.C <= 512) return rows(norm_rows_kernel<X, 64, 1, CODES>, 256, up(a.images, 4), 6);
    if (a.C <= 1024) return rows(norm_rows_kernel<X, 64, 2, CODES>, 256, up(a.images, 4), 4);
    if (a.C <= 2048) return rows(norm_rows_kernel<X, 256, 1, CODES>, 256, a.images, 6);
    if (a.C <= 4096) return rows(norm_rows_kernel<X, 256, 2, CODES>, 256, a.images, 4);
    if (a.C <= 8192) return rows(norm_rows_kernel<X, 512, 2, CODES>, 512, a.images, 2);
    return rows(norm_rows_kernel<X, 512, 4, CODES>, 512, a.images, 1);      // (1024 lanes of two vectors spill: 2048 rows of 16384 channels 56 us)
}

// LDS of workgroups of T threads with gpb groups each, the last of an image maybe fewer: that one has more rows of threads, and can have more pieces.
size_t groups_lds(const norm_args& a, int T) {
    auto bytes = [&](int groups) {
        const int cvec = (int)up((long long)groups * a.cg, 8);
        return norm_lds::bytes(groups, T / cvec, cvec);
    };
    return std::max(bytes(a.gpb), bytes(a.G - (a.nblk - 1) * a.gpb));
}

template <typename X>
hipError_t statistics(const norm_args& a, hipStream_t stream) {
    if (a.gpb == 0) return launch(norm_stats_wide_kernel<X>, a.images * a.G * a.chunks, 256, 0, stream, a);
    return launch(norm_stats_kernel<X>, a.images * a.nblk * a.chunks, 256, groups_lds(a, 256), stream, a);
}

template <typename X>
hipError_t norm(norm_args a, hipStream_t stream) {
    if (a.P == 1 && a.G == 1 && a.C <= 16384) return rows_form<X, false>(a, stream);
    for (int T : {64, 256, 512}) {
        // (small workgroups for whole small images, several for each compute unit: 2000 of 9 positions, 64 channels 5.9 us, 11.0 by larger ones)
        const int gpb = T > 64 || a.images > 512 ? one_launch<X>(a, T, T <= 256 ? 8 : 16) : 0;
        if (!gpb || (T == 64 && gpb < a.G)) continue;
        norm_args b = a;
        b.gpb = gpb, b.nblk = (int)up(a.G, gpb);
        const size_t lds = groups_lds(b, T);
        if (T == 64) return launch(norm_one_kernel<X, 64, 8>, b.images * b.nblk, T, lds, stream, b);
        return T == 256 ? launch(norm_one_kernel<X, 256, 8>, b.images * b.nblk, T, lds, stream, b) : launch(norm_one_kernel<X, 512, 16>, b.images * b.nblk, T, lds, stream, b);
    }
    const hipError_t e = statistics<X>(a, stream);
    if (e != hipSuccess) return e;
    cut_y(&a, a.token_major);
    const long long items = a.images * a.vblk * a.y_chunks;
    const size_t lds = 8 * ((size_t)std::min<long long>(a.G, a.vecs * 8) + 2) + (a.token_major ? 0 : 64 * 64 * 4);
    return a.token_major ? launch(norm_apply_kernel<X, true>, items, 256, lds, stream, a) : launch(norm_apply_kernel<X, false>, items, 256, lds, stream, a);
}
template <typename X>
hipError_t norm_codes(norm_args a, hipStream_t stream) {
    if (a.P == 1 && a.G == 1 && a.C <= 16384) return rows_form<X, true>(a, stream);
    const long long cvec = up(a.C, 8);
    // Whole images, positions of a thread at most 1, 4 or 8.  Against pieces, bf16: 49 positions of 512 channels, one image 9.8 us and 9.6, 2695 images 106 and 102; 40 of 400 in 4
    // groups 9.0 and 10.1, 91 and 107; 16 of 1280, which pieces read in rows of four wavefronts, 9.0 and 15.0, 96 and 190.
    size_t lds;
    auto whole_images = [&](int T, int NV) {
        const long long R = T / cvec, rows = R ? up(a.P, R) : NV + 1, pieces = sizeof(norm_piece) * R * (cvec + a.G);
        lds = 8 * (size_t)a.G + std::max<size_t>(pieces, 4 * ((size_t)NV * T + a.P));
        return rows <= NV && a.P * a.ldx <= INT32_MAX / 4 && lds <= 64 * 1024;
    };
    if (a.images > 512 && whole_images(64, 4)) return launch(norm_one_int8_kernel<X, 64, 4>, a.images, 64, lds, stream, a);
    if (whole_images(256, 4)) return launch(norm_one_int8_kernel<X, 256, 4>, a.images, 256, lds, stream, a);
    if (whole_images(512, 1)) return launch(norm_one_int8_kernel<X, 512, 1>, a.images, 512, lds, stream, a);
    if (whole_images(1024, 1)) return launch(norm_one_int8_kernel<X, 1024, 1>, a.images, 1024, lds, stream, a);
    if (whole_images(512, 8)) return launch(norm_one_int8_kernel<X, 512, 8>, a.images, 512, lds, stream, a);
    const hipError_t e = statistics<X>(a, stream);
    if (e != hipSuccess) return e;
    lds = 8 * (size_t)a.G;
    // up to 16 turns of a workgroup, about 512 workgroups: each joins the pieces of its image
    auto codes = [&](auto kernel, int positions) {
        a.y_rows = std::min<long long>(a.P, positions * std::max<long long>(1, std::min<long long>(16, up(a.images * a.P, 512 * positions))));
        a.y_chunks = up(a.P, a.y_rows);
        return launch(kernel, a.images * a.y_chunks, 256, lds, stream, a);
    };
    if (a.C <= 64) return codes(norm_int8_kernel<X, 8, 1>, 128);
    if (a.C <= 128) return codes(norm_int8_kernel<X, 16, 1>, 64);
    if (a.C <= 256) return codes(norm_int8_kernel<X, 32, 1>, 32);
    if (a.C <= 512) return codes(norm_int8_kernel<X, 64, 1>, 16);
    if (a.C <= 1024) return codes(norm_int8_kernel<X, 64, 2>, 8);
    if (a.C <= 2048) return codes(norm_int8_kernel<X, 256, 1>, 4);
    if (a.C <= 4096) return codes(norm_int8_kernel<X, 256, 2>, 2);
    a.y_rows = std::min<long long>(a.P, 4);
    a.y_chunks = up(a.P, a.y_rows);
    return launch(norm_int8_wide_kernel<X>, a.images * a.y_chunks, 256, lds, stream, a);
}

tsvd_status status_of(hipError_t e) { return e == hipSuccess ? TSVD_OK : e == hipErrorNotSupported ? TSVD_EUNSUPPORTED : TSVD_EDEVICE; }
bool bad_dtype(int t) { return t != TSVD_F32 && t != TSVD_BF16; }

tsvd_status common(const void* x, tsvd_dtype x_dtype, int64_t images, int64_t P, int64_t C, int64_t ldx, int64_t groups, const float* gamma, const float* beta, float eps,
                   tsvd_activation act, void* workspace, size_t workspace_bytes, norm_args* a) {
    if (!x || images < 1 || P < 1 || C < 1 || groups < 1 || bad_dtype(x_dtype) || ldx < C || !(eps > 0.f) || !std::isfinite(eps) || act < TSVD_ACT_NONE || act > TSVD_ACT_GELU)
        return TSVD_EINVAL;
    if (C % groups != 0) return TSVD_EINVAL;
    if (C > (1 << 20) || groups > MAX_GROUPS || images > INT32_MAX / P) return TSVD_EUNSUPPORTED;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < tsvd_group_norm_workspace_bytes(images, P, C, groups)) return TSVD_EINVAL;
    a->x = x, a->ldx = ldx;
    a->gamma = gamma, a->beta = beta, a->eps = eps, a->act = act;
    cut(images, P, (int)C, (int)groups, a);
    a->parts = static_cast<float4*>(workspace);
    return TSVD_OK;
}

}  // namespace

extern "C" size_t tsvd_group_norm_workspace_bytes(int64_t images, int64_t positions, int64_t C, int64_t groups) {
    if (images < 1 || positions < 1 || C < 1 || groups < 1 || C % groups != 0 || C > (1 << 20) || groups > MAX_GROUPS || images > INT32_MAX / positions) return 0;
    norm_args a = {};
    cut(images, positions, (int)C, (int)groups, &a);
    return round256((size_t)images * groups * a.chunks * sizeof(float4));
}

extern "C" tsvd_status tsvd_group_norm(const void* x_dev, tsvd_dtype x_dtype, int64_t images, int64_t positions, int64_t C, int64_t ldx, int64_t groups,
                                       const float* gamma_dev, const float* beta_dev, float eps, tsvd_activation act, void* y_dev, tsvd_dtype y_dtype,
                                       tsvd_layout y_layout, int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
    norm_args a = {};
    if (!y_dev || bad_dtype(y_dtype) || (y_layout != TSVD_FEATURE_MAJOR && y_layout != TSVD_TOKEN_MAJOR)) return TSVD_EINVAL;
    const tsvd_status st = common(x_dev, x_dtype, images, positions, C, ldx, groups, gamma_dev, beta_dev, eps, act, workspace, workspace_bytes, &a);
    if (st != TSVD_OK) return st;
    if (ldy < (y_layout == TSVD_TOKEN_MAJOR ? C : images * positions)) return TSVD_EINVAL;
    a.y = y_dev, a.ldy = ldy, a.out_bf16 = y_dtype == TSVD_BF16, a.token_major = y_layout == TSVD_TOKEN_MAJOR;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return status_of(x_dtype == TSVD_BF16 ? norm<uint16_t>(a, s) : norm<float>(a, s));
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
    return status_of(x_dtype == TSVD_BF16 ? norm_codes<uint16_t>(a, s) : norm_codes<float>(a, s));
}
