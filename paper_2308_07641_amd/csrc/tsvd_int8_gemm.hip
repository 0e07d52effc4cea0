// Products of 8-bit codes (include/tsvd_int8.h) for many tokens: y = (Q W^T) s t + bias on v_mfma_i32_32x32x32_i8, sums exact in int32.
//
// A workgroup of 2 x 2 wavefronts takes a tile of rows x tokens, a wavefront a quarter of it; both operands pass through LDS in stages of 128 indices of the
// contraction, moved there straight from memory (buffer_load ... lds) one stage or more ahead.
//
// Weights lie in tiles of 16 rows x 64 indices in operand order (tsvd_int8.h), and do so in LDS.  Codes of activations are rows: a request takes eight
// rows of 128 bytes, whole lines, piece c of row r to place c ^ (r & 7) of the row, so that the sixteen-byte reads of eight lanes (eight rows, one piece) hit all banks.
//
// The one barrier of a stage stands before its last quarter: by then a wavefront has read all that it needs of the stage, so the space may be
// filled again, and the first operands of the next stage are read behind it while the last quarter is multiplied.
#include "tsvd_int8.h"

#include <algorithm>
#include <type_traits>

#include "tsvd_epilogue.h"

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct gemm8_args {
    const uint8_t* tiles;
    int nkt;                      // tiles of a strip (even)
    int strips;
    const uint8_t* q;
    long long ldq;
    int N;
    const float *t, *s, *bias;
    void* y;
    long long ldy;
    long long M, B;
    int token_major, out_bf16;
    int row_tiles, token_tiles;
};

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

__device__ __forceinline__ void barrier() {
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Tile (row, token) of a workgroup: workgroups go round the XCDs, so each gets a run of the tiles, in bands of eight token tiles, rows outermost: what runs
// side by side on an XCD shares rows and tokens in its L2.
__device__ __forceinline__ void tile_of(const gemm8_args& p, int* row, int* token) {
    const int total = p.row_tiles * p.token_tiles, id = blockIdx.x, xcd = id & 7, each = total >> 3, more = total & 7;
    const int at = xcd * each + min(xcd, more) + (id >> 3);
    const int band = at / (8 * p.row_tiles), in = at - band * 8 * p.row_tiles, width = min(8, p.token_tiles - 8 * band);
    *row = in / width;
    *token = 8 * band + in % width;
}

// The results of a wavefront.  Sums go through LDS (of the wavefront's own) in pieces of 32 tokens (token-major y) or 32 rows, so that they leave 16 bytes a lane, whole lines at a time.
// A lane's result block: token r, rows 8 (v / 4) + 4 h + v % 4.
template <int RM, int RN, bool TOKENS>
__device__ __forceinline__ void store_tile(const gemm8_args& p, i32x16 (&acc)[RM][RN], uint8_t* smem, int row_of_tile, long long b0, int wm, int wn, int wave, int lane) {
    constexpr int WIDTH = 32 * (TOKENS ? RM : RN), PITCH = WIDTH + 4, OUTER = TOKENS ? RN : RM;
    const int r = lane & 31, h = lane >> 5;
    int* mine = reinterpret_cast<int*>(smem) + wave * 32 * PITCH;
    const int row0 = row_of_tile + wm * RM * 32;
    const long long token0 = b0 + wn * RN * 32;
    const int rows = (int)min((long long)RM * 32, p.M - row0), tokens = (int)min((long long)RN * 32, p.B - token0);       // (may be negative)
    auto pass = [&](auto wide) {
        constexpr int E = decltype(wide)::value;                 // values a lane stores at once: 16 bytes
        constexpr int LANES = WIDTH / E, STEP = 64 / LANES;
        const int at = lane % LANES * E, line0 = lane / LANES, valid = (TOKENS ? rows : tokens) - at;
        float along_t[E], along_b[E], along_s[E];                // what belongs to the lane's own values
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const bool there = e < valid;
            if (TOKENS) {
                along_t[e] = there ? p.t[row0 + at + e] : 0.f;
                along_b[e] = there && p.bias ? p.bias[row0 + at + e] : 0.f;
            } else {
                along_s[e] = there ? p.s[token0 + at + e] : 0.f;
            }
        }
#pragma unroll
        for (int o = 0; o < OUTER; ++o) {
#pragma unroll
            for (int i = 0; i < (TOKENS ? RM : RN); ++i) {
                const i32x16& d = acc[TOKENS ? i : o][TOKENS ? o : i];
#pragma unroll
                for (int v4 = 0; v4 < 4; ++v4) {
                    if (TOKENS) {
                        *reinterpret_cast<i32x4*>(mine + r * PITCH + i * 32 + 8 * v4 + 4 * h) = i32x4{d[4 * v4], d[4 * v4 + 1], d[4 * v4 + 2], d[4 * v4 + 3]};
                    } else {
#pragma unroll
                        for (int v = 0; v < 4; ++v) mine[(8 * v4 + 4 * h + v) * PITCH + i * 32 + r] = d[4 * v4 + v];
                    }
                }
            }
            __builtin_amdgcn_wave_barrier();
            const int lines = min(32, (TOKENS ? tokens : rows) - 32 * o);
            for (int line = line0; line < lines; line += STEP) {
                const long long outer = (TOKENS ? token0 : (long long)row0) + 32 * o + line;
                const float so = TOKENS ? p.s[outer] : p.t[outer], bo = TOKENS || !p.bias ? 0.f : p.bias[outer];
                float f[E];
#pragma unroll
                for (int e = 0; e < E; e += 4) {
                    const i32x4 d = *reinterpret_cast<const i32x4*>(mine + line * PITCH + at + e);
#pragma unroll
                    for (int k = 0; k < 4; ++k) f[e + k] = TOKENS ? int8_result(d[k], along_t[e + k], so, along_b[e + k]) : int8_result(d[k], so, along_s[e + k], bo);
                }
                const size_t to = (size_t)outer * p.ldy + (TOKENS ? (size_t)(row0 + at) : (size_t)(token0 + at));
                if (valid >= E) {
                    if constexpr (E == 8) {
                        typedef u32x4 u32x4_at __attribute__((aligned(2)));
                        *reinterpret_cast<u32x4_at*>(static_cast<uint16_t*>(p.y) + to) =
                            u32x4{tsvd_pack_bf16(f[0], f[1]), tsvd_pack_bf16(f[2], f[3]), tsvd_pack_bf16(f[4], f[5]), tsvd_pack_bf16(f[6], f[7])};
                    } else {
                        typedef f32x4 f32x4_at __attribute__((aligned(4)));
                        *reinterpret_cast<f32x4_at*>(static_cast<float*>(p.y) + to) = f32x4{f[0], f[1], f[2], f[3]};
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < E - 1; ++e)
                        if (e < valid) tsvd_store_y(p.y, to + e, f[e], E == 8);
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
    };
    if (p.out_bf16) pass(std::integral_constant<int, 8>());
    else pass(std::integral_constant<int, 4>());
}

// RM x RN blocks of 32 x 32 a wavefront, STAGES stages in LDS.
template <int RM, int RN, int STAGES>
__global__ void __launch_bounds__(256)
int8_gemm_kernel(gemm8_args p) {
    constexpr int BM = 64 * RM, BN = 64 * RN;
    constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128, STAGE = A_BYTES + B_BYTES;
    constexpr int A_LOADS = A_BYTES / 4096, B_LOADS = B_BYTES / 4096, LOADS = A_LOADS + B_LOADS;     // of a wavefront, for a stage
    constexpr int PART = (LOADS + 2 * RM - 1) / (2 * RM);        // ... requested beside one row of blocks, in the first two quarters
    extern __shared__ __align__(1024) uint8_t smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 31, h = lane >> 5, wm = wave & 1, wn = wave >> 1;
    int row_tile, token_tile;
    tile_of(p, &row_tile, &token_tile);
    const int strip0 = row_tile * (BM / 16), stages = p.nkt / 2;
    const long long b0 = (long long)token_tile * BN;
    const int tokens = (int)min((long long)BN, p.B - b0), strips = min(BM / 16, p.strips - strip0);

    // strips and tokens beyond the last are outside of the buffers: zeros
    const i32x4 wbuf = buffer_of(p.tiles + (size_t)strip0 * p.nkt * 1024, (uint32_t)strips * p.nkt * 1024);
    const i32x4 qbuf = buffer_of(p.q + b0 * p.ldq, (uint32_t)((tokens - 1) * p.ldq) + (uint32_t)((p.N + 15) & ~15));
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)smem;
    // a wavefront's loads of a stage: pieces wave, wave + 4 ... of the strips (two tiles each), rows 8 (wave + 4 j) ... of the codes
    int w_voff[A_LOADS], q_voff[B_LOADS];
#pragma unroll
    for (int j = 0; j < A_LOADS; ++j) w_voff[j] = ((wave + 4 * j) >> 1) * p.nkt * 1024 + ((wave + 4 * j) & 1) * 1024 + lane * 16;
#pragma unroll
    for (int j = 0; j < B_LOADS; ++j) q_voff[j] = (8 * (wave + 4 * j) + (lane >> 3)) * (int)p.ldq + ((lane & 7) ^ (lane >> 3)) * 16;
    // requests first ... of a stage's
    auto issue = [&](int stage, int slot, int first, int count) {
        const int k = min(stage, stages - 1) * 128;              // (behind the end: the last again, not used)
        const uint32_t lds = lds0 + slot * STAGE + wave * 1024;
#pragma unroll
        for (int j = first; j < first + count && j < LOADS; ++j) {
            if (j < A_LOADS) load_to_lds(wbuf, lds + j * 4096, w_voff[j], k * 16);
            else load_to_lds(qbuf, lds + j * 4096, q_voff[j - A_LOADS], k);
        }
    };
    // operands of quarter j of a stage
    const int a_at = ((wm * RM * 2 + (r >> 4)) * 2048) + (r & 15) * 16 + h * 256, b_at = A_BYTES + (wn * RN * 32 + r) * 128;
    i32x16 acc[RM][RN] = {};
    i32x4 w[2][RM], x[2][RN];
    // Reads the operands of quarter j of a stage into set `to`, multiplies set 1 - to, and requests a part of a later stage: in this order, and in pieces so that
    // the reads stand well before their use and the matrix unit has work between any two of the others.
    auto quarter = [&](int slot, int j, int to, bool multiply, int stage, int into, int first) {
        const uint8_t* base = smem + slot * STAGE;
        const int c = ((2 * j + h) ^ (r & 7)) * 16;
#pragma unroll
        for (int a = 0; a < RM; ++a) {
            if (a == 0) {
#pragma unroll
                for (int b = 0; b < RN; ++b) x[to][b] = *reinterpret_cast<const i32x4*>(base + b_at + b * 4096 + c);
                w[to][0] = *reinterpret_cast<const i32x4*>(base + a_at + j * 512);
            }
            if (a + 1 < RM) w[to][a + 1] = *reinterpret_cast<const i32x4*>(base + a_at + (a + 1) * 4096 + j * 512);
            if (first >= 0) issue(stage, into, first + a * PART, PART);
            if (multiply) {
#pragma unroll
                for (int b = 0; b < RN; ++b) acc[a][b] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[1 - to][a], x[1 - to][b], acc[a][b], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) issue(s, s, 0, LOADS);
    wait_vmcnt<(STAGES - 2) * LOADS>();
    barrier();
    quarter(0, 0, 0, false, 0, 0, -1);
    int slot = 0;
    for (int s = 0; s < stages; ++s) {
        const int last = slot == 0 ? STAGES - 1 : slot - 1, next = slot == STAGES - 1 ? 0 : slot + 1;
        quarter(slot, 1, 1, true, s + STAGES - 1, last, 0);
        quarter(slot, 2, 0, true, s + STAGES - 1, last, RM * PART);
        quarter(slot, 3, 1, true, 0, 0, -1);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // the stage is read
        wait_vmcnt<(STAGES - 2) * LOADS>();                      // ... and this wavefront's part of the next one is there
        barrier();
        quarter(next, 0, 0, true, 0, 0, -1);
        slot = next;
    }
    wait_vmcnt<0>();
    barrier();                                                   // (the stages' space is free)
    if (p.token_major) store_tile<RM, RN, true>(p, acc, smem, row_tile * BM, b0, wm, wn, wave, lane);
    else store_tile<RM, RN, false>(p, acc, smem, row_tile * BM, b0, wm, wn, wave, lane);
}

template <int RM, int RN, int STAGES>
hipError_t launch(gemm8_args a, hipStream_t stream) {
    constexpr int BM = 64 * RM, BN = 64 * RN, LDS = STAGES * (BM + BN) * 128;
    a.row_tiles = (int)((a.M + BM - 1) / BM);
    a.token_tiles = (int)((a.B + BN - 1) / BN);
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(int8_gemm_kernel<RM, RN, STAGES>), hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((int8_gemm_kernel<RM, RN, STAGES>), dim3((unsigned)(a.row_tiles * a.token_tiles)), dim3(256), LDS, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t tsvd_int8_gemm(const tsvd_int8_problem& p, hipStream_t stream) {
    const tsvd_int8_handle& h = *p.h;
    gemm8_args a = {};
    a.tiles = h.tiles(), a.nkt = h.nkt, a.strips = (int)h.strips, a.N = (int)h.N, a.t = h.scales(), a.M = h.M;
    a.q = reinterpret_cast<const uint8_t*>(p.codes), a.ldq = p.ldq, a.s = p.scales, a.B = p.B;
    a.bias = p.bias, a.y = p.y, a.ldy = p.ldy, a.token_major = p.token_major, a.out_bf16 = p.out_bf16;
    const long long big = ((h.M + 255) / 256) * ((p.B + 255) / 256), mid = ((h.M + 127) / 128) * ((p.B + 127) / 128);
    if (big >= h.cu_count) return launch<4, 4, 2>(a, stream);
    if (mid >= h.cu_count / 2) return launch<2, 2, 2>(a, stream);
    return launch<1, 1, 4>(a, stream);
}
