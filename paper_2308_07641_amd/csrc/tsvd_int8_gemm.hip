// Products of 8-bit codes (include/tsvd_int8.h) for many tokens: y = (Q W^T) s t + bias on v_mfma_i32_32x32x32_i8, sums exact in int32.
//
// A workgroup of 2 x 2 wavefronts takes a tile of rows x tokens, a wavefront a quarter of it, in stages of 128 indices of the contraction, each in four quarters of one matrix
// instruction a block.  Codes of activations pass through LDS, moved there straight from memory (buffer_load ... lds) several stages ahead: a request takes eight rows of 128
// bytes, whole lines, piece c of row r to place c ^ (r & 7) of the row, so that the sixteen-byte reads of eight lanes (eight rows, one piece) hit all banks.  Weights lie in memory in
// operand order (tsvd_int8.h); tiles of 128 rows and more load them into registers, one or two stages ahead, which halves what LDS has to pass (256 x 256 with both
// operands through LDS: 0.66 ms against 0.60 for 36864 x 9216 at 2048 tokens); the 64 x 64 tile, bound by latency, takes both through LDS.
//
// The one barrier of a stage stands before its last quarter: by then a wavefront has read all that it needs of the stage, so the space may be filled again, and the first operands of the
// next stage are read behind it while the last quarter is multiplied.
//
// What bounds it: with these operands the matrix unit alone, fed from registers, reaches 3.4e15 operations a second (5.0e15 with zeros: the clock follows the power), 36864 x 9216 at 2048
// tokens runs at 2.2e15 to 2.35e15, by the card; half the compute units busy run at the higher clock, so a last round that is half empty costs little.
#include "tsvd_int8.h"

#include <algorithm>
#include <type_traits>
#include <utility>

#include "tsvd_epilogue.h"
#include "tsvd_kernels.h"

namespace {

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

// body(0), ..., body(N - 1), each with a constant of its own: a loop that the compiler does not unroll would move all results through one another's registers.
template <typename F, int... I>
__device__ __forceinline__ void each(F&& body, std::integer_sequence<int, I...>) { (body(std::integral_constant<int, I>()), ...); }
template <int N, typename F>
__device__ __forceinline__ void each(F&& body) { each(body, std::make_integer_sequence<int, N>()); }

// Token-major results of a wavefront of up to four blocks, from its registers: of a block a lane holds token r, rows 8 v4 + 4 h + v: four rows side by side, in bf16 eight after the two
// halves of the wavefront have swapped (16 bytes either way).
template <int RM, int RN>
__device__ __forceinline__ void store_registers(const gemm8_args& p, i32x16 (&acc)[RM][RN], const float2* row_of, const float (&token_scale)[RN], int row0, long long token0, int lane) {
    const int r = lane & 31, h = lane >> 5, M = (int)p.M, B = (int)p.B;
    each<RM>([&](auto a) {
        float2 own[16];                                          // scale and bias
#pragma unroll
        for (int v = 0; v < 16; ++v) own[v] = row_of[a * 32 + 8 * (v >> 2) + 4 * h + (v & 3)];
        const int row = row0 + a * 32;
        each<RN>([&](auto b) {
            const int token = (int)token0 + b * 32 + r;
            float f[16];
#pragma unroll
            for (int v = 0; v < 16; ++v) f[v] = int8_result(acc[a][b][v], own[v].x, token_scale[b], own[v].y);
            if (p.out_bf16) {
#pragma unroll
                for (int v = 0; v < 4; v += 2) {
                    uint32_t d[2][2];
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        const auto two = __builtin_amdgcn_permlane32_swap(tsvd_pack_bf16(f[4 * v + 2 * w], f[4 * v + 2 * w + 1]), tsvd_pack_bf16(f[4 * v + 4 + 2 * w], f[4 * v + 5 + 2 * w]), false, false);
                        d[0][w] = two[0], d[1][w] = two[1];
                    }
                    const int at = row + 8 * (v + h);
                    uint16_t* to = static_cast<uint16_t*>(p.y) + (size_t)token * p.ldy + at;
                    if (token < B && at + 8 <= M) {
                        typedef u32x4 u32x4_at __attribute__((aligned(2)));
                        *reinterpret_cast<u32x4_at*>(to) = u32x4{d[0][0], d[0][1], d[1][0], d[1][1]};
                    } else if (token < B) {
#pragma unroll
                        for (int e = 0; e < 7; ++e)
                            if (at + e < M) to[e] = (uint16_t)(d[e >> 2][e >> 1 & 1] >> (16 * (e & 1)));
                    }
                }
            } else {
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const int at = row + 8 * v + 4 * h;
                    float* to = static_cast<float*>(p.y) + (size_t)token * p.ldy + at;
                    if (token < B && at + 4 <= M) {
                        typedef f32x4 f32x4_at __attribute__((aligned(4)));
                        *reinterpret_cast<f32x4_at*>(to) = f32x4{f[4 * v], f[4 * v + 1], f[4 * v + 2], f[4 * v + 3]};
                    } else if (token < B) {
#pragma unroll
                        for (int e = 0; e < 3; ++e)
                            if (at + e < M) to[e] = f[4 * v + e];
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);                   // (one block at a time: else the registers do not suffice)
        });
    });
}
// Results of a wavefront by way of LDS (of its own), in pieces of 32 tokens (token-major y) or 32 rows, so that they leave 16 bytes a lane, whole lines at a time, and the code stays
// short: larger tiles from registers, block by block, are some thousand instructions that every tile fetches anew (256 x 256: 9 us against 6).
template <int RM, int RN>
constexpr int store_bytes() { return 32 * (32 * (RM > RN ? RM : RN) + 4) * 4; }      // for a wavefront
template <int RM, int RN, bool TOKENS>
__device__ __forceinline__ void store_lds(const gemm8_args& p, i32x16 (&acc)[RM][RN], int* mine, const float2* row_of, const float* token_of, int row0, long long token0, int lane) {
    constexpr int WIDTH = 32 * (TOKENS ? RM : RN), PITCH = WIDTH + 4, OUTER = TOKENS ? RN : RM;
    const int r = lane & 31, h = lane >> 5;
    const int rows = (int)min((long long)RM * 32, p.M - row0), tokens = (int)min((long long)RN * 32, p.B - token0);       // (may be negative)
    const int outers = TOKENS ? tokens : rows, inners = TOKENS ? rows : tokens;
    if (outers <= 0 || inners <= 0) return;
    auto pass = [&](auto wide) {
        constexpr int E = decltype(wide)::value;                 // values a lane stores at once: 16 bytes
        constexpr int LANES = WIDTH / E, STEP = 64 / LANES;
        const int at = lane % LANES * E, line0 = lane / LANES, valid = inners - at;
        float scale[E], bias[E];                                 // of the lane's own values
#pragma unroll
        for (int e = 0; e < E; ++e) {
            scale[e] = TOKENS ? row_of[at + e].x : token_of[at + e];
            bias[e] = TOKENS ? row_of[at + e].y : 0.f;
        }
        const size_t step = (size_t)STEP * p.ldy;
        size_t to = TOKENS ? (size_t)(token0 + line0) * p.ldy + row0 + at : (size_t)(row0 + line0) * p.ldy + token0 + at;
        each<OUTER>([&](auto o) {
            each<(TOKENS ? RM : RN)>([&](auto i) {
                const i32x16& d = acc[TOKENS ? (int)i : (int)o][TOKENS ? (int)o : (int)i];
#pragma unroll
                for (int v4 = 0; v4 < 4; ++v4) {
                    if (TOKENS) {
                        *reinterpret_cast<i32x4*>(mine + r * PITCH + i * 32 + 8 * v4 + 4 * h) = i32x4{d[4 * v4], d[4 * v4 + 1], d[4 * v4 + 2], d[4 * v4 + 3]};
                    } else {
#pragma unroll
                        for (int v = 0; v < 4; ++v) mine[(8 * v4 + 4 * h + v) * PITCH + i * 32 + r] = d[4 * v4 + v];
                    }
                }
            });
            __builtin_amdgcn_wave_barrier();
#pragma unroll 2
            for (int line = line0; line < 32; line += STEP, to += step) {
                const float2 own = TOKENS ? float2{token_of[32 * o + line], 0.f} : row_of[32 * o + line];
                float f[E];
#pragma unroll
                for (int e = 0; e < E; e += 4) {
                    const i32x4 d = *reinterpret_cast<const i32x4*>(mine + line * PITCH + at + e);
#pragma unroll
                    for (int k = 0; k < 4; ++k) f[e + k] = TOKENS ? int8_result(d[k], scale[e + k], own.x, bias[e + k]) : int8_result(d[k], own.x, scale[e + k], own.y);
                }
                if (32 * o + line >= outers) continue;
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
        });
    };
    if (p.out_bf16) pass(std::integral_constant<int, 8>());
    else pass(std::integral_constant<int, 4>());
}
// What a thread keeps for it from the start, and the end of a tile.
template <int RM, int RN>
struct tile_scales {
    float2 row[(RM + 3) / 4];
    float token[RN];
    __device__ __forceinline__ void load(const gemm8_args& p, int row0, long long token0, int lane) {
#pragma unroll
        for (int i = 0; i < (RM + 3) / 4; ++i) {
            const int at = min(row0 + (int)threadIdx.x + 256 * i, (int)p.M - 1);
            row[i] = float2{p.t[at], p.bias ? p.bias[at] : 0.f};
        }
#pragma unroll
        for (int b = 0; b < RN; ++b) token[b] = p.s[min(token0 + b * 32 + (lane & 31), p.B - 1)];
    }
};
template <int RM, int RN>
constexpr int finish_bytes() { return 64 * RM * 8 + 64 * RN * 4 + 4 * store_bytes<RM, RN>(); }
template <int RM, int RN>
__device__ __forceinline__ void finish_tile(const gemm8_args& p, i32x16 (&acc)[RM][RN], const tile_scales<RM, RN>& scales, uint8_t* smem, int row0, long long token0, int wm, int wn, int wave, int lane) {
    wait_vmcnt<0>();
    barrier();                                                   // (the stages' space is free)
    float2* row_of = reinterpret_cast<float2*>(smem);
    float* token_of = reinterpret_cast<float*>(smem + 64 * RM * 8);
#pragma unroll
    for (int i = 0; i < (RM + 3) / 4; ++i)
        if ((int)threadIdx.x + 256 * i < 64 * RM) row_of[threadIdx.x + 256 * i] = scales.row[i];
    if (wm == 0 && lane < 32)
#pragma unroll
        for (int b = 0; b < RN; ++b) token_of[wn * RN * 32 + b * 32 + lane] = scales.token[b];
    __syncthreads();
    row_of += wm * RM * 32;
    token_of += wn * RN * 32;
    row0 += wm * RM * 32;
    int* mine = reinterpret_cast<int*>(smem + 64 * RM * 8 + 64 * RN * 4 + wave * store_bytes<RM, RN>());
    if (!p.token_major) store_lds<RM, RN, false>(p, acc, mine, row_of, token_of, row0, token0, lane);
    else if constexpr (RM * RN <= 4) store_registers<RM, RN>(p, acc, row_of, scales.token, row0, token0, lane);
    else store_lds<RM, RN, true>(p, acc, mine, row_of, token_of, row0, token0, lane);
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
    tile_scales<RM, RN> scales;
    scales.load(p, row_tile * BM, b0 + wn * RN * 32, lane);

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
    finish_tile<RM, RN>(p, acc, scales, smem, row_tile * BM, b0 + wn * RN * 32, wm, wn, wave, lane);
}

// RM x RN blocks of 32 x 32 a wavefront, STAGES stages of the activations' codes in LDS, RING quarters of the weights' in registers (4 or 8).
template <int RM, int RN, int STAGES, int RING>
__global__ void __launch_bounds__(256)
int8_gemm_direct_kernel(gemm8_args p) {
    constexpr int BM = 64 * RM, BN = 64 * RN, STAGE = BN * 128;
    constexpr int LOADS = STAGE / 4096, PART = (LOADS + 3) / 4;      // of a wavefront, for a stage; beside one quarter
    // Requests that follow the last one of a stage's codes, at least, when they are waited for one barrier ahead (they are requested STAGES - 1 stages ahead, a part in each
    // quarter, and results come in the order of the requests): those of STAGES - 3 whole stages and of three quarters of one.
    constexpr int NEWER = (STAGES - 3) * (4 * RM + LOADS) + 3 * RM + (3 * PART < LOADS ? 3 * PART : LOADS);
    static_assert(STAGES >= 3 && NEWER <= 63 && RING >= 4 * (STAGES - 3) && (RING == 4 || RING == 8), "what the first stages' waits count on");
    extern __shared__ __align__(1024) uint8_t smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 31, h = lane >> 5, wm = wave & 1, wn = wave >> 1;
    int row_tile, token_tile;
    tile_of(p, &row_tile, &token_tile);
    const int strip0 = row_tile * (BM / 16), stages = p.nkt / 2;
    const long long b0 = (long long)token_tile * BN;
    const int tokens = (int)min((long long)BN, p.B - b0), strips = min(BM / 16, p.strips - strip0);
    tile_scales<RM, RN> scales;
    scales.load(p, row_tile * BM, b0 + wn * RN * 32, lane);

    // strips and tokens beyond the last are outside of the buffers: zeros
    const uint32_t w_bytes = (uint32_t)strips * p.nkt * 1024;
    const __amdgpu_buffer_rsrc_t wbuf = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p.tiles + (size_t)strip0 * p.nkt * 1024), 0, w_bytes, 0x00020000);
    const i32x4 qbuf = buffer_of(p.q + b0 * p.ldq, (uint32_t)((tokens - 1) * p.ldq) + (uint32_t)((p.N + 15) & ~15));
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)smem;
    int w_voff[RM], q_voff[LOADS];
#pragma unroll
    for (int a = 0; a < RM; ++a) w_voff[a] = ((wm * RM + a) * 2 + (r >> 4)) * p.nkt * 1024 + (r & 15) * 16 + h * 256;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) q_voff[j] = (8 * (wave + 4 * j) + (lane >> 3)) * (int)p.ldq + ((lane & 7) ^ (lane >> 3)) * 16;
    auto issue = [&](int stage, int slot, int first, int count) {
        const int k = min(stage, stages - 1) * 128;              // (behind the end: the last again, not used)
        const uint32_t lds = lds0 + slot * STAGE + wave * 1024;
#pragma unroll
        for (int j = first; j < first + count && j < LOADS; ++j) load_to_lds(qbuf, lds + j * 4096, q_voff[j], k);
    };
    i32x4 w[RING][RM], x[2][RN];
    // quarter j of a stage of the weights: row block a  (behind the end: zeros)
    auto load_w = [&](int stage, int j, int a) {
        const int at = stage < stages ? (2 * stage + (j >> 1)) * 1024 + (j & 1) * 512 : (int)w_bytes;
        return __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(wbuf, w_voff[a], at, 0));
    };
    const int b_at = (wn * RN * 32 + r) * 128;
    auto read_x = [&](int slot, int j, int to) {
        const int c = ((2 * j + h) ^ (r & 7)) * 16;
#pragma unroll
        for (int b = 0; b < RN; ++b) x[to][b] = *reinterpret_cast<const i32x4*>(smem + slot * STAGE + b_at + b * 4096 + c);
    };
    i32x16 acc[RM][RN] = {};
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) issue(s, s, 0, LOADS);
#pragma unroll
    for (int n = 0; n < RING; ++n)
#pragma unroll
        for (int a = 0; a < RM; ++a) w[n][a] = load_w(n >> 2, n & 3, a);
    // (the weights' loads were requested last: all that came before them is there when RING RM are left)
    wait_vmcnt<(RING * RM < 63 ? RING * RM : 63)>();
    barrier();
    read_x(0, 0, 0);
    int slot = 0;
    for (int s0 = 0; s0 < stages; s0 += RING / 4) {
#pragma unroll
        for (int u = 0; u < RING / 4; ++u) {
            const int s = s0 + u;                                // (behind the end: weights of zero)
            const int last = slot == 0 ? STAGES - 1 : slot - 1, next = slot == STAGES - 1 ? 0 : slot + 1;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int n = 4 * u + j;
                if (j == 3) {
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // the stage is read
                    wait_vmcnt<NEWER>();                                     // ... and this wavefront's part of the next one is there
                    barrier();
                    read_x(next, 0, 0);
                } else {
                    read_x(slot, j + 1, (j + 1) & 1);
                }
                // (the space of the stage before is free since the barrier in its last quarter)
                issue(s + STAGES - 1, last, j * PART, PART);
#pragma unroll
                for (int a = 0; a < RM; ++a) {
#pragma unroll
                    for (int b = 0; b < RN; ++b) acc[a][b] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[n][a], x[j & 1][b], acc[a][b], 0, 0, 0);
                    w[n][a] = load_w(s + RING / 4, j, a);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            slot = next;
        }
    }
    finish_tile<RM, RN>(p, acc, scales, smem, row_tile * BM, b0 + wn * RN * 32, wm, wn, wave, lane);
}
// A launch of one kind of tile.  DIRECT: RING quarters of the weights in registers, else (RING = 0) through LDS.
template <int RM, int RN, int STAGES, int RING>
constexpr int lds_bytes() { return std::max(STAGES * 64 * (RING ? RN : RM + RN) * 128, finish_bytes<RM, RN>()); }
template <int RM, int RN, int STAGES, int RING>
const void* kernel_of() {
    if constexpr (RING > 0) return reinterpret_cast<const void*>(int8_gemm_direct_kernel<RM, RN, STAGES, RING>);
    else return reinterpret_cast<const void*>(int8_gemm_kernel<RM, RN, STAGES>);
}
template <int RM, int RN, int STAGES, int RING>
hipError_t launch(gemm8_args a, hipStream_t stream) {
    a.row_tiles = (int)((a.M + 64 * RM - 1) / (64 * RM));
    a.token_tiles = (int)((a.B + 64 * RN - 1) / (64 * RN));
    if ((long long)a.row_tiles * a.token_tiles > 1 << 23) return hipErrorNotSupported;       // (a grid counts its threads in 32 bits)
    void* args[] = {&a};
    return hipLaunchKernel(kernel_of<RM, RN, STAGES, RING>(), dim3((unsigned)(a.row_tiles * a.token_tiles)), dim3(256), args, lds_bytes<RM, RN, STAGES, RING>(), stream);
}
template <int RM, int RN, int STAGES, int RING>
hipError_t allow() {
    return hipFuncSetAttribute(kernel_of<RM, RN, STAGES, RING>(), hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes<RM, RN, STAGES, RING>());
}

// The tiles, and what one takes a compute unit (us, all of them busy): to begin and store it (bf16, fp32), for each stage of 128 indices.  Fitted to the times of all five kinds on
// 256 CUs for 170 sizes (64 to 40000 rows, 64 to 16384 features, 65 to 16384 tokens, both types and layouts): the kind that they choose takes 0.4% longer than the quickest, in the
// mean, and 16% at most.  Two workgroups of a compute unit take twice as long as one, so only the number of tiles for each counts.
enum { TILE_64 = 1, TILE_128x64, TILE_128, TILE_256x128, TILE_256 };
constexpr struct {
    int rows, tokens;
    double begin, begin_f32, stage;
} tile_costs[] = {{}, {64, 64, 0.44, 0.67, 0.19}, {128, 64, 2.3, 2.3, 0.33}, {128, 128, 2.1, 2.7, 0.44}, {256, 128, 9.2, 9.9, 0.7}, {256, 256, 6.3, 11.1, 1.32}};

long long up(long long v, long long m) { return (v + m - 1) / m; }
hipError_t launch(int tile, const gemm8_args& a, int cus, hipStream_t stream) {
    switch (tile) {
        // (two stages let five workgroups share a compute unit, four hide more of one's latency: 104576 tokens, 273 rows of 128 features 30 us and 43; 696 tokens, 320 rows of 15296
        // 60 us and 26)
        case TILE_64: return up(a.M, 64) * up(a.B, 64) > cus ? launch<1, 1, 2, 0>(a, stream) : launch<1, 1, 4, 0>(a, stream);
        case TILE_128x64: return launch<2, 1, 4, 8>(a, stream);
        case TILE_128: return launch<2, 2, 4, 8>(a, stream);
        case TILE_256x128: return launch<4, 2, 4, 8>(a, stream);
        case TILE_256: return launch<4, 4, 4, 4>(a, stream);
    }
    return hipErrorInvalidValue;
}
// The kind that takes the least time by these figures.
int cheapest(long long rows, long long B, int stages, bool f32, int cus) {
    int best = 0;
    double least = 0;
    for (int t = TILE_64; t <= TILE_256; ++t) {
        const auto& c = tile_costs[t];
        const double cost = (double)up(up(rows, c.rows) * up(B, c.tokens), cus) * ((f32 ? c.begin_f32 : c.begin) + c.stage * stages);
        if (!best || cost < least) best = t, least = cost;
    }
    return best;
}

}  // namespace

hipError_t tsvd_int8_gemm_init() {
    hipError_t e = allow<1, 1, 2, 0>();
    if (e == hipSuccess) e = allow<1, 1, 4, 0>();
    if (e == hipSuccess) e = allow<2, 1, 4, 8>();
    if (e == hipSuccess) e = allow<2, 2, 4, 8>();
    if (e == hipSuccess) e = allow<4, 2, 4, 8>();
    if (e == hipSuccess) e = allow<4, 4, 4, 4>();
    return e;
}

hipError_t tsvd_int8_gemm(const tsvd_int8_problem& p, hipStream_t stream) {
    const tsvd_int8_handle& h = *p.h;
    gemm8_args a = {};
    a.tiles = h.tiles(), a.nkt = h.nkt, a.strips = (int)h.strips, a.N = (int)h.N, a.t = h.scales(), a.M = h.M;
    a.q = reinterpret_cast<const uint8_t*>(p.codes), a.ldq = p.ldq, a.s = p.scales, a.B = p.B;
    a.bias = p.bias, a.y = p.y, a.ldy = p.ldy, a.token_major = p.token_major, a.out_bf16 = p.out_bf16;
    return launch(tsvd_tune("TSVD_INT8_TILE", cheapest(h.M, p.B, h.nkt / 2, !p.out_bf16, h.cu_count)), a, h.cu_count, stream);
}
