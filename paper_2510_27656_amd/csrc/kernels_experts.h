// The experts' products on expert-major rows (gfx950 only): h = act(x Wg^T) * (x Wu^T), y = x W^T, their gradients,
// and both in e4m3 blocks of 128.
//
// One kernel walks tiles of (expert, rows of the expert, features of its output): how many rows an expert has is only
// known on the device, so every workgroup scans the counts once and takes every gridDim-th tile.
// A tile is a matrix product of two operands staged through LDS 128 bytes of the contraction at a time:
//   A: the features (weights, or for the weight gradient the columns of x) on the matrix instructions' rows,
//   B: the expert's rows (or for the weight gradient the columns of the output's gradient) on their columns,
// so that a lane holds four consecutive features of one row.  An operand whose memory is contiguous along the contraction
// is read from LDS as it lies; one that is contiguous along the features is transposed on its way into registers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/flmoe.h"

namespace flmoe {
namespace experts {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef unsigned v2u __attribute__((ext_vector_type(2)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));

constexpr int kWave = 64;
constexpr int kMaxExperts = FL_MAX_EXPERTS;

// The experts of a call and where their rows lie.
struct Groups {
    int El, first, n;              // local experts of a rank; first expert of the call and how many
    long long cap;                 // rows of a rank
    const int *expert_off;         // [N][El+1]
    const int *counts;             // [N][El]
};
struct Rows {
    long long first;               // among all ranks' rows
    int n;
};
// Rows of expert e; whatever the tables hold, none outside its rank's.
__device__ inline Rows rows_of(const Groups &G, int e) {
    const int d = e / G.El, j = e - d * G.El;
    const long long off = G.expert_off[(size_t)d * (G.El + 1) + j];
    long long n = G.counts[e];
    if (off < 0 || off >= G.cap || n < 0) n = 0;
    else if (n > G.cap - off) n = G.cap - off;
    return {n ? (long long)d * G.cap + off : 0, (int)n};
}

// A value that is the same in all lanes, in scalar registers.
__device__ inline long long same_in_wave(long long v) {
    const unsigned lo = __builtin_amdgcn_readfirstlane((int)(unsigned)v), hi = __builtin_amdgcn_readfirstlane((int)(v >> 32));
    return (long long)((unsigned long long)hi << 32 | lo);
}

// ---------------------------------------------------------------- numbers
__device__ inline float from_bf16(unsigned bits) { return __uint_as_float(bits << 16); }
__device__ inline unsigned to_bf16(float f) {
    unsigned u = __float_as_uint(f);
    if ((u & 0x7fffffffu) > 0x7f800000u) return (u >> 16) | 0x40u;      // NaN stays a quiet NaN
    return (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;                      // ties to even
}
__device__ inline unsigned to_bf16x2(float lo, float hi) { return to_bf16(lo) | to_bf16(hi) << 16; }

// silu(v) = v s, s = 1 / (1 + e^-v); gelu(v) = v s with s = 1 / (1 + e^(-2 a (v + 0.044715 v^3))), a = sqrt(2 / pi), which
// is the tanh form.  *slope receives the derivative; where s has reached 0 or 1 its own derivative is 0, whatever v.
constexpr float kGelu = 1.5957691216057308f;                            // 2 sqrt(2 / pi)
template <bool SLOPE>
__device__ inline float activate(int act, float v, float *slope) {
    const float arg = act == FL_ACT_SILU ? v : kGelu * (v + 0.044715f * v * v * v);
    const float s = 1.0f / (1.0f + __expf(-arg));
    if (SLOPE) {
        const float ds = s * (1.0f - s), inner = act == FL_ACT_SILU ? v : kGelu * (v + 3.0f * 0.044715f * v * v * v);
        *slope = ds == 0.0f ? s : s + inner * ds;
    }
    return v * s;
}

// Codes of four values of an e4m3 block (see FL_DTYPE_E4M3_BLOCK128): rounded to nearest even, saturating; what is NaN
// over the scale (a NaN, or an Inf in a block whose scale it made infinite) becomes the NaN code with the value's sign.
__device__ inline float block_scale(float amax) { return amax == 0.0f ? 1.0f : __fdiv_rn(amax, 448.0f); }
__device__ inline unsigned e4m3_codes(const float *v, float scale) {
    float q[4];
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        q[i] = __fdiv_rn(v[i], scale);
        odd |= q[i] != q[i];
        q[i] = fabsf(q[i]) >= 448.0f ? copysignf(448.0f, q[i]) : q[i];
    }
    unsigned w = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
    w = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], (int)w, true);
    if (odd) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (q[i] != q[i]) w = (w & ~(0xffu << (8 * i))) | ((__float_as_uint(v[i]) >> 24 & 0x80u) | 0x7fu) << (8 * i);
    }
    return w;
}

// ---------------------------------------------------------------- memory
// A lane's 16 (or 4) bytes straight into LDS, at the wave's place there plus 16 (4) times the lane.  Offsets of kNowhere
// read as zero; only offsets inside the tensor or kNowhere are ever passed, the limit is the largest there is.  Written
// out because the compiler, which knows that these loads write LDS, lets every read of LDS behind them wait for them:
// here the waits are the ones below, once per step.  Nothing is returned, so no register is written behind its back.
// (One wait state lies between a write of m0 and a load that goes by it.)
#define FLMOE_LDS __attribute__((address_space(3)))
constexpr unsigned kNowhere = 0x80000000u;
struct Window {
    v4u rsrc;
    __device__ explicit Window(const char *base) {
        const unsigned long long at = (unsigned long long)base;
        rsrc = v4u{(unsigned)at, (unsigned)(at >> 32) & 0xffffu, 0x7FFFFFFFu, 0x00020000u};
    }
};
__device__ inline unsigned lds_address(const char *lds) { return (unsigned)(uintptr_t)(FLMOE_LDS const char *)lds; }
__device__ inline void to_lds_16(const Window &w, unsigned offset, unsigned shift, unsigned lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 ::"s"(lds), "v"(offset), "s"(w.rsrc), "s"(shift) : "memory");
}
__device__ inline void to_lds_4(const Window &w, unsigned offset, unsigned shift, unsigned lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds"
                 ::"s"(lds), "v"(offset), "s"(w.rsrc), "s"(shift) : "memory");
}
// Every load of this wave but the last KEEP is done, and so is every wave's, and its reads of LDS, behind the barrier.
template <int KEEP>
__device__ inline void loads_done_and_barrier() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(KEEP) : "memory");
}

// ---------------------------------------------------------------- the tiles' geometry
constexpr int kThreads = 512, kWaves = kThreads / kWave;
constexpr int kStep = 128;                     // bytes of the contraction per step: 64 bf16, 128 e4m3 (one block of scales)
constexpr int kFeatures = 256;                 // features of a tile; gated: 128 gates and the 128 ups that belong to them
constexpr int kHalf = 128;                     // features that are written out together
constexpr int kEmitPitch = kHalf + 4;          // floats from row to row of the tile's output in LDS

enum Form { kForward, kRowGradient, kWeightGradient };

struct Product {
    const char *a, *b;
    long long a_expert;            // bytes from expert to expert of the weights
    int a_ld, b_ld;                // bytes from row to row
    int features, other, k;        // output features; weight gradient: columns of the other operand; contraction (not there)
    const float *a_scales, *b_scales;
    void *out;
    float *out_scales;             // e4m3 blocks out
    void *pre;                     // gated: the pre-activations, kept for the backward pass, or null
    float *pre_scales;             // ... in e4m3 blocks, or null: bf16
    int act;
};

// Place of a 16-byte chunk in a staged operand, so that the lanes that are served together fall into different banks
// (64 of 4 bytes; sixteen lanes of a 16-byte read, 32 of an 8-byte one).
// Contiguous along the contraction: rows of 128 bytes, chunk c of row r at c ^ (r >> 1 & 7): two rows fill the banks once.
// Contiguous along the features: 64 contraction rows of 512 bytes, chunk c of row r at c ^ (r & 3) << 2: the transposing
// reads take 64 bytes each of four rows at once.
__device__ inline int swizzle(int row) { return row >> 1 & 7; }
__device__ inline int spread(int row) { return (row & 3) << 2; }

// Four rows of the contraction for one feature per lane: lanes 16 i .. 16 i + 15 give the places of four rows by four
// chunks of 8 bytes, and lane j of them receives column j.
__device__ inline v4s read_transposed(const char *lds, int row, int feature) {
    const int l = threadIdx.x & 15;
    const int r = row + (l >> 2), c = (feature >> 3) + (l >> 1 & 1);
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((FLMOE_LDS v4s *)(lds + r * 512 + ((c ^ spread(r)) << 4) + (l & 1) * 8));
}

template <int FORM, bool E4M3, bool GATED, int ROWS, int STAGES>
struct Tile {
    static constexpr bool kTransA = FORM != kForward, kTransB = FORM == kWeightGradient;
    static constexpr int kWavesF = ROWS == 256 ? 2 : 4, kWavesR = kWaves / kWavesF;
    static constexpr int kSide = E4M3 ? 16 : 32;                       // of a matrix instruction's output
    static constexpr int kFragsF = kFeatures / kWavesF / kSide, kFragsR = ROWS / kWavesR / kSide;
    static constexpr int kBytesA = kFeatures * kStep, kBytesB = ROWS * kStep, kBytesS = E4M3 ? ROWS * 4 : 0;
    static constexpr int kStage = kBytesA + kBytesB + kBytesS;
    static constexpr int kEmit = ROWS * kEmitPitch * 4;
    static constexpr int kLds = STAGES * kStage > kEmit ? STAGES * kStage : kEmit;
    static constexpr int kOutput = GATED ? kHalf : kFeatures;          // output features of a tile
    static constexpr int kLoadsA = kBytesA / 1024 / kWaves, kLoadsB = kBytesB / 1024 / kWaves;
    static_assert(!kTransB || ROWS == 256, "transposed operands are 256 wide");
    using Acc = typename std::conditional<E4M3, v4f, v16f>::type;
    static constexpr int kAccs = E4M3 ? 4 : 16;

    // First feature, of the staged 256, of fragment i of this wave.
    __device__ static int frag_feature(int wf, int i) {
        if (!GATED) return (wf * kFragsF + i) * kSide;
        return (i < kFragsF / 2 ? 0 : kHalf) + (wf * (kFragsF / 2) + i % (kFragsF / 2)) * kSide;
    }

    // e: expert; first, n: its rows; f0: first output feature; r0: first row (weight gradient: first column of b).
    __device__ static void run(const Product &P, char *lds, int e, const Rows &rows, int f0, int r0) {
        const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
        const int wf = wave % kWavesF, wr = wave / kWavesF;
        const int size = E4M3 ? 1 : 2;
        const int k = FORM == kWeightGradient ? rows.n : P.k;          // contraction
        const int n_b = FORM == kWeightGradient ? P.other : rows.n;    // rows of operand b
        const int steps = (k * (long long)size + kStep - 1) / kStep;

        // where this lane's chunks come from: offsets inside the operands, places that must not be past the end
        const char *a0, *a1, *b0;                                      // a1: ups of a gated tile
        unsigned off_a[kLoadsA], off_b[kLoadsB];
        const int chunk = (lane & 7) ^ swizzle(wave * 8 + (lane >> 3));       // (eight waves on it is the same)
        if (kTransA) {
            a0 = FORM == kWeightGradient ? P.a + (size_t)rows.first * P.a_ld : P.a + (size_t)e * P.a_expert;
            a1 = a0;
#pragma unroll
            for (int j = 0; j < kLoadsA; ++j) {
                const int r = (j * kWaves + wave) * 2 + (lane >> 5);
                int f = f0 + ((lane & 31) ^ spread(r)) * 8;
                if (f >= P.features) f = 0;
                off_a[j] = (unsigned)r * P.a_ld + f * 2;
            }
        } else {
            const char *base = P.a + (size_t)e * P.a_expert;
            a0 = base + (size_t)f0 * P.a_ld;
            a1 = GATED ? a0 + (size_t)P.features * P.a_ld : a0;
#pragma unroll
            for (int j = 0; j < kLoadsA; ++j) {
                int r = (j * kWaves + wave) * 8 + (lane >> 3);
                if (GATED) r &= kHalf - 1;
                if (f0 + r >= P.features) r = 0;
                off_a[j] = (unsigned)r * P.a_ld + chunk * 16;
            }
        }
        if (kTransB) {
            b0 = P.b + (size_t)rows.first * P.b_ld;
#pragma unroll
            for (int j = 0; j < kLoadsB; ++j) {
                const int r = (j * kWaves + wave) * 2 + (lane >> 5);
                int f = r0 + ((lane & 31) ^ spread(r)) * 8;
                if (f >= n_b) f = 0;
                off_b[j] = (unsigned)r * P.b_ld + f * 2;
            }
        } else {
            b0 = P.b + (size_t)(rows.first + r0) * P.b_ld;
#pragma unroll
            for (int j = 0; j < kLoadsB; ++j) {
                int r = (j * kWaves + wave) * 8 + (lane >> 3);
                if (r0 + r >= n_b) r = 0;
                off_b[j] = (unsigned)r * P.b_ld + chunk * 16;
            }
        }
        const float *sa = nullptr, *sa1 = nullptr, *sb = nullptr;
        unsigned off_s = 0;
        if (E4M3) {                                                    // scales: one of a row and one of 128 features a step
            const int blocks = (P.features + 127) / 128 * (GATED ? 2 : 1), per_row = P.k / 128;
            const int first = f0 / 128 + (GATED ? 0 : frag_feature(wf, 0) / 128);
            const int last = (P.features - 1) / 128;
            sa = P.a_scales + ((size_t)e * blocks + (first < last ? first : last)) * per_row;
            sa1 = GATED ? sa + (size_t)(P.features / 128) * per_row : sa;
            sb = P.b_scales + (size_t)(rows.first + r0) * per_row;
            int r = wave * kWave + lane;
            if (r0 + r >= n_b) r = 0;
            off_s = (unsigned)r * per_row * 4;
        }

        const unsigned lds0 = lds_address(lds);
        auto stage = [&](int step, int s) {
            const unsigned at = lds0 + s * kStage;
            const int row = wave * 2 + (lane >> 5);                    // transposed operands: of the first load
            const bool there = step * kStep + chunk * 16 < k * size;   // the others
            const Window wa(kTransA ? a0 + (size_t)step * 64 * P.a_ld : a0), wa1(a1);
            const Window wb(kTransB ? b0 + (size_t)step * 64 * P.b_ld : b0);
#pragma unroll
            for (int j = 0; j < kLoadsA; ++j) {
                const bool valid = kTransA ? step * 64 + j * kWaves * 2 + row < k : there;
                to_lds_16(GATED && j >= kLoadsA / 2 ? wa1 : wa, valid ? off_a[j] : kNowhere, kTransA ? 0 : step * kStep,
                          at + (j * kWaves + wave) * 1024);
            }
#pragma unroll
            for (int j = 0; j < kLoadsB; ++j) {
                const bool valid = kTransB ? step * 64 + j * kWaves * 2 + row < k : there;
                to_lds_16(wb, valid ? off_b[j] : kNowhere, kTransB ? 0 : step * kStep, at + kBytesA + (j * kWaves + wave) * 1024);
            }
            if (E4M3 && wave < ROWS / kWave)
                to_lds_4(Window((const char *)sb), off_s, step * 4, at + kBytesA + kBytesB + wave * kWave * 4);
        };

        Acc acc[kFragsF][kFragsR];
#pragma unroll
        for (int i = 0; i < kFragsF; ++i)
#pragma unroll
            for (int j = 0; j < kFragsR; ++j)
#pragma unroll
                for (int t = 0; t < kAccs; ++t) acc[i][j][t] = 0.0f;

        auto multiply = [&](int step, int s) {
            const char *A = lds + s * kStage, *B = A + kBytesA;
            if constexpr (E4M3) {
                const float *S = (const float *)(B + kBytesB);
                const float wa = sa[step], wa1 = GATED ? sa1[step] : wa;
                v8i fb[kFragsR];
                float scale[kFragsR];
                auto frag = [&](const char *T, int row) {
                    const v4i lo = *(const v4i *)(T + row * kStep + (((lane >> 4) ^ swizzle(row)) << 4));
                    const v4i hi = *(const v4i *)(T + row * kStep + ((((lane >> 4) + 4) ^ swizzle(row)) << 4));
                    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                };
#pragma unroll
                for (int j = 0; j < kFragsR; ++j) {
                    const int row = (wr * kFragsR + j) * kSide + (lane & 15);
                    fb[j] = frag(B, row);
                    scale[j] = S[row];
                }
#pragma unroll
                for (int i = 0; i < kFragsF; ++i) {
                    const v8i fa = frag(A, frag_feature(wf, i) + (lane & 15));
                    const float w = GATED && i >= kFragsF / 2 ? wa1 : wa;
#pragma unroll
                    for (int j = 0; j < kFragsR; ++j) {
                        const v4f zero = {0.0f, 0.0f, 0.0f, 0.0f};
                        const v4f part = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa, fb[j], zero, 0, 0, 0, 0, 0, 0);
                        const float f = scale[j] * w;
#pragma unroll
                        for (int t = 0; t < 4; ++t) acc[i][j][t] = fmaf(part[t], f, acc[i][j][t]);
                    }
                }
            } else {
                auto frag = [&](const char *T, bool trans, int first, int part) {
                    if (trans) {
                        const int f = first + (lane & 16), r = part * 16 + (lane >> 5) * 8;
                        const v4s lo = read_transposed(T, r, f), hi = read_transposed(T, r + 4, f);
                        const v8s both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                        return __builtin_bit_cast(v8bf, both);
                    }
                    const int row = first + (lane & 31);
                    return *(const v8bf *)(T + row * kStep + (((part * 2 + (lane >> 5)) ^ swizzle(row)) << 4));
                };
#pragma unroll
                for (int part = 0; part < 4; ++part) {
                    v8bf fa[kFragsF], fb[kFragsR];
#pragma unroll
                    for (int i = 0; i < kFragsF; ++i) fa[i] = frag(A, kTransA, frag_feature(wf, i), part);
#pragma unroll
                    for (int j = 0; j < kFragsR; ++j) fb[j] = frag(B, kTransB, (wr * kFragsR + j) * kSide, part);
#pragma unroll
                    for (int i = 0; i < kFragsF; ++i)
#pragma unroll
                        for (int j = 0; j < kFragsR; ++j)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[i], fb[j], acc[i][j], 0, 0, 0);
                }
            }
        };

        __syncthreads();                           // the tile before is done with its LDS
        if (steps) stage(0, 0);
        for (int step = 0; step < steps; ++step) {
            loads_done_and_barrier<0>();           // this step's operands are there, those of the step before are done with
            if (step + 1 < steps) stage(step + 1, (step + 1) % STAGES);
            multiply(step, step % STAGES);
        }

        // ---- the tile's output, 128 features at a time through LDS, so that rows are written in whole lines
        float *out = (float *)lds;
        const int piece = tid & 15, n_rows = n_b - r0 < ROWS ? n_b - r0 : ROWS;
        // Moves value(i, j, t) of fragments [lo, hi) to LDS and from there, eight features a lane, to put(row, values).
        auto emit = [&](int lo, int hi, auto value, auto put) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kFragsF; ++i) {
                if (i < lo || i >= hi) continue;
                const int f = frag_feature(wf, i) & (kHalf - 1);
#pragma unroll
                for (int j = 0; j < kFragsR; ++j) {
                    const int row = (wr * kFragsR + j) * kSide + (lane & (kSide - 1));
#pragma unroll
                    for (int t = 0; t < kAccs; t += 4) {
                        const v4f v = {value(i, j, t), value(i, j, t + 1), value(i, j, t + 2), value(i, j, t + 3)};
                        *(v4f *)(out + row * kEmitPitch + f + (E4M3 ? (lane >> 4) * 4 : t * 2 + (lane >> 5) * 4)) = v;
                    }
                }
            }
            __syncthreads();
            for (int row = tid >> 4; row < n_rows; row += kThreads / 16) {
                const v4f x = *(const v4f *)(out + row * kEmitPitch + piece * 8), y = *(const v4f *)(out + row * kEmitPitch + piece * 8 + 4);
                const float v[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
                put(row, v);
            }
        };
        // the eight features from f on of row `row` of a tensor `width` features wide
        auto put_bf16 = [&](void *to, size_t row, int f, int width, const float *v) {
            const v4u w = {to_bf16x2(v[0], v[1]), to_bf16x2(v[2], v[3]), to_bf16x2(v[4], v[5]), to_bf16x2(v[6], v[7])};
            *(v4u *)((char *)to + (row * width + f) * 2) = w;
        };
        auto put_e4m3 = [&](void *to, float *scales, size_t row, int f, int width, const float *v) {
            float amax = 0.0f;                                         // NaN fails the comparison and is skipped
#pragma unroll
            for (int i = 0; i < 8; ++i) amax = fabsf(v[i]) > amax ? fabsf(v[i]) : amax;
#pragma unroll
            for (int o = 1; o < 16; o <<= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
            const float scale = block_scale(amax);
            const v2u w = {e4m3_codes(v, scale), e4m3_codes(v + 4, scale)};
            *(v2u *)((char *)to + row * width + f) = w;
            if (piece == 0) scales[row * (width / 128) + f / 128] = scale;
        };
        // output row of the tile's row
        const size_t row0 = FORM == kWeightGradient ? (size_t)e * P.other + r0 : (size_t)(rows.first + r0);
        const int f = f0 + piece * 8;
        if constexpr (GATED) {
            auto gate = [&](int i, int j, int t) { return acc[i][j][t]; };
            auto up = [&](int i, int j, int t) { return acc[i + kFragsF / 2 < kFragsF ? i + kFragsF / 2 : i][j][t]; };
            if (P.pre) {
                for (int second = 0; second < 2; ++second) {
                    auto keep = [&](int row, const float *v) {
                        if (f >= P.features) return;
                        if (P.pre_scales) put_e4m3(P.pre, P.pre_scales, row0 + row, second * P.features + f, 2 * P.features, v);
                        else put_bf16(P.pre, row0 + row, second * P.features + f, 2 * P.features, v);
                    };
                    if (second) emit(0, kFragsF / 2, up, keep);
                    else emit(0, kFragsF / 2, gate, keep);
                }
            }
            emit(0, kFragsF / 2,
                 [&](int i, int j, int t) { return activate<false>(P.act, gate(i, j, t), nullptr) * up(i, j, t); },
                 [&](int row, const float *v) {
                     if (f >= P.features) return;
                     if (E4M3) put_e4m3(P.out, P.out_scales, row0 + row, f, P.features, v);
                     else put_bf16(P.out, row0 + row, f, P.features, v);
                 });
        } else {
            // a wave's features lie in one half: the waves of the other one wait at the barriers
#pragma unroll
            for (int half = 0; half < 2; ++half)
                emit(frag_feature(wf, 0) / kHalf == half ? 0 : kFragsF, kFragsF, [&](int i, int j, int t) { return acc[i][j][t]; },
                     [&](int row, const float *v) {
                         if (f + half * kHalf < P.features) put_bf16(P.out, row0 + row, f + half * kHalf, P.features, v);
                     });
        }
    }
};

// Row tiles of the call's experts before each, in LDS: [n + 1].
__device__ inline void scan_tiles(const Groups &G, int rows_per_tile, int *before) {
    __shared__ int part[kThreads / kWave];
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    int carry = 0;
    if (tid == 0) before[0] = 0;
    for (int base = 0; base < G.n; base += kThreads) {
        int v = 0;
        if (base + tid < G.n) v = (int)(((long long)rows_of(G, G.first + base + tid).n + rows_per_tile - 1) / rows_per_tile);
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
            const int w = __shfl_up(v, o);
            if (lane >= o) v += w;
        }
        if (lane == kWave - 1) part[tid / kWave] = v;
        __syncthreads();
        int mine = carry;
        for (int w = 0; w < kWaves; ++w) {
            if (w < tid / kWave) mine += part[w];
            carry += part[w];
        }
        if (base + tid < G.n) before[base + tid + 1] = mine + v;
        __syncthreads();
    }
}

constexpr int kXcds = 8;
constexpr int kRowGroup = 8;                   // row tiles that walk the features together

template <int FORM, bool E4M3, bool GATED, int ROWS, int STAGES>
__global__ __launch_bounds__(kThreads) void expert_tiles_kernel(Groups G, Product P) {
    using T = Tile<FORM, E4M3, GATED, ROWS, STAGES>;
    __shared__ __align__(1024) char lds[T::kLds];
    __shared__ int before[kMaxExperts + 1];
    const int columns = (P.features + T::kOutput - 1) / T::kOutput;
    const int fixed = FORM == kWeightGradient ? (P.other + ROWS - 1) / ROWS : 0;
    if (FORM != kWeightGradient) scan_tiles(G, ROWS, before);
    const long long tiles = (long long)(FORM == kWeightGradient ? G.n * fixed : before[G.n]) * columns;
    // workgroups go to the XCDs in turn: those of one XCD take neighbouring tiles, whose operands its L2 then holds
    const int per_xcd = gridDim.x / kXcds;
    const long long mine = (long long)(blockIdx.x % kXcds) * per_xcd + blockIdx.x / kXcds;
    for (long long t = mine; t < tiles; t += gridDim.x) {
        const int row_tile = (int)(t / columns);                       // counted over the experts
        int lo = 0, hi = G.n, n_tiles, index;
        if constexpr (FORM == kWeightGradient) {
            lo = row_tile / fixed;
            n_tiles = fixed;
            index = (int)(t - (long long)lo * fixed * columns);
        } else {
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (before[mid] <= row_tile) lo = mid; else hi = mid;
            }
            n_tiles = before[lo + 1] - before[lo];
            index = (int)(t - (long long)before[lo] * columns);
        }
        const int group = index / (kRowGroup * columns), left = n_tiles - group * kRowGroup;
        const int in_group = left < kRowGroup ? left : kRowGroup, within = index - group * kRowGroup * columns;
        const int column = within / in_group, row = group * kRowGroup + within - column * in_group;
        const int e = G.first + __builtin_amdgcn_readfirstlane(lo);
        const Rows found = rows_of(G, e), rows = {same_in_wave(found.first), __builtin_amdgcn_readfirstlane(found.n)};
        // (tables that claim more rows than there can be may have wrapped the sums)
        if ((unsigned)column >= (unsigned)columns || row < 0 || (long long)row * ROWS >= (FORM == kWeightGradient ? P.other : rows.n)) continue;
        T::run(P, lds, e, rows, __builtin_amdgcn_readfirstlane(column) * T::kOutput, __builtin_amdgcn_readfirstlane(row) * ROWS);
    }
}

// ---------------------------------------------------------------- the gated block's own gradient
// dg = dh u act'(g), du = dh act(g) from the kept pre-activations, rounded to bf16 for the matrix products behind (they
// take bf16 operands; the rounding is of the size of the results' own); h = act(g) u again where asked for.  Bound by
// memory: three rows of inter read, two (three) written.  pre and dpre may be the same rows.
__global__ __launch_bounds__(256) void expert_gated_gradient_kernel(
    Groups G, int inter, int act, const char *pre, const float *pre_scales, const char *__restrict__ dh, char *dpre, char *__restrict__ h) {
    const Rows rows = rows_of(G, G.first + blockIdx.y);
    const int vecs = inter / 8;
    const long long all = (long long)rows.n * vecs;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < all; i += (long long)gridDim.x * 256) {
        const int r = (int)(i / vecs), f = (int)(i - (long long)r * vecs) * 8;
        const size_t row = (size_t)rows.first + r;
        float g[8], u[8], d[8];
        auto split = [](v4u w, float *to) {
#pragma unroll
            for (int t = 0; t < 4; ++t) { to[2 * t] = from_bf16(w[t] & 0xffffu); to[2 * t + 1] = __uint_as_float(w[t] & 0xffff0000u); }
        };
        split(*(const v4u *)(dh + (row * inter + f) * 2), d);
        if (pre_scales) {
            auto decode = [](v2u w, float scale, float *to) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    to[4 * t] = __builtin_amdgcn_cvt_f32_fp8((int)w[t], 0) * scale;
                    to[4 * t + 1] = __builtin_amdgcn_cvt_f32_fp8((int)w[t], 1) * scale;
                    to[4 * t + 2] = __builtin_amdgcn_cvt_f32_fp8((int)w[t], 2) * scale;
                    to[4 * t + 3] = __builtin_amdgcn_cvt_f32_fp8((int)w[t], 3) * scale;
                }
            };
            const int blocks = inter / 128;
            decode(*(const v2u *)(pre + row * 2 * inter + f), pre_scales[row * 2 * blocks + f / 128], g);
            decode(*(const v2u *)(pre + row * 2 * inter + inter + f), pre_scales[row * 2 * blocks + blocks + f / 128], u);
        } else {
            split(*(const v4u *)(pre + (row * 2 * inter + f) * 2), g);
            split(*(const v4u *)(pre + (row * 2 * inter + inter + f) * 2), u);
        }
        float a[8], dg[8], du[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            float slope;
            a[t] = activate<true>(act, g[t], &slope);
            dg[t] = d[t] * u[t] * slope;
            du[t] = d[t] * a[t];
        }
        auto join = [](const float *v) { return v4u{to_bf16x2(v[0], v[1]), to_bf16x2(v[2], v[3]), to_bf16x2(v[4], v[5]), to_bf16x2(v[6], v[7])}; };
        *(v4u *)(dpre + (row * 2 * inter + f) * 2) = join(dg);
        *(v4u *)(dpre + (row * 2 * inter + inter + f) * 2) = join(du);
        if (h) {
#pragma unroll
            for (int t = 0; t < 8; ++t) a[t] *= u[t];
            *(v4u *)(h + (row * inter + f) * 2) = join(a);
        }
    }
}

}  // namespace experts
}  // namespace flmoe
