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
__device__ inline unsigned to_bf16x2(float lo, float hi) {              // to nearest even, NaN stays a quiet NaN
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(unsigned, v2bf{(__bf16)lo, (__bf16)hi});
}

// silu(v) = v s, s = 1 / (1 + e^-v); gelu(v) = v s with s = 1 / (1 + e^(-2 a (v + 0.044715 v^3))), a = sqrt(2 / pi), which
// is the tanh form.  *slope receives the derivative; where s has reached 0 or 1 its own derivative is 0, whatever v.
constexpr float kGelu = 1.5957691216057308f;                            // 2 sqrt(2 / pi)
template <bool SLOPE>
__device__ inline float activate(int act, float v, float *slope) {
    const float arg = act == FL_ACT_SILU ? v : kGelu * (v + 0.044715f * v * v * v);
    const float s = __builtin_amdgcn_rcpf(1.0f + __expf(-arg));
    if (SLOPE) {
        const float ds = s * (1.0f - s), inner = act == FL_ACT_SILU ? v : kGelu * (v + 3.0f * 0.044715f * v * v * v);
        *slope = ds == 0.0f ? s : s + inner * ds;
    }
    return v * s;
}

// Codes of four values of an e4m3 block (see FL_DTYPE_E4M3_BLOCK128): rounded to nearest even, saturating; what is NaN
// over the scale (a NaN, or an Inf in a block whose scale it made infinite) becomes the NaN code with the value's sign.
// (A maximum below about 3e-43, which no bf16 row has but an fp32 product may, over 448 is 0: such a block is zeros too.)
__device__ inline float block_scale(float amax) {
    const float scale = __fdiv_rn(amax, 448.0f);
    return scale == 0.0f ? 1.0f : scale;
}
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
// (Lambdas that hold fragments or accumulators by reference: called instead of inlined they would put them into memory.)
#define FLMOE_INLINE __attribute__((always_inline))
// A lane's 16 (or 4) bytes straight into LDS, at the wave's place there plus 16 (4) times the lane.  Offsets of kNowhere
// read as zero; only offsets inside the tensor or kNowhere are ever passed, the limit is the largest there is.  Written
// out because the compiler, which knows that these loads write LDS, lets every read of LDS behind them wait for them:
// here the waits are the ones below, once per step.  Nothing is returned, so no register is written behind its back.
// One wait state lies between a write of m0 and a load that goes by it.  And five between a vector instruction that writes a
// scalar register (also v_readlane, which brings back a spilled one) and the load that reads it: the compiler sees to that
// before its own loads, not before inline assembly, so the first load here begins with them.
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
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 ::"s"(__builtin_amdgcn_readfirstlane((int)lds)), "v"(offset), "s"(w.rsrc), "s"(__builtin_amdgcn_readfirstlane((int)shift)) : "memory", "m0");
}
// Two of them, DISTANCE bytes of LDS apart.
template <int DISTANCE>
__device__ inline void two_to_lds_16(const Window &w, unsigned offset, unsigned offset2, unsigned shift, unsigned lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %3, %4 offen lds\n\t"
                 "s_add_u32 m0, m0, %5\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, %4 offen lds"
                 ::"s"(__builtin_amdgcn_readfirstlane((int)lds)), "v"(offset), "v"(offset2), "s"(w.rsrc),
                 "s"(__builtin_amdgcn_readfirstlane((int)shift)), "n"(DISTANCE) : "memory", "m0", "scc");
}
__device__ inline void to_lds_4(const Window &w, unsigned offset, unsigned shift, unsigned lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dword %1, %2, %3 offen lds"
                 ::"s"(__builtin_amdgcn_readfirstlane((int)lds)), "v"(offset), "s"(w.rsrc), "s"(__builtin_amdgcn_readfirstlane((int)shift)) : "memory", "m0");
}
// The compiler keeps what comes before apart from what comes behind.
__device__ inline void in_order() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}
// Every load of this wave but the last KEEP is done, and so are its reads of LDS; behind the barrier every wave's.
// (The compiler knows the wait's own form, so it does not wait for those reads again.)
template <int KEEP>
__device__ inline void loads_done_and_barrier() {
    in_order();
    __builtin_amdgcn_s_waitcnt((KEEP & 15) | KEEP >> 4 << 14 | 7 << 4);      // vmcnt, lgkmcnt 0
    __builtin_amdgcn_s_barrier();
    in_order();
}

// ---------------------------------------------------------------- the tiles
// 256 features by 256 rows, eight waves, two on each SIMD: 32 accumulators of 16 by 16 outputs a wave, half of what the
// registers hold; an operand's byte, once read, serves 128 operations in bf16, 256 in e4m3.  A step multiplies 128 bytes of
// the contraction (64 bf16, 128 e4m3).  Both operands of a step come in two units of 16 KB (A0, A1: 128 features each, of a gated tile the gates and
// their ups; B0, B1: 128 rows each), and each wave owns 64 of the features and 32 of the rows of every unit.  A step has
// two phases; each reads from LDS what the products behind it take, over what has been used up, while the ones before it are
// under way:
//   phase 1: reads B1; A0 B0; A0 B1, reading A1 over A0 fragment by fragment
//   phase 2: reads B0 of the next step; A1 B1; A1 B0, reading A0 of the next step over A1
// A phase ends with: this wave's reads are done, its loads for the next phase's units have arrived, barrier; then the
// units just read are loaded for two steps later.  So with two places for each unit the loads that fill one have a step
// and a half to arrive, and 64 to 96 KB are on their way to a compute unit all the time.  (Four phases of one quadrant
// each, a barrier behind each: the row gradient took 6 % longer.)
// Full tiles with contractions of 7168 and more reach 1280 to 1330 Tflop/s in bf16 (a large library product on this card 1400
// to 1600), the loop by itself 1350; what begins and ends a tile takes 8 us, as long as five of its steps (32 x 1024 rows, 1024
// wide, contractions of 512 to 7168: 82 to 735 us).  e4m3 reaches 1880 to 2030: there the block scales' fused multiplications
// take about an eighth of the time and the loads into LDS a fifth.
constexpr int kStep = 128;                     // bytes of the contraction per step
constexpr int kXcds = 8;

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

// Place of a 16-byte chunk in a unit, so that the lanes that are served together fall into different banks (64 of 4
// bytes; sixteen lanes of a 16-byte read, 32 of an 8-byte one).
// Contiguous along the contraction: rows of 128 bytes, chunk c of row r at c ^ (r >> 1 & 7): two rows fill the banks once.
// Contiguous along the features: 64 contraction rows of 256 bytes; the transposing reads take 32 bytes each of rows
// 8 m .. 8 m + 3 (or + 4) and of the same of the next eight rows at once, which the row's bits 0, 1 and 3 keep apart.
__device__ inline int swizzle(int row) { return row >> 1 & 7; }
__device__ inline int spread(int row) { return (row & 3) << 2 | (row >> 2 & 2); }

// ROWS: 256; or for experts of few rows 64 or 32, with HALF features to a unit of A, a wave for every 16 of them.
template <int FORM, bool E4M3, bool GATED, int ROWS, int HALF>
struct Tile {
    static constexpr bool kTransA = FORM != kForward, kTransB = FORM == kWeightGradient;
    static_assert((ROWS == 256 && HALF == 128) || (FORM == kForward && ((ROWS == 64 && HALF == 128) || (ROWS <= 64 && HALF == 64))), "");
    static constexpr int kThreads = ROWS == 256 ? 512 : HALF * 4, kWaves = kThreads / kWave;
    // Matrix instructions of 16 by 16 outputs, 64 bytes of bf16 or 128 of e4m3 deep.  (Alone on the machine they reach
    // 2370 Tflop/s in bf16, 1930 with random operands; those of 32 by 32 outputs 1600 and 1310.)
    static constexpr int kSide = 16, kParts = E4M3 ? 1 : 2;
    static constexpr int kHalves = ROWS == 256 ? 2 : 1;                // units of B
    static constexpr int kUnitRows = ROWS / kHalves, kUnitA = HALF * kStep, kUnitB = kUnitRows * kStep;
    static constexpr int kWavesF = ROWS == 256 ? 2 : kWaves, kWavesR = kWaves / kWavesF;
    static constexpr int kOwnF = HALF / kWavesF, kOwnR = kUnitRows / kWavesR;         // of a wave in a unit
    static constexpr int kFragsF = kOwnF / kSide, kFragsR = kOwnR / kSide;
    static constexpr int kLoadsB = kUnitRows / kWaves / 8;             // of a wave for a unit of B
    static constexpr int kRing = 4 * kUnitA + 2 * kHalves * kUnitB;    // [two][A0, A1], [two][B0, B1]
    // scales of the rows of a step: those of its own rows for each wave, or of all
    static constexpr int kScales = !E4M3 ? 0 : ROWS == 256 ? kWaves * kWave * 4 : ROWS * 4, kScaleSlots = 4;
    static constexpr int kScalesAt = kRing, kScalesEnd = kScalesAt + kScaleSlots * kScales;
    // The output passes through LDS: a wave's 64 lanes write eight features each of kEmitRows rows at a time.  In blocks of
    // e4m3 the largest values of a row in each wave's features pass through it as well.
    static constexpr int kPieces = kOwnF / 8, kEmitRows = kWave / kPieces, kEmitPitch = kOwnF + 4;
    static constexpr int kEmit = kWaves * kEmitRows * kEmitPitch * 4;
    // Tiles of 256 rows have it apart from the ring: the next tile's first loads are on their way meanwhile.
    static constexpr bool kEarly = ROWS == 256;
    static constexpr int kEmitAt = kEarly ? kScalesEnd : 0, kLargestAt = kEmitAt + kEmit;
    static constexpr int kEmitEnd = kLargestAt + (GATED ? kWavesF * ROWS * 4 : 0);
    static constexpr int kLds = kEmitEnd > kScalesEnd ? kEmitEnd : kScalesEnd;
    static constexpr int kOutput = GATED ? HALF : 2 * HALF;          // output features of a tile
    using Acc = v4f;
    using Frag = typename std::conditional<E4M3, v8i, v8bf>::type;
    enum Unit { A0, A1, B0, B1 };
    struct Place {
        int e;                                     // expert
        Rows rows;                                 // its rows
        int f0, r0;                                // first output feature; first row (weight gradient: first column of b)
    };

    // next(place): the workgroup's next tile, if there is one.
    template <class Next>
    __device__ static void run(const Product &P, char *lds, Next next_place) {
        const int tid = threadIdx.x, lane = tid & (kWave - 1);
        const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
        const int wf = wave % kWavesF, wr = wave / kWavesF;
        const int size = E4M3 ? 1 : 2;
        Place tile;
        int k, n_b, steps;                         // contraction; rows of operand b; steps
        // Few rows: one unit of B.  The weights are then read once and their reading is what takes time, and where rows are
        // a power of two apart one step's loads all fall on a few memory channels.  So tiles begin at different steps and
        // wrap round: 128 experts of 2 x 768 x 2048 at 16 rows 196 -> 153 us.  (With more rows it would part the
        // workgroups that share operands: 487 -> 499 us.)  Where a tile begins goes by its expert and its 128 features alone,
        // one step on from the 128 before, so that a sum's order is the same whatever tiles, grid, ranks or other experts'
        // rows there are (spread over the steps by the golden section instead: 141.3 -> 143.9 us).
        bool few;
        int shift;
        using Turned = std::integral_constant<bool, true>;
        using Straight = std::integral_constant<bool, false>;
        auto place_of = [&](int step, auto turn) {
            if constexpr (turn()) return step + shift < steps ? step + shift : step + shift - steps;
            else return step;
        };

        // Where this lane's chunks come from.  Past the end of the features there are others that are as good (what is
        // computed from them is not written); past the rows and past the contraction there are zeros.
        unsigned off[2][4];                        // [operand][loads of both units]
        int steps_here[2];                         // steps in which this lane's chunk of a load is there (transposed: of both)
        int depth;                                 // transposed: row of this lane's chunk of a unit's first load
        const char *a0, *a1, *b0;                  // a1: ups of a gated tile
        // e4m3: scales of 128 features (weights never change while a kernel runs: scalar loads) and of the rows, one a step
        typedef const __attribute__((address_space(4))) float *Constant;
        Constant sa[2] = {nullptr, nullptr};
        const char *sb = nullptr;
        unsigned off_s = 0;
        const int per_row = P.k / 128;
        auto set_out = [&]() FLMOE_INLINE {
            // (opaque, so that what follows from it is worked out here and not kept in registers from tile to tile)
            int l = lane;
            asm volatile("" : "+v"(l));
            const int e = tile.e, f0 = tile.f0, r0 = tile.r0;
            const Rows rows = tile.rows;
            k = FORM == kWeightGradient ? rows.n : P.k;
            n_b = FORM == kWeightGradient ? P.other : rows.n;
            steps = (int)(((long long)k * size + kStep - 1) / kStep);
            few = kHalves == 1 || n_b - r0 <= kUnitRows;
            shift = steps > 0 ? (e * ((P.features + 127) / 128) + f0 / 128) % steps : 0;
            depth = wave * 4 + (l >> 4);
            const int column = ((l & 15) ^ spread(depth)) * 8;
#pragma unroll
            for (int o = 0; o < 2; ++o) {
                const bool trans = o ? kTransB : kTransA;
                const int ld = o ? P.b_ld : P.a_ld, end = o ? n_b - r0 : P.features - f0;
                const int chunk = (l & 7) ^ swizzle(wave * 8 + (l >> 3));               // contiguous along the contraction
#pragma unroll
                for (int j = 0; j < (o ? kHalves * kLoadsB : 4); ++j) {
                    if (trans) {
                        const int f = (j >> 1) * HALF + column;
                        off[o][j] = (unsigned)(depth + (j & 1) * 32) * ld + (f < end ? f : 0) * 2;
                    } else {
                        int r = (j * kWaves + wave) * 8 + (l >> 3);
                        if (!o && GATED) r &= HALF - 1;
                        off[o][j] = r < end ? (unsigned)r * ld + chunk * 16 : o ? kNowhere : (unsigned)chunk * 16;
                    }
                }
                steps_here[o] = trans ? (k - depth + 63) / 64 : (k * size - chunk * 16 + kStep - 1) / kStep;
            }
            if (FORM == kWeightGradient) a0 = P.a + (size_t)rows.first * P.a_ld + f0 * 2;
            else a0 = P.a + (size_t)e * P.a_expert + (kTransA ? (size_t)f0 * 2 : (size_t)f0 * P.a_ld);
            a1 = GATED ? a0 + (size_t)P.features * P.a_ld : a0;
            b0 = kTransB ? P.b + (size_t)rows.first * P.b_ld + r0 * 2 : P.b + (size_t)(rows.first + r0) * P.b_ld;
            if (E4M3) {
                const int blocks = (P.features + 127) / 128;
                const Constant first = (Constant)(uintptr_t)P.a_scales + (size_t)e * blocks * (GATED ? 2 : 1) * per_row;
                const int block = f0 / 128, second = (f0 + HALF) / 128;
                sa[0] = first + (size_t)block * per_row;
                sa[1] = first + (size_t)(GATED ? blocks + block : second < blocks ? second : block) * per_row;
                sb = (const char *)(P.b_scales + (size_t)(rows.first + r0) * per_row);
                // this wave's in B0, then in B1; of 64 rows each wave a share
                int r = ROWS == 256 ? (l >> 5) * kUnitRows + wr * 32 + (l & 31) : wave * kLoadsB * 8 + (l & (kLoadsB * 8 - 1));
                if (r >= n_b - r0) r = 0;
                off_s = (unsigned)r * per_row * 4;
            }
        };

        const unsigned lds0 = lds_address(lds);
        // [slot][A0, A1], then [slot][B0, B1]: what one operand's reads span fits their instructions' offset
        auto place = [](int unit, int slot) constexpr {
            return unit < B0 ? (slot * 2 + unit) * kUnitA : 4 * kUnitA + (slot * kHalves + unit - B0) * kUnitB;
        };
        auto scales_at = [](int step, int wave) { return kScalesAt + ((step & (kScaleSlots - 1)) * kScales) + (ROWS == 256 ? wave * kWave * 4 : 0); };
        auto load = [&](int unit, int step, auto turn) FLMOE_INLINE {
            const int o = unit >= B0, u = o ? unit - B0 : unit;
            const bool trans = o ? kTransB : kTransA;
            const int ld = o ? P.b_ld : P.a_ld, at_k = place_of(step, turn);
            const char *base = o ? b0 : u ? a1 : a0;
            const Window from(trans ? base + (size_t)at_k * 64 * ld : base);
            const unsigned to = lds0 + place(unit, step & 1) + wave * 1024;
            auto offset = [&](int j) {
                const bool there = step < steps && (trans && j ? at_k * 64 + depth + 32 < k : at_k < steps_here[o]);
                return there ? off[o][u * 2 + j] : kNowhere;
            };
            const unsigned along = trans ? 0 : at_k * kStep;
            if (!o || kLoadsB == 2) two_to_lds_16<kWaves * 1024>(from, offset(0), offset(1), along, to);
            else to_lds_16(from, offset(0), along, to);
        };
        auto load_scales = [&](int step, auto turn) {
            if constexpr (E4M3) {
                const unsigned from = step < steps ? off_s : kNowhere, shift_by = place_of(step, turn) * 4;
                if (ROWS == 256) to_lds_4(Window(sb), from, shift_by, lds0 + scales_at(step, wave));
                else if (lane < kLoadsB * 8) to_lds_4(Window(sb), from, shift_by, lds0 + scales_at(step, 0) + wave * kLoadsB * 32);
            }
        };

        // This wave's fragments of a unit.  Their places differ from the first one's by constants and, where the swizzle
        // reaches into them, by one of a few patterns: those are kept as addresses.
        //   contiguous along the contraction: chunks lane >> 4 and that plus 4 of row lane & 15, bf16 one for each of two
        //   instructions, e4m3 both for one (any order of the contraction will do that both operands have)
        //   transposed: lanes 16 m .. 16 m + 15 give the places of four rows by four pieces of 8 bytes, and lane j of them
        //   receives column j; a pattern for each fragment
        constexpr int kPatterns = kTransA || kTransB ? 4 : 2;
        unsigned at[2][kPatterns];
#pragma unroll
        for (int o = 0; o < 2; ++o) {
            const int first = o ? wr * kOwnR : wf * kOwnF, unit = lds0 + place(o ? B0 : A0, 0);
#pragma unroll
            for (int p = 0; p < kPatterns; ++p) {
                if (o ? kTransB : kTransA) {
                    const int row = (lane >> 4) * 8 + (lane >> 2 & 3), c = (first + p * kSide) / 8 + (lane >> 1 & 1);
                    at[o][p] = unit + row * 256 + (c ^ spread(row)) * 16 + (lane & 1) * 8;
                } else {
                    const int row = lane & 15;
                    at[o][p] = unit + (first + row) * kStep + (((lane >> 4) + (p & 1) * 4) ^ swizzle(row)) * 16;
                }
                asm volatile("" : "+v"(at[o][p]));                     // not to be worked out again at every use
            }
        }
        // base: from the operand's first unit to the fragment's
        auto frag = [&](auto operand, int base, int i, int part) FLMOE_INLINE -> Frag {
            constexpr int o = operand();
            if constexpr (E4M3) {
                const v4i lo = *(FLMOE_LDS const v4i *)(uintptr_t)(at[o][0] + base + i * kSide * kStep);
                const v4i hi = *(FLMOE_LDS const v4i *)(uintptr_t)(at[o][1] + base + i * kSide * kStep);
                return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            } else if constexpr (o ? kTransB : kTransA) {
                const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((FLMOE_LDS v4s *)(uintptr_t)(at[o][i] + base + part * 8192));
                const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((FLMOE_LDS v4s *)(uintptr_t)(at[o][i] + base + part * 8192 + 1024));
                const v8s both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                return __builtin_bit_cast(v8bf, both);
            } else {
                return *(FLMOE_LDS const v8bf *)(uintptr_t)(at[o][part] + base + i * kSide * kStep);
            }
        };
        Acc acc[2][kHalves][kFragsF][kFragsR];
        Frag fa[kFragsF][kParts], fb0[2][kFragsR][kParts], fb1[kFragsR][kParts];
        float row_scale[kFragsR];
        // multiplies the fragments at hand into quadrant (h, g); next(i, part) follows a fragment's last use
        auto multiply = [&](auto half_a, auto half_b, const Frag (&b)[kFragsR][kParts], float w, auto next) FLMOE_INLINE {
            constexpr int h = decltype(half_a)::value, g = decltype(half_b)::value;
            if constexpr (E4M3) {
                // A block's sum enters the accumulators, times both scales, while the next two are on their way (with one, the
                // wave waits for the instruction's end: 16 x 2048 rows of 7168 x 2048 996 -> 987 us, the product behind
                // 555 -> 533).  The instruction cuts the products of eight neighbours 13 places below their largest before it
                // adds them (and adds those sums in fp32): the price of twice the rate of the same sums in bf16, which would
                // be exact products.
                v4f sum[3];
                auto add = [&](int n) {
                    const int i = n / kFragsR, j = n % kFragsR;
                    const float f = row_scale[j] * w;
#pragma unroll
                    for (int t = 0; t < 4; ++t) acc[h][g][i][j][t] = fmaf(sum[n % 3][t], f, acc[h][g][i][j][t]);
                };
#pragma unroll
                for (int n = 0; n < kFragsF * kFragsR; ++n) {
                    const int i = n / kFragsR, j = n % kFragsR;
                    const v4f zero = {0.0f, 0.0f, 0.0f, 0.0f};
                    sum[n % 3] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa[i][0], b[j][0], zero, 0, 0, 0, 0, 0, 0);
                    if (j == kFragsR - 1) next(i, 0);
                    __builtin_amdgcn_sched_barrier(0);
                    if (n > 1) add(n - 2);
                }
                if (kFragsF * kFragsR > 1) add(kFragsF * kFragsR - 2);
                add(kFragsF * kFragsR - 1);
            } else {
#pragma unroll
                for (int part = 0; part < kParts; ++part)
#pragma unroll
                    for (int i = 0; i < kFragsF; ++i) {
#pragma unroll
                        for (int j = 0; j < kFragsR; ++j)
                            acc[h][g][i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[i][part], b[j][part], acc[h][g][i][j], 0, 0, 0);
                        next(i, part);
                        __builtin_amdgcn_sched_barrier(0);
                    }
            }
        };
        using Zero = std::integral_constant<int, 0>;
        using One = std::integral_constant<int, 1>;
        auto nothing = [](int, int) {};
        // What one wave does for step `step`; s: step & 1.
        float w[2] = {0.0f, 0.0f};
        auto scales_of_weights = [&](int step, auto parity, auto turn) {
            if constexpr (E4M3) {
                const bool there = !parity() || step < steps;          // behind an odd last step there is one of zeros
                const int at_k = there ? place_of(step, turn) : 0;
                w[0] = sa[0][at_k]; w[1] = sa[1][at_k];
                if (!there) w[0] = w[1] = 0.0f;
            }
        };
        auto scales_of = [&](int step, int g) {                        // of the rows of a unit of B
            if constexpr (E4M3) {
                const float *S = (const float *)(lds + scales_at(step, wave)) + g * 32 + (lane & 15);
#pragma unroll
                for (int j = 0; j < kFragsR; ++j) row_scale[j] = S[j * kSide];
            }
        };
        auto read_b = [&](Frag (&to)[kFragsR][kParts], int base) FLMOE_INLINE {
#pragma unroll
            for (int part = 0; part < kParts; ++part)
#pragma unroll
                for (int j = 0; j < kFragsR; ++j) to[j][part] = frag(One(), base, j, part);
        };
        auto read_a = [&](int base) FLMOE_INLINE {
#pragma unroll
            for (int part = 0; part < kParts; ++part)
#pragma unroll
                for (int i = 0; i < kFragsF; ++i) fa[i][part] = frag(Zero(), base, i, part);
        };
        // multiplies while the next fragments of A are read over the present ones
        auto multiply_and_read_a = [&](auto half_a, auto half_b, const Frag (&b)[kFragsR][kParts], float w, int base) FLMOE_INLINE {
            multiply(half_a, half_b, b, w, [&](int i, int part) FLMOE_INLINE { fa[i][part] = frag(Zero(), base, i, part); });
        };

        auto two_units = [&](auto one) FLMOE_INLINE {                  // (a template, so that it is made where it is called only)
            using One = decltype(one);
            // Loads of this wave that may still be on their way between phases: all but the units that the next phase reads
            // and those before them, four units of two loads, and in e4m3 a load of scales among them.
            constexpr int kAhead = E4M3 ? 9 : 8;
            Straight t;
            loads_done_and_barrier<kAhead + 4>();
            read_a(0);
            read_b(fb0[0], 0);
            loads_done_and_barrier<kAhead>();
            load(B0, 2, t); load_scales(2, t); load(A0, 2, t);
            // full: whether this wave has rows in B1 as well
            auto body = [&](int step, auto parity, auto full) FLMOE_INLINE {
                constexpr int s = parity();
                constexpr bool both = full();
                constexpr int a_here = s * 2 * kUnitA, a_next = (1 - s) * 2 * kUnitA, b_here = s * 2 * kUnitB, b_next = (1 - s) * 2 * kUnitB;
                scales_of_weights(step, parity, t);
                scales_of(step, 0);
                if constexpr (both) {
                    read_b(fb1, b_here + kUnitB);
                    in_order();
                    multiply(Zero(), Zero(), fb0[s], w[0], nothing);
                    scales_of(step, 1);
                    multiply_and_read_a(Zero(), One(), fb1, w[0], a_here + kUnitA);
                } else {
                    multiply_and_read_a(Zero(), Zero(), fb0[s], w[0], a_here + kUnitA);
                }
                loads_done_and_barrier<kAhead>();
                load(B1, step + 2, t); load(A1, step + 2, t);
                read_b(fb0[1 - s], b_next);
                in_order();
                if constexpr (both) {
                    multiply(One(), One(), fb1, w[1], nothing);
                    scales_of(step, 0);
                }
                multiply_and_read_a(One(), Zero(), fb0[s], w[1], a_next);
                loads_done_and_barrier<kAhead>();
                load(B0, step + 3, t); load_scales(step + 3, t); load(A0, step + 3, t);
            };
            auto all = [&](auto full) FLMOE_INLINE {
                for (int step = 0; step < steps; step += 2) {          // behind an odd last step, one of zeros
                    body(step, Zero(), full);
                    body(step + 1, One(), full);
                }
            };
            if (kUnitRows + wr * kOwnR < n_b - tile.r0) all(One());
            else all(Zero());
        };
        auto one_unit = [&]() FLMOE_INLINE {
            // No B1, two phases: A0 B0 while A1 is read over A0, then A1 B0 while the next step's A0 and B0 are read.  Waves
            // whose rows there are none of only load.
            constexpr int kAhead = 4 + kLoadsB + (E4M3 ? 1 : 0);
            Turned t;
            loads_done_and_barrier<kAhead + 2>();
            auto start = [&]() FLMOE_INLINE {
                loads_done_and_barrier<kAhead>();
                load(B0, 2, t); load_scales(2, t); load(A0, 2, t);
            };
            auto body = [&](int step, auto parity, auto present) FLMOE_INLINE {
                constexpr int s = parity();
                constexpr bool here = present();
                constexpr int a_here = s * 2 * kUnitA, a_next = (1 - s) * 2 * kUnitA, b_next = (1 - s) * kHalves * kUnitB;
                if constexpr (here) {
                    scales_of_weights(step, parity, t);
                    scales_of(step, 0);
                    multiply_and_read_a(Zero(), Zero(), fb0[s], w[0], a_here + kUnitA);
                }
                loads_done_and_barrier<kAhead>();
                load(A1, step + 2, t);
                if constexpr (here) {
                    read_b(fb0[1 - s], b_next);
                    in_order();
                    multiply_and_read_a(One(), Zero(), fb0[s], w[1], a_next);
                }
                loads_done_and_barrier<kAhead>();
                load(B0, step + 3, t); load_scales(step + 3, t); load(A0, step + 3, t);
            };
            auto all = [&](auto present) FLMOE_INLINE {
                for (int step = 0; step < steps; step += 2) {          // behind an odd last step, one of zeros
                    body(step, Zero(), present);
                    body(step + 1, One(), present);
                }
            };
            if (kWavesR == 1 || wr * kOwnR < n_b - tile.r0) {
                read_a(0);
                read_b(fb0[0], 0);
                start();
                all(One());
            } else {
                start();
                all(Zero());
            }
        };
        // the tile's first loads: what the loops above begin with
        auto begin = [&]() FLMOE_INLINE {
#pragma unroll
            for (int step = 0; step < 2; ++step) {
                if (few) {
                    Turned t;
                    load(B0, step, t); load_scales(step, t); load(A0, step, t); load(A1, step, t);
                } else if constexpr (kHalves == 2) {
                    Straight t;
                    load_scales(step, t); load(B0, step, t); load(A0, step, t); load(B1, step, t); load(A1, step, t);
                }
            }
        };

        // ---- the tile's output: accumulators hold four features of a row a lane, memory wants whole lines
        float *largest = (float *)(lds + kLargestAt);                  // [kWavesF][ROWS]
        int el;                                                        // lane
        // Moves value(g, i, j, t) of a half of the features to put(row, values), eight features a lane.
        auto emit = [&](int n_rows, auto value, auto put) FLMOE_INLINE {
            float *mine = (float *)(lds + kEmitAt) + wave * kEmitRows * kEmitPitch;
            const int piece = el & (kPieces - 1);
#pragma unroll
            for (int g = 0; g < kHalves; ++g)
#pragma unroll
                for (int first = 0; first < kOwnR; first += kEmitRows) {
#pragma unroll
                    for (int j = 0; j < kFragsR; ++j) {
                        const int row = j * kSide + (el & 15) - first;
                        if (j * kSide + kSide <= first || j * kSide >= first + kEmitRows) continue;
                        if (row >= 0 && row < kEmitRows) {
#pragma unroll
                            for (int i = 0; i < kFragsF; ++i)
                                *(v4f *)(mine + row * kEmitPitch + i * kSide + (el >> 4) * 4) =
                                    v4f{value(g, i, j, 0), value(g, i, j, 1), value(g, i, j, 2), value(g, i, j, 3)};
                        }
                    }
                    asm volatile("" ::: "memory");         // (a wave's reads of LDS follow its writes)
                    const float *from = mine + (el / kPieces) * kEmitPitch + piece * 8;
                    const v4f x = *(const v4f *)from, y = *(const v4f *)(from + 4);
                    const float v[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
                    const int row = g * kUnitRows + wr * kOwnR + first + el / kPieces;
                    if (row < n_rows) put(row, v);
                    asm volatile("" ::: "memory");
                }
        };
        // Whole lines that the kernel does not read again go past the caches, which keep the operands: training step of 128 experts
        // of 1 to 1694 rows 1035 -> 1019 us, both e4m3 products of 64 x 128 rows 668 -> 649, that of 32 x 250 rows of 1024 x 2048
        // 28.0 -> 27.1.  Not rows that begin inside lines (2056 wide 42.7 -> 43.8), nor a gated block's output, which the next
        // product reads.
        const bool past = ROWS == 256 && !GATED && P.features % 64 == 0;
        auto put = [&](auto w, char *to) {
            if (past) {
                asm volatile("");                              // (or the compiler makes one plain store of the two)
                __builtin_nontemporal_store(w, (decltype(w) *)to);
                asm volatile("");
            } else {
                *(decltype(w) *)to = w;
            }
        };
        // the eight features from f on of row `row` of a tensor `width` features wide
        auto put_bf16 = [&](void *to, size_t row, int f, int width, const float *v) {
            const v4u w = {to_bf16x2(v[0], v[1]), to_bf16x2(v[2], v[3]), to_bf16x2(v[4], v[5]), to_bf16x2(v[6], v[7])};
            put(w, (char *)to + (row * width + f) * 2);
        };
        // in blocks of e4m3; the tile's 128 features are one block
        auto find_largest = [&](auto value) FLMOE_INLINE {
            __syncthreads();                                           // those found before have been read
#pragma unroll
            for (int g = 0; g < kHalves; ++g)
#pragma unroll
                for (int j = 0; j < kFragsR; ++j) {
                    float m = 0.0f;                                    // NaN fails the comparison and is skipped
#pragma unroll
                    for (int i = 0; i < kFragsF; ++i)
#pragma unroll
                        for (int t = 0; t < 4; ++t) { const float v = fabsf(value(g, i, j, t)); m = v > m ? v : m; }
                    m = fmaxf(m, __shfl_xor(m, 16));
                    m = fmaxf(m, __shfl_xor(m, 32));
                    if (el < kSide) largest[wf * ROWS + g * kUnitRows + wr * kOwnR + j * kSide + el] = m;
                }
            __syncthreads();
        };
        auto put_e4m3 = [&](void *to, float *scales, size_t row0, int row, int f, int width, const float *v) {
            float m = 0.0f;
#pragma unroll
            for (int i = 0; i < kWavesF; ++i) m = fmaxf(m, largest[i * ROWS + row]);
            const float scale = block_scale(m);
            const v2u w = {e4m3_codes(v, scale), e4m3_codes(v + 4, scale)};
            put(w, (char *)to + (row0 + row) * width + f);
            if (wf == 0 && (el & (kPieces - 1)) == 0) scales[(row0 + row) * (width / 128) + f / 128] = scale;
        };
        auto write = [&](const Place &done) FLMOE_INLINE {
            el = lane;
            asm volatile("" : "+v"(el));                               // as in set_out
            const int end = FORM == kWeightGradient ? P.other : done.rows.n, n_rows = end - done.r0 < ROWS ? end - done.r0 : ROWS;
            // output row of the tile's first row
            const size_t row0 = FORM == kWeightGradient ? (size_t)done.e * P.other + done.r0 : (size_t)(done.rows.first + done.r0);
            const int f = done.f0 + wf * kOwnF + (el & (kPieces - 1)) * 8;
            if constexpr (GATED) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (!P.pre) break;
                    auto value = [&](int g, int i, int j, int t) { return acc[h][g][i][j][t]; };
                    if (P.pre_scales) {
                        find_largest(value);
                        emit(n_rows, value, [&](int row, const float *v) {
                            put_e4m3(P.pre, P.pre_scales, row0, row, h * P.features + f, 2 * P.features, v);
                        });
                    } else {
                        emit(n_rows, value, [&](int row, const float *v) {
                            if (f < P.features) put_bf16(P.pre, row0 + row, h * P.features + f, 2 * P.features, v);
                        });
                    }
                }
#pragma unroll
                for (int g = 0; g < kHalves; ++g)
#pragma unroll
                    for (int i = 0; i < kFragsF; ++i)
#pragma unroll
                        for (int j = 0; j < kFragsR; ++j)
#pragma unroll
                            for (int t = 0; t < 4; ++t)
                                acc[0][g][i][j][t] = activate<false>(P.act, acc[0][g][i][j][t], nullptr) * acc[1][g][i][j][t];
                auto value = [&](int g, int i, int j, int t) { return acc[0][g][i][j][t]; };
                if constexpr (E4M3) {
                    find_largest(value);
                    emit(n_rows, value, [&](int row, const float *v) { put_e4m3(P.out, P.out_scales, row0, row, f, P.features, v); });
                } else {
                    emit(n_rows, value, [&](int row, const float *v) {
                        if (f < P.features) put_bf16(P.out, row0 + row, f, P.features, v);
                    });
                }
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    emit(n_rows, [&](int g, int i, int j, int t) { return acc[h][g][i][j][t]; },
                         [&](int row, const float *v) {
                             if (f + h * HALF < P.features) put_bf16(P.out, row0 + row, f + h * HALF, P.features, v);
                         });
            }
        };

        if (!next_place(&tile)) return;
        set_out();
        begin();
        for (;;) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int g = 0; g < kHalves; ++g)
#pragma unroll
                    for (int i = 0; i < kFragsF; ++i)
#pragma unroll
                        for (int j = 0; j < kFragsR; ++j) acc[h][g][i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
            if constexpr (kHalves == 1) one_unit();
            else if (few) one_unit();
            else two_units(One());
            loads_done_and_barrier<0>();           // also those of steps that are none; and the ring is free
            const Place done = tile;
            const bool more = next_place(&tile);
            if (kEarly && more) {
                set_out();
                begin();
            }
            write(done);
            if (!more) break;
            if (!kEarly) {
                __syncthreads();                   // the output is out of the ring
                set_out();
                begin();
            }
        }
    }
};

// What the workgroups share out, in LDS.  Row tiles, or cost, of the call's experts before each: [n + 1]; and the experts
// whose last, short row tile comes behind all others.
struct Shares {
    int before[kMaxExperts + 1];
    unsigned long long short_tile[kMaxExperts / 64];
};
// value(rows of an expert, &whether it has a tile of the second kind): what is summed.
template <int THREADS, class Value>
__device__ inline void scan(const Groups &G, Shares &S, Value value) {
    __shared__ int part[THREADS / kWave];
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    int carry = 0;
    if (tid == 0) S.before[0] = 0;
    for (int base = 0; base < G.n; base += THREADS) {
        int v = 0;
        bool second = false;
        if (base + tid < G.n) v = value(rows_of(G, G.first + base + tid).n, &second);
        const unsigned long long seconds = __ballot(second);
        if (lane == 0 && base + tid < kMaxExperts) S.short_tile[(base + tid) / 64] = seconds;
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
            const int w = __shfl_up(v, o);
            if (lane >= o) v += w;
        }
        if (lane == kWave - 1) part[tid / kWave] = v;
        __syncthreads();
        int mine = carry;
        for (int w = 0; w < THREADS / kWave; ++w) {
            if (w < tid / kWave) mine += part[w];
            carry += part[w];
        }
        if (base + tid < G.n) S.before[base + tid + 1] = mine + v;
        __syncthreads();
    }
}
// Largest i < n with before[i] <= x.
__device__ inline int expert_at(const Shares &S, int n, int x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (S.before[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

constexpr int kRowGroup = 8;                   // row tiles that walk the features together
// An expert of this many row tiles has a last one of at most half the rows behind all others, so that what is left for the last
// turns is short as well; with fewer, whoever reads the weights for the others had better have it, too.
constexpr int kTilesBeforeShort = 4;
constexpr int kTileCost = 8;                   // weight gradient: what begins and ends a tile, in steps of the contraction

template <int FORM, bool E4M3, bool GATED, int ROWS, int HALF>
__global__ __launch_bounds__((Tile<FORM, E4M3, GATED, ROWS, HALF>::kThreads), 2) void expert_tiles_kernel(Groups G, Product P) {
    using T = Tile<FORM, E4M3, GATED, ROWS, HALF>;
    constexpr bool kWeights = FORM == kWeightGradient;
    __shared__ __align__(1024) char lds[T::kLds];
    __shared__ Shares S;
    const int columns = (P.features + T::kOutput - 1) / T::kOutput;
    // Workgroups go to the XCDs in turn.  Each XCD has a share of the tiles, neighbours, whose operands its L2 then holds, and its
    // workgroups take them in turn.
    const int xcd = blockIdx.x % kXcds;
    long long first, whole, first_short = 0, all;      // this XCD's: first tile, number of them, first short one, number of both
    int per_expert = 0;                                // weight gradient: tiles
    if constexpr (kWeights) {
        per_expert = (P.other + ROWS - 1) / ROWS * columns;
        scan<T::kThreads>(G, S, [](int n, bool *) { return (n < 1 << 26 ? (n + 63) / 64 : 1 << 20) + kTileCost; });
        // Shares of equal cost, experts' contractions differ (128 experts of 1 to 1694 rows 464 -> 425 us), begun at whole turns of an
        // XCD's workgroups, since a part of a turn takes as long as a whole one (shares to the tile: 64 experts of 2048 rows
        // 481 -> 496). One grid for all starts keeps them in order. Less than a turn for each: equal numbers.
        auto start = [&](int x) -> long long {
            const long long tiles = (long long)G.n * per_expert, turn = gridDim.x / kXcds;
            if (x == 0 || x == kXcds || tiles < kXcds * turn) return tiles * x / kXcds;
            const long long cost = (long long)S.before[G.n] * x / kXcds;
            const int e = expert_at(S, G.n, (int)cost);
            const long long at = (long long)e * per_expert + (cost - S.before[e]) * per_expert / (S.before[e + 1] - S.before[e]);
            const long long even = (at + turn / 2) / turn * turn;
            return even < tiles ? even : tiles;
        };
        first = start(xcd);
        all = whole = start(xcd + 1) - first;
    } else {
        scan<T::kThreads>(G, S, [](int n, bool *second) {
            *second = ROWS == 256 && n / ROWS >= kTilesBeforeShort && n % ROWS && n % ROWS <= ROWS / 2;
            return n / ROWS + (n % ROWS && !*second);
        });
        const long long tiles = (long long)S.before[G.n] * columns;
        first = tiles * xcd / kXcds;
        all = whole = tiles * (xcd + 1) / kXcds - first;
        if (ROWS == 256) {
            int n = 0;
            for (int w = 0; w * 64 < G.n; ++w) n += __popcll(S.short_tile[w]);
            const long long shorts = (long long)n * columns;
            first_short = shorts * xcd / kXcds;
            all += shorts * (xcd + 1) / kXcds - first_short;
        }
    }
    long long t = blockIdx.x / kXcds;
    T::run(P, lds, [&](typename T::Place *to) {
        for (; t < all; t += gridDim.x / kXcds) {
            int lo, column, row;                       // expert, column of tiles, row of tiles
            if (t < whole) {
                const long long tile = first + t;
                int n_tiles, index;
                if constexpr (kWeights) {
                    lo = (int)(tile / per_expert);
                    n_tiles = per_expert / columns;
                    index = (int)(tile - (long long)lo * per_expert);
                } else {
                    lo = expert_at(S, G.n, (int)(tile / columns));
                    n_tiles = S.before[lo + 1] - S.before[lo];
                    index = (int)(tile - (long long)S.before[lo] * columns);
                }
                const int group = index / (kRowGroup * columns), left = n_tiles - group * kRowGroup;
                const int in_group = left < kRowGroup ? left : kRowGroup, within = index - group * kRowGroup * columns;
                column = within / in_group;
                row = group * kRowGroup + within - column * in_group;
            } else {
                const long long tile = first_short + t - whole;
                int nth = (int)(tile / columns), w = 0;
                column = (int)(tile - (long long)nth * columns);
                unsigned long long have = S.short_tile[0];
                for (int n; nth >= (n = __popcll(have)) && (w + 1) * 64 < G.n; have = S.short_tile[++w]) nth -= n;
                for (; nth > 0; --nth) have &= have - 1;
                lo = w * 64 + __ffsll(have) - 1;
                row = -1;
            }
            if (lo < 0) continue;
            const int e = G.first + __builtin_amdgcn_readfirstlane(lo);
            const Rows found = rows_of(G, e), rows = {same_in_wave(found.first), __builtin_amdgcn_readfirstlane(found.n)};
            if (row < 0) row = rows.n / ROWS;
            // (tables that claim more rows than there can be may have wrapped the sums)
            if ((unsigned)column >= (unsigned)columns || row < 0 || (long long)row * ROWS >= (kWeights ? P.other : rows.n)) continue;
            *to = {e, rows, __builtin_amdgcn_readfirstlane(column) * T::kOutput, __builtin_amdgcn_readfirstlane(row) * ROWS};
            t += gridDim.x / kXcds;
            return true;
        }
        return false;
    });
}

// ---------------------------------------------------------------- the gated block's own gradient
// dg = dh u act'(g), du = dh act(g) from the kept pre-activations, rounded to bf16 for the matrix products behind (they
// take bf16 operands; the rounding is of the size of the results' own); h = act(g) u again where asked for.  Bound by
// memory: three rows of inter read, two (three) written, 32768 x 1024 in bf16 57 us, 5.9 TB/s.  pre and dpre may be the same rows.
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
