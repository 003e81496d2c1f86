// Host side of the experts' products: argument checks and launches.  No context, no workspace, nothing kept.
// (Part of flmoe.hip.)
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <initializer_list>

#include "../../include/flmoe.h"
#include "kernels_experts.h"

namespace flmoe {
namespace experts {

constexpr int kMaxWidth = 1 << 20;             // as fl_moe_config.hidden
constexpr int kUnits = 256;                    // compute units of the part

// What a call's configuration and tables come to.
inline int groups_of(const fl_moe_config *cfg, int rank_begin, int rank_count, const int32_t *expert_off,
              const int32_t *tokens_per_expert, Groups *G) {
    fl_moe_sizes sizes;
    const int e = fl_moe_query_sizes(cfg, &sizes);
    if (e != FL_OK) return e;
    if (rank_begin < 0 || rank_count < 1 || rank_count > cfg->n_ranks - rank_begin) return FL_ERR_INVALID_ARG;
    if (!expert_off || !tokens_per_expert) return FL_ERR_INVALID_ARG;
    if (((uintptr_t)expert_off & 3) || ((uintptr_t)tokens_per_expert & 3)) return FL_ERR_ALIGNMENT;
    const int El = cfg->n_experts / cfg->n_ranks;
    *G = Groups{El, rank_begin * El, rank_count * El, sizes.expert_capacity_rows, expert_off, tokens_per_expert};
    return FL_OK;
}

inline long long mean_rows(const fl_moe_config *cfg, const Groups &G) {
    return std::max(1ll, (long long)cfg->max_tokens * cfg->top_k / G.El);
}

inline int check_width(int width, int multiple) {
    if (width < 1 || width > kMaxWidth) return FL_ERR_INVALID_ARG;
    return width % multiple ? FL_ERR_ALIGNMENT : FL_OK;
}

// Every pointer there and 16-byte aligned (scales: 4).
inline int check_tensors(std::initializer_list<const void *> rows, std::initializer_list<const float *> scales = {}) {
    for (const void *p : rows) if (!p) return FL_ERR_INVALID_ARG;
    for (const float *p : scales) if (!p) return FL_ERR_INVALID_ARG;
    for (const void *p : rows) if ((uintptr_t)p & 15) return FL_ERR_ALIGNMENT;
    for (const float *p : scales) if ((uintptr_t)p & 3) return FL_ERR_ALIGNMENT;
    return FL_OK;
}

inline int compute_units() {
    static std::atomic<int> known[64];
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return kUnits;
    n = known[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1) n = kUnits;
        known[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

inline int launched() { return hipGetLastError() == hipSuccess ? FL_OK : FL_ERR_HIP; }

// mean: rows an expert would have if the tokens of the configuration were spread evenly.
// Experts of few rows are bound by the reading of their weights; smaller tiles leave less of the machine idle at the beginning
// and the end of each and spread few experts over more compute units.  A real routing scatters the counts round their mean, and an
// expert with one row more than a tile has its weights read twice, which is why the lines lie below 32 and 64.  us with a random
// top 8 of 128 experts of 2 x 768 x 2048 in bf16, tiles of 32, 64 and 256 rows, gated block and product behind:
//   mean 16  140 / 78,  142 / 78,  144 / 86      40  182 / 103, 146 / 88, 148 / 88
//        20  154 / 84,  143 / 79,  146 / 86      48  193 / 106, 160 / 96, 151 / 88
//        32  158 / 92,  146 / 85,  147 / 87      64  212 / 117, 184 / 107, 155 / 91
// e4m3, the product of 64 experts of 4096 x 2048: 16 rows 104, 110, 113; 24 110, 108, 111; 40 135, 114, 113; 48 141, 121, 114; the
// gated block there, in tiles of 64 and 256: 40 194, 205; 48 219, 207.
constexpr long long kRowsFor32 = 16, kRowsFor64 = 40;
// Workgroups of small tiles on a compute unit: what is on its way to one is best 64 to 96 KB (32 KB each); the third pays where a
// tile is short.  us with two and with three, 128 experts, tiles of 32 rows: bf16, 2048 outputs, 512 long 49 and 44, 1024 103 and
// 102, 1792 166 and 167; e4m3, 4096 outputs, 512 63 and 55, 1024 114 and 108, 2048 200 and 202 (64 experts of
// 7168 x 2048, both products, 4 rows: 474 and 467).  Tiles of 64 rows: bf16, 512 52 and 48, 768 87 and 88; e4m3 never (768 103 and 118,
// 2048 223 and 252).
constexpr int kShortBytes = 2048;

template <int FORM, bool E4M3, bool GATED>
int launch_tiles(const Groups &G, long long mean, const Product &P, hipStream_t st) {
    using std::integral_constant;
    const int units = std::max(1, compute_units() / kXcds) * kXcds;
    auto go = [&](auto rows, auto half, int per_unit) {
        using T = Tile<FORM, E4M3, GATED, rows(), half()>;
        expert_tiles_kernel<FORM, E4M3, GATED, rows(), half()><<<dim3(units * per_unit), dim3(T::kThreads), 0, st>>>(G, P);
        return launched();
    };
    if constexpr (FORM == kForward) {
        if constexpr (GATED) {                     // what answers in blocks of 128 features has them in one tile
            if (mean <= kRowsFor64 && (E4M3 || P.pre_scales))
                return go(integral_constant<int, 64>(), integral_constant<int, 128>(), 1);
        }
        if constexpr (!(E4M3 && GATED)) {
            const bool small = P.k * (E4M3 ? 1 : 2) <= kShortBytes;
            if (mean <= kRowsFor32) return go(integral_constant<int, 32>(), integral_constant<int, 64>(), small ? 3 : 2);
            if (mean <= kRowsFor64) return go(integral_constant<int, 64>(), integral_constant<int, 64>(), small && !E4M3 ? 3 : 2);
        }
    }
    return go(integral_constant<int, 256>(), integral_constant<int, 128>(), 1);
}

// y = x W^T, W [experts][out][in]
inline Product forward(const void *x, const void *w, void *y, int in, int out) {
    Product P = {};
    P.a = (const char *)w; P.b = (const char *)x; P.out = y;
    P.a_ld = P.b_ld = 2 * in;
    P.a_expert = (long long)out * in * 2;
    P.features = out; P.k = in;
    return P;
}
// dx = dy W
inline Product row_gradient(const void *dy, const void *w, void *dx, int in, int out) {
    Product P = {};
    P.a = (const char *)w; P.b = (const char *)dy; P.out = dx;
    P.a_ld = 2 * in; P.b_ld = 2 * out;
    P.a_expert = (long long)out * in * 2;
    P.features = in; P.k = out;
    return P;
}
// dW = dy^T x
inline Product weight_gradient(const void *dy, const void *x, void *dw, int in, int out) {
    Product P = {};
    P.a = (const char *)x; P.b = (const char *)dy; P.out = dw;
    P.a_ld = 2 * in; P.b_ld = 2 * out;
    P.features = in; P.other = out;
    return P;
}

#define FL_CHECK(call) do { const int code = (call); if (code != FL_OK) return code; } while (0)

}  // namespace experts
}  // namespace flmoe

extern "C" {

int fl_moe_expert_gated(const fl_moe_config *cfg, int rb, int rc, const int32_t *expert_off, const int32_t *tokens_per_expert,
                        int inter, int activation, const void *x, const void *w, void *h, void *pre, float *pre_scales,
                        void *stream) {
    using namespace flmoe::experts;
    Groups G;
    FL_CHECK(groups_of(cfg, rb, rc, expert_off, tokens_per_expert, &G));
    FL_CHECK(check_width(inter, pre_scales ? 128 : 8));
    if (activation != FL_ACT_SILU && activation != FL_ACT_GELU) return FL_ERR_INVALID_ARG;
    if (pre_scales && !pre) return FL_ERR_INVALID_ARG;
    FL_CHECK(check_tensors({x, w, h}));
    if (((uintptr_t)pre & 15) || ((uintptr_t)pre_scales & 3)) return FL_ERR_ALIGNMENT;
    Product P = forward(x, w, h, cfg->hidden, inter);
    P.a_expert *= 2;
    P.pre = pre; P.pre_scales = pre_scales; P.act = activation;
    return launch_tiles<kForward, false, true>(G, mean_rows(cfg, G), P, (hipStream_t)stream);
}

int fl_moe_expert_gated_backward(const fl_moe_config *cfg, int rb, int rc, const int32_t *expert_off,
                                 const int32_t *tokens_per_expert, int inter, int activation, const void *x, const void *w,
                                 const void *pre, const float *pre_scales, const void *dh, void *dpre, void *dx, void *dw,
                                 void *h, void *stream) {
    using namespace flmoe::experts;
    Groups G;
    FL_CHECK(groups_of(cfg, rb, rc, expert_off, tokens_per_expert, &G));
    FL_CHECK(check_width(inter, pre_scales ? 128 : 8));
    if (activation != FL_ACT_SILU && activation != FL_ACT_GELU) return FL_ERR_INVALID_ARG;
    FL_CHECK(check_tensors({pre, dh, dpre}));
    if ((dx && !w) || (dw && !x) || (pre_scales && dpre == pre)) return FL_ERR_INVALID_ARG;
    if (((uintptr_t)x | (uintptr_t)w | (uintptr_t)dx | (uintptr_t)dw | (uintptr_t)h) & 15 || (uintptr_t)pre_scales & 3)
        return FL_ERR_ALIGNMENT;
    hipStream_t st = (hipStream_t)stream;
    const long long mean = mean_rows(cfg, G);
    const long long blocks = std::min(std::max(1ll, (mean * (inter / 8) + 1023) / 1024), (1ll << 18) / G.n);
    expert_gated_gradient_kernel<<<dim3((unsigned)blocks, G.n), dim3(256), 0, st>>>(
        G, inter, activation, (const char *)pre, pre_scales, (const char *)dh, (char *)dpre, (char *)h);
    FL_CHECK(launched());
    if (dx) FL_CHECK((launch_tiles<kRowGradient, false, false>(G, 0, row_gradient(dpre, w, dx, cfg->hidden, 2 * inter), st)));
    if (dw) FL_CHECK((launch_tiles<kWeightGradient, false, false>(G, 0, weight_gradient(dpre, x, dw, cfg->hidden, 2 * inter), st)));
    return FL_OK;
}

int fl_moe_expert_product(const fl_moe_config *cfg, int rb, int rc, const int32_t *expert_off, const int32_t *tokens_per_expert,
                          int in, int out, const void *x, const void *w, void *y, void *stream) {
    using namespace flmoe::experts;
    Groups G;
    FL_CHECK(groups_of(cfg, rb, rc, expert_off, tokens_per_expert, &G));
    FL_CHECK(check_width(in, 8));
    FL_CHECK(check_width(out, 8));
    FL_CHECK(check_tensors({x, w, y}));
    return launch_tiles<kForward, false, false>(G, mean_rows(cfg, G), forward(x, w, y, in, out), (hipStream_t)stream);
}

int fl_moe_expert_product_backward(const fl_moe_config *cfg, int rb, int rc, const int32_t *expert_off,
                                   const int32_t *tokens_per_expert, int in, int out, const void *x, const void *w,
                                   const void *dy, void *dx, void *dw, void *stream) {
    using namespace flmoe::experts;
    Groups G;
    FL_CHECK(groups_of(cfg, rb, rc, expert_off, tokens_per_expert, &G));
    FL_CHECK(check_width(in, 8));
    FL_CHECK(check_width(out, 8));
    FL_CHECK(check_tensors({dy}));
    if ((!dx && !dw) || (dx && !w) || (dw && !x)) return FL_ERR_INVALID_ARG;
    if (((uintptr_t)x | (uintptr_t)w | (uintptr_t)dx | (uintptr_t)dw) & 15) return FL_ERR_ALIGNMENT;
    hipStream_t st = (hipStream_t)stream;
    if (dx) FL_CHECK((launch_tiles<kRowGradient, false, false>(G, 0, row_gradient(dy, w, dx, in, out), st)));
    if (dw) FL_CHECK((launch_tiles<kWeightGradient, false, false>(G, 0, weight_gradient(dy, x, dw, in, out), st)));
    return FL_OK;
}

int fl_moe_expert_gated_e4m3(const fl_moe_config *cfg, int rb, int rc, const int32_t *expert_off,
                             const int32_t *tokens_per_expert, int inter, int activation, const void *x, const float *x_scales,
                             const void *w, const float *w_scales, void *h, float *h_scales, void *stream) {
    using namespace flmoe::experts;
    Groups G;
    FL_CHECK(groups_of(cfg, rb, rc, expert_off, tokens_per_expert, &G));
    FL_CHECK(check_width(inter, 128));
    FL_CHECK(check_width(cfg->hidden, 128));
    if (activation != FL_ACT_SILU && activation != FL_ACT_GELU) return FL_ERR_INVALID_ARG;
    FL_CHECK(check_tensors({x, w, h}, {x_scales, w_scales, h_scales}));
    Product P = {};
    P.a = (const char *)w; P.b = (const char *)x; P.a_scales = w_scales; P.b_scales = x_scales;
    P.out = h; P.out_scales = h_scales; P.act = activation;
    P.a_ld = P.b_ld = P.k = cfg->hidden;
    P.features = inter;
    P.a_expert = 2ll * inter * cfg->hidden;
    return launch_tiles<kForward, true, true>(G, mean_rows(cfg, G), P, (hipStream_t)stream);
}

int fl_moe_expert_product_e4m3(const fl_moe_config *cfg, int rb, int rc, const int32_t *expert_off,
                               const int32_t *tokens_per_expert, int in, int out, const void *x, const float *x_scales,
                               const void *w, const float *w_scales, void *y, void *stream) {
    using namespace flmoe::experts;
    Groups G;
    FL_CHECK(groups_of(cfg, rb, rc, expert_off, tokens_per_expert, &G));
    FL_CHECK(check_width(in, 128));
    FL_CHECK(check_width(out, 8));
    FL_CHECK(check_tensors({x, w, y}, {x_scales, w_scales}));
    Product P = {};
    P.a = (const char *)w; P.b = (const char *)x; P.a_scales = w_scales; P.b_scales = x_scales;
    P.out = y;
    P.a_ld = P.b_ld = P.k = in;
    P.features = out;
    P.a_expert = (long long)out * in;
    return launch_tiles<kForward, true, false>(G, mean_rows(cfg, G), P, (hipStream_t)stream);
}

}  // extern "C"
