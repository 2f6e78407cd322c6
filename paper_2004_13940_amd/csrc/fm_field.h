// Shared by the kernels over the candidates of a field and their entry points.
#pragma once

#include "fm_device.h"

// Best candidates are found by way of the largest logit of every FM_GROUP candidates: of the `top` groups with the largest
// ones (lower groups first among equal ones) every other candidate is behind `top` better ones.  FM_GROUPS such groups
// make one of a second level.
constexpr int FM_GROUP = 64;
constexpr int FM_GROUPS = 64;
constexpr int FM_FIELD_TOP = 64;

constexpr float FM_LOG2E = 1.44269504088896340736f, FM_LN2 = 0.69314718055994530942f;

// Statistics of a part of a row's candidates: reference m, S = sum 2^(x - m), U = sum 2^(x - m) (x - m), with
// x = scale log2(e) z.  S = 0: no allowed candidate.
struct FieldPart {
    float m, S, U;
};

__device__ __forceinline__ FieldPart fm_field_merge(FieldPart a, FieldPart b)
{
    if (b.S == 0.f) return a;  // not so if S is NaN
    if (a.S == 0.f) return b;
    FieldPart r;
    r.m = fmaxf(a.m, b.m);
    const float da = a.m - r.m, db = b.m - r.m;
    const float fa = __builtin_amdgcn_exp2f(da), fb = __builtin_amdgcn_exp2f(db);
    r.S = fa * a.S + fb * b.S;
    // 0 times -infinity (a part 2^200 below the other) must not become NaN
    r.U = (fa > 0.f ? fa * (a.U + da * a.S) : 0.f) + (fb > 0.f ? fb * (b.U + db * b.S) : 0.f);
    return r;
}

struct FieldArgs {
    const void* V;
    const float* w;
    const uint32_t* mask;
    int64_t v_stride, mask_stride;
    const float* G;
    int64_t g_stride;
    int64_t C;
    int32_t n, K;
    float scale, sl;  // sl = scale log2(e)
    // rows against parts of the candidates
    int32_t row_tiles, splits;
    int64_t chunk;    // candidates to a split, a multiple of FM_GROUP
    float4* part;     // [splits][n] FieldPart
    float* opart;     // [splits][n][KP] sum 2^(x - m) v_j (distillation)
    float* gmax;      // [n][ngroups] largest logit of every group, or nullptr
    int64_t ngroups;
    // logprobs
    const int32_t* ids;
    float *logprob, *lse, *entropy, *top_logprob;
    int32_t* top_ids;
    int32_t T, top;
    // distillation
    const float *teacher, *weight;
    float *loss, *grad_G, *grad_V, *grad_w;
    int32_t npad;     // n in whole tiles of 16 rows
    float* rm;        // [npad] reference m of the row's exponentials
    float* rs;        // [npad] weight scale / S; 0: no part in the gradient
    float2* rq;       // [npad] largest scaled teacher logit; S / Q, the share of the teacher in units of the exponentials
    float* g0;        // [npad][KP] G, 0 for rows without a part in the gradient, NaN for rows that are NaN
    float* gs;        // [npad][KP] rs G, finite
    uint32_t* hits;   // [npad / 16][hit_words] blocks of 2^hit_shift candidates that some row of the tile names
    int32_t hit_words, hit_shift;
    int32_t col_tiles, row_splits, row_chunk;  // candidates against parts of the rows, multiples of 16 rows
    float* vpart;     // [row_splits][C][KP] parts of grad_V, and [row_splits][C] of grad_w
    float* wpart;
};

__device__ __forceinline__ float fm_field_value(const float* p) { return *p; }
__device__ __forceinline__ float fm_field_value(const _Float16* p) { return (float)*p; }
__device__ __forceinline__ float fm_field_value(const __bf16* p) { return (float)*p; }

__device__ __forceinline__ bool fm_field_allowed(const FieldArgs& A, int64_t row, int64_t j)
{
    return A.mask == nullptr || (A.mask[row * A.mask_stride + (j >> 5)] >> (j & 31) & 1u) != 0;
}

// Logit of candidate j in a row: -infinity where it is not allowed.
template <typename TV>
__device__ __forceinline__ float fm_field_logit(const FieldArgs& A, int64_t row, const float* g, int64_t j)
{
    if (!fm_field_allowed(A, row, j)) return -INFINITY;
    const TV* v = static_cast<const TV*>(A.V) + j * A.v_stride;
    float z = A.w != nullptr ? A.w[j] : 0.f;
    for (int k = 0; k < A.K; ++k) z = fmaf(g[k], fm_field_value(v + k), z);
    return z;
}
