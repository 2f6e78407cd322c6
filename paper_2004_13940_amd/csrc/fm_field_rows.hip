// Rows against the candidates: statistics of the softmax, the largest logit of every group, and for distillation the sum of
// the candidates weighted by their probabilities.
#include "fm_field_tiles.h"

namespace {

// A wavefront takes 16 NT rows and a part of the candidates, 16 of them at a time.  The tile of logits has candidates down
// and rows across, so that a lane has four candidates of one row of every 16: maxima and sums stay in the lane, and the tile
// is the B operand of the second product (candidates are what it sums over) as it stands.
// The reference m of the exponentials follows the maximum only when that has risen by more than 2^8 over it.
template <typename TV, int KC, bool FULL, int NT, bool DISTILL>
__global__ __launch_bounds__(FM_BLOCK, 2) void k_field_rows(const FieldArgs A)
{
    constexpr int KP = 16 * KC;
    const int lane = threadIdx.x % 64, lo = lane % 16, g = lane / 16;
    const int64_t item = (int64_t)blockIdx.x * FM_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    if constexpr (DISTILL) {  // the bits that the next kernel sets
        const int64_t words = (int64_t)(A.npad / 16) * A.hit_words;
        for (int64_t i = (int64_t)blockIdx.x * FM_BLOCK + threadIdx.x; i < words; i += (int64_t)gridDim.x * FM_BLOCK) A.hits[i] = 0;
    }
    if (item >= (int64_t)A.row_tiles * A.splits) return;
    const int split = (int)(item / A.row_tiles), row0 = (int)(item % A.row_tiles) * 16 * NT;
    const int64_t beg = split * A.chunk, end = min(A.C, beg + A.chunk);
    const TV* V = static_cast<const TV*>(A.V);

    float b[NT][KC][4];
    int64_t mask_row[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int64_t row = min(row0 + 16 * t + lo, A.n - 1);
        mask_row[t] = row * A.mask_stride;
#pragma unroll
        for (int c = 0; c < KC; ++c) load4<float, FULL>(A.G + row * A.g_stride, 16 * c + 4 * g, A.K, b[t][c]);
    }
    float m[NT], S[NT], U[NT];
    f32x4 o[DISTILL ? KC : 1][NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        m[t] = -3e38f;
        S[t] = U[t] = 0.f;
#pragma unroll
        for (int c = 0; c < (DISTILL ? KC : 1); ++c) o[c][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    for (int64_t j0 = beg; j0 < end; j0 += FM_GROUP) {
        f32x4 z[4][NT];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float a[KC][4];
            const TV* v = V + min(j0 + 16 * i + lo, A.C - 1) * A.v_stride;
#pragma unroll
            for (int c = 0; c < KC; ++c) load4<TV, FULL>(v, 16 * c + 4 * g, A.K, a[c]);
            f32x4 w = {0.f, 0.f, 0.f, 0.f};
            if (A.w != nullptr)
#pragma unroll
                for (int r = 0; r < 4; ++r) w[r] = A.w[min(j0 + 16 * i + 4 * g + r, A.C - 1)];
#pragma unroll
            for (int t = 0; t < NT; ++t) z[i][t] = w;
#pragma unroll
            for (int c = 0; c < KC; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int t = 0; t < NT; ++t) z[i][t] = mfma4(a[c][e], b[t][c][e], z[i][t]);
        }
        if (A.mask != nullptr || j0 + FM_GROUP > end) {
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                uint32_t bits[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int64_t left = end - j0 - 32 * h;
                    bits[h] = left <= 0 ? 0u : left < 32 ? (1u << left) - 1u : ~0u;
                    if (A.mask != nullptr && left > 0) bits[h] &= A.mask[mask_row[t] + (j0 >> 5) + h];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t four = bits[i / 2] >> (16 * (i % 2) + 4 * g);
#pragma unroll
                    for (int r = 0; r < 4; ++r) z[i][t][r] = four >> r & 1u ? z[i][t][r] : -INFINITY;
                }
            }
        }
        float top[NT];
        bool rise = false;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            float x = fmaxf(fmaxf(z[0][t][0], z[0][t][1]), z[0][t][2]);
            x = fmaxf(fmaxf(x, z[0][t][3]), z[1][t][0]);
            x = fmaxf(fmaxf(x, z[1][t][1]), z[1][t][2]);
            x = fmaxf(fmaxf(x, z[1][t][3]), z[2][t][0]);
            x = fmaxf(fmaxf(x, z[2][t][1]), z[2][t][2]);
            x = fmaxf(fmaxf(x, z[2][t][3]), z[3][t][0]);
            x = fmaxf(fmaxf(x, z[3][t][1]), z[3][t][2]);
            top[t] = fmaxf(x, z[3][t][3]);
            rise |= top[t] * A.sl > m[t] + 8.f;
        }
        if (!DISTILL && A.gmax != nullptr) {
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                float x = fmaxf(top[t], fm_xor_lane<16>(top[t]));
                x = fmaxf(x, fm_xor_lane<32>(x));
                const int row = row0 + 16 * t + lo;
                if (g == 0 && row < A.n) A.gmax[row * A.ngroups + j0 / FM_GROUP] = x;
            }
        }
        if (__any(rise)) {
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                float to = fmaxf(m[t], top[t] * A.sl);
                if constexpr (DISTILL) {  // the four lanes of a row share its sums of candidates
                    to = fmaxf(to, fm_xor_lane<16>(to));
                    to = fmaxf(to, fm_xor_lane<32>(to));
                }
                const float d = m[t] - to, f = __builtin_amdgcn_exp2f(d);
                if constexpr (!DISTILL) U[t] = f > 0.f ? f * (U[t] + d * S[t]) : 0.f;
                S[t] *= f;
                m[t] = to;
                if constexpr (DISTILL)
#pragma unroll
                    for (int c = 0; c < KC; ++c)
#pragma unroll
                        for (int r = 0; r < 4; ++r) o[c][t][r] *= f;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float x = fmaf(z[i][t][r], A.sl, -m[t]), e = __builtin_amdgcn_exp2f(x);
                    S[t] += e;
                    if constexpr (DISTILL)
                        z[i][t][r] = e;
                    else
                        U[t] = fmaf(e, fmaxf(x, -200.f), U[t]);  // e is 0 where x is -infinity
                }
            if constexpr (DISTILL) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const TV* v = V + min(j0 + 16 * i + 4 * g + r, A.C - 1) * A.v_stride;
#pragma unroll
                    for (int c = 0; c < KC; ++c) {
                        // what is left out has probability 0, which is to stay 0 whatever its values are
                        const float a = finite(FULL || 16 * c + lo < A.K ? fm_field_value(v + 16 * c + lo) : 0.f);
#pragma unroll
                        for (int t = 0; t < NT; ++t) o[c][t] = mfma4(a, z[i][t][r], o[c][t]);
                    }
                }
            }
        }
    }

#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int row = row0 + 16 * t + lo;
        FieldPart p = {m[t], S[t], U[t]};
        p = fm_field_merge(p, {fm_xor_lane<16>(p.m), fm_xor_lane<16>(p.S), fm_xor_lane<16>(p.U)});
        p = fm_field_merge(p, {fm_xor_lane<32>(p.m), fm_xor_lane<32>(p.S), fm_xor_lane<32>(p.U)});
        if (row >= A.n) continue;
        const int64_t at = (int64_t)split * A.n + row;
        if (g == 0) A.part[at] = make_float4(p.m, p.S, p.U, 0.f);
        if constexpr (DISTILL)
#pragma unroll
            for (int c = 0; c < KC; ++c) *reinterpret_cast<f32x4*>(A.opart + at * KP + 16 * c + 4 * g) = o[c][t];
    }
}

template <typename TV, int KC, bool FULL, int NT, bool DISTILL>
void launch(const FieldArgs& A, hipStream_t st)
{
    const int64_t items = (int64_t)A.row_tiles * A.splits;
    k_field_rows<TV, KC, FULL, NT, DISTILL><<<(uint32_t)((items + FM_WAVES - 1) / FM_WAVES), FM_BLOCK, 0, st>>>(A);
}

template <bool DISTILL>
void rows(int32_t v_type, const FieldArgs& A, hipStream_t st)
{
    fm_field_shape(v_type, A.K, [&](auto type, auto kc, auto full) {
        using TV = decltype(type);
        constexpr int KC = decltype(kc)::value;
        constexpr bool FULL = decltype(full)::value;
        if (A.n <= 16) return launch<TV, KC, FULL, 1, DISTILL>(A, st);
        launch<TV, KC, FULL, fm_field_row_tiles(KC, DISTILL), DISTILL>(A, st);
    });
}

}  // namespace

int fm_field_rows_per_wave(bool distill, int32_t K, int64_t n)
{
    return n <= 16 ? 16 : 16 * fm_field_row_tiles(fm_field_chunks(K), distill);
}

void fm_field_rows(bool distill, int32_t v_type, const FieldArgs& A, hipStream_t st)
{
    if (distill)
        rows<true>(v_type, A, st);
    else
        rows<false>(v_type, A, st);
}
