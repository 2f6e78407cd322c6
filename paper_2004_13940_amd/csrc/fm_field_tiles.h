// Tiles of 16 x 16 logits on the matrix cores (v_mfma_f32_16x16x4_f32: full fp32 products and sums).
//
// Operand layout of C[16 x 16] += A[16 x 4] B[4 x 16] over the 64 lanes of a wavefront, lo = lane % 16, g = lane / 16:
//   A: A[lo][g];   B: B[g][lo];   C: register r holds C[4 g + r][lo].
// The order in which a product runs through k is free as long as both operands have the same: step e of chunk c takes
// k = 16 c + 4 g + e, so that a lane reads four consecutive values of a row.
#pragma once

#include <float.h>

#include "fm_field.h"

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4_unaligned __attribute__((ext_vector_type(4), aligned(4)));
typedef _Float16 f16x4_unaligned __attribute__((ext_vector_type(4), aligned(2)));
typedef __bf16 bf16x4_unaligned __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ f32x4 mfma4(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// The nearest finite value: times a probability of 0 it is 0.
__device__ __forceinline__ float finite(float v) { return __builtin_amdgcn_fmed3f(v, -FLT_MAX, FLT_MAX); }

template <typename T> struct Unaligned4;
template <> struct Unaligned4<float> { using type = f32x4_unaligned; };
template <> struct Unaligned4<_Float16> { using type = f16x4_unaligned; };
template <> struct Unaligned4<__bf16> { using type = bf16x4_unaligned; };

// Values k..k+3 of a row of K; 0 beyond.  FULL: there is nothing beyond.
template <typename T, bool FULL>
__device__ __forceinline__ void load4(const T* row, int k, int K, float (&v)[4])
{
    if constexpr (FULL) {
        const auto x = *reinterpret_cast<const typename Unaligned4<T>::type*>(row + k);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (float)x[e];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = k + e < K ? (float)row[k + e] : 0.f;
    }
}

// Chunks of 16 latent values that the kernels for K have: 1, 2, 4, 8 or 16.
constexpr int fm_field_chunks(int32_t K) { return K <= 16 ? 1 : K <= 32 ? 2 : K <= 64 ? 4 : K <= 128 ? 8 : 16; }
// Tiles of 16 rows, or of 16 candidates, that stay in a wavefront's registers: 256 of them are to do.
constexpr int fm_field_row_tiles(int KC, bool distill) { return KC <= (distill ? 2 : 4) ? 4 : KC <= 8 ? 2 : 1; }
constexpr int fm_field_col_tiles(int KC) { return KC <= 4 ? 4 : KC == 8 ? 2 : 1; }

template <int V> using IntC = std::integral_constant<int, V>;

// Calls run(a value of V's type, chunks, whether K fills them).
template <typename F>
void fm_field_shape(int32_t v_type, int32_t K, F run)
{
    const auto by_k = [&](auto type) {
        const int kc = fm_field_chunks(K);
        const bool full = K == 16 * kc;
        const auto of = [&](auto chunks) { full ? run(type, chunks, std::true_type{}) : run(type, chunks, std::false_type{}); };
        switch (kc) {
            case 1: return of(IntC<1>{});
            case 2: return of(IntC<2>{});
            case 4: return of(IntC<4>{});
            case 8: return of(IntC<8>{});
            default: return of(IntC<16>{});
        }
    };
    switch (v_type) {
        case FM_TYPE_F16: return by_k(_Float16{});
        case FM_TYPE_BF16: return by_k(__bf16{});
        default: return by_k(float{});
    }
}

int fm_field_rows_per_wave(bool distill, int32_t K, int64_t n);
void fm_field_rows(bool distill, int32_t v_type, const FieldArgs& A, hipStream_t st);
int fm_field_cols_per_wave(int32_t K);
void fm_field_cols(int32_t v_type, const FieldArgs& A, hipStream_t st);
