// Few rows (up to 16): every product is bound by reading the class weights and writing their gradient, so the weights are read where
// they lie, by every wavefront its own classes, and D (16 fp32 values per class) is kept.  1 x 1024 against 32,768 bfloat16 classes: scores 13.5 us,
// 5 TB/s.  Gradients of 1 x 4096 against 32,000, with the scores made again: 192 us, 4.1 TB/s.
#pragma once
#include "product_device.h"

namespace qgbdt {

constexpr int FEW_ROWS = 16;

struct FewArgs {
    const uint16_t* x;  // rows of dp values in pieces, as they are laid out for the products
    int64_t x_ld, x_piece;
    const void* w;
    int64_t w_ld;
    int n, dim;
    int64_t n_classes;
    int parts;
    float2* part;       // scores for the loss: [n][workgroups] maximum and sum of exponentials, or
    float* d;           // D: [n][d_ld]
    int64_t d_ld;
    const float *lse, *weight, *common;
    const void* target;
    int target_bytes;
};

__device__ __forceinline__ int64_t target_of(const void* t, int bytes, int64_t i, int64_t n_classes) {
    const int64_t v = bytes == 8 ? static_cast<const int64_t*>(t)[i] : (int64_t)static_cast<const int32_t*>(t)[i];
    return v >= 0 && v < n_classes ? v : -1;
}

// nearest of 8 bits; a finite value never becomes infinite
__device__ __forceinline__ uint16_t piece_of(float v) {
    const uint16_t b = to_bf16(v);
    return (b & 0x7fffu) == 0x7f80u && fabsf(v) < __builtin_inff() ? (uint16_t)(__float_as_uint(v) >> 16) : b;
}
__device__ __forceinline__ void three_pieces(float v, uint16_t* q) {
    q[0] = piece_of(v);
    const float r1 = v - from_bf16(q[0]);
    const bool finite = fabsf(v) < __builtin_inff();
    q[1] = finite ? to_bf16(r1) : 0x7fc0;  // (an infinity: NaN, so that its scores are NaN whatever the signs of the other's pieces)
    q[2] = finite ? to_bf16(r1 - from_bf16(q[1])) : 0;
}

// As three_pieces(), of eight values: two are rounded by one instruction, and the first piece is kept finite by a bound before it, not by a check
// after it (infinities become NaN with their second piece).
__device__ __forceinline__ void eight_in_pieces(const float* v, bf16x8* out) {
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    constexpr float MOST = 3.3895313892515355e38f;  // of bfloat16
    union { uint32_t u[4]; bf16x8 v; } o[3];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        f32x2 r = {v[2 * h], v[2 * h + 1]};
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            const f32x2 held = {__builtin_amdgcn_fmed3f(r[0], -MOST, MOST), __builtin_amdgcn_fmed3f(r[1], -MOST, MOST)};
            o[p].u[h] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p == 0 ? held : r, bf16x2));
            if (p < 2) r = f32x2{r[0] - __uint_as_float(o[p].u[h] << 16), r[1] - __uint_as_float(o[p].u[h] & 0xffff0000u)};
        }
    }
#pragma unroll
    for (int p = 0; p < 3; ++p) out[p] = o[p].v;
}

// 8 values of a row of weights from k on, as they come from memory; zeros beyond the row's end
template <class E>
struct Eight {
    Piece<E> q[8 / E::PER16];
};
template <class E>
__device__ __forceinline__ Eight<E> load_eight(const typename E::T* row, int k, int dim) {
    Eight<E> v;
    if (k + 8 <= dim) {
#pragma unroll
        for (int h = 0; h < 8 / E::PER16; ++h) __builtin_memcpy(&v.q[h], row + k + h * E::PER16, 16);
    } else {
#pragma unroll
        for (int h = 0; h < 8; ++h) v.q[h / E::PER16].v[h % E::PER16] = k + h < dim ? row[k + h] : E::put(0.0f);
    }
    return v;
}

// Scores of all rows against 16 classes per wavefront and turn (parts = 1), or per workgroup, whose wavefronts share the rows' values
// (parts = 4: few classes); a lane has row lane % 16 and classes 4 (lane / 16) + 0..3.
template <class E, int PIECES, bool GRAD>
__global__ __launch_bounds__(256) void few_scores_kernel(FewArgs a) {
    constexpr int U = 4;  // steps of 32 values whose loads are under way together
    __shared__ float2 both[4][FEW_ROWS];
    __shared__ float4 acc_of[3][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, s = lane & 15;
    const int64_t blocks = (a.n_classes + 15) / 16, waves = (int64_t)gridDim.x * 4;
    const uint16_t* const xr = a.x + (int64_t)(s < a.n ? s : a.n - 1) * a.x_ld;
    const int dp = (a.dim + 7) / 8 * 8;
    float u = 0.0f, b = 0.0f;
    int64_t t = -1;
    if (GRAD && s < a.n) {
        t = target_of(a.target, a.target_bytes, s, a.n_classes);
        if (t >= 0) u = a.weight[s] / *a.common;
        if (u != 0.0f) b = -a.lse[s] * LOG2E;
    }
    float top = -__builtin_inff(), sum = 0.0f;
    for (int64_t block = a.parts > 1 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + wave; block < blocks; block += a.parts > 1 ? (int64_t)gridDim.x : waves) {
        const int64_t c0 = block * 16, c = c0 + s;
        const typename E::T* const wr = static_cast<const typename E::T*>(a.w) + (c < a.n_classes ? c : a.n_classes - 1) * a.w_ld;
        f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int k0 = a.parts > 1 ? wave * 32 * U : 0; k0 < a.dim; k0 += 32 * U * a.parts) {
            Eight<E> w[U];
            uint4 x[U][PIECES];
#pragma unroll
            for (int q = 0; q < U; ++q) w[q] = load_eight<E>(wr, k0 + q * 32 + g * 8, a.dim);
#pragma unroll
            for (int q = 0; q < U; ++q)
#pragma unroll
                for (int p = 0; p < PIECES; ++p) {
                    const int k = k0 + q * 32 + g * 8;
                    x[q][p] = k < dp ? *reinterpret_cast<const uint4*>(xr + p * a.x_piece + k) : make_uint4(0, 0, 0, 0);
                }
#pragma unroll
            for (int q = 0; q < U; ++q) {
                bf16x8 y[PIECES], z[PIECES];
#pragma unroll
                for (int p = 0; p < PIECES; ++p) z[p] = __builtin_bit_cast(bf16x8, x[q][p]);
                if constexpr (PIECES == 1) {
                    y[0] = __builtin_bit_cast(bf16x8, w[q]);
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y[0], z[0], acc, 0, 0, 0);
                } else {
                    float v[8];
                    bf16x8 o[3];
#pragma unroll
                    for (int h = 0; h < 8; ++h) v[h] = w[q].q[h / 4].v[h % 4];
                    eight_in_pieces(v, o);
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(o[0], z[2], acc, 0, 0, 0);
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(o[1], z[1], acc, 0, 0, 0);
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(o[2], z[0], acc, 0, 0, 0);
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(o[0], z[1], acc, 0, 0, 0);
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(o[1], z[0], acc, 0, 0, 0);
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(o[0], z[0], acc, 0, 0, 0);
                }
            }
        }
        if (a.parts > 1) {
            __syncthreads();
            if (wave) acc_of[wave - 1][lane] = make_float4(acc[0], acc[1], acc[2], acc[3]);
            __syncthreads();
            if (wave) continue;
#pragma unroll
            for (int q = 0; q < 3; ++q) {
                const float4 o = acc_of[q][lane];
                acc[0] += o.x; acc[1] += o.y; acc[2] += o.z; acc[3] += o.w;
            }
        }
        const int64_t first = c0 + g * 4;
        if constexpr (GRAD) {
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] = u != 0.0f ? u * __builtin_amdgcn_exp2f(fmaf(acc[e], LOG2E, b)) : 0.0f;  // (left out: whatever the score is)
                if (first + e == t) v[e] -= u;
            }
            if (s < a.n) {
                float* const o = a.d + s * a.d_ld + first;  // (d_ld is a multiple of 16: classes beyond the last one have room)
                *reinterpret_cast<float4*>(o) = make_float4(v[0], v[1], v[2], v[3]);
            }
        } else {
            float m = top;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (first + e >= a.n_classes) acc[e] = -__builtin_inff();
                m = fmaxf(m, acc[e]);
            }
            const float m0 = m == -__builtin_inff() ? 0.0f : m;
            sum *= __builtin_amdgcn_exp2f((top - m0) * LOG2E);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f((acc[e] - m0) * LOG2E);
            top = m;
        }
    }
    if constexpr (!GRAD) {
        auto join = [&](float mo, float so) {
            const float m = fmaxf(top, mo), m0 = m == -__builtin_inff() ? 0.0f : m;
            sum = sum * __builtin_amdgcn_exp2f((top - m0) * LOG2E) + so * __builtin_amdgcn_exp2f((mo - m0) * LOG2E);
            top = m;
        };
#pragma unroll
        for (int o = 16; o < 64; o <<= 1) {
            const float mo = __shfl_xor(top, o), so = __shfl_xor(sum, o);
            join(mo, so);
        }
        if (g == 0) both[wave][s] = make_float2(top, sum);
        __syncthreads();
        if (threadIdx.x < a.n) {
            top = both[0][s].x; sum = both[0][s].y;
            for (int w = 1; w < 4; ++w) join(both[w][s].x, both[w][s].y);
            a.part[(int64_t)s * gridDim.x + blockIdx.x] = make_float2(top, sum);
        }
    }
}

// Both gradients from D: a thread has 4 values of a row of weights; classes first .. first + classes_each - 1 are a workgroup's, its groups of
// `lanes` threads take them in turn.  dW of a class is written at once, dX is added up over the workgroup's classes: a slab each.  ROWS
// rows: n of them, then zeros.
struct FewGradArgs {
    const void *x, *w;  // as the caller has them
    int64_t x_ld, w_ld;
    int n, dim, lanes, column_blocks;
    int64_t n_classes, each;
    const float* d;
    int64_t d_ld;
    const float* common;
    void* grad_w;       // null: not wanted
    float* slab;        // [workgroups along the classes][n][slab_ld], null: not wanted
    int64_t slab_ld;
    const void* target; // rows without a class or weight are zeros in D; their x is not looked at
    int target_bytes;
    const float* weight;
};

template <class E>
__device__ __forceinline__ void load_four(const typename E::T* p, int have, float* v) {
    if (have >= 4) {
        typename E::T q[4];
        __builtin_memcpy(q, p, sizeof(q));
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = E::get(q[k]);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = k < have ? E::get(p[k]) : 0.0f;
    }
}

template <class E, int ROWS>
__global__ __launch_bounds__(256) void few_gradients_kernel(FewGradArgs a) {
    constexpr int CHUNK = 64;
    __shared__ __align__(16) float ds[CHUNK][ROWS];
    __shared__ __align__(16) float sums[256][4];
    typedef typename E::T T;
    const int sub = threadIdx.x % a.lanes, group = threadIdx.x / a.lanes, groups = 256 / a.lanes;
    const int cb = blockIdx.x % a.column_blocks;
    const int64_t block = blockIdx.x / a.column_blocks, c0 = block * a.each, c1 = c0 + a.each < a.n_classes ? c0 + a.each : a.n_classes;
    const int col = (cb * a.lanes + sub) * 4, have = a.dim - col;
    const float by = *a.common;
    float x[ROWS][4], acc[ROWS][4];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
#pragma unroll
        for (int k = 0; k < 4; ++k) x[r][k] = acc[r][k] = 0.0f;
        if (r < a.n && a.weight[r] != 0.0f && target_of(a.target, a.target_bytes, r, a.n_classes) >= 0)
            load_four<E>(static_cast<const T*>(a.x) + r * a.x_ld + col, have, x[r]);
    }
    for (int64_t base = c0; base < c1; base += CHUNK) {
        const int m = (int)(c1 - base < CHUNK ? c1 - base : CHUNK);
        __syncthreads();
        for (int i = threadIdx.x; i < CHUNK * ROWS; i += 256) {
            const int r = i / CHUNK, c = i % CHUNK;
            ds[c][r] = r < a.n && c < m ? a.d[r * a.d_ld + base + c] : 0.0f;
        }
        __syncthreads();
        if (have <= 0) continue;
        for (int c = group; c < m; c += 2 * groups) {
            float w[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (a.slab && c + h * groups < m) load_four<E>(static_cast<const T*>(a.w) + (base + c + h * groups) * a.w_ld + col, have, w[h]);
                else w[h][0] = w[h][1] = w[h][2] = w[h][3] = 0.0f;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int ch = c + h * groups;
                if (ch >= m) continue;
                float o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    const float d = ds[ch][r];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        o[k] = fmaf(d, x[r][k], o[k]);
                        acc[r][k] = fmaf(d, w[h][k], acc[r][k]);
                    }
                }
                if (a.grad_w) {
                    T* const p = static_cast<T*>(a.grad_w) + (base + ch) * a.dim + col;
                    const T q[4] = {E::put(o[0] * by), E::put(o[1] * by), E::put(o[2] * by), E::put(o[3] * by)};
                    if (have >= 4) __builtin_memcpy(p, q, sizeof(q));
                    else
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (k < have) p[k] = q[k];
                }
            }
        }
    }
    if (!a.slab) return;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        if (r < a.n && groups > 1) {  // the groups' sums in their order
            __syncthreads();
            *reinterpret_cast<float4*>(sums[threadIdx.x]) = make_float4(acc[r][0], acc[r][1], acc[r][2], acc[r][3]);
            __syncthreads();
            if (group == 0)
                for (int k = 1; k < groups; ++k) {
                    const float4 o = *reinterpret_cast<const float4*>(sums[k * a.lanes + sub]);
                    acc[r][0] += o.x; acc[r][1] += o.y; acc[r][2] += o.z; acc[r][3] += o.w;
                }
        }
        if (r < a.n && group == 0 && have > 0)
            *reinterpret_cast<float4*>(a.slab + (block * a.n + r) * a.slab_ld + col) = make_float4(acc[r][0], acc[r][1], acc[r][2], acc[r][3]);
    }
}

}  // namespace qgbdt
