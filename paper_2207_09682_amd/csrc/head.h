// What the operators on token tables and class scores share: element types, conversions, launchers.
#pragma once
#include "common.h"

namespace qgbdt {

// bfloat16 keeps the sign, the exponent and 7 bits of a float; to the nearest, ties to even, NaN stays NaN.
__device__ __forceinline__ float from_bf16(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ uint16_t to_bf16(float v) {
    const __bf16 b = (__bf16)v;
    return __builtin_bit_cast(uint16_t, b);
}
__device__ __forceinline__ float from_f16(uint16_t v) { return (float)__builtin_bit_cast(_Float16, v); }
__device__ __forceinline__ uint16_t to_f16(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }

// Element types: how many values 16 bytes hold, and their conversion.
struct F32 {
    typedef float T;
    static constexpr int PER16 = 4;
    static __device__ __forceinline__ float get(float v) { return v; }
    static __device__ __forceinline__ float put(float v) { return v; }
};
struct BF16 {
    typedef uint16_t T;
    static constexpr int PER16 = 8;
    static __device__ __forceinline__ float get(uint16_t v) { return from_bf16(v); }
    static __device__ __forceinline__ uint16_t put(float v) { return to_bf16(v); }
};
struct F16 {
    typedef uint16_t T;
    static constexpr int PER16 = 8;
    static __device__ __forceinline__ float get(uint16_t v) { return from_f16(v); }
    static __device__ __forceinline__ uint16_t put(float v) { return to_f16(v); }
};

// 16 bytes that may begin at any element: global loads and stores of gfx950 take any address.
template <class E>
struct __attribute__((packed, aligned(sizeof(typename E::T)))) Piece {
    typename E::T v[E::PER16];
};

template <class E>
__device__ __forceinline__ void load_piece(const typename E::T* p, float* v) {
    Piece<E> q;
    __builtin_memcpy(&q, p, 16);
#pragma unroll
    for (int i = 0; i < E::PER16; ++i) v[i] = E::get(q.v[i]);
}
template <class E>
__device__ __forceinline__ void store_piece(typename E::T* p, const float* v) {
    Piece<E> q;
#pragma unroll
    for (int i = 0; i < E::PER16; ++i) q.v[i] = E::put(v[i]);
    __builtin_memcpy(p, &q, 16);
}
// the same for the first m < PER16 values of a row's last piece
template <class E>
__device__ __forceinline__ void load_part(const typename E::T* p, int m, float* v) {
#pragma unroll
    for (int i = 0; i < E::PER16; ++i) v[i] = i < m ? E::get(p[i]) : 0.0f;
}
template <class E>
__device__ __forceinline__ void store_part(typename E::T* p, int m, const float* v) {
#pragma unroll
    for (int i = 0; i < E::PER16; ++i)
        if (i < m) p[i] = E::put(v[i]);
}

// A sum that keeps what its roundings lose (the exact error of an addition of two floats, after Knuth), so that its own error does not grow with its length.
// An infinite sum stays one.
struct LongSum {
    float sum = 0.0f, lost = 0.0f;
    __device__ __forceinline__ void add(float v) {
        const float s = sum + v, b = s - sum;
        lost += (sum - (s - b)) + (v - b);
        sum = s;
    }
    __device__ __forceinline__ float value() const { return fabsf(sum) < __builtin_inff() ? sum + lost : sum; }
};

// LDS writes of a wavefront's lanes are there for its other lanes
__device__ __forceinline__ void wavefront_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

inline size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }
inline int dtype_bytes(int dtype) { return dtype == QGBDT_F32 ? 4 : 2; }

size_t embed_gradient_bytes(int64_t n, int bag, int64_t n_vocab, int dim, int dtype);
int run_embed_tokens(qgbdt_ctx* ctx, const void* table, int dtype, int64_t n_vocab, int dim, int64_t table_stride,
                     const void* tokens, int token_bytes, int64_t n, int bag, float scale, void* out);
int run_embed_gradient(qgbdt_ctx* ctx, const void* tokens, int token_bytes, int64_t n, int bag, const void* grad, int dtype,
                       int64_t n_vocab, int dim, float scale, void* grad_table, int accumulate, void* scratch);
size_t softmax_bytes(int64_t n, int dim, int64_t n_classes, int dtype, int64_t x_stride, int64_t w_stride, bool gradients);
int run_softmax_loss(qgbdt_ctx* ctx, const void* x, const void* w, int dtype, int64_t n, int dim, int64_t n_classes, int64_t x_stride,
                     int64_t w_stride, const void* target, int target_bytes, float* loss, float* lse, void* scratch);
int run_softmax_gradients(qgbdt_ctx* ctx, const void* x, const void* w, int dtype, int64_t n, int dim, int64_t n_classes, int64_t x_stride,
                          int64_t w_stride, const void* target, int target_bytes, const float* lse, const float* row_weight,
                          void* grad_x, void* grad_w, void* scratch);
size_t clip_bytes(int n_tensors);
int run_clip_gradients(qgbdt_ctx* ctx, const void* const* in, void* const* out, const int64_t* counts, const int32_t* dtypes,
                       int n_tensors, double max_norm, float* norm_out, void* scratch);

}  // namespace qgbdt
