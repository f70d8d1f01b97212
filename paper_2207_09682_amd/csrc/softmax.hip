// Softmax cross entropy over many classes with a weight vector each, and its gradient, without the matrix of scores.
//   s_ij = x_i . w_j,  lse_i = log sum_j exp s_ij,  loss_i = lse_i - s_it
//   p_ij = exp(s_ij - lse_i),  D_ij = u_i (p_ij - [j = t]),  dX = D W,  dW = D^T X
// The scores leave the product kernel as a maximum and a sum of exponentials per row and strip of classes.  The gradients make
// the scores again, strip of classes by strip: D of a strip (in bfloat16, for fp32 inputs in three pieces) is all that
// is kept of them, and two more products take it to dX and dW.
#include <type_traits>

#include "few_device.h"
#include "middle_device.h"
#include "sweep_device.h"

namespace qgbdt {

// What rows are left out by, and what the gradients need of them; all null or zero: no row is left out.
struct LeftOut {
    const void* target;
    int target_bytes;
    int64_t n_classes;
    const float* weight;
    const float* lse;
    const uint32_t* tops;  // not null: of weight_kernel
    int n_tops;
    float* common;      // not null: written
    RowTerms* terms;    // not null: written, up to a multiple of SWEEP_TILE with rows that are left out
    __device__ __forceinline__ bool live(int64_t row) const { return !target || (target_of(target, target_bytes, row, n_classes) >= 0 && weight[row] != 0.0f); }
    __device__ __forceinline__ RowTerms of(int64_t row, int64_t rows, float unit, float back) const {
        if (row < rows && live(row)) return {-lse[row] * LOG2E, weight[row] / unit, (int)target_of(target, target_bytes, row, n_classes), back};
        return {-__builtin_inff(), 0.0f, -1, back};
    }
    // bits of a row's weight without its sign, 0 where it does not count or is not finite
    __device__ __forceinline__ uint32_t size_of_weight(int64_t row) const {
        const int64_t t = target_of(target, target_bytes, row, n_classes);  // (both are requested at once)
        const uint32_t b = __float_as_uint(weight[row]) & 0x7fffffffu;
        return t >= 0 && b < 0x7f800000u ? b : 0u;
    }
};

__device__ __forceinline__ uint32_t largest_of_workgroup(uint32_t v) {
    __shared__ uint32_t part[4];
    for (int o = 32; o > 0; o >>= 1) { const uint32_t b = __shfl_xor(v, o); v = b > v ? b : v; }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    const uint32_t a = part[0] > part[1] ? part[0] : part[1], b = part[2] > part[3] ? part[2] : part[3];
    return a > b ? a : b;
}

// The common weight: the largest finite one among the rows that count, 1 where none does.  D in units of it is at most 1 in size, and where all
// weights are the same, as for a mean, D keeps p - 1 and p without a second rounding.  For a whole workgroup, from all rows where they are
// few, else from the maxima of weight_kernel: every workgroup that lays rows out needs it, wherever the rows that count begin.
constexpr int64_t WEIGHTS_AT_ONCE = 2048;  // (gradients of 2000 x 250 bf16 against 20,000 classes: 313 us, with the launch 319)
constexpr int WEIGHT_BLOCKS = 256;
__device__ __forceinline__ float common_weight(const LeftOut& src, int64_t rows) {
    uint32_t top = 0;
    if (src.tops) {
        if ((int)threadIdx.x < src.n_tops) top = src.tops[threadIdx.x];
    } else {
#pragma unroll
        for (int k = 0; k < (int)(WEIGHTS_AT_ONCE / 256); ++k) {
            const int64_t i = threadIdx.x + k * 256;
            const uint32_t b = i < rows ? src.size_of_weight(i) : 0u;
            top = b > top ? b : top;
        }
    }
    top = largest_of_workgroup(top);
    return top ? __uint_as_float(top) : 1.0f;
}

// Up to WEIGHT_BLOCKS maxima of the rows' weights.  Bound by latency, with very many rows by memory (100,003 rows: 5 us).
__global__ __launch_bounds__(256) void weight_kernel(LeftOut src, int64_t rows, uint32_t* __restrict__ tops, uint32_t* __restrict__ range) {
    uint32_t top = 0;
    if (range && blockIdx.x == 0 && threadIdx.x == 0) *range = 0;  // (for lay_out_fp32_kernel)
    const int64_t step = (int64_t)gridDim.x * 256;
#pragma unroll 4
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows; i += step) { const uint32_t b = src.size_of_weight(i); top = b > top ? b : top; }
    top = largest_of_workgroup(top);
    if (threadIdx.x == 0) tops[blockIdx.x] = top;
}

// A matrix as the products read it: rows of `dp` elements (a multiple of 8, zeros behind the row's end), fp32 values in three
// pieces.  Rows that are left out become zeros, whatever they hold.  Bound by memory (8192 x 2048 bf16: 14 us, 4.8 TB/s).
template <class E, int PIECES>
__global__ __launch_bounds__(256) void lay_out_kernel(const typename E::T* __restrict__ in, int64_t stride, int64_t rows, int dim, int dp,
                                                      uint16_t* __restrict__ out, int64_t piece, LeftOut src) {
    const int64_t t0 = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, step = (int64_t)gridDim.x * blockDim.x;
    if (src.terms || (src.common && blockIdx.x == 0)) {
        const float unit = common_weight(src, rows);
        if (t0 == 0) *src.common = unit;
        if (src.terms)
            for (int64_t i = t0; i < (rows + SWEEP_TILE - 1) / SWEEP_TILE * SWEEP_TILE; i += step) src.terms[i] = src.of(i, rows, unit, 1.0f);
    }
    const int per_row = dp >> 3;
    const int64_t total = rows * per_row;
    for (int64_t i = t0; i < total; i += step) {
        const int64_t row = i / per_row;
        const int c = (int)(i - row * per_row) * 8;
        float v[8];
        if (!src.live(row)) {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = 0.0f;
        } else {
            const Eight<E> e = load_eight<E>(in + row * stride, c, dim);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = E::get(e.q[k / E::PER16].v[k % E::PER16]);
        }
        union { uint16_t h[8]; uint4 q; } u[PIECES];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if constexpr (PIECES == 1) {
                u[0].h[k] = to_bf16(v[k]);
            } else {
                uint16_t q[3];
                three_pieces(v[k], q);
                u[0].h[k] = q[0]; u[1].h[k] = q[1]; u[2].h[k] = q[2];
            }
        }
#pragma unroll
        for (int s = 0; s < PIECES; ++s) *reinterpret_cast<uint4*>(out + s * piece + row * dp + c) = u[s].q;
    }
}

constexpr int LAY_OUT_BLOCKS = 2048;  // workgroups per matrix: as many as the chip holds

// A matrix of fp32 rows and where its pieces go.
struct Fp32Rows {
    const float* in;
    int64_t stride, rows;
    uint16_t* halves;  // two fp16 pieces, rows of dp values
    uint16_t* three;   // three bfloat16 pieces, null in a loss
    float* back;       // per row: takes scores of the fp16 pieces back
};

// fp32 rows in two fp16 pieces for the scores, each row brought to 2^14 .. 2^15 by a power of two, which `back` undoes, and with THREE in
// three bfloat16 pieces too, for the second products.  `lanes` threads have a row.  The first w_blocks workgroups lay out the weights, the others x.  What
// the rows say about their pieces (RANGE_...) goes to a byte per workgroup or into *range.  Bound by memory (100,003 x 64
// and 10,007 classes with all pieces: 22 us, 4.5 TB/s; without the bfloat16 ones 16).
template <bool THREE>
__global__ __launch_bounds__(256) void lay_out_fp32_kernel(Fp32Rows w, Fp32Rows x, int w_blocks, int dim, int dp, int lanes, LeftOut of_x, uint8_t* __restrict__ marks,
                                                           uint32_t* __restrict__ range) {
    __shared__ uint32_t found;
    if (threadIdx.x == 0) found = 0;
    const bool weights = (int)blockIdx.x < w_blocks;
    const Fp32Rows m = weights ? w : x;
    const LeftOut src = weights ? LeftOut{} : of_x;
    const int block = (int)blockIdx.x - (weights ? 0 : w_blocks), blocks = weights ? w_blocks : (int)gridDim.x - w_blocks;
    const int sub = threadIdx.x & (lanes - 1), per = 256 / lanes;
    const int64_t step = (int64_t)blocks * per, rows = m.rows, piece = rows * dp;
    float unit = 1.0f;
    if (src.terms || (src.common && block == 0)) {
        unit = common_weight(src, rows);
        if (block == 0 && threadIdx.x == 0) *src.common = unit;
    }
    __syncthreads();
    uint32_t marked = 0;
    const int64_t filled = src.terms ? (rows + SWEEP_TILE - 1) / SWEEP_TILE * SWEEP_TILE : rows;
    for (int64_t row = (int64_t)block * per + threadIdx.x / lanes; row < filled; row += step) {
        if (row >= rows) {
            if (sub == 0) src.terms[row] = src.of(row, rows, unit, 1.0f);
            continue;
        }
        const bool live = src.live(row);
        const float* const p = m.in + row * m.stride;
        uint32_t top = 0;  // bits of the largest magnitude: infinities and NaN are above all others
        for (int c = sub * 8; c < dim; c += lanes * 8) {
            const Eight<F32> v = load_eight<F32>(p, c, dim);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t b = __float_as_uint(v.q[k / 4].v[k % 4]) & 0x7fffffffu;
                top = b > top ? b : top;
            }
        }
        for (int o = lanes >> 1; o > 0; o >>= 1) {  // (lanes of a row go through this together)
            const uint32_t b = __shfl_xor(top, o);
            top = b > top ? b : top;
        }
        const int e = (int)(top >> 23);
        const bool finite = e != 255 && top != 0 && live;  // (and not all zeros, which any pieces hold)
        int shift = finite ? 14 + 127 - e : 0;
        if (shift > 120) shift = 120;
        const float by = __uint_as_float((uint32_t)(127 + shift) << 23), undo = __uint_as_float((uint32_t)(127 - shift) << 23);
        if (sub == 0) {
            m.back[row] = undo;
            if (src.terms) src.terms[row] = src.of(row, rows, unit, undo);
        }
        const uint32_t large = top > (9u << 23) ? top - (9u << 23) : 0u, faint = top > (17u << 23) ? top - (17u << 23) : 0u;
        int of_size = 0;
        for (int c = sub * 8; c < dp; c += lanes * 8) {
            const Eight<F32> v = load_eight<F32>(p, c, dim);
            union { uint16_t h[8]; uint4 q; } hi, lo, u[3];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float value = live ? v.q[k / 4].v[k % 4] : 0.0f, x = value * by;
                const uint32_t b = __float_as_uint(value) & 0x7fffffffu;
                of_size += b >= large ? 1 : 0;
                if (finite && b != 0 && b < faint) marked |= RANGE_FAINT;
                hi.h[k] = to_f16(x);
                const float r = x - from_f16(hi.h[k]);
                lo.h[k] = fabsf(x) < __builtin_inff() ? to_f16(r) : 0x7e00;  // (an infinity: NaN, as in three_pieces())
                if constexpr (THREE) {
                    uint16_t q[3];
                    three_pieces(value, q);
                    u[0].h[k] = q[0]; u[1].h[k] = q[1]; u[2].h[k] = q[2];
                }
            }
            *reinterpret_cast<uint4*>(m.halves + row * dp + c) = hi.q;
            *reinterpret_cast<uint4*>(m.halves + piece + row * dp + c) = lo.q;
            if constexpr (THREE)
#pragma unroll
                for (int s = 0; s < 3; ++s) *reinterpret_cast<uint4*>(m.three + s * piece + row * dp + c) = u[s].q;
        }
        for (int o = lanes >> 1; o > 0; o >>= 1) of_size += __shfl_xor(of_size, o);
        if (finite && (dim - of_size) * 4 > dim) marked |= RANGE_LOOSE;
        if (finite && (e < 127 - 50 || e > 127 + 50)) marked |= RANGE_WIDE;
    }
    if (marked) atomicOr(&found, marked);
    __syncthreads();
    if (threadIdx.x == 0) {
        if (marks) marks[blockIdx.x] = (uint8_t)found;
        else if (found) atomicOr(range, found);
    }
}

// Between the layout and the scores of a loss: the range of all rows, and where it asks for them three bfloat16 pieces in place of the two of fp16.  before:
// of the rows before these, whose pieces of the weights stay.  Bound by latency (5 us), by memory where pieces are made.
__global__ __launch_bounds__(256) void settle_kernel(Fp32Rows w, Fp32Rows x, int dim, int dp, const uint8_t* __restrict__ marks, int n_marks, const uint32_t* __restrict__ before,
                                                     uint32_t* __restrict__ range) {
    __shared__ uint32_t found;
    const uint32_t old = before ? *before : 0;
    if (threadIdx.x == 0) found = old;
    __syncthreads();
    uint32_t marked = 0;
    static_assert(2 * LAY_OUT_BLOCKS <= 16 * 256, "a thread has 16 bytes of the marks");
    const int i0 = threadIdx.x * 16;
    if (i0 < n_marks) {
        union { uint4 q; uint8_t b[16]; } v;
        v.q = *reinterpret_cast<const uint4*>(marks + i0);
#pragma unroll
        for (int i = 0; i < 16; ++i) marked |= i0 + i < n_marks ? v.b[i] : 0;
    }
    if (marked) atomicOr(&found, marked);
    __syncthreads();
    const uint32_t all = found;
    if (blockIdx.x == 0 && threadIdx.x == 0) *range = all;
    if (!in_three_pieces(all)) return;
    const int per_row = dp >> 3;
    const int64_t of_w = in_three_pieces(old) ? 0 : w.rows * per_row, total = of_w + x.rows * per_row;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const Fp32Rows m = i < of_w ? w : x;
        const int64_t j = i < of_w ? i : i - of_w, row = j / per_row;
        const int c = (int)(j - row * per_row) * 8;
        const Eight<F32> v = load_eight<F32>(m.in + row * m.stride, c, dim);
        union { uint16_t h[8]; uint4 q; } u[3];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            uint16_t q[3];
            three_pieces(v.q[k / 4].v[k % 4], q);
            u[0].h[k] = q[0]; u[1].h[k] = q[1]; u[2].h[k] = q[2];
        }
#pragma unroll
        for (int s = 0; s < 3; ++s) *reinterpret_cast<uint4*>(m.halves + s * m.rows * dp + row * dp + c) = u[s].q;
    }
}

// ---- epilogues ------------------------------------------------------------------------------------

// Scores of fp32 rows as they were before their rows were scaled.
template <int NL, int NR>
__device__ __forceinline__ void scale_back(f32x4 (&acc)[NL][NR], const float* back_l, const float* back_r, int row0, int col0, int rows, int cols, int lane) {
    float r[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        const int row = row0 + i * 16 + (lane & 15);
        r[i] = back_l[row < rows ? row : rows - 1];
    }
#pragma unroll
    for (int j = 0; j < NR; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int col = col0 + j * 16 + (lane >> 4) * 4 + e;
            const float c = back_r[col < cols ? col : cols - 1];
#pragma unroll
            for (int i = 0; i < NL; ++i) acc[i][j][e] = acc[i][j][e] * r[i] * c;
        }
}

// Maximum and sum of exponentials of a row's scores over a wavefront's strip of classes.  SCALED: of fp32 rows, in fp16 pieces where back_l is not null.
template <bool SCALED>
struct StatsEpilogue {
    float2* part;  // [rows][strips]
    int strips;
    int rows, cols;
    const float *back_l, *back_r;
    static constexpr bool TURNS = false;
    template <int NL, int NR>
    __device__ __forceinline__ void finish(f32x4 (&acc)[NL][NR], int row0, int col0, int strip, int, int lane, uint16_t*) const {
        if (SCALED && back_l) scale_back(acc, back_l, back_r, row0, col0, rows, cols, lane);
        const int h4 = (lane >> 4) * 4;
        const bool whole = col0 + NR * 16 <= cols;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int row = row0 + i * 16 + (lane & 15);
            float m = -__builtin_inff();
#pragma unroll
            for (int j = 0; j < NR; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (!whole && col0 + j * 16 + h4 + e >= cols) acc[i][j][e] = -__builtin_inff();
                    m = fmaxf(m, acc[i][j][e]);
                }
            m = fmaxf(m, __shfl_xor(m, 16));
            m = fmaxf(m, __shfl_xor(m, 32));
            const float m0 = m == -__builtin_inff() ? 0.0f : m, mb = -m0 * LOG2E;
            float s = 0.0f;
#pragma unroll
            for (int j = 0; j < NR; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) s += __builtin_amdgcn_exp2f(fmaf(acc[i][j][e], LOG2E, mb));
            s += __shfl_xor(s, 16);
            s += __shfl_xor(s, 32);
            if (lane < 16 && row < rows) part[(int64_t)row * strips + strip] = make_float2(m, s);
        }
    }
};

// D of a strip of classes, in units of the common weight.  PIECES = 1 rounds it to bfloat16, 2^-8 of each value, as the operand of the two products that
// follow: two pieces would double these, two of the three products of a step, for gradients that are rounded to the same type.  PIECES = 3 keeps 24 bits.  Rows and columns beyond the last ones, as far as the products read
// them, are zeros.  A lane has 4 consecutive values of a row: they are turned in LDS, so that 16 bytes per lane
// and whole rows of the wavefront's part go to memory (8192 rows x 16,384 classes x 2048: 473 us; D^T X, a product of the same size, 412).
template <int PIECES>
struct GradEpilogue {
    uint16_t* d;  // [pieces][rows_out][ld]
    int64_t ld, piece;
    const float *lse, *weight, *common;
    const void* target;
    int target_bytes;
    int rows, rows_out, cols, cols_out;
    int64_t first;  // class of column 0
    int64_t n_classes;
    const float *back_l, *back_r;  // not null: the scores are of rows in fp16 pieces
    static constexpr bool TURNS = true;
    template <int NL, int NR>
    __device__ __forceinline__ void finish(f32x4 (&acc)[NL][NR], int row0, int col0, int, int, int lane, uint16_t* own) const {
        constexpr int CW = NR * 16, C = CW / 8;  // columns, 16-byte pieces of a row
        const int h4 = (lane >> 4) * 4;
        const float unit = *common;
        const bool whole = col0 + CW <= cols;
        if (PIECES > 1 && back_l) scale_back(acc, back_l, back_r, row0, col0, rows, cols, lane);
        // Rows that are left out, bit i: zeros, chosen when the values are packed and not multiplied, since their x of zeros makes scores that are no
        // numbers with infinite weights.
        uint32_t left = 0;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int row = row0 + i * 16 + (lane & 15);
            float u = 0.0f, b = 0.0f;
            int64_t t = -1;
            if (row < rows) {
                t = target_of(target, target_bytes, row, n_classes);
                if (t >= 0) u = weight[row] / unit;
                if (u != 0.0f) b = -lse[row] * LOG2E;
            }
            const int64_t at = t - first - col0 - h4;
            const int want = t >= 0 && at >= 0 && at < CW ? (int)at : -1;
#pragma unroll
            for (int j = 0; j < NR; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] = u * __builtin_amdgcn_exp2f(fmaf(acc[i][j][e], LOG2E, b));
            left |= (u == 0.0f ? 1u : 0u) << i;
            if (__ballot(want >= 0) != 0)
#pragma unroll
                for (int j = 0; j < NR; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (want == j * 16 + e) acc[i][j][e] -= u;
            if (!whole)
#pragma unroll
                for (int j = 0; j < NR; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (col0 + j * 16 + h4 + e >= cols) acc[i][j][e] = 0.0f;
        }
        const bool any_left = __ballot(left != 0) != 0;
#pragma unroll 1
        for (int s = 0; s < PIECES; ++s) {
            // (16 consecutive rows put the same piece into 16 different places of 256 bytes)
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                const int r = i * 16 + (lane & 15), turn = (r / (16 / C)) & (C - 1);
#pragma unroll
                for (int j = 0; j < NR; ++j) {
                    union { uint16_t h[4]; uint2 v; } o;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        o.h[e] = to_bf16(acc[i][j][e]);
                        if (PIECES > 1) acc[i][j][e] -= from_bf16(o.h[e]);
                    }
                    if (any_left) { o.v.x = left >> i & 1 ? 0u : o.v.x; o.v.y = left >> i & 1 ? 0u : o.v.y; }
                    *reinterpret_cast<uint2*>(own + r * CW + ((j * 2 + (lane >> 5)) ^ turn) * 8 + (h4 & 4)) = o.v;
                }
            }
            wavefront_sync();
#pragma unroll
            for (int n = 0; n < NL * 16 * C / 64; ++n) {
                const int k = n * 64 + lane, r = k / C, c = k % C;
                const uint4 v = *reinterpret_cast<const uint4*>(own + r * CW + (c ^ ((r / (16 / C)) & (C - 1))) * 8);
                if (row0 + r < rows_out && col0 + c * 8 < cols_out) *reinterpret_cast<uint4*>(d + s * piece + (row0 + r) * ld + col0 + c * 8) = v;
            }
            wavefront_sync();
        }
    }
};

// C itself: to a fp32 slab of this split, added to what it holds or not, or as the result's type.
template <class E>
struct StoreEpilogue {
    typename E::T* out;
    float* slab;  // not null: [splits][rows][slab_ld]
    int64_t ld, slab_ld, slab_size;
    int rows, cols;
    int add;
    const float* unit;  // of D, for the result's type
    static constexpr bool TURNS = false;
    template <int NL, int NR>
    __device__ __forceinline__ void finish(f32x4 (&acc)[NL][NR], int row0, int col0, int, int split, int lane, uint16_t*) const {
        const int h4 = (lane >> 4) * 4;
        const float by = slab ? 1.0f : *unit;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int row = row0 + i * 16 + (lane & 15);
            if (row >= rows) continue;
#pragma unroll
            for (int j = 0; j < NR; ++j) {
                const int col = col0 + j * 16 + h4;
                if (col >= cols) continue;
                const f32x4 v = acc[i][j];
                if (slab) {
                    float4* p = reinterpret_cast<float4*>(slab + split * slab_size + row * slab_ld + col);
                    float4 o = make_float4(v[0], v[1], v[2], v[3]);
                    if (add) { const float4 b = *p; o.x += b.x; o.y += b.y; o.z += b.z; o.w += b.w; }
                    *p = o;
                } else {
                    typename E::T* p = out + row * ld + col;
                    typename E::T c[4] = {E::put(v[0] * by), E::put(v[1] * by), E::put(v[2] * by), E::put(v[3] * by)};
                    if (col + 4 <= cols) __builtin_memcpy(p, c, sizeof(c));
                    else
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (col + e < cols) p[e] = c[e];
                }
            }
        }
    }
};

// Slabs of fp32 sums -> the result.  Bound by memory (100,003 x 64 of 4 slabs: 27 us).
template <class E>
__global__ __launch_bounds__(256) void join_kernel(const float* __restrict__ slab, int64_t slab_size, int slab_ld, int splits, int64_t rows, int cols,
                                                   typename E::T* __restrict__ out, int64_t ld, const float* __restrict__ unit) {
    const float by = *unit;
    const int per_row = slab_ld >> 2;
    const int64_t total = rows * per_row, step = (int64_t)gridDim.x * blockDim.x;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += step) {
        const int64_t row = i / per_row;
        const int c = (int)(i - row * per_row) * 4;
        const float* p = slab + row * slab_ld + c;
        float4 s = *reinterpret_cast<const float4*>(p);
        for (int k = 1; k < splits; ++k) {
            const float4 b = *reinterpret_cast<const float4*>(p + k * slab_size);
            s.x += b.x; s.y += b.y; s.z += b.z; s.w += b.w;
        }
        typename E::T* o = out + row * ld + c;
        const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < cols) o[e] = E::put(v[e] * by);
    }
}

// The same for many slabs and few values: 16 pieces of 4 values by 16 groups of slabs, whose sums are added up in their order.
template <class E>
__global__ __launch_bounds__(256) void join_many_kernel(const float* __restrict__ slab, int64_t slab_size, int slab_ld, int splits, int64_t rows, int cols,
                                                        typename E::T* __restrict__ out, int64_t ld, const float* __restrict__ unit) {
    __shared__ float4 sums[16][16];
    const int per_row = slab_ld >> 2, piece = threadIdx.x & 15, group = threadIdx.x >> 4;
    const int64_t i = (int64_t)blockIdx.x * 16 + piece, row = i / per_row;
    const int c = (int)(i - row * per_row) * 4;
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (row < rows) {
        const float* const p = slab + row * slab_ld + c;
        for (int k = group; k < splits; k += 64) {
            float4 v[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = k + q * 16 < splits ? *reinterpret_cast<const float4*>(p + (k + q * 16) * slab_size) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int q = 0; q < 4; ++q) { s.x += v[q].x; s.y += v[q].y; s.z += v[q].z; s.w += v[q].w; }
        }
    }
    sums[group][piece] = s;
    __syncthreads();
    if (group || row >= rows) return;
    for (int k = 1; k < 16; ++k) { const float4 v = sums[k][piece]; s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w; }
    const float by = *unit;
    const float v[4] = {s.x, s.y, s.z, s.w};
    typename E::T* const o = out + row * ld + c;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (c + e < cols) o[e] = E::put(v[e] * by);
}

// One wavefront per row: the strips' maxima and sums to the log of the normaliser, and the target's score as a product
// of its own.  The log and the difference are taken in fp64: they are two per row.  Bound by latency (1 row: 4.4 us), with many rows by the
// scattered rows of weights and the parts (100,003 x 64 fp32: 53 us).
template <class E>
__global__ __launch_bounds__(256) void loss_kernel(const float2* __restrict__ part, int strips, const typename E::T* __restrict__ x, int64_t x_stride,
                                                   const typename E::T* __restrict__ w, int64_t w_stride, int64_t n, int dim, int64_t n_classes,
                                                   const void* target, int target_bytes, float* __restrict__ loss, float* __restrict__ lse) {
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * (blockDim.x >> 6) + (threadIdx.x >> 6);
    if (row >= n) return;
    const int64_t t = target_of(target, target_bytes, row, n_classes);
    float m = -__builtin_inff(), s = 0.0f;
    const float2* const p = part + row * strips;
    for (int i = lane; i < strips; i += 64 * 8) {
        float2 q[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) q[k] = i + k * 64 < strips ? p[i + k * 64] : make_float2(-__builtin_inff(), 0.0f);
        float top = m;
#pragma unroll
        for (int k = 0; k < 8; ++k) top = fmaxf(top, q[k].x);
        const float t0 = top == -__builtin_inff() ? 0.0f : top;
        s *= __builtin_amdgcn_exp2f((m - t0) * LOG2E);
#pragma unroll
        for (int k = 0; k < 8; ++k) s += q[k].y * __builtin_amdgcn_exp2f((q[k].x - t0) * LOG2E);
        m = top;
    }
    float dot = 0.0f;
    if (t >= 0) {
        const typename E::T *xr = x + row * x_stride, *wr = w + t * w_stride;
        int c = lane * E::PER16;
        for (; c + 3 * 64 * E::PER16 + E::PER16 <= dim; c += 4 * 64 * E::PER16) {
            float a[4][E::PER16], b[4][E::PER16];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                load_piece<E>(xr + c + q * 64 * E::PER16, a[q]);
                load_piece<E>(wr + c + q * 64 * E::PER16, b[q]);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int k = 0; k < E::PER16; ++k) dot = fmaf(a[q][k], b[q][k], dot);
        }
        for (; c + E::PER16 <= dim; c += 64 * E::PER16) {
            float a[E::PER16], b[E::PER16];
            load_piece<E>(xr + c, a);
            load_piece<E>(wr + c, b);
#pragma unroll
            for (int k = 0; k < E::PER16; ++k) dot = fmaf(a[k], b[k], dot);
        }
        for (; c < dim; ++c) dot = fmaf(E::get(xr[c]), E::get(wr[c]), dot);
    }
    for (int o = 32; o > 0; o >>= 1) {
        const float mo = __shfl_xor(m, o), so = __shfl_xor(s, o);
        const float top = fmaxf(m, mo), t0 = top == -__builtin_inff() ? 0.0f : top;
        s = s * __builtin_amdgcn_exp2f((m - t0) * LOG2E) + so * __builtin_amdgcn_exp2f((mo - t0) * LOG2E);
        m = top;
        dot += __shfl_xor(dot, o);
    }
    if (lane == 0) {
        const double l = (double)m + log((double)s);
        lse[row] = (float)l;
        loss[row] = t >= 0 ? (float)(l - (double)dot) : 0.0f;
    }
}

// ---- host -----------------------------------------------------------------------------------------

// Tiles of C: 256 x 256 by 8 wavefronts, 128 x 128, 128 x 64, 64 x 64 and 32 x 128 by 4.
enum { TILE_256, TILE_128, TILE_128x64, TILE_64, TILE_32 };
static int tile_l(int t) { return t == TILE_256 ? 256 : t == TILE_32 ? 32 : t == TILE_64 ? 64 : 128; }
static int tile_r(int t) { return t == TILE_256 ? 256 : t == TILE_128x64 || t == TILE_64 ? 64 : 128; }
static int strips_per_tile(int t) { return t == TILE_32 ? 4 : t == TILE_128x64 ? 1 : 2; }

// What a product is expected to take, in us: whole rounds of workgroups over the chip (256 of the largest tile, else 512: two to a compute unit), each
// of `steps` times 64 values of k, and what its parts cost to be joined.  Per step and round the tiles take about 1.7 (1.25 PFLOP/s), 1.15, 0.7
// and 0.6 us, a round's start and end 3 us.  (13,834 x 1152 fp32 against 5628 classes: D W has 54 x 5 of the largest tiles, two rounds of which
// the second is nearly empty: 800 us per strip, 128 x 128 tiles 590.)
static double product_cost(int tile, int64_t rows_l, int64_t rows_r, int64_t steps, int splits) {
    const int64_t n = ((rows_l + tile_l(tile) - 1) / tile_l(tile)) * ((rows_r + tile_r(tile) - 1) / tile_r(tile)) * splits;
    const double rounds = (double)((n + (tile == TILE_256 ? 255 : 511)) / (tile == TILE_256 ? 256 : 512));
    const double step = tile == TILE_256 ? 1.7 : tile == TILE_128 ? 1.15 : tile == TILE_64 ? 0.6 : 0.7;
    const double join = splits > 1 ? 4.0 + (double)splits * (double)rows_l * (double)rows_r * 8.0 / 4.0e6 : 0.0;
    return rounds * ((double)((steps + splits - 1) / splits) * step + 3.0) + join;
}

struct Choice {
    int tile, splits;
};
// Tile and parts of the sum; 32 rows of l where there are no more: r is then read once.
static Choice choose(int64_t rows_l, int64_t rows_r, int64_t steps, int most) {
    Choice best = {TILE_256, 1};
    double best_cost = 1e300;
    for (int tile = TILE_256; tile <= TILE_32; ++tile) {
        if ((tile == TILE_32) != (rows_l <= 32) || (tile == TILE_128x64 && rows_r > 64)) continue;
        for (int s = 1; s <= most && (s == 1 || steps / s >= 4); s += s < 8 ? 1 : s < 16 ? 2 : 8) {
            const double c = product_cost(tile, rows_l, rows_r, steps, s);
            if (c < best_cost) { best_cost = c; best = {tile, s}; }
        }
    }
    return best;
}
static int pick_tile(int64_t rows_l, int64_t rows_r, int64_t steps) { return choose(rows_l, rows_r, steps, 1).tile; }

// Tells the runtime once per context that a kernel takes more than the default limit of dynamic LDS.
static void allow_lds(qgbdt_ctx* ctx, const void* kernel, int lds) {
    if (lds <= 65536) return;
    for (int i = 0; i < ctx->lds_told; ++i)
        if (ctx->lds_kernels[i] == kernel) return;
    if (ctx->lds_told < LDS_KERNELS) ctx->lds_kernels[ctx->lds_told++] = kernel;
    (void)hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
}

static unsigned cut(ProductArgs& a, int tile, int64_t rows_l, int64_t rows_r) {
    a.tiles_l = (int)((rows_l + tile_l(tile) - 1) / tile_l(tile));
    a.tiles_r = (int)((rows_r + tile_r(tile) - 1) / tile_r(tile));
    return (unsigned)((a.tiles_l * a.tiles_r * a.splits + 7) / 8 * 8);
}

template <bool LT, bool RT, class Epilogue>
static void launch_product(qgbdt_ctx* ctx, int tile, ProductArgs a, const Epilogue& e, int64_t rows_l, int64_t rows_r) {
    const dim3 grid(cut(a, tile, rows_l, rows_r));
    auto go = [&](auto kernel, int threads, int lds) {
        allow_lds(ctx, reinterpret_cast<const void*>(kernel), lds);
        hipLaunchKernelGGL(kernel, grid, dim3(threads), lds, ctx->stream, a, e);
    };
    if (tile == TILE_256) go(product_kernel<256, 256, 4, 2, 2, LT, RT, Epilogue>, 512, product_lds(256, 256, 2));
    else if (tile == TILE_128) go(product_kernel<128, 128, 2, 2, 2, LT, RT, Epilogue>, 256, product_lds(128, 128, 2));
    else if (tile == TILE_128x64) go(product_kernel<128, 64, 4, 1, 3, LT, RT, Epilogue>, 256, product_lds(128, 64, 3));
    else if (tile == TILE_64) go(product_kernel<64, 64, 2, 2, 3, LT, RT, Epilogue>, 256, product_lds(64, 64, 3));
    else if constexpr (!Epilogue::TURNS) go(product_kernel<32, 128, 1, 4, 6, LT, RT, Epilogue>, 256, product_lds(32, 128, 6));  // (D has 64 rows at least)
}

// Scores of fp32 rows; `three`: where their three bfloat16 pieces lie, of x and of the weights.
template <class Epilogue>
static void launch_scores(qgbdt_ctx* ctx, int tile, ProductArgs a, const uint16_t* three_l, const uint16_t* three_r, const uint32_t* range, const Epilogue& e, int64_t rows_l,
                          int64_t rows_r) {
    const dim3 grid(cut(a, tile, rows_l, rows_r));
    ProductArgs b = a;
    b.l.p = three_l; b.r.p = three_r; b.segs = 6; b.pieces_l = SIX_L; b.pieces_r = SIX_R;
    auto go = [&](auto kernel, int threads, int lds) {
        allow_lds(ctx, reinterpret_cast<const void*>(kernel), lds);
        hipLaunchKernelGGL(kernel, grid, dim3(threads), lds, ctx->stream, a, b, range, e);
    };
    if (tile == TILE_256) go(score_kernel<256, 256, 4, 2, 2, Epilogue>, 512, product_lds(256, 256, 2));
    else if (tile == TILE_128) go(score_kernel<128, 128, 2, 2, 2, Epilogue>, 256, product_lds(128, 128, 2));
    else if (tile == TILE_128x64) go(score_kernel<128, 64, 4, 1, 3, Epilogue>, 256, product_lds(128, 64, 3));
    else if (tile == TILE_64) go(score_kernel<64, 64, 2, 2, 3, Epilogue>, 256, product_lds(64, 64, 3));
    else if constexpr (!Epilogue::TURNS) go(score_kernel<32, 128, 1, 4, 6, Epilogue>, 256, product_lds(32, 128, 6));
}

// Whether the products read fp32 weights where they lie (middle_device.h).  Scores of pieces that are made once take half the products: the loss of
// 256 x 1024 against 20,000 classes takes 84 us with them and 94 without, of 128 x 512 48 and 34; few classes leave most of the chip idle
// either way, and pieces cost launches (512 x 2048 against 2000: 53 and 46).  The gradients have two products of six pieces anyway, and reading D W's
// operands once for all of them decides: 300 x 1000 against 30,000: 556 and 424, 1024 x 1024 against 20,000: 783 and 758, 2048 x 512: 702 and
// 798; 1127 x 2425 against 623, few tiles of long sums: 152 and 130.  Where all is small, D W and D^T X in one launch are worth more (128 x 200
// against 1000: 33 and 44).
static bool middle_rows(int64_t n, int dim, int64_t n_classes, int dtype, int64_t w_stride, bool gradients) {
    if (dtype != QGBDT_F32 || dim <= 128 || w_stride > (1 << 21)) return false;
    if (n <= FEW_ROWS) return !gradients && n_classes >= 12000 && (dim >= 768 || (dim >= 384 && n * dim > 2560));
    const bool small = n * n_classes <= 1200000;
    if (!gradients) return n <= 128 || (n <= 512 && n_classes <= 8192) || small;
    return n <= 64 || ((n <= 1024 || small) && n_classes * dim >= 500000);
}
// Whether few rows go to the kernels that stream the classes (few_device.h).  Their wavefronts read the rows from the caches for every 16 classes, a tile
// in LDS has them once for 32 or 64: with many classes long rows are better off there (loss of 4 x 1792 against 34,840 fp32 classes: 79 -> 61 us, of
// 1 x 2048 against 30,000 bfloat16 ones 33 -> 24; of 1 x 512 against 60,000 fp32 ones it would be 32 -> 35).  Gradients of 9 to 16
// bfloat16 rows that are not swept take a third longer in them (16 x 1024 against 60,000: 160 us, 104), fp32 ones do not (233, 252).
static bool few_rows(int64_t n, int dim, int64_t n_classes, int dtype, bool gradients, bool middle) {
    if (n > FEW_ROWS || middle) return false;
    if (dtype == QGBDT_F32 || dim <= 256) return true;
    return gradients ? n <= 8 : n_classes < 25000 || (dim < 2048 && n * dim < 8192);
}
// Rows of a tile; fewer where the scores' tiles would leave most of the chip idle (loss of 100 x 3392 against 1404: tiles of 128 rows 138 us, of 64 65;
// loss and gradients of 135 rows: tiles of 64 rows 178 us, of 32 152).
static int middle_rows_of(int64_t n, int64_t n_classes, bool classes) {
    if (n <= 32 || (classes && ((n + 63) / 64) * ((n_classes + 63) / 64) <= 128)) return 32;
    return n <= 64 || (classes && n_classes <= 8192) ? 64 : 128;
}
static int middle_cols(int rows) { return rows <= 64 ? 64 : 128; }
// Parts of the sum over the classes for D W, as choose() has them: a step takes about 1.8 us.
static int middle_splits(int64_t n, int dim, int64_t steps) {
    const int rows = middle_rows_of(n, 0, false), cols = middle_cols(rows);
    const int64_t tiles = (dim + cols - 1) / cols * ((n + rows - 1) / rows), room = rows <= 64 ? 512 : 256;
    int best = 1;
    double best_cost = 1e300;
    for (int s = 1; s <= 256 && (s == 1 || steps / s >= 4); ++s) {
        const double cost = (double)((tiles * s + room - 1) / room) * ((double)((steps + s - 1) / s) * 1.8 + 3.0) + (s > 1 ? 4.0 + (double)s * (double)n * dim * 8.0 / 4.0e6 : 0.0);
        if (cost < best_cost) { best_cost = cost; best = s; }
    }
    return best;
}

// C of all rows and `cols` columns of the weights (TR) or classes.
template <bool TR, class Epilogue>
static void launch_middle(qgbdt_ctx* ctx, MiddleArgs a, const Epilogue& e, int64_t n, int rows) {
    const int across = middle_cols(rows);
    a.tiles_l = (int)((n + rows - 1) / rows);
    a.tiles = (a.cols + across - 1) / across;
    a.steps = (a.k + PK - 1) / PK;
    const dim3 grid((unsigned)((a.tiles_l * a.tiles * a.splits + 7) / 8 * 8));
    auto go = [&](auto kernel, int threads, int lds) {
        allow_lds(ctx, reinterpret_cast<const void*>(kernel), lds);
        hipLaunchKernelGGL(kernel, grid, dim3(threads), lds, ctx->stream, a, e);
    };
    // (loss and gradients of 19 x 664 against 53,200, four at a time: 210 us, of 665 values, one at a time: 213, as pieces 466)
    auto pick = [&](auto wide) {
        constexpr bool W = decltype(wide)::value;
        if (rows <= 32) go(middle_kernel<32, 64, 1, 4, 2, TR, W, Epilogue>, 256, middle_lds(32, 64, 2));
        else if (rows <= 64) go(middle_kernel<64, 64, 1, 4, 2, TR, W, Epilogue>, 256, middle_lds(64, 64, 2));
        else go(middle_kernel<128, 128, 2, 4, 2, TR, W, Epilogue>, 512, middle_lds(128, 128, 2));
    };
    if (((reinterpret_cast<uintptr_t>(a.w) | (uintptr_t)a.ld * 4) & 15) == 0 && (TR ? a.cols : a.k) % 4 == 0) pick(std::true_type());
    else pick(std::false_type());
}

constexpr int64_t ROW_BLOCK = 131072;       // rows whose scores, or gradients, are taken together
constexpr int64_t BLOCK_SCORES = 1ll << 37; // scores of such a block in the loss: 8 GB of maxima and sums, 2^21 tiles of the largest kind, 2^30 threads
constexpr int64_t D_VALUES = 128ll << 20;   // values of D that are kept at a time

// Whether the rows are short enough to be swept (sweep_device.h), and to how many values they are filled up; 0: not.
static int sweep_values(int dim, int dtype) {
    if (dtype == QGBDT_F32) return dim <= 64 ? 64 : dim <= 128 ? 128 : 0;
    return dim <= 64 ? 64 : dim <= 128 ? 128 : dim <= 256 ? 256 : 0;
}

// Parts of the swept rows, at most `most`, of at least 2 steps each: what is expected to take the least, in us.  A round of workgroups takes about
// 2.2 us per step of 64 fp32 rows and 0.8 of bf16 ones, and 3 to begin and end; the parts' join a launch of 5 (`joined`).
static int sweep_splits(int64_t kept, int64_t swept, int dtype, int most, bool joined) {
    const int64_t tiles = (kept + SWEEP_KEPT - 1) / SWEEP_KEPT, steps = (swept + SWEEP_TILE - 1) / SWEEP_TILE;
    const double step = dtype == QGBDT_F32 ? 2.2 : 0.8;
    int best = 1;
    double best_cost = 1e300;
    for (int k = 1; k <= most && (k == 1 || steps / k >= 2); ++k) {
        const double rounds = (double)((tiles * k + 511) / 512), cost = rounds * ((double)((steps + k - 1) / k) * step + 3.0) + (k > 1 ? (joined ? 5.0 : 0.0) + 0.02 * k : 0.0);
        if (cost < best_cost) { best_cost = cost; best = k; }
    }
    return best;
}

// most parts of a gradient whose slabs take at most 256 MB
static int sweep_parts(int64_t rows, int dim) {
    const int64_t most = (256 << 20) / (rows * ((dim + 3) / 4 * 16));
    return (int)(most < 1 ? 1 : most > 512 ? 512 : most);
}

// Few rows: parts of the rows' values, and workgroups along the classes.  Up to 2048 blocks of 16 classes a workgroup has one block at a
// time, so that there are enough wavefronts (3 x 1200 fp32 against 12,257 classes: 31 -> 18 us).
static int few_parts(int64_t n_classes) { return n_classes <= 2048 * 16 ? 4 : 1; }
static int few_blocks(int64_t n_classes) {
    const int64_t b = few_parts(n_classes) > 1 ? (n_classes + 15) / 16 : (n_classes + 63) / 64;
    return (int)(few_parts(n_classes) > 1 || b < 1024 ? b : 1024);
}

struct SoftmaxPlan {
    bool few;     // few rows (few_device.h)
    bool middle;  // fp32 weights are read where they lie (middle_device.h)
    int lanes, column_blocks;
    int64_t each;  // few rows: classes per workgroup of the gradients
    int sweep;  // values of a row when they are swept, 0: not
    int pieces, dp;
    bool copy_x, copy_w;
    int64_t row_block, row_blocks, strip, strips;  // gradients: rows together, classes together
    int tile;                                      // loss: of the scores; `strips` is then the wavefronts' strips of classes
    int x_splits, w_splits, x_tile, w_tile;
    bool x_slabs, w_slabs;
    int64_t ld_d, slab_ld;
    // offsets in the scratch block
    size_t common, tops, range, marks, terms, x16, w16, x_back, w_back, x, w, part, d, xs, ws, bytes;
};

static SoftmaxPlan make_softmax_plan(int64_t n, int dim, int64_t n_classes, int dtype, int64_t x_stride, int64_t w_stride, bool gradients) {
    SoftmaxPlan p = {};
    p.pieces = dtype == QGBDT_F32 ? 3 : 1;
    p.dp = (dim + 7) / 8 * 8;
    p.sweep = sweep_values(dim, dtype);
    const bool odd = dtype != QGBDT_BF16 || dim % 8 != 0;
    // (offsets inside a tile of 256 rows are 32-bit)
    p.copy_x = gradients || odd || x_stride % 8 != 0 || x_stride > (1 << 21);
    p.copy_w = odd || w_stride % 8 != 0 || w_stride > (1 << 21);
    p.middle = middle_rows(n, dim, n_classes, dtype, w_stride, gradients);
    p.few = few_rows(n, dim, n_classes, dtype, gradients, p.middle);
    if (p.few || p.middle) p.copy_w = false;  // (read where it lies)
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align256(bytes); return o; };
    const bool halves = p.pieces > 1 && !p.few && !p.middle;  // scores of rows in fp16 pieces
    // (the loss has room for the three bfloat16 pieces in the place of the fp16 ones)
    const size_t half_bytes = gradients ? 4 : 6;
    if (halves) {
        p.range = take(8);
        p.marks = take(2 * LAY_OUT_BLOCKS);
        p.w16 = take((size_t)n_classes * p.dp * half_bytes);
        p.w_back = take((size_t)((n_classes + SWEEP_TILE - 1) / SWEEP_TILE * SWEEP_TILE) * 4);
    }
    // (the loss reads no other pieces than those)
    p.w = p.copy_w && (gradients || !halves) ? take((size_t)n_classes * p.dp * 2 * p.pieces) : 0;
    p.row_block = ROW_BLOCK;
    while (!gradients && p.row_block * n_classes > BLOCK_SCORES) p.row_block /= 2;
    if (p.row_block > n) p.row_block = n;
    p.row_blocks = n > 0 ? (n + p.row_block - 1) / p.row_block : 0;
    if (!gradients) {
        if (halves) {
            p.x16 = take((size_t)p.row_block * p.dp * half_bytes);
            p.x_back = take((size_t)p.row_block * 4);
        }
        p.x = p.copy_x && !halves ? take((size_t)p.row_block * p.dp * 2 * p.pieces) : 0;
        p.tile = pick_tile(p.row_block, n_classes, (int64_t)(p.dp + PK - 1) / PK * (p.pieces > 1 ? 3 : 1));
        if (p.few) p.strips = few_blocks(n_classes);
        else if (p.middle) p.strips = (n_classes + middle_cols(middle_rows_of(n, n_classes, true)) - 1) / middle_cols(middle_rows_of(n, n_classes, true)) * 4;
        else p.strips = p.sweep ? sweep_splits(p.row_block, n_classes, dtype, 512, false) : (n_classes + tile_r(p.tile) - 1) / tile_r(p.tile) * strips_per_tile(p.tile);
        p.part = take((size_t)p.row_block * p.strips * 8);
        p.bytes = at;
        return p;
    }
    p.slab_ld = (dim + 3) / 4 * 4;
    p.common = take(4);
    p.tops = take(WEIGHT_BLOCKS * 4);
    if (p.few) {
        const int pieces = (dim + 3) / 4;
        p.lanes = 1;
        while (p.lanes < pieces && p.lanes < 256) p.lanes <<= 1;
        p.column_blocks = (pieces + p.lanes - 1) / p.lanes;
        // about 1024 workgroups in all, of at least 16 classes per group of threads
        const int64_t most = 1024 / p.column_blocks > 0 ? 1024 / p.column_blocks : 1, least = 4 * (256 / p.lanes);
        p.each = (n_classes + most - 1) / most;
        if (p.each < least) p.each = least;
        p.strips = (n_classes + p.each - 1) / p.each;
        p.ld_d = (n_classes + 15) / 16 * 16;
        p.x = take((size_t)n * p.dp * 2 * p.pieces);
        p.d = take((size_t)n * p.ld_d * 4);
        p.xs = take((size_t)p.strips * n * p.slab_ld * 4);
        p.bytes = at;
        return p;
    }
    if (p.sweep) {  // nothing is kept of D: all rows together
        p.row_block = n; p.row_blocks = 1;
        p.x_splits = sweep_splits(n, n_classes, dtype, sweep_parts(n, dim), true);
        p.w_splits = sweep_splits(n_classes, n, dtype, sweep_parts(n_classes, dim), true);
        p.x_slabs = p.x_splits > 1;
        p.w_slabs = p.w_splits > 1;
        if (halves) {
            p.x16 = take((size_t)n * p.dp * 4);
            p.x_back = take((size_t)n * 4);
        }
        p.terms = take((size_t)((n + SWEEP_TILE - 1) / SWEEP_TILE * SWEEP_TILE) * sizeof(RowTerms));
        p.x = take((size_t)n * p.dp * 2 * p.pieces);
        p.xs = p.x_slabs ? take((size_t)p.x_splits * n * p.slab_ld * 4) : 0;
        p.ws = p.w_slabs ? take((size_t)p.w_splits * n_classes * p.slab_ld * 4) : 0;
        p.bytes = at;
        return p;
    }
    const int64_t rows_out = (p.row_block + 63) / 64 * 64;
    p.strip = D_VALUES / p.pieces / (rows_out > 0 ? rows_out : 1) / 256 * 256;
    if (p.strip < 1024) p.strip = 1024;
    const int64_t most = (n_classes + 255) / 256 * 256;
    if (p.strip > most) p.strip = most;
    p.strips = (n_classes + p.strip - 1) / p.strip;
    // (of one size: 20,051 x 1312 fp32 against 2930 classes in strips of 2048 and 882, with tiles and parts for the former: 3270 us, of 1536 and 1394
    // 2910; 3000 x 512 bf16 against 50,000: 830 and 724)
    p.strip = ((n_classes + p.strips - 1) / p.strips + 255) / 256 * 256;
    p.strips = (n_classes + p.strip - 1) / p.strip;
    p.ld_d = p.strip;
    const int64_t segs = p.pieces > 1 ? 6 : 1;
    const Choice cx = choose(p.row_block, dim, p.strip / PK * segs, 64), cw = choose(p.strip < n_classes ? p.strip : n_classes, dim, rows_out / PK * segs, 64);
    p.x_tile = cx.tile; p.x_splits = cx.splits; p.w_tile = cw.tile; p.w_splits = cw.splits;
    if (p.middle) p.x_splits = middle_splits(n, dim, p.strip / PK);
    p.x_slabs = p.x_splits > 1 || p.strips > 1;
    p.w_slabs = p.w_splits > 1 || p.row_blocks > 1;
    if (halves) {
        p.x16 = take((size_t)p.row_block * p.dp * 4);
        p.x_back = take((size_t)p.row_block * 4);
    }
    p.x = take((size_t)rows_out * p.dp * 2 * p.pieces);
    p.d = take((size_t)rows_out * p.ld_d * 2 * p.pieces);
    p.xs = p.x_slabs ? take((size_t)p.x_splits * p.row_block * p.slab_ld * 4) : 0;
    p.ws = p.w_slabs ? take((size_t)p.w_splits * (p.row_blocks > 1 ? n_classes : p.strip) * p.slab_ld * 4) : 0;
    p.bytes = at;
    return p;
}

size_t softmax_bytes(int64_t n, int dim, int64_t n_classes, int dtype, int64_t x_stride, int64_t w_stride, bool gradients) {
    return make_softmax_plan(n, dim, n_classes, dtype, x_stride, w_stride, gradients).bytes;
}

static int stream_blocks(int64_t items) {
    const int64_t b = (items + 255) / 256;
    return (int)(b < 1 ? 1 : b > 8192 ? 8192 : b);
}

static void lay_out(qgbdt_ctx* ctx, const SoftmaxPlan& p, const void* in, int64_t stride, int64_t rows, int dim, void* out, const LeftOut& src = {}) {
    const dim3 grid(stream_blocks(rows * (p.dp / 8)));
    if (p.pieces > 1)
        hipLaunchKernelGGL((lay_out_kernel<F32, 3>), grid, dim3(256), 0, ctx->stream, static_cast<const float*>(in), stride, rows, dim, p.dp, static_cast<uint16_t*>(out), rows * p.dp, src);
    else
        hipLaunchKernelGGL((lay_out_kernel<BF16, 1>), grid, dim3(256), 0, ctx->stream, static_cast<const uint16_t*>(in), stride, rows, dim, p.dp, static_cast<uint16_t*>(out), rows * p.dp,
                           src);
}

// Workgroups that lay out `rows` rows.
static int lay_out_blocks(int dp, int64_t rows, int* lanes) {
    *lanes = 1;
    while (*lanes < 64 && *lanes * 8 < dp) *lanes <<= 1;
    const int64_t blocks = (rows + 256 / *lanes - 1) / (256 / *lanes);
    return (int)(blocks < LAY_OUT_BLOCKS ? blocks : LAY_OUT_BLOCKS);
}

// w.rows = 0: x alone
static void lay_out_fp32(qgbdt_ctx* ctx, const SoftmaxPlan& p, const Fp32Rows& w, const Fp32Rows& x, int dim, const LeftOut& of_x, uint8_t* marks, uint32_t* range) {
    int lanes;
    const int w_blocks = lay_out_blocks(p.dp, w.rows, &lanes), x_blocks = lay_out_blocks(p.dp, x.rows, &lanes);
    const dim3 grid((unsigned)(w_blocks + x_blocks));
    if (x.three) hipLaunchKernelGGL(lay_out_fp32_kernel<true>, grid, dim3(256), 0, ctx->stream, w, x, w_blocks, dim, p.dp, lanes, of_x, marks, range);
    else hipLaunchKernelGGL(lay_out_fp32_kernel<false>, grid, dim3(256), 0, ctx->stream, w, x, w_blocks, dim, p.dp, lanes, of_x, marks, range);
}

template <class E, int PIECES, int MODE>
static void launch_sweep(qgbdt_ctx* ctx, int values, SweepArgs a) {
    a.tiles = (int)(((int64_t)a.n_kept + SWEEP_KEPT - 1) / SWEEP_KEPT);
    const int total = a.tiles * a.splits;
    const dim3 grid((unsigned)((total + 7) / 8 * 8));
    auto go = [&](auto kernel, int lds) {
        allow_lds(ctx, reinterpret_cast<const void*>(kernel), lds);
        hipLaunchKernelGGL(kernel, grid, dim3(512), lds, ctx->stream, a);
    };
    if (values == 64) go(sweep_kernel<E, 64, PIECES, MODE>, sweep_lds<64, PIECES, MODE>());
    else if (values == 128) go(sweep_kernel<E, 128, PIECES, MODE>, sweep_lds<128, PIECES, MODE>());
    else if constexpr (PIECES == 1) go(sweep_kernel<E, 256, PIECES, MODE>, sweep_lds<256, PIECES, MODE>());
}

int run_softmax_loss(qgbdt_ctx* ctx, const void* x, const void* w, int dtype, int64_t n, int dim, int64_t n_classes, int64_t x_stride,
                     int64_t w_stride, const void* target, int target_bytes, float* loss, float* lse, void* scratch) {
    if (n == 0) return QGBDT_OK;
    const SoftmaxPlan p = make_softmax_plan(n, dim, n_classes, dtype, x_stride, w_stride, false);
    unsigned char* const s = static_cast<unsigned char*>(scratch);
    const bool halves = p.pieces > 1 && !p.few && !p.middle;
    ProductArgs a = {};
    a.r = {static_cast<const uint16_t*>(w), w_stride, 0, (int)n_classes, p.dp};
    const Fp32Rows of_w = {static_cast<const float*>(w), w_stride, n_classes, reinterpret_cast<uint16_t*>(s + p.w16), nullptr, reinterpret_cast<float*>(s + p.w_back)};
    uint32_t* range = reinterpret_cast<uint32_t*>(s + p.range);
    if (halves) {
        a.r = {reinterpret_cast<const uint16_t*>(s + p.w16), p.dp, n_classes * p.dp, (int)n_classes, p.dp};
    } else if (p.copy_w) {
        lay_out(ctx, p, w, w_stride, n_classes, dim, s + p.w);
        a.r = {reinterpret_cast<const uint16_t*>(s + p.w), p.dp, n_classes * p.dp, (int)n_classes, p.dp};
    }
    a.steps = (p.dp + PK - 1) / PK; a.segs = halves ? 3 : 1; a.splits = 1;
    a.pieces_l = halves ? THREE_L : 0; a.pieces_r = halves ? THREE_R : 0;
    float2* const part = reinterpret_cast<float2*>(s + p.part);
    const float *const x_back = reinterpret_cast<const float*>(s + p.x_back), *const w_back = reinterpret_cast<const float*>(s + p.w_back);
    for (int64_t r0 = 0; r0 < n; r0 += p.row_block) {
        const int64_t rows = n - r0 < p.row_block ? n - r0 : p.row_block;
        const char* const xb = static_cast<const char*>(x) + r0 * x_stride * dtype_bytes(dtype);
        const char* const tg = static_cast<const char*>(target) + r0 * target_bytes;
        a.l = {reinterpret_cast<const uint16_t*>(xb), x_stride, 0, (int)rows, p.dp};
        if (halves) {
            const Fp32Rows of_x = {reinterpret_cast<const float*>(xb), x_stride, rows, reinterpret_cast<uint16_t*>(s + p.x16), nullptr, reinterpret_cast<float*>(s + p.x_back)};
            int lanes;
            uint8_t* const marks = s + p.marks;
            const int w_blocks = lay_out_blocks(p.dp, n_classes, &lanes), x_blocks = lay_out_blocks(p.dp, rows, &lanes);
            Fp32Rows w_now = of_w;
            if (r0 > 0) w_now.rows = 0;  // (laid out already)
            lay_out_fp32(ctx, p, w_now, of_x, dim, LeftOut{}, marks + (r0 > 0 ? w_blocks : 0), nullptr);
            // (the range in two words by turns: that of the rows before these is read)
            const uint32_t* const before = r0 > 0 ? range : nullptr;
            range = reinterpret_cast<uint32_t*>(s + p.range) + (r0 / p.row_block & 1);
            const int blocks = stream_blocks((n_classes + rows) * (p.dp / 8));
            hipLaunchKernelGGL(settle_kernel, dim3(blocks < 1024 ? blocks : 1024), dim3(256), 0, ctx->stream, of_w, of_x, dim, p.dp, marks, w_blocks + x_blocks,
                               before, range);
            a.l = {reinterpret_cast<const uint16_t*>(s + p.x16), p.dp, rows * p.dp, (int)rows, p.dp};
        } else if (p.copy_x) {
            lay_out(ctx, p, xb, x_stride, rows, dim, s + p.x);
            a.l = {reinterpret_cast<const uint16_t*>(s + p.x), p.dp, rows * p.dp, (int)rows, p.dp};
        }
        if (p.few) {
            FewArgs v = {};
            v.x = a.l.p; v.x_ld = a.l.ld; v.x_piece = a.l.piece; v.w = w; v.w_ld = w_stride; v.n = (int)rows; v.dim = dim; v.n_classes = n_classes; v.part = part;
            v.parts = few_parts(n_classes);
            if (p.pieces > 1) hipLaunchKernelGGL((few_scores_kernel<F32, 3, false>), dim3((unsigned)p.strips), dim3(256), 0, ctx->stream, v);
            else hipLaunchKernelGGL((few_scores_kernel<BF16, 1, false>), dim3((unsigned)p.strips), dim3(256), 0, ctx->stream, v);
        } else if (p.middle) {
            MiddleArgs v = {};
            v.l = a.l; v.w = static_cast<const float*>(w); v.ld = w_stride; v.cols = (int)n_classes; v.k = dim; v.splits = 1;
            launch_middle<false>(ctx, v, StatsEpilogue<false>{part, (int)p.strips, (int)rows, (int)n_classes, nullptr, nullptr}, rows, middle_rows_of(n, n_classes, true));
        } else if (p.sweep) {
            SweepArgs v = {};
            v.kept = a.l.p; v.kept_ld = a.l.ld; v.kept_piece = a.l.piece; v.n_kept = (int)rows;
            v.swept = a.r.p; v.swept_ld = a.r.ld; v.swept_piece = a.r.piece; v.n_swept = (int)n_classes;
            v.dp = p.dp; v.splits = (int)p.strips; v.part = part; v.kept_back = x_back; v.swept_back = w_back; v.range = range;
            if (halves) launch_sweep<F32, 3, SWEEP_STATS>(ctx, p.sweep, v);
            else launch_sweep<BF16, 1, SWEEP_STATS>(ctx, p.sweep, v);
        } else if (halves) {
            launch_scores(ctx, p.tile, a, a.l.p, a.r.p, range, StatsEpilogue<true>{part, (int)p.strips, (int)rows, (int)n_classes, x_back, w_back}, rows, n_classes);
        } else {
            launch_product<false, false>(ctx, p.tile, a, StatsEpilogue<false>{part, (int)p.strips, (int)rows, (int)n_classes, nullptr, nullptr}, rows, n_classes);
        }
        const dim3 grid((unsigned)((rows + 3) / 4));
        if (dtype == QGBDT_F32)
            hipLaunchKernelGGL(loss_kernel<F32>, grid, dim3(256), 0, ctx->stream, part, (int)p.strips, reinterpret_cast<const float*>(xb), x_stride,
                               static_cast<const float*>(w), w_stride, rows, dim, n_classes, tg, target_bytes, loss + r0, lse + r0);
        else
            hipLaunchKernelGGL(loss_kernel<BF16>, grid, dim3(256), 0, ctx->stream, part, (int)p.strips, reinterpret_cast<const uint16_t*>(xb), x_stride,
                               static_cast<const uint16_t*>(w), w_stride, rows, dim, n_classes, tg, target_bytes, loss + r0, lse + r0);
    }
    QG_HIP(ctx, hipGetLastError());
    return QGBDT_OK;
}

template <class E>
static void join_slabs(qgbdt_ctx* ctx, const float* slab, int64_t slab_size, int64_t slab_ld, int splits, int64_t rows, int dim, typename E::T* out, const float* common) {
    const int64_t pieces = rows * (slab_ld / 4);
    // (one thread per 4 values is enough where there are many, and reads 16 slabs in a row; few values of many slabs are shared out)
    if (splits > 16 && pieces < 1 << 18)
        hipLaunchKernelGGL(join_many_kernel<E>, dim3((unsigned)((pieces + 15) / 16)), dim3(256), 0, ctx->stream, slab, slab_size, (int)slab_ld, splits, rows, dim, out, (int64_t)dim, common);
    else
        hipLaunchKernelGGL(join_kernel<E>, dim3(stream_blocks(pieces)), dim3(256), 0, ctx->stream, slab, slab_size, (int)slab_ld, splits, rows, dim, out, (int64_t)dim, common);
}

template <class E, int PIECES>
static void gradients(qgbdt_ctx* ctx, const SoftmaxPlan& p, const typename E::T* x, const typename E::T* w, int64_t n, int dim, int64_t n_classes,
                      int64_t x_stride, int64_t w_stride, const void* target, int target_bytes, const float* lse, const float* weight,
                      typename E::T* grad_x, typename E::T* grad_w, unsigned char* s) {
    typedef typename E::T T;
    const uint16_t* wp = reinterpret_cast<const uint16_t*>(w);
    int64_t w_ld = w_stride, w_piece = 0;
    const bool halves = PIECES > 1 && !p.few && !p.middle;
    if (p.copy_w) {
        if (!halves) lay_out(ctx, p, w, w_stride, n_classes, dim, s + p.w);
        wp = reinterpret_cast<const uint16_t*>(s + p.w); w_ld = p.dp; w_piece = n_classes * p.dp;
    }
    const uint16_t* const xp = reinterpret_cast<const uint16_t*>(s + p.x);
    const uint16_t *const x16 = reinterpret_cast<const uint16_t*>(s + p.x16), *const w16 = reinterpret_cast<const uint16_t*>(s + p.w16);
    const float *const x_back = reinterpret_cast<const float*>(s + p.x_back), *const w_back = reinterpret_cast<const float*>(s + p.w_back);
    uint32_t* const tops = n > WEIGHTS_AT_ONCE || halves ? reinterpret_cast<uint32_t*>(s + p.tops) : nullptr;
    const int n_tops = (int)(n < WEIGHT_BLOCKS * 1024 ? (n + 1023) / 1024 : WEIGHT_BLOCKS);
    uint32_t* const range = halves ? reinterpret_cast<uint32_t*>(s + p.range) : nullptr;
    if (tops)
        hipLaunchKernelGGL(weight_kernel, dim3(n_tops), dim3(256), 0, ctx->stream, LeftOut{target, target_bytes, n_classes, weight, lse, nullptr, 0, nullptr, nullptr}, n,
                           tops, range);
    auto lay_out_x = [&](int64_t r0, int64_t rows, float* common, RowTerms* terms) {
        const LeftOut src = {static_cast<const char*>(target) + r0 * target_bytes, target_bytes, n_classes, weight + r0, lse + r0, tops, n_tops, common, terms};
        if constexpr (PIECES > 1) {
            if (halves) {  // (with the first rows the weights)
                const Fp32Rows of_w = {w, w_stride, r0 ? 0 : n_classes, reinterpret_cast<uint16_t*>(s + p.w16), reinterpret_cast<uint16_t*>(s + p.w), reinterpret_cast<float*>(s + p.w_back)};
                const Fp32Rows of_x = {x + r0 * x_stride, x_stride, rows, reinterpret_cast<uint16_t*>(s + p.x16), reinterpret_cast<uint16_t*>(s + p.x), reinterpret_cast<float*>(s + p.x_back)};
                lay_out_fp32(ctx, p, of_w, of_x, dim, src, nullptr, range);
                return;
            }
        }
        lay_out(ctx, p, x + r0 * x_stride, x_stride, rows, dim, s + p.x, src);
    };
    if (p.few) {
        float* const common = reinterpret_cast<float*>(s + p.common);
        float* const d = reinterpret_cast<float*>(s + p.d);
        lay_out_x(0, n, common, nullptr);
        FewArgs v = {};
        v.x = xp; v.x_ld = p.dp; v.x_piece = n * p.dp; v.w = w; v.w_ld = w_stride; v.n = (int)n; v.dim = dim; v.n_classes = n_classes;
        v.parts = few_parts(n_classes); v.d = d; v.d_ld = p.ld_d; v.lse = lse; v.weight = weight; v.common = common; v.target = target; v.target_bytes = target_bytes;
        hipLaunchKernelGGL((few_scores_kernel<E, PIECES, true>), dim3(few_blocks(n_classes)), dim3(256), 0, ctx->stream, v);
        FewGradArgs q = {};
        q.x = x; q.w = w; q.x_ld = x_stride; q.w_ld = w_stride; q.n = (int)n; q.dim = dim; q.lanes = p.lanes; q.column_blocks = p.column_blocks;
        q.n_classes = n_classes; q.each = p.each; q.d = d; q.d_ld = p.ld_d; q.common = common; q.grad_w = grad_w;
        q.slab = grad_x ? reinterpret_cast<float*>(s + p.xs) : nullptr; q.slab_ld = p.slab_ld; q.target = target; q.target_bytes = target_bytes; q.weight = weight;
        const dim3 grid((unsigned)(p.strips * p.column_blocks));
        if (n <= 2) hipLaunchKernelGGL((few_gradients_kernel<E, 2>), grid, dim3(256), 0, ctx->stream, q);
        else if (n <= 8) hipLaunchKernelGGL((few_gradients_kernel<E, 8>), grid, dim3(256), 0, ctx->stream, q);
        else hipLaunchKernelGGL((few_gradients_kernel<E, 16>), grid, dim3(256), 0, ctx->stream, q);
        if (grad_x) join_slabs<E>(ctx, q.slab, n * p.slab_ld, p.slab_ld, (int)p.strips, n, dim, grad_x, common);
        return;
    }
    if (p.sweep) {
        float* const common = reinterpret_cast<float*>(s + p.common);
        RowTerms* const terms = reinterpret_cast<RowTerms*>(s + p.terms);
        lay_out_x(0, n, common, terms);
        SweepArgs v = {};
        v.dp = p.dp; v.dim = dim; v.terms = terms; v.unit = common; v.slab_ld = p.slab_ld; v.range = range;
        if (grad_x) {
            v.swept = wp; v.swept_ld = w_ld; v.swept_piece = w_piece; v.n_swept = (int)n_classes; v.swept16 = w16; v.swept_back = w_back;
            v.kept_ld = p.dp; v.kept_piece = n * p.dp; v.splits = p.x_splits;
            v.slab = p.x_slabs ? reinterpret_cast<float*>(s + p.xs) : nullptr; v.slab_size = n * p.slab_ld;
            for (int64_t r0 = 0; r0 < n; r0 += SWEEP_MOST) {  // (so many rows are never in slabs)
                v.kept = xp + r0 * p.dp; v.kept16 = x16 + r0 * p.dp; v.kept_back = x_back + r0; v.terms = terms + r0; v.out = grad_x + r0 * dim;
                v.n_kept = (int)(n - r0 < SWEEP_MOST ? n - r0 : SWEEP_MOST);
                launch_sweep<E, PIECES, SWEEP_ROWS>(ctx, p.sweep, v);
            }
            v.terms = terms;
            if (v.slab) join_slabs<E>(ctx, v.slab, v.slab_size, p.slab_ld, p.x_splits, n, dim, grad_x, common);
        }
        if (grad_w) {
            v.kept = wp; v.kept16 = w16; v.kept_ld = w_ld; v.kept_piece = n_classes * p.dp; v.n_kept = (int)n_classes; v.swept16 = x16; v.kept_back = w_back;
            v.swept = xp; v.swept_ld = p.dp; v.swept_piece = n * p.dp; v.n_swept = (int)n;
            v.splits = p.w_splits; v.out = grad_w; v.slab = p.w_slabs ? reinterpret_cast<float*>(s + p.ws) : nullptr; v.slab_size = n_classes * p.slab_ld;
            launch_sweep<E, PIECES, SWEEP_CLASSES>(ctx, p.sweep, v);
            if (v.slab) join_slabs<E>(ctx, v.slab, v.slab_size, p.slab_ld, p.w_splits, n_classes, dim, grad_w, common);
        }
        return;
    }
    uint16_t* const d = reinterpret_cast<uint16_t*>(s + p.d);
    float* const common = reinterpret_cast<float*>(s + p.common);
    float* const xs = p.x_slabs ? reinterpret_cast<float*>(s + p.xs) : nullptr;
    float* const ws = p.w_slabs ? reinterpret_cast<float*>(s + p.ws) : nullptr;
    ProductArgs base = {};
    base.segs = PIECES > 1 ? 6 : 1;
    base.pieces_l = PIECES > 1 ? SIX_L : 0; base.pieces_r = PIECES > 1 ? SIX_R : 0;
    for (int64_t b = 0; b < p.row_blocks; ++b) {
        const int64_t r0 = b * p.row_block, rows = n - r0 < p.row_block ? n - r0 : p.row_block, rows_out = (rows + 63) / 64 * 64;
        const void* const tg = static_cast<const char*>(target) + r0 * target_bytes;
        const int64_t x_piece = rows * p.dp, d_piece = rows_out * p.ld_d;
        lay_out_x(r0, rows, b == 0 ? common : nullptr, nullptr);
        const int64_t xs_size = rows * p.slab_ld;
        for (int64_t c = 0; c < p.strips; ++c) {
            const int64_t c0 = c * p.strip, cols = n_classes - c0 < p.strip ? n_classes - c0 : p.strip, cols_out = (cols + 63) / 64 * 64;
            ProductArgs a = base;
            a.l = {xp, p.dp, x_piece, (int)rows, p.dp};
            a.r = {wp + c0 * w_ld, w_ld, w_piece, (int)cols, p.dp};
            if (PIECES > 1) {
                a.l.p = x16;
                a.r = {w16 + c0 * p.dp, p.dp, n_classes * p.dp, (int)cols, p.dp};
                a.segs = 3; a.pieces_l = THREE_L; a.pieces_r = THREE_R;
            }
            a.steps = (p.dp + PK - 1) / PK; a.splits = 1;
            GradEpilogue<PIECES> g = {};
            g.d = d; g.ld = p.ld_d; g.piece = d_piece; g.lse = lse + r0; g.weight = weight + r0; g.common = common; g.target = tg; g.target_bytes = target_bytes;
            g.rows = (int)rows; g.rows_out = (int)rows_out; g.cols = (int)cols; g.cols_out = (int)cols_out; g.first = c0; g.n_classes = n_classes;
            if (!p.middle) {
                g.back_l = x_back; g.back_r = w_back + c0;
                const int tile = pick_tile(rows_out, cols_out, a.steps * a.segs);
                if constexpr (PIECES > 1) launch_scores(ctx, tile, a, xp, wp + c0 * w_ld, range, g, rows_out, cols_out);
                else launch_product<false, false>(ctx, tile, a, g, rows_out, cols_out);
            }
            // dX += D W, dW of the strip (+)= D^T X
            ProductArgs ax = base, aw = base;
            ax.l = {d, p.ld_d, d_piece, (int)rows, (int)cols_out};
            ax.r = {wp + c0 * w_ld, w_ld, w_piece, p.dp, (int)cols};
            ax.steps = (int)(cols_out / PK); ax.splits = p.x_splits;
            const StoreEpilogue<E> ex = {grad_x ? grad_x + r0 * dim : nullptr, xs, dim, p.slab_ld, xs_size, (int)rows, dim, c > 0, common};
            const int64_t ws_rows = p.row_blocks > 1 ? n_classes : cols;
            float* const slab = ws ? ws + (p.row_blocks > 1 ? c0 * p.slab_ld : 0) : nullptr;
            aw.l = {d, p.ld_d, d_piece, (int)cols_out, (int)rows_out};
            aw.r = {xp, p.dp, x_piece, p.dp, (int)rows};
            aw.steps = (int)(rows_out / PK); aw.splits = p.w_splits;
            const StoreEpilogue<E> ew = {grad_w ? grad_w + c0 * dim : nullptr, slab, dim, p.slab_ld, ws_rows * p.slab_ld, (int)cols, dim, b > 0, common};
            const int tx = p.x_tile, tw = p.w_tile;
            // (256 x 4099 x 512: 8 and 10 us one after the other, 14 us together)
            ProductArgs sx = ax, sw = aw;
            const unsigned bx = cut(sx, TILE_64, rows, dim), bw = cut(sw, TILE_64, cols, dim);
            if constexpr (PIECES > 1) {
                if (p.middle) {
                    MiddleArgs v = {};
                    v.l = a.l; v.l.p = xp; v.w = w + c0 * w_stride; v.ld = w_stride; v.cols = (int)cols; v.k = dim; v.splits = 1;
                    launch_middle<false>(ctx, v, g, rows, middle_rows_of(n, n_classes, true));
                    v.l = ax.l; v.cols = dim; v.k = (int)cols; v.splits = p.x_splits;
                    if (grad_x) launch_middle<true>(ctx, v, ex, rows, middle_rows_of(n, n_classes, false));
                    if (middle_rows_of(n, n_classes, true) == 32) aw.l.k = (int)((rows + 31) / 32 * 32);  // (all rows of D that the tiles write)
                }
            }
            if (p.middle) {
                if (grad_w) launch_product<true, true>(ctx, tw, aw, ew, cols, dim);
            } else if (grad_x && grad_w && bx + bw <= 1024 && (int64_t)ax.steps * ax.segs <= 16 * ax.splits && (int64_t)aw.steps * aw.segs <= 16 * aw.splits) {
                hipLaunchKernelGGL((product_pair_kernel<64, 64, 2, 2, 3, false, true, true, true, StoreEpilogue<E>>), dim3(bx + bw), dim3(256), product_lds(64, 64, 3),
                                   ctx->stream, sx, ex, sw, ew, (int)bx);
            } else {
                if (grad_x) launch_product<false, true>(ctx, tx, ax, ex, rows, dim);
                if (grad_w) launch_product<true, true>(ctx, tw, aw, ew, cols, dim);
            }
            if (grad_w && slab && b == p.row_blocks - 1) join_slabs<E>(ctx, slab, ws_rows * p.slab_ld, p.slab_ld, p.w_splits, cols, dim, grad_w + c0 * dim, common);
        }
        if (grad_x && xs) join_slabs<E>(ctx, xs, xs_size, p.slab_ld, p.x_splits, rows, dim, grad_x + r0 * dim, common);
    }
}

template <class E>
__global__ __launch_bounds__(256) void fill_zero_kernel(typename E::T* p, int64_t n) {
    const int64_t step = (int64_t)gridDim.x * blockDim.x;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += step) p[i] = 0;
}

int run_softmax_gradients(qgbdt_ctx* ctx, const void* x, const void* w, int dtype, int64_t n, int dim, int64_t n_classes, int64_t x_stride,
                          int64_t w_stride, const void* target, int target_bytes, const float* lse, const float* row_weight,
                          void* grad_x, void* grad_w, void* scratch) {
    if (n == 0) {
        const int64_t m = n_classes * dim;
        if (grad_w && dtype == QGBDT_F32) hipLaunchKernelGGL(fill_zero_kernel<F32>, dim3(stream_blocks(m)), dim3(256), 0, ctx->stream, static_cast<float*>(grad_w), m);
        else if (grad_w) hipLaunchKernelGGL(fill_zero_kernel<BF16>, dim3(stream_blocks(m)), dim3(256), 0, ctx->stream, static_cast<uint16_t*>(grad_w), m);
        QG_HIP(ctx, hipGetLastError());
        return QGBDT_OK;
    }
    const SoftmaxPlan p = make_softmax_plan(n, dim, n_classes, dtype, x_stride, w_stride, true);
    unsigned char* const s = static_cast<unsigned char*>(scratch);
    if (dtype == QGBDT_F32)
        gradients<F32, 3>(ctx, p, static_cast<const float*>(x), static_cast<const float*>(w), n, dim, n_classes, x_stride, w_stride, target,
                          target_bytes, lse, row_weight, static_cast<float*>(grad_x), static_cast<float*>(grad_w), s);
    else
        gradients<BF16, 1>(ctx, p, static_cast<const uint16_t*>(x), static_cast<const uint16_t*>(w), n, dim, n_classes, x_stride, w_stride, target,
                           target_bytes, lse, row_weight, static_cast<uint16_t*>(grad_x), static_cast<uint16_t*>(grad_w), s);
    QG_HIP(ctx, hipGetLastError());
    return QGBDT_OK;
}

}  // namespace qgbdt
