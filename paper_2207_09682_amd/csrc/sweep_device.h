// Short rows (up to 128 fp32 or 256 bfloat16 values): a wavefront keeps 32 rows of one matrix in registers and goes through the rows of the
// other, tile by tile, and what it makes of their scores never leaves the registers.
//   STATS  rows of x against all classes: maximum and sum of exponentials
//   ROWS   rows of x against all classes: D, and at once D W
//   CLASSES  classes against all rows of x: D^T, and at once D^T x
// The gradients make the scores twice, which costs as much as one more product of `dim` values, 2 dim per score; writing D and
// reading it twice costs 6 bytes per score (18 in pieces), more than 256 values' worth at this chip's rates.
// Bound by the matrix units and the exponentials between their instructions, and by power: 100,003 x 64 fp32 against 10,007 classes, in products of
// pieces: STATS 0.43 ms (3 of them, 890 TFLOP/s), ROWS 1.10 and CLASSES 1.20 ms (9 of them, 1050 and 960 TFLOP/s).
#pragma once
#include "product_device.h"

namespace qgbdt {

enum { SWEEP_STATS, SWEEP_ROWS, SWEEP_CLASSES };
constexpr int SWEEP_KEPT = 256;   // rows that a workgroup of 8 wavefronts keeps
constexpr int SWEEP_TILE = 64;    // rows of the other matrix are filled up to a multiple of this
constexpr int64_t SWEEP_MOST = 1 << 30;  // rows kept by a launch: fewer than 2^32 threads

// A row of x: p = exp2(score * log2(e) + b), its weight in units of the common one, its class or -1.  A row that is left out has
// b = -infinity and weight 0.
struct RowTerms {
    float b, u;
    int t;
    float back;  // in fp16 pieces: takes the row's scores back
};

struct SweepArgs {
    const uint16_t *kept, *swept;  // rows of 8-element pieces
    int64_t kept_ld, swept_ld, kept_piece, swept_piece;
    // fp32 rows: `kept`, and `swept` for STATS, are in the pieces that the scores are made of, which `range` says; else `swept` is in three bfloat16
    // pieces for the second product, swept16 and kept16 are in two fp16 ones for the scores (rows of dp values, pieces a matrix apart)
    const uint16_t *swept16, *kept16;
    const uint32_t* range;
    const float *kept_back, *swept_back;  // (CLASSES: the swept rows' are in their terms)
    int n_kept, n_swept, dp;       // n_kept: at most SWEEP_MOST; dp: values of a row that exist, a multiple of 8
    int tiles, splits;             // workgroups along the kept rows; parts of the swept ones
    const RowTerms* terms;         // of the rows of x, padded to a multiple of SWEEP_TILE
    const float* unit;
    float2* part;                  // STATS: [n_kept][splits]
    void* out;                     // ROWS, CLASSES: the result, or
    float* slab;                   // not null: [splits][n_kept][slab_ld]
    int64_t slab_ld, slab_size;
    int dim;
};

// Piece c of a row lies at c ^ swept_turn(row).  A read of 16 bytes per lane takes lanes 0-3, 12-15 and 20-27 together, and their like: the pieces of
// one column of 8 rows of a block of 16 and of its neighbour (which differs in bit 0) of the other 8.  They are in 16 different places of 256
// bytes, and so are the 32 bytes each of 8 consecutive rows (transposing reads).
template <int CB>
__device__ __forceinline__ int swept_turn(int row) {
    return CB == 8 ? ((row >> 1) & 3) << 1 : (row & 7) << 1;
}

// Pieces of a swept row in LDS: for the scores, and behind them for the second product where those are others.  HALVES: fp32 rows whose scores are of
// two fp16 pieces.
template <int PIECES, int MODE, bool HALVES>
struct SweepPieces {
    static constexpr bool F16 = HALVES;
    static constexpr int SCORE = F16 ? 2 : PIECES, SECOND = MODE == SWEEP_STATS ? 0 : PIECES, ALL = F16 ? SCORE + SECOND : PIECES;
    static constexpr int SECOND_AT = F16 ? SCORE : 0;
    static constexpr bool TERMS = MODE == SWEEP_CLASSES, BACK = F16 && MODE != SWEEP_CLASSES;
};
// Swept rows per step (32 where the tile of 64 would leave LDS for two stages only), stages, bytes of LDS (1 KB of each for the rows' terms).
template <int DP, int PIECES, int MODE, bool HALVES>
struct SweepShape {
    typedef SweepPieces<PIECES, MODE, HALVES> P;
    static constexpr int TILE = P::ALL * 64 * DP * 2 * 3 > 150 * 1024 ? 32 : 64;
    static constexpr int STAGES = 3;
    static constexpr int TERMS = P::ALL * TILE * DP, STAGE = TERMS + (P::TERMS || P::BACK ? 512 : 0);  // elements
    static constexpr int LDS = STAGES * STAGE * 2;
};

template <class E, int DP, int PIECES, int MODE, bool HALVES>
__device__ __forceinline__ void sweep(const SweepArgs& a) {
    typedef SweepPieces<PIECES, MODE, HALVES> SP;
    typedef SweepShape<DP, PIECES, MODE, HALVES> SH;
    constexpr int CB = DP / 8, NK = DP / 32, NM = DP / 16, TILE = SH::TILE, STAGES = SH::STAGES, STAGE = SH::STAGE, TERMS = SH::TERMS;
    constexpr int ROUNDS = SP::ALL * TILE * CB / 512, LOADS = ROUNDS + (SP::TERMS || SP::BACK ? 1 : 0);
    static_assert(TILE * CB % 512 == 0, "a round's loads are of one piece");
    extern __shared__ __align__(1024) uint16_t product_tiles[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, s = lane & 15;
    const int total = a.tiles * a.splits, per = (total + 7) >> 3, in = (int)(blockIdx.x >> 3);
    const int id = (int)(blockIdx.x & 7) * per + in;  // neighbouring tiles on one XCD
    if (in >= per || id >= total) return;
    const int split = id / a.tiles, kept0 = (id - split * a.tiles) * SWEEP_KEPT + wave * 32;
    const int steps = (int)(((int64_t)a.n_swept + TILE - 1) / TILE);
    const int t0 = (int)((int64_t)steps * split / a.splits), t1 = (int)((int64_t)steps * (split + 1) / a.splits);

    // the kept rows: lane % 16 of a block of 16, values 32 k + 8 (lane / 16) + 0..7
    bf16x8 x[2][NK][SP::SCORE];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int row = kept0 + i * 16 + s;
        const uint16_t* const p = (SP::F16 && MODE != SWEEP_STATS ? a.kept16 : a.kept) + (int64_t)(row < a.n_kept ? row : a.n_kept - 1) * a.kept_ld + g * 8;
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
            for (int q = 0; q < SP::SCORE; ++q) {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (k * 32 + g * 8 < a.dp) v = *reinterpret_cast<const uint4*>(p + k * 32 + q * a.kept_piece);
                x[i][k][q] = __builtin_bit_cast(bf16x8, v);
            }
    }
    // Whether a class that is kept has weights that are not finite: only then is a score of a row that is left out, and so all zeros, no zero.
    bool odd = false;
    if constexpr (MODE == SWEEP_CLASSES) {
        constexpr uint32_t EXPONENT = SP::F16 ? 0x7c007c00u : 0x7f807f80u, ONE = SP::F16 ? 0x04000400u : 0x00800080u;
        uint32_t over = 0;  // exponents of ones run over into the sign's place
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int k = 0; k < NK; ++k) {
                const uint4 v = __builtin_bit_cast(uint4, x[i][k][0]);
                over |= ((v.x & EXPONENT) + ONE) | ((v.y & EXPONENT) + ONE) | ((v.z & EXPONENT) + ONE) | ((v.w & EXPONENT) + ONE);
            }
        odd = __ballot((over & 0x80008000u) != 0) != 0;
    }
    float b[2], u[2];
    int t[2];
    if constexpr (MODE == SWEEP_ROWS) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = kept0 + i * 16 + s;
            const RowTerms r = a.terms[row < a.n_kept ? row : a.n_kept - 1];
            b[i] = r.b; u[i] = r.u; t[i] = r.u != 0.0f ? r.t : -1;
        }
    }

    float kept_back[2] = {1.0f, 1.0f};
    if constexpr (SP::F16) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = kept0 + i * 16 + s;
            kept_back[i] = a.kept_back[row < a.n_kept ? row : a.n_kept - 1];
        }
    }

    const float kept_log2[2] = {kept_back[0] * LOG2E, kept_back[1] * LOG2E};

    // loads of a step
    uint32_t off[ROUNDS];
    int at_row[ROUNDS];
#pragma unroll
    for (int j = 0; j < ROUNDS; ++j) {
        const int q = j * 512 + tid, row = (q / CB) % TILE, c = (q % CB) ^ swept_turn<CB>(row);
        const int64_t ld = SP::F16 && MODE != SWEEP_STATS && q / (TILE * CB) < SP::SCORE ? a.dp : a.swept_ld;
        off[j] = (uint32_t)row * (uint32_t)(ld * 2) + (uint32_t)c * 16u;
        at_row[j] = c * 8 < a.dp ? row : 0x7fffffff;  // (never below the rows that are left)
    }
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint16_t*)product_tiles;
    typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
    auto to_lds = [&](const void* base, uint32_t o, uint32_t to) {
        const uint64_t at = (uint64_t)base;
        const u32x4 rsrc = {(uint32_t)at, (uint32_t)(at >> 32) & 0xffffu, 0x7fffffffu, 0x00020000u};
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(o), "s"(rsrc), "s"(__builtin_amdgcn_readfirstlane(to)) : "m0");
    };
    auto bring = [&](int step, int stage) {  // (beyond the last step: zeros)
        const int64_t row0 = (int64_t)step * TILE;
        const int left = step < t1 ? (int)(a.n_swept - row0) : 0;
        const uint32_t to = lds + (uint32_t)stage * (STAGE * 2) + (uint32_t)wave * 1024u;
#pragma unroll
        for (int j = 0; j < ROUNDS; ++j) {
            const int piece = j * 512 / (TILE * CB);
            const uint16_t* base;
            if (SP::F16 && MODE != SWEEP_STATS && piece < SP::SCORE) base = a.swept16 + (int64_t)piece * a.n_swept * a.dp + row0 * a.dp;
            else base = a.swept + (int64_t)(piece - (MODE == SWEEP_STATS ? 0 : SP::SECOND_AT)) * a.swept_piece + row0 * a.swept_ld;
            to_lds(base, at_row[j] < left ? off[j] : 0xfffffff0u, to + j * 8192u);
        }
        if constexpr (SP::TERMS)  // (every wavefront the same: all have as many loads in flight)
            to_lds(a.terms + row0, step < t1 && lane < TILE ? (uint32_t)lane * 16u : 0xfffffff0u, to - (uint32_t)wave * 1024u + TERMS * 2);
        if constexpr (SP::BACK)
            to_lds(a.swept_back + row0, step < t1 && lane < TILE / 4 ? (uint32_t)lane * 16u : 0xfffffff0u, to - (uint32_t)wave * 1024u + TERMS * 2);
    };

    f32x4 out[2][MODE == SWEEP_STATS ? 1 : NM];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int m = 0; m < (MODE == SWEEP_STATS ? 1 : NM); ++m) out[i][m] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    float top[2] = {-__builtin_inff(), -__builtin_inff()}, sum[2] = {0.0f, 0.0f};

    f32x4 acc[2][2];
    bf16x8 d[2][PIECES];
    // scores of 32 swept rows: the lane has those of kept row s and swept rows 16 j + 4 g + e
    auto scores = [&](const uint16_t* tile, int h) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < NK; ++k) {
            bf16x8 y[2][SP::SCORE];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int q = 0; q < SP::SCORE; ++q)
                    y[j][q] = *reinterpret_cast<const bf16x8*>(tile + (q * TILE + (h * 2 + j) * 16 + s) * DP + (((k * 4 + g) ^ swept_turn<CB>(s)) << 3));
            constexpr int PRODUCTS = SP::SCORE == 3 ? 6 : SP::SCORE == 2 ? 3 : 1;  // (of pieces, smallest first)
            constexpr uint32_t OF_L = SP::SCORE == 3 ? SIX_L : SP::SCORE == 2 ? THREE_R : 0, OF_R = SP::SCORE == 3 ? SIX_R : SP::SCORE == 2 ? THREE_L : 0;
#pragma unroll
            for (int p = 0; p < PRODUCTS; ++p)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int i = 0; i < 2; ++i) acc[i][j] = matrix_product<SP::F16>(y[j][(OF_R >> (4 * p)) & 0xf], x[i][k][(OF_L >> (4 * p)) & 0xf], acc[i][j]);
        }
    };
    // what becomes of them: the running maximum and sum, or D as an operand
    auto values = [&](const uint16_t* tile, int h, int first) {
        const bool whole = first + 32 <= a.n_swept;
        if constexpr (MODE == SWEEP_STATS) {
            if constexpr (SP::BACK) {
                const float* const back = reinterpret_cast<const float*>(tile + TERMS) + h * 32;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float4 c = *reinterpret_cast<const float4*>(back + j * 16 + g * 4);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        acc[i][j][0] = acc[i][j][0] * kept_back[i] * c.x; acc[i][j][1] = acc[i][j][1] * kept_back[i] * c.y;
                        acc[i][j][2] = acc[i][j][2] * kept_back[i] * c.z; acc[i][j][3] = acc[i][j][3] * kept_back[i] * c.w;
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float m = top[i];
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (!whole && first + j * 16 + g * 4 + e >= a.n_swept) acc[i][j][e] = -__builtin_inff();
                        m = fmaxf(m, acc[i][j][e]);
                    }
                const float m0 = m == -__builtin_inff() ? 0.0f : m, mb = -m0 * LOG2E;
                float v = sum[i] * __builtin_amdgcn_exp2f((top[i] - m0) * LOG2E);
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) v += __builtin_amdgcn_exp2f(fmaf(acc[i][j][e], LOG2E, mb));
                sum[i] = v;
                top[i] = m;
            }
        } else if constexpr (MODE == SWEEP_ROWS) {
            const float* const back = reinterpret_cast<const float*>(tile + TERMS) + h * 32;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float c[4] = {LOG2E, LOG2E, LOG2E, LOG2E};
                    if constexpr (SP::BACK) {
                        const float4 v = *reinterpret_cast<const float4*>(back + j * 16 + g * 4);
                        c[0] = v.x; c[1] = v.y; c[2] = v.z; c[3] = v.w;
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] = __builtin_amdgcn_exp2f(fmaf(SP::F16 ? acc[i][j][e] * kept_log2[i] : acc[i][j][e], c[e], b[i]));
                }
                const unsigned want = (unsigned)(t[i] - first);
                if (__ballot(want < 32u) != 0)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (want == (unsigned)(j * 16 + g * 4 + e)) acc[i][j][e] -= 1.0f;
                if (!whole)  // (zeros times what exp2(b) is)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (first + j * 16 + g * 4 + e >= a.n_swept) acc[i][j][e] = 0.0f;
            }
        } else {
            const RowTerms* const terms = reinterpret_cast<const RowTerms*>(tile + TERMS) + h * 32;
            const bool any = __ballot((unsigned)(terms[lane & 31].t - kept0) < 32u) != 0;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const RowTerms r = terms[j * 16 + g * 4 + e];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float v = r.u * __builtin_amdgcn_exp2f(SP::F16 ? fmaf(acc[i][j][e] * kept_log2[i], r.back, r.b) : fmaf(acc[i][j][e], LOG2E, r.b));
                        if (any && r.t == kept0 + i * 16 + s) v -= r.u;
                        acc[i][j][e] = v;
                    }
                }
            if (odd) {
                asm volatile("" ::: "memory");  // (the weights are read again, not kept)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bool left_out = terms[j * 16 + g * 4 + e].u == 0.0f;
#pragma unroll
                        for (int i = 0; i < 2; ++i) acc[i][j][e] = left_out ? 0.0f : acc[i][j][e];
                    }
            }
        }
        // its k-th value is that of swept row 16 (k / 4 % 2) + 4 (k / 8) + k % 4, and so are the other operand's
        if constexpr (MODE != SWEEP_STATS)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int q = 0; q < PIECES; ++q)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const __bf16 v = (__bf16)acc[i][j][e];
                            d[i][q][j * 4 + e] = v;
                            if (q + 1 < PIECES) acc[i][j][e] -= (float)v;
                        }
    };
    // D times the same 32 swept rows
    auto second = [&](const uint16_t* tile, int h) {
        if constexpr (MODE != SWEEP_STATS)
#pragma unroll
            for (int m = 0; m < NM; ++m) {
                bf16x8 z[PIECES];
                const int row = h * 32 + g * 4 + (s >> 2), c = m * 2 + ((s >> 1) & 1);
                typedef __attribute__((address_space(3))) short4v* lp;
#pragma unroll
                for (int q = 0; q < PIECES; ++q) {
                    const uint16_t* const p = tile + ((SP::SECOND_AT + q) * TILE + row) * DP + ((c ^ swept_turn<CB>(row & 15)) << 3) + ((s & 1) << 2);
                    union { short4v w[2]; bf16x8 v; } o;
                    o.w[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)p);
                    o.w[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(p + 16 * DP));
                    z[q] = o.v;
                }
#pragma unroll
                for (int n = PIECES == 3 ? 0 : 5; n < 6; ++n) {  // the six products of pieces, smallest first
                    const int pl = PIECES == 3 ? (SIX_L >> (4 * n)) & 0xf : 0, pr = PIECES == 3 ? (SIX_R >> (4 * n)) & 0xf : 0;
#pragma unroll
                    for (int i = 0; i < 2; ++i) out[i][m] = matrix_product<false>(z[pr], d[i][pl], out[i][m]);
                }
            }
    };

    int into = 0, stage = 0;
#pragma unroll
    for (int k = 0; k < STAGES - 1; ++k) bring(t0 + k, into++);
    for (int step = t0; step < t1; ++step) {
        // (lgkmcnt: what is brought now goes to the place that the step before was read from)
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((STAGES - 2) * LOADS) : "memory");
        bring(step + STAGES - 1, into);
        into = into + 1 == STAGES ? 0 : into + 1;
        const uint16_t* const tile = product_tiles + stage * STAGE;
        stage = stage + 1 == STAGES ? 0 : stage + 1;
#pragma unroll
        for (int h = 0; h < TILE / 32; ++h) {
            scores(tile, h);
            values(tile, h, MODE == SWEEP_CLASSES ? 0 : step * TILE + h * 32);  // (classes; of rows there may be more than fit)
            second(tile, h);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // nothing on its way to LDS when the workgroup ends

#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int row = kept0 + i * 16 + s;
        if constexpr (MODE == SWEEP_STATS) {
            float m = top[i], v = sum[i];
#pragma unroll
            for (int o = 16; o < 64; o <<= 1) {
                const float mo = __shfl_xor(m, o), vo = __shfl_xor(v, o);
                const float big = fmaxf(m, mo), m0 = big == -__builtin_inff() ? 0.0f : big;
                v = v * __builtin_amdgcn_exp2f((m - m0) * LOG2E) + vo * __builtin_amdgcn_exp2f((mo - m0) * LOG2E);
                m = big;
            }
            if (g == 0 && row < a.n_kept) a.part[(int64_t)row * a.splits + split] = make_float2(m, v);
        } else {
            if (row >= a.n_kept) continue;
            const float by = (MODE == SWEEP_ROWS ? u[i] : 1.0f) * (a.slab ? 1.0f : *a.unit);
            const bool left_out = MODE == SWEEP_ROWS && u[i] == 0.0f;  // (zeros, whatever its sums are)
#pragma unroll
            for (int m = 0; m < NM; ++m) {
                const int col = m * 16 + g * 4;
                if (col >= a.dim) continue;
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = left_out ? 0.0f : out[i][m][e] * by;
                if (a.slab) {
                    *reinterpret_cast<float4*>(a.slab + split * a.slab_size + row * a.slab_ld + col) = make_float4(v[0], v[1], v[2], v[3]);
                } else {
                    typename E::T* const o = static_cast<typename E::T*>(a.out) + (int64_t)row * a.dim + col;
                    typename E::T c[4] = {E::put(v[0]), E::put(v[1]), E::put(v[2]), E::put(v[3])};
                    if (col + 4 <= a.dim) __builtin_memcpy(o, c, sizeof(c));
                    else
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (col + e < a.dim) o[e] = c[e];
                }
            }
        }
    }
}

template <class E, int DP, int PIECES, int MODE>
__global__ __launch_bounds__(512) void sweep_kernel(SweepArgs a) {
    if constexpr (PIECES == 3) {
        if (in_three_pieces(*a.range)) sweep<E, DP, PIECES, MODE, false>(a);
        else sweep<E, DP, PIECES, MODE, true>(a);
    } else {
        sweep<E, DP, PIECES, MODE, false>(a);
    }
}

template <int DP, int PIECES, int MODE>
constexpr int sweep_lds() {
    constexpr int halves = PIECES == 3 ? SweepShape<DP, PIECES, MODE, PIECES == 3>::LDS : 0, all = SweepShape<DP, PIECES, MODE, false>::LDS;
    return halves > all ? halves : all;
}

}  // namespace qgbdt
