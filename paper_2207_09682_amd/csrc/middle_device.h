// Products of some rows with fp32 class weights.  With few rows it is the weights' bytes that count, so they come to LDS as they lie in memory and a
// wavefront takes its own values of them apart in registers; laid out in pieces, they would be read once more, written and read again (10
// bytes written and 16 read for 4).  The rows, or D, are in three bfloat16 pieces, six products per value, of which LDS is read once for all six.
// Loss and gradients of 30 x 1000 against 30,000 classes: 381 -> 154 us, of 100 x 512 against 60,000: 434 -> 263.  At 50 x 1000 the scores read
// the weights at 2.8 TB/s and D W at 3.4; at 100 rows the matrix units have as much to do as the memory (123 MB in 57 us).
#pragma once
#include "few_device.h"

namespace qgbdt {

struct MiddleArgs {
    ProductOperand l;  // rows, in three pieces, k consecutive
    const float* w;
    int64_t ld;
    int cols, k;       // of the product: classes and the weights' values (not TR), or the weights' values and classes (TR)
    int tiles_l, tiles, steps, splits;
};

// One step's tile of the weights to LDS: BR classes x PK values (256 bytes of a row), or, TR, PK classes x BR values.  Four values at c of row r lie
// at c ^ r % 16, so that 16 lanes that read the same four of consecutive rows meet all 64 banks; TR: of class k at c ^ 4 (k / 8 % 4), so that
// four runs of 16 values, 8 classes apart, do.  A lane brings four values, WIDE, where rows start at multiples of 16 bytes and have whole
// fours, or one.
template <int BR, int T, bool TR, bool WIDE>
struct WeightLoader {
    static constexpr int P = WIDE ? 4 : 1, CB = (TR ? BR : PK) / P, ROUNDS = BR * PK / P / T, PER_ROUND = T / CB;
    uint32_t off[ROUNDS];
    const float* base;
    int64_t advance;
    int k, kk;
    static __device__ __forceinline__ int turned(int row) { return TR ? ((row >> 3) & 3) << 2 : row & 15; }
    // what lies at value v of row r
    static __device__ __forceinline__ int at(int v, int r) { return ((((v >> 2) ^ turned(r)) << 2) | (v & 3)); }
    __device__ __forceinline__ void init(const MiddleArgs& a, int col0, int step, int tid) {
        k = a.k;
        const int row = tid / CB, v = tid % CB * P;
#pragma unroll
        for (int j = 0; j < ROUNDS; ++j) {
            const int r = row + j * PER_ROUND, c = at(v, r), last = TR ? a.cols - P - col0 : a.cols - 1 - col0;
            off[j] = TR ? (uint32_t)r * (uint32_t)(a.ld * 4) + (uint32_t)(c < last ? c : last) * 4u : (uint32_t)(r < last ? r : last) * (uint32_t)(a.ld * 4) + (uint32_t)c * 4u;
        }
        kk = TR ? row : (row << 8) | v;
        advance = TR ? PK * a.ld : PK;
        base = a.w + (TR ? col0 : col0 * a.ld) + step * advance;
    }
    __device__ __forceinline__ void load(int j, uint32_t lds, int wave, int step, bool more) const {
        typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
        const uint64_t from = (uint64_t)base;
        const u32x4 rsrc = {(uint32_t)from, (uint32_t)(from >> 32) & 0xffffu, 0x7fffffffu, 0x00020000u};
        const int left = (more ? k : -(1 << 30)) - step * PK, mine = TR ? kk + j * PER_ROUND : at(kk & 255, (kk >> 8) + j * PER_ROUND);
        const uint32_t o = left > mine ? off[j] : 0xfffffff0u;
        const uint32_t to = __builtin_amdgcn_readfirstlane(lds + (uint32_t)(j * T + wave * 64) * (P * 4u));
        if constexpr (WIDE) asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(o), "s"(rsrc), "s"(to) : "m0");
        else asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(o), "s"(rsrc), "s"(to) : "m0");
    }
};

__host__ __device__ constexpr int middle_lds(int bl, int br, int stages) { return stages * (bl * PK * 6 + br * PK * 4); }

// As product(): WL x WR wavefronts, a lane has C[l][r] of l = lane % 16 and r = 4 (lane / 16) + 0..3 of each block of 16 x 16.
template <int BL, int BR, int WL, int WR, int STAGES, bool TR, bool WIDE, class Epilogue>
__global__ __launch_bounds__(64 * WL * WR) void middle_kernel(MiddleArgs a, Epilogue epi) {
    constexpr int T = 64 * WL * WR, NL = BL / WL / 16, NR = BR / WR / 16, L = BL * PK, STAGE = 3 * L * 2 + BR * PK * 4;  // (elements; bytes)
    extern __shared__ __align__(1024) uint16_t product_tiles[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wl = wave % WL, wr = wave / WL, g = lane >> 4, s = lane & 15;
    const int total = a.tiles_l * a.tiles * a.splits, per = (total + 7) >> 3, id = ((int)blockIdx.x & 7) * per + ((int)blockIdx.x >> 3);  // (neighbours on one XCD)
    if (((int)blockIdx.x >> 3) >= per || id >= total) return;
    const int tl = id % a.tiles_l, across = id / a.tiles_l, split = across / a.tiles, tr = across - split * a.tiles;
    const int t0 = (int)((int64_t)a.steps * split / a.splits), t1 = (int)((int64_t)a.steps * (split + 1) / a.splits);

    TileLoader<BL, T, false> ll;
    WeightLoader<BR, T, TR, WIDE> lw;
    ll.init(a.l, tl * BL, tid);
    lw.init(a, tr * BR, t0, tid);
    FragReader<BL, false> fl;
    fl.init(wl * (BL / WL), lane);
    constexpr int LOADS_L = TileLoader<BL, T, false>::ROUNDS, LOADS = 3 * LOADS_L + WeightLoader<BR, T, TR, WIDE>::ROUNDS;
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint16_t*)product_tiles;
    int next = t0;
    auto load = [&](int stage) {  // (beyond the last step: zeros, so that the loads in flight are always as many)
        const uint32_t to = lds + (uint32_t)stage * STAGE;
#pragma unroll
        for (int j = 0; j < WeightLoader<BR, T, TR, WIDE>::ROUNDS; ++j) lw.load(j, to + 3 * L * 2, wave, next, next < t1);
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            ll.seek(next, p);
#pragma unroll
            for (int j = 0; j < LOADS_L; ++j) ll.load(j, to + p * L * 2, wave, next, next < t1);
        }
        lw.base += lw.advance;
        ++next;
    };
    f32x4 acc[NL][NR];
#pragma unroll
    for (int i = 0; i < NL; ++i)
#pragma unroll
        for (int j = 0; j < NR; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][e] = 0.0f;
    for (int q = 0; q < STAGES; ++q) load(q);
    int stage = 0;
    for (int t = t0; t < t1; ++t) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((STAGES - 1) * LOADS) : "memory");
        const uint16_t* const x_lds = product_tiles + stage * (STAGE / 2);
        const float* const w_lds = reinterpret_cast<const float*>(x_lds + 3 * L);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            bf16x8 y[NR][3], x[NL][3];
#pragma unroll
            for (int j = 0; j < NR; ++j) {
                const int r0 = wr * (BR / WR) + j * 16, k0 = kk * 32 + g * 8;
                float v[8];
                if constexpr (TR) {  // (k0 is a multiple of 8: the eight classes are turned alike)
                    const float* const p = w_lds + k0 * BR + (((r0 / 4) ^ WeightLoader<BR, T, TR, WIDE>::turned(k0)) << 2) + s;
#pragma unroll
                    for (int h = 0; h < 8; ++h) v[h] = p[h * BR];
                } else {
                    const float* const p = w_lds + (r0 + s) * PK;
#pragma unroll
                    for (int h = 0; h < 2; ++h) __builtin_memcpy(v + 4 * h, __builtin_assume_aligned(p + ((((k0 >> 2) + h) ^ s) << 2), 16), 16);
                }
                eight_in_pieces(v, y[j]);
            }
#pragma unroll
            for (int i = 0; i < NL; ++i)
#pragma unroll
                for (int p = 0; p < 3; ++p) x[i][p] = fl.read(x_lds + p * L, i, kk);
#pragma unroll
            for (int q = 0; q < 6; ++q)
#pragma unroll
                for (int i = 0; i < NL; ++i)
#pragma unroll
                    for (int j = 0; j < NR; ++j) acc[i][j] = matrix_product<false>(y[j][(SIX_R >> (4 * q)) & 0xf], x[i][(SIX_L >> (4 * q)) & 0xf], acc[i][j]);
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // nobody reads the stage any more
        load(stage);
        stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    static_assert(!Epilogue::TURNS || BL * BR * 2 <= STAGES * STAGE, "the wavefronts' values fit");
    epi.template finish<NL, NR>(acc, tl * BL + wl * (BL / WL), tr * BR + wr * (BR / WR), tr * WR + wr, split, lane, product_tiles + wave * (NL * 16 * NR * 16));
}

}  // namespace qgbdt
