// C[l][r] = sum over k of L[l][k] R[r][k] on the matrix cores, operands in bfloat16, sums in fp32: the product that the
// softmax loss and its gradients are made of.  What becomes of C is the epilogue's affair.  Bound by the matrix units and, in large
// products, by power (the clock falls to 1.6 GHz).  Tiles of 256 x 256 take the fewest bytes from the L2s and LDS per product and one fills a
// compute unit; 16 x 16 x 32 instructions draw less than 32 x 32 x 16 ones.  8192 x 2048 against 131,072 bfloat16: scores 3.41 ms, 1290 TFLOP/s; per
// strip of 16,384 classes D 0.47 ms, D W 0.43 and D^T X 0.41 (1330 TFLOP/s).
#pragma once
#include "head.h"

namespace qgbdt {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) short short4v;
typedef __attribute__((ext_vector_type(4))) float f32x4;

constexpr float LOG2E = 1.44269504088896340736f;
constexpr int PK = 64;  // k values per step: 128 bytes of a row, a cache line

template <bool F16>
__device__ __forceinline__ f32x4 matrix_product(bf16x8 a, bf16x8 b, f32x4 c) {
    if constexpr (F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// An operand as it lies in memory.  Not transposed: [rows][k], `ld` elements from row to row, k consecutive.  Transposed:
// [k][rows], rows consecutive.  Both are read in 16-byte pieces that start at multiples of 16 bytes.
struct ProductOperand {
    const uint16_t* p;
    int64_t ld;
    int64_t piece;  // elements from one piece of a split fp32 value to the next (0: one piece)
    int rows;       // rows that exist (a multiple of 8 when transposed); reads beyond are held to the last ones
    int k;          // values of k that exist (a multiple of 8 when not transposed); what is beyond is read as zeros
};

struct ProductArgs {
    ProductOperand l, r;
    int tiles_l, tiles_r;
    int steps;   // of PK values of k per segment
    int segs;    // 1, or products of pieces for split fp32 values
    uint32_t pieces_l, pieces_r;  // of the segments
    int splits;  // parts of the k range, each with a C of its own
};

// fp32 values in pieces.
//  * Three of bfloat16, hi + mid + lo (8 bits each, to the nearest): any value, and the six products whose size is at least 2^-18 of the largest,
//    smallest first.  What is left out is below 2^-26 of |l||r|, less than fp32's own rounding.
//  * Two of fp16, hi + lo (11 bits each), of rows scaled by a power of two that brings their largest value to 2^14 .. 2^15: half the
//    products.  Values down to 2^-17 of their row's largest keep 22 bits, smaller ones what lies above 2^-39 of it; what is left out, lo lo, is
//    below 2^-22 of |l||r|.  For scores, where the rows allow it (in_three_pieces).
// Nibble s of these: the piece of segment s.
constexpr uint32_t SIX_L = 0x001012, SIX_R = 0x010210, THREE_L = 0x001, THREE_R = 0x010;

// What rows of fp32 values say about two pieces of fp16, found when they are laid out.  A value below 2^-17 of its row's largest, a FAINT one, is off by
// up to 2^-39 of that.  Without such a value in any row a score is off by 3 2^-22 of the sum of its terms' magnitudes at most.  With them it depends on
// what they meet: a LOOSE row has more than a quarter of its values below 2^-9 of its largest, zeros among them.  Where no row of either matrix is
// loose, any two have half of their `dim` values above that in common, so the magnitudes add up to dim / 2 * 2^-18 * |largest l||largest r| at
// least, and the faint ones, a quarter of each row at most, add an error of dim / 2 * 2^-39 of the same: 2^-21.  Together 20 units of fp32.
// WIDE: a row's largest value is beyond 2^-50 .. 2^50, and scaling the scores back could leave fp32's range on the way.
// Scores are of three bfloat16 pieces where that does not hold, of two fp16 ones where it does.
enum { RANGE_LOOSE = 1, RANGE_FAINT = 2, RANGE_WIDE = 4 };
__device__ __forceinline__ bool in_three_pieces(uint32_t range) { return (range & RANGE_WIDE) || (range & (RANGE_LOOSE | RANGE_FAINT)) == (RANGE_LOOSE | RANGE_FAINT); }

// A read of 16 bytes per lane takes 16 lanes at a time from 64 banks, so 16 consecutive rows (128 bytes each) have to put the same piece
// into 16 different places of 256 bytes: piece c of row r lies at c ^ (r / 2) % 8.
//
// Position of 16-byte piece c of k row `k` of a transposed tile that is `CB` pieces wide: a transposing read takes 32 lanes at a time, 32
// bytes each of 4 rows of k and of the 4 that lie 8 rows further on; they come from different banks.
template <int CB>
__device__ __forceinline__ int turned(int k) {
    return CB >= 16 ? (((k & 3) | ((k >> 1) & 4)) << 1) : CB == 8 ? ((((k >> 1) & 1) | ((k >> 2) & 2)) << 1) : (((k >> 3) & 1) << 1);
}

// Brings one step's tile of an operand to LDS: B rows x PK values, by T threads, 16 bytes each at a time.  The loads go through a
// buffer descriptor whose base is the tile's place in this step; a lane whose place does not exist asks beyond the
// descriptor's range and gets zeros.  They write LDS and no register, so they are issued as they stand (the compiler, which would wait for
// them before any read of LDS, does not see them): who reads waits for vmcnt.
template <int B, int T, bool TR>
struct TileLoader {
    static constexpr int CB = B / 8;
    static constexpr int PIECES = B * PK / 8;                       // of 16 bytes
    static constexpr int ROUNDS = PIECES / T;
    static_assert(PIECES % T == 0 && PIECES >= T, "every wavefront has a part in every round");
    static constexpr int PER_ROUND = TR ? T / CB : T / (PK / 8);    // rows (of k when transposed) per round
    uint32_t off[ROUNDS];  // bytes from the base
    const uint16_t* base;  // of the next step
    const uint16_t* start;
    int64_t advance, piece;
    int k, kk;  // values of k; this lane's place in a step (transposed: of round 0)

    __device__ __forceinline__ void init(const ProductOperand& o, int row0, int tid) {
        piece = o.piece;
        k = o.k;
        if constexpr (TR) {
            const int kr = tid / CB, last = o.rows / 8 - 1 - row0 / 8;
#pragma unroll
            for (int j = 0; j < ROUNDS; ++j) {
                const int krj = kr + j * PER_ROUND, c = (tid % CB) ^ turned<CB>(krj);
                off[j] = (uint32_t)krj * (uint32_t)(o.ld * 2) + (uint32_t)(c < last ? c : last) * 16u;
            }
            start = o.p + row0;
            advance = (int64_t)PK * o.ld;
            kk = kr;
        } else {
            const int chunk = (tid & 7) ^ ((tid >> 4) & 7), last = o.rows - 1 - row0;
#pragma unroll
            for (int j = 0; j < ROUNDS; ++j) {
                const int row = (tid >> 3) + j * PER_ROUND;
                off[j] = (uint32_t)(row < last ? row : last) * (uint32_t)(o.ld * 2) + (uint32_t)chunk * 16u;
            }
            start = o.p + (int64_t)row0 * o.ld;
            advance = PK;
            kk = chunk * 8;
        }
    }
    __device__ __forceinline__ void seek(int step, int pc) { base = start + (int64_t)pc * piece + step * advance; }

    // Round j of a step's loads.  lds: byte address of the tile
    __device__ __forceinline__ void load(int j, uint32_t lds, int wave, int step, bool more) const {
        typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
        const uint64_t at = (uint64_t)base;
        const u32x4 rsrc = {(uint32_t)at, (uint32_t)(at >> 32) & 0xffffu, 0x7fffffffu, 0x00020000u};
        const int left = (more ? k : -(1 << 30)) - step * PK - kk;
        const uint32_t o = left > (TR ? j * PER_ROUND : 0) ? off[j] : 0xfffffff0u;
        const uint32_t to = __builtin_amdgcn_readfirstlane(lds + (uint32_t)(j * T + wave * 64) * 16u);
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(o), "s"(rsrc), "s"(to) : "m0");
    }
};

// Reads a wavefront's fragments: 16 rows x 32 values of k; a lane has row lane % 16 and k = 8 (lane / 16) + 0..7.
template <int B, bool TR>
struct FragReader {
    static constexpr int CB = B / 8;
    int lane, row0;
    __device__ __forceinline__ void init(int row0_, int lane_) { lane = lane_; row0 = row0_; }
    __device__ __forceinline__ bf16x8 read(const uint16_t* lds, int t, int kk) const {
        const int g = lane >> 4, s = lane & 15;
        if constexpr (TR) {
            const int m = row0 + t * 16 + (s & 3) * 4, k0 = kk * 32 + g * 8 + (s >> 2);
            const uint16_t* p = lds + k0 * B + (((m >> 3) ^ turned<CB>(k0)) << 3) + (m & 4);
            typedef __attribute__((address_space(3))) short4v* lp;
            union { short4v h[2]; bf16x8 v; } u;
            // (4 rows of k on: the same position, since bit 2 does not go into it)
            u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)p);
            u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(p + 4 * B));
            return u.v;
        } else {
            const int c = (kk * 4 + g) ^ ((s >> 1) & 7);
            return *reinterpret_cast<const bf16x8*>(lds + (row0 + s) * PK + c * 8 + t * 16 * PK);
        }
    }
};

__host__ __device__ constexpr int product_lds(int bl, int br, int stages) { return stages * (bl + br) * PK * 2; }  // bytes

struct ProductPlace {
    int tl, tr, split;  // tile of l and of r, part of k
};
// Neighbouring tiles on one XCD: workgroups go to the XCDs in turn, so XCD x takes the x-th eighth of the tiles, in
// bands of 8 tiles of l, along r.  False: a workgroup without a tile.
__device__ __forceinline__ bool product_place(const ProductArgs& a, int block, ProductPlace& p) {
    const int total = a.tiles_l * a.tiles_r * a.splits, per = (total + 7) >> 3;
    const int id = (block & 7) * per + (block >> 3);
    if ((block >> 3) >= per || id >= total) return false;
    const int per_split = a.tiles_l * a.tiles_r, in = id % per_split;
    p.split = id / per_split;
    const int band = in / (8 * a.tiles_r), left = a.tiles_l - band * 8, height = left < 8 ? left : 8;
    const int inb = in - band * 8 * a.tiles_r;
    p.tl = band * 8 + inb % height;
    p.tr = inb / height;
    return true;
}

// WL x WR wavefronts, each with (BL / WL) x (BR / WR) values of C.  A step is 64 values of k, two halves of 32, and STAGES steps are in
// LDS or on their way.  Early in the second half of step t, whose operands are in registers by then, the wavefronts meet: everybody
// has step t + 1 and has left the place of step t, which t + STAGES takes.  So operands of t + 1 are read during that half, and
// the loads have STAGES - 1 steps to arrive.  Operands of r are read again into the registers of those just used.
// A lane has C[l][r] of l = lane % 16 and r = 4 (lane / 16) + 0..3 of each block of 16 x 16: what is summed or stored along r lies in
// few lanes.
template <int BL, int BR, int WL, int WR, int STAGES, bool F16, bool LT, bool RT>
__device__ __forceinline__ void product_sums(const ProductArgs& a, const ProductPlace& at, f32x4 (&acc)[BL / WL / 16][BR / WR / 16]) {
    constexpr int T = 64 * WL * WR, NL = BL / WL / 16, NR = BR / WR / 16, STAGE = (BL + BR) * PK;
    extern __shared__ __align__(1024) uint16_t product_tiles[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wl = wave % WL, wr = wave / WL, tl = at.tl, tr = at.tr, split = at.split;

#pragma unroll
    for (int i = 0; i < NL; ++i)
#pragma unroll
        for (int j = 0; j < NR; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][e] = 0.0f;

    TileLoader<BL, T, LT> ll;
    TileLoader<BR, T, RT> lr;
    ll.init(a.l, tl * BL, tid);
    lr.init(a.r, tr * BR, tid);
    FragReader<BL, LT> fl;
    FragReader<BR, RT> fr;
    fl.init(wl * (BL / WL), lane);
    fr.init(wr * (BR / WR), lane);

    const int all = a.steps * a.segs;
    const int t0 = (int)((int64_t)all * split / a.splits), t1 = (int)((int64_t)all * (split + 1) / a.splits);
    int seg = t0 / a.steps, step = t0 - seg * a.steps, next = t0;  // of the next load
    auto seek = [&]() {
        ll.seek(step, (a.pieces_l >> (4 * seg)) & 0xf);
        lr.seek(step, (a.pieces_r >> (4 * seg)) & 0xf);
    };
    seek();
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint16_t*)product_tiles;
    int into = 0;  // stage of the next load
    constexpr int LOADS_L = TileLoader<BL, T, LT>::ROUNDS, LOADS = LOADS_L + TileLoader<BR, T, RT>::ROUNDS;  // of a step
    // load i of step `next` (beyond the last step: zeros, so that the loads in flight are always as many)
    auto load = [&](int i) {
        const uint32_t to = lds + (uint32_t)into * (STAGE * 2);
        if (i < LOADS_L) ll.load(i, to, wave, step, next < t1);
        else lr.load(i - LOADS_L, to + BL * PK * 2, wave, step, next < t1);
    };
    auto loaded = [&]() {
        into = into + 1 == STAGES ? 0 : into + 1;
        ++next;
        ll.base += ll.advance;
        lr.base += lr.advance;
        if (++step == a.steps) {
            step = 0;
            if (++seg < a.segs) seek();
        }
    };
    bf16x8 x[2][NL], y[NR];
    auto read_l = [&](int i, int of, int kk) { x[kk][i] = fl.read(product_tiles + of * STAGE, i, kk); };
    auto read_r = [&](int j, int of, int kk) { y[j] = fr.read(product_tiles + of * STAGE + BL * PK, j, kk); };
    for (int s = 0; s < STAGES; ++s) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load(i);
        loaded();
    }
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((STAGES - 1) * LOADS) : "memory");
#pragma unroll
    for (int i = 0; i < NL; ++i) read_l(i, 0, 0);
#pragma unroll
    for (int j = 0; j < NR; ++j) read_r(j, 0, 0);
    int stage = 0;
    // The matrix instructions take 16 cycles each and everything else is issued between them: the order is kept.
    constexpr int MEET = NR >= 4 ? 2 : 1;                                // blocks of the second half in front of the meeting
    constexpr int LATER = LOADS / 2, NOW = LOADS - LATER;                // loads in the half after, in the second half
    constexpr int PER_NOW = (NOW + NR - MEET - 1) / (NR - MEET > 0 ? NR - MEET : 1), PER_LATER = (LATER + NR - 1) / NR;
    constexpr int PER_L = (NL + NR - 1) / NR, PER_L2 = (NL + (NR - MEET > 0 ? NR - MEET : 1) - 1) / (NR - MEET > 0 ? NR - MEET : 1);
    for (int t = t0; t < t1; ++t) {
        const bool loading = t > t0;  // (the rest of the loads of the step before)
#pragma unroll
        for (int j = 0; j < NR; ++j) {
#pragma unroll
            for (int i = 0; i < NL; ++i) acc[i][j] = matrix_product<F16>(y[j], x[0][i], acc[i][j]);
            read_r(j, stage, 1);
#pragma unroll
            for (int i = j * PER_L; i < (j + 1) * PER_L && i < NL; ++i) read_l(i, stage, 1);
            if (loading)
#pragma unroll
                for (int i = NOW + j * PER_LATER; i < NOW + (j + 1) * PER_LATER && i < LOADS; ++i) load(i);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (loading) loaded();
        const int after = stage + 1 == STAGES ? 0 : stage + 1;
#pragma unroll
        for (int j = 0; j < NR; ++j) {
            if (j == MEET) {
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((STAGES - 2) * LOADS) : "memory");
#pragma unroll
                for (int q = 0; q < MEET; ++q) read_r(q, after, 0);
            }
#pragma unroll
            for (int i = 0; i < NL; ++i) acc[i][j] = matrix_product<F16>(y[j], x[1][i], acc[i][j]);
            if (j >= MEET) {
                read_r(j, after, 0);
#pragma unroll
                for (int i = (j - MEET) * PER_L2; i < (j - MEET + 1) * PER_L2 && i < NL; ++i) read_l(i, after, 0);
#pragma unroll
                for (int i = (j - MEET) * PER_NOW; i < (j - MEET + 1) * PER_NOW && i < NOW; ++i) load(i);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        stage = after;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");  // nothing on its way to LDS, nobody reading
}

template <int BL, int BR, int WL, int WR, int STAGES, class Epilogue>
__device__ __forceinline__ void product_finish(const ProductPlace& at, const Epilogue& epi, f32x4 (&acc)[BL / WL / 16][BR / WR / 16]) {
    constexpr int NL = BL / WL / 16, NR = BR / WR / 16, STAGE = (BL + BR) * PK;
    extern __shared__ __align__(1024) uint16_t product_tiles[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wl = wave % WL, wr = wave / WL;
    // (LDS in which an epilogue turns its values: a wavefront's own part)
    static_assert(!Epilogue::TURNS || NL * 16 * NR * 16 * WL * WR <= STAGES * STAGE, "the wavefronts' values fit");
    uint16_t* const own = product_tiles + wave * (NL * 16 * NR * 16);
    epi.template finish<NL, NR>(acc, at.tl * BL + wl * (BL / WL), at.tr * BR + wr * (BR / WR), at.tr * WR + wr, at.split, lane, own);
}

template <int BL, int BR, int WL, int WR, int STAGES, bool LT, bool RT, class Epilogue>
__device__ __forceinline__ void product(const ProductArgs& a, const Epilogue& epi, int block) {
    ProductPlace at;
    if (!product_place(a, block, at)) return;
    f32x4 acc[BL / WL / 16][BR / WR / 16];
    product_sums<BL, BR, WL, WR, STAGES, false, LT, RT>(a, at, acc);
    product_finish<BL, BR, WL, WR, STAGES>(at, epi, acc);
}

template <int BL, int BR, int WL, int WR, int STAGES, bool LT, bool RT, class Epilogue>
__global__ __launch_bounds__(64 * WL * WR) void product_kernel(ProductArgs a, Epilogue epi) {
    product<BL, BR, WL, WR, STAGES, LT, RT>(a, epi, blockIdx.x);
}

// Scores of fp32 rows, in the pieces that the rows ask for: of the same tiles, two fp16 ones (a16) or three bfloat16 ones (a3).
template <int BL, int BR, int WL, int WR, int STAGES, class Epilogue>
__global__ __launch_bounds__(64 * WL * WR) void score_kernel(ProductArgs a16, ProductArgs a3, const uint32_t* __restrict__ range, Epilogue epi) {
    ProductPlace at;
    if (!product_place(a16, blockIdx.x, at)) return;
    f32x4 acc[BL / WL / 16][BR / WR / 16];
    if (in_three_pieces(*range)) {
        epi.back_l = epi.back_r = nullptr;
        product_sums<BL, BR, WL, WR, STAGES, false, false, false>(a3, at, acc);
    } else {
        product_sums<BL, BR, WL, WR, STAGES, true, false, false>(a16, at, acc);
    }
    product_finish<BL, BR, WL, WR, STAGES>(at, epi, acc);
}

// Two products that do not depend on each other, in one launch: the first `blocks` workgroups (a multiple of 8) have one.
template <int BL, int BR, int WL, int WR, int STAGES, bool LT1, bool RT1, bool LT2, bool RT2, class Epilogue>
__global__ __launch_bounds__(64 * WL * WR) void product_pair_kernel(ProductArgs a1, Epilogue epi1, ProductArgs a2, Epilogue epi2, int blocks) {
    if ((int)blockIdx.x < blocks) product<BL, BR, WL, WR, STAGES, LT1, RT1>(a1, epi1, blockIdx.x);
    else product<BL, BR, WL, WR, STAGES, LT2, RT2>(a2, epi2, blockIdx.x - blocks);
}

}  // namespace qgbdt
