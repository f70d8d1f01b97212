// Rows of a token table by token, scaled and added up over a bag of tokens, and the table's gradient.
//   out_i = scale * sum_b T[tok_ib],   dT[v] = scale * sum over (i, b) with tok_ib = v of g_i
// Both are bound by memory.  Tokens outside 0 .. n_vocab - 1 are padding: they add nothing and get no gradient.
#include "head.h"

namespace qgbdt {

template <class I>
__device__ __forceinline__ int64_t token_at(const void* t, int64_t i) { return (int64_t)static_cast<const I*>(t)[i]; }

// Lanes that share a row: a power of two of which the row's 16-byte pieces leave the fewest idle (155 pieces: 5 times 32 lanes, not 256),
// the most of those; more where `rows` rows at work together would not fill the chip, since a lane takes its pieces one after the other (35
// bags of 26 rows of 656 bf16 values: 8 lanes 59 us, 128 lanes 8 us).
static int lanes_of_row(int dim, int per16, int64_t rows) {
    const int pieces = (dim + per16 - 1) / per16;
    int best = 1;
    for (int l = 2; l <= 256 && l < 2 * pieces; l <<= 1)
        if ((pieces + l - 1) / l * l <= (pieces + best - 1) / best * best + pieces / 16) best = l;
    while (best < pieces && best < 256 && rows * best < 131072) best <<= 1;
    return best;
}

// A row's values are taken in pieces of 16 bytes, wherever they begin; the last piece of a row whose length is no multiple
// of that overlaps the one before (its values are the same).  TINY: rows shorter than a piece.
template <class E, bool TINY>
__device__ __forceinline__ int piece_at(int c, int dim) { return TINY ? 0 : c + E::PER16 <= dim ? c : dim - E::PER16; }
template <class E, bool TINY>
__device__ __forceinline__ void get_piece(const typename E::T* p, int dim, float* v) {
    if constexpr (TINY) load_part<E>(p, dim, v);
    else load_piece<E>(p, v);
}
template <class E, bool TINY>
__device__ __forceinline__ void put_piece(typename E::T* p, int dim, const float* v) {
    if constexpr (TINY) store_part<E>(p, dim, v);
    else store_piece<E>(p, v);
}

// A group of `lanes` threads per row; BAG rows of a bag are requested at a time (1: a plain lookup, then two rows are in flight).  Bound by
// memory (16,384 x 2048 bf16: 16.5 us, 5.8 TB/s), with short rows by the requests to the caches (5.2 M rows of 256 bytes: 102 us, 13 TB/s of which
// 5.5 come from memory).
//
// LONG: bags of more than 64 rows, whose sums would lose more with every row (65,536 equal values: up to 14,000 units of 2^-24), keep what the
// additions lose.  In shorter ones that would cost registers and, where rows come from the caches, time (5000 bags of 26 x 512 fp16: 16.1 us, with it 17.8).
template <class E, class I, bool TINY, int BAG, bool LONG>
__global__ __launch_bounds__(256) void embed_kernel(const typename E::T* __restrict__ table, int64_t n_vocab, int dim, int64_t stride,
                                                    const void* __restrict__ tokens, int64_t n, int bag, float scale,
                                                    typename E::T* __restrict__ out, int lanes) {
    constexpr int P = E::PER16, ROWS = BAG == 1 ? 2 : 1;
    const int sub = threadIdx.x & (lanes - 1), per = 256 / lanes;
    const int64_t groups = (int64_t)gridDim.x * per;
    for (int64_t i = (int64_t)blockIdx.x * per + threadIdx.x / lanes; i < n; i += groups * ROWS)
        for (int c = sub * P; c < dim; c += lanes * P) {
            const int at = piece_at<E, TINY>(c, dim);
            LongSum sum[ROWS][P];
            for (int b = 0; b < bag; b += BAG) {
                // (no token, padding: row 0 is read and not used)
                bool on[ROWS * BAG];
                float v[ROWS * BAG][P];
#pragma unroll
                for (int q = 0; q < ROWS * BAG; ++q) {
                    const int64_t row = i + (ROWS > 1 ? q * groups : 0);
                    const int place = ROWS > 1 ? 0 : b + q;
                    const bool there = place < bag && row < n;
                    const int64_t t = there ? token_at<I>(tokens, row * bag + place) : -1;
                    on[q] = t >= 0 && t < n_vocab;
                    get_piece<E, TINY>(table + (on[q] ? t : 0) * stride + at, dim, v[q]);
                }
                float part[ROWS][P];
#pragma unroll
                for (int r = 0; r < ROWS; ++r)
#pragma unroll
                    for (int k = 0; k < P; ++k) part[r][k] = LONG ? 0.0f : sum[r][k].sum;
#pragma unroll
                for (int q = 0; q < ROWS * BAG; ++q)
#pragma unroll
                    for (int k = 0; k < P; ++k) part[ROWS > 1 ? q : 0][k] += on[q] ? v[q][k] : 0.0f;
#pragma unroll
                for (int r = 0; r < ROWS; ++r)
#pragma unroll
                    for (int k = 0; k < P; ++k) {
                        if constexpr (LONG) sum[r][k].add(part[r][k]);
                        else sum[r][k].sum = part[r][k];
                    }
            }
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                float o[P];
#pragma unroll
                for (int k = 0; k < P; ++k) o[k] = (LONG ? sum[r][k].value() : sum[r][k].sum) * scale;
                if (r == 0 || i + r * groups < n) put_piece<E, TINY>(out + (i + r * groups) * dim + at, dim, o);
            }
        }
}

// ---- the gradient -----------------------------------------------------------------------------------
// The entries (i, b) are sorted by token, ties by position, so that every sum has a fixed order.  A stable radix sort, least digit
// first, of one or two digits of up to 10 bits (three beyond 2^20 tokens, four beyond 2^30): a count per workgroup's tile and digit, sums over the tiles, and
// the move.  An entry is its token and its position; padding has the token n_vocab and comes last.

constexpr int DIGIT_BITS = 10, DIGITS = 1 << DIGIT_BITS;
constexpr int SORT_THREADS = 256;
constexpr int SORT_PER = 16, SORT_PER_FEW = 4;  // entries per thread; where they are few, more workgroups
constexpr int SCAN_TILES = 64;                  // up to so many tiles every workgroup of the move adds up the counts itself

// what the first digit's kernels read (tokens), and the later ones (entries)
template <class I>
struct FromTokens {
    const void* tokens;
    int64_t n_vocab;
    __device__ __forceinline__ uint2 get(int64_t i) const {
        const int64_t t = token_at<I>(tokens, i);
        return make_uint2((uint32_t)(t >= 0 && t < n_vocab ? t : n_vocab), (uint32_t)i);
    }
};
struct FromEntries {
    const uint2* entry;
    __device__ __forceinline__ uint2 get(int64_t i) const { return entry[i]; }
};

// The sort by token: a stable radix sort, ten bits at a time, of (token, entry).  Bound by latency in small sorts and by the moves' scattered
// stores in large ones (2.6 M entries of two digits: counts 10 and 14 us, scans 5 each, moves 28 and 22).
// counts: [digit][tile].  Workgroups behind the tiles clear the tokens' ranges.
template <class From, int PER>
__global__ __launch_bounds__(SORT_THREADS) void sort_count_kernel(From from, int64_t m, int shift, int digits, int tiles, int32_t* __restrict__ counts,
                                                                  int2* __restrict__ range, int64_t n_range) {
    __shared__ int32_t bins[SORT_THREADS / 64][DIGITS];  // (one per wavefront: not all of them add to a frequent token's count)
    if ((int)blockIdx.x >= tiles) {
        const int64_t step = (int64_t)(gridDim.x - tiles) * SORT_THREADS;
        for (int64_t i = (int64_t)(blockIdx.x - tiles) * SORT_THREADS + threadIdx.x; i < n_range; i += step) range[i] = make_int2(0, 0);
        return;
    }
    for (int d = threadIdx.x; d < digits; d += SORT_THREADS)
#pragma unroll
        for (int w = 0; w < SORT_THREADS / 64; ++w) bins[w][d] = 0;
    __syncthreads();
    const int64_t base = (int64_t)blockIdx.x * (SORT_THREADS * PER);
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int64_t i = base + j * SORT_THREADS + threadIdx.x;
        if (i < m) atomicAdd(&bins[threadIdx.x >> 6][(from.get(i).x >> shift) & (digits - 1)], 1);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += SORT_THREADS) counts[(int64_t)d * tiles + blockIdx.x] = bins[0][d] + bins[1][d] + bins[2][d] + bins[3][d];
}

// A workgroup per digit: exclusive sums over the tiles, and the digit's total.
__global__ __launch_bounds__(256) void sort_scan_kernel(int32_t* __restrict__ counts, int tiles, int32_t* __restrict__ totals) {
    __shared__ int32_t part[4];
    int32_t* const row = counts + (int64_t)blockIdx.x * tiles;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t carry = 0;
    for (int at = 0; at < tiles; at += 256) {
        const int i = at + threadIdx.x;
        const int32_t v = i < tiles ? row[i] : 0;
        int32_t s = v;
        for (int o = 1; o < 64; o <<= 1) { const int32_t b = __shfl_up(s, o); if (lane >= o) s += b; }
        __syncthreads();
        if (lane == 63) part[wave] = s;
        __syncthreads();
        int32_t before = carry;
        for (int w = 0; w < wave; ++w) before += part[w];
        if (i < tiles) row[i] = before + s - v;
        carry += part[0] + part[1] + part[2] + part[3];
    }
    if (threadIdx.x == 0) totals[blockIdx.x] = carry;
}

// Each wavefront has a consecutive stretch of the tile; equal digits of 64 entries are ranked by ballots.  totals null: the counts are
// as they were counted (few tiles).
template <class From, int PER>
__global__ __launch_bounds__(SORT_THREADS) void sort_move_kernel(From from, int64_t m, int shift, int bits, int tiles, const int32_t* __restrict__ counts,
                                                                 const int32_t* __restrict__ totals, uint2* __restrict__ out) {
    constexpr int WAVES = SORT_THREADS / 64, MOST = DIGITS / SORT_THREADS;
    __shared__ int32_t wave_bins[WAVES][DIGITS];
    __shared__ int32_t first[DIGITS];
    __shared__ int32_t part[WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int digits = 1 << bits, each = digits > SORT_THREADS ? digits / SORT_THREADS : 1;  // consecutive digits of a thread
    // the entries, requested first
    const int64_t base = (int64_t)blockIdx.x * (SORT_THREADS * PER) + wave * (64 * PER);
    uint2 k[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int64_t i = base + j * 64 + lane;
        k[j] = i < m ? from.get(i) : make_uint2(0, 0);
    }
    // where each digit begins: totals of the lower ones, and of this digit in the tiles before
    {
        int32_t mine[MOST], sum = 0;
#pragma unroll
        for (int q = 0; q < MOST; ++q) {
            mine[q] = 0;
            const int d = threadIdx.x * each + q;
            if (q >= each || d >= digits) continue;
            const int32_t* const c = counts + (int64_t)d * tiles;
            int32_t before, total;
            if (totals) {
                before = c[blockIdx.x];
                total = totals[d];
            } else {
                before = total = 0;
#pragma unroll 8
                for (int t = 0; t < tiles; ++t) {
                    const int32_t v = c[t];
                    before += t < (int)blockIdx.x ? v : 0;
                    total += v;
                }
            }
            first[d] = sum + before;
            mine[q] = total;
            sum += total;
        }
        int32_t s = sum;
        for (int o = 1; o < 64; o <<= 1) { const int32_t b = __shfl_up(s, o); if (lane >= o) s += b; }
        if (lane == 63) part[wave] = s;
        for (int w = 0; w < WAVES; ++w)
            for (int d = threadIdx.x; d < digits; d += SORT_THREADS) wave_bins[w][d] = 0;
        __syncthreads();
        s -= sum;
        for (int w = 0; w < wave; ++w) s += part[w];
#pragma unroll
        for (int q = 0; q < MOST; ++q) {
            const int d = threadIdx.x * each + q;
            if (q < each && d < digits) first[d] += s;
        }
    }
    int32_t rank[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const bool on = base + j * 64 + lane < m;
        const uint32_t d = (k[j].x >> shift) & (digits - 1);
        unsigned long long same = __ballot(on);
        for (int b = 0; b < bits; ++b) {
            const unsigned long long set = __ballot((d >> b) & 1);
            same &= (d >> b) & 1 ? set : ~set;
        }
        const int before = __popcll(same & ((1ull << lane) - 1));
        rank[j] = on ? wave_bins[wave][d] + before : 0;
        wavefront_sync();
        if (on && before == 0) wave_bins[wave][d] += __popcll(same);
        wavefront_sync();
    }
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += SORT_THREADS) {
        int32_t s = first[d];
        for (int w = 0; w < WAVES; ++w) { const int32_t c = wave_bins[w][d]; wave_bins[w][d] = s; s += c; }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < PER; ++j)
        if (base + j * 64 + lane < m) out[wave_bins[wave][(k[j].x >> shift) & (digits - 1)] + rank[j]] = k[j];
}

// first and last + 1 of each token's entries
__global__ __launch_bounds__(256) void ranges_kernel(const uint2* __restrict__ entry, int64_t m, int64_t n_vocab, int2* __restrict__ range) {
    const int64_t step = (int64_t)gridDim.x * blockDim.x;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < m; i += step) {
        const uint32_t k = entry[i].x;
        if (k >= n_vocab) continue;
        if (i == 0 || entry[i - 1].x != k) range[k].x = (int)i;
        if (i == m - 1 || entry[i + 1].x != k) range[k].y = (int)i + 1;
    }
}

__global__ __launch_bounds__(256) void clear_ranges_kernel(int2* range, int64_t n) {
    const int64_t step = (int64_t)gridDim.x * blockDim.x;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += step) range[i] = make_int2(0, 0);
}

// Few entries, in one launch: an entry's place is the number of entries with a smaller token, or with the same one and in front of it.  A
// workgroup has all tokens in LDS and places 32 entries, by 8 threads each that look at every eighth four tokens (371 bags of 5: 42 ->
// 25 us for the whole gradient, whose launches are 4 instead of 7).
constexpr int SORT_FEW = 4096, SORT_FEW_ENTRIES = 32;
template <class I>
__global__ __launch_bounds__(256) void sort_few_kernel(FromTokens<I> from, int m, int64_t n_vocab, uint2* __restrict__ out, int2* __restrict__ range) {
    __shared__ __align__(16) uint32_t key[SORT_FEW];
    const int whole = (m + 31) / 32 * 32;
    for (int i = threadIdx.x; i < whole; i += 256) key[i] = i < m ? from.get(i).x : 0xffffffffu;  // (behind all, padding's n_vocab among them)
    __syncthreads();
    const int i = blockIdx.x * SORT_FEW_ENTRIES + (threadIdx.x >> 3), part = threadIdx.x & 7;
    const uint32_t k = i < m ? key[i] : 0u;
    int less = 0, before = 0, same = 0;
    for (int j = part * 4; j < whole; j += 32) {
        const uint4 q = *reinterpret_cast<const uint4*>(key + j);
        const uint32_t v[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            less += v[e] < k ? 1 : 0;
            same += v[e] == k ? 1 : 0;
            before += v[e] == k && j + e < i ? 1 : 0;
        }
    }
    for (int o = 4; o > 0; o >>= 1) {
        less += __shfl_xor(less, o);
        same += __shfl_xor(same, o);
        before += __shfl_xor(before, o);
    }
    if (part == 0 && i < m) {
        out[less + before] = make_uint2(k, (uint32_t)i);
        if (before == 0 && k < n_vocab) range[k] = make_int2(less, less + same);
    }
}

// adds the gradient rows of entries a .. b - 1, in order
template <class E, bool TINY>
__device__ __forceinline__ void add_rows(const typename E::T* __restrict__ grad, const uint2* __restrict__ entry, int bag, int dim, int at, int a, int b, float* sum) {
    constexpr int P = E::PER16, U = 8;
    for (uint32_t i = a, end = b; i < end; i += U) {  // (unsigned: b may be 2^31 - 1)
        uint32_t r[U];
#pragma unroll
        for (int q = 0; q < U; ++q) r[q] = entry[i + q < end ? i + q : end - 1].y;
        Piece<E> v[U];
#pragma unroll
        for (int q = 0; q < U; ++q) {
            const typename E::T* const p = grad + (int64_t)(bag == 1 ? r[q] : r[q] / (uint32_t)bag) * dim + at;
            if constexpr (TINY) {
#pragma unroll
                for (int k = 0; k < P; ++k) v[q].v[k] = k < dim ? p[k] : E::put(0.0f);
            } else {
                __builtin_memcpy(&v[q], p, 16);
            }
        }
        // (eight at a time, as a tree: equal values, whose roundings go one way, lose little)
#pragma unroll
        for (int k = 0; k < P; ++k) {
            float t[U];
#pragma unroll
            for (int q = 0; q < U; ++q) t[q] = i + q < end ? E::get(v[q].v[k]) : 0.0f;
            sum[k] += ((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7]));
            __builtin_amdgcn_sched_barrier(0);  // (the others stay as they came: 77 registers instead of 106)
        }
    }
}

// scale times the sum to the row's piece at c, or added to what is there
template <class E, bool TINY>
__device__ __forceinline__ void put_row(typename E::T* row, int c, int dim, const float* sum, float scale, int accumulate) {
    constexpr int P = E::PER16;
    const int at = piece_at<E, TINY>(c, dim);
    float v[P];
    if (accumulate) {  // (values that overlap the piece before are that piece's)
        for (int q = c - at; q < P && at + q < dim; ++q) row[at + q] = E::put(E::get(row[at + q]) + sum[q] * scale);
        return;
    }
#pragma unroll
    for (int q = 0; q < P; ++q) v[q] = sum[q] * scale;
    put_piece<E, TINY>(row + at, dim, v);
}

// What has no part in anything else, in one launch.  `lanes` threads work together on a row of the gradient or the table.
//  * Units of unit consecutive entries: what they have of tokens of more entries than that goes to `part`.  A unit meets at most
//    two such tokens; slot 0: the one of its first entry, slot 1: another.
//  * Rows of the table that no token names: zeros.  Every workgroup of the next kind writes a share of them first, so that its stores
//    go on while it waits for its tokens.
//  * Tokens of up to unit entries: added up by the group that has the first one, `each` consecutive entries per group.
// Bound by the zeros where the table is large (131,072 x 2048 bf16: 110 us of stores, 4.9 TB/s) and by requests to the caches where rows are short
// (2.6 M rows of 256 bytes: 161 us, 4.2 TB/s: a group waits for an entry, its token's range, the token's entries and then two rows).
template <class E, bool TINY>
__global__ __launch_bounds__(256) void embed_sums_kernel(const typename E::T* __restrict__ grad, const uint2* __restrict__ entry, const int2* __restrict__ range,
                                                         int64_t m, int64_t n_vocab, int bag, int dim, int lanes, int unit, int unit_blocks, int each,
                                                         float* __restrict__ part, float scale, typename E::T* __restrict__ out, int accumulate) {
    constexpr int P = E::PER16;
    const int sub = threadIdx.x & (lanes - 1), per = 256 / lanes, group = threadIdx.x / lanes;
    const int pd = (dim + 7) / 8 * 8;
    if ((int)blockIdx.x < unit_blocks) {
        for (int64_t u = (int64_t)blockIdx.x * per + group; u * unit < m; u += (int64_t)unit_blocks * per) {
            const int64_t a0 = u * unit;
            const int a = (int)a0, b = (int)(a0 + unit < m ? a0 + unit : m);
            const uint32_t k0 = entry[a].x, k1 = entry[b - 1].x;
            for (int slot = 0; slot < 2; ++slot) {
                const uint32_t k = slot ? k1 : k0;
                if (k >= n_vocab || (slot && k1 == k0)) continue;
                const int2 r = range[k];
                if (r.y - r.x <= unit) continue;
                const int from = r.x > a ? r.x : a, to = r.y < b ? r.y : b;
                for (int c = sub * P; c < dim; c += lanes * P) {
                    const int at = piece_at<E, TINY>(c, dim);
                    float sum[P];
#pragma unroll
                    for (int q = 0; q < P; ++q) sum[q] = 0.0f;
                    add_rows<E, TINY>(grad, entry, bag, dim, at, from, to, sum);
                    float* const o = part + (u * 2 + slot) * pd + at;
#pragma unroll
                    for (int q = 0; q < P; q += 4) store_piece<F32>(o + q, sum + q);  // (pd holds a whole piece of a tiny row)
                }
            }
        }
        return;
    }
    const int64_t blocks = (int64_t)gridDim.x - unit_blocks, block = (int64_t)blockIdx.x - unit_blocks, groups = blocks * per;
    const int64_t first = (block * per + group) * each, end = first + each < m ? first + each : m;
    // (requested before the zeros)
    uint32_t next = first < end ? entry[first].x : 0u, last = first < end && first > 0 ? entry[first - 1].x : 0xffffffffu;
    if (!accumulate) {
        const float zero[P] = {};
        for (int64_t v = (block * per + group) * 4; v < n_vocab; v += 4 * groups) {
            int used[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) used[q] = v + q < n_vocab ? range[v + q].y : 1;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (!used[q])
                    for (int c = sub * P; c < dim; c += lanes * P)
                        put_piece<E, TINY>(out + (v + q) * dim + piece_at<E, TINY>(c, dim), dim, zero);
        }
    }
    for (int64_t i = first; i < end; ++i) {
        const uint32_t k = next;
        if (i + 1 < end) next = entry[i + 1].x;
        if (k >= n_vocab) break;  // padding: the rest
        if (k == last) continue;  // (not the token's first entry: its range is not looked up)
        last = k;
        const int2 r = range[k];
        if (r.y - r.x > unit) continue;
        if (r.y - r.x <= 2) {  // most tokens: both rows' pieces of all columns are requested as they come
            const uint32_t p0 = entry[i].y, p1 = entry[r.y - 1].y;
            const typename E::T* const g0 = grad + (int64_t)(bag == 1 ? p0 : p0 / (uint32_t)bag) * dim;
            const typename E::T* const g1 = grad + (int64_t)(bag == 1 ? p1 : p1 / (uint32_t)bag) * dim;
            const float second = r.y - r.x > 1 ? 1.0f : 0.0f;
#pragma unroll 4
            for (int c = sub * P; c < dim; c += lanes * P) {
                const int at = piece_at<E, TINY>(c, dim);
                float a[P], b[P];
                get_piece<E, TINY>(g0 + at, dim, a);
                get_piece<E, TINY>(g1 + at, dim, b);
#pragma unroll
                for (int q = 0; q < P; ++q) a[q] += second != 0.0f ? b[q] : 0.0f;
                put_row<E, TINY>(out + (int64_t)k * dim, c, dim, a, scale, accumulate);
            }
            continue;
        }
        for (int c = sub * P; c < dim; c += lanes * P) {
            float sum[P];
#pragma unroll
            for (int q = 0; q < P; ++q) sum[q] = 0.0f;
            add_rows<E, TINY>(grad, entry, bag, dim, piece_at<E, TINY>(c, dim), r.x, r.y, sum);
            put_row<E, TINY>(out + (int64_t)k * dim, c, dim, sum, scale, accumulate);
        }
    }
}

// Tokens of more than unit entries: such a token's entries go beyond the unit in which they begin, so a unit begins at most one.  A
// workgroup looks at `each` units; its groups of lanes take the parts in turn and are added up in their order.
constexpr int MERGE_THREADS = 256;  // (2.6 M entries, the most frequent token's 3750 parts: 30 us; with 1024: 109)
template <class E, bool TINY>
__global__ __launch_bounds__(MERGE_THREADS) void embed_merge_kernel(const uint2* __restrict__ entry, const int2* __restrict__ range, int64_t m, int64_t n_vocab, int unit, int64_t units, int each, int dim,
                                                          int lanes, const float* __restrict__ part, float scale, typename E::T* __restrict__ out, int accumulate) {
    constexpr int P = E::PER16;
    __shared__ float sums[MERGE_THREADS][P + 1];
    const int sub = threadIdx.x & (lanes - 1), per = MERGE_THREADS / lanes, group = threadIdx.x / lanes;
    const int pd = (dim + 7) / 8 * 8;
    const int64_t u0 = (int64_t)blockIdx.x * each;
    for (int64_t u = u0; u < u0 + each && u < units; ++u) {
        const int64_t a = u * unit, b = a + unit < m ? a + unit : m;
        const uint32_t k = entry[b - 1].x;
        if (k >= n_vocab) continue;
        const int2 r = range[k];
        if (r.x < a || r.y - r.x <= unit) continue;
        const int64_t last = (r.y - 1) / unit;
        for (int c0 = 0; c0 < dim; c0 += lanes * P) {
            const int c = c0 + sub * P;
            LongSum parts[P];  // (a token of all of 2^31 entries has 33 million parts)
            if (c < dim)
                for (int64_t w0 = u + group; w0 <= last; w0 += 4 * per) {
                    float v[4][P];
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        const int64_t w = w0 + h * per;
#pragma unroll
                        for (int q = 0; q < P; ++q) v[h][q] = 0.0f;
                        if (w > last) continue;
                        const float* const p = part + (w * 2 + (w == u && r.x > a ? 1 : 0)) * pd + piece_at<E, TINY>(c, dim);
#pragma unroll
                        for (int q = 0; q < P; q += 4) load_piece<F32>(p + q, v[h] + q);
                    }
#pragma unroll
                    for (int q = 0; q < P; ++q) parts[q].add((v[0][q] + v[1][q]) + (v[2][q] + v[3][q]));
                }
            float sum[P];
#pragma unroll
            for (int q = 0; q < P; ++q) sum[q] = parts[q].value();
            for (int half = per >> 1; half > 0; half >>= 1) {  // the groups' sums, as a tree
                __syncthreads();
#pragma unroll
                for (int q = 0; q < P; ++q) sums[threadIdx.x][q] = sum[q];
                __syncthreads();
                if (group < half)
#pragma unroll
                    for (int q = 0; q < P; ++q) sum[q] += sums[threadIdx.x + half * lanes][q];
            }
            if (group == 0 && c < dim) put_row<E, TINY>(out + (int64_t)k * dim, c, dim, sum, scale, accumulate);
        }
    }
}

// ---- host -----------------------------------------------------------------------------------------

struct EmbedPlan {
    int64_t m, tiles, units;
    int passes, bits, unit;
    bool few, sorted;
    size_t entry[2], counts, totals, range, part, bytes;
};

static EmbedPlan make_embed_plan(int64_t n, int bag, int64_t n_vocab, int dim, int dtype) {
    EmbedPlan p = {};
    p.m = n * bag;
    p.few = p.m <= 256 * 1024;  // (65 k entries: 16 tiles of 4096 leave most of the chip idle)
    const int tile = SORT_THREADS * (p.few ? SORT_PER_FEW : SORT_PER);
    p.tiles = (p.m + tile - 1) / tile;
    p.sorted = p.m <= SORT_FEW;
    // Entries that are added up in one go: 64; 16 where that would leave too few at work (28,369 rows of 440 bf16 values, the whole
    // gradient: 167 -> 41 us; 16,384 of 2048 values: 166 us with 64, 172 with 16, whose parts take longer to join).
    const int64_t pieces = (dim * (int64_t)dtype_bytes(dtype) + 15) / 16;
    p.unit = p.m > 64 && p.m / 64 * (pieces < 256 ? pieces : 256) < 49152 ? 16 : 64;
    int bits = 1;
    while (bits < 32 && (n_vocab >> bits) > 0) ++bits;  // keys 0 .. n_vocab
    p.passes = (bits + DIGIT_BITS - 1) / DIGIT_BITS;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.units = (p.m + p.unit - 1) / p.unit;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align256(bytes); return o; };
    for (int k = 0; k < 2; ++k) p.entry[k] = take((size_t)p.m * 8);
    p.counts = take(((size_t)p.tiles << p.bits) * 4);
    p.totals = take(DIGITS * 4);
    p.range = take((size_t)n_vocab * 8);
    p.part = take(p.m > p.unit ? (size_t)p.units * 2 * ((dim + 7) / 8 * 8) * 4 : 0);
    p.bytes = at;
    return p;
}

size_t embed_gradient_bytes(int64_t n, int bag, int64_t n_vocab, int dim, int dtype) { return make_embed_plan(n, bag, n_vocab, dim, dtype).bytes; }

static int blocks_for(int64_t items, int per, int most) {
    const int64_t b = (items + per - 1) / per;
    return (int)(b < 1 ? 1 : b > most ? most : b);
}

template <class E, class I>
static void embed_tokens(qgbdt_ctx* ctx, const void* table, int64_t n_vocab, int dim, int64_t stride, const void* tokens, int64_t n, int bag, float scale, void* out) {
    const int lanes = lanes_of_row(dim, E::PER16, n);
    const dim3 grid(blocks_for(n, 256 / lanes * (bag == 1 ? 2 : 1), 1 << 20)), threads(256);
    const typename E::T* const t = static_cast<const typename E::T*>(table);
    typename E::T* const o = static_cast<typename E::T*>(out);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, threads, 0, ctx->stream, t, n_vocab, dim, stride, tokens, n, bag, scale, o, lanes); };
    const bool longer = bag > 64;
    if (dim < E::PER16) longer ? go(embed_kernel<E, I, true, 4, true>) : go(embed_kernel<E, I, true, 4, false>);
    else if (bag == 1) go(embed_kernel<E, I, false, 1, false>);
    else longer ? go(embed_kernel<E, I, false, 8, true>) : go(embed_kernel<E, I, false, 8, false>);
}

int run_embed_tokens(qgbdt_ctx* ctx, const void* table, int dtype, int64_t n_vocab, int dim, int64_t table_stride, const void* tokens, int token_bytes, int64_t n,
                     int bag, float scale, void* out) {
    if (n == 0) return QGBDT_OK;
    auto go = [&](auto e) {
        typedef decltype(e) E;
        if (token_bytes == 8) embed_tokens<E, int64_t>(ctx, table, n_vocab, dim, table_stride, tokens, n, bag, scale, out);
        else embed_tokens<E, int32_t>(ctx, table, n_vocab, dim, table_stride, tokens, n, bag, scale, out);
    };
    if (dtype == QGBDT_F32) go(F32());
    else if (dtype == QGBDT_BF16) go(BF16());
    else go(F16());
    QG_HIP(ctx, hipGetLastError());
    return QGBDT_OK;
}

template <class From>
static void sort_pass(qgbdt_ctx* ctx, const EmbedPlan& p, From from, int pass, int32_t* counts, int32_t* totals, uint2* out, int2* range, int64_t n_vocab) {
    const int shift = pass * p.bits, clear = pass == 0 ? blocks_for(n_vocab, 1024, 1024) : 0;
    const dim3 count_grid((unsigned)(p.tiles + clear)), move_grid((unsigned)p.tiles), threads(SORT_THREADS);
    const bool scan = p.tiles > SCAN_TILES;
    if (p.few) hipLaunchKernelGGL((sort_count_kernel<From, SORT_PER_FEW>), count_grid, threads, 0, ctx->stream, from, p.m, shift, 1 << p.bits, (int)p.tiles, counts, range, n_vocab);
    else hipLaunchKernelGGL((sort_count_kernel<From, SORT_PER>), count_grid, threads, 0, ctx->stream, from, p.m, shift, 1 << p.bits, (int)p.tiles, counts, range, n_vocab);
    if (scan) hipLaunchKernelGGL(sort_scan_kernel, dim3(1 << p.bits), dim3(256), 0, ctx->stream, counts, (int)p.tiles, totals);
    if (p.few) hipLaunchKernelGGL((sort_move_kernel<From, SORT_PER_FEW>), move_grid, threads, 0, ctx->stream, from, p.m, shift, p.bits, (int)p.tiles, counts, scan ? totals : nullptr, out);
    else hipLaunchKernelGGL((sort_move_kernel<From, SORT_PER>), move_grid, threads, 0, ctx->stream, from, p.m, shift, p.bits, (int)p.tiles, counts, scan ? totals : nullptr, out);
}

template <class E>
static void embed_sums(qgbdt_ctx* ctx, const EmbedPlan& p, const uint2* entry, const int2* range, float* part, int bag, const void* grad, int64_t n_vocab, int dim,
                       float scale, void* grad_table, int accumulate) {
    typedef typename E::T T;
    const int lanes = lanes_of_row(dim, E::PER16, p.units), per = 256 / lanes;
    const bool many = p.m > p.unit;
    // (at most 2^22 workgroups of either kind, so that a launch has fewer than 2^32 threads)
    const int unit_blocks = many ? blocks_for(p.units, per, 1 << 22) : 0;
    int each = 1;
    while ((each < 16 && p.m / per / each > 16384) || p.m / per / each >= 1 << 22) each *= 2;
    const int64_t span = (int64_t)per * each, token_blocks = (p.m + span - 1) / span;
    const int zero_blocks = accumulate ? 0 : blocks_for(n_vocab, per * 4, 4096);
    const int blocks = token_blocks > zero_blocks ? (int)token_blocks : zero_blocks;
    if (blocks == 0) return;
    const int merge = p.units > 8192 ? 8 : 1;
    const dim3 sums((unsigned)(unit_blocks + blocks)), merges((unsigned)((p.units + merge - 1) / merge)), threads(256);
    const T* const g = static_cast<const T*>(grad);
    T* const out = static_cast<T*>(grad_table);
    if (dim < E::PER16) {
        hipLaunchKernelGGL((embed_sums_kernel<E, true>), sums, threads, 0, ctx->stream, g, entry, range, p.m, n_vocab, bag, dim, lanes, p.unit, unit_blocks, each, part, scale, out, accumulate);
        if (many) hipLaunchKernelGGL((embed_merge_kernel<E, true>), merges, dim3(MERGE_THREADS), 0, ctx->stream, entry, range, p.m, n_vocab, p.unit, p.units, merge, dim, lanes, part, scale, out, accumulate);
    } else {
        hipLaunchKernelGGL((embed_sums_kernel<E, false>), sums, threads, 0, ctx->stream, g, entry, range, p.m, n_vocab, bag, dim, lanes, p.unit, unit_blocks, each, part, scale, out, accumulate);
        if (many) hipLaunchKernelGGL((embed_merge_kernel<E, false>), merges, dim3(MERGE_THREADS), 0, ctx->stream, entry, range, p.m, n_vocab, p.unit, p.units, merge, dim, lanes, part, scale, out, accumulate);
    }
}

int run_embed_gradient(qgbdt_ctx* ctx, const void* tokens, int token_bytes, int64_t n, int bag, const void* grad, int dtype, int64_t n_vocab, int dim, float scale,
                       void* grad_table, int accumulate, void* scratch) {
    const EmbedPlan p = make_embed_plan(n, bag, n_vocab, dim, dtype);
    unsigned char* const s = static_cast<unsigned char*>(scratch);
    uint2* entry[2] = {reinterpret_cast<uint2*>(s + p.entry[0]), reinterpret_cast<uint2*>(s + p.entry[1])};
    int32_t* const counts = reinterpret_cast<int32_t*>(s + p.counts);
    int32_t* const totals = reinterpret_cast<int32_t*>(s + p.totals);
    int2* const range = reinterpret_cast<int2*>(s + p.range);
    int at = 0;
    if (p.m > 0 && p.sorted) {
        hipLaunchKernelGGL(clear_ranges_kernel, dim3(blocks_for(n_vocab, 1024, 1024)), dim3(256), 0, ctx->stream, range, n_vocab);
        const dim3 grid((unsigned)((p.m + SORT_FEW_ENTRIES - 1) / SORT_FEW_ENTRIES));
        if (token_bytes == 8) hipLaunchKernelGGL(sort_few_kernel<int64_t>, grid, dim3(256), 0, ctx->stream, FromTokens<int64_t>{tokens, n_vocab}, (int)p.m, n_vocab, entry[0], range);
        else hipLaunchKernelGGL(sort_few_kernel<int32_t>, grid, dim3(256), 0, ctx->stream, FromTokens<int32_t>{tokens, n_vocab}, (int)p.m, n_vocab, entry[0], range);
    } else if (p.m > 0) {
        for (int k = 0; k < p.passes; ++k) {
            if (k > 0) sort_pass(ctx, p, FromEntries{entry[at]}, k, counts, totals, entry[at ^ 1], range, n_vocab);
            else if (token_bytes == 8) sort_pass(ctx, p, FromTokens<int64_t>{tokens, n_vocab}, k, counts, totals, entry[at ^ 1], range, n_vocab);
            else sort_pass(ctx, p, FromTokens<int32_t>{tokens, n_vocab}, k, counts, totals, entry[at ^ 1], range, n_vocab);
            at ^= 1;
        }
        hipLaunchKernelGGL(ranges_kernel, dim3(blocks_for(p.m, 256, 4096)), dim3(256), 0, ctx->stream, entry[at], p.m, n_vocab, range);
    } else {
        hipLaunchKernelGGL(clear_ranges_kernel, dim3(blocks_for(n_vocab, 1024, 1024)), dim3(256), 0, ctx->stream, range, n_vocab);
    }
    float* const part = reinterpret_cast<float*>(s + p.part);
    if (dtype == QGBDT_F32) embed_sums<F32>(ctx, p, entry[at], range, part, bag, grad, n_vocab, dim, scale, grad_table, accumulate);
    else if (dtype == QGBDT_BF16) embed_sums<BF16>(ctx, p, entry[at], range, part, bag, grad, n_vocab, dim, scale, grad_table, accumulate);
    else embed_sums<F16>(ctx, p, entry[at], range, part, bag, grad, n_vocab, dim, scale, grad_table, accumulate);
    QG_HIP(ctx, hipGetLastError());
    return QGBDT_OK;
}

}  // namespace qgbdt
