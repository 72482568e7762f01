// One layer of every expert on the rows that chose it, and its gradients (gfx950).
//
// Three products of matrices whose rows are cut into ranges by expert:
//   forward   y[p, n]  = sum over k of x[row(p), k] * W_e[n, k]        p in the range of e
//   by input  dx[p, k] = sum over n of dz[p, n] * W_e[n, k]            p in the range of e
//   by weight dW_e[n, k] = sum over p in the range of e of dz[p, n] * x[row(p), k]
//
// Products and sums are in single precision; a result is rounded to the type once, at the end.  dx is one row a slot, rounded as such: the sum over a
// row's slots is another call (gr_expert_combine), so nothing here is added up by atomics and every result is the same from run to run.
//
// Bound by matrix instructions where an expert has hundreds of rows, by reading the weights where it has few, by reading x or writing dx where it has
// few output features.  Each of these has a form of its own; which one a call takes is decided in `product` at the end, with both sides' times.
#include <type_traits>

#include "experts.h"

namespace gr {
namespace {

constexpr int kBlock = 256;
constexpr int kWave = 64;

enum Product { kForward = 0, kByInput, kByWeight };

struct LinearArgs {
    const int *off, *slot;
    const void *x, *w, *bias, *dz;
    void* out;
    int64_t n_pos;
    int n_expert, n_in, n_out, top_k, relu;
    int tiles;      // in the direction of columns
    int64_t down;   // and of rows
    int block;      // rows of tiles taken together
    int parts_n;    // by weight: parts of an expert's positions that are summed apart,
    float* parts;   // and where: [parts_n][n_expert][n_out][n_in]
    uint32_t k_mul;      // slot / top_k: the upper half of slot * k_mul (the slot itself for 0), by 2^k_shift
    int k_shift;
};

// Bounds of a range, whatever the offsets hold.
__device__ __forceinline__ int64_t bound(const int* off, int e, int n_expert, int64_t n_pos)
{
    if (!off) return e == 0 ? 0 : n_pos;
    const int64_t v = off[e];
    return v < 0 ? 0 : v > n_pos ? n_pos : v;
}

// The row of a slot: a product in the place of a division (exact below 2^30, see args_of).
__device__ __forceinline__ uint32_t row_of_slot(const LinearArgs& a, uint32_t s) { return (a.k_mul ? __umulhi(s, a.k_mul) : s) >> a.k_shift; }

__device__ __forceinline__ int64_t row_of(const LinearArgs& a, int64_t p)
{
    if (!a.slot) return p;
    int s = a.slot[p];
    if (s < 0) s = -1 - s;
    return row_of_slot(a, s < a.n_pos ? s : (uint32_t)a.n_pos - 1);
}

// A part of an expert's positions (all of them where they are not cut), in whole slices of the reduction.
constexpr int kDepth = 64;

__device__ __forceinline__ void part_of(const LinearArgs& a, int e, int part, int64_t& lo, int64_t& depth)
{
    const int64_t from = bound(a.off, e, a.n_expert, a.n_pos), until = bound(a.off, e + 1, a.n_expert, a.n_pos);
    const int64_t slices = (until - from + kDepth - 1) / kDepth, each = (slices + a.parts_n - 1) / a.parts_n * kDepth;
    lo = from + part * each;
    depth = until - lo < each ? until - lo : each;
    if (depth < 0) depth = 0;
}

// A block of rows of the output: an expert (n_expert: rows without one) and positions lo .. hi - 1.
struct RowTile {
    int expert;
    int64_t lo, hi;
};

// The t-th tile of `rows` rows, no tile reaching from one expert's range into the next; lo = hi where there are fewer.
// Every lane of a wave calls it.
__device__ __forceinline__ RowTile row_tile(const int* off, int n_expert, int64_t n_pos, int rows, int64_t t)
{
    const int lane = threadIdx.x % kWave;
    int64_t before = 0;
    for (int e0 = 0; e0 <= n_expert; e0 += kWave) {
        const int e = e0 + lane;
        int64_t lo = 0, hi = 0;
        if (e <= n_expert) {
            lo = bound(off, e, n_expert, n_pos);
            hi = e < n_expert ? bound(off, e + 1, n_expert, n_pos) : n_pos;
        }
        const int own = hi > lo ? (int)((uint32_t)(hi - lo + rows - 1) / (uint32_t)rows) : 0;
        int v = own;
        for (int d = 1; d < kWave; d *= 2) {
            const int o = __shfl_up(v, d);
            if (lane >= d) v += o;
        }
        const int64_t end = before + v;
        const unsigned long long mine = __ballot(t >= end - own && t < end);
        if (mine) {
            const int l = __ffsll((long long)mine) - 1;
            const int64_t first = __shfl(lo, l) + (t - (__shfl(end, l) - __shfl(own, l))) * rows;
            const int64_t last = __shfl(hi, l);
            return {e0 + l, first, first + rows < last ? first + rows : last};
        }
        before = __shfl(end, kWave - 1);
    }
    return {n_expert, 0, 0};
}

// Tiles of all experts before one, and its own; every lane of a wave calls it.
__device__ __forceinline__ void tiles_before(const int* off, int n_expert, int64_t n_pos, int rows, int expert, int64_t& before, int64_t& own)
{
    int64_t sum = 0;
    own = 0;
    for (int e = threadIdx.x % kWave; e <= expert; e += kWave) {
        const int64_t lo = bound(off, e, n_expert, n_pos), hi = bound(off, e + 1, n_expert, n_pos);
        const int64_t tiles = hi > lo ? (uint32_t)(hi - lo + rows - 1) / (uint32_t)rows : 0;
        if (e < expert) sum += tiles;
        else own = tiles;
    }
    own = __shfl(own, expert % kWave);
    for (int d = 1; d < kWave; d *= 2) sum += __shfl_xor(sum, d);
    before = sum;
}

// Which tile workgroup j takes.  Workgroups go to the eight dies in turn, each with a cache of its own: a die takes blocks of neighbouring tiles, 32
// at a time, `block` rows down and the rest across, so that what they share is fetched into a die once.
constexpr int kDies = 8, kTogether = 32;

struct TileNo {
    int64_t row;      // -1: none
    int col;
};

// Tile t in the order of blocks.
__device__ __forceinline__ TileNo tile_at(int64_t t, int64_t down, int across, int block)
{
    const int64_t band = t / ((int64_t)block * across), in = t - band * block * across, left = down - band * block;
    const int rows = left < block ? (int)left : block;
    return {band * block + in % rows, (int)(in / rows)};
}

__device__ __forceinline__ TileNo tile_no(int64_t j, int64_t down, int across, int block)
{
    const int64_t all = down * across, each = (all + kDies - 1) / kDies;
    const int run = each < kTogether ? (int)each : kTogether;      // tiles that a die takes together (fewer where there are not 32 for each)
    if (run == 0) return {-1, 0};
    const int64_t at = j / kDies, t = (at / run * kDies + j % kDies) * run + at % run;
    return t < all ? tile_at(t, down, across, block) : TileNo{-1, 0};
}

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));

// acc += a * b over the reduction indexes that a lane's 16 bytes of each operand hold: lane l has row l % 16, indexes (l / 16) *
// n to (l / 16) * n + n - 1.  (For single precision four products of four indexes each; the order within a sum is free as long as
// both operands have the same.)
__device__ __forceinline__ f32x4 mfma(f32x4 a, f32x4 b, f32x4 acc)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], acc, 0, 0, 0);
    return acc;
}
__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 acc) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, acc, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma(f16x8 a, f16x8 b, f32x4 acc) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, acc, 0, 0, 0); }

// ---- any sizes, any alignment -------------------------------------------------------------------
//
// Tiles of 64 by 64, four waves of 32 by 32, 64 bytes of the reduction at a time: loaded into registers, four neighbours in memory at a time
// whatever their alignment, while the tile before is multiplied, and laid into shared memory with the reduction contiguous.  Small tiles, eight
// workgroups to a compute unit: their waits for memory and at barriers fall into each other's products.  Single precision, 8 198 positions of nine
// experts x 1 023 -> 511: 100 us alone, 112 one after the other: 77 to 86 TFLOP/s of the 153 that a large product reaches: 1 037 tiles are four or
// five to a unit, so a fifth of it is the last ones' (65 536 x 1 024 -> 512: 100 TFLOP/s; 20 000 x 4 096 -> 1 024: 109).  Loaded element by
// element the first took 149; twice the reduction at a time gains nothing there (118) and loses a third at short ones (131 072 x 100 -> 64 in
// bfloat16 30 / 41).

constexpr int kAnyTile = 64;

template <typename T>
constexpr int kAnyDepth = 64 / sizeof(T);

template <typename T, Product kProduct, int kVec>
__global__ __launch_bounds__(kBlock) void k_linear_any(LinearArgs a)
{
    constexpr int kRows = kAnyTile, kCols = kAnyTile;
    constexpr int D = kAnyDepth<T>, kLd = D + Chunk<T>::n, kPerP = kRows * D / kBlock / kVec, kPerQ = kCols * D / kBlock / kVec;
    typedef typename Chunk<T>::Vec Vec;
    constexpr int n = Chunk<T>::n;
    typedef Elements<T, kVec> Get;
    __shared__ __attribute__((aligned(16))) T lds_p[kRows * kLd], lds_q[kCols * kLd];

    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const TileNo no = tile_no(blockIdx.x, a.down, a.tiles, a.block);
    const int64_t row_no = no.row;
    if (row_no < 0) return;
    const T* const x = static_cast<const T*>(a.x);
    const T* const dz = static_cast<const T*>(a.dz);
    const int I = a.n_in, O = a.n_out;

    // the output's rows p0 .. p0 + p_n - 1 (positions, or output features of an expert), columns q0 .. q0 + q_n - 1
    int e, part = 0;
    int64_t p0, lo = 0, depth;
    int p_n, q0 = no.col * kCols, q_n;
    if constexpr (kProduct == kByWeight) {
        const int tiles = (O + kRows - 1) / kRows, of = (int)(row_no / tiles);
        e = of / a.parts_n;
        part = of - e * a.parts_n;
        p0 = (row_no - (int64_t)of * tiles) * kRows;
        p_n = O - p0 < kRows ? (int)(O - p0) : kRows;
        q_n = I - q0 < kCols ? I - q0 : kCols;
        part_of(a, e, part, lo, depth);
    } else {
        const RowTile t = row_tile(a.off, a.n_expert, a.n_pos, kRows, row_no);
        if (t.hi <= t.lo) return;
        e = t.expert;
        p0 = t.lo;
        p_n = (int)(t.hi - t.lo);
        const int width = kProduct == kForward ? O : I;
        q_n = width - q0 < kCols ? width - q0 : kCols;
        depth = e == a.n_expert ? 0 : kProduct == kForward ? I : O;
    }
    const T* const w = static_cast<const T*>(a.w) + (kProduct == kByWeight || e == a.n_expert ? 0 : (int64_t)e * O * I);

    // which of the tile's elements a thread loads, kVec neighbours in memory at a time
    constexpr bool kPLong = kProduct != kByWeight, kQLong = kProduct == kForward;      // those along the reduction
    // Rows past the edge are loaded from within it: what becomes of them is not stored.  Where neighbours are rows, the ones at the edge reach
    // back from it, before the tile if it has fewer rows than they are.
    const auto place = [&](bool along, int size, int rows, int i, int& row, int& r) __attribute__((always_inline)) {
        const int at = (i * kBlock + tid) * kVec;
        if (along) { row = at / D; r = at % D; }
        else { r = at / size; row = at % size; }
        const int last = rows - (along ? 1 : kVec);
        if (row > last) row = last;
    };
    const T *from_p[kPerP], *from_q[kPerQ];
#pragma unroll
    for (int i = 0; i < kPerP; ++i) {
        int row, r;
        place(kPLong, kRows, p_n, i, row, r);
        if constexpr (kProduct == kForward) from_p[i] = x + (e < a.n_expert ? row_of(a, p0 + row) : 0) * I + r;
        if constexpr (kProduct == kByInput) from_p[i] = dz + (p0 + row) * O + r;
        if constexpr (kProduct == kByWeight) from_p[i] = dz + (lo + r) * O + p0 + row;
    }
#pragma unroll
    for (int i = 0; i < kPerQ; ++i) {
        int row, r;
        place(kQLong, kCols, q_n, i, row, r);
        if constexpr (kProduct == kForward) from_q[i] = w + (int64_t)(q0 + row) * I + r;
        if constexpr (kProduct == kByInput) from_q[i] = w + (int64_t)r * I + q0 + row;
        if constexpr (kProduct == kByWeight) from_q[i] = x + q0 + row;
    }
    const int64_t step_p = kPLong ? D : (int64_t)D * O, step_q = kQLong ? D : (int64_t)D * I;
    Get get_p[kPerP], get_q[kPerQ];
    // past the end of the reduction there are zeros
    const auto get = [&](const T* from, bool along, int64_t r, bool whole) __attribute__((always_inline)) {
        Get v{};
        if (whole || r + (along ? kVec : 1) <= depth) v = Get::load(from);
        else if (along)
#pragma unroll
            for (int k = 0; k < kVec - 1; ++k)
                if (r + k < depth) v.v[k] = from[k];
        return v;
    };
    const auto load = [&](int64_t r0, bool whole) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kPerP; ++i) {
            int row, r;
            place(kPLong, kRows, p_n, i, row, r);
            get_p[i] = get(from_p[i], kPLong, r0 + r, whole);
            from_p[i] += step_p;
        }
#pragma unroll
        for (int i = 0; i < kPerQ; ++i) {
            int row, r;
            place(kQLong, kCols, q_n, i, row, r);
            const bool in = whole || r0 + r < depth;
            get_q[i] = get(from_q[i] + (kProduct == kByWeight && in ? row_of(a, lo + r0 + r) * I : 0), kQLong, r0 + r, whole);
            if (kProduct != kByWeight) from_q[i] += step_q;
        }
    };

    const auto put = [&](T* lds, bool along, int row, int r, const Get& v) __attribute__((always_inline)) {
        if (along) __builtin_memcpy(__builtin_assume_aligned(&lds[row * kLd + r], kVec * sizeof(T)), &v, sizeof v);
        else
#pragma unroll
            for (int k = 0; k < kVec; ++k)
                if (row + k >= 0) lds[(row + k) * kLd + r] = v.v[k];
    };
    constexpr int kP = kRows / 32, kQ = kCols / 32;      // fragments of a wave
    f32x4 acc[kP][kQ] = {};
    const int wp = wave / 2 * (kRows / 2), wq = wave % 2 * (kCols / 2);
    if (depth > 0) load(0, depth >= D);
    for (int64_t r0 = 0; r0 < depth; r0 += D) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kPerP; ++i) {
            int row, r;
            place(kPLong, kRows, p_n, i, row, r);
            put(lds_p, kPLong, row, r, get_p[i]);
        }
#pragma unroll
        for (int i = 0; i < kPerQ; ++i) {
            int row, r;
            place(kQLong, kCols, q_n, i, row, r);
            put(lds_q, kQLong, row, r, get_q[i]);
        }
        __syncthreads();
        if (r0 + 2 * D <= depth) load(r0 + D, true);
        else if (r0 + D < depth) load(r0 + D, false);
#pragma unroll
        for (int d = 0; d < D; d += 4 * n) {
            Vec p[kP], q[kQ];
#pragma unroll
            for (int i = 0; i < kP; ++i) p[i] = *reinterpret_cast<const Vec*>(&lds_p[(wp + i * 16 + lane % 16) * kLd + d + lane / 16 * n]);
#pragma unroll
            for (int i = 0; i < kQ; ++i) q[i] = *reinterpret_cast<const Vec*>(&lds_q[(wq + i * 16 + lane % 16) * kLd + d + lane / 16 * n]);
            // (columns as the first operand: a lane then holds four neighbours of a row)
#pragma unroll
            for (int i = 0; i < kP; ++i)
#pragma unroll
                for (int j = 0; j < kQ; ++j) acc[i][j] = mfma(q[j], p[i], acc[i][j]);
        }
    }

    const int width = kProduct == kForward ? O : I;
    const int64_t at = ((kProduct == kByWeight ? ((int64_t)part * a.n_expert + e) * O : 0) + p0) * width + q0;
    T* const out = static_cast<T*>(a.out) + at;
    const T* const bias = kProduct == kForward && a.bias && e < a.n_expert ? static_cast<const T*>(a.bias) + (int64_t)e * O + q0 : nullptr;
#pragma unroll
    for (int i = 0; i < kP; ++i) {
        const int row = wp + i * 16 + lane % 16;
        if (row >= p_n) continue;
#pragma unroll
        for (int j = 0; j < kQ; ++j) {
            const int col = wq + j * 16 + lane / 16 * 4;
            Elements<T, 4> o;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float v = acc[i][j][k] + (bias && col + k < q_n ? (float)bias[col + k] : 0.0f);
                if (kProduct == kForward && a.relu && v < 0) v = 0;
                o.v[k] = (T)v;
            }
            const int64_t to = (int64_t)row * width + col;
            if (kProduct == kByWeight && a.parts) {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (col + k < q_n) a.parts[at + to + k] = acc[i][j][k];
            } else if (col + 4 <= q_n) {
                o.store(out + to);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (col + k < q_n) out[to + k] = o.v[k];
            }
        }
    }
}

// ---- 16-bit types, rows of whole 16 bytes -------------------------------------------------------
//
// Tiles of kSize by kSize, 64 reduction indexes (a slice) at a time, four waves of half by half each.  Slices go from memory straight into shared
// memory.  An operand lies there as it does in memory:
//   long    its reduction is contiguous: [row][64 indexes]; a lane's eight indexes are one read of 16 bytes
//   across  its rows are contiguous: [64 indexes][row]; a lane's eight indexes are two reads that transpose 4 by 16
// What is written is one after the other, 16 bytes a lane, so which 16 bytes of memory a lane fetches decides the layout: their number
// within a line of the tile is exclusive-ored with one made of the line's, so that the lanes of a read meet no bank twice.
//
// Bound by the matrix units and, with them, by power: 131 072 positions of nine experts x 4 096 -> 1 024 in bfloat16 (1.1 TFLOP) forward 880 to
// 930 us (up to 1 250 TFLOP/s; the library's plain product of one such matrix 874), where the units are busy 59 % of the time at 1.89 GHz. Tiles
// of 256 by 256 because a fragment read from shared memory then serves eight products of a wave (at 128 by 128 four) and each operand is fetched
// half as often; the sums of a wave's 128 by 128 take half of all registers. Five slots of an operand's slice, 32 KB each, are all the shared
// memory there is. By input 65 536 x 4 096 <- 1 024 540 us (1 018 TFLOP/s, units busy 44 %: a tile is 16 slices, and writing it, 128 KB from each
// unit at the same time, holds up the loads behind it); by weight 670 us (820), of 128 by 128 (2 304 tiles on 512 places: 4.5 rounds, units busy
// 35 %: loads into shared memory, 32 KB a slice, take as long as its products; of 256, 576 on 256, 2.25 rounds, it takes 780).

constexpr int kSlots = 5, kWaves = 4;

__device__ const uint4 kZeros = {0, 0, 0, 0};      // where lanes read that are past the end of the reduction

typedef __attribute__((address_space(3))) char LdsChar;

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v)
{
    return (int64_t)((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32 | (uint32_t)uniform((int)v));
}

// 16 bytes a lane into shared memory at `to` and after (the compiler hands that over in m0), from an address of the lane's own, or from an offset
// to one of the wave's.  That one may come from the vector unit, a spilled register at the least: five wait states before memory's reads it, which
// the compiler does not add for a statement of this kind.  Backward, 65 536 x 4 096 -> 1 024, they are 6 us of 1 275.
__device__ __forceinline__ void fetch16(const char* from, uint32_t to)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "{m0}"(to) : "memory");
}
__device__ __forceinline__ void fetch16(const char* base, uint32_t offset, uint32_t to)
{
    asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(base), "{m0}"(to) : "memory");
}

__device__ __forceinline__ int across_swizzle(int r) { return (r & 3) << 1 | (r >> 3 & 1) << 3; }

// A lane's part of fragment `no` (16 rows or columns, 32 indexes), and where in a slice those of a wave start for it: everything that is not the
// lane's is a constant beside it.
template <bool kLong, int kSize>
__device__ __forceinline__ uint32_t fragments_at(int first, int lane)
{
    const int g = lane / 16, i = lane % 16;
    if constexpr (kLong) return (first + i) * (kDepth * 2) + (g ^ (i & 7)) * 16;
    const int r = g * 8 + i / 4;
    return r * (kSize * 2) + ((first / 8 + i % 4 / 2) ^ across_swizzle(r)) * 16 + i % 2 * 8;
}

template <typename T, bool kLong, int kSize>
__device__ __forceinline__ typename Chunk<T>::Vec fragment(const char* lds, uint32_t at, int half, int no)
{
    typedef typename Chunk<T>::Vec Vec;
    if constexpr (kLong) {
        return *reinterpret_cast<const Vec*>(lds + (at ^ half * 64) + no * (16 * kDepth * 2));
    } else {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 Lds4;
        union { s16x4 part[2]; Vec all; } v;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            v.part[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4*)(lds + (at ^ no * 32) + (half * 32 + h * 4) * (kSize * 2)));
        return v.all;
    }
}

// A lane's share of an operand's slice: load i of a wave, 1 KB each, brings line(i) (the reduction's index across, the row
// else), its piece(i) of 16 bytes.
template <bool kLong, int kSize>
struct Share {
    static constexpr int kLoads = kSize * kDepth * 2 / 1024 / kWaves;
    static constexpr int kPerLine = kLong ? 8 : kSize / 8;
    static constexpr int kLines = kWave / kPerLine;      // of a load
    static __device__ __forceinline__ int line(int i, int wave, int lane) { return ((wave * kLoads + i) * kWave + lane) / kPerLine; }
    static __device__ __forceinline__ int piece(int i, int wave, int lane)
    {
        const int l = line(i, wave, lane);
        return lane % kPerLine ^ (kLong ? l & 7 : across_swizzle(l));
    }
    // whether it is past the end of a reduction of which `left` indexes are left
    static __device__ __forceinline__ bool past(int i, int wave, int lane, int64_t left)
    {
        return (kLong ? piece(i, wave, lane) * 8 : line(i, wave, lane)) >= left;
    }
};

// acc += a * b with the sums where the compiler leaves them alone: there are as many as there are registers of their kind, and it moves them
// about. For the same reason no vector register of a kernel with these may be spilled: a variant that had some gave wrong sums, and the build fails
// where one does. (Scalar registers are, 24 to 96 a kernel, to lanes of vector registers.)
__device__ __forceinline__ void mfma_in_place(f32x4& acc, bf16x8 a, bf16x8 b)
{
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
}
__device__ __forceinline__ void mfma_in_place(f32x4& acc, f16x8 a, f16x8 b)
{
    asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
}

// An expert's range and its tiles, by lane, where a wave has a lane for each (kept from tile to tile).
struct Ranges {
    int lo, hi, tiles, end;      // `end`: tiles up to and with this expert's
};

struct Tile {
    int e, part, p_n, q0, q_n;
    int64_t p0, lo, depth;      // rows from p0 on (positions, or by weight output features); the reduction's start, by weight, and length
};

// A last round of large tiles that at most half of the units would have work in is left to tiles of 128 by 128, four in the place of each (kRest).
// Without / with: 65 536 x 4 096 -> 1 024 of nine experts 490 / 466 us, 65 536 x 1 024 -> 1 024 178 / 166, 131 072 x 4 096 -> 1 024 915 / 905;
// where nothing is left, 270 000 x 512 -> 1 024, 410 / 411.
constexpr int kUnits = 256;          // compute units: workgroups of large tiles that run at a time

__device__ __forceinline__ int64_t whole_rounds(int64_t all) { return all % kUnits <= kUnits / 2 ? all / kUnits * kUnits : all; }

template <typename T, Product kProduct, int kSize, bool kParts, bool kRest>
__global__ __launch_bounds__(kWaves * kWave, kSize > 128 ? 1 : 2) void k_linear_tiles(LinearArgs a)
{
    constexpr int kUnit = kRest ? 2 * kSize : kSize;      // rows and columns of what is numbered
    constexpr int kFrag = kSize / 2 / 16;      // fragments of a wave, either way
    constexpr bool kPLong = kProduct != kByWeight, kQLong = kProduct == kForward;
    constexpr int kSlotBytes = kSize * kDepth * 2;
    typedef typename Chunk<T>::Vec Vec;
    typedef Share<kPLong, kSize> ShareP;
    typedef Share<kQLong, kSize> ShareQ;
    constexpr int kLoads = ShareP::kLoads;
    __shared__ __attribute__((aligned(1024))) char lds[kSlots * kSlotBytes];

    const int lane = threadIdx.x % kWave, wave = uniform((int)threadIdx.x / kWave);
    const T* const x = static_cast<const T*>(a.x);
    const T* const dz = static_cast<const T*>(a.dz);
    const int I = a.n_in, O = a.n_out, width = kProduct == kForward ? O : I;
    const uint32_t lds_base = uniform((int)(uint32_t)(uintptr_t)(LdsChar*)lds) + wave * kLoads * 1024;

    // The lane's number, anew: what is made of it is not kept over the products, whose registers are all there are.
    const auto lane_now = [&]() __attribute__((always_inline)) {
        int l = lane;
        asm volatile("" : "+v"(l));
        return l;
    };

    // ---- which tiles
    Ranges mine{};
    int64_t down = a.down;
    const bool by_lane = a.n_expert < kWave;
    if constexpr (kProduct != kByWeight) {
        if (by_lane) {
            if (lane <= a.n_expert) {
                mine.lo = (int)bound(a.off, lane, a.n_expert, a.n_pos);
                mine.hi = lane < a.n_expert ? (int)bound(a.off, lane + 1, a.n_expert, a.n_pos) : (int)a.n_pos;
            }
            mine.tiles = mine.hi > mine.lo ? (mine.hi - mine.lo + kUnit - 1) / kUnit : 0;
            mine.end = mine.tiles;
            for (int d = 1; d < kWave; d *= 2) {
                const int o = __shfl_up(mine.end, d);
                if (lane >= d) mine.end += o;
            }
            down = __builtin_amdgcn_readlane(mine.end, kWave - 1);
        }
    }
    const auto quarter_of = [](Tile& t, int quarter) __attribute__((always_inline)) {      // false where it is past the edge
        const int down = quarter / 2 * kSize, right = quarter % 2 * kSize;
        t.p0 += down;
        t.p_n = t.p_n - down < kSize ? t.p_n - down : kSize;
        t.q0 += right;
        t.q_n = t.q_n - right < kSize ? t.q_n - right : kSize;
        return t.p_n > 0 && t.q_n > 0;
    };
    const auto find = [&](int64_t j, Tile& t) __attribute__((always_inline)) {
        TileNo no;
        int quarter = 0;
        const int64_t all = down * a.tiles, whole = whole_rounds(all);
        if constexpr (kRest) {      // the quarters of a tile go to one die
            const int64_t in = j / kDies, at = whole + in / 4 * kDies + j % kDies;
            if (at >= all) return false;
            no = tile_at(at, down, a.tiles, a.block);
            quarter = (int)(in % 4);
        } else {
            if (kSize > 128 && whole < all && j >= whole) return false;      // (a round of numbers is the same tiles in `tile_no`'s order)
            no = tile_no(j, down, a.tiles, a.block);
            if (no.row < 0) return false;
        }
        t.q0 = no.col * kUnit;
        t.q_n = width - t.q0 < kUnit ? width - t.q0 : kUnit;
        t.lo = 0;
        if constexpr (kProduct == kByWeight) {
            const int tiles = (O + kUnit - 1) / kUnit, part = (int)(no.row / tiles);
            t.e = part / a.parts_n;
            t.part = part - t.e * a.parts_n;
            t.p0 = (no.row - (int64_t)part * tiles) * kUnit;
            t.p_n = O - t.p0 < kUnit ? (int)(O - t.p0) : kUnit;
            if (kRest && !quarter_of(t, quarter)) return false;
            part_of(a, t.e, t.part, t.lo, t.depth);
            t.lo = uniform(t.lo);
            t.depth = uniform(t.depth);
        } else {
            RowTile r{a.n_expert, 0, 0};
            if (by_lane) {
                const unsigned long long here = __ballot(no.row >= mine.end - mine.tiles && no.row < mine.end);
                if (here) {
                    const int l = __ffsll((long long)here) - 1;
                    const int64_t first = __builtin_amdgcn_readlane(mine.lo, l) + (no.row - (__builtin_amdgcn_readlane(mine.end, l) - __builtin_amdgcn_readlane(mine.tiles, l))) * kUnit;
                    const int64_t last = __builtin_amdgcn_readlane(mine.hi, l);
                    r = {l, first, first + kUnit < last ? first + kUnit : last};
                }
            } else {
                r = row_tile(a.off, a.n_expert, a.n_pos, kUnit, no.row);
            }
            t.e = uniform(r.expert);
            t.p0 = uniform(r.lo);
            t.p_n = uniform((int)(r.hi - r.lo));
            if (kRest && !quarter_of(t, quarter)) return false;
            t.depth = t.e == a.n_expert || t.p_n <= 0 ? 0 : kProduct == kForward ? I : O;
        }
        return true;
    };

    // ---- where their slices come from: an address of the wave's that moves on from slice to slice, and a lane's offset to it; but rows of x are a
    // lane's own.  (Rows and columns past the edge are fetched from within it: what becomes of them is not stored.)
    const char *base_p = nullptr, *base_q = nullptr;
    const int64_t step_p = kPLong ? kDepth * 2 : (int64_t)kDepth * 2 * O, step_q = kQLong ? kDepth * 2 : (int64_t)kDepth * 2 * I;
    uint32_t off_p[kLoads], off_q[kLoads];
    const char* x_at[kLoads];      // forward: a lane's rows of x; by weight: those of a slice
    int x_row[kLoads];             // forward: the rows of the next tile
    const auto look_up = [&](const Tile& t) __attribute__((always_inline)) {
        const int lane = lane_now();
        if constexpr (kProduct == kForward)
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int line = ShareP::line(i, wave, lane);
                x_row[i] = t.depth > 0 ? (int)row_of(a, t.p0 + (line < t.p_n ? line : t.p_n - 1)) : 0;
            }
    };
    const auto aim = [&](const Tile& t) __attribute__((always_inline)) {
        const int lane = lane_now();
        const T* const w = static_cast<const T*>(a.w) + (t.depth > 0 ? (int64_t)t.e * O * I : 0);
        if constexpr (kProduct == kForward) base_q = reinterpret_cast<const char*>(w + (int64_t)t.q0 * I);
        if constexpr (kProduct == kByInput) {
            base_p = reinterpret_cast<const char*>(dz + t.p0 * O);
            base_q = reinterpret_cast<const char*>(w + t.q0);
        }
        if constexpr (kProduct == kByWeight) {
            base_p = reinterpret_cast<const char*>(dz + t.lo * O + t.p0);
            base_q = reinterpret_cast<const char*>(x + t.q0);
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int line = ShareP::line(i, wave, lane), piece = ShareP::piece(i, wave, lane), row = line < t.p_n ? line : t.p_n - 1;
            if constexpr (kProduct == kForward) x_at[i] = reinterpret_cast<const char*>(x + (int64_t)x_row[i] * I + piece * 8);
            if constexpr (kProduct == kByInput) off_p[i] = (uint32_t)row * O * 2 + piece * 16;
            if constexpr (kProduct == kByWeight) off_p[i] = (uint32_t)line * O * 2 + (piece * 8 < t.p_n ? piece * 16 : 0);
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int line = ShareQ::line(i, wave, lane), piece = ShareQ::piece(i, wave, lane);
            if constexpr (kProduct == kForward) off_q[i] = (uint32_t)(line < t.q_n ? line : t.q_n - 1) * I * 2 + piece * 16;
            if constexpr (kProduct == kByInput) off_q[i] = (uint32_t)line * I * 2 + (piece * 8 < t.q_n ? piece * 16 : 0);
            if constexpr (kProduct == kByWeight) off_q[i] = piece * 8 < t.q_n ? piece * 16 : 0;
        }
    };
    // By weight: the rows of x of 16 slices, a wave's lines of four slices in a register; a slice's are handed to the lanes that fetch them.
    constexpr int kLinesOfWave = kDepth / kWaves, kRowRegs = 16 * kLinesOfWave / kWave;
    typedef int RowRegs __attribute__((ext_vector_type(kRowRegs)));
    RowRegs rows{}, rows_later{};
    const auto load_rows = [&](int64_t p) __attribute__((always_inline)) {
        RowRegs to;
        const int lane = lane_now();
#pragma unroll
        for (int r = 0; r < kRowRegs; ++r) {
            const int line = r * kWave + lane;
            int64_t at = p + line / kLinesOfWave * kDepth + wave * kLinesOfWave + line % kLinesOfWave;
            if (at >= a.n_pos) at = a.n_pos - 1;
            uint32_t s = a.slot ? (uint32_t)a.slot[at] : (uint32_t)at;
            if (s >= a.n_pos) s = (uint32_t)a.n_pos - 1;
            if (a.slot) s = row_of_slot(a, s);
            to[r] = (int)s;
        }
        return to;
    };
    const auto aim_rows = [&](int slice) __attribute__((always_inline)) {
        constexpr int kOfReg = kWave / kLinesOfWave;
        const int lane = lane_now(), c = slice % 16;
        int from = rows[0];
#pragma unroll
        for (int r = 1; r < kRowRegs; ++r) from = c / kOfReg == r ? rows[r] : from;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int row = __builtin_amdgcn_ds_bpermute((c % kOfReg * kLinesOfWave + i * ShareQ::kLines + lane / ShareQ::kPerLine) * 4, from);
            x_at[i] = base_q + ((uint64_t)(uint32_t)row * ((uint32_t)I * 2) + off_q[i]);
        }
    };
    // what slice `slice` of a tile needs of them (the first 16 are there)
    const auto turn_rows = [&](const Tile& t, int slice) __attribute__((always_inline)) {
        if (slice % 16 == 8) rows_later = load_rows(t.lo + (int64_t)(slice / 16 + 1) * (16 * kDepth));
        if (slice % 16 == 0) rows = rows_later;
        aim_rows(slice);
    };

    const char* const zeros = reinterpret_cast<const char*>(&kZeros);
    const auto fetch_p = [&](int i, uint32_t slot, int64_t left, bool whole) __attribute__((always_inline)) {
        const uint32_t to = lds_base + slot + i * 1024;
        if constexpr (kProduct == kForward) {
            fetch16(!whole && ShareP::past(i, wave, lane_now(), left) ? zeros : x_at[i], to);
            x_at[i] += kDepth * 2;
        } else if (whole) {
            fetch16(base_p, off_p[i], to);
        } else {
            fetch16(ShareP::past(i, wave, lane_now(), left) ? zeros : base_p + off_p[i], to);
        }
        if (i == kLoads - 1) base_p += step_p;
    };
    const auto fetch_q = [&](int i, uint32_t slot, int64_t left, bool whole) __attribute__((always_inline)) {
        const uint32_t to = lds_base + slot + i * 1024;
        if constexpr (kProduct == kByWeight) {
            fetch16(!whole && ShareQ::past(i, wave, lane_now(), left) ? zeros : x_at[i], to);
        } else if (whole) {
            fetch16(base_q, off_q[i], to);
        } else {
            fetch16(ShareQ::past(i, wave, lane_now(), left) ? zeros : base_q + off_q[i], to);
        }
        if (kProduct != kByWeight && i == kLoads - 1) base_q += step_q;
    };

    // ---- multiplication.  A slice is multiplied in two halves of its depth.  While one is multiplied the other is read from shared memory, a fragment
    // after every few products.  Between them the slice has been read whole, and the next one has to be there.  Of five places in shared memory the
    // operands of a slice take two; in the first half the left operand two slices on is asked for, in the second the right one, a load
    // after every eight products: more at a time than memory's queue takes would hold the products up.
    constexpr int kGroups = 2 * kFrag;
    f32x4 acc[kFrag][kFrag];
    const int wp = wave / 2 * (kSize / 2), wq = wave % 2 * (kSize / 2);
    const uint32_t p_at = fragments_at<kPLong, kSize>(wp, lane), q_at = fragments_at<kQLong, kSize>(wq, lane);
    Vec p[2][kFrag], q[2][kFrag];
    const auto read = [&](uint32_t slot_p, uint32_t slot_q, int half, int no) __attribute__((always_inline)) {
        if (no < kFrag) q[half][no] = fragment<T, kQLong, kSize>(lds, q_at + slot_q, half, no);
        else p[half][no - kFrag] = fragment<T, kPLong, kSize>(lds, p_at + slot_p, half, no - kFrag);
    };
    // `fetch(g)` is called before the products of group g
    const auto multiply = [&](int half, bool reads, uint32_t slot_p, uint32_t slot_q, auto fetch) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            __builtin_amdgcn_sched_barrier(0);
            if (reads) read(slot_p, slot_q, half ^ 1, g);
            fetch(g);
            asm volatile("s_nop 1");      // (between what the vector unit has written and a product that might read it)
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < kFrag / 2; ++j) {
                const int col = g % 2 * (kFrag / 2) + j;
                mfma_in_place(acc[g / 2][col], q[half][col], p[half][g / 2]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    const auto settle = [&]() __attribute__((always_inline)) {      // (products write their sums some cycles after they are issued)
        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
        for (int i = 0; i < kFrag; ++i)
#pragma unroll
            for (int j = 0; j < kFrag; ++j) asm volatile("" : "+a"(acc[i][j]));
    };
    // (through a descriptor, whose bounds drop what is past the edge: the same stores whatever the tile's size)
    const auto store = [&](const Tile& t) __attribute__((always_inline)) {
        typedef T Four __attribute__((ext_vector_type(4)));
        typedef uint32_t Two __attribute__((ext_vector_type(2)));
        constexpr uint32_t kNowhere = ~0u;
        typedef std::conditional_t<kParts, float, T> Out;
        const int64_t first = kProduct == kByWeight ? ((int64_t)t.part * a.n_expert + t.e) * O : 0;
        Out* const out = (kParts ? reinterpret_cast<Out*>(a.parts) : static_cast<Out*>(a.out)) + (first + t.p0) * width + t.q0;
        const int lane = lane_now();
        const __amdgpu_buffer_rsrc_t to = __builtin_amdgcn_make_buffer_rsrc(out, 0, 0x7fffffff, 0x00027000);
        const bool biased = kProduct == kForward && a.bias && t.e < a.n_expert;
        const T* const bias = static_cast<const T*>(a.bias) + (int64_t)t.e * O + t.q0;
        if constexpr (kParts) {
#pragma unroll
            for (int j = 0; j < kFrag; ++j) {
                const int col = wq + j * 16 + lane / 16 * 4;
#pragma unroll
                for (int i = 0; i < kFrag; ++i) {
                    const int row = wp + i * 16 + lane % 16;
                    typedef uint32_t Bits __attribute__((ext_vector_type(4)));
                    union { f32x4 value; Bits bits; } o;
                    o.value = acc[i][j];
                    __builtin_amdgcn_raw_buffer_store_b128(
                        o.bits, to, row < t.p_n && col < t.q_n ? (uint32_t)(row * width + col) * (uint32_t)sizeof(Out) : kNowhere, 0, 0);
                }
            }
            return;
        }
        // Two fragments' columns at a time: a lane has four of each; exchanged between the wave's rows of 16 lanes they are eight in a row, so that
        // a store writes 64 bytes of a line instead of 32.
#pragma unroll
        for (int j = 0; j < kFrag; j += 2) {
            float b[2][4] = {};
#pragma unroll
            for (int f = 0; f < 2; ++f) {
                const int of = wq + (j + f) * 16 + lane / 16 * 4;
                if (biased && of < t.q_n) {
                    const Elements<T, 4> v = Elements<T, 4>::load(bias + of);
#pragma unroll
                    for (int k = 0; k < 4; ++k) b[f][k] = (float)v.v[k];
                }
            }
            const int col = wq + j * 16 + lane / 16 * 8;
#pragma unroll
            for (int i = 0; i < kFrag; ++i) {
                const int row = wp + i * 16 + lane % 16;
                const uint32_t at = row < t.p_n && col < t.q_n ? (uint32_t)(row * width + col) * (uint32_t)sizeof(Out) : kNowhere;
                union { Four value; Two bits; } o[2];
#pragma unroll
                for (int f = 0; f < 2; ++f)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        float v = acc[i][j + f][k] + b[f][k];
                        if (kProduct == kForward && a.relu && v < 0) v = 0;
                        o[f].value[k] = (T)v;
                    }
                typedef uint32_t Bits __attribute__((ext_vector_type(4)));
                Bits all;
#pragma unroll
                for (int d = 0; d < 2; ++d) {
                    const auto half = __builtin_amdgcn_permlane32_swap(o[0].bits[d], o[1].bits[d], false, false);
                    const auto both = __builtin_amdgcn_permlane16_swap(half[0], half[1], false, false);
                    all[d] = both[0];
                    all[2 + d] = both[1];
                }
                __builtin_amdgcn_raw_buffer_store_b128(all, to, at, 0, 0);
                __builtin_amdgcn_sched_barrier(0);      // (sums of one fragment's are in the other registers at a time)
            }
        }
    };

    constexpr uint32_t kRing = kSlots * kSlotBytes;
    const auto further = [](uint32_t slot) { return slot + 2 * kSlotBytes < kRing ? slot + 2 * kSlotBytes : slot + 2 * kSlotBytes - kRing; };
    const auto after = [](uint32_t slot) { return slot + kSlotBytes < kRing ? slot + kSlotBytes : 0; };
    const auto nothing = [](int) {};

    // The first two slices of a tile, into the first four places: part g of kGroups.
    const auto begin = [&](const Tile& t, int g) __attribute__((always_inline)) {
        constexpr int kEach = 4 * kLoads / kGroups;
#pragma unroll
        for (int l = g * kEach; l < (g + 1) * kEach; ++l) {
            const int slice = l / (2 * kLoads), in = l % (2 * kLoads);
            const int64_t left = t.depth - slice * kDepth;
            if (kProduct == kByWeight && in == 0) aim_rows(slice);
            if (in < kLoads) fetch_p(in, slice * 2 * kSlotBytes, left, false);
            else fetch_q(in - kLoads, (slice * 2 + 1) * kSlotBytes, left, false);
        }
    };

    Tile now, then;
    int64_t j = blockIdx.x;
    if (!find(j, now)) return;
    look_up(now);
    if constexpr (kProduct == kByWeight) rows = load_rows(now.lo);
    aim(now);
#pragma unroll
    for (int g = 0; g < kGroups; ++g) begin(now, g);
    bool behind = false;      // whether a tile's stores are behind those loads
    for (;;) {
        j += gridDim.x;
        const bool more = find(j, then);
        if (!more) then = Tile{0, 0, 1, 0, 8, 0, 0, 0};      // (nothing is fetched of a tile without depth)
        look_up(then);
#pragma unroll
        for (int i = 0; i < kFrag; ++i)
#pragma unroll
            for (int k = 0; k < kFrag; ++k) acc[i][k] = f32x4{0, 0, 0, 0};
        settle();
        const int slices = (int)((now.depth + kDepth - 1) / kDepth), whole = (int)(now.depth / kDepth);
        if (slices > 0) {
            // the first slice: behind it there may be the second, and the stores
            constexpr int kStores = kParts ? kFrag * kFrag : kFrag * kFrag / 2;
            if (slices == 1) asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
            else if (behind) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(2 * kLoads + kStores < 63 ? 2 * kLoads + kStores : 63) : "memory");
            else asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(2 * kLoads) : "memory");
#pragma unroll
            for (int no = 0; no < 2 * kFrag; ++no) read(0, kSlotBytes, 0, no);
            uint32_t slot = 0;      // of the left operand of slice s; the right one's is the next
            int s = 0;
            for (; s + 2 < whole; ++s) {
                const uint32_t next = further(slot), far = further(next);
                multiply(0, true, slot, after(slot), [&](int g) __attribute__((always_inline)) {
                    if (g % (kGroups / kLoads) == 0) fetch_p(g / (kGroups / kLoads), far, 0, true);
                });
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kLoads) : "memory");
                if constexpr (kProduct == kByWeight) turn_rows(now, s + 2);
                multiply(1, true, next, after(next), [&](int g) __attribute__((always_inline)) {
                    if (g % (kGroups / kLoads) == 0) fetch_q(g / (kGroups / kLoads), after(far), 0, true);
                });
                slot = next;
            }
            for (; s + 1 < slices; ++s) {
                const uint32_t next = further(slot), far = further(next);
                const int64_t left = now.depth - (int64_t)(s + 2) * kDepth;
                if (left > 0)
#pragma unroll
                    for (int i = 0; i < kLoads; ++i) fetch_p(i, far, left, false);
                multiply(0, true, slot, after(slot), nothing);
                if (left > 0) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kLoads) : "memory");
                else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
                if (left > 0) {
                    if constexpr (kProduct == kByWeight) turn_rows(now, s + 2);
#pragma unroll
                    for (int i = 0; i < kLoads; ++i) fetch_q(i, after(far), left, false);
                }
                multiply(1, true, next, after(next), nothing);
                slot = next;
            }
            multiply(0, true, slot, after(slot), nothing);
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        }
        // (shared memory has been read to the end by all waves)
        aim(then);
        if constexpr (kProduct == kByWeight) rows = load_rows(then.lo);
        if (slices > 0) {
            multiply(1, false, 0, 0, [&](int g) __attribute__((always_inline)) { begin(then, g); });
        } else {
#pragma unroll
            for (int g = 0; g < kGroups; ++g) begin(then, g);
        }
        settle();
        store(now);
        if (!more) break;
        behind = true;
        now = then;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// The parts of sums, added in their order whatever order they came in; N at a time.  Bound by reading them (9 x 33 x 1 024 in 14 parts, 17 MB: 5.8
// us).
template <typename T, int N>
__global__ __launch_bounds__(kBlock) void k_join(const float* parts, int n, int64_t count, T* out)
{
    typedef float Sums __attribute__((ext_vector_type(N)));
    typedef T Out __attribute__((ext_vector_type(N)));
    const int64_t i = ((int64_t)blockIdx.x * kBlock + threadIdx.x) * N;
    if (i >= count) return;
    Sums sum = *reinterpret_cast<const Sums*>(parts + i);
    for (int k = 1; k < n; ++k) sum += *reinterpret_cast<const Sums*>(parts + k * count + i);
    Out o;
#pragma unroll
    for (int k = 0; k < N; ++k) o[k] = (T)sum[k];
    *reinterpret_cast<Out*>(out + i) = o;
}

// Adds up what the groups of a workgroup have, halving them, into the first one's; all threads call it.
template <int N>
__device__ __forceinline__ void sum_groups(float* part, float (&sum)[N], int group, int groups)
{
    const int across = kBlock / groups;
    __syncthreads();
    for (int half = groups / 2; half > 0; half /= 2) {
        if (group >= half && group < 2 * half)
#pragma unroll
            for (int n = 0; n < N; ++n) part[(threadIdx.x - half * across) * N + n] = sum[n];
        __syncthreads();
        if (group < half)
#pragma unroll
            for (int n = 0; n < N; ++n) sum[n] += part[threadIdx.x * N + n];
        __syncthreads();
    }
}

// ---- few output features -----------------------------------------------------------------------
//
// Up to 16 (a predictor's last layer has one): a tile of 64 would be mostly empty.  Bound by reading x, or writing dx, once; rows of any length and
// alignment.  147 456 positions x 512 -> 1 in bfloat16: forward 25 us (151 MB, from the cache: 6 TB/s), backward 67; in tiles 51 and 404.
// 32 768 x 2 703 -> 8, bfloat16: forward 132 (rows on odd addresses of two bytes, which 16-byte loads take at half the rate; single precision 99
// for twice the bytes), backward 161; in tiles, element by element, 600.

constexpr int kNarrow = 16;

// Elements k and after of a row of `size`, zeros past its end.
template <typename T>
__device__ __forceinline__ typename Chunk<T>::Vec chunk_of(const T* row, int k, int size)
{
    constexpr int n = Chunk<T>::n;
    typename Chunk<T>::Vec v{};
    if (k + n <= size) {
        const Elements<T, n> e = Elements<T, n>::load(row + k);
#pragma unroll
        for (int j = 0; j < n; ++j) v[j] = e.v[j];
    } else {
#pragma unroll
        for (int j = 0; j < n - 1; ++j)
            if (k + j < size) v[j] = row[k + j];
    }
    return v;
}

// Forward: a wave takes 16 positions and all features, straight from memory into registers, as the operands of one 16 by 16 product after another.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_linear_narrow(LinearArgs a)
{
    typedef typename Chunk<T>::Vec Vec;
    constexpr int n = Chunk<T>::n, kStep = 4 * n, kAsked = 4;      // indexes of a product (or four); products asked for together
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, g = lane / 16, i = lane % 16, I = a.n_in, O = a.n_out;
    const RowTile t = row_tile(a.off, a.n_expert, a.n_pos, 16 * (kBlock / kWave), blockIdx.x);
    const int64_t p0 = t.lo + wave * 16;
    if (p0 >= t.hi) return;
    const bool any = t.expert < a.n_expert;
    const int64_t p = p0 + i < t.hi ? p0 + i : t.hi - 1;
    const T* const x = static_cast<const T*>(a.x) + (any ? row_of(a, p) : 0) * I;
    const T* const w = static_cast<const T*>(a.w) + ((int64_t)(any ? t.expert : 0) * O + (i < O ? i : O - 1)) * I;
    f32x4 acc = {0, 0, 0, 0};
    const int depth = any ? I : 0;
    int k0 = 0;
    for (; k0 + kAsked * kStep <= depth; k0 += kAsked * kStep) {      // (no lane asks whether it is within the row)
        Elements<T, n> xv[kAsked], wv[kAsked];
#pragma unroll
        for (int s = 0; s < kAsked; ++s) {
            xv[s] = Elements<T, n>::load(x + k0 + s * kStep + g * n);
            wv[s] = Elements<T, n>::load(w + k0 + s * kStep + g * n);
        }
#pragma unroll
        for (int s = 0; s < kAsked; ++s) acc = mfma(__builtin_bit_cast(Vec, wv[s]), __builtin_bit_cast(Vec, xv[s]), acc);
    }
    for (; k0 < depth; k0 += kStep) acc = mfma(chunk_of(w, k0 + g * n, depth), chunk_of(x, k0 + g * n, depth), acc);
    if (p0 + i >= t.hi) return;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int o = g * 4 + k;
        if (o >= O) continue;
        float v = acc[k] + (a.bias && any ? (float)static_cast<const T*>(a.bias)[(int64_t)t.expert * O + o] : 0.0f);
        if (a.relu && v < 0) v = 0;
        static_cast<T*>(a.out)[(p0 + i) * O + o] = (T)v;
    }
}

// Backward, no matrix instructions: up to 16 multiplications for every element that moves.
// Threads across a row of n_in, each with neighbouring columns, and down a block of rows.  Where a row is no whole number of those, its last
// thread's columns reach back into the one's before: both come to the same values.
struct NarrowShape {
    int lg, across;      // threads across as a power of two; workgroups across
};

constexpr int kNarrowRows = 64, kNarrowLeast = 8;      // rows of a block, most (they are held in shared memory) and least

// By input: dx[p] = the sum over the features of dz[p, o] * W[o]; a thread keeps its columns of W.
template <typename T, int N, int kOut>
__global__ __launch_bounds__(kBlock) void k_narrow_by_input(LinearArgs a, NarrowShape s, int most)
{
    __shared__ float dzs[kNarrowRows][kOut];
    const int I = a.n_in, O = a.n_out, lane = threadIdx.x & ((1 << s.lg) - 1), group = threadIdx.x >> s.lg, groups = kBlock >> s.lg;
    const RowTile t = row_tile(a.off, a.n_expert, a.n_pos, most, blockIdx.x / s.across);
    if (t.hi <= t.lo) return;
    const int rows = (int)(t.hi - t.lo);
    const bool any = t.expert < a.n_expert;
    for (int i = threadIdx.x; i < kNarrowRows * kOut; i += kBlock) {
        const int r = i / kOut, o = i % kOut;
        dzs[r][o] = any && r < rows && o < O ? (float)static_cast<const T*>(a.dz)[(t.lo + r) * O + o] : 0.0f;
    }
    __syncthreads();
    int c = ((int)(blockIdx.x % s.across) << s.lg | lane) * N;
    if (c >= I) return;
    if (c + N > I) c = I - N;
    const T* const w = static_cast<const T*>(a.w) + (int64_t)(any ? t.expert : 0) * O * I + c;
    float wv[kOut][N];
#pragma unroll
    for (int o = 0; o < kOut; ++o) {
        const Elements<T, N> e = Elements<T, N>::load(w + (int64_t)(o < O ? o : 0) * I);
#pragma unroll
        for (int j = 0; j < N; ++j) wv[o][j] = any && o < O ? (float)e.v[j] : 0.0f;
    }
#pragma unroll 2
    for (int r = group; r < rows; r += groups) {
        float sum[N] = {};
#pragma unroll
        for (int o = 0; o < kOut; ++o)
#pragma unroll
            for (int j = 0; j < N; ++j) sum[j] = fmaf(dzs[r][o], wv[o][j], sum[j]);
        Elements<T, N> e;
#pragma unroll
        for (int j = 0; j < N; ++j) e.v[j] = (T)sum[j];
        e.store(static_cast<T*>(a.out) + (t.lo + r) * I + c);
    }
}

// By weight: the sums of a block of rows, [block][n_out][n_in], which k_sum_blocks adds up; a thread keeps its columns' sums, and what it reads of x
// is used for all features at once.
template <typename T, int N, int kOut>
__global__ __launch_bounds__(kBlock) void k_narrow_by_weight(LinearArgs a, NarrowShape s, int rows)
{
    __shared__ float part[kBlock * N], dzs[kNarrowRows][kOut];
    __shared__ uint32_t xs[kNarrowRows];
    const int I = a.n_in, O = a.n_out, lane = threadIdx.x & ((1 << s.lg) - 1), group = threadIdx.x >> s.lg, groups = kBlock >> s.lg;
    const int64_t block = blockIdx.x / s.across;
    const RowTile t = row_tile(a.off, a.n_expert, a.n_pos, rows, block);
    if (t.expert == a.n_expert) return;
    int c = ((int)(blockIdx.x % s.across) << s.lg | lane) * N;
    const bool in = c < I;
    if (c + N > I) c = I - N;
    float sum[kOut][N] = {};
    for (int64_t p0 = t.lo; p0 < t.hi; p0 += kNarrowRows) {
        const int own = t.hi - p0 < kNarrowRows ? (int)(t.hi - p0) : kNarrowRows;
        __syncthreads();
        for (int i = threadIdx.x; i < kNarrowRows * kOut; i += kBlock) {
            const int r = i / kOut, o = i % kOut;
            dzs[r][o] = r < own && o < O ? (float)static_cast<const T*>(a.dz)[(p0 + r) * O + o] : 0.0f;
        }
        if (threadIdx.x < own) xs[threadIdx.x] = (uint32_t)row_of(a, p0 + threadIdx.x);
        __syncthreads();
        if (!in) continue;
#pragma unroll 4
        for (int r = group; r < own; r += groups) {
            const Elements<T, N> e = Elements<T, N>::load(static_cast<const T*>(a.x) + (int64_t)xs[r] * I + c);
#pragma unroll
            for (int o = 0; o < kOut; ++o)
#pragma unroll
                for (int j = 0; j < N; ++j) sum[o][j] = fmaf(dzs[r][o], (float)e.v[j], sum[o][j]);
        }
    }
#pragma unroll
    for (int o = 0; o < kOut; ++o) {
        if (o >= O) continue;
        sum_groups<N>(part, sum[o], group, groups);
        if (group > 0 || !in) continue;
#pragma unroll
        for (int j = 0; j < N; ++j) a.parts[(block * O + o) * I + c + j] = sum[o][j];
    }
}

// ---- few rows an expert ------------------------------------------------------------------------
//
// Bound by reading the weights, each once: a workgroup takes 16 output features of an expert, its waves a part of the reduction each, straight
// from memory into registers; their sums meet in shared memory.  Rows of x are taken 16 at a time.  Nothing is shared between waves but a row of
// x, which the cache holds, so shared memory would only add a wait.  9 positions of nine experts x 4 096 -> 1 024 in bfloat16 (75 MB): 17.7 us,
// 4.3 TB/s (a copy reaches 5.0); single precision 30.5, 5.0 TB/s.  (Four loads at a time or sixteen: the same.)

constexpr int kFewWaves = 4, kFewAhead = 8;      // loads of an operand asked for together

template <typename T>
__global__ __launch_bounds__(kFewWaves * kWave) void k_linear_few(LinearArgs a)
{
    typedef typename Chunk<T>::Vec Vec;
    constexpr int n = Chunk<T>::n, kStep = 4 * n;
    __shared__ f32x4 sums[kFewWaves - 1][kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, g = lane / 16, i = lane % 16;
    const int e = blockIdx.x / a.tiles, n0 = blockIdx.x % a.tiles * 16, I = a.n_in, O = a.n_out;
    const int64_t lo = bound(a.off, e, a.n_expert, a.n_pos), hi = e < a.n_expert ? bound(a.off, e + 1, a.n_expert, a.n_pos) : a.n_pos;
    const T* const w = static_cast<const T*>(a.w) + ((int64_t)(e < a.n_expert ? e : 0) * O + (n0 + i < O ? n0 + i : O - 1)) * I;
    const int depth = e < a.n_expert ? I : 0, each = (depth + kFewWaves * kStep - 1) / (kFewWaves * kStep) * kStep;
    const int from = wave * each, until = from + each < depth ? from + each : depth;
    for (int64_t p0 = lo; p0 < hi; p0 += 16) {
        const int64_t p = p0 + i < hi ? p0 + i : hi - 1;
        const T* const x = static_cast<const T*>(a.x) + (e < a.n_expert ? row_of(a, p) : 0) * I;
        f32x4 acc = {0, 0, 0, 0};
        int d = from;
        for (; d + kFewAhead * kStep <= until; d += kFewAhead * kStep) {
            Elements<T, n> wv[kFewAhead], xv[kFewAhead];
#pragma unroll
            for (int k = 0; k < kFewAhead; ++k) {
                wv[k] = Elements<T, n>::load(w + d + k * kStep + g * n);
                xv[k] = Elements<T, n>::load(x + d + k * kStep + g * n);
            }
#pragma unroll
            for (int k = 0; k < kFewAhead; ++k) acc = mfma(__builtin_bit_cast(Vec, wv[k]), __builtin_bit_cast(Vec, xv[k]), acc);
        }
        if (d < until) {
            Vec wv[kFewAhead], xv[kFewAhead];
#pragma unroll
            for (int k = 0; k < kFewAhead; ++k) {
                wv[k] = chunk_of(w, d + k * kStep + g * n, until);
                xv[k] = chunk_of(x, d + k * kStep + g * n, until);
            }
#pragma unroll
            for (int k = 0; k < kFewAhead; ++k) acc = mfma(wv[k], xv[k], acc);
        }
        if (wave > 0) sums[wave - 1][lane] = acc;
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int k = 0; k < kFewWaves - 1; ++k) acc += sums[k][lane];
            const int at = n0 + g * 4;
            if (p0 + i < hi && at < O) {
                Elements<T, 4> o;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float v = acc[k] + (a.bias && e < a.n_expert && at + k < O ? (float)static_cast<const T*>(a.bias)[(int64_t)e * O + at + k] : 0.0f);
                    if (a.relu && v < 0) v = 0;
                    o.v[k] = (T)v;
                }
                T* const out = static_cast<T*>(a.out) + (p0 + i) * O + at;
                if (at + 4 <= O) o.store(out);
                else
#pragma unroll
                    for (int k = 0; k < 3; ++k)
                        if (at + k < O) out[k] = o.v[k];
            }
        }
        __syncthreads();
    }
}

// dz = dy where y > 0, and db = its sums over each expert's rows: one pass over dy and y, sums over blocks of rows (no block reaching from one
// expert's range into the next) and then over blocks, in a fixed order.  Bound by memory: 65 536 x 1 024 in bfloat16, 403 MB read and written, 80 us
// (5.0 TB/s), and 7 for the second.
// A thread takes N neighbouring columns of every (kBlock >> lg)-th row of the block.
struct SumArgs {
    const int* off;
    const void *y, *dy;
    void *dz, *db;
    float* parts;      // [blocks of rows][columns]; null: no sums
    int64_t n_pos;
    int n_expert, width, first, cols;      // columns first .. first + cols - 1
    int lg, across, rows;                  // lanes across, workgroups across, rows of a block
    int64_t blocks;                        // that there are
};

template <typename T, int N>
__global__ __launch_bounds__(kBlock) void k_unrelu_sums(SumArgs a)
{
    typedef Elements<T, N> Of;
    __shared__ float part[kBlock * N];
    const int64_t t = blockIdx.x / a.across;
    const RowTile r = row_tile(a.off, a.n_expert, a.n_pos, a.rows, t);
    const int lane = threadIdx.x & ((1 << a.lg) - 1), group = threadIdx.x >> a.lg, groups = kBlock >> a.lg;
    // (the last columns reach back into the ones before where they are no whole number: both come to the same values)
    int c = ((int)(blockIdx.x % a.across) << a.lg | lane) * N;
    const bool in = c < a.cols;
    if (c + N > a.cols) c = a.cols - N;
    float sum[N] = {};
    if (in) {
        const int64_t at = a.first + c;
#pragma unroll 2
        for (int64_t p = r.lo + group; p < r.hi; p += groups) {
            Of d = Of::load(static_cast<const T*>(a.dy) + p * a.width + at);
            if (a.y) {
                const Of v = Of::load(static_cast<const T*>(a.y) + p * a.width + at);
#pragma unroll
                for (int n = 0; n < N; ++n) d.v[n] = (float)v.v[n] > 0 ? d.v[n] : (T)0.0f;
                d.store(static_cast<T*>(a.dz) + p * a.width + at);
            }
#pragma unroll
            for (int n = 0; n < N; ++n) sum[n] += (float)d.v[n];
        }
    }
    if (!a.parts || r.expert == a.n_expert) return;
    sum_groups<N>(part, sum, group, groups);
    if (group > 0 || !in) return;
#pragma unroll
    for (int n = 0; n < N; ++n) a.parts[t * a.cols + c + n] = sum[n];
}

// The sums over an expert's blocks: 32 columns a workgroup, eight threads a column.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_sum_blocks(SumArgs a)
{
    __shared__ float part[kBlock];
    const int across = (a.cols + 31) / 32, e = blockIdx.x / across, c = blockIdx.x % across * 32 + threadIdx.x % 32;
    int64_t before, own;
    tiles_before(a.off, a.n_expert, a.n_pos, a.rows, e, before, own);
    if (own > a.blocks - before) own = a.blocks - before;      // (offsets that are none)
    float sum = 0;
    if (c < a.cols)
        for (int64_t t = threadIdx.x / 32; t < own; t += kBlock / 32) sum += a.parts[(before + t) * a.cols + c];
    part[threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.x >= 32 || c >= a.cols) return;
    for (int g = 1; g < kBlock / 32; ++g) sum += part[g * 32 + threadIdx.x];
    static_cast<T*>(a.db)[(int64_t)e * a.width + a.first + c] = (T)sum;
}

int64_t row_tiles(const LinearIn& in, int rows)
{
    return (in.n_pos + rows - 1) / rows + (in.off ? in.n_expert : 0);
}

LinearArgs args_of(const LinearIn& in)
{
    LinearArgs a{};
    a.off = in.off; a.slot = in.n_pos > 0 ? in.slot : nullptr; a.x = in.x; a.w = in.w; a.bias = in.bias; a.n_pos = in.n_pos;
    a.n_expert = in.off ? in.n_expert : 1; a.n_in = in.n_in; a.n_out = in.n_out; a.top_k = in.top_k; a.relu = in.relu;
    while ((int64_t(2) << a.k_shift) <= in.top_k) ++a.k_shift;
    if (in.top_k & (in.top_k - 1)) a.k_mul = (uint32_t)(((uint64_t(1) << (32 + a.k_shift)) + in.top_k - 1) / in.top_k);
    return a;
}

int tiles_of(int width, int tile) { return (width + tile - 1) / tile; }

// Whether rows of both widths are whole 16 bytes, on boundaries of 16.
template <typename T>
bool in_tiles(const LinearIn& in, const void* a, const void* b, const void* c)
{
    return in.n_in % Chunk<T>::n == 0 && in.n_out % Chunk<T>::n == 0 && aligned16(a) && aligned16(b) && aligned16(c);
}

// Which form a product takes.  Times are of nine experts, in bfloat16 where nothing else is said, without the form / with it. Tiles of 256 by 256
// from four rounds of them on, of 128 by 128 before.  Forward, 128 / 256: 8 192 x 4 096 -> 1 024 (165 tiles) 93 / 101 us, 65 536 x 1 024 -> 512
// (530) 85 / 104, 65 536 x 4 096 -> 1 024 (1 060) 607 / 535; by input 65 536 x 1 024 -> 512 (1 060) 111 / 112, 65 536 x 1 024 -> 4 096 (4 240) 703
// / 614.
constexpr int kLargeRounds = 4;
// Few rows: up to 16 an expert on average (32 in single precision), 16 times that in all (an expert may have them all, and its weights are read
// again for every 16).  Nine experts of 4 096 -> 1 024, tiles / this: bfloat16 9 positions 39 / 18 us, 72 39 / 20, 144 39 / 24 (36 where one expert
// has most), 288 38 / 59; single precision 9 125 / 30, 144 123 / 45, 288 125 / 89, 432 128 / 133; bfloat16 from 4 095: 153 77 / 118.
template <typename T>
constexpr int kFewRows = sizeof(T) == 2 ? 16 : 32;
constexpr int kFewExperts = 16;
// By weight, where the tiles are fewer than two rounds: as many parts of the positions as fill those, of at least 1 024 positions each.
// One part / several: 131 072 x 512 -> 128 (36 tiles) 279 / 56 us, 65 536 x 1 024 -> 512 (288) 172 / 137, 16 384 x 1 024 -> 512 50 / 52.
constexpr int kPartRounds = 2, kPartRows = 1024;
// The tiles for any sizes: by weight in parts, of at least 256 positions each, up to eight workgroups to a compute unit.  65 536 x 257 -> 129 590
// / 156 us (both before the loads by four); least 1 024 positions / 256: 2 000 x 768 -> 768, one matrix, single precision 216 / 114, 131 072 x 100
// -> 64 167 / 102; 128 and 512 are slower than 256 there.
constexpr int kAnyEnough = 8 * kUnits, kAnyPartRows = 256;

// Few output features, unless the tiles for 16 bits have one for every compute unit forward.  Tiles / this form, forward 2 000 x 1 024 -> 8 14 / 9
// us, 32 000 x 512 -> 8 11.8 / 10.7, 131 072 x 1 024 -> 8 52 / 56, -> 16 53 / 66; single precision, -> 16, 178 / 132; backward, -> 8 216 / 172, ->
// 16 219 / 257, 32 768 x 4 096 -> 16 241 / 202, 600 x 2 048 -> 8 26 / 30; single precision 481 / 259 and 477 / 296. The products of a layer of few
// output features; false where they are not for these sizes.
template <typename T, Product kProduct>
bool narrow(gr_experts* h, const LinearIn& in, LinearArgs a, hipStream_t s)
{
    if constexpr (kProduct == kForward) {
        k_linear_narrow<T><<<(unsigned)row_tiles(in, 16 * (kBlock / kWave)), kBlock, 0, s>>>(a);
        return true;
    } else {
        constexpr int n = Chunk<T>::n;
        if (in.n_in < n || in.n_pos == 0) return false;
        const int pieces = (in.n_in + n - 1) / n;
        NarrowShape shape{0, 0};
        while ((1 << shape.lg) < pieces && shape.lg < 8) ++shape.lg;
        shape.across = ((pieces - 1) >> shape.lg) + 1;
        // rows of a block: as many as leave four workgroups to each compute unit
        const int64_t enough = in.n_pos * shape.across / (4 * kUnits);
        int64_t rows = enough < kNarrowLeast ? kNarrowLeast : enough > kNarrowRows ? kNarrowRows : enough;
        if constexpr (kProduct == kByWeight) {      // and as there is room for the sums of all blocks
            int64_t most = (int64_t)kPartFloats / ((int64_t)in.n_out * in.n_in) - a.n_expert;
            if (most < kUnits) return false;
            if (most > 4 * kUnits) most = 4 * kUnits;
            if (rows < (in.n_pos + most - 1) / most) rows = (in.n_pos + most - 1) / most;
            a.parts = h->parts;
        }
        const int64_t blocks = row_tiles(in, (int)rows);
        const auto launch = [&](auto out) {
            constexpr int kOut = decltype(out)::value;
            if constexpr (kProduct == kByInput) k_narrow_by_input<T, n, kOut><<<(unsigned)(blocks * shape.across), kBlock, 0, s>>>(a, shape, (int)rows);
            else k_narrow_by_weight<T, n, kOut><<<(unsigned)(blocks * shape.across), kBlock, 0, s>>>(a, shape, (int)rows);
        };
        if (in.n_out == 1) launch(std::integral_constant<int, 1>{});
        else if (in.n_out <= 4) launch(std::integral_constant<int, 4>{});
        else if (in.n_out <= 8) launch(std::integral_constant<int, 8>{});
        else launch(std::integral_constant<int, 16>{});
        if constexpr (kProduct == kByWeight) {
            SumArgs sums{};
            sums.off = in.off; sums.db = a.out; sums.parts = h->parts; sums.n_pos = in.n_pos; sums.n_expert = a.n_expert;
            sums.width = sums.cols = in.n_out * in.n_in; sums.rows = (int)rows; sums.blocks = blocks;
            k_sum_blocks<T><<<a.n_expert * ((sums.cols + 31) / 32), kBlock, 0, s>>>(sums);
        }
        return true;
    }
}

template <typename T, Product kProduct>
void product(gr_experts* h, const LinearIn& in, LinearArgs a, bool tiles, hipStream_t s)
{
    const int width = kProduct == kForward ? in.n_out : in.n_in;
    const auto grid = [&](int size) {
        a.tiles = tiles_of(width, size);
        a.block = a.tiles < 8 ? 8 : 4;
        a.down = kProduct == kByWeight ? (int64_t)a.n_expert * tiles_of(in.n_out, size) * a.parts_n : row_tiles(in, size);
        const int64_t all = a.down * a.tiles, round = all < kDies * kTogether ? kDies : kDies * kTogether;
        return (all + round - 1) / round * round;
    };
    a.parts_n = 1;
    // by weight: where the tiles are few, parts of the positions apart, as many as make up for it
    const int64_t one = (int64_t)a.n_expert * in.n_out * in.n_in;
    const auto cut = [&](int size, int64_t enough, int rows) {
        int64_t parts = enough / grid(size);
        if (parts > (int64_t)kPartFloats / one) parts = (int64_t)kPartFloats / one;
        if (parts > in.n_pos / a.n_expert / rows) parts = in.n_pos / a.n_expert / rows;
        if (kProduct != kByWeight || parts < 2) return false;
        a.parts_n = (int)parts;
        a.parts = h->parts;
        return true;
    };
    const auto join = [&]() {
        if (one % 4 == 0 && reinterpret_cast<uintptr_t>(a.out) % (4 * sizeof(T)) == 0)
            k_join<T, 4><<<(unsigned)((one / 4 + kBlock - 1) / kBlock), kBlock, 0, s>>>(h->parts, a.parts_n, one, static_cast<T*>(a.out));
        else
            k_join<T, 1><<<(unsigned)((one + kBlock - 1) / kBlock), kBlock, 0, s>>>(h->parts, a.parts_n, one, static_cast<T*>(a.out));
    };
    if constexpr (kProduct == kForward) {
        if (in.n_pos <= kFewRows<T> * (a.n_expert < kFewExperts ? a.n_expert : kFewExperts)) {
            a.tiles = tiles_of(width, 16);
            k_linear_few<T><<<(a.n_expert + 1) * a.tiles, kFewWaves * kWave, 0, s>>>(a);
            return;
        }
    }
    const bool whole = kProduct == kForward && sizeof(T) == 2 && tiles && row_tiles(in, 128) >= kUnits;
    if (in.n_out <= kNarrow && !whole && narrow<T, kProduct>(h, in, a, s)) return;
    if constexpr (sizeof(T) == 2) {
        if (tiles) {
            if (grid(256) >= kLargeRounds * kUnits) {
                k_linear_tiles<T, kProduct, 256, false, false><<<kUnits, kWaves * kWave, 0, s>>>(a);
                k_linear_tiles<T, kProduct, 128, false, true><<<2 * kUnits, kWaves * kWave, 0, s>>>(a);
                return;
            }
            if constexpr (kProduct == kByWeight) {
                if (cut(128, 2 * kUnits * kPartRounds, kPartRows)) {
                    const int64_t n = grid(128);
                    k_linear_tiles<T, kProduct, 128, true, false><<<(unsigned)(n < 2 * kUnits ? n : 2 * kUnits), kWaves * kWave, 0, s>>>(a);
                    return join();
                }
            }
            const int64_t n = grid(128);
            k_linear_tiles<T, kProduct, 128, false, false><<<(unsigned)(n < 2 * kUnits ? n : 2 * kUnits), kWaves * kWave, 0, s>>>(a);
            return;
        }
    }
    const bool parts = cut(kAnyTile, kAnyEnough, kAnyPartRows);
    const unsigned n = (unsigned)grid(kAnyTile);
    if (in.n_in >= 4 && in.n_out >= 4) k_linear_any<T, kProduct, 4><<<n, kBlock, 0, s>>>(a);
    else k_linear_any<T, kProduct, 1><<<n, kBlock, 0, s>>>(a);
    if (parts) join();
}

// Whether the smallest tiles of results [positions, width], or of weights, are more than a launch may have.
constexpr int64_t kMostTiles = kMostBlocks - kDies * kTogether;

bool too_many_tiles(const LinearIn& in, int width) { return row_tiles(in, kAnyTile) > kMostTiles / tiles_of(width, kAnyTile); }

bool too_many_weights(const LinearIn& in)
{
    return (int64_t)(in.off ? in.n_expert : 1) * tiles_of(in.n_in, kAnyTile) * tiles_of(in.n_out, kAnyTile) > kMostTiles;
}

// dz and db
template <typename T>
void unrelu_sums(gr_experts* h, const LinearIn& in, void* dz, void* db, hipStream_t s)
{
    constexpr int64_t kMost = 1024;      // blocks of rows, but for what a range does not fill
    SumArgs a{};
    a.off = in.off; a.y = in.y; a.dy = in.dy; a.dz = dz; a.db = db; a.n_pos = in.n_pos;
    a.n_expert = in.off ? in.n_expert : 1; a.width = in.n_out;
    a.rows = in.n_pos > 128 * kMost ? (int)((in.n_pos + kMost - 1) / kMost) : 128;
    const int64_t blocks = a.blocks = row_tiles(in, a.rows) + 1;      // (one more: no positions and no experts leave none)
    const int64_t fit = (int64_t)kPartFloats / blocks / Chunk<T>::n * Chunk<T>::n;
    const int most = fit < in.n_out ? (int)fit : in.n_out;      // columns whose parts there is room for
    for (a.first = 0; a.first < in.n_out; a.first += most) {
        a.cols = in.n_out - a.first < most ? in.n_out - a.first : most;
        a.parts = db ? h->parts : nullptr;
        const bool chunks = a.cols >= Chunk<T>::n;
        const int n = chunks ? Chunk<T>::n : 1, pieces = (a.cols + n - 1) / n;
        a.lg = 0;
        while ((1 << a.lg) < pieces && a.lg < 5) ++a.lg;
        a.across = ((pieces - 1) >> a.lg) + 1;
        if (in.n_pos > 0) {
            if (chunks) k_unrelu_sums<T, Chunk<T>::n><<<blocks * a.across, kBlock, 0, s>>>(a);
            else k_unrelu_sums<T, 1><<<blocks * a.across, kBlock, 0, s>>>(a);
        }
        if (db) k_sum_blocks<T><<<a.n_expert * ((a.cols + 31) / 32), kBlock, 0, s>>>(a);
    }
}

}  // namespace

int launch_linear(gr_experts* h, const LinearIn& in, int dtype, void* out_y, hipStream_t s)
{
    if (too_many_tiles(in, in.n_out)) return GR_ERR_TOO_LARGE;
    LinearArgs a = args_of(in);
    a.out = out_y;
    return by_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        product<T, kForward>(h, in, a, in_tiles<T>(in, in.x, in.w, out_y), s);
        return launched();
    });
}

int launch_linear_backward(gr_experts* h, const LinearIn& in, int dtype, void* dz, void* dx, void* dw, void* db, hipStream_t s)
{
    if ((dx && too_many_tiles(in, in.n_in)) || (dw && too_many_weights(in))) return GR_ERR_TOO_LARGE;
    return by_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        LinearArgs a = args_of(in);
        a.dz = in.dy;
        if (db || (in.y && in.n_pos > 0)) unrelu_sums<T>(h, in, dz, db, s);
        if (in.y) a.dz = dz;
        if (dx && in.n_pos > 0) {
            a.out = dx;
            product<T, kByInput>(h, in, a, in_tiles<T>(in, a.dz, in.w, dx), s);
        }
        if (dw) {
            a.out = dw;
            product<T, kByWeight>(h, in, a, in_tiles<T>(in, a.dz, in.x, dw), s);
        }
        return launched();
    });
}

}  // namespace gr
