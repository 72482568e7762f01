// One layer of every expert on the rows that chose it, and its gradients (gfx950).
//
// Three products of matrices whose rows are cut into ranges by expert:
//   forward   y[p, n]  = sum over k of x[row(p), k] * W_e[n, k]        p in the range of e
//   by input  dx[p, k] = sum over n of dz[p, n] * W_e[n, k]            p in the range of e
//   by weight dW_e[n, k] = sum over p in the range of e of dz[p, n] * x[row(p), k]
#include "experts.h"

namespace gr {
namespace {

constexpr int kBlock = 256;
constexpr int kWave = 64;

enum Product { kForward = 0, kByInput, kByWeight };

struct LinearArgs {
    const int *off, *slot;
    const void *x, *w, *bias, *dz;
    void *out, *db;
    int64_t n_pos;
    int n_expert, n_in, n_out, top_k, relu;
    int tiles;      // in the direction of columns
};

// Bounds of a range, whatever the offsets hold.
__device__ __forceinline__ int64_t bound(const int* off, int e, int n_expert, int64_t n_pos)
{
    if (!off) return e == 0 ? 0 : n_pos;
    const int64_t v = off[e];
    return v < 0 ? 0 : v > n_pos ? n_pos : v;
}

__device__ __forceinline__ int64_t row_of(const LinearArgs& a, int64_t p)
{
    if (!a.slot) return p;
    int64_t s = a.slot[p];
    if (s < 0) s = -1 - s;
    if (s >= a.n_pos) s = a.n_pos - 1;
    return s / a.top_k;
}

// A block of rows of the output: an expert (n_expert: rows without one) and positions lo .. hi - 1.
struct RowTile {
    int expert;
    int64_t lo, hi;
};

// The t-th tile of kRows rows, no tile reaching from one expert's range into the next; lo = hi where there are fewer.
// Every lane of a wave calls it.
template <int kRows>
__device__ __forceinline__ RowTile row_tile(const LinearArgs& a, int64_t t)
{
    const int lane = threadIdx.x % kWave;
    int64_t before = 0;
    for (int e0 = 0; e0 <= a.n_expert; e0 += kWave) {
        const int e = e0 + lane;
        int64_t lo = 0, hi = 0;
        if (e <= a.n_expert) {
            lo = bound(a.off, e, a.n_expert, a.n_pos);
            hi = e < a.n_expert ? bound(a.off, e + 1, a.n_expert, a.n_pos) : a.n_pos;
        }
        const int own = hi > lo ? (int)((hi - lo + kRows - 1) / kRows) : 0;
        int v = own;
        for (int d = 1; d < kWave; d *= 2) {
            const int o = __shfl_up(v, d);
            if (lane >= d) v += o;
        }
        const int64_t end = before + v;
        const unsigned long long mine = __ballot(t >= end - own && t < end);
        if (mine) {
            const int l = __ffsll((long long)mine) - 1;
            const int64_t first = __shfl(lo, l) + (t - (__shfl(end, l) - __shfl(own, l))) * kRows;
            const int64_t last = __shfl(hi, l);
            return {e0 + l, first, first + kRows < last ? first + kRows : last};
        }
        before = __shfl(end, kWave - 1);
    }
    return {a.n_expert, 0, 0};
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
// Tiles of 128 rows by 128 columns, 64 bytes of the reduction at a time, loaded element by element into registers while the
// tile before is multiplied, and laid into shared memory with the reduction contiguous.

constexpr int kAnyTile = 128;

template <typename T>
constexpr int kAnyDepth = 64 / sizeof(T);

template <typename T, Product kProduct>
__global__ __launch_bounds__(kBlock) void k_linear_any(LinearArgs a)
{
    constexpr int D = kAnyDepth<T>, kLd = D + Chunk<T>::n, kPer = kAnyTile * D / kBlock;
    typedef typename Chunk<T>::Vec Vec;
    constexpr int n = Chunk<T>::n;
    __shared__ __attribute__((aligned(16))) T lds_p[kAnyTile * kLd], lds_q[kAnyTile * kLd];

    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const int col_tile = blockIdx.x % a.tiles;
    const int64_t row_no = blockIdx.x / a.tiles;
    const T* const x = static_cast<const T*>(a.x);
    const T* const dz = static_cast<const T*>(a.dz);
    const int I = a.n_in, O = a.n_out;

    // the output's rows p0 .. p0 + p_n - 1 (positions, or output features of an expert), columns q0 .. q0 + q_n - 1
    int e;
    int64_t p0, lo = 0, depth;
    int p_n, q0 = col_tile * kAnyTile, q_n;
    if constexpr (kProduct == kByWeight) {
        const int tiles = (O + kAnyTile - 1) / kAnyTile;
        e = (int)(row_no / tiles);
        p0 = (row_no - (int64_t)e * tiles) * kAnyTile;
        p_n = O - p0 < kAnyTile ? (int)(O - p0) : kAnyTile;
        q_n = I - q0 < kAnyTile ? I - q0 : kAnyTile;
        lo = bound(a.off, e, a.n_expert, a.n_pos);
        depth = bound(a.off, e + 1, a.n_expert, a.n_pos) - lo;
    } else {
        const RowTile t = row_tile<kAnyTile>(a, row_no);
        if (t.hi <= t.lo) return;
        e = t.expert;
        p0 = t.lo;
        p_n = (int)(t.hi - t.lo);
        const int width = kProduct == kForward ? O : I;
        q_n = width - q0 < kAnyTile ? width - q0 : kAnyTile;
        depth = e == a.n_expert ? 0 : kProduct == kForward ? I : O;
    }
    const T* const w = static_cast<const T*>(a.w) + (kProduct == kByWeight || e == a.n_expert ? 0 : (int64_t)e * O * I);

    // which of the tile's elements a thread loads: kPer of each operand, along the direction that is contiguous in memory
    constexpr bool kPLong = kProduct != kByWeight, kQLong = kProduct == kForward;      // that is the reduction's
    const auto place = [&](bool along, int i, int& row, int& r) {
        const int at = i * kBlock + tid;
        if (along) { row = at / D; r = at % D; }
        else { r = at / kAnyTile; row = at % kAnyTile; }
    };
    int64_t p_row[kPer];      // where the rows of the left operand start
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        int row, r;
        place(kPLong, i, row, r);
        p_row[i] = 0;
        if (kProduct == kForward && row < p_n && e < a.n_expert) p_row[i] = row_of(a, p0 + row) * I;
        if (kProduct == kByInput) p_row[i] = (p0 + row) * O;
    }
    T get_p[kPer], get_q[kPer];
    const auto load = [&](int64_t r0) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            int row, r;
            place(kPLong, i, row, r);
            const bool in = row < p_n && r0 + r < depth;
            get_p[i] = (T)0.0f;
            if (in) get_p[i] = kProduct == kForward ? x[p_row[i] + r0 + r] : kProduct == kByInput ? dz[p_row[i] + r0 + r] : dz[(lo + r0 + r) * O + p0 + row];
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            int row, r;
            place(kQLong, i, row, r);
            const bool in = row < q_n && r0 + r < depth;
            get_q[i] = (T)0.0f;
            if (in) get_q[i] = kProduct == kForward ? w[(int64_t)(q0 + row) * I + r0 + r] : kProduct == kByInput ? w[(r0 + r) * I + q0 + row] : x[row_of(a, lo + r0 + r) * I + q0 + row];
        }
    };

    f32x4 acc[4][4] = {};
    float db = 0;
    const bool sums = kProduct == kByWeight && a.db && col_tile == 0;
    const int wp = (wave / 2) * 64, wq = (wave % 2) * 64;      // a wave's 64 by 64
    if (depth > 0) load(0);
    for (int64_t r0 = 0; r0 < depth; r0 += D) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            int row, r;
            place(kPLong, i, row, r);
            lds_p[row * kLd + r] = get_p[i];
            place(kQLong, i, row, r);
            lds_q[row * kLd + r] = get_q[i];
        }
        __syncthreads();
        if (r0 + D < depth) load(r0 + D);
        Vec p[4], q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[i] = *reinterpret_cast<const Vec*>(&lds_p[(wp + i * 16 + lane % 16) * kLd + lane / 16 * n]);
            q[i] = *reinterpret_cast<const Vec*>(&lds_q[(wq + i * 16 + lane % 16) * kLd + lane / 16 * n]);
        }
        // (columns as the first operand: a lane then holds four neighbours of a row)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = mfma(q[j], p[i], acc[i][j]);
        if (sums && tid < p_n)
            for (int r = 0; r < D; ++r) db += (float)lds_p[tid * kLd + r];
    }
    if (sums && tid < p_n) static_cast<T*>(a.db)[(int64_t)e * O + p0 + tid] = (T)db;

    if (kProduct == kByWeight && !a.out) return;      // (sums of dz alone)
    const int width = kProduct == kForward ? O : I;
    T* const out = static_cast<T*>(a.out) + ((kProduct == kByWeight ? (int64_t)e * O : 0) + p0) * width + q0;
    const T* const bias = kProduct == kForward && a.bias && e < a.n_expert ? static_cast<const T*>(a.bias) + (int64_t)e * O + q0 : nullptr;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = wp + i * 16 + lane % 16;
        if (row >= p_n) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int col = wq + j * 16 + lane / 16 * 4 + k;
                if (col >= q_n) continue;
                float v = acc[i][j][k] + (bias ? (float)bias[col] : 0.0f);
                if (kProduct == kForward && a.relu && v < 0) v = 0;
                out[(int64_t)row * width + col] = (T)v;
            }
    }
}

// ---- 16-bit types, rows of whole 16 bytes -------------------------------------------------------
//
// Tiles of kRows by kCols, 64 reduction indexes at a time, that go from memory straight into shared memory (two tiles in turn: one
// is filled while the other is multiplied).  An operand lies there as it does in memory:
//   long    its reduction is contiguous: [row][64 indexes]; a lane's eight indexes are one read of 16 bytes
//   across  its rows are contiguous: [64 indexes][row]; a lane's eight indexes are two reads that transpose 4 by 16
// What is written is one after the other, 16 bytes a lane, so which 16 bytes of memory a lane fetches decides the layout: their number
// within a row is exclusive-ored with one made of the row's, so that the lanes of a read meet no bank twice.

constexpr int kDepth = 64;

__device__ const uint4 kZeros = {0, 0, 0, 0};      // where lanes read that are past the end of the reduction

typedef __attribute__((address_space(3))) char LdsChar;
typedef const __attribute__((address_space(1))) char GlobalChar;

__device__ __forceinline__ void fetch16(const void* from, char* to)
{
    const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(LdsChar*)to);
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(at) : "memory");
}

__device__ __forceinline__ int across_swizzle(int r) { return (r & 3) << 1 | (r >> 3 & 1) << 3; }

// A lane's part of a fragment of 16 rows (or columns) by 32 indexes.
template <typename T, bool kLong, int kSize>
__device__ __forceinline__ typename Chunk<T>::Vec fragment(const char* tile, int first, int half, int lane)
{
    typedef typename Chunk<T>::Vec Vec;
    const int g = lane / 16, i = lane % 16;
    if constexpr (kLong) {
        const int row = first + i;
        return *reinterpret_cast<const Vec*>(tile + row * (kDepth * 2) + ((half * 4 + g) ^ (row & 7)) * 16);
    } else {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 Lds4;
        union { s16x4 part[2]; Vec all; } v;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = half * 32 + g * 8 + h * 4 + i / 4;
            const int chunk = (first / 8 + i % 4 / 2) ^ across_swizzle(r);
            v.part[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4*)(tile + r * (kSize * 2) + chunk * 16 + i % 2 * 8));
        }
        return v.all;
    }
}

// Where a lane fetches its share of an operand's tiles from, one tile of the reduction after the other.
template <typename T, bool kLong, int kSize, int kWaves>
struct Source {
    static constexpr int kLoads = kSize * kDepth * 2 / 1024 / kWaves;      // of a wave, 1 KB each
    static constexpr int kPerRow = kSize / 8;                              // across: pieces of 16 bytes
    const char* at[kLoads];
    int64_t step;      // bytes from one tile to the next

    // The number within the tile of what load i of a lane brings: across its index, long its row; and its piece of 16 bytes.
    static __device__ __forceinline__ int line(int i, int wave, int lane)
    {
        const int no = (wave * kLoads + i) * kWave + lane;
        return kLong ? no / 8 : no / kPerRow;
    }
    static __device__ __forceinline__ int piece(int i, int wave, int lane)
    {
        const int no = (wave * kLoads + i) * kWave + lane;
        return kLong ? no % 8 ^ (no / 8 & 7) : no % kPerRow ^ across_swizzle(no / kPerRow);
    }

    // left: indexes of the reduction from this tile on
    __device__ __forceinline__ void fetch(char* tile, int64_t left, int wave, int lane)
    {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const char* from = at[i];
            if (left < kDepth && (kLong ? piece(i, wave, lane) * 8 : line(i, wave, lane)) >= left) from = reinterpret_cast<const char*>(&kZeros);
            fetch16(from, tile + (wave * kLoads + i) * 1024);
            at[i] += step;
        }
    }
};

template <typename T, Product kProduct, int kRows, int kCols, int kWavesP, int kWavesQ>
__global__ __launch_bounds__(kWavesP * kWavesQ * kWave, kWavesP * kWavesQ / 4) void k_linear_tiles(LinearArgs a)
{
    constexpr int kWaves = kWavesP * kWavesQ, kP = kRows / kWavesP / 16, kQ = kCols / kWavesQ / 16;      // fragments of a wave
    constexpr bool kPLong = kProduct != kByWeight, kQLong = kProduct == kForward;
    constexpr int kPBytes = kRows * kDepth * 2, kBytes = (kRows + kCols) * kDepth * 2;
    typedef typename Chunk<T>::Vec Vec;
    __shared__ __attribute__((aligned(1024))) char lds[2 * kBytes];

    const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const T* const x = static_cast<const T*>(a.x);
    const T* const dz = static_cast<const T*>(a.dz);
    const int I = a.n_in, O = a.n_out;

    const int col_tile = blockIdx.x % a.tiles;
    const int64_t row_no = blockIdx.x / a.tiles;
    int e;
    int64_t p0, lo = 0, depth;
    int p_n, q0 = col_tile * kCols, q_n;
    if constexpr (kProduct == kByWeight) {
        const int tiles = (O + kRows - 1) / kRows;
        e = (int)(row_no / tiles);
        p0 = (row_no - (int64_t)e * tiles) * kRows;
        p_n = O - p0 < kRows ? (int)(O - p0) : kRows;
        q_n = I - q0 < kCols ? I - q0 : kCols;
        lo = bound(a.off, e, a.n_expert, a.n_pos);
        depth = bound(a.off, e + 1, a.n_expert, a.n_pos) - lo;
    } else {
        const RowTile t = row_tile<kRows>(a, row_no);
        if (t.hi <= t.lo) return;
        e = t.expert;
        p0 = t.lo;
        p_n = (int)(t.hi - t.lo);
        const int width = kProduct == kForward ? O : I;
        q_n = width - q0 < kCols ? width - q0 : kCols;
        depth = e == a.n_expert ? 0 : kProduct == kForward ? I : O;
    }
    const T* const w = static_cast<const T*>(a.w) + (kProduct == kByWeight || e == a.n_expert ? 0 : (int64_t)e * O * I);

    // (rows and columns past the edge are fetched from within it: what becomes of them is not stored)
    Source<T, kPLong, kRows, kWaves> from_p;
    Source<T, kQLong, kCols, kWaves> from_q;
#pragma unroll
    for (int i = 0; i < from_p.kLoads; ++i) {
        const int line = from_p.line(i, wave, lane), piece = from_p.piece(i, wave, lane);
        const T* at;
        if constexpr (kPLong) {
            const int64_t p = p0 + (line < p_n ? line : p_n - 1);
            at = (kProduct == kForward ? x + (e < a.n_expert ? row_of(a, p) : 0) * I : dz + p * O) + piece * 8;
        } else {
            at = dz + (lo + line) * O + p0 + (piece * 8 < p_n ? piece * 8 : 0);
        }
        from_p.at[i] = reinterpret_cast<const char*>(at);
    }
    from_p.step = kPLong ? kDepth * 2 : (int64_t)kDepth * 2 * O;
    int64_t next[from_q.kLoads];      // by weight: rows of x of the next tile
#pragma unroll
    for (int i = 0; i < from_q.kLoads; ++i) {
        const int line = from_q.line(i, wave, lane), piece = from_q.piece(i, wave, lane);
        const T* at;
        if constexpr (kQLong) at = w + (int64_t)(q0 + (line < q_n ? line : q_n - 1)) * I + piece * 8;
        else at = (kProduct == kByInput ? w + (int64_t)line * I : x) + q0 + (piece * 8 < q_n ? piece * 8 : 0);
        from_q.at[i] = reinterpret_cast<const char*>(at);
    }
    from_q.step = kQLong ? kDepth * 2 : kProduct == kByInput ? (int64_t)kDepth * 2 * I : 0;
    const auto look_up = [&](int64_t r0) {
#pragma unroll
        for (int i = 0; i < from_q.kLoads; ++i) {
            const int64_t r = r0 + from_q.line(i, wave, lane);
            next[i] = r < depth ? row_of(a, lo + r) * I * 2 : 0;
        }
    };
    const auto fetch = [&](int64_t r0, char* to) {
        from_p.fetch(to, depth - r0, wave, lane);
        if constexpr (kProduct == kByWeight) {
            Source<T, kQLong, kCols, kWaves> now = from_q;
#pragma unroll
            for (int i = 0; i < from_q.kLoads; ++i) now.at[i] += next[i];
            now.fetch(to + kPBytes, depth - r0, wave, lane);
            look_up(r0 + kDepth);
        } else {
            from_q.fetch(to + kPBytes, depth - r0, wave, lane);
        }
    };

    f32x4 acc[kP][kQ] = {};
    const int wp = wave / kWavesQ * (kP * 16), wq = wave % kWavesQ * (kQ * 16);
    if (depth > 0) {
        if constexpr (kProduct == kByWeight) look_up(0);
        fetch(0, lds);
    }
    int turn = 0;
    for (int64_t r0 = 0; r0 < depth; r0 += kDepth, turn ^= 1) {
        // this tile is there, and the one before has been read
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (r0 + kDepth < depth) fetch(r0 + kDepth, lds + (turn ^ 1) * kBytes);
        const char* const tile = lds + turn * kBytes;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            Vec p[kP], q[kQ];
#pragma unroll
            for (int j = 0; j < kQ; ++j) q[j] = fragment<T, kQLong, kCols>(tile + kPBytes, wq + j * 16, half, lane);
#pragma unroll
            for (int i = 0; i < kP; ++i) p[i] = fragment<T, kPLong, kRows>(tile, wp + i * 16, half, lane);
#pragma unroll
            for (int i = 0; i < kP; ++i)
#pragma unroll
                for (int j = 0; j < kQ; ++j) acc[i][j] = mfma(q[j], p[i], acc[i][j]);
        }
    }

    const int width = kProduct == kForward ? O : I;
    T* const out = static_cast<T*>(a.out) + ((kProduct == kByWeight ? (int64_t)e * O : 0) + p0) * width + q0;
    const T* const bias = kProduct == kForward && a.bias && e < a.n_expert ? static_cast<const T*>(a.bias) + (int64_t)e * O + q0 : nullptr;
    typedef T Four __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int j = 0; j < kQ; ++j) {
        const int col = wq + j * 16 + lane / 16 * 4;
        if (col >= q_n) continue;
        float b[4] = {};
        if (bias)
#pragma unroll
            for (int k = 0; k < 4; ++k) b[k] = (float)bias[col + k];
#pragma unroll
        for (int i = 0; i < kP; ++i) {
            const int row = wp + i * 16 + lane % 16;
            if (row >= p_n) continue;
            Four o;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float v = acc[i][j][k] + b[k];
                if (kProduct == kForward && a.relu && v < 0) v = 0;
                o[k] = (T)v;
            }
            *reinterpret_cast<Four*>(out + (int64_t)row * width + col) = o;
        }
    }
}

// dz = dy where y > 0; rows without an expert are rows as any other (no product reads them).
template <typename T>
__global__ __launch_bounds__(kBlock) void k_unrelu(const T* y, const T* dy, T* dz, int64_t count, int64_t chunks)
{
    typedef typename Chunk<T>::Vec Vec;
    constexpr int n = Chunk<T>::n;
    const int64_t stride = (int64_t)gridDim.x * kBlock, from = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    for (int64_t i = from; i < chunks; i += stride) {
        const Vec v = reinterpret_cast<const Vec*>(y)[i];
        Vec d = reinterpret_cast<const Vec*>(dy)[i];
#pragma unroll
        for (int j = 0; j < n; ++j) d[j] = (float)v[j] > 0 ? d[j] : (T)0.0f;
        reinterpret_cast<Vec*>(dz)[i] = d;
    }
    for (int64_t i = chunks * n + from; i < count; i += stride) dz[i] = (float)y[i] > 0 ? dy[i] : (T)0.0f;
}

int64_t row_tiles(const LinearIn& in, int rows)
{
    return (in.n_pos + rows - 1) / rows + (in.off ? in.n_expert : 0);
}

LinearArgs args_of(const LinearIn& in)
{
    LinearArgs a{};
    a.off = in.off; a.slot = in.slot; a.x = in.x; a.w = in.w; a.bias = in.bias; a.n_pos = in.n_pos;
    a.n_expert = in.off ? in.n_expert : 1; a.n_in = in.n_in; a.n_out = in.n_out; a.top_k = in.top_k; a.relu = in.relu;
    return a;
}

int tiles_of(int width, int tile) { return (width + tile - 1) / tile; }

// Whether rows of both widths are whole 16 bytes, on boundaries of 16.
template <typename T>
bool in_tiles(const LinearIn& in, const void* a, const void* b, const void* c)
{
    return sizeof(T) == 2 && in.n_in % 8 == 0 && in.n_out % 8 == 0 && aligned16(a) && aligned16(b) && aligned16(c);
}

template <typename T, Product kProduct>
void product(const LinearIn& in, LinearArgs a, bool tiles, hipStream_t s)
{
    constexpr int kRows = 256, kCols = 256;
    const int width = kProduct == kForward ? in.n_out : in.n_in;
    const auto grid = [&](int rows, int cols) {
        a.tiles = tiles_of(width, cols);
        const int64_t down = kProduct == kByWeight ? (int64_t)a.n_expert * tiles_of(in.n_out, rows) : row_tiles(in, rows);
        return (unsigned)(down * a.tiles);
    };
    if constexpr (sizeof(T) == 2) {
        if (tiles) {
            const unsigned n = grid(kRows, kCols);
            k_linear_tiles<T, kProduct, kRows, kCols, 2, 4><<<n, 512, 0, s>>>(a);
            return;
        }
    }
    const unsigned n = grid(kAnyTile, kAnyTile);
    k_linear_any<T, kProduct><<<n, kBlock, 0, s>>>(a);
}

}  // namespace

int launch_linear(gr_experts*, const LinearIn& in, int dtype, void* out_y, hipStream_t s)
{
    LinearArgs a = args_of(in);
    a.out = out_y;
    return by_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        product<T, kForward>(in, a, in_tiles<T>(in, in.x, in.w, out_y), s);
        return launched();
    });
}

int launch_linear_backward(gr_experts*, const LinearIn& in, int dtype, void* dz, void* dx, void* dw, void* db, hipStream_t s)
{
    return by_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        LinearArgs a = args_of(in);
        a.dz = in.dy;
        if (in.y && in.n_pos > 0) {
            const int64_t count = in.n_pos * in.n_out;
            const int64_t chunks = aligned16(in.y) && aligned16(in.dy) && aligned16(dz) ? count / Chunk<T>::n : 0;
            const int64_t blocks = ((chunks ? chunks : count) + kBlock - 1) / kBlock;
            k_unrelu<T><<<blocks < 4096 ? blocks : 4096, kBlock, 0, s>>>(static_cast<const T*>(in.y), static_cast<const T*>(in.dy),
                                                                         static_cast<T*>(dz), count, chunks);
            a.dz = dz;
        }
        if (dx && in.n_pos > 0) {
            a.out = dx;
            product<T, kByInput>(in, a, in_tiles<T>(in, a.dz, in.w, dx), s);
        }
        if (dw || db) {
            a.out = dw;
            a.db = db;
            const bool tiles = dw && in_tiles<T>(in, a.dz, in.x, dw);
            if (tiles) {
                product<T, kByWeight>(in, a, true, s);
                a.out = nullptr;
            }
            if (!tiles || db) {
                a.tiles = a.out ? tiles_of(in.n_in, kAnyTile) : 1;
                k_linear_any<T, kByWeight><<<(int64_t)a.n_expert * tiles_of(in.n_out, kAnyTile) * a.tiles, kBlock, 0, s>>>(a);
            }
        }
        return launched();
    });
}

}  // namespace gr
