// The global norm of many gradients, and clipping by it (gfx950).
//
//   norm = sqrt(sum of g^2 over all elements of all gradients),  out = g * min(1, max_norm / norm)
//
// Bound by memory: two reads and a write of every gradient, the second read from the cache where all fit it (256 MB).  The norm has to be known
// before anything is written, so there are two launches: one for the sums of workgroups, one whose workgroups all add those up (in one order, so all
// come to the same norm) and scale.  20 gradients, 45 million elements in bfloat16 (90 MB): the sums 16.5 us (5.5 TB/s), scaling 30 (180 MB at
// 6 TB/s), 56 us in all with the launches; 60 gradients, 60 million in single precision (240 MB) 167 us.
//
// Squares are summed in double precision: they cannot overflow there, and the order of a sum shows in no digit that is kept.
#include "experts.h"

namespace gr {
namespace {

constexpr int kBlock = 256;
constexpr int kWave = 64;
// Few gradients go in one launch (k_clip_few).  One launch / two, single precision, results apart: 3 gradients of 240 KB in all 7.4 / 9.9 us, of
// 520 KB 10.2 / 11, of 1 MB 13 / 10; 9 of 32 KB 7.4 / 7.6, 12 of 64 KB 9.5 / 8.2, 40 of 80 KB 21 / 12.  In place, where one workgroup does it: 3
// of 32 KB 7.0 / 8.5, of 64 KB 9.7 / 7.4; 9 of 32 KB 13.8 / 7.9.
constexpr int kFewThreads = 1024, kFewTensors = 8, kAloneTensors = 4;
constexpr int64_t kFewBytes = 512 << 10, kAloneBytes = 32 << 10;
constexpr int kPiece = kBlock * 4 * 16;      // bytes of a gradient that a workgroup takes at a time

struct ClipTable {
    const void* grad[kClipTensors];
    void* out[kClipTensors];
    int64_t count_type[kClipTensors];      // 4 * elements + type
    int pieces_before[kClipTensors + 1];
    int n;
};

struct Piece {
    const char* grad;
    char* out;
    int64_t bytes;
    int type;
};

__device__ __forceinline__ Piece piece_of(const ClipTable& t, int at)
{
    int lo = 0, hi = t.n - 1;      // the last gradient that starts at or before the piece
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (t.pieces_before[mid] <= at) lo = mid;
        else hi = mid - 1;
    }
    const int type = (int)(t.count_type[lo] & 3);
    const int64_t bytes = (t.count_type[lo] >> 2) * (type == GR_F32 ? 4 : 2), from = (int64_t)(at - t.pieces_before[lo]) * kPiece;
    return {static_cast<const char*>(t.grad[lo]) + from, static_cast<char*>(t.out[lo]) + from, bytes - from < kPiece ? bytes - from : kPiece, type};
}

// `f` of every element of a piece: of chunks of 16 bytes where both sides allow, of single ones else and behind
template <typename T, typename F, typename G>
__device__ __forceinline__ void each(const Piece& p, bool aligned, F chunk, G one)
{
    const int count = (int)(p.bytes / sizeof(T)), chunks = aligned ? count / Chunk<T>::n : 0;
#pragma unroll 4
    for (int i = threadIdx.x; i < chunks; i += blockDim.x) chunk(i);
    for (int i = chunks * Chunk<T>::n + threadIdx.x; i < count; i += blockDim.x) one(i);
}

template <typename T>
__device__ __forceinline__ double squares_of(const Piece& p)
{
    typedef typename Chunk<T>::Vec Vec;
    const T* const g = reinterpret_cast<const T*>(p.grad);
    double sum = 0;
    const auto add = [&](T v) { sum = fma((double)(float)v, (double)(float)v, sum); };
    each<T>(p, reinterpret_cast<uintptr_t>(g) % 16 == 0,
            [&](int i) {
                const Vec v = reinterpret_cast<const Vec*>(g)[i];
#pragma unroll
                for (int j = 0; j < Chunk<T>::n; ++j) add(v[j]);
            },
            [&](int i) { add(g[i]); });
    return sum;
}

// `by`(an element) of each.
template <typename T, typename F>
__device__ __forceinline__ void scale(const Piece& p, F by)
{
    typedef typename Chunk<T>::Vec Vec;
    const T* const g = reinterpret_cast<const T*>(p.grad);
    T* const o = reinterpret_cast<T*>(p.out);
    each<T>(p, reinterpret_cast<uintptr_t>(g) % 16 == 0 && reinterpret_cast<uintptr_t>(o) % 16 == 0,
            [&](int i) {
                Vec v = reinterpret_cast<const Vec*>(g)[i];
#pragma unroll
                for (int j = 0; j < Chunk<T>::n; ++j) v[j] = (T)by((float)v[j]);
                reinterpret_cast<Vec*>(o)[i] = v;
            },
            [&](int i) { o[i] = (T)by((float)g[i]); });
}

// The workgroup's sum, in thread 0.
template <int kThreads>
__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double part[kThreads / kWave];
    for (int m = 1; m < kWave; m *= 2) v += __shfl_xor(v, m);
    if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = v;
    __syncthreads();
    for (int w = 1; w < kThreads / kWave; ++w) v += threadIdx.x == 0 ? part[w] : 0.0;
    return v;
}

__device__ __forceinline__ double squares_of(const Piece& p, int)
{
    return p.type == GR_F32 ? squares_of<float>(p) : p.type == GR_BF16 ? squares_of<bf16>(p) : squares_of<f16>(p);
}

template <typename F>
__device__ __forceinline__ void scale(const Piece& p, F by, int)
{
    if (p.type == GR_F32) scale<float>(p, by);
    else if (p.type == GR_BF16) scale<bf16>(p, by);
    else scale<f16>(p, by);
}

// What gradients are multiplied by.
__device__ __forceinline__ double factor(double norm, double max_norm)
{
    return norm > max_norm && norm < __builtin_inf() ? max_norm / norm : 1.0;
}

// A factor that single precision holds whole is one of single precision; with a smaller one (gradients near the end of their range, clipped to
// little) products are in double precision, as the results may well be whole.
constexpr float kLeastFactor = 0x1p-126f;

__device__ __forceinline__ void scale(const Piece& p, double by)
{
    const float f = (float)by;
    if (f >= kLeastFactor || by == 0) scale(p, [f](float v) { return v * f; }, 0);
    else scale(p, [by](float v) { return (float)((double)v * by); }, 0);
}

__global__ __launch_bounds__(kBlock) void k_norm(ClipTable t, double* squares)
{
    double sum = 0;
    for (int at = blockIdx.x; at < t.pieces_before[t.n]; at += gridDim.x) {
        const Piece p = piece_of(t, at);
        sum += squares_of(p, 0);
    }
    sum = block_sum<kBlock>(sum);
    if (threadIdx.x == 0) squares[blockIdx.x] = sum;
}

__global__ __launch_bounds__(kBlock) void k_clip(ClipTable t, const double* squares, int parts, double max_norm, float* norm)
{
    __shared__ double by;
    double sum = 0;
    for (int i = threadIdx.x; i < parts; i += kBlock) sum += squares[i];
    sum = block_sum<kBlock>(sum);
    if (threadIdx.x == 0) {
        const double all = sqrt(sum);
        by = factor(all, max_norm);
        if (norm && blockIdx.x == 0) *norm = (float)all;
    }
    __syncthreads();
    const double f = by;
    for (int at = blockIdx.x; at < t.pieces_before[t.n]; at += gridDim.x) {
        const Piece p = piece_of(t, at);
        if ((float)f == 1.0f && p.grad == p.out) continue;
        scale(p, f);
    }
}

// Little enough that every workgroup reads all of it, and one launch does: the same sum in each, and a share of the pieces.
__global__ __launch_bounds__(kFewThreads) void k_clip_few(ClipTable t, double max_norm, float* norm)
{
    __shared__ double by;
    double sum = 0;
    for (int i = 0; i < t.n; ++i) {
        const int type = (int)(t.count_type[i] & 3);
        sum += squares_of(Piece{static_cast<const char*>(t.grad[i]), nullptr, (t.count_type[i] >> 2) * (type == GR_F32 ? 4 : 2), type}, 0);
    }
    sum = block_sum<kFewThreads>(sum);
    if (threadIdx.x == 0) {
        const double all = sqrt(sum);
        by = factor(all, max_norm);
        if (norm && blockIdx.x == 0) *norm = (float)all;
    }
    __syncthreads();
    const double f = by;
    for (int at = blockIdx.x; at < t.pieces_before[t.n]; at += gridDim.x) scale(piece_of(t, at), f);
}

}  // namespace

int launch_clip(gr_experts* h, int n, const void* const* grad, void* const* out, const int64_t* count, const int* dtype,
                float max_norm, float* norm, hipStream_t s)
{
    // a table for each launch, made anew for either pass
    const auto each_table = [&](auto launch) -> int {
        int parts = 0, i = 0;
        do {
            ClipTable t{};
            while (i < n && t.n < kClipTensors) {
                const int64_t pieces = (count[i] * (int64_t)size_of(dtype[i]) + kPiece - 1) / kPiece;
                if (pieces > INT32_MAX - t.pieces_before[t.n]) { if (t.n == 0) return GR_ERR_TOO_LARGE; break; }
                t.grad[t.n] = grad[i]; t.out[t.n] = out[i]; t.count_type[t.n] = count[i] * 4 + dtype[i];
                t.pieces_before[t.n + 1] = t.pieces_before[t.n] + (int)pieces;
                ++t.n;
                ++i;
            }
            const int blocks = t.pieces_before[t.n] < 1 ? 1 : t.pieces_before[t.n] < kClipBlocks ? t.pieces_before[t.n] : kClipBlocks;
            if ((size_t)(parts + blocks) > kClipParts) return GR_ERR_TOO_LARGE;
            launch(t, blocks, parts);
            parts += blocks;
        } while (i < n);
        return parts;
    };
    int64_t bytes = 0;
    bool apart = true;      // (a workgroup may be done while another still reads: in place only one may do all)
    for (int i = 0; i < n && bytes <= kFewBytes; ++i) {
        bytes += count[i] * (int64_t)size_of(dtype[i]);
        apart = apart && (out[i] != grad[i] || count[i] == 0);
    }
    if (n <= (apart ? kFewTensors : kAloneTensors) && bytes <= (apart ? kFewBytes : kAloneBytes)) {
        each_table([&](const ClipTable& t, int blocks, int) { k_clip_few<<<apart ? blocks : 1, kFewThreads, 0, s>>>(t, max_norm, norm); });
        return launched();
    }
    const int parts = each_table([&](const ClipTable& t, int blocks, int at) { k_norm<<<blocks, kBlock, 0, s>>>(t, h->squares + at); });
    if (parts < 0) return parts;
    each_table([&](const ClipTable& t, int blocks, int at) { k_clip<<<blocks, kBlock, 0, s>>>(t, h->squares, parts, max_norm, at == 0 ? norm : nullptr); });
    return launched();
}

}  // namespace gr
