// Rows of a table by token, and their gradient by sorted tokens (gfx950).
//
//   out[t] = scale * table[token[t]];  dtable[v] = scale * sum of dout[t] over the t with token[t] = v
//
// Forward: the rows that are written, and those of the tokens that occur.  Backward: the tokens are sorted first, in passes of up to nine bits, each
// stable, so that the rows of a token are summed in the order in which they stand, in single precision: no atomics, the same bits every time.
#include "tokens.h"

namespace gr {
namespace {

constexpr int kBlock = 256, kWave = 64, kWaves = kBlock / kWave;

// log2 of the lanes that share a row of so many pieces
int lanes_log(int pieces)
{
    int lg = 0;
    while (lg < 6 && (1 << lg) < pieces) ++lg;
    return lg;
}

// Pieces of 16 bytes at any address of an element; the last one of a row reaches back into the one before.
template <typename T, int N>
__global__ __launch_bounds__(kBlock) void k_embed(const int* token, const T* table, float scale, T* out, int64_t n, int vocab, int width, int lg)
{
    typedef Elements<T, N> Of;
    const int64_t row = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> lg;
    if (row >= n) return;
    const int v = token[row];
    const bool there = v >= 0 && v < vocab;
    const T* const from = table + (int64_t)(there ? v : 0) * width;
    for (int p = (threadIdx.x & ((1 << lg) - 1)) * N; p < width; p += N << lg) {
        const int c = p + N > width ? width - N : p;
        Of e{};
        if (there) e = Of::load(from + c);
#pragma unroll
        for (int j = 0; j < N; ++j) e.v[j] = (T)((float)e.v[j] * scale);
        if (!there) e = Of{};
        e.store(out + row * width + c);
    }
}

// ---- the sort ----------------------------------------------------------------------------------
//
// A pass: how many tokens of each digit every unit of 2 048 has; for each digit the sums over units; the places.

struct SortArgs {
    const int *key, *slot;      // slot: null in the first pass, where they are the places themselves
    int *to_key, *to_slot;
    int* digits;
    int64_t n;      // tokens (in later passes: most)
    const int* left;      // null in the first pass: how many there are
    int units, vocab, shift, mask;
};

__device__ __forceinline__ int64_t count_of(const SortArgs& a) { return a.left ? *a.left : a.n; }

// The digit of the token at i, -1 if there is none or it has no row.
__device__ __forceinline__ int digit_of(const SortArgs& a, int64_t i, int64_t n, int* key)
{
    if (i >= n) return -1;
    *key = a.key[i];
    return *key < 0 || *key >= a.vocab ? -1 : *key >> a.shift & a.mask;
}

__global__ __launch_bounds__(kBlock) void k_digit_count(SortArgs a)
{
    __shared__ int hist[kDigits];
    for (int d = threadIdx.x; d <= a.mask; d += kBlock) hist[d] = 0;
    __syncthreads();
    const int64_t from = (int64_t)blockIdx.x * kSortUnit, n = count_of(a);
    for (int i = threadIdx.x; i < kSortUnit; i += kBlock) {
        int key;
        const int d = digit_of(a, from + i, n, &key);
        if (d >= 0) atomicAdd(&hist[d], 1);
    }
    __syncthreads();
    for (int d = threadIdx.x; d <= a.mask; d += kBlock) a.digits[(int64_t)d * a.units + blockIdx.x] = hist[d];
}

// Over a workgroup: the sum of the values of lower threads, and that of all.
__device__ __forceinline__ int before_me(int own, int* part, int* all)
{
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    int v = own;
    for (int d = 1; d < kWave; d *= 2) {
        const int o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    if (lane == kWave - 1) part[wave] = v;
    __syncthreads();
    int base = 0, sum = 0;
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) base += part[w];
        sum += part[w];
    }
    __syncthreads();
    *all = sum;
    return base + v - own;
}

__global__ __launch_bounds__(kBlock) void k_digit_sum(SortArgs a)
{
    __shared__ int part[kWaves];
    int* const at = a.digits + (int64_t)blockIdx.x * a.units;
    int before = 0;
    for (int u0 = 0; u0 < a.units; u0 += kBlock) {
        const int u = u0 + threadIdx.x, own = u < a.units ? at[u] : 0;
        int all;
        const int b = before_me(own, part, &all);
        if (u < a.units) at[u] = before + b;
        before += all;
    }
    if (threadIdx.x == 0) a.digits[(int64_t)kDigits * a.units + blockIdx.x] = before;
}

// What a wave's lanes wrote to shared memory is there for its others.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Waves take 512 tokens each, 64 at a time; lanes of one digit find each other bit by bit.
__global__ __launch_bounds__(kBlock) void k_digit_place(SortArgs a, int bits, int* left)
{
    __shared__ int part[kWaves], next[kWaves][kDigits];
    constexpr int kPer = kSortUnit / kWaves;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    for (int i = threadIdx.x; i < kWaves * kDigits; i += kBlock) (&next[0][0])[i] = 0;
    __syncthreads();
    const int64_t from = (int64_t)blockIdx.x * kSortUnit + wave * kPer, n = count_of(a);
    for (int i = lane; i < kPer; i += kWave) {
        int key;
        const int d = digit_of(a, from + i, n, &key);
        if (d >= 0) atomicAdd(&next[wave][d], 1);
    }
    __syncthreads();
    int before = 0;
    for (int d0 = 0; d0 <= a.mask; d0 += kBlock) {
        const int d = d0 + threadIdx.x;
        int all;
        int at = before + before_me(d <= a.mask ? a.digits[(int64_t)kDigits * a.units + d] : 0, part, &all);
        before += all;
        if (d > a.mask) continue;
        at += a.digits[(int64_t)d * a.units + blockIdx.x];
        for (int w = 0; w < kWaves; ++w) {
            const int own = next[w][d];
            next[w][d] = at;
            at += own;
        }
    }
    if (left && blockIdx.x == 0 && threadIdx.x == 0) *left = before;
    __syncthreads();
    for (int i = lane; i < kPer; i += kWave) {
        int key = 0;
        const int d = digit_of(a, from + i, n, &key);
        uint64_t same = __ballot(d >= 0);
        for (int b = 0; b < bits; ++b) {
            const uint64_t set = __ballot(d >> b & 1);
            same &= d >> b & 1 ? set : ~set;
        }
        if (d >= 0) {
            const int rank = __popcll(same & ((uint64_t(1) << lane) - 1)), at = next[wave][d] + rank;
            a.to_key[at] = key;
            a.to_slot[at] = a.slot ? a.slot[from + i] : (int)(from + i);
        }
        wave_sync();
        if (d >= 0 && (same >> lane) == 1) next[wave][d] += __popcll(same);
        wave_sync();
    }
}

// The place of the first key that is at least v.
__device__ __forceinline__ int64_t first_of(const int* key, int64_t n, int v)
{
    int64_t lo = 0, hi = n;
    while (lo < hi) {
        const int64_t mid = (lo + hi) / 2;
        if (key[mid] < v) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

template <typename T, int N>
__global__ __launch_bounds__(kBlock) void k_embed_sums(const int* key, const int* slot, const int* left, const T* dout, float scale, T* dtable,
                                                       int vocab, int width, int lg)
{
    typedef Elements<T, N> Of;
    const int64_t v = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> lg;
    if (v >= vocab) return;
    const int64_t n = left ? *left : 0, from = first_of(key, n, (int)v), to = first_of(key, n, (int)v + 1);
    for (int p = (threadIdx.x & ((1 << lg) - 1)) * N; p < width; p += N << lg) {
        const int c = p + N > width ? width - N : p;
        float sum[N] = {};
        for (int64_t i = from; i < to; ++i) {
            const Of e = Of::load(dout + (int64_t)slot[i] * width + c);
#pragma unroll
            for (int j = 0; j < N; ++j) sum[j] += (float)e.v[j];
        }
        Of o;
#pragma unroll
        for (int j = 0; j < N; ++j) o.v[j] = (T)(sum[j] * scale);
        o.store(dtable + v * width + c);
    }
}

}  // namespace

int launch_embed(int64_t n, int vocab, int width, int dtype, const int* token, const void* table, float scale, void* out, hipStream_t s)
{
    return by_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        const auto go = [&](auto kernel, int per) -> int {
            const int lg = lanes_log((width + per - 1) / per);
            const int64_t blocks = ((n << lg) + kBlock - 1) / kBlock;
            if (blocks > kMostBlocks) return GR_ERR_TOO_LARGE;
            kernel<<<(unsigned)blocks, kBlock, 0, s>>>(token, static_cast<const T*>(table), scale, static_cast<T*>(out), n, vocab, width, lg);
            return launched();
        };
        return width >= Chunk<T>::n ? go(k_embed<T, Chunk<T>::n>, Chunk<T>::n) : go(k_embed<T, 1>, 1);
    });
}

int launch_embed_backward(gr_tokens* h, int64_t n, int vocab, int width, int dtype, const int* token, const void* dout, float scale,
                          void* dtable, hipStream_t s)
{
    int bits = 1;
    while ((int64_t(1) << bits) < vocab) ++bits;
    const int passes = (bits + kDigitBits - 1) / kDigitBits;
    int *const key[2] = {h->order, h->order + h->max_tokens}, *const slot[2] = {h->order + 2 * h->max_tokens, h->order + 3 * h->max_tokens};
    SortArgs a{};
    a.digits = h->digits; a.n = n; a.units = (int)sort_units(n); a.vocab = vocab;
    int* const left = h->digits + (sort_units(h->max_tokens) + 1) * kDigits;
    int at = 0;
    for (int p = 0; p < passes && n > 0; ++p) {
        const int from = bits * p / passes, to = bits * (p + 1) / passes;
        a.key = p ? key[at] : token;
        a.slot = p ? slot[at] : nullptr;
        a.left = p ? left : nullptr;
        at = p & 1;
        a.to_key = key[at]; a.to_slot = slot[at];
        a.shift = from; a.mask = (1 << (to - from)) - 1;
        k_digit_count<<<a.units, kBlock, 0, s>>>(a);
        k_digit_sum<<<a.mask + 1, kBlock, 0, s>>>(a);
        k_digit_place<<<a.units, kBlock, 0, s>>>(a, to - from, p ? nullptr : left);
    }
    return by_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        const auto go = [&](auto kernel, int per) -> int {
            const int lg = lanes_log((width + per - 1) / per);
            const int64_t blocks = (((int64_t)vocab << lg) + kBlock - 1) / kBlock;
            if (blocks > kMostBlocks) return GR_ERR_TOO_LARGE;
            kernel<<<(unsigned)blocks, kBlock, 0, s>>>(key[at], slot[at], n > 0 ? left : nullptr, static_cast<const T*>(dout), scale,
                                                       static_cast<T*>(dtable), vocab, width, lg);
            return launched();
        };
        return width >= Chunk<T>::n ? go(k_embed_sums<T, Chunk<T>::n>, Chunk<T>::n) : go(k_embed_sums<T, 1>, 1);
    });
}

}  // namespace gr
