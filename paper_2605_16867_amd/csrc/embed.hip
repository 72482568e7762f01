// Rows of a table by token, and their gradient by sorted tokens (gfx950).
//
//   out[t] = scale * table[token[t]];  dtable[v] = scale * sum of dout[t] over the t with token[t] = v
//
// Forward: the rows that are written, and those of the tokens that occur.  Backward: the tokens are sorted first, in passes of up to nine bits, each
// stable, so that the rows of a token are summed in the order in which they stand, in single precision: no atomics, the same bits every time.
#include <type_traits>

#include "tokens.h"

namespace gr {
namespace {

constexpr int kBlock = 256, kWave = 64, kWaves = kBlock / kWave, kSumWaves = 16384;

// log2 of the lanes that share a row of so many pieces
int lanes_log(int pieces)
{
    int lg = 0;
    while (lg < 6 && (1 << lg) < pieces) ++lg;
    return lg;
}

// N elements, past the cache.
template <typename T, int N>
__device__ __forceinline__ void store_past(T* at, const Elements<T, N>& e)
{
    typedef T Vec __attribute__((ext_vector_type(N), aligned(sizeof(T))));
    Vec v;
    __builtin_memcpy(&v, &e, sizeof e);
    __builtin_nontemporal_store(v, reinterpret_cast<Vec*>(at));
}

constexpr int kRowsAtOnce = 4;      // rows of a group of lanes whose loads are under way together

// Pieces of 16 bytes at any address of an element; the last one of a row reaches back into the one before.  What is written is not asked for again soon:
// it goes past the cache, which the rows of frequent tokens then stay in.
template <typename T, int N>
__global__ __launch_bounds__(kBlock) void k_embed(const int* token, const T* table, float scale, T* out, int64_t n, int vocab, int width, int lg)
{
    typedef Elements<T, N> Of;
    const int groups = kBlock >> lg, group = threadIdx.x >> lg;
    const int64_t first = (int64_t)blockIdx.x * groups * kRowsAtOnce + group;
    const T* from[kRowsAtOnce];
#pragma unroll
    for (int u = 0; u < kRowsAtOnce; ++u) {
        const int64_t row = first + u * groups;
        const int v = row < n ? token[row] : -1;
        from[u] = v >= 0 && v < vocab ? table + (int64_t)v * width : nullptr;
    }
    for (int p = (threadIdx.x & ((1 << lg) - 1)) * N; p < width; p += N << lg) {
        const int c = p + N > width ? width - N : p;
        Of e[kRowsAtOnce];
#pragma unroll
        for (int u = 0; u < kRowsAtOnce; ++u) {
            e[u] = Of{};
            if (from[u]) e[u] = Of::load(from[u] + c);
        }
#pragma unroll
        for (int u = 0; u < kRowsAtOnce; ++u) {
            const int64_t row = first + u * groups;
#pragma unroll
            for (int j = 0; j < N; ++j) e[u].v[j] = from[u] ? (T)((float)e[u].v[j] * scale) : (T)0.0f;
            if (row < n) store_past(out + row * width + c, e[u]);
        }
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

// ---- the sums ----------------------------------------------------------------------------------
//
// Sorted places and rows of the table are one line of work: the places of a row, then the row itself, which is written.  A wave takes kPiece items
// of it and a block of channels, and finds its first place by the line's order: that of place p is p + key[p], of row v the places up to its last plus v.
// A row of at most kPiece places is summed where its first place is, as far as it goes; a longer one in every piece that it has places in, whose
// sums a second launch adds up in their order.

struct SumArgs {
    const int *key, *slot, *left;      // left: how many there are; null: none
    const void* dout;
    void* dtable;
    float *head, *trail;      // [pieces][width] of long rows: of the piece that has the row's end, of the others
    float scale;
    int vocab, width, piece, pieces, blocks;
};

// How many of [lo, hi) are before the first that `before` is not true for; by a wave.
template <typename F>
__device__ __forceinline__ int first_not(int lo, int hi, F before)
{
    const int lane = threadIdx.x % kWave;
    while (lo < hi) {
        const int step = (hi - lo + kWave - 1) / kWave, at = lo + lane * step;
        const uint64_t not_yet = ~__ballot(at < hi && before(at < hi ? at : lo));
        const int c = not_yet ? __builtin_ctzll(not_yet) : kWave;
        if (c == 0) break;
        hi = lo + c * step < hi ? lo + c * step : hi;
        lo += (c - 1) * step + 1;
    }
    return lo;
}

__device__ __forceinline__ int place_at(const SumArgs& a, int n, int64_t item)
{
    return first_not(0, n, [&](int p) { return (int64_t)p + a.key[p] < item; });
}

// More than kPiece places, from the first one.
__device__ __forceinline__ bool is_long(const SumArgs& a, int n, int first, int v) { return first + a.piece < n && a.key[first + a.piece] == v; }

template <typename T, int N>
__global__ __launch_bounds__(kBlock) void k_embed_sums(SumArgs a)
{
    typedef Elements<T, N> Of;
    constexpr int kAtOnce = 8;
    const int lane = threadIdx.x % kWave;
    const int64_t id = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int piece = (int)(id / a.blocks), block = (int)(id - (int64_t)piece * a.blocks);
    if (piece >= a.pieces) return;
    const int n = a.left ? *a.left : 0;
    const int64_t item = (int64_t)piece * a.piece, all = (int64_t)a.vocab + n, end = item + a.piece < all ? item + a.piece : all;
    if (item >= end) return;
    const int c_own = (block * kWave + lane) * N, c = c_own + N > a.width ? a.width - N : c_own;
    const bool on = c_own < a.width;
    const T* const dout = static_cast<const T*>(a.dout) + c;
    T* const dtable = static_cast<T*>(a.dtable) + c;
    float sum[N] = {};
    const auto put = [&](float* to) {
        if (on) reinterpret_cast<Elements<float, N>*>(sum)->store(to + (int64_t)piece * a.width + c);
    };
    const auto clear = [&] {
#pragma unroll
        for (int e = 0; e < N; ++e) sum[e] = 0;
    };
    int p = place_at(a, n, item), v = (int)(item - p);
    int ends = first_not(p, n, [&](int q) { return (int64_t)q + a.key[q] < end; });      // places up to the piece's end
    const int v_end = (int)(end - ends);
    // a row from before: long, or not this piece's
    bool headed = p > 0 && a.key[p - 1] == v;
    if (headed) {
        const int back = p > a.piece ? p - a.piece : 0, first = first_not(back, p, [&](int q) { return a.key[q] < v; });
        if (!((first == back && back > 0 && a.key[back - 1] == v) || is_long(a, n, first, v))) {
            headed = false;
            p = first_not(p, n < first + a.piece ? n : first + a.piece, [&](int q) { return a.key[q] == v; });
            ++v;
        }
    }
    // a row that has places here and does not end here: to its last place, where it is not long
    const bool open = ends > p && a.key[ends - 1] == v_end;
    bool trailing = open;
    if (open && !(headed && v == v_end)) {
        const int first = first_not(p, ends, [&](int q) { return a.key[q] < v_end; });
        if (!is_long(a, n, first, v_end)) {
            trailing = false;
            ends = first_not(ends, n < first + a.piece ? n : first + a.piece, [&](int q) { return a.key[q] == v_end; });
        }
    }
    const int last = open && !trailing ? v_end + 1 : v_end;      // rows before it are ended here
    const auto finish = [&] {
        if (headed) put(a.head);
        else if (on) {
            Of o;
#pragma unroll
            for (int e = 0; e < N; ++e) o.v[e] = (T)(sum[e] * a.scale);
            o.store(dtable + (int64_t)v * a.width);
        }
        headed = false;
        ++v;
        clear();
    };
    for (; p < ends; p += kWave) {
        const int here = ends - p < kWave ? ends - p : kWave, at = p + (lane < here ? lane : here - 1);
        const int key = a.key[at], slot = a.slot[at];
        for (int j0 = 0; j0 < here; j0 += kAtOnce) {
            Of row[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const int j = j0 + u < here ? j0 + u : here - 1;
                row[u] = Of::load(dout + (int64_t)__builtin_amdgcn_readlane(slot, j) * a.width);
            }
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                if (j0 + u >= here) break;
                const int k = __builtin_amdgcn_readlane(key, j0 + u);
                while (v < k) finish();
#pragma unroll
                for (int e = 0; e < N; ++e) sum[e] += (float)row[u].v[e];
            }
        }
    }
    while (v < last) finish();
    if (trailing) put(a.trail);
}

// A wave for each piece and block of channels: what a long row has, in the piece that it ends in.
template <typename T, int N>
__global__ __launch_bounds__(kBlock) void k_embed_join(SumArgs a)
{
    const int lane = threadIdx.x % kWave;
    const int64_t id = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int piece = (int)(id / a.blocks), block = (int)(id - (int64_t)piece * a.blocks);
    if (piece >= a.pieces) return;
    const int n = *a.left;
    const int64_t item = (int64_t)piece * a.piece, all = (int64_t)a.vocab + n, end = item + a.piece < all ? item + a.piece : all;
    if (item >= end) return;
    const int p = place_at(a, n, item), v = (int)(item - p);
    if (p == 0 || a.key[p - 1] != v) return;
    const int ends = first_not(p, n, [&](int q) { return (int64_t)q + a.key[q] < end; });
    if (v == (int)(end - ends)) return;      // the row does not end here
    const int first = first_not(0, p, [&](int q) { return a.key[q] < v; });
    if (!is_long(a, n, first, v)) return;
    const int c_own = (block * kWave + lane) * N, c = c_own + N > a.width ? a.width - N : c_own;
    if (c_own >= a.width) return;
    typedef Elements<float, N> Sum;
    float sum[N] = {};
    const auto add = [&](const Sum& s) {
#pragma unroll
        for (int e = 0; e < N; ++e) sum[e] += s.v[e];
    };
    constexpr int kAtOnce = 8;
    const float* const trail = a.trail + c;
    int i = (int)(((int64_t)first + v) / a.piece);
    for (; i + kAtOnce <= piece; i += kAtOnce) {
        Sum s[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) s[u] = Sum::load(trail + (int64_t)(i + u) * a.width);
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) add(s[u]);
    }
    for (; i < piece; ++i) add(Sum::load(trail + (int64_t)i * a.width));
    add(Sum::load(a.head + (int64_t)piece * a.width + c));
    Elements<T, N> o;
#pragma unroll
    for (int e = 0; e < N; ++e) o.v[e] = (T)(sum[e] * a.scale);
    o.store(static_cast<T*>(a.dtable) + (int64_t)v * a.width + c);
}

}  // namespace

int launch_embed(int64_t n, int vocab, int width, int dtype, const int* token, const void* table, float scale, void* out, hipStream_t s)
{
    return by_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        const auto go = [&](auto kernel, int per) -> int {
            const int lg = lanes_log((width + per - 1) / per);
            const int64_t rows = (int64_t)(kBlock >> lg) * kRowsAtOnce, blocks = (n + rows - 1) / rows;
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
        const auto go = [&](auto count) -> int {
            constexpr int N = decltype(count)::value;
            SumArgs b{};
            b.key = key[at]; b.slot = slot[at]; b.left = n > 0 ? left : nullptr; b.dout = dout; b.dtable = dtable; b.scale = scale; b.vocab = vocab;
            b.width = width;
            b.blocks = (width + kWave * N - 1) / (kWave * N);
            // as many pieces as there are waves in a few rounds; no less than 64 items each
            const int64_t items = vocab + n, most = kSumWaves / b.blocks > 1 ? kSumWaves / b.blocks : 1;
            const int64_t piece = (items + most - 1) / most > 64 ? (items + most - 1) / most : 64;
            b.piece = (int)piece;
            b.pieces = (int)((items + piece - 1) / piece);
            b.head = h->parts;
            b.trail = h->parts + (int64_t)b.pieces * width;
            if (2 * (int64_t)b.pieces * width > h->n_parts) return GR_ERR_TOO_LARGE;
            const int64_t waves = (int64_t)b.pieces * b.blocks, blocks = (waves + kWaves - 1) / kWaves;
            k_embed_sums<T, N><<<(unsigned)blocks, kBlock, 0, s>>>(b);
            if (n > piece) k_embed_join<T, N><<<(unsigned)blocks, kBlock, 0, s>>>(b);
            return launched();
        };
        // 16 bytes a lane, fewer where a row has not as many for all lanes
        constexpr int kMost = Chunk<T>::n;
        if (width >= kWave * kMost) return go(std::integral_constant<int, kMost>{});
        if (width >= kWave * kMost / 2) return go(std::integral_constant<int, kMost / 2>{});
        return go(std::integral_constant<int, 1>{});
    });
}

// (blocks of channels of 64 lanes: a wave's sums are 64 * 8 channels at most, and there are kSumWaves or one a block)
int64_t embed_parts(int width)
{
    const int64_t most = 2 * (int64_t)kWave * 8 * kSumWaves, one = 2 * (int64_t)width;
    return most > one ? most : one;
}

}  // namespace gr
