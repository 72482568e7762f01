// Rows of a table by token, and their gradient by sorted tokens (gfx950).
//
//   out[t] = scale * table[token[t]];  dtable[v] = scale * sum of dout[t] over the t with token[t] = v
//
// Bound by memory.  Forward: the rows that are written, and those of the tokens that occur: 524 288 rows of 1 024 in bfloat16 1.2 GB, 227 us while the table
// stands in the cache, 290 where it does not.  Backward: the tokens are sorted first, in passes of up to nine bits, each stable, so that the rows of a
// token are summed in single precision in an order that hangs on where they stand alone: no atomics, the same bits every time.  Of 283 us at the same
// sizes 234 are the sums (1.2 GB, 5.2 TB/s), 7 the joining of those that pieces share, 33 the sort; of 56 at 49 999 of 511 in single precision 35, 5 and 17.
#include <type_traits>

#include "tokens.h"

namespace gr {
namespace {

constexpr int kBlock = 256, kWave = 64, kWaves = kBlock / kWave, kDies = 8;

// log2 of the lanes that share a row of so many pieces
int lanes_log(int pieces)
{
    int lg = 0;
    while (lg < 6 && (1 << lg) < pieces) ++lg;
    return lg;
}

constexpr int kRowsAtOnce = 2;      // rows of a group of lanes whose loads are under way together

// Pieces of 16 bytes at any address of an element; the last one of a row reaches back into the one before.  What is written goes past the cache, which the
// rows of frequent tokens then stay in: faster at every size (bfloat16, 65 536 rows of 256 7.9 us for 10.0, of 1 024 30 for 43.5, 524 288 of 1 024 226 for
// 328; 512 of 256 in single precision 3.3 for 3.3 to 3.7).  A product that reads the rows next finds them there only up to some 100 MB: with one, 512 of 256 15.8 us
// for 14.3, 16 384 of 256 in bfloat16 20.1 for 19.8, 65 536 50.4 for 44.1, but 65 536 of 1 024 185 for 188, 524 288 590 for 628.
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
            if (row < n) store_of<true>(out + row * width + c, e[u]);
        }
    }
}

// ---- the sort ----------------------------------------------------------------------------------
//
// A pass: how many tokens of each digit every unit of 2 048 has; for each digit the sums over units; the places.  4 MB of tokens and places are in the cache
// throughout: what counts is launches and the loads that wait for each other, 4, 3 and 7 us at 524 288 tokens.  A unit is 16 waves of 128 tokens (four of 512: 13 us
// for the places).  Token and place are a pair: as two arrays, in two stores, 9.

constexpr int kFewUnits = 64;      // up to so many each workgroup of the places adds them up itself, one launch less

struct SortArgs {
    const int* token;      // the first pass's, which stand at their places
    const int2* from;      // later ones': token and place
    int2* to;
    int* digits;
    int64_t n;      // tokens (in later passes: most)
    const int* left;      // null in the first pass: how many there are
    int units, vocab, shift, mask;
    int summed;      // digits holds what is before a unit, and those of all; else each unit's own
};

__device__ __forceinline__ int64_t count_of(const SortArgs& a) { return a.left ? *a.left : a.n; }

// A die's workgroups, every eighth, take units that follow each other: what they write is side by side in its cache (the places of 1 000 000 tokens 13.6 us for 15.5).
__device__ __forceinline__ int unit_of(const SortArgs& a)
{
    return (int)(a.summed ? blockIdx.x % kDies * (gridDim.x / kDies) + blockIdx.x / kDies : blockIdx.x);
}

// The digit of the token at i, -1 if there is none or it has no row.
__device__ __forceinline__ int digit_of(const SortArgs& a, int64_t i, int64_t n, int2* pair)
{
    if (i >= n) return -1;
    *pair = a.from ? a.from[i] : int2{a.token[i], (int)i};
    const int key = pair->x;
    return key < 0 || key >= a.vocab ? -1 : key >> a.shift & a.mask;
}

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / kWave, kSortRounds = kSortUnit / kSortThreads;

__global__ __launch_bounds__(kSortThreads) void k_digit_count(SortArgs a)
{
    __shared__ int hist[kDigits];
    const int unit = unit_of(a);
    if (unit >= a.units) return;
    if (threadIdx.x < kDigits) hist[threadIdx.x] = 0;
    const int64_t from = (int64_t)unit * kSortUnit + threadIdx.x, n = count_of(a);
    int d[kSortRounds];
    int2 pair;
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) d[r] = digit_of(a, from + r * kSortThreads, n, &pair);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r)
        if (d[r] >= 0) atomicAdd(&hist[d[r]], 1);
    __syncthreads();
    const int t = threadIdx.x;
    if (t <= a.mask) a.digits[a.summed ? (int64_t)t * a.units + unit : (int64_t)unit * kDigits + t] = hist[t];
}

// The sum over the lanes up to this one.
__device__ __forceinline__ int up_to_me(int v)
{
    const int lane = threadIdx.x % kWave;
    for (int d = 1; d < kWave; d *= 2) {
        const int o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}

// Of a digit: what is before each unit, and the sum of all.
__global__ __launch_bounds__(kBlock) void k_digit_sum(SortArgs a)
{
    __shared__ int part[kWaves];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    int* const at = a.digits + (int64_t)blockIdx.x * a.units;
    int before = 0;
    for (int u0 = 0; u0 < a.units; u0 += kBlock) {
        const int u = u0 + threadIdx.x, own = u < a.units ? at[u] : 0, upto = up_to_me(own);
        if (lane == kWave - 1) part[wave] = upto;
        __syncthreads();
        int base = before;
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) base += part[w];
            before += part[w];
        }
        if (u < a.units) at[u] = base + upto - own;
        __syncthreads();
    }
    if (threadIdx.x == 0) a.digits[(int64_t)kDigits * a.units + blockIdx.x] = before;
}

// What a wave's lanes wrote to shared memory is there for its others.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The lanes of a wave that have the same digit, of so many bits; none for a digit of -1.
__device__ __forceinline__ uint64_t lanes_of(int digit, int bits)
{
    uint64_t same = __ballot(digit >= 0);
    for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot(digit >> b & 1);
        same &= digit >> b & 1 ? set : ~set;
    }
    return same;
}

// Each lane's place among its wave's tokens of the same digit, 64 tokens at a time, lanes of one digit finding each other bit by bit; `next`, the wave's own,
// is left with how many there are.
template <int kRounds>
__device__ __forceinline__ void ranks(const int (&d)[kRounds], int rounds, int bits, int* next, int digits, int (&rank)[kRounds])
{
    const int lane = threadIdx.x % kWave;
    for (int i = lane; i < digits; i += kWave) next[i] = 0;
    uint64_t same[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
        if (r < rounds) same[r] = lanes_of(d[r], bits);
    wave_sync();
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        if (r >= rounds) break;
        const int before = d[r] >= 0 ? next[d[r]] : 0;
        rank[r] = before + __popcll(same[r] & ((uint64_t(1) << lane) - 1));
        wave_sync();
        if (d[r] >= 0 && (same[r] >> lane) == 1) next[d[r]] = rank[r] + 1;
        wave_sync();
    }
}

// Waves take 128 tokens each.
__global__ __launch_bounds__(kSortThreads) void k_digit_place(SortArgs a, int bits, int* left)
{
    __shared__ int part[kDigits / kWave], next[kSortWaves][kDigits];
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, unit = unit_of(a);
    if (unit >= a.units) return;
    const int64_t from = (int64_t)unit * kSortUnit + wave * (kSortUnit / kSortWaves) + lane, n = count_of(a);
    int2 pair[kSortRounds];
    int d[kSortRounds], rank[kSortRounds];
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) d[r] = digit_of(a, from + r * kWave, n, &pair[r]);
    int earlier = 0, whole = 0;
    if (tid <= a.mask) {
        if (a.summed) {
            earlier = a.digits[(int64_t)tid * a.units + unit];
            whole = a.digits[(int64_t)kDigits * a.units + tid];
        } else
            for (int u0 = 0; u0 < a.units; u0 += 16) {
                int own[16];
#pragma unroll
                for (int u = 0; u < 16; ++u) own[u] = a.digits[(int64_t)(u0 + u < a.units ? u0 + u : u0) * kDigits + tid];
#pragma unroll
                for (int u = 0; u < 16; ++u) {
                    earlier += u0 + u < unit ? own[u] : 0;
                    whole += u0 + u < a.units ? own[u] : 0;
                }
            }
    }
    ranks(d, kSortRounds, bits, next[wave], kDigits, rank);
    const int upto = up_to_me(whole);
    if (tid < kDigits && lane == kWave - 1) part[wave] = upto;
    __syncthreads();
    if (tid < kDigits) {
        int at = earlier + upto - whole, all = 0, own[kSortWaves];
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) own[w] = next[w][tid];
        for (int w = 0; w < kDigits / kWave; ++w) {
            if (w < wave) at += part[w];
            all += part[w];
        }
        if (left && unit == 0 && tid == 0) *left = all;
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            next[w][tid] = at;
            at += own[w];
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r)
        if (d[r] >= 0) a.to[next[wave][d[r]] + rank[r]] = pair[r];
}

// Few tokens are sorted by one workgroup in one launch, in shared memory between the passes: 512 of 32 000 in 5 us where six launches take 16; 8 192 of them
// 22, where four launches take 18.
constexpr int kFewTokens = 4096, kFewThreads = 1024, kFewWaves = kFewThreads / kWave, kFewRounds = kFewTokens / kFewThreads;

__global__ __launch_bounds__(kFewThreads) void k_sort_few(const int* token, int n, int vocab, int bits, int2* to, int* left)
{
    __shared__ int2 order[kFewTokens];
    __shared__ int next[kFewWaves][kDigits], part[kDigits / kWave];
    const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave), passes = (bits + kDigitBits - 1) / kDigitBits;
    for (int pass = 0; pass < passes; ++pass) {
        const int shift = bits * pass / passes, width = bits * (pass + 1) / passes - shift, mask = (1 << width) - 1;
        const int most = (n + kFewThreads - 1) / kFewThreads, first = wave * most * kWave, from = first + lane, rounds = first < n ? most : 0;
        int2 pair[kFewRounds];
        int d[kFewRounds], rank[kFewRounds];
#pragma unroll
        for (int r = 0; r < kFewRounds; ++r) {
            const int i = from + r * kWave;
            pair[r] = int2{-1, 0};
            if (r < rounds && i < n) pair[r] = pass ? order[i] : int2{token[i], i};
            d[r] = pair[r].x < 0 || pair[r].x >= vocab ? -1 : pair[r].x >> shift & mask;
        }
        ranks(d, rounds, width, next[wave], mask + 1, rank);
        __syncthreads();
        int before = 0, own[kFewWaves], upto = 0, all = 0;
        if (tid < kDigits) {
#pragma unroll
            for (int w = 0; w < kFewWaves; ++w) {
                own[w] = tid <= mask ? next[w][tid] : 0;
                before += own[w];
            }
            upto = up_to_me(before);
            if (lane == kWave - 1) part[wave] = upto;
        }
        __syncthreads();
        before = upto - before;
        for (int w = 0; w < kDigits / kWave; ++w) {
            if (w < wave) before += part[w];
            all += part[w];
        }
        if (tid <= mask) {
#pragma unroll
            for (int w = 0; w < kFewWaves; ++w) {
                next[w][tid] = before;
                before += own[w];
            }
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kFewRounds; ++r)
            if (d[r] >= 0) (pass + 1 == passes ? to : order)[next[wave][d[r]] + rank[r]] = pair[r];
        n = all;
        __syncthreads();
    }
    if (tid == 0) *left = n;
}

// ---- the sums ----------------------------------------------------------------------------------
//
// Sorted places and rows of the table are one line of work: the places of a row, then the row itself, which is written.  A workgroup takes a piece's items
// of it, 64 to 1 024, and a block of channels, and finds its first place by the line's order: that of place p is p + key[p], of row v the places up
// to its last plus v.  Its places stand in shared memory.  As many lanes as a row has chunks are a team, up to a wave; a team takes places that follow each
// other, eight rows under way at a time, and writes the rows that it has all of.  What it has of one that goes on behind it is passed on from team to team
// by a scan, whose order hangs on places alone, and what a piece has of one that goes on behind the piece by a second launch.  So it does not matter how the
// places are shared out among rows: 1 000 000 of 16 channels, where a token is 4 % of all of them, 26 us.

struct SumArgs {
    const int2* place;      // tokens in order, and where each stood
    const int* left;        // how many there are; null: none
    const void* dout;
    void* dtable;
    float *head, *trail;      // [pieces][width] of rows that pieces share: of the piece that has the row's end, of the others
    int2* ended;              // [pieces] such a row that ends there, or -1; whether one goes through
    float scale;
    int vocab, width, piece, pieces, blocks;
    int lg;      // log2 of the lanes of a team
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
    return first_not(0, n, [&](int p) { return (int64_t)p + a.place[p].x < item; });
}

// The sum of a row that goes on behind these places; of all of them, the row having begun before them?
template <int N>
struct Open {
    Elements<float, N> sum;
    bool through;
    __device__ __forceinline__ void behind(const Open& o)      // o is what stands before
    {
#pragma unroll
        for (int e = 0; e < N; ++e) sum.v[e] = through ? o.sum.v[e] + sum.v[e] : sum.v[e];
        through = through && o.through;
    }
    __device__ __forceinline__ Open up(int lanes) const
    {
        Open o;
#pragma unroll
        for (int e = 0; e < N; ++e) o.sum.v[e] = __shfl_up(sum.v[e], lanes);
        o.through = __shfl_up((int)through, lanes);
        return o;
    }
};

// kPast: rows are read past the cache.
template <typename T, int N, bool kPast>
__global__ __launch_bounds__(kBlock) void k_embed_sums(SumArgs a)
{
    typedef Elements<T, N> Of;
    typedef Elements<float, N> Sum;
    constexpr int kAtOnce = 8;
    __shared__ int keys[kPieceItems], slots[kPieceItems], occurs[kPieceItems], bound[2];
    __shared__ Open<N> of_wave[kWaves][kWave];
    const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int lg = a.lg, teams = kBlock >> lg, team = tid >> lg, mine = tid & ((1 << lg) - 1), n = a.left ? *a.left : 0;
    // (the blocks of a piece share lines at their edges: one die's workgroups, every eighth, take them one after the other)
    const int block = (int)(blockIdx.x / kDies % a.blocks), piece = (int)(blockIdx.x / (kDies * a.blocks) * kDies + blockIdx.x % kDies);
    const int64_t item = (int64_t)piece * a.piece, all = (int64_t)a.vocab + n, end = item + a.piece < all ? item + a.piece : all;
    if (item >= end) return;
    for (int i = tid; i < kPieceItems; i += kBlock) occurs[i] = 0;
    if (wave < 2) {
        const int p = place_at(a, n, wave ? end : item);
        if (lane == 0) bound[wave] = p;
    }
    __syncthreads();
    const int p0 = bound[0], count = bound[1] - p0, v0 = (int)(item - p0), v1 = (int)(end - bound[1]);      // rows from v0 to v1 end here
    const bool headed = p0 > 0 && a.place[p0 - 1].x == v0;
    for (int i = tid; i < count; i += kBlock) {
        const int2 at = a.place[p0 + i];
        keys[i] = at.x;
        slots[i] = at.y;
        if (at.x < v1) occurs[at.x - v0] = 1;
    }
    __syncthreads();
    const int per = (count + teams - 1) / teams, from = team * per, to = from + per < count ? from + per : count;
    bool before = false, after = false;      // the first row began before this team's places, the last goes on behind them
    if (from < to) {
        before = from > 0 ? keys[from - 1] == keys[from] : headed && keys[0] == v0;
        after = keys[to - 1] == (to < count ? keys[to] : v1);
    }
    const int c0 = (block * kWave + mine) * N, c = c0 + N > a.width ? a.width - N : c0;
    const bool on = c0 < a.width;
    const T* const dout = static_cast<const T*>(a.dout) + c;
    T* const dtable = static_cast<T*>(a.dtable) + c;
    const auto write = [&](int v, const Sum& sum) {
        Of o;
#pragma unroll
        for (int e = 0; e < N; ++e) o.v[e] = (T)(sum.v[e] * a.scale);
        if (on) o.store(dtable + (int64_t)v * a.width);
    };
    const auto keep = [&](float* to, const Sum& sum) {
        if (on) sum.store(to + (int64_t)piece * a.width + c);
    };
    int ended = -1;      // a row that began before and ends here, and what this team has of it
    Sum head{}, sum{};
    for (int i0 = from; i0 < to; i0 += kAtOnce) {
        Of row[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) row[u] = load_of<kPast, T, N>(dout + (int64_t)slots[i0 + u < to ? i0 + u : to - 1] * a.width);
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int i = i0 + u;
            if (i >= to) break;
#pragma unroll
            for (int e = 0; e < N; ++e) sum.v[e] += (float)row[u].v[e];
            if (i + 1 < to ? keys[i + 1] == keys[i] : after) continue;
            if (before) {
                ended = keys[i];
                head = sum;
            } else write(keys[i], sum);
            before = false;
            sum = Sum{};
        }
    }
    Open<N> open{sum, after && before};
    for (int d = 1 << lg; d < kWave; d *= 2) {
        const Open<N> o = open.up(d);
        if (lane >= d) open.behind(o);
    }
    if (lane >= kWave - (1 << lg)) of_wave[wave][mine] = open;
    Open<N> earlier = open.up(1 << lg);      // before this team
    __syncthreads();
    Open<N> first{Sum{}, true};      // before this wave
    for (int w = 0; w < wave; ++w) {
        Open<N> o = of_wave[w][mine];
        o.behind(first);
        first = o;
    }
    if (lane < 1 << lg) earlier = first;
    else earlier.behind(first);
    if (ended >= 0) {
#pragma unroll
        for (int e = 0; e < N; ++e) head.v[e] += earlier.sum.v[e];
        if (earlier.through) keep(a.head, head);
        else write(ended, head);
    }
    if (to == count && from < to && after) {
        open.behind(first);
        keep(a.trail, open.sum);
    }
    if (team == 0 && headed && v0 < v1 && (count == 0 || keys[0] != v0)) keep(a.head, Sum{});
    for (int r = team * a.blocks + block; r < v1 - v0; r += teams * a.blocks)
        if (!occurs[r] && !(r == 0 && headed)) {
            T* const row = static_cast<T*>(a.dtable) + (int64_t)(v0 + r) * a.width;
            for (int c0 = mine * N; c0 < a.width; c0 += kWave * N) Of{}.store(row + (c0 + N > a.width ? a.width - N : c0));
        }
    // (a row that goes through this piece: no place of another is in it, and it does not end here)
    if (tid == 0 && block == 0) a.ended[piece] = int2{headed && v0 < v1 ? v0 : -1, headed && v0 == v1};
}

// A workgroup a piece that a row from before ends in: the parts of it, shared by the teams.
template <typename T, int N>
__global__ __launch_bounds__(kBlock) void k_embed_join(SumArgs a)
{
    typedef Elements<float, N> Sum;
    __shared__ Sum of_wave[kWaves][kWave];
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, lg = a.lg, teams = kBlock >> lg, team = tid >> lg, mine = tid & ((1 << lg) - 1);
    const int piece = blockIdx.x;
    // (behind the last item there may be pieces that nothing was written for)
    if ((int64_t)piece * a.piece >= (int64_t)a.vocab + *a.left) return;
    const int v = a.ended[piece].x;
    if (v < 0) return;
    int start = piece - 1;      // the piece that it begins in: the last before this one that it does not go through
    for (;;) {
        const uint64_t not_through = __ballot(start - lane <= 0 || !a.ended[start - lane > 0 ? start - lane : 0].y);
        start -= not_through ? __builtin_ctzll(not_through) : kWave;
        if (not_through) break;
    }
    const int c_own = (blockIdx.y * kWave + mine) * N, c = c_own + N > a.width ? a.width - N : c_own, parts = piece - start, per = (parts + teams - 1) / teams;
    const int from = start + team * per, to = from + per < piece ? from + per : piece;
    Sum sum{};
    constexpr int kAtOnce = 8;
    for (int i = from; i < to; i += kAtOnce) {
        Sum s[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) s[u] = Sum::load(a.trail + (int64_t)(i + u < to ? i + u : i) * a.width + c);
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
            for (int e = 0; e < N; ++e) sum.v[e] += i + u < to ? s[u].v[e] : 0.0f;
    }
    for (int d = 1 << lg; d < kWave; d *= 2)
#pragma unroll
        for (int e = 0; e < N; ++e) sum.v[e] += __shfl_xor(sum.v[e], d);
    if (lane < 1 << lg) of_wave[wave][mine] = sum;
    __syncthreads();
    if (tid >= 1 << lg || c_own >= a.width) return;
    const Sum head = Sum::load(a.head + (int64_t)piece * a.width + c);
    Elements<T, N> o;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        float all = of_wave[0][mine].v[e];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) all += of_wave[w][mine].v[e];
        o.v[e] = (T)((all + head.v[e]) * a.scale);
    }
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

// How many pieces there are, as long as they have 64 items at least and 1 024 at most.  1 000 000 rows of 16 channels in bfloat16 with 1 024 pieces 81 us, with 2 048 83,
// with 4 096 87; 300 000 of 400 with 2 048 95, with 4 096 100; 524 288 of 1 024, two blocks, with 1 024 295, with 2 048 286, with 4 096 289; 50 000 of 2 000, four
// blocks, with 1 024 91, with 2 048 96.  At least 32 items: 49 999 of 511 in single precision 61 us for 57; at least 128: 16 000 of 512 33 for 31.
constexpr int kTeamPieces = 1024, kMostPieces = 2048, kBlockPieces = 4096, kLeastItems = 64;

int pieces_of(int lg, int blocks)
{
    const int most = lg < 6 ? kTeamPieces : kBlockPieces / blocks;
    return most > kMostPieces ? kMostPieces : most < 1 ? 1 : most;
}

int launch_embed_backward(gr_tokens* h, int64_t n, int vocab, int width, int dtype, const int* token, const void* dout, float scale,
                          void* dtable, hipStream_t s)
{
    int bits = 1;
    while ((int64_t(1) << bits) < vocab) ++bits;
    const int passes = (bits + kDigitBits - 1) / kDigitBits;
    int2* const order[2] = {h->order, h->order + h->max_tokens};
    SortArgs a{};
    a.digits = h->digits; a.n = n; a.units = (int)sort_units(n); a.vocab = vocab; a.summed = a.units > kFewUnits;
    int* const left = h->digits + (sort_units(h->max_tokens) + 1) * kDigits;
    const int grid = a.summed ? (a.units + kDies - 1) / kDies * kDies : a.units;
    int at = 0;
    if (n > 0 && n <= kFewTokens) k_sort_few<<<1, kFewThreads, 0, s>>>(token, (int)n, vocab, bits, order[0], left);
    for (int p = 0; p < passes && n > kFewTokens; ++p) {
        const int from = bits * p / passes, to = bits * (p + 1) / passes;
        a.token = token;
        a.from = p ? order[at] : nullptr;
        a.left = p ? left : nullptr;
        at = p & 1;
        a.to = order[at];
        a.shift = from; a.mask = (1 << (to - from)) - 1;
        k_digit_count<<<grid, kSortThreads, 0, s>>>(a);
        if (a.summed) k_digit_sum<<<a.mask + 1, kBlock, 0, s>>>(a);
        k_digit_place<<<grid, kSortThreads, 0, s>>>(a, to - from, p ? nullptr : left);
    }
    return by_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        const auto go = [&](auto count) -> int {
            constexpr int N = decltype(count)::value;
            SumArgs b{};
            b.place = order[at]; b.left = n > 0 ? left : nullptr; b.dout = dout; b.dtable = dtable; b.scale = scale; b.vocab = vocab;
            b.width = width;
            b.blocks = (width + kWave * N - 1) / (kWave * N);
            b.lg = lanes_log((width + N - 1) / N);
            const int64_t items = vocab + n, least = (items + pieces_of(b.lg, b.blocks) - 1) / pieces_of(b.lg, b.blocks);
            b.piece = (int)(least < kLeastItems ? kLeastItems : least > kPieceItems ? kPieceItems : least);
            b.pieces = (int)((items + b.piece - 1) / b.piece);
            b.head = h->parts;
            b.ended = h->ended;
            b.trail = h->parts + (int64_t)b.pieces * width;
            if (2 * (int64_t)b.pieces * width > h->n_parts) return GR_ERR_TOO_LARGE;
            const int64_t blocks = (int64_t)(b.pieces + kDies - 1) / kDies * kDies * b.blocks;
            if (blocks > kMostBlocks) return GR_ERR_TOO_LARGE;
            if (past_cache((n + vocab) * width * (int64_t)sizeof(T))) k_embed_sums<T, N, true><<<(unsigned)blocks, kBlock, 0, s>>>(b);
            else k_embed_sums<T, N, false><<<(unsigned)blocks, kBlock, 0, s>>>(b);
            if (n > 0 && b.pieces > 1) k_embed_join<T, N><<<dim3(b.pieces, b.blocks), kBlock, 0, s>>>(b);
            return launched();
        };
        return width >= Chunk<T>::n ? go(std::integral_constant<int, Chunk<T>::n>{}) : go(std::integral_constant<int, 1>{});
    });
}

int64_t embed_pieces(int64_t n, int vocab)
{
    const int64_t whole = (n + vocab + kPieceItems - 1) / kPieceItems;
    return whole > kMostPieces ? whole : kMostPieces;
}

// (pieces of less than kPieceItems are no more than pieces_of)
int64_t embed_parts(int64_t n, int vocab, int width)
{
    const int64_t less = 2 * (int64_t)kWave * 8 * kBlockPieces, whole = 2 * (int64_t)width * ((n + vocab + kPieceItems - 1) / kPieceItems);
    return less > whole ? less : whole;
}

}  // namespace gr
