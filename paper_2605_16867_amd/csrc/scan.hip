// A gated recurrence along sequences of tokens, forward and backward (gfx950).
//
//   f = sigmoid(gate), i = sigmoid(-gate);  h_t = f_t h_{t-1} + i_t x_t
//   D_t = dy_t + c_{t+1}, c_t = f_t D_t;  dx_t = i_t D_t, dgate_t = f_t i_t D_t (h_{t-1} - x_t)
//
// Bound by memory: three arrays forward, six backward, read once and written once; near it by vector instructions, 29 for an element forward (half of them
// the two sigmoids, to two units of single precision's last digit), which keep the units busy for 57 % of the time in 16 bits.  The step from token to token
// is linear, so a stretch of tokens is two numbers a channel, and stretches join: work is split over the tokens however long a sequence is.
// MI355X, us: 262 144 tokens of 1 024 sequences x 1 024 in bfloat16 380 (1.6 GB, 4.2 TB/s), backward 659 (3.2 GB, 4.9 TB/s; 582
// without dy); 100 000 x 1 024 in single precision 211 (5.8 TB/s); one sequence of 65 536 x 1 024 in float16 115; 3 000 tokens x 256 7.7; a token of 4 096
// requests x 1 024 10, backward 20.5.
#include <type_traits>
#include <utility>

#include "tokens.h"

namespace gr {
namespace {

constexpr int kBlock = 256;

struct Gate {
    float keep, take;      // sigmoid(gate), sigmoid(-gate)
};

// With e = exp(-|gate|) the smaller one is e / (1 + e), which is no difference and has its digits however far the gate is from 0; the larger one is
// what it leaves of 1, rounded once: states pass through thousands of those.  The exponent is |gate| log2(e) in single precision; what the product lost
// and what the constant lost, |gate| * 2^-24 and |gate| * 2^-26, are made good: without the second, which has one sign, the smaller one is 3.0 units of 2^-23
// off at a gate of 10 and 10.6 at 85, with it 2.1 and 1.1.  An infinite gate's product has lost what is no number; the median of three makes a number of
// it, and e is 0.  A gate that is no number stays one.
__device__ __forceinline__ Gate gate_of(float g)
{
    constexpr float kLog2e = 1.44269504089f, kLog2eRest = 1.92596299e-8f, kLn2 = 0.693147181f;
    const float a = fabsf(g), p = a * -kLog2e;
    const float lost = __builtin_amdgcn_fmed3f(fmaf(fmaf(a, -kLog2e, -p), kLn2, a * (-kLog2eRest * kLn2)), -1.0f, 1.0f);
    float e = __builtin_amdgcn_exp2f(p);
    e = fmaf(e, lost, e);
    const float far = e * __builtin_amdgcn_rcpf(1.0f + e), near = 1.0f - far;
    return g >= 0 ? Gate{near, far} : Gate{far, near};
}

// Both in one word: the smaller one, negative where it is the first; the other is what it leaves of 1.
__device__ __forceinline__ float packed(Gate g) { return g.keep < g.take ? -g.keep : g.take; }

__device__ __forceinline__ Gate unpacked(float v)
{
    const float s = fabsf(v), rest = 1.0f - s;
    return __float_as_int(v) >= 0 ? Gate{rest, s} : Gate{s, rest};
}

// ---- many tokens: tiles of rows -----------------------------------------------------------------
//
// Rows are taken in the direction of the recurrence (backward: the last one first), a tile of them by a workgroup, a run of kRun by the lanes
// that share a row; a lane has N channels.  A stretch of rows takes a state c to F c + B, F the product of its f.  For a tile a workgroup
//   1. reads its rows once, holds f and what is added in registers, and finds (F, B) of its runs, and of the tile, which it publishes;
//   2. finds the state that the tile starts from: of the tiles since the one that its sequence starts in, or since the last multiple of kGroup tiles,
//      whose last tile publishes the state itself;
//   3. goes through its rows once more, in registers, and writes.
// The order in which stretches are joined hangs on the places of rows and sequences alone, so the bits are the same every time.
//
// Published words are 64 bits, a value and the number of the call: complete or not there, with nothing to order between words.  Workgroups take
// tiles by a ticket, one counter for each block of channels, so that those that a tile waits for are always held by workgroups that run already, and
// wait for none behind them: every wait ends.  A counter holds the number of the call and the next ticket in one word; whoever draws the last one of
// all counters sets them for the next call (all others have what they need by then).  Draws at one counter follow each other in 43 ns: with one for
// all blocks, and another for workgroups that are done, 262 144 tokens of 1 024 took 1.4 ms whatever else was done.
//
// Of the 11.7 us of a workgroup there (of which two share a unit) 0.5 are the draw, 2.7 the loads, 2.3 the sigmoids, 3.9 the join with the tiles before,
// 2 the second pass.  A sequence's marks are looked up beside the loads; offsets of up to 2 047 sequences are in shared memory by then (1 us less).

constexpr int kThreads = 512, kWaves = kThreads / 64;
// Of 16 tiles the last publishes a state: one of eight is a longer chain (300 000 x 64 89 us for 71), one of 32 more words to look at (65 536 x 1 024 131
// for 116).
constexpr int kGroup = 16, kLeastLanesLog = 2, kNearOffsets = 2048, kMostRuns = kThreads >> kLeastLanesLog;
// Rows of a run: as many as leave a unit two workgroups (forward 115 registers, backward 124); few where there would not be a tile a unit: 3 000 x 256 in
// single precision 8.9 us with four (9.8 with two, 9.9 with eight), but 16 000 x 512, 504 tiles of eight, 20 us (24 with four, 33 with two).
constexpr int kRunForward = 8, kRunBackward = 6, kRunFew = 4;
constexpr int64_t kFewTiles = 256;
// Blocks of channels.  A row is split into as few as 32 lanes allow, all with as many lanes.  Where rows lie on lines, or halves of lines, blocks start there as well:
// two that share a line both ask for it (200 000 x 224 in bfloat16 86 us for 89, 100 000 x 352 backward 107 for 120, single precision 100 000 x 416 106 for
// 118).  There 16 lanes are taken if that leaves fewer without a piece (bfloat16, 300 000 x 192 96 us for 131, 200 000 x 160 67 for 82, 100 000 x 1 088 156 for 194,
// backward 262 for 346; elsewhere 200 000 x 270 128 for 124, backward 244 for 215), and, where rows are whole sixteens, with rows of 512 bytes at most
// (a block has a counter, and 300 000 x 128 are 2 300 draws: 69 us for 76) and with a round of tiles (16 000 x 512 17.3 for 18.5, 3 000 x 256 in single
// precision 7.7 for 8.3); other rows are faster by 32 (200 000 x 512 152 for 154, 262 144 x 1 024 380 for 390).  Eight lanes, blocks of 64 bytes, are slower.
constexpr int kFewLanesLog = 4, kFewLanesBytes = 512;
constexpr int64_t kFewLanesTiles = 512;

struct TileArgs {
    ScanIn in;
    void *y, *dgate, *dx;
    float* last;      // states after the last rows (backward: gradients of the first states)
    uint64_t *sums, *states;
    uint64_t* control;      // see Control
    int n, n_seq, tiles, blocks, lanes, lg, rows;      // blocks of channels, lanes of a row in use, log2 of lanes of a row, rows of a tile
    int gate_stride, x_stride, dgate_stride, dx_stride;
    int counters;      // all of the handle's, and its words
    size_t n_words;
};

__device__ __forceinline__ void publish(uint64_t* at, float v, unsigned call)
{
    __hip_atomic_store(at, (uint64_t)call << 32 | __float_as_uint(v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ uint64_t look(const uint64_t* at) { return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

__device__ __forceinline__ float wait_for(const uint64_t* at, uint64_t seen, unsigned call)
{
    while ((unsigned)(seen >> 32) != call) {
        __builtin_amdgcn_s_sleep(1);
        seen = look(at);
    }
    return __uint_as_float((unsigned)seen);
}

__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ int bound(int v, int n) { return v < 0 ? 0 : v > n ? n : v; }

// What the words of a handle's control are; each counter has a line of memory of its own.
enum Control { kBlocksDrawn = 0, kDone = 1, kCounters = kScanLine };

// By one wave.
__device__ void ready(const TileArgs& a, unsigned call)
{
    const int lane = threadIdx.x & 63;
    if (lane == 0) a.control[kBlocksDrawn] = a.control[kDone] = 0;
    for (int i = lane; i < a.counters; i += 64) a.control[kCounters + i * kScanLine] = (uint64_t)call << 32;
}

__device__ __forceinline__ uint64_t draw(uint64_t* at) { return __hip_atomic_fetch_add(at, uint64_t(1), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// By the wave whose workgroup has drawn the last tile of a block of channels.
__device__ void last_tile(const TileArgs& a, unsigned call)
{
    uint64_t v = 0;
    if ((threadIdx.x & 63) == 0) v = draw(a.control + kBlocksDrawn);
    if (__builtin_amdgcn_readfirstlane((int)v) == a.blocks - 1 && call != ~0u) ready(a, call + 1);
}

// Where sequences enter and leave the rows of a tile.
template <int kRun>
struct Marks {
    int start;                                        // the row, of all, that the sequence of the tile's first row starts with
    unsigned enter[kMostRuns], leave[kMostRuns];      // a bit for each row of a run
    int entering[kMostRuns * kRun], leaving[kMostRuns * kRun];      // the sequences, where a bit is set
};

// By one wave; `off` is in shared memory where there are few enough sequences.
template <int kRun, bool kBack>
__device__ __forceinline__ void mark(const TileArgs& a, Marks<kRun>& m, int tile, const int* off)
{
    const int lane = threadIdx.x & 63, p0 = tile * a.rows, end = p0 + a.rows < a.n ? p0 + a.rows : a.n;
    for (int r = lane; r < a.rows / kRun; r += 64) m.enter[r] = m.leave[r] = 0;
    if (lane == 0) m.start = p0;
    wave_sync();
    const int from = kBack ? a.n - end : p0, to = kBack ? a.n - p0 : end;      // as tokens
    // how many sequences start at or before `from`: 64 at a time
    int lo = 0, hi = a.n_seq + 1;
    while (lo < hi) {
        const int step = (hi - lo + 63) / 64, at = lo + lane * step;
        const uint64_t not_yet = ~__ballot(at < hi && off[at < hi ? at : 0] <= from);
        const int c = not_yet ? __builtin_ctzll(not_yet) : 64;
        if (c == 0) break;
        hi = lo + c * step < hi ? lo + c * step : hi;
        lo += (c - 1) * step + 1;
    }
    for (int base = lo > 0 ? lo - 1 : 0; base < a.n_seq; base += 64) {
        const int s = base + lane;
        int end_here = a.n;
        if (s < a.n_seq) {
            const int b = bound(off[s], a.n), e = bound(off[s + 1], a.n);
            end_here = e;
            if (b < e) {
                const int enter = kBack ? a.n - e : b, leave = kBack ? a.n - 1 - b : e - 1;      // as rows
                if (enter >= p0 && enter < end) {
                    m.entering[enter - p0] = s;
                    atomicOr(&m.enter[(enter - p0) / kRun], 1u << (enter - p0) % kRun);
                }
                if (leave >= p0 && leave < end) {
                    m.leaving[leave - p0] = s;
                    atomicOr(&m.leave[(leave - p0) / kRun], 1u << (leave - p0) % kRun);
                }
                if (enter < p0 && leave >= p0) m.start = enter;
            }
        }
        if (__shfl(end_here, 63) >= to) break;
    }
    wave_sync();
}

// What follows from v is found anew where it is asked for, not kept in registers from before.
template <typename V>
__device__ __forceinline__ V anew(V v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// What a lane holds of its rows between the passes.
template <int N, int kRun, bool kBack>
struct Held {
    float f[kRun][N], b[kRun][N];           // forward: what the state is multiplied with, and what is added; backward: both sigmoids, and dy
    float by[kBack ? kRun : 1][N];          // dgate is D times this
};

// f(0), ... f(M - 1), as constants: what they index is in registers.
template <typename F, int... I>
__device__ __forceinline__ void each_of(F f, std::integer_sequence<int, I...>)
{
    (f(std::integral_constant<int, I>{}), ...);
}

template <int M, typename F>
__device__ __forceinline__ void each(F f)
{
    each_of(f, std::make_integer_sequence<int, M>{});
}

// The rows of one lane.  Whether sequences enter or leave at a row, or rows are not there, is asked for the wave; lanes choose by selects: no branch by
// lanes has what is held live on both of its sides.
template <typename T, int N, int kRun, bool kBack, bool kPast>
struct Rows {
    typedef Elements<T, N> Of;
    typedef Elements<float, N> State;
    const TileArgs& a;
    int q, first, rows_here;       // the lane's first row in the tile; the tile's lowest token, and how many there are from it
    int c;                         // first channel
    unsigned enter, leave;         // bits of rows
    const int *entering, *leaving; // sequences, where a bit is set

    // The bits that any lane has.
    __device__ __forceinline__ static unsigned of_wave(unsigned bits)
    {
        unsigned all = 0;
        for (uint64_t lanes = __ballot(bits != 0); lanes; lanes = __ballot((bits & ~all) != 0))
            all |= (unsigned)__builtin_amdgcn_readlane((int)bits, __builtin_ctzll(lanes));
        return all;
    }

    // Distances in bytes, from the tile's lowest token, of the lane's rows of an array, in 32 bits by the limit on strides: row j is `step` from the one
    // before.  Rows that are not there (past the last, or wrapped round) are the highest one that is, or lie between rows that are.
    struct Lines {
        unsigned from, step, most;
        __device__ __forceinline__ unsigned operator[](int j) const
        {
            const unsigned off = kBack ? from - j * step : from + j * step;
            return off < most ? off : most;
        }
    };

    __device__ __forceinline__ Lines lines(int stride) const
    {
        const unsigned step = (unsigned)stride * (unsigned)sizeof(T), at = (unsigned)c * (unsigned)sizeof(T);
        return {(unsigned)(kBack ? rows_here - 1 - q : q) * step + at, step, (unsigned)(rows_here - 1) * step + at};
    }

    template <typename P>
    __device__ __forceinline__ static auto* byte(P* p, unsigned off)
    {
        typedef std::conditional_t<std::is_const<P>::value, const char, char> Byte;
        return reinterpret_cast<P*>(reinterpret_cast<Byte*>(p) + off);
    }

    __device__ __forceinline__ void load(Of (&to)[kRun], const void* p, int stride) const
    {
        const T* const base = static_cast<const T*>(p) + (int64_t)first * stride;
        const Lines at = lines(stride);
        each<kRun>([&](auto j) { to[j] = load_of<kPast, T, N>(byte(base, at[j])); });
    }

    // The state of row j's sequence; the first one's for lanes that have no mark there.
    __device__ __forceinline__ State state_of(const float* state, const int* seq, bool here, int j) const
    {
        return state ? State::load(state + (int64_t)(here ? seq[q + j] : 0) * a.in.width + c) : State{};
    }

    struct Raw {
        Of g[kRun], x[kRun], up[kBack ? kRun : 1], was[kBack ? kRun : 1];
    };

    __device__ __forceinline__ void read(Raw& r) const
    {
        const ScanIn& in = a.in;
        load(r.g, in.gate, a.gate_stride);
        load(r.x, in.x, a.x_stride);
        if constexpr (kBack) {
            if (in.dy) load(r.up, in.dy, in.width);
            else each<kRun>([&](auto j) { r.up[j] = Of{}; });
            // (the row before the first token is not there, and not asked for: a sequence leaves at it)
            const T* const base = static_cast<const T*>(in.y) + (int64_t)(first - 1) * in.width;
            const Lines at = lines(in.width);
            const unsigned least = first == 0 ? at.step : 0;
            each<kRun>([&](auto j) {
                const unsigned off = at[j];
                r.was[j] = load_of<kPast, T, N>(byte(base, off < least ? off + least : off));
            });
        }
    }

    __device__ __forceinline__ void first_pass(const Raw& r, Held<N, kRun, kBack>& held, float (&F)[N], float (&B)[N]) const
    {
        const ScanIn& in = a.in;
        const bool some_missing = rows_here < a.rows;
        const unsigned any_enter = of_wave(enter), any_leave = kBack ? of_wave(leave) : 0;
        each<kRun>([&](auto j) {
            float before[N] = {};
            if constexpr (kBack) {
                const bool here = leave >> j & 1;
                each<N>([&](auto e) { before[e] = (float)r.was[j].v[e]; });
                if (any_leave >> j & 1) {
                    const State h0 = state_of(in.h0, leaving, here, j);
                    each<N>([&](auto e) { before[e] = here ? +h0.v[e] : +before[e]; });
                }
            }
            float f[N];
            const bool there = !some_missing || q + j < rows_here;
            each<N>([&](auto e) {
                const float v = (float)r.x[j].v[e];
                const Gate k = gate_of((float)r.g[j].v[e]);
                f[e] = k.keep;
                if constexpr (!kBack) held.b[j][e] = k.take * v;
                else {
                    held.f[j][e] = anew(packed(k));
                    held.b[j][e] = (float)r.up[j].v[e];
                    held.by[j][e] = anew(k.keep * k.take * (before[e] - v));
                }
            });
            if (some_missing)      // rows that are not there change nothing (and nothing is written for them)
                each<N>([&](auto e) {
                    f[e] = there ? +f[e] : 1.0f;
                    held.b[j][e] = there ? +held.b[j][e] : 0.0f;
                });
            if constexpr (!kBack) each<N>([&](auto e) { held.f[j][e] = f[e]; });
            if (j == 0) each<N>([&](auto e) { F[e] = 1.0f; B[e] = 0.0f; });
            const bool here = enter >> j & 1;
            if (any_enter >> j & 1) {
                const State from = state_of(kBack ? in.dh : in.h0, entering, here, j);
                each<N>([&](auto e) {
                    B[e] = here ? +from.v[e] : +B[e];
                    F[e] = here ? 0.0f : +F[e];
                });
            }
            each<N>([&](auto e) {
                B[e] = kBack ? f[e] * (held.b[j][e] + B[e]) : fmaf(f[e], B[e], held.b[j][e]);
                F[e] *= f[e];
            });
        });
    }

    __device__ __forceinline__ void second_pass(const Held<N, kRun, kBack>& held, float (&h)[N], bool on, int lowest, int highest) const
    {
        const unsigned any_enter = of_wave(enter), any_leave = of_wave(leave);
        const Lines at_y = lines(kBack ? a.dx_stride : a.in.width), at_g = lines(a.dgate_stride);
        const bool edge = rows_here < a.rows || first < lowest || first + rows_here > highest;      // some rows are not there, or of no sequence
        each<kRun>([&](auto j) {
            const bool here = enter >> j & 1, leaves = leave >> j & 1;
            if (any_enter >> j & 1) {
                const State from = state_of(kBack ? a.in.dh : a.in.h0, entering, here, j);
                each<N>([&](auto e) { h[e] = here ? +from.v[e] : +h[e]; });
            }
            Of o, p;
            each<N>([&](auto e) {
                if constexpr (kBack) {
                    const Gate k = unpacked(held.f[j][e]);
                    const float d = held.b[j][e] + h[e];
                    o.v[e] = (T)(d * k.take);
                    p.v[e] = (T)(d * held.by[j][e]);
                    h[e] = k.keep * d;
                } else {
                    h[e] = fmaf(held.f[j][e], h[e], held.b[j][e]);
                    o.v[e] = (T)h[e];
                }
            });
            bool write = on;
            if (edge) {
                const int t = first + (kBack ? rows_here - 1 - (q + j) : q + j);
                write = on && q + j < rows_here && t >= lowest && t < highest;
            }
            if (write) {
                if constexpr (!kBack) {
                    if (a.y) store_of<kPast>(byte(static_cast<T*>(a.y) + (int64_t)first * a.in.width, at_y[j]), o);
                } else {
                    store_of<kPast>(byte(static_cast<T*>(a.dx) + (int64_t)first * a.dx_stride, at_y[j]), o);
                    store_of<kPast>(byte(static_cast<T*>(a.dgate) + (int64_t)first * a.dgate_stride, at_g[j]), p);
                }
            }
            if (a.last && any_leave >> j & 1) {
                State v;
                each<N>([&](auto e) { v.v[e] = h[e]; });
                if (leaves && on) v.store(a.last + (int64_t)leaving[q + j] * a.in.width + c);
            }
        });
    }
};

constexpr int kJoined = 4;      // runs that a thread joins for a channel

// Stretches one after the other, kJoined at a time: `step`(which, whether a sequence enters in it, F, B).
template <typename F>
__device__ __forceinline__ void each_stretch(int n, int channels, int ch, const bool* cut, const float* f, const float* b, F step)
{
#pragma unroll 1
    for (int r = 0; r < n; r += kJoined) {
        float rf[kJoined], rb[kJoined];
#pragma unroll
        for (int u = 0; u < kJoined; ++u) {
            rf[u] = f[(r + u) * channels + ch];
            rb[u] = b[(r + u) * channels + ch];
        }
#pragma unroll
        for (int u = 0; u < kJoined; ++u) step(r + u, cut[r + u], rf[u], rb[u]);
    }
}

// (F, B) of a channel of the tile from those of its stretches, published; the state that it starts from; those that its stretches start from, in the place of F.
__device__ __forceinline__ void join(const TileArgs& a, int tile, int start, unsigned call, const bool* cuts, float* f, const float* b, int n, int channels, int block,
                                     int ch)
{
    const int p0 = tile * a.rows;
    const int64_t pitch = (int64_t)a.blocks * channels, word = block * channels + ch;
    float tf = 1, tb = 0;
    bool cut = false;
    each_stretch(n, channels, ch, cuts, f, b, [&](int, bool here, float rf, float rb) {
        tb = here ? rb : fmaf(rf, tb, rb);
        tf = here ? 0.0f : tf * rf;
        cut = cut || here;
    });
    const bool more = tile + 1 < a.tiles;
    uint64_t* const sums = a.sums + word;
    if (more) {
        publish(sums + (int64_t)tile * 2 * pitch, tf, call);
        publish(sums + ((int64_t)tile * 2 + 1) * pitch, tb, call);
        __atomic_signal_fence(__ATOMIC_SEQ_CST);      // (before anything is waited for)
    }
    float state = 0;
    if (start < p0) {
        const int from = start / a.rows, group = tile / kGroup * kGroup;
        // what it starts from: the end of the tile that the sequence starts in, or the state at a group's end; then the tiles since, which are joined
        // first: nothing but a word and a product is between the state at a group's end and that at the next
        const uint64_t* const begin = from >= group ? sums + ((int64_t)from * 2 + 1) * pitch : a.states + (int64_t)(group / kGroup - 1) * pitch + word;
        const uint64_t seen = look(begin);
        float cf = 1, cb = 0;
        for (int k = from >= group ? from + 1 : group; k < tile; k += 4) {
            uint64_t sf[4], sb[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int64_t w = (int64_t)(k + u < tile ? k + u : k) * 2;
                sf[u] = look(sums + w * pitch);
                sb[u] = look(sums + (w + 1) * pitch);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (k + u < tile) {
                    const int64_t w = (int64_t)(k + u) * 2;
                    const float kf = wait_for(sums + w * pitch, sf[u], call), kb = wait_for(sums + (w + 1) * pitch, sb[u], call);
                    cb = fmaf(kf, cb, kb);
                    cf *= kf;
                }
        }
        state = fmaf(cf, wait_for(begin, seen, call), cb);
    }
    if (more && tile % kGroup == kGroup - 1) publish(a.states + (int64_t)(tile / kGroup) * pitch + word, cut ? tb : fmaf(tf, state, tb), call);
    each_stretch(n, channels, ch, cuts, f, b, [&](int r, bool here, float rf, float rb) {
        f[r * channels + ch] = state;
        state = here ? rb : fmaf(rf, state, rb);
    });
}

// Sequences of no token: their states stay.
__device__ void stay(const TileArgs& a, int s0, const float* state)
{
    const int s = s0 + (threadIdx.x & 63), width = a.in.width;
    uint64_t none = __ballot(s < a.n_seq && bound(a.in.off[s < a.n_seq ? s : 0], a.n) >= bound(a.in.off[s < a.n_seq ? s + 1 : 0], a.n));
    for (; none; none &= none - 1) {
        const int64_t at = (int64_t)(s0 + __builtin_ctzll(none)) * width;
        for (int c = threadIdx.x; c < width; c += kThreads) a.last[at + c] = state ? state[at + c] : 0.0f;
    }
}

template <typename T, int N, int kRun, bool kBack, bool kPast>
__global__ __launch_bounds__(kThreads) void k_scan_tiles(TileArgs a)
{
    typedef Rows<T, N, kRun, kBack, kPast> Of;
    __shared__ float part_f[kThreads * N], part_b[kThreads * N], stretch_f[kThreads], stretch_b[kThreads];
    __shared__ bool cuts[kMostRuns / kJoined];
    __shared__ Marks<kRun> m;
    __shared__ uint64_t drawn;
    __shared__ int near_off[kNearOffsets];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const ScanIn& in = a.in;
    const int width = in.width, workers = a.tiles * a.blocks;
    if (blockIdx.x >= (unsigned)workers) return stay(a, (int)(blockIdx.x - workers) * 64, kBack ? in.dh : in.h0);
    const int block = blockIdx.x % a.blocks;
    const bool few = a.n_seq < kNearOffsets;
    if (few)
        for (int i = tid; i <= a.n_seq; i += kThreads) near_off[i] = in.off[i];
    if (tid == 0) drawn = draw(a.control + kCounters + block * kScanLine);
    __syncthreads();
    const int tile = __builtin_amdgcn_readfirstlane((int)(unsigned)drawn), p0 = tile * a.rows;
    const unsigned call = __builtin_amdgcn_readfirstlane((int)(drawn >> 32));
    const int l = tid & ((1 << a.lg) - 1), run = tid >> a.lg, channels = a.lanes * N;
    // channels: those of a last lane that is not whole reach back, and both come to the same values
    const int c_own = block * channels + (l < a.lanes ? l : 0) * N, c = c_own + N > width ? width - N : c_own;
    const bool on = l < a.lanes && c_own < width;
    const int q = run * kRun, rows_here = a.n - p0 < a.rows ? a.n - p0 : a.rows, first = kBack ? a.n - p0 - rows_here : p0;
    Held<N, kRun, kBack> held;
    {
        float F[N], B[N];
        typename Of::Raw raw;
        Of{a, q, first, rows_here, c, 0, 0, nullptr, nullptr}.read(raw);
        if (wave == kWaves - 1) {
            if (few) mark<kRun, kBack>(a, m, tile, near_off);
            else mark<kRun, kBack>(a, m, tile, in.off);
        } else if (wave == 0 && tile == a.tiles - 1) last_tile(a, call);
        __syncthreads();
        Of{a, anew(q), first, rows_here, anew(c), m.enter[run], m.leave[run], m.entering, m.leaving}.first_pass(raw, held, F, B);
        if (l < a.lanes) each<N>([&](auto e) {
            part_f[run * channels + l * N + e] = F[e];
            part_b[run * channels + l * N + e] = B[e];
        });
    }
    __syncthreads();
    {
        // four runs of a channel by each thread, then those by a thread for each channel, and back
        const int stretch = tid / channels, ch = tid - stretch * channels, stretches = (kThreads >> a.lg) / kJoined;
        float rf[kJoined], rb[kJoined], f = 1, b = 0;
        bool enters[kJoined], cut = false;
        if (stretch < stretches) {
#pragma unroll
            for (int u = 0; u < kJoined; ++u) {
                const int r = stretch * kJoined + u;
                rf[u] = part_f[r * channels + ch];
                rb[u] = part_b[r * channels + ch];
                enters[u] = m.enter[r] != 0;
                b = enters[u] ? rb[u] : fmaf(rf[u], b, rb[u]);
                f = enters[u] ? 0.0f : f * rf[u];
                cut = cut || enters[u];
            }
            stretch_f[tid] = f;
            stretch_b[tid] = b;
            if (ch == 0) cuts[stretch] = cut;
        }
        __syncthreads();
        if (tid < channels) join(a, tile, m.start, call, cuts, stretch_f, stretch_b, stretches, channels, block, tid);
        __syncthreads();
        if (stretch < stretches) {
            float state = stretch_f[tid];
#pragma unroll
            for (int u = 0; u < kJoined; ++u) {
                part_f[(stretch * kJoined + u) * channels + ch] = state;
                state = enters[u] ? rb[u] : fmaf(rf[u], state, rb[u]);
            }
        }
    }
    __syncthreads();
    {
        float h[N];
        each<N>([&](auto e) { h[e] = part_f[l < a.lanes ? run * channels + l * N + e : 0]; });
        const Of rows{a, anew(q), first, rows_here, anew(c), m.enter[run], m.leave[run], m.entering, m.leaving};
        const int lowest = bound(in.off[0], a.n), highest = bound(in.off[a.n_seq], a.n);
        rows.second_pass(held, h, on, lowest, highest);
    }
    // after the last number that there is all words are cleared, and 0 is no call's number
    if (call != ~0u) return;
    __syncthreads();
    if (tid == 0) drawn = draw(a.control + kDone);
    __syncthreads();
    if (drawn != (uint64_t)workers - 1) return;
    for (size_t i = tid; i < a.n_words; i += kThreads) a.sums[i] = 0;
    if (wave == 0) ready(a, 1);
}

// ---- a token of every sequence ------------------------------------------------------------------

// Bound by memory, most of it the states in single precision: 4 096 requests x 1 024 in bfloat16 59 MB, 10 us, backward 101 MB, 20.5 us.  Pieces of N channels of a row; a last one
// that is not whole goes by single channels, as states may be in place.
template <typename T, int N, bool kBack>
__global__ __launch_bounds__(kBlock) void k_scan_step(ScanIn in, T* y, T* dgate, T* dx, float* last, int pieces)
{
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x, s = i / pieces;
    if (s >= in.n_seq) return;
    const int c = (int)(i - s * pieces) * N;
    const auto go = [&](auto count, int c) {
        constexpr int M = decltype(count)::value;
        typedef Elements<T, M> Of;
        typedef Elements<float, M> State;
        const int64_t at = s * in.width + c;
        const Of g = Of::load(static_cast<const T*>(in.gate) + s * in.gate_stride + c), x = Of::load(static_cast<const T*>(in.x) + s * in.x_stride + c);
        State h0{}, h;
        if (in.h0) h0 = State::load(in.h0 + at);
        if (!kBack) {
            Of o;
#pragma unroll
            for (int e = 0; e < M; ++e) {
                const Gate k = gate_of((float)g.v[e]);
                h.v[e] = fmaf(k.keep, h0.v[e], k.take * (float)x.v[e]);
                o.v[e] = (T)h.v[e];
            }
            if (y) o.store(y + at);
        } else {
            Of up{}, og, ox;
            State dh{};
            if (in.dy) up = Of::load(static_cast<const T*>(in.dy) + at);
            if (in.dh) dh = State::load(in.dh + at);
#pragma unroll
            for (int e = 0; e < M; ++e) {
                const Gate k = gate_of((float)g.v[e]);
                const float d = (float)up.v[e] + dh.v[e], by = d * k.take;
                ox.v[e] = (T)by;
                og.v[e] = (T)(by * k.keep * (h0.v[e] - (float)x.v[e]));
                h.v[e] = d * k.keep;
            }
            ox.store(dx + s * in.dx_stride + c);
            og.store(dgate + s * in.dgate_stride + c);
        }
        if (last) h.store(last + at);
    };
    if (c + N <= in.width) go(std::integral_constant<int, N>{}, c);
    else
        for (int one = c; one < in.width; ++one) go(std::integral_constant<int, 1>{}, one);
}

template <typename T, int N, int kRun, bool kBack, bool kPast>
int launch_tiles(gr_tokens* h, TileArgs a, hipStream_t s)
{
    static_assert((kThreads >> kScanLanesLog) % (kJoined * kJoined) == 0, "runs and stretches are joined four at a time");
    static_assert((int64_t)kMostRuns * kRun * GR_MAX_STRIDE <= int64_t(1) << 30, "distances within a tile are in 32 bits, in bytes");
    a.rows = (kThreads >> a.lg) * kRun;
    a.tiles = (int)(((int64_t)a.n + a.rows - 1) / a.rows);
    const int64_t pitch = (int64_t)a.blocks * a.lanes * N;
    a.states = a.sums + (int64_t)a.tiles * 2 * pitch;
    if (a.blocks > a.counters || (size_t)(((int64_t)a.tiles * 2 + a.tiles / kGroup + 1) * pitch) > a.n_words) return GR_ERR_TOO_LARGE;
    const int64_t total = (int64_t)a.tiles * a.blocks + (a.last ? ((int64_t)a.n_seq + 63) / 64 : 0);
    if (total > kMostBlocks * kBlock / kThreads) return GR_ERR_TOO_LARGE;
    if (total == 0) return GR_OK;
    k_scan_tiles<T, N, kRun, kBack, kPast><<<(unsigned)total, kThreads, 0, s>>>(a);
    return launched();
}

template <bool kBack>
int launch(gr_tokens* h, const ScanIn& in, int dtype, void* y, void* dgate, void* dx, float* last, hipStream_t s)
{
    if (!in.off)
        return by_type(dtype, [&](auto t) {
            typedef decltype(t) T;
            constexpr int N = 4;
            const int pieces = (in.width + N - 1) / N;
            const int64_t blocks = (in.n_seq * pieces + kBlock - 1) / kBlock;
            if (blocks > kMostBlocks) return (int)GR_ERR_TOO_LARGE;
            k_scan_step<T, N, kBack><<<(unsigned)blocks, kBlock, 0, s>>>(in, static_cast<T*>(y), static_cast<T*>(dgate), static_cast<T*>(dx), last, pieces);
            return launched();
        });
    TileArgs a{};
    a.in = in; a.y = y; a.dgate = dgate; a.dx = dx; a.last = last;
    a.gate_stride = (int)in.gate_stride; a.x_stride = (int)in.x_stride; a.dgate_stride = (int)in.dgate_stride; a.dx_stride = (int)in.dx_stride;
    a.n = (int)in.n; a.n_seq = (int)in.n_seq;
    a.control = h->control; a.counters = h->counters; a.sums = h->words; a.n_words = h->n_words;
    const int per = in.width < kScanChannels ? 1 : kScanChannels, pieces = (in.width + per - 1) / per;
    constexpr int kRun = kBack ? kRunBackward : kRunForward;
    const auto split = [&](int most) {
        a.blocks = (pieces + most - 1) / most;
        a.lanes = (pieces + a.blocks - 1) / a.blocks;
        a.lg = kLeastLanesLog;
        while ((1 << a.lg) < a.lanes) ++a.lg;
        const int rows = (kThreads >> a.lg) * kRun;
        return (in.n + rows - 1) / rows * a.blocks;
    };
    const int64_t tiles = split(1 << kScanLanesLog);
    const bool few = tiles <= kFewTiles;
    const int bytes = in.width * (int)size_of(dtype), line = bytes % 128 == 0 ? 128 : bytes % 64 == 0 ? 64 : 1;
    const auto lanes_of = [&](int most) { return (pieces + most - 1) / most * most; };
    const bool fewer = lanes_of(1 << kFewLanesLog) < lanes_of(1 << kScanLanesLog), whole = in.width % (kScanChannels << kFewLanesLog) == 0;
    if ((line > 1 && fewer) || (whole && (bytes <= kFewLanesBytes || tiles <= kFewLanesTiles))) split(1 << kFewLanesLog);
    const int per_line = line / (kScanChannels * (int)size_of(dtype));
    if (a.blocks > 1 && per_line > 1) a.lanes = (a.lanes + per_line - 1) / per_line * per_line;
    return by_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        if (per == 1) return launch_tiles<T, 1, kRun, kBack, false>(h, a, s);
        if (few) return launch_tiles<T, kScanChannels, kRunFew, kBack, false>(h, a, s);
        return past_cache(in.n * in.width * (int64_t)sizeof(T) * (kBack ? 6 : 3)) ? launch_tiles<T, kScanChannels, kRun, kBack, true>(h, a, s)
                                                                                 : launch_tiles<T, kScanChannels, kRun, kBack, false>(h, a, s);
    });
}

}  // namespace

int scan_counters(int width) { return (width / kScanChannels >> kFewLanesLog) + 1; }

size_t scan_words(int64_t n, int width)
{
    // a word for F and one for B of every channel of every tile, and one of every group's state: of the least tiles and the most channels in use
    // (all blocks have as many lanes, and a block that is not the only one 32 at most)
    constexpr int kWide = kScanChannels << kScanLanesLog;
    const int64_t channels = width > kWide ? (width + (int64_t)kWide - 1) / kWide * kWide : width + kScanChannels - 1;
    const auto words = [&](int64_t tiles) { return (size_t)((tiles * 2 + tiles / kGroup + 1) * channels); };
    const auto tiles = [&](int run) {
        const int64_t rows = (int64_t)(kThreads >> kScanLanesLog) * run;
        return (n + rows - 1) / rows;
    };
    constexpr int kMost = kRunForward > kRunBackward ? kRunForward : kRunBackward, kLeast = kRunForward < kRunBackward ? kRunForward : kRunBackward;
    // runs of few rows are for few tiles
    const int64_t few = tiles(kRunFew), of_few = kFewTiles * ((kMost + kRunFew - 1) / kRunFew);
    const size_t a = words(tiles(kLeast)), b = words(few < of_few ? few : of_few);
    return a > b ? a : b;
}

int launch_scan(gr_tokens* h, const ScanIn& in, int dtype, void* y, float* last, hipStream_t s)
{
    return launch<false>(h, in, dtype, y, nullptr, nullptr, last, s);
}

int launch_scan_backward(gr_tokens* h, const ScanIn& in, int dtype, void* dgate, void* dx, float* dh0, hipStream_t s)
{
    return launch<true>(h, in, dtype, nullptr, dgate, dx, dh0, s);
}

}  // namespace gr
