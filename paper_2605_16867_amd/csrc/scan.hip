// A gated recurrence along sequences of tokens, forward and backward (gfx950).
//
//   f = sigmoid(gate), i = sigmoid(-gate);  h_t = f_t h_{t-1} + i_t x_t
//   D_t = dy_t + c_{t+1}, c_t = f_t D_t;  dx_t = i_t D_t, dgate_t = f_t i_t D_t (h_{t-1} - x_t)
#include <type_traits>

#include "tokens.h"

namespace gr {
namespace {

constexpr int kBlock = 256;

struct Gate {
    float keep, take;      // sigmoid(gate), sigmoid(-gate)
};

// Both from exp(-|gate|) =: e, as 1 / (1 + e) and e / (1 + e): neither is a difference, so both have all their digits however far the gate is from 0.
// The exponent's rounding, |gate| log2(e) * 2^-24, is made good where results are in single precision.  (A gate that is no number stays one.)
template <typename T>
__device__ __forceinline__ Gate gate_of(float g)
{
    constexpr float kLog2e = 1.44269504089f, kLog2eRest = 1.92596299e-8f, kLn2 = 0.693147181f;
    float a = fabsf(g);
    a = a > 88.0f ? 88.0f : a;      // (behind that e is no whole number of single precision, and 0 is as good)
    const float p = a * -kLog2e;
    float e = __builtin_amdgcn_exp2f(p);
    if (sizeof(T) == 4) e = fmaf(e, fmaf(a, -kLog2eRest, fmaf(a, -kLog2e, -p)) * kLn2, e);
    const float near = __builtin_amdgcn_rcpf(1.0f + e), far = e * near;
    return g >= 0 ? Gate{near, far} : Gate{far, near};
}

// ---- many tokens: tiles of rows -----------------------------------------------------------------
//
// Rows are taken in the direction of the recurrence (backward: the last one first), a tile of them by a workgroup, a run of kRun by the lanes
// that share a row; a lane has N channels.  A stretch of rows takes a state c to F c + B, F the product of its f.  A tile
//   1. reads its rows once, holds f and what is added in registers, and finds (F, B) of its runs, and of itself, which it publishes;
//   2. finds the state that it starts from: of the tiles since the one that its sequence starts in, or since the last multiple of kGroup tiles, whose
//      last tile publishes the state itself;
//   3. goes through its rows once more, in registers, and writes.
// The order in which stretches are joined hangs on the places of rows and sequences alone, so the bits are the same every time.
//
// Published words are 64 bits, a value and the number of the call: complete or not there, with nothing to order between words.  Workgroups take
// tiles by a ticket, one counter for each block of channels, so that those that a tile waits for are always held by workgroups that run already, and
// wait for none behind them: every wait ends.  A counter holds the number of the call and the next ticket in one word; whoever draws the last one of
// all counters sets them for the next call (all others have what they need by then).  Draws at one counter follow each other in 43 ns: with one for all
// blocks, and another for workgroups that are done, 262 144 tokens of 1 024 took 1.4 ms whatever else was done.

constexpr int kTileBlock = 512, kGroup = 16, kLeastLanesLog = 2;
constexpr int kMostRuns = kTileBlock >> kLeastLanesLog;

struct TileArgs {
    ScanIn in;
    void *y, *dgate, *dx;
    float* last;      // states after the last rows (backward: gradients of the first states)
    uint64_t *sums, *states;
    uint64_t* control;      // see Control
    int n, n_seq, tiles, blocks, lanes, lg, rows;      // blocks of channels, lanes of a row in use, log2 of lanes of a row, rows of a tile
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

__device__ void ready(const TileArgs& a, unsigned call)
{
    if (threadIdx.x == 0) a.control[kBlocksDrawn] = a.control[kDone] = 0;
    for (int i = threadIdx.x; i < a.counters; i += kTileBlock) a.control[kCounters + i * kScanLine] = (uint64_t)call << 32;
}

__device__ __forceinline__ uint64_t draw(uint64_t* at) { return __hip_atomic_fetch_add(at, uint64_t(1), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Where sequences enter and leave the rows of a tile.
struct Marks {
    unsigned enter[kMostRuns], leave[kMostRuns];      // a bit for each row of a run
    int start;                                        // the row, of all, that the sequence of the tile's first row starts with
};

// The wave's own runs: rows q0 .. q0 + count - 1 of the tile, whose first row is row p0 of all.  `entering` and `leaving` get the sequences.
template <int kRun, bool kBack>
__device__ void mark(const TileArgs& a, Marks& m, int* entering, int* leaving, int p0, int q0, int count)
{
    const int lane = threadIdx.x & 63, first = p0 + q0, end = first + count < a.n ? first + count : a.n;
    for (int r = lane; r < count / kRun; r += 64) m.enter[q0 / kRun + r] = m.leave[q0 / kRun + r] = 0;
    if (q0 == 0 && lane == 0) m.start = p0;
    wave_sync();
    if (first >= end) return;
    const int from = kBack ? a.n - end : first, to = kBack ? a.n - first : end;      // as tokens
    // how many sequences start at or before `from`: 64 at a time
    int lo = 0, hi = a.n_seq + 1;
    while (lo < hi) {
        const int step = (hi - lo + 63) / 64, at = lo + lane * step;
        const uint64_t not_yet = ~__ballot(at < hi && a.in.off[at < hi ? at : 0] <= from);
        const int c = not_yet ? __builtin_ctzll(not_yet) : 64;
        if (c == 0) break;
        hi = lo + c * step < hi ? lo + c * step : hi;
        lo += (c - 1) * step + 1;
    }
    for (int base = lo > 0 ? lo - 1 : 0; base < a.n_seq; base += 64) {
        const int s = base + lane;
        int end_here = a.n;
        if (s < a.n_seq) {
            const int b = bound(a.in.off[s], a.n), e = bound(a.in.off[s + 1], a.n);
            end_here = e;
            if (b < e) {
                const int enter = kBack ? a.n - e : b, leave = kBack ? a.n - 1 - b : e - 1;      // as rows
                if (enter >= first && enter < end) {
                    entering[enter - p0] = s;
                    atomicOr(&m.enter[(enter - p0) / kRun], 1u << (enter - p0) % kRun);
                }
                if (leave >= first && leave < end) {
                    leaving[leave - p0] = s;
                    atomicOr(&m.leave[(leave - p0) / kRun], 1u << (leave - p0) % kRun);
                }
                if (q0 == 0 && enter < p0 && leave >= p0) m.start = enter;
            }
        }
        if (__shfl(end_here, 63) >= to) break;
    }
    wave_sync();
}

// Rows of T as the lane has them: N channels from c, of which it writes those from `own`.
template <typename T, int N>
__device__ __forceinline__ void store(T* at, const float (&v)[N], int own)
{
    Elements<T, N> o;
#pragma unroll
    for (int e = 0; e < N; ++e) o.v[e] = (T)v[e];
    if (own == 0) o.store(at);
    else
        for (int e = 0; e < N; ++e)
            if (e >= own) at[e] = o.v[e];
}

template <typename T, int N, int kRun, bool kBack>
__global__ __launch_bounds__(kTileBlock) void k_scan_tiles(TileArgs a)
{
    typedef Elements<T, N> Of;
    __shared__ float part_f[kTileBlock * N], part_b[kTileBlock * N];
    __shared__ int entering[kMostRuns * kRun], leaving[kMostRuns * kRun];
    __shared__ Marks m;
    __shared__ uint64_t drawn;
    __shared__ bool last_drawn;
    const int tid = threadIdx.x;
    const ScanIn& in = a.in;
    const int width = in.width;
    if (blockIdx.x >= (unsigned)a.tiles * a.blocks) {      // sequences of no token: their states stay
        const int lane = tid & 63, s0 = (int)(blockIdx.x - (unsigned)a.tiles * a.blocks) * 64, s = s0 + lane;
        const float* const state = kBack ? in.dh : in.h0;
        uint64_t none = __ballot(s < a.n_seq && bound(in.off[s < a.n_seq ? s : 0], a.n) >= bound(in.off[s < a.n_seq ? s + 1 : 0], a.n));
        for (; none; none &= none - 1) {
            const int64_t at = (int64_t)(s0 + __builtin_ctzll(none)) * width;
            for (int c = tid; c < width; c += kTileBlock) a.last[at + c] = state ? state[at + c] : 0.0f;
        }
        return;
    }
    const int block = blockIdx.x % a.blocks;
    if (tid == 0) {
        drawn = draw(a.control + kCounters + block * kScanLine);
        last_drawn = (int)(unsigned)drawn == a.tiles - 1 && draw(a.control + kBlocksDrawn) == (uint64_t)a.blocks - 1;
    }
    __syncthreads();
    const int tile = (int)(unsigned)drawn;
    const unsigned now = (unsigned)(drawn >> 32);
    if (last_drawn && now != ~0u) ready(a, now + 1);
    {
        const int p0 = tile * a.rows;
        const int l = tid & ((1 << a.lg) - 1), run = tid >> a.lg, runs = kTileBlock >> a.lg, channels = a.lanes * N;
        const int wave_rows = (64 >> a.lg) * kRun;
        mark<kRun, kBack>(a, m, entering, leaving, p0, (tid >> 6) * wave_rows, wave_rows);
        const int lowest = bound(in.off[0], a.n), highest = bound(in.off[a.n_seq], a.n);
        // channels: those of the last lane reach back, and it writes only its own
        const int c_own = block * channels + l * N, c = c_own + N > width ? width - N : c_own, own = c_own - c;
        const bool on = l < a.lanes && c_own < width;
        const unsigned enter = m.enter[run], leave = m.leave[run];
        float f[kRun][N], b[kRun][N];      // backward: b is dy
        Of xs[kBack ? kRun : 1], before[kBack ? kRun : 1];
        float i_of[kBack ? kRun : 1][N];
        float F[N], B[N];
#pragma unroll
        for (int e = 0; e < N; ++e) { F[e] = 1; B[e] = 0; }
        const int q = run * kRun, p_run = p0 + q;
        const auto token_of = [&](int j) { return kBack ? a.n - 1 - (p_run + j) : p_run + j; };
        if (on && p_run < a.n) {
            Of g[kRun], v[kRun];
#pragma unroll
            for (int j = 0; j < kRun; ++j) {
                const int t0 = token_of(j), t = t0 < 0 ? 0 : t0 >= a.n ? a.n - 1 : t0;
                g[j] = Of::load(static_cast<const T*>(in.gate) + t * in.gate_stride + c);
                if (!kBack) v[j] = Of::load(static_cast<const T*>(in.x) + t * in.x_stride + c);
                else {
                    v[j] = Of{};
                    if (in.dy) v[j] = Of::load(static_cast<const T*>(in.dy) + (int64_t)t * width + c);
                    xs[j] = Of::load(static_cast<const T*>(in.x) + t * in.x_stride + c);
                    before[j] = Of::load(static_cast<const T*>(in.y) + (int64_t)(t > 0 ? t - 1 : 0) * width + c);
                }
            }
#pragma unroll
            for (int j = 0; j < kRun; ++j) {
                const bool there = p_run + j < a.n;
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const Gate k = gate_of<T>((float)g[j].v[e]);
                    f[j][e] = there ? k.keep : 1.0f;
                    if (!kBack) b[j][e] = there ? k.take * (float)v[j].v[e] : 0.0f;
                    else {
                        i_of[j][e] = k.take;
                        b[j][e] = there ? (float)v[j].v[e] : 0.0f;
                    }
                }
                if (enter >> j & 1) {
                    const float* const state = kBack ? in.dh : in.h0;
                    const int64_t at = (int64_t)entering[q + j] * width + c;
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const float from = state ? state[at + e] : 0.0f;
                        b[j][e] = kBack ? b[j][e] + from : fmaf(f[j][e], from, b[j][e]);
                        B[e] = kBack ? f[j][e] * b[j][e] : b[j][e];
                        F[e] = 0;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        B[e] = kBack ? f[j][e] * (b[j][e] + B[e]) : fmaf(f[j][e], B[e], b[j][e]);
                        F[e] *= f[j][e];
                    }
                }
            }
        }
        if (l < a.lanes) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                part_f[run * channels + l * N + e] = F[e];
                part_b[run * channels + l * N + e] = B[e];
            }
        }
        __syncthreads();
        for (int ch = tid; ch < channels; ch += kTileBlock) {
            const int64_t pitch = (int64_t)a.blocks * channels, word = block * channels + ch;
            float tf = 1, tb = 0;
            bool cut = false;
            for (int r = 0; r < runs; ++r) {
                const float rf = part_f[r * channels + ch], rb = part_b[r * channels + ch];
                const bool here = m.enter[r] != 0;
                tb = here ? rb : fmaf(rf, tb, rb);
                tf = here ? 0.0f : tf * rf;
                cut = cut || here;
            }
            const bool more = tile + 1 < a.tiles;
            uint64_t* const sums = a.sums + word;
            if (more) {
                publish(sums + (int64_t)tile * 2 * pitch, tf, now);
                publish(sums + ((int64_t)tile * 2 + 1) * pitch, tb, now);
                __atomic_signal_fence(__ATOMIC_SEQ_CST);      // (before anything is waited for)
            }
            float state = 0;
            if (m.start < p0) {
                const int from = m.start / a.rows, group = tile / kGroup * kGroup;
                int k = from;
                if (from >= group) {
                    const uint64_t* const at = sums + ((int64_t)k++ * 2 + 1) * pitch;
                    state = wait_for(at, look(at), now);
                } else {
                    const uint64_t* const at = a.states + (int64_t)(group / kGroup - 1) * pitch + word;
                    k = group;
                    state = wait_for(at, look(at), now);
                }
                for (; k < tile; k += 4) {
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
                            const float kf = wait_for(sums + w * pitch, sf[u], now), kb = wait_for(sums + (w + 1) * pitch, sb[u], now);
                            state = fmaf(kf, state, kb);
                        }
                }
            }
            if (more && tile % kGroup == kGroup - 1) publish(a.states + (int64_t)(tile / kGroup) * pitch + word, cut ? tb : fmaf(tf, state, tb), now);
            for (int r = 0; r < runs; ++r) {
                const float rf = part_f[r * channels + ch], rb = part_b[r * channels + ch];
                part_f[r * channels + ch] = state;
                state = m.enter[r] ? rb : fmaf(rf, state, rb);
            }
        }
        __syncthreads();
        if (on && p_run < a.n) {
            float h[N];
#pragma unroll
            for (int e = 0; e < N; ++e) h[e] = part_f[run * channels + l * N + e];
#pragma unroll
            for (int j = 0; j < kRun; ++j) {
                const int t = token_of(j);
                const bool enters = enter >> j & 1;
                if (!kBack) {
#pragma unroll
                    for (int e = 0; e < N; ++e) h[e] = enters ? b[j][e] : fmaf(f[j][e], h[e], b[j][e]);
                    if (a.y && t >= lowest && t < highest) store<T, N>(static_cast<T*>(a.y) + (int64_t)t * width + c, h, own);
                } else {
                    float d[N], dg[N], dx[N], was[N];
#pragma unroll
                    for (int e = 0; e < N; ++e) was[e] = (float)before[j].v[e];
                    if (leave >> j & 1) {
                        const int64_t at = (int64_t)leaving[q + j] * width + c;
#pragma unroll
                        for (int e = 0; e < N; ++e) was[e] = in.h0 ? in.h0[at + e] : 0.0f;
                    }
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        d[e] = enters ? b[j][e] : b[j][e] + h[e];
                        dx[e] = d[e] * i_of[j][e];
                        dg[e] = dx[e] * f[j][e] * (was[e] - (float)xs[j].v[e]);
                        h[e] = d[e] * f[j][e];
                    }
                    if (t >= lowest && t < highest) {
                        store<T, N>(static_cast<T*>(a.dx) + t * in.dx_stride + c, dx, own);
                        store<T, N>(static_cast<T*>(a.dgate) + t * in.dgate_stride + c, dg, own);
                    }
                }
                if (a.last && leave >> j & 1) store<float, N>(a.last + (int64_t)leaving[q + j] * width + c, h, own);
            }
        }
    }
    // after the last number that there is all words are cleared, and 0 is no call's number
    if (now != ~0u) return;
    __syncthreads();
    if (tid == 0) last_drawn = draw(a.control + kDone) == (uint64_t)a.tiles * a.blocks - 1;
    __syncthreads();
    if (!last_drawn) return;
    for (size_t i = tid; i < a.n_words; i += kTileBlock) a.sums[i] = 0;
    ready(a, 1);
}

// ---- a token of every sequence ------------------------------------------------------------------

// Pieces of N channels of a row; a last one that is not whole goes by single channels, as states may be in place.
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
                const Gate k = gate_of<T>((float)g.v[e]);
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
                const Gate k = gate_of<T>((float)g.v[e]);
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
    a.n = (int)in.n; a.n_seq = (int)in.n_seq;
    const int per = in.width >= kScanChannels ? kScanChannels : 1, pieces = (in.width + per - 1) / per;
    const int most = 1 << kScanLanesLog;
    a.blocks = (pieces + most - 1) / most;
    a.lanes = (pieces + a.blocks - 1) / a.blocks;
    a.lg = kLeastLanesLog;
    while ((1 << a.lg) < a.lanes) ++a.lg;
    a.rows = (kTileBlock >> a.lg) * kScanRun;
    a.tiles = (int)((in.n + a.rows - 1) / a.rows);
    a.control = h->control;
    a.sums = h->words;
    a.n_words = h->n_words;
    a.counters = h->counters;
    a.states = a.sums + (int64_t)a.tiles * 2 * a.blocks * a.lanes * per;
    const int64_t total = (int64_t)a.tiles * a.blocks + (last ? (in.n_seq + 63) / 64 : 0);
    if (total > kMostBlocks / 2) return GR_ERR_TOO_LARGE;
    if (total == 0) return GR_OK;
    return by_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        if (per == 1) k_scan_tiles<T, 1, kScanRun, kBack><<<(unsigned)total, kTileBlock, 0, s>>>(a);
        else k_scan_tiles<T, kScanChannels, kScanRun, kBack><<<(unsigned)total, kTileBlock, 0, s>>>(a);
        return launched();
    });
}

}  // namespace

int scan_counters(int width) { return (width / kScanChannels >> kScanLanesLog) + 1; }

size_t scan_words(int64_t n, int width)
{
    // a word for F and one for B of every channel of every tile, and one of every group's state: of the least tiles and the most channels in use
    const int64_t rows = (int64_t)(kTileBlock >> kScanLanesLog) * kScanRun, tiles = (n + rows - 1) / rows;
    // (lanes are as many in every block of channels: less than a piece a block more in all, and two pieces)
    return (size_t)(tiles * 2 + tiles / kGroup + 1) * (width + (scan_counters(width) + 2) * kScanChannels);
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
