// recurrence.cu -- the gated linear recurrence of relaylayers.h, forward and
// backward, on GB300 (sm_103a):
//
//   h_t = f_t h_{t-1} + (1 - f_t) v_t,  f = sigma(gate)
//
// Every channel runs on its own, so a stretch of tokens is a pair (A, B) for the state
// behind it, h -> A h + B, and stretches join in any grouping.  A warp takes 64 channels,
// two a lane, and a run of tokens: from zero to get its (A, B), then, once the stretches
// before it are joined, again from the state that reaches it.  What both sweeps need stays
// in registers, so that the rows cross the chip once.
//
// A token that begins a sequence takes nothing from the state, not even 0 times it (it may
// hold an infinity or NaN): its factor is -0, which no sigmoid is, and a stretch that holds
// one has A = -0.
#include <type_traits>

#include "layers.cuh"

namespace {

constexpr int kWide = 64;  // channels of a warp

// ------------------------------------------------------------- a lane's channels

// kVector: channels 2 l and 2 l + 1 as one access (rows on boundaries of two elements, d
// even); kDirect: channels l and 32 + l.
template <Way kWay>
__device__ __forceinline__ int channel(int lane, int k) { return kWay == kVector ? 2 * lane + k : 32 * k + lane; }

template <typename T>
struct alignas(2 * sizeof(T)) Two {
    T e[2];
    __device__ __forceinline__ float get(int k) const { return widen(e[k]); }
};

template <Way kWay, typename T>
__device__ __forceinline__ Two<T> load_two(const T* p, int lane, int left, bool on) {
    Two<T> v;
    v.e[0] = v.e[1] = T(0.0f);
    if constexpr (kWay == kVector) {
        if (on && 2 * lane < left) v = *reinterpret_cast<const Two<T>*>(p + 2 * lane);
    } else {
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (on && 32 * k + lane < left) v.e[k] = p[32 * k + lane];
    }
    return v;
}

template <Way kWay, typename T>
__device__ __forceinline__ void store_two(T* p, int lane, int left, const float (&v)[2]) {
    if constexpr (kWay == kVector) {
        Two<T> w;
        w.e[0] = narrow<T>(v[0]), w.e[1] = narrow<T>(v[1]);
        if (2 * lane < left) *reinterpret_cast<Two<T>*>(p + 2 * lane) = w;
    } else {
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (32 * k + lane < left) p[32 * k + lane] = narrow<T>(v[k]);
    }
}

// fp32 values of the lane's channels; 0 where there are none.
template <Way kWay>
__device__ __forceinline__ void load_state(const float* p, int lane, int left, float (&v)[2]) {
#pragma unroll
    for (int k = 0; k < 2; ++k) v[k] = p != nullptr && channel<kWay>(lane, k) < left ? p[channel<kWay>(lane, k)] : 0.0f;
}

template <Way kWay>
__device__ __forceinline__ void store_state(float* p, int lane, int left, const float (&v)[2]) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (channel<kWay>(lane, k) < left) p[channel<kWay>(lane, k)] = v[k];
}

// ------------------------------------------------------------------ the arithmetic

__device__ __forceinline__ bool starts(float a) { return __float_as_uint(a) == 0x80000000u; }

// The state behind a token or a stretch (a, b).
__device__ __forceinline__ float carry(float h, float a, float b) { return starts(a) ? b : fmaf(a, h, b); }

// The stretch (a, b) with the one after it.
__device__ __forceinline__ void join(float& a, float& b, float a2, float b2) {
    b = carry(b, a2, b2);
    a = starts(a2) ? a2 : a * a2;
}

// ------------------------------------------------------------------- the kernels

template <typename T>
struct RecurrenceArgs {
    View<const T> gate, value, out_in, dout;  // out_in, dout: of the backward pass
    View<T> out, dgate, dvalue;
    const float* initial;  // the state before the first token, or NULL
    float* last;           // the state behind the last one (backward: its gradient's, of the first state), or NULL
    const float* dlast;
    int64_t initial_stride, last_stride, dlast_stride;
    const uint8_t* begins;
    const int32_t* lengths;
    float *a, *b;  // [n][segments][d], with several segments: A, then the state that reaches the segment; B
    int32_t n, tokens, d, strips, segments, segment;  // segment: tokens
};

// What a warp works on.
template <typename T>
struct Place {
    int strip, segment, worker, length, first;
    int64_t at;  // of its channels in a and b
    bool on;
    __device__ __forceinline__ Place(const RecurrenceArgs<T>& a, int64_t unit) {
        on = unit < static_cast<int64_t>(a.n) * a.segments * a.strips;
        if (!on) unit = 0;
        const int64_t row = unit / a.strips;
        strip = static_cast<int>(unit - row * a.strips) * kWide;
        worker = static_cast<int>(row / a.segments);
        segment = static_cast<int>(row - static_cast<int64_t>(worker) * a.segments);
        length = !on ? 0 : a.lengths == nullptr ? a.tokens : min(max(a.lengths[worker], 0), a.tokens);
        first = segment * a.segment;
        at = row * a.d + strip;
    }
};

// Tokens of a warp's run.
template <typename T>
constexpr int kRun = sizeof(T) == 2 ? 8 : 4;

// A run's rows as they lie in memory, so that the next ones can be on their way.
template <typename T, Way kWay>
struct Run {
    Two<T> gate[kRun<T>], value[kRun<T>];
    uint32_t begin;  // lane r: of token r
    // tokens from `to` on are not asked for
    __device__ __forceinline__ void ask(const RecurrenceArgs<T>& a, const Place<T>& p, int token, int to, int lane) {
        const int left = a.d - p.strip;
#pragma unroll
        for (int r = 0; r < kRun<T>; ++r) {
            const bool on = token + r < to;
            gate[r] = load_two<kWay>(a.gate.row(p.worker, token + r) + p.strip, lane, left, on);
            value[r] = load_two<kWay>(a.value.row(p.worker, token + r) + p.strip, lane, left, on);
        }
        begin = 0;
        if (a.begins != nullptr && lane < kRun<T> && token + lane < to)
            begin = a.begins[static_cast<int64_t>(p.worker) * a.tokens + token + lane];
    }
};

// Factor and addend of the run's tokens, and the run as one stretch; tokens from `to` on
// change nothing.
template <typename T, Way kWay>
__device__ __forceinline__ void stretch(const Run<T, kWay>& run, int token, int to, float (&f)[kRun<T>][2],
                                        float (&b)[kRun<T>][2], float (&ends)[4]) {
    const uint32_t begins = __ballot_sync(0xffffffffu, run.begin != 0);
    ends[0] = ends[1] = 1.0f;
    ends[2] = ends[3] = 0.0f;
#pragma unroll
    for (int r = 0; r < kRun<T>; ++r)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const Gate<T> g(run.gate[r].get(k));
            const bool on = token + r < to;
            f[r][k] = !on ? 1.0f : begins >> r & 1 ? -0.0f : g.at;
            b[r][k] = on ? g.rest * run.value[r].get(k) : 0.0f;
            join(ends[k], ends[2 + k], f[r][k], b[r][k]);
        }
}

// The stretches of the kTime warps that share a tile, in their order: `h` goes from the
// state before the tile to the one behind it, `mine` gets the one before warp `part`.
template <int kTime>
__device__ __forceinline__ void through(const float4 (*shared)[32], int part, int lane, float (&h)[2], float (&mine)[2]) {
#pragma unroll
    for (int j = 0; j < kTime; ++j) {
        if (j == part) mine[0] = h[0], mine[1] = h[1];
        const float4 e = shared[j][lane];
        h[0] = carry(h[0], e.x, e.z);
        h[1] = carry(h[1], e.y, e.w);
    }
}

constexpr int kWarps = 16, kBackWarps = 8;

// A segment's tokens tile by tile: kTime warps take a run each, the CTA's other warps
// other strips.
template <typename T, Way kWay, int kTime>
__global__ void __launch_bounds__(32 * kWarps, 2) relay_recurrence_kernel(RecurrenceArgs<T> a) {
    constexpr int kSide = kWarps / kTime, kTile = kTime * kRun<T>;
    __shared__ float4 shared[2][kSide][kTime][32];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, slot = warp / kTime, part = warp % kTime;
    const Place<T> p(a, static_cast<int64_t>(blockIdx.x) * kSide + slot);
    const int left = p.on ? a.d - p.strip : 0, tiles = (min(a.segment, a.tokens) + kTile - 1) / kTile;
    const int end = min(p.first + a.segment, a.tokens), to = min(end, p.length);
    float h[2];
    if (a.segments == 1)
        load_state<kWay>(a.initial == nullptr ? nullptr : a.initial + p.worker * a.initial_stride + p.strip, lane, left, h);
    else
        load_state<kWay>(a.a + p.at, lane, left, h);
    Run<T, kWay> run;
    run.ask(a, p, p.first + part * kRun<T>, to, lane);
    for (int i = 0; i < tiles; ++i) {
        const int token = p.first + i * kTile + part * kRun<T>;
        float f[kRun<T>][2], b[kRun<T>][2], ends[4], x[2];
        stretch(run, token, to, f, b, ends);
        if (i + 1 < tiles) run.ask(a, p, token + kTile, to, lane);
        if constexpr (kTime > 1) {
            shared[i & 1][slot][part][lane] = make_float4(ends[0], ends[1], ends[2], ends[3]);
            __syncthreads();
            through<kTime>(shared[i & 1][slot], part, lane, h, x);
        } else {
            x[0] = h[0], x[1] = h[1];
        }
#pragma unroll
        for (int r = 0; r < kRun<T>; ++r) {
            float y[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                x[k] = carry(x[k], f[r][k], b[r][k]);
                y[k] = token + r < p.length ? x[k] : 0.0f;
            }
            if (token + r < end) store_two<kWay>(a.out.row(p.worker, token + r) + p.strip, lane, left, y);
        }
        if constexpr (kTime == 1) h[0] = x[0], h[1] = x[1];
    }
    if (a.segments == 1 && a.last != nullptr && part == 0)
        store_state<kWay>(a.last + p.worker * a.last_stride + p.strip, lane, left, h);
}

// A segment as one stretch: each of the CTA's warps takes a part of its tokens.
template <typename T, Way kWay>
__global__ void __launch_bounds__(32 * kWarps, 2) relay_recurrence_ends_kernel(RecurrenceArgs<T> a) {
    __shared__ float4 shared[kWarps][32];
    const int lane = threadIdx.x % 32, part = threadIdx.x / 32;
    const Place<T> p(a, blockIdx.x);
    const int left = a.d - p.strip, each = (a.segment + kWarps - 1) / kWarps;
    const int first = p.first + part * each, to = min(min(first + each, p.first + a.segment), p.length);
    float whole[4] = {1.0f, 1.0f, 0.0f, 0.0f};
    Run<T, kWay> run;
    run.ask(a, p, first, to, lane);
    for (int token = first; token < to; token += kRun<T>) {
        float f[kRun<T>][2], b[kRun<T>][2], ends[4];
        stretch(run, token, to, f, b, ends);
        run.ask(a, p, token + kRun<T>, to, lane);
#pragma unroll
        for (int k = 0; k < 2; ++k) join(whole[k], whole[2 + k], ends[k], ends[2 + k]);
    }
    shared[part][lane] = make_float4(whole[0], whole[1], whole[2], whole[3]);
    __syncthreads();
    if (part > 0) return;
    for (int j = 1; j < kWarps; ++j) {
        const float4 e = shared[j][lane];
        join(whole[0], whole[2], e.x, e.z);
        join(whole[1], whole[3], e.y, e.w);
    }
    const float one[2] = {whole[0], whole[1]}, two[2] = {whole[2], whole[3]};
    store_state<kWay>(a.a + p.at, lane, left, one);
    store_state<kWay>(a.b + p.at, lane, left, two);
}

// Through a channel's segments (from the last to the first: kBack): a gets the state that
// reaches each of them, `last` what leaves the last of them.
template <bool kBack>
__global__ void __launch_bounds__(64)
relay_recurrence_carry_kernel(float* a, const float* b, int segments, int d, const float* initial, int64_t initial_stride,
                              float* last, int64_t last_stride) {
    const int c = blockIdx.x * 64 + threadIdx.x, worker = blockIdx.y;
    if (c >= d) return;
    constexpr int kAtOnce = 8;
    const int64_t base = static_cast<int64_t>(worker) * segments * d + c;
    float h = initial == nullptr ? 0.0f : initial[worker * initial_stride + c];
    for (int s0 = 0; s0 < segments; s0 += kAtOnce) {
        float fa[kAtOnce], fb[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int s = kBack ? segments - 1 - s0 - j : s0 + j;
            fa[j] = 0.0f, fb[j] = 0.0f;
            if (s0 + j < segments) fa[j] = a[base + int64_t(s) * d], fb[j] = b[base + int64_t(s) * d];
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int s = kBack ? segments - 1 - s0 - j : s0 + j;
            if (s0 + j < segments) {
                a[base + int64_t(s) * d] = h;
                h = carry(h, fa[j], fb[j]);
            }
        }
    }
    if (last != nullptr) last[worker * last_stride + c] = h;
}

// ------------------------------------------------------------------ the backward pass
//
// With l_t the gradient that reaches h_t and m_t = f_t l_t what goes on to h_{t-1},
//   l_t = dout_t + m_{t+1},  dv_t = l_t (1 - f_t),  dgate_t = l_t (h_{t-1} - v_t) f_t (1 - f_t):
// from the last token to the first m is the same kind of recurrence, m -> f_t m + f_t dout_t.

template <typename T, Way kWay>
struct BackRun {
    Two<T> gate[kRun<T>], dout[kRun<T>];
    uint32_t begin;
    __device__ __forceinline__ void ask(const RecurrenceArgs<T>& a, const Place<T>& p, int token, int to, int lane) {
        const int left = a.d - p.strip;
#pragma unroll
        for (int r = 0; r < kRun<T>; ++r) {
            const bool on = token + r < to && token + r >= 0;
            gate[r] = load_two<kWay>(a.gate.row(p.worker, token + r) + p.strip, lane, left, on);
            dout[r] = load_two<kWay>(a.dout.row(p.worker, token + r) + p.strip, lane, left, on);
        }
        begin = 0;
        if (a.begins != nullptr && lane < kRun<T> && token + lane < to && token + lane >= 0)
            begin = a.begins[static_cast<int64_t>(p.worker) * a.tokens + token + lane];
    }
    // The run as one stretch, from its last token to its first.
    __device__ __forceinline__ void stretch(int token, int to, uint32_t begins, float (&ends)[4]) const {
        ends[0] = ends[1] = 1.0f;
        ends[2] = ends[3] = 0.0f;
#pragma unroll
        for (int r = kRun<T> - 1; r >= 0; --r)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const Gate<T> g(gate[r].get(k));
                const bool on = token + r < to;
                const float f = !on ? 1.0f : begins >> r & 1 ? -0.0f : g.at;
                join(ends[k], ends[2 + k], f, on && !starts(f) ? f * dout[r].get(k) : 0.0f);
            }
    }
};

// The forward kernel's tiles, from the segment's end to its start.  What the second sweep
// needs of the gate is made again from the row.
template <typename T, Way kWay, int kTime>
__global__ void __launch_bounds__(32 * kBackWarps, 2) relay_recurrence_backward_kernel(RecurrenceArgs<T> a) {
    constexpr int kSide = kBackWarps / kTime, kTile = kTime * kRun<T>;
    __shared__ float4 shared[2][kSide][kTime][32];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, slot = warp / kTime, part = warp % kTime;
    const Place<T> p(a, static_cast<int64_t>(blockIdx.x) * kSide + slot);
    const int left = p.on ? a.d - p.strip : 0, tiles = (min(a.segment, a.tokens) + kTile - 1) / kTile;
    const int end = min(p.first + a.segment, a.tokens), to = min(end, p.length);
    float m[2], first[2];
    if (a.segments == 1)
        load_state<kWay>(a.dlast == nullptr ? nullptr : a.dlast + p.worker * a.dlast_stride + p.strip, lane, left, m);
    else
        load_state<kWay>(a.a + p.at, lane, left, m);
    load_state<kWay>(a.initial == nullptr ? nullptr : a.initial + p.worker * a.initial_stride + p.strip, lane, left, first);
    BackRun<T, kWay> run;
    Two<T> value[kRun<T>], before[kRun<T>];
    const auto ask = [&](int token) {
        run.ask(a, p, token, to, lane);
#pragma unroll
        for (int r = 0; r < kRun<T>; ++r) {
            const int t = token + r;
            value[r] = load_two<kWay>(a.value.row(p.worker, t) + p.strip, lane, left, t < to && t >= 0);
            before[r] = load_two<kWay>(a.out_in.row(p.worker, t - 1) + p.strip, lane, left, t < to && t > 0);
        }
    };
    // warp 0 of a tile takes its last tokens
    const auto token_of = [&](int i) { return p.first + (tiles - 1 - i) * kTile + (kTime - 1 - part) * kRun<T>; };
    ask(token_of(0));
    for (int i = 0; i < tiles; ++i) {
        const int token = token_of(i);
        const BackRun<T, kWay> now = run;
        Two<T> v[kRun<T>], h[kRun<T>];
#pragma unroll
        for (int r = 0; r < kRun<T>; ++r) v[r] = value[r], h[r] = before[r];
        if (i + 1 < tiles) ask(token_of(i + 1));
        const uint32_t begins = __ballot_sync(0xffffffffu, now.begin != 0);
        float ends[4], x[2];
        if constexpr (kTime > 1) {
            now.stretch(token, to, begins, ends);
            shared[i & 1][slot][part][lane] = make_float4(ends[0], ends[1], ends[2], ends[3]);
            __syncthreads();
            through<kTime>(shared[i & 1][slot], part, lane, m, x);
        } else {
            x[0] = m[0], x[1] = m[1];
        }
#pragma unroll
        for (int r = kRun<T> - 1; r >= 0; --r) {
            const bool on = token + r < to, begin = begins >> r & 1;
            float dg[2] = {0.0f, 0.0f}, dv[2] = {0.0f, 0.0f};
            if (on) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const Gate<T> g(now.gate[r].get(k));
                    const float l = now.dout[r].get(k) + x[k];
                    const float h0 = begin ? 0.0f : token + r == 0 ? first[k] : h[r].get(k);
                    dv[k] = l * g.rest;
                    dg[k] = dv[k] * g.at * (h0 - v[r].get(k));
                    x[k] = begin ? 0.0f : g.at * l;
                }
            }
            if (token + r < end && token + r >= p.first) {
                store_two<kWay>(a.dgate.row(p.worker, token + r) + p.strip, lane, left, dg);
                store_two<kWay>(a.dvalue.row(p.worker, token + r) + p.strip, lane, left, dv);
            }
        }
        if constexpr (kTime == 1) m[0] = x[0], m[1] = x[1];
    }
    if (a.segments == 1 && a.last != nullptr && part == 0)
        store_state<kWay>(a.last + p.worker * a.last_stride + p.strip, lane, left, m);
}

template <typename T, Way kWay>
__global__ void __launch_bounds__(32 * kWarps, 2) relay_recurrence_backward_ends_kernel(RecurrenceArgs<T> a) {
    __shared__ float4 shared[kWarps][32];
    const int lane = threadIdx.x % 32, part = threadIdx.x / 32;
    const Place<T> p(a, blockIdx.x);
    const int left = a.d - p.strip, each = (a.segment + kWarps - 1) / kWarps;
    const int first = p.first + part * each, to = min(min(first + each, p.first + a.segment), p.length);
    float whole[4] = {1.0f, 1.0f, 0.0f, 0.0f};
    const int runs = to > first ? (to - first + kRun<T> - 1) / kRun<T> : 0;
    BackRun<T, kWay> run;
    if (runs > 0) run.ask(a, p, first + (runs - 1) * kRun<T>, to, lane);
    for (int i = runs - 1; i >= 0; --i) {
        const BackRun<T, kWay> now = run;
        if (i > 0) run.ask(a, p, first + (i - 1) * kRun<T>, to, lane);
        float ends[4];
        now.stretch(first + i * kRun<T>, to, __ballot_sync(0xffffffffu, now.begin != 0), ends);
#pragma unroll
        for (int k = 0; k < 2; ++k) join(whole[k], whole[2 + k], ends[k], ends[2 + k]);
    }
    shared[part][lane] = make_float4(whole[0], whole[1], whole[2], whole[3]);
    __syncthreads();
    if (part > 0) return;
    const float4 e0 = shared[kWarps - 1][lane];  // the last tokens come first
    whole[0] = e0.x, whole[1] = e0.y, whole[2] = e0.z, whole[3] = e0.w;
    for (int j = kWarps - 2; j >= 0; --j) {
        const float4 e = shared[j][lane];
        join(whole[0], whole[2], e.x, e.z);
        join(whole[1], whole[3], e.y, e.w);
    }
    const float one[2] = {whole[0], whole[1]}, two[2] = {whole[2], whole[3]};
    store_state<kWay>(a.a + p.at, lane, left, one);
    store_state<kWay>(a.b + p.at, lane, left, two);
}

// ---------------------------------------------------------------- launching

// How a call is cut.
struct Cut {
    int strips, segments, segment;
};

// Segments only where the strips alone leave most SMs idle and the tokens are many: they
// cost a second reading of two rows in three (four in six).
Cut recurrence_cut(int64_t n, int64_t tokens, int64_t d) {
    const int64_t strips = (d + kWide - 1) / kWide, units = n * strips;
    int64_t segments = 1;
    if (units < 152 && tokens >= 1024) {
        segments = 608 / units;
        if (segments > tokens / 256) segments = tokens / 256;
        if (segments > 128) segments = 128;
    }
    int64_t segment = (tokens + segments - 1) / segments;
    segment = (segment + 127) / 128 * 128;
    if (segments > 1) segments = (tokens + segment - 1) / segment;
    if (segments <= 1) return Cut{static_cast<int>(strips), 1, static_cast<int>(tokens)};
    return Cut{static_cast<int>(strips), static_cast<int>(segments), static_cast<int>(segment)};
}

int check_recurrence(int32_t type, int32_t n, int64_t tokens, int64_t d) {
    if (type < RELAY_BF16 || type > RELAY_FP32 || n < 1 || tokens < 0 || d < 1) return RELAY_EINVAL;
    if (n > RELAY_RECURRENCE_MAX_N || tokens >= kMaxRows || tokens * n >= kMaxRows || d > kMaxD) return RELAY_EUNSUPPORTED;
    if (n * ((d + kWide - 1) / kWide) > (int64_t(1) << 30)) return RELAY_EUNSUPPORTED;
    return RELAY_OK;
}

// Whether [n][d] fp32 values may be used (NULL: there are none).
bool state_fits(const float* p, int64_t stride, int32_t n, int64_t d, bool output) {
    if (p == nullptr) return true;
    return aligned(p, 4) && stride >= 0 && (!output || n == 1 || stride >= d);
}

// Whether an output state may lie where an input one does: nowhere, or on its very rows.
bool apart(const float* out, int64_t out_stride, const float* in, int64_t in_stride, int32_t n) {
    return out == nullptr || out != in || n == 1 || out_stride == in_stride;
}

// Rows whose channels go two at a time.
bool pairs(const relay_rows* r, int32_t type, int32_t n, int64_t tokens) {
    return aligned(r->data, 2 * element_size(type)) && (n == 1 || r->worker_stride % 2 == 0) &&
           (tokens <= 1 || r->token_stride % 2 == 0);
}

// f(warps that share a strip's tile) as a constant.
template <int kMost, typename F>
int by_time(int64_t tokens, int run, F f) {
    if (tokens <= run) return f(std::integral_constant<int, 1>());
    if (tokens <= 4 * run) return f(std::integral_constant<int, 4>());
    return f(std::integral_constant<int, kMost>());
}

}  // namespace

extern "C" {

int64_t relay_recurrence_workspace(int32_t n, int64_t tokens, int64_t d) {
    if (const int rc = check_recurrence(RELAY_FP32, n, tokens, d)) return rc;
    const Cut cut = recurrence_cut(n, tokens, d);
    return cut.segments > 1 ? 8 * static_cast<int64_t>(n) * cut.segments * d : 0;
}

int relay_recurrence(int32_t type, int32_t n, int64_t tokens, int64_t d, const relay_rows* gate, const relay_rows* value,
                     const float* initial, int64_t initial_stride, const uint8_t* begins, const int32_t* lengths,
                     const relay_rows* out, float* last, int64_t last_stride, void* workspace, int64_t workspace_bytes,
                     relay_stream_t stream) {
    if (const int rc = check_recurrence(type, n, tokens, d)) return rc;
    if (!rows_fit(gate, type, n, tokens, d, false) || !rows_fit(value, type, n, tokens, d, false) ||
        !rows_fit(out, type, n, tokens, d, true))
        return RELAY_EINVAL;
    if (!state_fits(initial, initial_stride, n, d, false) || !state_fits(last, last_stride, n, d, true) ||
        !apart(last, last_stride, initial, initial_stride, n) || !aligned(lengths, 4))
        return RELAY_EINVAL;
    const int64_t need = relay_recurrence_workspace(n, tokens, d);
    if (workspace_bytes < need || (need > 0 && (workspace == nullptr || !aligned(workspace, 16)))) return RELAY_EINVAL;
    if (tokens > 0 && (out->data == gate->data || out->data == value->data)) return RELAY_EINVAL;
    if (tokens == 0 && last == nullptr) return RELAY_OK;
    const Cut cut = recurrence_cut(n, tokens, d);
    const bool vec = tokens == 0 || (d % 2 == 0 && pairs(gate, type, n, tokens) && pairs(value, type, n, tokens) &&
                                     pairs(out, type, n, tokens));
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        RecurrenceArgs<T> a{};
        a.gate = view<const T>(gate, n, tokens), a.value = view<const T>(value, n, tokens), a.out = view<T>(out, n, tokens);
        a.initial = initial, a.initial_stride = n > 1 ? initial_stride : 0;
        a.last = last, a.last_stride = n > 1 ? last_stride : 0;
        a.begins = begins, a.lengths = lengths;
        a.a = static_cast<float*>(workspace), a.b = a.a + static_cast<int64_t>(n) * cut.segments * d;
        a.n = n, a.tokens = static_cast<int32_t>(tokens), a.d = static_cast<int32_t>(d);
        a.strips = cut.strips, a.segments = cut.segments, a.segment = cut.segment;
        const int64_t units = static_cast<int64_t>(n) * cut.segments * cut.strips;
        if (cut.segments > 1) {
            (vec ? relay_recurrence_ends_kernel<T, kVector> : relay_recurrence_ends_kernel<T, kDirect>)
                <<<static_cast<unsigned>(units), 32 * kWarps, 0, stream>>>(a);
            relay_recurrence_carry_kernel<false><<<dim3(static_cast<unsigned>((d + 63) / 64), n), 64, 0, stream>>>(
                a.a, a.b, cut.segments, a.d, initial, a.initial_stride, last, a.last_stride);
        }
        return by_time<kWarps>(cut.segment, kRun<T>, [&](auto time) {
            constexpr int kTime = decltype(time)::value, kSide = kWarps / kTime;
            (vec ? relay_recurrence_kernel<T, kVector, kTime> : relay_recurrence_kernel<T, kDirect, kTime>)
                <<<static_cast<unsigned>((units + kSide - 1) / kSide), 32 * kWarps, 0, stream>>>(a);
            return status_of_launch();
        });
    });
}

int relay_recurrence_backward(int32_t type, int32_t n, int64_t tokens, int64_t d, const relay_rows* dout,
                              const relay_rows* gate, const relay_rows* value, const relay_rows* out, const float* initial,
                              int64_t initial_stride, const float* dlast, int64_t dlast_stride, const uint8_t* begins,
                              const int32_t* lengths, const relay_rows* dgate, const relay_rows* dvalue, float* dinitial,
                              int64_t dinitial_stride, void* workspace, int64_t workspace_bytes, relay_stream_t stream) {
    if (const int rc = check_recurrence(type, n, tokens, d)) return rc;
    for (const relay_rows* r : {dout, gate, value, out})
        if (!rows_fit(r, type, n, tokens, d, false)) return RELAY_EINVAL;
    for (const relay_rows* r : {dgate, dvalue})
        if (!rows_fit(r, type, n, tokens, d, true)) return RELAY_EINVAL;
    if (!state_fits(initial, initial_stride, n, d, false) || !state_fits(dlast, dlast_stride, n, d, false) ||
        !state_fits(dinitial, dinitial_stride, n, d, true) || (dinitial != nullptr && dinitial == initial) ||
        !apart(dinitial, dinitial_stride, dlast, dlast_stride, n) || !aligned(lengths, 4))
        return RELAY_EINVAL;
    const int64_t need = relay_recurrence_workspace(n, tokens, d);
    if (workspace_bytes < need || (need > 0 && (workspace == nullptr || !aligned(workspace, 16)))) return RELAY_EINVAL;
    if (tokens > 0) {
        for (const relay_rows* o : {dgate, dvalue})
            for (const relay_rows* r : {dout, gate, value, out})
                if (o->data == r->data) return RELAY_EINVAL;
        if (dgate->data == dvalue->data) return RELAY_EINVAL;
    }
    if (tokens == 0 && dinitial == nullptr) return RELAY_OK;
    const Cut cut = recurrence_cut(n, tokens, d);
    bool vec = d % 2 == 0 || tokens == 0;
    if (tokens > 0)
        for (const relay_rows* r : {dout, gate, value, out, dgate, dvalue}) vec = vec && pairs(r, type, n, tokens);
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        RecurrenceArgs<T> a{};
        a.gate = view<const T>(gate, n, tokens), a.value = view<const T>(value, n, tokens);
        a.out_in = view<const T>(out, n, tokens), a.dout = view<const T>(dout, n, tokens);
        a.dgate = view<T>(dgate, n, tokens), a.dvalue = view<T>(dvalue, n, tokens);
        a.initial = initial, a.initial_stride = n > 1 ? initial_stride : 0;
        a.dlast = dlast, a.dlast_stride = n > 1 ? dlast_stride : 0;
        a.last = dinitial, a.last_stride = n > 1 ? dinitial_stride : 0;
        a.begins = begins, a.lengths = lengths;
        a.a = static_cast<float*>(workspace), a.b = a.a + static_cast<int64_t>(n) * cut.segments * d;
        a.n = n, a.tokens = static_cast<int32_t>(tokens), a.d = static_cast<int32_t>(d);
        a.strips = cut.strips, a.segments = cut.segments, a.segment = cut.segment;
        const int64_t units = static_cast<int64_t>(n) * cut.segments * cut.strips;
        if (cut.segments > 1) {
            (vec ? relay_recurrence_backward_ends_kernel<T, kVector> : relay_recurrence_backward_ends_kernel<T, kDirect>)
                <<<static_cast<unsigned>(units), 32 * kWarps, 0, stream>>>(a);
            relay_recurrence_carry_kernel<true><<<dim3(static_cast<unsigned>((d + 63) / 64), n), 64, 0, stream>>>(
                a.a, a.b, cut.segments, a.d, dlast, a.dlast_stride, dinitial, a.last_stride);
        }
        return by_time<kBackWarps>(cut.segment, kRun<T>, [&](auto time) {
            constexpr int kTime = decltype(time)::value, kSide = kBackWarps / kTime;
            (vec ? relay_recurrence_backward_kernel<T, kVector, kTime> : relay_recurrence_backward_kernel<T, kDirect, kTime>)
                <<<static_cast<unsigned>((units + kSide - 1) / kSide), 32 * kBackWarps, 0, stream>>>(a);
            return status_of_launch();
        });
    });
}

}  // extern "C"
