// recurrence.cu -- the gated linear recurrence of relaylayers.h, forward and
// backward, on GB300 (sm_103a):
//
//   h_t = f_t h_{t-1} + (1 - f_t) v_t,  f = sigma(gate)
//
// Every channel runs on its own, so a stretch of tokens is a pair (A, B) for the state
// behind it, h -> A h + B, and stretches join in any grouping.  A warp takes 64 channels,
// two a lane, and a run of tokens: from zero to get its (A, B), then, once the stretches
// before it are joined, again from the state that reaches it.  What both sweeps need stays
// on the SM, so that the rows cross the chip once.  A CTA's 8 warps take runs one behind the
// other; where strips of 64 channels are few, clusters of CTAs do, or segments of the tokens
// go their own ways, their stretches first.  Every join is in a fixed order: the same bits
// every time.
//
// A token that begins a sequence takes nothing from the state, not even 0 times it (it may
// hold an infinity or NaN): its factor is -0, which no sigmoid is, and a stretch that holds
// one has A = -0.
//
// Memory bounds it where strips are many: [4][4096][4096] in bf16 takes 66 us forward (403 MB,
// 6.1 TB/s) and 127 to 138 us backward (805 MB, 5.9 to 6.3 TB/s); issue slots are 61 % taken.  With few strips the
// chain of joins bounds it: [1][4096][1024] 13 us; [1][50021][257] in fp32, whose rows TMA does
// not take and whose segments read two rows in three twice, 84 us (154 MB, 1.8 TB/s).
#include <type_traits>

#include "blackwell.cuh"
#include "layers.cuh"

namespace {

constexpr int kWide = 64;  // channels of a warp

// ------------------------------------------------------------- a lane's channels

// kVector: channels 2 l and 2 l + 1 as one access (rows on boundaries of two elements, d
// even); kDirect: channels l and 32 + l.
template <Way kWay>
__device__ __forceinline__ int channel(int lane, int k) { return kWay == kVector ? 2 * lane + k : 32 * k + lane; }

// Two channels as they lie in memory: 16-bit ones that come together share a register, and ones
// that come apart have one each, since putting them together would wait for them.
template <typename T, Way kWay = kVector>
struct Two {
    uint32_t w;
    __device__ __forceinline__ float get(int k) const {
        if constexpr (std::is_same_v<T, __nv_bfloat16>) return __uint_as_float(k == 0 ? w << 16 : w & 0xffff0000u);
        return widen(reinterpret_cast<const T*>(&w)[k]);
    }
    __device__ __forceinline__ void set(T a, T b) {
        reinterpret_cast<T*>(&w)[0] = a;
        reinterpret_cast<T*>(&w)[1] = b;
    }
};
template <typename T>
struct Two<T, kDirect> {
    uint32_t e[2];
    __device__ __forceinline__ float get(int k) const {
        if constexpr (std::is_same_v<T, __nv_bfloat16>) return __uint_as_float(e[k] << 16);
        return widen(*reinterpret_cast<const T*>(&e[k]));
    }
    __device__ __forceinline__ void set(T a, T b) {
        e[0] = *reinterpret_cast<const uint16_t*>(&a);
        e[1] = *reinterpret_cast<const uint16_t*>(&b);
    }
};
template <>
struct alignas(8) Two<float> {
    float v[2];
    __device__ __forceinline__ float get(int k) const { return v[k]; }
    __device__ __forceinline__ void set(float a, float b) { v[0] = a, v[1] = b; }
};
template <>
struct Two<float, kDirect> : Two<float> {};

template <Way kWay, typename T>
__device__ __forceinline__ void store_two(T* p, int lane, int left, const float (&v)[2]) {
    if constexpr (kWay == kVector) {
        Two<T> w;
        w.set(narrow<T>(v[0]), narrow<T>(v[1]));
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

// The state behind a token or a stretch (a, b).  kBegins: there may be beginnings.
template <bool kBegins>
__device__ __forceinline__ float carry(float h, float a, float b) { return kBegins && starts(a) ? b : fmaf(a, h, b); }

// The stretch (a, b) with the one after it.
template <bool kBegins>
__device__ __forceinline__ void join(float& a, float& b, float a2, float b2) {
    b = carry<kBegins>(b, a2, b2);
    a = kBegins && starts(a2) ? a2 : a * a2;
}

// A wait for rows that ran out: whatever reaches the run and whatever begins in it, its states and
// the stretch that it leaves are NaN, up to the next beginning in rows that did come.
template <int kRun>
__device__ __forceinline__ void lose(float (&b)[kRun][2]) {
#pragma unroll
    for (int r = 0; r < kRun; ++r) b[r][0] = b[r][1] = NAN;
}

// The same on the way back, where a run's gradients are made of f and 1 - f.
template <int kRun>
__device__ __forceinline__ void lose(float (&at)[kRun][2], float (&rest)[kRun][2], float (&ends)[4]) {
#pragma unroll
    for (int r = 0; r < kRun; ++r) at[r][0] = at[r][1] = rest[r][0] = rest[r][1] = NAN;
    ends[2] = ends[3] = NAN;
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
    float *a, *b, *first;  // with several segments: their A and B, [n][segments][d], and the state before them, [n][d]
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

// Row addresses: aligned rows have strides below 2^30 elements (pairs()), which leaves one
// instruction an address.
template <Way kWay, typename T>
__device__ __forceinline__ T* token_of(T* base, int64_t stride, int r) {
    if constexpr (kWay == kVector) return base + static_cast<int64_t>(r) * static_cast<int32_t>(stride);
    return base + r * stride;
}

// `bits` or, where `on`, what lies at p.  In one instruction stream whether on or not, so that
// no move waits for the load before its value is needed: with a branch around the loads of whole
// runs every run waited for the next one's (310 us for [4][4096][4096] in bf16).
__device__ __forceinline__ void load_if(uint32_t& v, const uint32_t* p, bool on) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %2, 0;\n@p ld.global.b32 %0, [%1];\n}" : "+r"(v) : "l"(p), "r"(uint32_t(on)));
}
__device__ __forceinline__ void load_if(float (&v)[2], const float* p, bool on) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %3, 0;\n@p ld.global.v2.f32 {%0, %1}, [%2];\n}"
                 : "+f"(v[0]), "+f"(v[1])
                 : "l"(p), "r"(uint32_t(on)));
}
__device__ __forceinline__ void load_if(float& v, const float* p, bool on) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %2, 0;\n@p ld.global.f32 %0, [%1];\n}" : "+f"(v) : "l"(p), "r"(uint32_t(on)));
}
__device__ __forceinline__ void load_if(uint32_t& v, const uint16_t* p, bool on) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %2, 0;\n@p ld.global.u16 %0, [%1];\n}" : "+r"(v) : "l"(p), "r"(uint32_t(on)));
}

// kRun tokens of one activation as they lie in memory; those that do not count (from number
// `counts` on, and the first one where `skip` says so, and channels from `left` on) are
// `rest`.
template <Way kWay, int kRun, typename T>
__device__ __forceinline__ void load_run(Two<T, kWay> (&to)[kRun], const View<const T>& v, int worker, int token, int column,
                                         int lane, int left, int counts, float rest = 0.0f, bool skip = false) {
    const T* from = v.row(worker, token) + column + (kWay == kVector ? 2 * lane : lane);
    if constexpr (kWay == kVector) {
        if (2 * lane >= left) counts = 0;
#pragma unroll
        for (int r = 0; r < kRun; ++r) {
            to[r].set(narrow<T>(rest), narrow<T>(rest));
            if constexpr (sizeof(T) == 2)
                load_if(to[r].w, reinterpret_cast<const uint32_t*>(token_of<kWay>(from, v.ts, r)),
                        r < counts && (r > 0 || !skip));
            else
                load_if(to[r].v, token_of<kWay>(from, v.ts, r), r < counts && (r > 0 || !skip));
        }
    } else {
        const int first = lane < left ? counts : 0, second = 32 + lane < left ? counts : 0;
#pragma unroll
        for (int r = 0; r < kRun; ++r) {
            const T* p = token_of<kWay>(from, v.ts, r);
            const bool on = r > 0 || !skip;
            to[r].set(narrow<T>(rest), narrow<T>(rest));
            if constexpr (sizeof(T) == 2) {
                load_if(to[r].e[0], reinterpret_cast<const uint16_t*>(p), on && r < first);
                load_if(to[r].e[1], reinterpret_cast<const uint16_t*>(p + 32), on && r < second);
            } else {
                load_if(to[r].v[0], p, on && r < first);
                load_if(to[r].v[1], p + 32, on && r < second);
            }
        }
    }
}

constexpr float kKeeps = INFINITY;  // a gate that leaves the state as it is

// Lane r: whether token r of the run begins a sequence; 0 where nothing says so.
template <int kRun, bool kBegins, typename T>
__device__ __forceinline__ uint32_t load_begins(const RecurrenceArgs<T>& a, int worker, int token, int lane, int counts) {
    if (kBegins && a.begins != nullptr && lane < kRun && lane < counts) return a.begins[static_cast<int64_t>(worker) * a.tokens + token + lane];
    return 0;
}

// Factor and addend of the run's tokens, and the run as one stretch.
template <bool kBegins, int kRun, typename T, Way kWay>
__device__ __forceinline__ void stretch(const Two<T, kWay> (&gate)[kRun], const Two<T, kWay> (&value)[kRun], uint32_t begin,
                                        float (&f)[kRun][2], float (&b)[kRun][2], float (&ends)[4]) {
    const uint32_t begins = kBegins ? __ballot_sync(0xffffffffu, begin != 0) : 0u;
#pragma unroll
    for (int r = 0; r < kRun; ++r)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const Gate<T> g(gate[r].get(k));
            f[r][k] = kBegins && (begins >> r & 1) ? -0.0f : g.at;
            b[r][k] = g.rest * value[r].get(k);
            if (r == 0)
                ends[k] = f[r][k], ends[2 + k] = b[r][k];
            else
                join<kBegins>(ends[k], ends[2 + k], f[r][k], b[r][k]);
        }
}

// The stretches of the kTime warps that share a tile, in their order: `h` goes from the
// state before the tile to the one behind it, `mine` gets the one before warp `part`.
template <int kTime, bool kBegins>
__device__ __forceinline__ void through(const float4 (*shared)[32], int part, int lane, float (&h)[2], float (&mine)[2]) {
#pragma unroll
    for (int j = 0; j < kTime; ++j) {
        if (j == part) mine[0] = h[0], mine[1] = h[1];
        const float4 e = shared[j][lane];
        h[0] = carry<kBegins>(h[0], e.x, e.z);
        h[1] = carry<kBegins>(h[1], e.y, e.w);
    }
}

constexpr int kWarps = 8;  // of a CTA, all of them a strip's, or kTime of them and the others other strips'

// Tokens of a warp's run: as many as leave the next ones on their way too.
template <typename T, Way kWay = kVector>
constexpr int kRunOf = sizeof(T) == 2 && kWay == kVector ? 16 : 8;
template <typename T, Way kWay = kVector>
constexpr int kBackRunOf = kRunOf<T, kWay> / 2;

// The state that reaches segment p.segment, from the stretches of those before it (behind it:
// kBack), which the CTA's warps join side by side.  The first one's holds the incoming state
// (keep_ends) and lets nothing through.
template <Way kWay, bool kBack, typename T>
__device__ __forceinline__ void reach(const RecurrenceArgs<T>& a, const Place<T>& p, int part, int lane, int left,
                                      float4 (&shared)[kWarps][32], float (&h)[2]) {
    const int before = kBack ? a.segments - 1 - p.segment : p.segment, each = (before + kWarps - 1) / kWarps;
    if (before == 0) {
        load_state<kWay>(a.first + static_cast<int64_t>(p.worker) * a.d + p.strip, lane, left, h);
        return;
    }
    float whole[4] = {1.0f, 1.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int j = part * each; j < min(part * each + each, before); ++j) {
        const int64_t at = p.at + static_cast<int64_t>(kBack ? a.segments - 1 - j - p.segment : j - p.segment) * a.d;
        float f[2], b[2];
        load_state<kWay>(a.a + at, lane, left, f);
        load_state<kWay>(a.b + at, lane, left, b);
#pragma unroll
        for (int k = 0; k < 2; ++k) join<true>(whole[k], whole[2 + k], f[k], b[k]);
    }
    shared[part][lane] = make_float4(whole[0], whole[1], whole[2], whole[3]);
    __syncthreads();
    h[0] = h[1] = 0.0f;
#pragma unroll
    for (int j = 0; j < kWarps; ++j) {
        const float4 e = shared[j][lane];
        h[0] = carry<true>(h[0], e.x, e.z);
        h[1] = carry<true>(h[1], e.y, e.w);
    }
}

// Puts a segment's stretch away, that of the first segment with the incoming state in it.
template <Way kWay, typename T>
__device__ __forceinline__ void keep_ends(const RecurrenceArgs<T>& a, const Place<T>& p, int lane, int left, bool first,
                                          const float* state, int64_t stride, float (&whole)[4]) {
    if (first) {
        float h[2];
        load_state<kWay>(state == nullptr ? nullptr : state + p.worker * stride + p.strip, lane, left, h);
        store_state<kWay>(a.first + static_cast<int64_t>(p.worker) * a.d + p.strip, lane, left, h);
#pragma unroll
        for (int k = 0; k < 2; ++k) whole[2 + k] = carry<true>(h[k], whole[k], whole[2 + k]), whole[k] = -0.0f;
    }
    const float one[2] = {whole[0], whole[1]}, two[2] = {whole[2], whole[3]};
    store_state<kWay>(a.a + p.at, lane, left, one);
    store_state<kWay>(a.b + p.at, lane, left, two);
}

// A segment's tokens tile by tile: kTime warps take a run each.
template <typename T, Way kWay, int kTime, int kRun, bool kBegins>
__global__ void __launch_bounds__(32 * kWarps, 2) relay_recurrence_kernel(RecurrenceArgs<T> a) {
    constexpr int kSide = kWarps / kTime, kTile = kTime * kRun;
    __shared__ float4 shared[2][kSide][kTime][32];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, slot = warp / kTime, part = warp % kTime;
    const Place<T> p(a, static_cast<int64_t>(blockIdx.x) * kSide + slot);
    const int left = p.on ? a.d - p.strip : 0, tiles = (min(a.segment, a.tokens) + kTile - 1) / kTile;
    const int end = p.on ? min(p.first + a.segment, a.tokens) : 0, to = min(end, p.length);
    float h[2];
    if (kTime < kWarps || a.segments == 1)
        load_state<kWay>(a.initial == nullptr ? nullptr : a.initial + p.worker * a.initial_stride + p.strip, lane, left, h);
    else if constexpr (kTime == kWarps)
        reach<kWay, false>(a, p, part, lane, left, shared[1][0], h);
    Two<T, kWay> gate[kRun], value[kRun];
    uint32_t begin;
    const auto ask = [&](int token) {
        load_run<kWay>(gate, a.gate, p.worker, token, p.strip, lane, left, to - token, kKeeps);
        load_run<kWay>(value, a.value, p.worker, token, p.strip, lane, left, to - token);
        begin = load_begins<kRun, kBegins>(a, p.worker, token, lane, to - token);
    };
    ask(p.first + part * kRun);
    for (int i = 0; i < tiles; ++i) {
        const int token = p.first + i * kTile + part * kRun;
        float f[kRun][2], b[kRun][2], ends[4], x[2];
        stretch<kBegins>(gate, value, begin, f, b, ends);
        if (i + 1 < tiles) ask(token + kTile);
        if constexpr (kTime > 1) {
            shared[i & 1][slot][part][lane] = make_float4(ends[0], ends[1], ends[2], ends[3]);
            __syncthreads();
            through<kTime, kBegins>(shared[i & 1][slot], part, lane, h, x);
        } else {
            x[0] = h[0], x[1] = h[1];
        }
        T* out = a.out.row(p.worker, token) + p.strip;
        if (token + kRun <= to) {
#pragma unroll
            for (int r = 0; r < kRun; ++r) {
#pragma unroll
                for (int k = 0; k < 2; ++k) x[k] = carry<kBegins>(x[k], f[r][k], b[r][k]);
                store_two<kWay>(token_of<kWay>(out, a.out.ts, r), lane, left, x);
            }
        } else {
#pragma unroll
            for (int r = 0; r < kRun; ++r) {
#pragma unroll
                for (int k = 0; k < 2; ++k) x[k] = carry<kBegins>(x[k], f[r][k], b[r][k]);
                const float y[2] = {token + r < to ? x[0] : 0.0f, token + r < to ? x[1] : 0.0f};
                if (token + r < end) store_two<kWay>(token_of<kWay>(out, a.out.ts, r), lane, left, y);
            }
        }
        if constexpr (kTime == 1) h[0] = x[0], h[1] = x[1];
    }
    if (p.segment == a.segments - 1 && a.last != nullptr && part == 0)
        store_state<kWay>(a.last + p.worker * a.last_stride + p.strip, lane, left, h);
}

// ------------------------------------------------------------- rows by tensor copies
//
// Rows that TMA takes (16-byte addresses and strides) come as boxes of 64 channels x a tile's
// tokens to shared memory, kStages tiles of them, so that neither registers nor addresses are
// spent on what is on its way.  A box may reach past the segment or the length: what it brings
// from there is left out.

constexpr int kStages = 3;

// Where the strips alone leave most SMs idle, clusters of kCtas CTAs take kCtas tiles side by
// side: the warps' stretches are joined to one a CTA, which goes to all of them.

template <typename T>
struct TileMaps {
    CUtensorMap gate, value, dout, out;
};

// Stages of kBoxes boxes of kTile tokens: the copies' barriers and the order of their places.
template <typename T, int kBoxes, int kTile>
struct Boxes {
    static constexpr int kBox = kTile * kWide * static_cast<int>(sizeof(T)), kStage = kBoxes * kBox;
    static constexpr int kShared = kStages * kStage + 128;
    Numbers<kStages, 1> tiles;
    uint32_t ring;  // in shared memory
    const uint8_t* at;
    __device__ __forceinline__ Boxes(uint64_t* barriers, uint8_t* raw) {
        const uint32_t pad = (128 - shared_address(raw) % 128) % 128;
        tiles.bars = shared_address(barriers), ring = shared_address(raw) + pad, at = raw + pad;
        if (threadIdx.x < kStages) barrier_init(tiles.bar(threadIdx.x), 1);
        barriers_ready();
        __syncthreads();
    }
    __device__ __forceinline__ uint32_t expect(int tile) const {  // returns the stage's place
        barrier_expect(tiles.bar(tile), kStage);
        return ring + tiles.place(tile) * kStage;
    }
    // The lane's two channels of token `token` of box `box`.
    __device__ __forceinline__ Two<T> get(int tile, int box, int token, int lane) const {
        return reinterpret_cast<const Two<T>*>(at + tiles.place(tile) * kStage + box * kBox)[token * (kWide / 2) + lane];
    }
};

// The stretches of a cluster's CTAs, in shared memory of each of them.
template <int kCtas>
struct Joined {
    float4 of[2][kCtas][32];
};

__device__ __forceinline__ void put_there(uint32_t at, float4 v) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}

// `h` goes from the state before the cluster's tiles to the one behind them, `mine` gets the one
// that reaches this warp: first through the CTAs before this one, then through its warps.
// Called by all threads of the cluster; on return all warps are done with the tile before.
template <int kCtas, bool kBegins>
__device__ __forceinline__ void hand_on(float4 (&shared)[kWarps][32], Joined<kCtas>& joined, int turn, int rank, int part, int lane,
                                        const float (&ends)[4], float (&h)[2], float (&mine)[2]) {
    shared[part][lane] = make_float4(ends[0], ends[1], ends[2], ends[3]);
    __syncthreads();
    if constexpr (kCtas == 1) {
        through<kWarps, kBegins>(shared, part, lane, h, mine);
    } else {
        if (part == 0) {
            float whole[4] = {ends[0], ends[1], ends[2], ends[3]};
#pragma unroll
            for (int j = 1; j < kWarps; ++j) {
                const float4 e = shared[j][lane];
                join<kBegins>(whole[0], whole[2], e.x, e.z);
                join<kBegins>(whole[1], whole[3], e.y, e.w);
            }
            const uint32_t at = shared_address(&joined.of[turn][rank][lane]);
#pragma unroll
            for (int q = 0; q < kCtas; ++q) put_there(in_cta(at, q), make_float4(whole[0], whole[1], whole[2], whole[3]));
        }
        cluster_sync();
        float first[2], behind[2];
        through<kCtas, kBegins>(joined.of[turn], rank, lane, h, first);
        behind[0] = first[0], behind[1] = first[1];
        through<kWarps, kBegins>(shared, part, lane, behind, mine);
    }
}

template <typename T, bool kBegins, int kCtas>
__global__ void __launch_bounds__(32 * kWarps, 2)
relay_recurrence_tiles_kernel(const __grid_constant__ RecurrenceArgs<T> a, const __grid_constant__ TileMaps<T> maps) {
    constexpr int kRun = kRunOf<T>, kTile = kWarps * kRun;
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t barriers[kStages];
    __shared__ float4 shared[2][kWarps][32];
    __shared__ Joined<kCtas> joined;
    Boxes<T, 2, kTile> boxes(barriers, raw);
    const int lane = threadIdx.x % 32, part = threadIdx.x / 32, rank = kCtas == 1 ? 0 : static_cast<int>(cluster_rank());
    const Place<T> p(a, blockIdx.x / kCtas);
    // rounds of kCtas tiles; this CTA's tile of a round
    const int left = a.d - p.strip, tiles = (min(a.segment, a.tokens) + kCtas * kTile - 1) / (kCtas * kTile);
    const auto first_of = [&](int i) { return p.first + (i * kCtas + rank) * kTile; };
    const int end = min(p.first + a.segment, a.tokens), to = min(end, p.length);
    const auto bring = [&](int i) {  // one thread
        const uint32_t at = boxes.expect(i);
        copy_box(at, &maps.gate, p.strip, first_of(i), p.worker, boxes.tiles.bar(i));
        copy_box(at + boxes.kBox, &maps.value, p.strip, first_of(i), p.worker, boxes.tiles.bar(i));
    };
    if (threadIdx.x == 0)
        for (int i = 0; i < min(kStages, tiles); ++i) bring(i);
    if (kCtas > 1) cluster_sync();  // the others have started
    float h[2];
    if (kCtas > 1 || a.segments == 1)
        load_state<kVector>(a.initial == nullptr ? nullptr : a.initial + p.worker * a.initial_stride + p.strip, lane, left, h);
    else
        reach<kVector, false>(a, p, part, lane, left, shared[1], h);
    const int start = first_of(0) + part * kRun;
    uint32_t begin = load_begins<kRun, kBegins>(a, p.worker, start, lane, to - start);
    for (int i = 0; i < tiles; ++i) {
        const int token = first_of(i) + part * kRun, counts = to - token;
        const uint32_t begins = kBegins ? __ballot_sync(0xffffffffu, begin != 0) : 0u;
        if (kBegins && i + 1 < tiles)
            begin = load_begins<kRun, kBegins>(a, p.worker, token + kCtas * kTile, lane, counts - kCtas * kTile);
        const bool ok = boxes.tiles.wait(i);
        float f[kRun][2], b[kRun][2], ends[4], x[2];
#pragma unroll
        for (int r = 0; r < kRun; ++r) {
            const Two<T> gate = boxes.get(i, 0, part * kRun + r, lane), value = boxes.get(i, 1, part * kRun + r, lane);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const Gate<T> g(gate.get(k));
                f[r][k] = kBegins && (begins >> r & 1) ? -0.0f : g.at;
                b[r][k] = g.rest * value.get(k);
            }
        }
        if (!ok) lose(b);
        if (counts < kRun) {
#pragma unroll
            for (int r = 0; r < kRun; ++r)
                if (r >= counts) f[r][0] = f[r][1] = 1.0f, b[r][0] = b[r][1] = 0.0f;
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            ends[k] = f[0][k], ends[2 + k] = b[0][k];
#pragma unroll
            for (int r = 1; r < kRun; ++r) join<kBegins>(ends[k], ends[2 + k], f[r][k], b[r][k]);
        }
        hand_on<kCtas, kBegins>(shared[i & 1], joined, i & 1, rank, part, lane, ends, h, x);
        const int next = boxes.tiles.asks(i) && boxes.tiles.next(i) < tiles ? boxes.tiles.next(i) : -1;
        if (threadIdx.x == 0 && next >= 0) bring(next);
        T* out = a.out.row(p.worker, token) + p.strip;
        if (counts >= kRun) {
#pragma unroll
            for (int r = 0; r < kRun; ++r) {
#pragma unroll
                for (int k = 0; k < 2; ++k) x[k] = carry<kBegins>(x[k], f[r][k], b[r][k]);
                store_two<kVector>(token_of<kVector>(out, a.out.ts, r), lane, left, x);
            }
        } else {
#pragma unroll
            for (int r = 0; r < kRun; ++r) {
#pragma unroll
                for (int k = 0; k < 2; ++k) x[k] = carry<kBegins>(x[k], f[r][k], b[r][k]);
                const float y[2] = {r < counts ? x[0] : 0.0f, r < counts ? x[1] : 0.0f};
                if (token + r < end) store_two<kVector>(token_of<kVector>(out, a.out.ts, r), lane, left, y);
            }
        }
    }
    if (threadIdx.x == 0) boxes.tiles.drain(tiles);
    if (p.segment == a.segments - 1 && a.last != nullptr && part == 0 && rank == 0)
        store_state<kVector>(a.last + p.worker * a.last_stride + p.strip, lane, left, h);
}

// A segment as one stretch: each of the CTA's warps takes a part of its tokens.
template <typename T, Way kWay, bool kBegins>
__global__ void __launch_bounds__(32 * kWarps, 2) relay_recurrence_ends_kernel(RecurrenceArgs<T> a) {
    constexpr int kRun = kRunOf<T, kWay>;
    __shared__ float4 shared[kWarps][32];
    const int lane = threadIdx.x % 32, part = threadIdx.x / 32;
    const Place<T> p(a, blockIdx.x);
    const int left = a.d - p.strip, each = (a.segment + kWarps - 1) / kWarps;
    const int first = p.first + part * each, to = min(min(first + each, p.first + a.segment), p.length);
    float whole[4] = {1.0f, 1.0f, 0.0f, 0.0f};
    Two<T, kWay> gate[kRun], value[kRun];
    uint32_t begin;
    const auto ask = [&](int token) {
        load_run<kWay>(gate, a.gate, p.worker, token, p.strip, lane, left, to - token, kKeeps);
        load_run<kWay>(value, a.value, p.worker, token, p.strip, lane, left, to - token);
        begin = load_begins<kRun, kBegins>(a, p.worker, token, lane, to - token);
    };
    ask(first);
    for (int token = first; token < to; token += kRun) {
        float f[kRun][2], b[kRun][2], ends[4];
        stretch<kBegins>(gate, value, begin, f, b, ends);
        ask(token + kRun);
#pragma unroll
        for (int k = 0; k < 2; ++k) join<kBegins>(whole[k], whole[2 + k], ends[k], ends[2 + k]);
    }
    shared[part][lane] = make_float4(whole[0], whole[1], whole[2], whole[3]);
    __syncthreads();
    if (part > 0) return;
    for (int j = 1; j < kWarps; ++j) {
        const float4 e = shared[j][lane];
        join<kBegins>(whole[0], whole[2], e.x, e.z);
        join<kBegins>(whole[1], whole[3], e.y, e.w);
    }
    keep_ends<kWay>(a, p, lane, left, p.segment == 0, a.initial, a.initial_stride, whole);
}

// ------------------------------------------------------------------ the backward pass
//
// With l_t the gradient that reaches h_t and m_t = f_t l_t what goes on to h_{t-1},
//   l_t = dout_t + m_{t+1},  dv_t = l_t (1 - f_t),  dgate_t = l_t (h_{t-1} - v_t) f_t (1 - f_t):
// from the last token to the first m is the same kind of recurrence, m -> f_t m + f_t dout_t.

// One token on the way back: `m` comes from behind it and goes on before it.
__device__ __forceinline__ void back_step(bool starts, float at, float rest, float dout, float before, float value, float& m,
                                          float& dg, float& dv) {
    const float l = dout + m;
    dv = l * rest;
    dg = dv * at * (before - value);
    m = starts ? 0.0f : at * l;
}

// The stretch (a, b) with the token before it.
__device__ __forceinline__ void back_join(bool starts, float at, float dout, float& a, float& b) {
    a = starts ? -0.0f : a * at;
    b = starts ? 0.0f : at * (b + dout);
}

// The run as one stretch, from its last token to its first.
template <bool kBegins, int kRun, typename T, Way kWay>
__device__ __forceinline__ void back_stretch(const Two<T, kWay> (&gate)[kRun], const Two<T, kWay> (&dout)[kRun], uint32_t begins,
                                             float (&ends)[4]) {
    ends[0] = ends[1] = 1.0f;
    ends[2] = ends[3] = 0.0f;
#pragma unroll
    for (int r = kRun - 1; r >= 0; --r)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const Gate<T> g(gate[r].get(k));
            back_join(kBegins && (begins >> r & 1), g.at, dout[r].get(k), ends[k], ends[2 + k]);
        }
}

// The forward kernel's tiles, from the segment's end to its start.  What the second sweep
// needs of the gate is made again from the row.
template <typename T, Way kWay, int kTime, int kRun, bool kBegins>
__global__ void __launch_bounds__(32 * kWarps, 2) relay_recurrence_backward_kernel(RecurrenceArgs<T> a) {
    constexpr int kSide = kWarps / kTime, kTile = kTime * kRun;
    __shared__ float4 shared[2][kSide][kTime][32];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, slot = warp / kTime, part = warp % kTime;
    const Place<T> p(a, static_cast<int64_t>(blockIdx.x) * kSide + slot);
    const int left = p.on ? a.d - p.strip : 0, tiles = (min(a.segment, a.tokens) + kTile - 1) / kTile;
    const int end = p.on ? min(p.first + a.segment, a.tokens) : 0, to = min(end, p.length);
    float m[2], first[2];
    if (kTime < kWarps || a.segments == 1)
        load_state<kWay>(a.dlast == nullptr ? nullptr : a.dlast + p.worker * a.dlast_stride + p.strip, lane, left, m);
    else if constexpr (kTime == kWarps)
        reach<kWay, true>(a, p, part, lane, left, shared[1][0], m);
    load_state<kWay>(a.initial == nullptr ? nullptr : a.initial + p.worker * a.initial_stride + p.strip, lane, left, first);
    Two<T, kWay> gate[kRun], dout[kRun], value[kRun], before[kRun];
    uint32_t begin;
    const auto ask = [&](int token) {
        const int counts = to - token;
        load_run<kWay>(gate, a.gate, p.worker, token, p.strip, lane, left, counts, kKeeps);
        load_run<kWay>(dout, a.dout, p.worker, token, p.strip, lane, left, counts);
        load_run<kWay>(value, a.value, p.worker, token, p.strip, lane, left, counts);
        // there is no row before the first
        load_run<kWay>(before, a.out_in, p.worker, token - 1, p.strip, lane, left, counts, 0.0f, token == 0);
        begin = load_begins<kRun, kBegins>(a, p.worker, token, lane, counts);
    };
    // warp 0 of a tile takes its last tokens
    const auto token_at = [&](int i) { return p.first + (tiles - 1 - i) * kTile + (kTime - 1 - part) * kRun; };
    if (tiles > 0) ask(token_at(0));  // (without tokens there is no tile, and nothing to read)
    for (int i = 0; i < tiles; ++i) {
        const int token = token_at(i);
        Two<T, kWay> g[kRun], dh[kRun], v[kRun], h[kRun];
#pragma unroll
        for (int r = 0; r < kRun; ++r) g[r] = gate[r], dh[r] = dout[r], v[r] = value[r], h[r] = before[r];
        const uint32_t begins = kBegins ? __ballot_sync(0xffffffffu, begin != 0) : 0u;
        if (i + 1 < tiles) ask(token_at(i + 1));
        float ends[4], x[2];
        if constexpr (kTime > 1) {
            back_stretch<kBegins>(g, dh, begins, ends);
            shared[i & 1][slot][part][lane] = make_float4(ends[0], ends[1], ends[2], ends[3]);
            __syncthreads();
            through<kTime, kBegins>(shared[i & 1][slot], part, lane, m, x);
        } else {
            x[0] = m[0], x[1] = m[1];
        }
        T *to_gate = a.dgate.row(p.worker, token) + p.strip, *to_value = a.dvalue.row(p.worker, token) + p.strip;
        const auto step = [&](int r, float (&dg)[2], float (&dv)[2]) {
            const bool starts = kBegins && (begins >> r & 1);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const Gate<T> s(g[r].get(k));
                const float h0 = starts ? 0.0f : r == 0 && token == 0 ? first[k] : h[r].get(k);
                back_step(starts, s.at, s.rest, dh[r].get(k), h0, v[r].get(k), x[k], dg[k], dv[k]);
            }
        };
        if (token + kRun <= to) {
#pragma unroll
            for (int r = kRun - 1; r >= 0; --r) {
                float dg[2], dv[2];
                step(r, dg, dv);
                store_two<kWay>(token_of<kWay>(to_gate, a.dgate.ts, r), lane, left, dg);
                store_two<kWay>(token_of<kWay>(to_value, a.dvalue.ts, r), lane, left, dv);
            }
        } else {
#pragma unroll
            for (int r = kRun - 1; r >= 0; --r) {
                float dg[2] = {0.0f, 0.0f}, dv[2] = {0.0f, 0.0f};
                if (token + r < to) step(r, dg, dv);
                if (token + r < end) {
                    store_two<kWay>(token_of<kWay>(to_gate, a.dgate.ts, r), lane, left, dg);
                    store_two<kWay>(token_of<kWay>(to_value, a.dvalue.ts, r), lane, left, dv);
                }
            }
        }
        if constexpr (kTime == 1) m[0] = x[0], m[1] = x[1];
    }
    if (p.segment == 0 && a.last != nullptr && part == 0)
        store_state<kWay>(a.last + p.worker * a.last_stride + p.strip, lane, left, m);
}

// The same with the rows by tensor copies.  What the first sweep makes of the gates stays for
// the second one.
template <typename T, bool kBegins, int kCtas>
__global__ void __launch_bounds__(32 * kWarps, 2)
relay_recurrence_backward_tiles_kernel(const __grid_constant__ RecurrenceArgs<T> a, const __grid_constant__ TileMaps<T> maps) {
    constexpr int kRun = kBackRunOf<T>, kTile = kWarps * kRun;
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t barriers[kStages];
    __shared__ float4 shared[2][kWarps][32];
    __shared__ Joined<kCtas> joined;
    Boxes<T, 4, kTile> boxes(barriers, raw);
    const int lane = threadIdx.x % 32, part = threadIdx.x / 32, rank = kCtas == 1 ? 0 : static_cast<int>(cluster_rank());
    const Place<T> p(a, blockIdx.x / kCtas);
    const int left = a.d - p.strip, tiles = (min(a.segment, a.tokens) + kCtas * kTile - 1) / (kCtas * kTile);
    // this CTA's tile of a round; CTA 0 has the last tokens
    const auto first_of = [&](int i) { return p.first + ((tiles - 1 - i) * kCtas + kCtas - 1 - rank) * kTile; };
    const int end = min(p.first + a.segment, a.tokens), to = min(end, p.length);
    const auto bring = [&](int i) {  // one thread
        const uint32_t at = boxes.expect(i), bar = boxes.tiles.bar(i);
        const int token = first_of(i);
        copy_box(at, &maps.gate, p.strip, token, p.worker, bar);
        copy_box(at + boxes.kBox, &maps.dout, p.strip, token, p.worker, bar);
        copy_box(at + 2 * boxes.kBox, &maps.value, p.strip, token, p.worker, bar);
        copy_box(at + 3 * boxes.kBox, &maps.out, p.strip, token - 1, p.worker, bar);  // (row -1 reads as 0)
    };
    if (threadIdx.x == 0)
        for (int i = 0; i < min(kStages, tiles); ++i) bring(i);
    if (kCtas > 1) cluster_sync();  // the others have started
    float m[2], first[2];
    if (kCtas > 1 || a.segments == 1)
        load_state<kVector>(a.dlast == nullptr ? nullptr : a.dlast + p.worker * a.dlast_stride + p.strip, lane, left, m);
    else
        reach<kVector, true>(a, p, part, lane, left, shared[1], m);
    load_state<kVector>(a.initial == nullptr ? nullptr : a.initial + p.worker * a.initial_stride + p.strip, lane, left, first);
    // warp 0 of a tile takes its last tokens
    const int place = (kWarps - 1 - part) * kRun;
    const auto token_at = [&](int i) { return first_of(i) + place; };
    uint32_t begin = tiles > 0 ? load_begins<kRun, kBegins>(a, p.worker, token_at(0), lane, to - token_at(0)) : 0;
    for (int i = 0; i < tiles; ++i) {
        const int token = token_at(i), counts = to - token;
        const uint32_t begins = kBegins ? __ballot_sync(0xffffffffu, begin != 0) : 0u;
        if (kBegins && i + 1 < tiles)
            begin = load_begins<kRun, kBegins>(a, p.worker, token - kCtas * kTile, lane, counts + kCtas * kTile);
        const bool ok = boxes.tiles.wait(i);
        float at[kRun][2], rest[kRun][2], ends[4] = {1.0f, 1.0f, 0.0f, 0.0f}, x[2];
#pragma unroll
        for (int r = kRun - 1; r >= 0; --r) {
            const Two<T> gate = boxes.get(i, 0, place + r, lane), dout = boxes.get(i, 1, place + r, lane);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const Gate<T> g(gate.get(k));
                at[r][k] = g.at, rest[r][k] = g.rest;
                if (r < counts) back_join(kBegins && (begins >> r & 1), g.at, dout.get(k), ends[k], ends[2 + k]);
            }
        }
        if (!ok && counts > 0) lose(at, rest, ends);
        hand_on<kCtas, kBegins>(shared[i & 1], joined, i & 1, rank, part, lane, ends, m, x);
        const int next = boxes.tiles.asks(i) && boxes.tiles.next(i) < tiles ? boxes.tiles.next(i) : -1;
        if (threadIdx.x == 0 && next >= 0) bring(next);
        T *to_gate = a.dgate.row(p.worker, token) + p.strip, *to_value = a.dvalue.row(p.worker, token) + p.strip;
        const auto step = [&](int r, float (&dg)[2], float (&dv)[2]) {
            const Two<T> dout = boxes.get(i, 1, place + r, lane), value = boxes.get(i, 2, place + r, lane),
                         before = boxes.get(i, 3, place + r, lane);
            const bool starts = kBegins && (begins >> r & 1);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float h0 = starts ? 0.0f : r == 0 && token == 0 ? first[k] : before.get(k);
                back_step(starts, at[r][k], rest[r][k], dout.get(k), h0, value.get(k), x[k], dg[k], dv[k]);
            }
        };
        if (counts >= kRun) {
#pragma unroll
            for (int r = kRun - 1; r >= 0; --r) {
                float dg[2], dv[2];
                step(r, dg, dv);
                store_two<kVector>(token_of<kVector>(to_gate, a.dgate.ts, r), lane, left, dg);
                store_two<kVector>(token_of<kVector>(to_value, a.dvalue.ts, r), lane, left, dv);
            }
        } else {
#pragma unroll
            for (int r = kRun - 1; r >= 0; --r) {
                float dg[2] = {0.0f, 0.0f}, dv[2] = {0.0f, 0.0f};
                if (r < counts) step(r, dg, dv);
                if (token + r < end) {
                    store_two<kVector>(token_of<kVector>(to_gate, a.dgate.ts, r), lane, left, dg);
                    store_two<kVector>(token_of<kVector>(to_value, a.dvalue.ts, r), lane, left, dv);
                }
            }
        }
    }
    if (threadIdx.x == 0) boxes.tiles.drain(tiles);
    if (p.segment == 0 && a.last != nullptr && part == 0 && rank == 0)
        store_state<kVector>(a.last + p.worker * a.last_stride + p.strip, lane, left, m);
}

template <typename T, Way kWay, bool kBegins>
__global__ void __launch_bounds__(32 * kWarps, 2) relay_recurrence_backward_ends_kernel(RecurrenceArgs<T> a) {
    constexpr int kRun = kRunOf<T, kWay>;
    __shared__ float4 shared[kWarps][32];
    const int lane = threadIdx.x % 32, part = threadIdx.x / 32;
    const Place<T> p(a, blockIdx.x);
    const int left = a.d - p.strip, each = (a.segment + kWarps - 1) / kWarps;
    const int first = p.first + part * each, to = min(min(first + each, p.first + a.segment), p.length);
    float whole[4] = {1.0f, 1.0f, 0.0f, 0.0f};
    const int runs = to > first ? (to - first + kRun - 1) / kRun : 0;
    Two<T, kWay> gate[kRun], dout[kRun];
    uint32_t begin = 0;
    const auto ask = [&](int token) {
        load_run<kWay>(gate, a.gate, p.worker, token, p.strip, lane, left, to - token, kKeeps);
        load_run<kWay>(dout, a.dout, p.worker, token, p.strip, lane, left, to - token);
        begin = load_begins<kRun, kBegins>(a, p.worker, token, lane, to - token);
    };
    if (runs > 0) ask(first + (runs - 1) * kRun);
    for (int i = runs - 1; i >= 0; --i) {
        Two<T, kWay> g[kRun], dh[kRun];
#pragma unroll
        for (int r = 0; r < kRun; ++r) g[r] = gate[r], dh[r] = dout[r];
        const uint32_t begins = kBegins ? __ballot_sync(0xffffffffu, begin != 0) : 0u;
        if (i > 0) ask(first + (i - 1) * kRun);
        float ends[4];
        back_stretch<kBegins>(g, dh, begins, ends);
#pragma unroll
        for (int k = 0; k < 2; ++k) join<kBegins>(whole[k], whole[2 + k], ends[k], ends[2 + k]);
    }
    shared[part][lane] = make_float4(whole[0], whole[1], whole[2], whole[3]);
    __syncthreads();
    if (part > 0) return;
    const float4 e0 = shared[kWarps - 1][lane];  // the last tokens come first
    whole[0] = e0.x, whole[1] = e0.y, whole[2] = e0.z, whole[3] = e0.w;
    for (int j = kWarps - 2; j >= 0; --j) {
        const float4 e = shared[j][lane];
        join<kBegins>(whole[0], whole[2], e.x, e.z);
        join<kBegins>(whole[1], whole[3], e.y, e.w);
    }
    keep_ends<kWay>(a, p, lane, left, p.segment == a.segments - 1, a.dlast, a.dlast_stride, whole);
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
    if (units < 152 && tokens >= 512) {
        segments = 304 / units;
        if (segments > tokens / 128) segments = tokens / 128;
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
           (tokens <= 1 || (r->token_stride % 2 == 0 && r->token_stride < (int64_t(1) << 30)));
}

// Whether TMA takes the rows: 16-byte steps, no row read twice.
bool boxed(const relay_rows* r, int32_t type, int32_t n, int64_t tokens, int64_t d) {
    constexpr int64_t kMost = int64_t(1) << 36;  // elements: a map's strides end at 2^40 bytes
    return vectors(r, type, n, tokens) && r->token_stride >= d && r->token_stride < kMost &&
           (n == 1 || (r->worker_stride >= d && r->worker_stride < kMost));
}

// The map of such rows for boxes of 64 channels x `high` tokens.
bool map_tiles(CUtensorMap* map, const relay_rows* r, int32_t type, int32_t n, int64_t tokens, int64_t d, int high) {
    const cuuint64_t e = static_cast<cuuint64_t>(element_size(type)), row = static_cast<cuuint64_t>(r->token_stride) * e;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(d), static_cast<cuuint64_t>(tokens), static_cast<cuuint64_t>(n)};
    const cuuint64_t strides[2] = {row, n > 1 ? static_cast<cuuint64_t>(r->worker_stride) * e : row};
    const cuuint32_t box[3] = {kWide, static_cast<cuuint32_t>(high), 1}, steps[3] = {1, 1, 1};
    const CUtensorMapDataType as = type == RELAY_BF16   ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                   : type == RELAY_FP16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                        : CU_TENSOR_MAP_DATA_TYPE_FLOAT32;
    return encoder()(map, as, 3, r->data, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
                     CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <auto Kernel, typename T>
int launch_tiles(const RecurrenceArgs<T>& a, const TileMaps<T>& maps, int64_t units, int ctas, int shared, cudaStream_t stream) {
    if (!allow_shared<Kernel>(shared)) return RELAY_ECUDA;
    cudaLaunchAttribute with = {};
    with.id = cudaLaunchAttributeClusterDimension;
    with.val.clusterDim.x = static_cast<unsigned>(ctas), with.val.clusterDim.y = 1, with.val.clusterDim.z = 1;
    cudaLaunchConfig_t how = {};
    how.gridDim = dim3(static_cast<unsigned>(units * ctas)), how.blockDim = dim3(32 * kWarps);
    how.dynamicSmemBytes = static_cast<size_t>(shared), how.stream = stream, how.attrs = &with, how.numAttrs = 1;
    if (cudaLaunchKernelEx(&how, Kernel, a, maps) == cudaSuccess) return RELAY_OK;
    (void)cudaGetLastError();
    return RELAY_ECUDA;
}

// CTAs that work side by side on a strip whose rows come by tensor copies, tiles of `tile`
// tokens: as many as come near to filling the SMs twice (a cluster of 8 leaves a few of them
// out), no more than there are tiles.  A round of a cluster costs a microsecond more than one
// CTA's, so that from half the SMs on a CTA a strip is faster.  0: segments are faster, which is
// so for a few strips and very many tokens.  Forward and backward in us, bf16, four calls one
// behind the other, as one CTA a strip / segments / clusters (of 4 from 64 strips on, else of 8):
//   [2][4096][4096]  43  75 / 63  90 /  57  99     [1][4096][4096]  38  67 / 32  47 /  26  50
//   [1][65536][256] 545 963 / 32  46 / 127 234     [1][4096][1024]  37  63 / 12  15 /  14  23
//   [1][2048][1024]           9  10 /   9  13
// The rule is from before segments found their states without a launch of their own; since then
// they are ahead of clusters at 16 strips of 4096 tokens, which it does not know.
int cluster_of(int64_t units, int64_t tokens, int tile) {
    if (units < 10 && tokens > 96 * tile) return 0;
    if (units <= 30 && tokens > 4 * tile) return 8;
    if (units <= 70 && tokens > 2 * tile) return 4;
    return 1;
}

// f(CTAs of a cluster) as a constant.
template <typename F>
int by_cluster(int ctas, F f) {
    return ctas == 8   ? f(std::integral_constant<int, 8>())
           : ctas == 4 ? f(std::integral_constant<int, 4>())
                       : f(std::integral_constant<int, 1>());
}

// f(way, warps that share a strip's tile, tokens of a warp's run) as constants: one warp a strip
// where its run holds all tokens, with a short run for few of them, and two where two runs do.
template <int kRun, typename W, typename F>
int by_time(W way, int64_t tokens, F f) {
    if (tokens <= 1) return f(way, std::integral_constant<int, 1>(), std::integral_constant<int, 1>());
    if (tokens <= 4) return f(way, std::integral_constant<int, 1>(), std::integral_constant<int, 4>());
    if (tokens <= kRun) return f(way, std::integral_constant<int, 1>(), std::integral_constant<int, kRun>());
    if (tokens <= 2 * kRun) return f(way, std::integral_constant<int, 2>(), std::integral_constant<int, kRun>());
    return f(way, std::integral_constant<int, kWarps>(), std::integral_constant<int, kRun>());
}

}  // namespace

extern "C" {

int64_t relay_recurrence_workspace(int32_t n, int64_t tokens, int64_t d) {
    if (const int rc = check_recurrence(RELAY_FP32, n, tokens, d)) return rc;
    const Cut cut = recurrence_cut(n, tokens, d);
    return cut.segments > 1 ? (8 * static_cast<int64_t>(cut.segments) + 4) * n * d : 0;
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
    Cut cut = recurrence_cut(n, tokens, d);
    const bool vec = tokens == 0 || (d % 2 == 0 && pairs(gate, type, n, tokens) && pairs(value, type, n, tokens) &&
                                     pairs(out, type, n, tokens));
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        constexpr int kTile = kWarps * kRunOf<T>;
        const bool boxes = vec && tokens > 2 * kRunOf<T> && boxed(gate, type, n, tokens, d) && boxed(value, type, n, tokens, d) &&
                           encoder() != nullptr;
        const int ctas = boxes ? cluster_of(static_cast<int64_t>(n) * cut.strips, tokens, kTile) : 0;
        if (ctas > 0) cut.segments = 1, cut.segment = static_cast<int>(tokens);
        RecurrenceArgs<T> a{};
        a.gate = view<const T>(gate, n, tokens), a.value = view<const T>(value, n, tokens), a.out = view<T>(out, n, tokens);
        a.initial = initial, a.initial_stride = n > 1 ? initial_stride : 0;
        a.last = last, a.last_stride = n > 1 ? last_stride : 0;
        a.begins = begins, a.lengths = lengths;
        a.a = static_cast<float*>(workspace), a.b = a.a + static_cast<int64_t>(n) * cut.segments * d;
        a.first = a.b + static_cast<int64_t>(n) * cut.segments * d;
        a.n = n, a.tokens = static_cast<int32_t>(tokens), a.d = static_cast<int32_t>(d);
        a.strips = cut.strips, a.segments = cut.segments, a.segment = cut.segment;
        const int64_t units = static_cast<int64_t>(n) * cut.segments * cut.strips;
        TileMaps<T> maps{};  // before anything is enqueued
        if (boxes && (!map_tiles(&maps.gate, gate, type, n, tokens, d, kTile) || !map_tiles(&maps.value, value, type, n, tokens, d, kTile)))
            return RELAY_ECUDA;
        if (cut.segments > 1) {
            (vec ? (begins != nullptr ? relay_recurrence_ends_kernel<T, kVector, true> : relay_recurrence_ends_kernel<T, kVector, false>)
                 : relay_recurrence_ends_kernel<T, kDirect, true>)
                <<<static_cast<unsigned>(units), 32 * kWarps, 0, stream>>>(a);
            if (const int rc = status_of_launch()) return rc;
        }
        if (boxes) {
            return by_cluster(ctas, [&](auto with) {
                constexpr int kCtas = decltype(with)::value, kShared = Boxes<T, 2, kTile>::kShared;
                return begins != nullptr
                           ? launch_tiles<relay_recurrence_tiles_kernel<T, true, kCtas>>(a, maps, units, kCtas, kShared, stream)
                           : launch_tiles<relay_recurrence_tiles_kernel<T, false, kCtas>>(a, maps, units, kCtas, kShared, stream);
            });
        }
        const auto go = [&](auto way, auto time, auto run) {
            constexpr Way kWay = decltype(way)::value;
            constexpr int kTime = decltype(time)::value, kRun = decltype(run)::value, kSide = kWarps / kTime;
            (kWay == kVector && begins == nullptr ? relay_recurrence_kernel<T, kWay, kTime, kRun, kWay == kDirect>
                                                  : relay_recurrence_kernel<T, kWay, kTime, kRun, true>)
                <<<static_cast<unsigned>((units + kSide - 1) / kSide), 32 * kWarps, 0, stream>>>(a);
            return status_of_launch();
        };
        return vec ? by_time<kRunOf<T, kVector>>(std::integral_constant<Way, kVector>(), cut.segment, go)
                   : by_time<kRunOf<T, kDirect>>(std::integral_constant<Way, kDirect>(), cut.segment, go);
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
    Cut cut = recurrence_cut(n, tokens, d);
    bool vec = d % 2 == 0 || tokens == 0;
    if (tokens > 0)
        for (const relay_rows* r : {dout, gate, value, out, dgate, dvalue}) vec = vec && pairs(r, type, n, tokens);
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        constexpr int kTile = kWarps * kBackRunOf<T>;
        bool boxes = vec && tokens > 2 * kBackRunOf<T> && encoder() != nullptr;
        if (boxes)
            for (const relay_rows* r : {dout, gate, value, out}) boxes = boxes && boxed(r, type, n, tokens, d);
        const int ctas = boxes ? cluster_of(static_cast<int64_t>(n) * cut.strips, tokens, kTile) : 0;
        if (ctas > 0) cut.segments = 1, cut.segment = static_cast<int>(tokens);
        RecurrenceArgs<T> a{};
        a.gate = view<const T>(gate, n, tokens), a.value = view<const T>(value, n, tokens);
        a.out_in = view<const T>(out, n, tokens), a.dout = view<const T>(dout, n, tokens);
        a.dgate = view<T>(dgate, n, tokens), a.dvalue = view<T>(dvalue, n, tokens);
        a.initial = initial, a.initial_stride = n > 1 ? initial_stride : 0;
        a.dlast = dlast, a.dlast_stride = n > 1 ? dlast_stride : 0;
        a.last = dinitial, a.last_stride = n > 1 ? dinitial_stride : 0;
        a.begins = begins, a.lengths = lengths;
        a.a = static_cast<float*>(workspace), a.b = a.a + static_cast<int64_t>(n) * cut.segments * d;
        a.first = a.b + static_cast<int64_t>(n) * cut.segments * d;
        a.n = n, a.tokens = static_cast<int32_t>(tokens), a.d = static_cast<int32_t>(d);
        a.strips = cut.strips, a.segments = cut.segments, a.segment = cut.segment;
        const int64_t units = static_cast<int64_t>(n) * cut.segments * cut.strips;
        TileMaps<T> maps{};  // before anything is enqueued
        if (boxes && (!map_tiles(&maps.gate, gate, type, n, tokens, d, kTile) || !map_tiles(&maps.value, value, type, n, tokens, d, kTile) ||
                      !map_tiles(&maps.dout, dout, type, n, tokens, d, kTile) || !map_tiles(&maps.out, out, type, n, tokens, d, kTile)))
            return RELAY_ECUDA;
        if (cut.segments > 1) {
            (vec ? (begins != nullptr ? relay_recurrence_backward_ends_kernel<T, kVector, true>
                                      : relay_recurrence_backward_ends_kernel<T, kVector, false>)
                 : relay_recurrence_backward_ends_kernel<T, kDirect, true>)
                <<<static_cast<unsigned>(units), 32 * kWarps, 0, stream>>>(a);
            if (const int rc = status_of_launch()) return rc;
        }
        if (boxes) {
            return by_cluster(ctas, [&](auto with) {
                constexpr int kCtas = decltype(with)::value, kShared = Boxes<T, 4, kTile>::kShared;
                return begins != nullptr
                           ? launch_tiles<relay_recurrence_backward_tiles_kernel<T, true, kCtas>>(a, maps, units, kCtas, kShared, stream)
                           : launch_tiles<relay_recurrence_backward_tiles_kernel<T, false, kCtas>>(a, maps, units, kCtas, kShared, stream);
            });
        }
        const auto go = [&](auto way, auto time, auto run) {
            constexpr Way kWay = decltype(way)::value;
            constexpr int kTime = decltype(time)::value, kRun = decltype(run)::value, kSide = kWarps / kTime;
            (kWay == kVector && begins == nullptr ? relay_recurrence_backward_kernel<T, kWay, kTime, kRun, kWay == kDirect>
                                                  : relay_recurrence_backward_kernel<T, kWay, kTime, kRun, true>)
                <<<static_cast<unsigned>((units + kSide - 1) / kSide), 32 * kWarps, 0, stream>>>(a);
            return status_of_launch();
        };
        return vec ? by_time<kBackRunOf<T, kVector>>(std::integral_constant<Way, kVector>(), cut.segment, go)
                   : by_time<kBackRunOf<T, kDirect>>(std::integral_constant<Way, kDirect>(), cut.segment, go);
    });
}

}  // extern "C"
