// block_norm.cu -- the step from one block of a model to the next (relaylayers.h), forward
// and backward, on GB300 (sm_103a): the block's output is normalised, gated and joined to
// the residual, and the sum normalised for the next block,
//
//   m = x s_x w_post;  h = rho r + sigma(z) m;  y = h s_h w_pre
//
// All rows in and all rows out once.  Any rows go through registers, kParts warps a row; many
// aligned ones come by bulk copies to shared memory, so that what is on its way takes no
// registers, and groups of warps wait only for their own row and sums.  Measured in bf16 with
// gate and scale, [4][4096][4096]: forward with the 8-bit output 125 us (740 MB, 5.9 TB/s), backward with
// dtotal 206 us and 5 us for the weights' sums (1074 MB, 5.1 TB/s).  Issue slots are 69 % and 64 %
// taken: a feature takes 52 and 78 instructions, and waits for sums and copies have 24 and 16
// warps to hide among.
#include <type_traits>

#include "blackwell.cuh"
#include "layers.cuh"

// Compiled once per pass (RELAY_PASS: 1 forward, 2 backward): the two halves build side by side.
namespace {

struct Weight {  // fp32, from worker to worker
    const float* p;
    int64_t stride;
    bool quads;
    template <Way kWay>
    __device__ __forceinline__ void load(int worker, int base, int lane, int left, float (&v)[8], float* turn) const {
        load_weight<kWay>(p + worker * stride + base, lane, left, quads, v, turn);
    }
};

constexpr int kQuads = 128;  // features that a warp takes four a lane

// Four features of a weight of any alignment, from feature `at` on.
__device__ __forceinline__ void load_quad_of(const Weight& w, int worker, int at, bool on, Pair (&v)[2]) {
    const float* p = w.p + worker * w.stride + at;
    if (w.quads) {
        load_quad(p, on, v);
    } else {
#pragma unroll
        for (int k = 0; k < 2; ++k) v[k] = on ? Pair(p[2 * k], p[2 * k + 1]) : Pair(0.0f);
    }
}

template <typename T>
struct BlockArgs {
    View<const T> x, gate, residual;
    View<T> total, y;
    Weight post, pre, scale;
    float eps;
    float* rstd;  // [2][n][tokens]
    int8_t* codes;
    uint8_t* scales;
    int32_t tokens, d, pitch;
};

template <typename T, Way kWay, int kParts, int kStrips>
__global__ void __launch_bounds__(32 * kNormWarps<kParts>, (kParts > 16 || kStrips > 2 ? 1 : kParts == 16 ? 2 : 4))
relay_block_norm_kernel(BlockArgs<T> a) {
    constexpr int kRows = kNormWarps<kParts> / kParts;
    __shared__ float shared[kNormWarps<kParts>];
    WARP_TURN(kNormWarps<kParts>, true);  // kVector: for unaligned weights
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, slot = warp / kParts, part = warp % kParts;
    const int worker = blockIdx.y, token = static_cast<int>(blockIdx.x) * kRows + slot;
    const bool on = token < a.tokens;
    const int64_t row = static_cast<int64_t>(worker) * a.tokens + token;
    const auto base_of = [&](int j) { return (part + kParts * j) * kStrip; };
    const auto left_of = [&](int j) { return on ? a.d - base_of(j) : 0; };

    Piece<T, kWay> x[kStrips], z[kStrips], r[kStrips];
    float h[kStrips][8], squares = 0.0f;
#pragma unroll
    for (int j = 0; j < kStrips; ++j) {
        x[j].load(a.x.row(worker, token) + base_of(j), lane, left_of(j));
        if (a.gate.p != nullptr) z[j].load(a.gate.row(worker, token) + base_of(j), lane, left_of(j));
        r[j].load(a.residual.row(worker, token) + base_of(j), lane, left_of(j));
    }
#pragma unroll
    for (int j = 0; j < kStrips; ++j) {
        x[j].get(h[j]);
#pragma unroll
        for (int k = 0; k < 8; ++k) squares = fmaf(h[j][k], h[j][k], squares);
    }
    squares = row_sum<kParts>(squares, shared, slot, part);
    const float sx = 1.0f / sqrtf(squares / static_cast<float>(a.d) + a.eps);
    squares = 0.0f;
#pragma unroll
    for (int j = 0; j < kStrips; ++j) {
        const int left = left_of(j);
        float w[8], v[8];
        a.post.template load<kWay>(worker, base_of(j), lane, left, w, turn);
#pragma unroll
        for (int k = 0; k < 8; ++k) h[j][k] *= sx * w[k];
        if (a.gate.p != nullptr) {
            z[j].get(v);
#pragma unroll
            for (int k = 0; k < 8; ++k) h[j][k] *= Gate<T>(v[k]).at;
        }
        r[j].get(v);
        if (a.scale.p != nullptr) {
            a.scale.template load<kWay>(worker, base_of(j), lane, left, w, turn);
#pragma unroll
            for (int k = 0; k < 8; ++k) h[j][k] = fmaf(w[k], v[k], h[j][k]);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) h[j][k] += v[k];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) squares = fmaf(h[j][k], h[j][k], squares);
    }
    squares = row_sum<kParts>(squares, shared, slot, part);
    if (!on) return;
    const float sh = 1.0f / sqrtf(squares / static_cast<float>(a.d) + a.eps);
    if (a.rstd != nullptr && part == 0 && lane == 0) {
        a.rstd[row] = sx;
        a.rstd[static_cast<int64_t>(gridDim.y) * a.tokens + row] = sh;
    }
#pragma unroll
    for (int j = 0; j < kStrips; ++j) {
        const int base = base_of(j), left = a.d - base;
        if (base >= a.pitch) break;
        if (a.total.p != nullptr) store_strip<kWay>(a.total.row(worker, token) + base, lane, left, h[j]);
#pragma unroll
        for (int k = 0; k < 8; ++k) h[j][k] *= sh;
        clear_past<kWay>(h[j], lane, left);
        if (a.codes != nullptr)
            put_strip<kWay>(a.codes + row * a.pitch, a.scales + row * (a.pitch / kBlock), base, lane, a.pitch, h[j],
                            kWay == kVector ? largest(h[j]) : 0u, turn);
        float w[8];
        a.pre.template load<kWay>(worker, base, lane, left, w, turn);
#pragma unroll
        for (int k = 0; k < 8; ++k) h[j][k] *= w[k];
        store_strip<kWay>(a.y.row(worker, token) + base, lane, left, h[j]);
    }
}

#if RELAY_PASS == 1

// The 8-bit format of four features a lane, a block on eight lanes: layers.cuh's put_strip.  `on`:
// there are any; past d v is 0, or NaN in a row whose factors are, and such a block's scale stays 7.
__device__ __forceinline__ void put_quad(int8_t* codes, uint8_t* scales, int at, int lane, bool on, const Pair (&v)[2]) {
    const float e[4] = {v[0].v.x, v[0].v.y, v[1].v.x, v[1].v.y};
    uint32_t most = max(max(magnitude(e[0]), magnitude(e[1])), max(magnitude(e[2]), magnitude(e[3])));
#pragma unroll
    for (int m = 1; m < 8; m *= 2) most = max(most, __shfl_xor_sync(0xffffffffu, most, m));
    const uint32_t c = scale_byte(most);
    const uint32_t ab = __byte_perm(code_bits(e[0], c), code_bits(e[1], c), 0x0040);
    const uint32_t cd = __byte_perm(code_bits(e[2], c), code_bits(e[3], c), 0x0040);
    *reinterpret_cast<uint32_t*>(codes + at) = c == 255u ? 0u : __byte_perm(ab, cd, 0x5410);
    if (lane % 8 == 0) scales[at / kBlock] = static_cast<uint8_t>(on ? c : 7u);
}

#endif  // RELAY_PASS

// Many aligned rows of up to 8192 features (4096 in fp32): they come by bulk copies to shared memory and h stays in
// registers.  The groups wait only for themselves; while one waits for its row or for one
// of the two sums, others are at work.
template <typename T, int kParts_, int kInputs>
struct Ring {
    static constexpr int kParts = kParts_;
    // the forward pass: 24 warps of 8 quads a lane, a row of each group at a time; the backward
    // pass: 16 (in fp32 8) of 4 quads, two rows of each group
    static constexpr bool kBack = kInputs == 5;
    static constexpr int kWarps = (kBack ? 16 : 24) / (sizeof(T) == 2 ? 1 : 2), kGroups = kWarps / kParts;
    static constexpr int kHold = kBack ? 4 : 8, kStages = kBack ? 2 : 1;
    static constexpr int kWide = kParts * kHold * kQuads;  // features of a row at most
    static constexpr int kRow = kWide * static_cast<int>(sizeof(T)), kStage = kInputs * kRow;  // bytes
    static constexpr bool kWeights = kWide <= 4096;  // there is room for the three weights too
    static constexpr int kRows = kGroups * kStages * kStage, kShared = kRows + (kWeights ? 3 * 4 * kWide : 0) + 16;
    static_assert(kShared <= 232448 - 2048, "shared memory of a CTA");
};

// The three weights, next to one another in shared memory: 0 past d, 1 where there are none.
template <typename R>
__device__ __forceinline__ void bring_weights(float* to, const Weight& post, const Weight& pre, const Weight& scale, int worker, int d) {
    const Weight* from[3] = {&post, &pre, &scale};
#pragma unroll
    for (int e = 0; e < 3; ++e)
        for (int k = threadIdx.x; k < R::kWide; k += 32 * R::kWarps)
            to[e * R::kWide + k] = k >= d ? 0.0f : from[e]->p == nullptr ? 1.0f : from[e]->p[worker * from[e]->stride + k];
}

// Features past d up to the next 128, which a row's copies leave out, are 0 from the start, so
// that a warp reads its 128 without asking which are there.
template <typename R, typename T>
__device__ __forceinline__ void clear_rest(uint8_t* ring, int d) {
    const int rest = (d + kQuads - 1) / kQuads * kQuads - d;
    for (int at = threadIdx.x; at < R::kRows / R::kRow * rest; at += 32 * R::kWarps)
        reinterpret_cast<T*>(ring + at / rest * R::kRow)[d + at % rest] = T(0.0f);
}

// Weight number e at feature `at`, from there or, in the widest rows, from memory.
template <typename R>
__device__ __forceinline__ void weight_at(const float* weights, int e, const Weight& w, int worker, int at, bool on, Pair (&v)[2]) {
    if constexpr (R::kWeights) {
        load_quad(weights + e * R::kWide + at, true, v);
    } else if (w.p != nullptr) {
        load_quad_of(w, worker, at, on, v);
    } else {
        v[0] = v[1] = Pair(1.0f);
    }
}

// Sums of kCount values over a group's warps, their lanes included.
template <int kParts, int kCount>
__device__ __forceinline__ void group_sum(float (&v)[kCount], float (&shared)[kParts][kCount], int group, int part, int lane) {
#pragma unroll
    for (int e = 0; e < kCount; ++e)
#pragma unroll
        for (int m = 16; m > 0; m >>= 1) v[e] += __shfl_xor_sync(0xffffffffu, v[e], m);
    if constexpr (kParts > 1) {
#pragma unroll
        for (int e = 0; e < kCount; ++e)
            if (lane == e) shared[part][e] = v[e];
        asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(32 * kParts) : "memory");
#pragma unroll
        for (int e = 0; e < kCount; ++e) {
            v[e] = 0.0f;
#pragma unroll
            for (int w = 0; w < kParts; ++w) v[e] += shared[w][e];
        }
    } else {
        __syncwarp();
    }
}

// kWhole: every warp has all its quads.  A wait that runs out makes a group's results from there
// on NaN.
template <typename T, int kParts, bool kWhole>
__global__ void __launch_bounds__(32 * Ring<T, kParts, 3>::kWarps, 1) relay_block_norm_rows_kernel(BlockArgs<T> a) {
    using R = Ring<T, kParts, 3>;
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[R::kGroups][R::kStages];
    __shared__ float shared[2][R::kGroups][kParts][1];
    uint8_t* ring = raw + (16 - shared_address(raw) % 16) % 16;
    float* weights = reinterpret_cast<float*>(ring + R::kRows);
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, group = warp / kParts, part = warp % kParts;
    const int worker = blockIdx.y;
    const bool gated = a.gate.p != nullptr;
    if (threadIdx.x < R::kGroups * R::kStages) barrier_init(shared_address(&bars[0][0] + threadIdx.x), 1);
    barriers_ready();
    if (R::kWeights) bring_weights<R>(weights, a.post, a.pre, a.scale, worker, a.d);
    const uint32_t bytes = static_cast<uint32_t>(a.d) * sizeof(T);
    clear_rest<R, T>(ring, a.d);
    __syncthreads();

    const int step = static_cast<int>(gridDim.x) * R::kGroups, begin = static_cast<int>(blockIdx.x) * R::kGroups + group;
    const bool brings = part == 0 && elected();
    uint8_t* mine = ring + group * (R::kStages * R::kStage);
    Numbers<R::kStages, 0> numbers{shared_address(&bars[group][0])};
    const auto bring = [&](int token, int i) {  // one thread of the group: its row number i
        const uint32_t bar = numbers.bar(i), to = shared_address(mine + numbers.place(i) * R::kStage);
        barrier_expect(bar, bytes * (2 + gated));
        copy_row(to, a.x.row(worker, token), bytes, bar);
        copy_row(to + R::kRow, a.residual.row(worker, token), bytes, bar);
        if (gated) copy_row(to + 2 * R::kRow, a.gate.row(worker, token), bytes, bar);
    };
    if (brings)
        for (int i = 0; i < R::kStages; ++i)
            if (begin + i * step < a.tokens) bring(begin + i * step, i);
    const float over_d = 1.0f / static_cast<float>(a.d);
    int i = 0;
    for (int token = begin; token < a.tokens; token += step, ++i) {
        const int64_t row = static_cast<int64_t>(worker) * a.tokens + token;
        const bool ok = numbers.wait(i);
        const T* from = reinterpret_cast<const T*>(mine + numbers.place(i) * R::kStage);
        constexpr int kNext = R::kRow / static_cast<int>(sizeof(T));
        Pair h[R::kHold][2], squares(0.0f);
#pragma unroll
        for (int j = 0; j < R::kHold; ++j) {
            const int base = (part + kParts * j) * kQuads, at = base + 4 * lane;
            if (!kWhole && base >= a.d) break;
            load_quad(from + at, true, h[j]);
#pragma unroll
            for (int k = 0; k < 2; ++k) squares = fma(h[j][k], h[j][k], squares);
        }
        float sum[1] = {ok ? squares.sum() : __int_as_float(0x7fffffff)};
        group_sum(sum, shared[0][group], group, part, lane);
        const float sx = 1.0f / sqrtf(sum[0] * over_d + a.eps);
        squares = Pair(0.0f);
#pragma unroll
        for (int j = 0; j < R::kHold; ++j) {
            const int base = (part + kParts * j) * kQuads, at = base + 4 * lane;
            const bool on = at < a.d;
            if (!kWhole && base >= a.d) break;
            Pair w[2], rho[2], z[2], r[2];
            load_quad(from + kNext + at, true, r);
            if (gated) load_quad(from + 2 * kNext + at, true, z);
            weight_at<R>(weights, 0, a.post, worker, at, on, w);
            weight_at<R>(weights, 2, a.scale, worker, at, on, rho);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                h[j][k] = h[j][k] * Pair(sx) * w[k];
                if (gated) h[j][k] = h[j][k] * Pair(Gate<T>(z[k].v.x).at, Gate<T>(z[k].v.y).at);
                h[j][k] = fma(rho[k], r[k], h[j][k]);
                squares = fma(h[j][k], h[j][k], squares);
            }
        }
        sum[0] = squares.sum();
        group_sum(sum, shared[1][group], group, part, lane);
        // here every warp of the group is done with the row in shared memory
        if (brings && numbers.asks(i) && token + R::kStages * step < a.tokens) bring(token + R::kStages * step, numbers.next(i));
        const float sh = 1.0f / sqrtf(sum[0] * over_d + a.eps);
        if (a.rstd != nullptr && part == 0 && lane == 0) {
            a.rstd[row] = sx;
            a.rstd[static_cast<int64_t>(gridDim.y) * a.tokens + row] = sh;
        }
#pragma unroll
        for (int j = 0; j < R::kHold; ++j) {
            const int base = (part + kParts * j) * kQuads, at = base + 4 * lane;
            const bool on = at < a.d;
            if (!kWhole && base >= a.d) break;  // (the pitch ends with d's last 128)
            Pair w[2];
            if (a.total.p != nullptr) store_quad(a.total.row(worker, token) + at, on, h[j]);
            weight_at<R>(weights, 1, a.pre, worker, at, on, w);
#pragma unroll
            for (int k = 0; k < 2; ++k) h[j][k] = h[j][k] * Pair(sh);
            if (a.codes != nullptr) put_quad(a.codes + row * a.pitch, a.scales + row * (a.pitch / kBlock), at, lane, on, h[j]);
#pragma unroll
            for (int k = 0; k < 2; ++k) h[j][k] = h[j][k] * w[k];
            store_quad(a.y.row(worker, token) + at, on, h[j]);
        }
    }
    if (brings) numbers.drain(i);
}

#if RELAY_PASS == 2

// ------------------------------------------------------------------ the backward pass
//
//   u = dy w_pre;  dh = s_h (u - hhat mean(u hhat)) + dtotal;  dr = rho dh;  drho = sum_t dh r
//   p = sigma(z);  dz = dh m p (1 - p);  v = dh p w_post;  dx = s_x (v - xhat mean(v xhat))
//   dw_post = sum_t dh p xhat;  dw_pre = sum_t dy hhat
//
// with xhat = x s_x and hhat = h s_h made again from the rows.  With a = p xhat w_post (h is
// rho r + a) the second mean is known with the first,
//
//   mean(v xhat) = mean(a (s_h u + dtotal)) - s_h mean(u hhat) mean(a hhat),
//
// so that a row waits for one sum over its warps, of three values.

template <typename T>
struct BlockBackwardArgs {
    View<const T> dy, dtotal, x, gate, residual;
    View<T> dx, dgate, dresidual;
    Weight post, pre, scale;
    const float* rstd;
    const int32_t* lengths;
    float* partial;  // [3][n][gridDim.x][pitch]: of w_post, w_pre, rho
    int32_t tokens, d, pitch;
};

// The factor of a row's norm where the row has come; NaN where the wait for it ran out, which
// makes everything NaN that Features make of the row.
__device__ __forceinline__ float factor_of(bool came, float s) { return came ? s : NAN; }

// What a lane makes again of 2 kPairs features of a row, two at a time: `xhat`, `p`, `r` come as x,
// gate and residual; w and rho are w_post and rho (1 without).
template <typename T, int kPairs>
struct Features {
    Pair xhat[kPairs], p[kPairs], q[kPairs], m[kPairs], r[kPairs], hhat[kPairs];
    __device__ __forceinline__ void make(const Pair (&w)[kPairs], const Pair (&rho)[kPairs], bool gated, float sx, float sh) {
#pragma unroll
        for (int k = 0; k < kPairs; ++k) {
            xhat[k] = xhat[k] * Pair(sx);
            m[k] = xhat[k] * w[k];
            if (gated) {
                const Gate<T> a(p[k].v.x), b(p[k].v.y);
                p[k] = Pair(a.at, b.at), q[k] = Pair(a.rest, b.rest);
            } else {
                p[k] = Pair(1.0f), q[k] = Pair(0.0f);
            }
            hhat[k] = fma(rho[k], r[k], p[k] * m[k]) * Pair(sh);
        }
    }
    // Adds to the three sums and to dw_pre.
    __device__ __forceinline__ void add(const Pair (&dy)[kPairs], const Pair (&pre)[kPairs], const Pair (&over)[kPairs], float sh,
                                        Pair (&sums)[3], Pair (&dpre)[kPairs]) const {
#pragma unroll
        for (int k = 0; k < kPairs; ++k) {
            const Pair u = dy[k] * pre[k], a = p[k] * m[k];
            dpre[k] = fma(dy[k], hhat[k], dpre[k]);
            sums[0] = fma(u, hhat[k], sums[0]);
            sums[1] = fma(a, fma(Pair(sh), u, over[k]), sums[1]);
            sums[2] = fma(a, hhat[k], sums[2]);
        }
    }
    // The three gradients of the rows (dy becomes dx), and what w_post and rho get of them.
    __device__ __forceinline__ void leave(Pair (&dy)[kPairs], const Pair (&pre)[kPairs], const Pair (&over)[kPairs], const Pair (&w)[kPairs],
                                          const Pair (&rho)[kPairs], float sx, float sh, float along, float along_x, Pair (&dz)[kPairs],
                                          Pair (&dr)[kPairs], Pair (&dpost)[kPairs], Pair (&dscale)[kPairs]) const {
#pragma unroll
        for (int k = 0; k < kPairs; ++k) {
            const Pair d = fma(Pair(sh), fma(hhat[k], Pair(-along), dy[k] * pre[k]), over[k]), dp = d * p[k];
            dr[k] = rho[k] * d;
            dz[k] = dp * m[k] * q[k];
            dscale[k] = fma(d, r[k], dscale[k]);
            dpost[k] = fma(dp, xhat[k], dpost[k]);
            dy[k] = Pair(sx) * fma(dp, w[k], xhat[k] * Pair(-along_x));
        }
    }
};

__device__ __forceinline__ void to_pairs(const float (&v)[8], Pair (&to)[4]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) to[k] = Pair(v[2 * k], v[2 * k + 1]);
}
__device__ __forceinline__ void from_pairs(const Pair (&v)[4], float (&to)[8]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) to[2 * k] = v[k].v.x, to[2 * k + 1] = v[k].v.y;
}

// Any rows: kParts warps share one, kStrips strips each, with what they need of it in
// registers.  CTA (p, i) takes tokens p, p + gridDim.x, ... (kRows at a time) of worker i and
// leaves their sums in its rows of `partial`.
template <typename T, Way kWay, int kParts, int kStrips>
__global__ void __launch_bounds__(32 * kNormWarps<kParts>, kNormWarps<kParts> > 8 ? 1 : 2)
relay_block_norm_backward_kernel(BlockBackwardArgs<T> a) {
    constexpr int kRows = kNormWarps<kParts> / kParts;
    __shared__ float shared[3][kNormWarps<kParts>];
    WARP_TURN(kNormWarps<kParts>, true);
    extern __shared__ float sums[];  // kRows > 1: [kRows - 1][kStrips][kParts][256]
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, slot = warp / kParts, part = warp % kParts;
    const int worker = blockIdx.y, n = gridDim.y;
    const int length = a.lengths == nullptr ? a.tokens : min(max(a.lengths[worker], 0), a.tokens);
    const auto base_of = [&](int j) { return (part + kParts * j) * kStrip; };

    Pair dpost[kStrips][4], dpre[kStrips][4], dscale[kStrips][4];
#pragma unroll
    for (int j = 0; j < kStrips; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) dpost[j][k] = dpre[j][k] = dscale[j][k] = Pair(0.0f);
    const int step = static_cast<int>(gridDim.x) * kRows;
    for (int first = static_cast<int>(blockIdx.x) * kRows; first < a.tokens; first += step) {
        const int token = first + slot;
        const bool counts = token < length;
        const int64_t row = static_cast<int64_t>(worker) * a.tokens + token;
        const float sx = counts ? a.rstd[row] : 0.0f, sh = counts ? a.rstd[static_cast<int64_t>(n) * a.tokens + row] : 0.0f;
        Piece<T, kWay> x[kStrips], z[kStrips], r[kStrips], dy[kStrips], dtotal[kStrips];
#pragma unroll
        for (int j = 0; j < kStrips; ++j) {
            const int base = base_of(j), left = counts ? a.d - base : 0;
            x[j].load(a.x.row(worker, token) + base, lane, left);
            if (a.gate.p != nullptr) z[j].load(a.gate.row(worker, token) + base, lane, left);
            r[j].load(a.residual.row(worker, token) + base, lane, left);
            dy[j].load(a.dy.row(worker, token) + base, lane, left);
            dtotal[j].load(a.dtotal.row(worker, token) + base, lane, a.dtotal.p != nullptr ? left : 0);
        }
        const auto remake = [&](int j, Features<T, 4>& o, Pair (&w)[4], Pair (&rho)[4], Pair (&pre)[4], Pair (&u)[4], Pair (&over)[4]) {
            const int base = base_of(j), left = counts ? a.d - base : 0;
            float v[8];
            x[j].get(v), to_pairs(v, o.xhat);
            r[j].get(v), to_pairs(v, o.r);
            dy[j].get(v), to_pairs(v, u);
            dtotal[j].get(v), to_pairs(v, over);
            if (a.gate.p != nullptr) z[j].get(v), to_pairs(v, o.p);
            a.post.template load<kWay>(worker, base, lane, left, v, turn), to_pairs(v, w);
            a.pre.template load<kWay>(worker, base, lane, left, v, turn), to_pairs(v, pre);
            if (a.scale.p != nullptr) {
                a.scale.template load<kWay>(worker, base, lane, left, v, turn), to_pairs(v, rho);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) rho[k] = Pair(1.0f);
            }
            o.make(w, rho, a.gate.p != nullptr, sx, sh);
        };
        Pair parts[3] = {Pair(0.0f), Pair(0.0f), Pair(0.0f)};
        float three[3];
#pragma unroll
        for (int j = 0; j < kStrips; ++j) {
            Features<T, 4> o;
            Pair w[4], rho[4], pre[4], u[4], over[4];
            remake(j, o, w, rho, pre, u, over);
            o.add(u, pre, over, sh, parts, dpre[j]);
        }
#pragma unroll
        for (int e = 0; e < 3; ++e) three[e] = row_sum<kParts>(parts[e].sum(), shared[e], slot, part) / static_cast<float>(a.d);
        if (token >= a.tokens) continue;
        const float along = three[0], along_x = three[1] - sh * along * three[2];
#pragma unroll
        for (int j = 0; j < kStrips; ++j) {
            const int base = base_of(j), left = a.d - base;
            if (left <= 0) break;
            Features<T, 4> o;
            Pair w[4], rho[4], pre[4], u[4], over[4], dz[4], dr[4];
            if (counts) {
                remake(j, o, w, rho, pre, u, over);
                o.leave(u, pre, over, w, rho, sx, sh, along, along_x, dz, dr, dpost[j], dscale[j]);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) u[k] = dz[k] = dr[k] = Pair(0.0f);
            }
            float v[8];
            from_pairs(u, v), store_strip<kWay>(a.dx.row(worker, token) + base, lane, left, v);
            from_pairs(dr, v), store_strip<kWay>(a.dresidual.row(worker, token) + base, lane, left, v);
            if (a.dgate.p != nullptr) from_pairs(dz, v), store_strip<kWay>(a.dgate.row(worker, token) + base, lane, left, v);
        }
    }
    const auto leave = [&](Pair (&pairs)[kStrips][4], int which) {
        float v[kStrips][8];
#pragma unroll
        for (int j = 0; j < kStrips; ++j) from_pairs(pairs[j], v[j]);
        if (kRows > 1) {  // the rows that went side by side, in their order
            __syncthreads();
            if (slot > 0) {
#pragma unroll
                for (int j = 0; j < kStrips; ++j)
#pragma unroll
                    for (int k = 0; k < 8; ++k) sums[(((slot - 1) * kStrips + j) * kParts + part) * kStrip + 32 * k + lane] = v[j][k];
            }
            __syncthreads();
            if (slot > 0) return;
            for (int s = 0; s < kRows - 1; ++s)
#pragma unroll
                for (int j = 0; j < kStrips; ++j)
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[j][k] += sums[((s * kStrips + j) * kParts + part) * kStrip + 32 * k + lane];
        }
        float* out = a.partial + ((static_cast<int64_t>(which) * n + worker) * gridDim.x + blockIdx.x) * a.pitch;
#pragma unroll
        for (int j = 0; j < kStrips; ++j) store_strip<kWay>(out + base_of(j), lane, a.pitch - base_of(j), v[j]);
    };
    leave(dpost, 0);
    leave(dpre, 1);
    if (a.scale.p != nullptr) leave(dscale, 2);
}

// The rows that the forward pass's kernel of bulk copies takes, here with two sweeps over a
// row in shared memory, so that registers are left for the sums over the tokens.  The groups of a CTA take rows of their own and wait only for themselves.
// kWhole: every warp has all its quads.  A wait that runs out makes a group's results from there
// on NaN.
template <typename T, int kParts, bool kWhole>
__global__ void __launch_bounds__(32 * Ring<T, kParts, 5>::kWarps, 1) relay_block_norm_backward_rows_kernel(BlockBackwardArgs<T> a) {
    using R = Ring<T, kParts, 5>;
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[R::kGroups][R::kStages];
    __shared__ float shared[2][R::kGroups][kParts][3];
    uint8_t* ring = raw + (16 - shared_address(raw) % 16) % 16;
    float* weights = reinterpret_cast<float*>(ring + R::kRows);  // post, pre, rho
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, group = warp / kParts, part = warp % kParts;
    const int worker = blockIdx.y, n = gridDim.y;
    const int length = a.lengths == nullptr ? a.tokens : min(max(a.lengths[worker], 0), a.tokens);
    const bool gated = a.gate.p != nullptr, over_too = a.dtotal.p != nullptr, scaled = a.scale.p != nullptr;
    if (threadIdx.x < R::kGroups * R::kStages) barrier_init(shared_address(&bars[0][0] + threadIdx.x), 1);
    barriers_ready();
    if (R::kWeights) bring_weights<R>(weights, a.post, a.pre, a.scale, worker, a.d);
    const uint32_t bytes = static_cast<uint32_t>(a.d) * sizeof(T);
    clear_rest<R, T>(ring, a.d);
    __syncthreads();

    const int step = static_cast<int>(gridDim.x) * R::kGroups, begin = static_cast<int>(blockIdx.x) * R::kGroups + group;
    const bool brings = part == 0 && elected();
    uint8_t* mine = ring + group * (R::kStages * R::kStage);
    Numbers<R::kStages, 1> numbers{shared_address(&bars[group][0])};
    const auto bring = [&](int token, int i) {  // one thread of the group: its row number i
        const uint32_t bar = numbers.bar(i), to = shared_address(mine + numbers.place(i) * R::kStage);
        barrier_expect(bar, bytes * (3 + gated + over_too));
        copy_row(to, a.x.row(worker, token), bytes, bar);
        copy_row(to + R::kRow, a.residual.row(worker, token), bytes, bar);
        copy_row(to + 2 * R::kRow, a.dy.row(worker, token), bytes, bar);
        if (gated) copy_row(to + 3 * R::kRow, a.gate.row(worker, token), bytes, bar);
        if (over_too) copy_row(to + 4 * R::kRow, a.dtotal.row(worker, token), bytes, bar);
    };
    if (brings)
        for (int i = 0; i < R::kStages; ++i)
            if (begin + i * step < length) bring(begin + i * step, i);
    Pair dpost[4][2], dpre[4][2], dscale[4][2];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int k = 0; k < 2; ++k) dpost[j][k] = dpre[j][k] = dscale[j][k] = Pair(0.0f);
    const float* factors = a.rstd + static_cast<int64_t>(worker) * a.tokens;
    const int64_t second = static_cast<int64_t>(n) * a.tokens;
    float next_x = begin < length ? factors[begin] : 0.0f, next_h = begin < length ? factors[second + begin] : 0.0f;
    const float over_d = 1.0f / static_cast<float>(a.d);
    int i = 0;
    for (int token = begin; token < length; token += step, ++i) {
        const float row_x = next_x, row_h = next_h;
        if (token + step < length) next_x = factors[token + step], next_h = factors[second + token + step];
        const bool ok = numbers.wait(i);
        const float sx = factor_of(ok, row_x), sh = factor_of(ok, row_h);
        const auto remake = [&](int j, Features<T, 2>& o, Pair (&w)[2], Pair (&rho)[2], Pair (&pre)[2], Pair (&u)[2], Pair (&over)[2]) {
            const int at = (part + kParts * j) * kQuads + 4 * lane;
            const bool on = at < a.d;
            const T* from = reinterpret_cast<const T*>(mine + numbers.place(i) * R::kStage) + at;
            constexpr int kNext = R::kRow / static_cast<int>(sizeof(T));
            load_quad(from, true, o.xhat);
            load_quad(from + kNext, true, o.r);
            load_quad(from + 2 * kNext, true, u);
            if (gated) load_quad(from + 3 * kNext, true, o.p);
            load_quad(from + 4 * kNext, over_too, over);
            weight_at<R>(weights, 0, a.post, worker, at, on, w);
            weight_at<R>(weights, 1, a.pre, worker, at, on, pre);
            weight_at<R>(weights, 2, a.scale, worker, at, on, rho);
            o.make(w, rho, gated, sx, sh);
        };
        Pair parts[3] = {Pair(0.0f), Pair(0.0f), Pair(0.0f)};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (!kWhole && (part + kParts * j) * kQuads >= a.d) break;
            Features<T, 2> o;
            Pair w[2], rho[2], pre[2], u[2], over[2];
            remake(j, o, w, rho, pre, u, over);
            o.add(u, pre, over, sh, parts, dpre[j]);
        }
        float three[3];
#pragma unroll
        for (int e = 0; e < 3; ++e) three[e] = parts[e].sum();
        group_sum(three, shared[i & 1][group], group, part, lane);
        // here every warp of the group is done with the row before this one
        if (brings && numbers.asks(i) && token + step < length) bring(token + step, numbers.next(i));
        const float along = three[0] * over_d, along_x = three[1] * over_d - sh * along * (three[2] * over_d);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int base = (part + kParts * j) * kQuads, at = base + 4 * lane;
            const bool on = at < a.d;
            if (!kWhole && base >= a.d) break;
            Features<T, 2> o;
            Pair w[2], rho[2], pre[2], u[2], over[2], dz[2], dr[2];
            remake(j, o, w, rho, pre, u, over);
            o.leave(u, pre, over, w, rho, sx, sh, along, along_x, dz, dr, dpost[j], dscale[j]);
            store_quad(a.dx.row(worker, token) + at, on, u);
            store_quad(a.dresidual.row(worker, token) + at, on, dr);
            if (gated) store_quad(a.dgate.row(worker, token) + at, on, dz);
        }
    }
    if (brings) numbers.drain(i);
    // padding
    for (int token = begin + i * step; token < a.tokens; token += step) {
        const Pair none[2] = {Pair(0.0f), Pair(0.0f)};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int at = (part + kParts * j) * kQuads + 4 * lane;
            const bool on = at < a.d;
            store_quad(a.dx.row(worker, token) + at, on, none);
            store_quad(a.dresidual.row(worker, token) + at, on, none);
            if (gated) store_quad(a.dgate.row(worker, token) + at, on, none);
        }
    }
    // the groups' sums in their order, through the ring's memory: [kGroups - 1][kWide]
    float* others = reinterpret_cast<float*>(ring);
    const auto leave = [&](Pair (&v)[4][2], int which) {
        if (R::kGroups > 1) {
            __syncthreads();
            if (group > 0) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    store_quad(others + (group - 1) * R::kWide + (part + kParts * j) * kQuads + 4 * lane, true, v[j]);
            }
            __syncthreads();
            if (group > 0) return;
            for (int g = 0; g < R::kGroups - 1; ++g)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    Pair add[2];
                    load_quad(others + g * R::kWide + (part + kParts * j) * kQuads + 4 * lane, true, add);
#pragma unroll
                    for (int k = 0; k < 2; ++k) v[j][k] = fma(add[k], Pair(1.0f), v[j][k]);
                }
        }
        float* out = a.partial + ((static_cast<int64_t>(which) * n + worker) * gridDim.x + blockIdx.x) * a.pitch;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int at = (part + kParts * j) * kQuads + 4 * lane;
            store_quad(out + at, at < a.pitch, v[j]);
        }
    };
    leave(dpost, 0);
    leave(dpre, 1);
    if (scaled) leave(dscale, 2);
}

struct Sums {  // where the three sums go
    float* p[3];
    int64_t stride[3];
};

// out[i][k] = sum_p partial[i][p][k]: a CTA sums 128 columns, 8 rows at a time.
__global__ void __launch_bounds__(256) relay_block_norm_join_kernel(const float* partial, int parts, int d, int pitch, Sums to) {
    __shared__ float4 shared[8][32];
    const int lane = threadIdx.x % 32, column = blockIdx.x * 128 + 4 * lane, lead = threadIdx.x / 32, which = blockIdx.z;
    if (to.p[which] == nullptr) return;
    const float* p = partial + (static_cast<int64_t>(which) * gridDim.y + blockIdx.y) * parts * pitch;
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const auto add = [&](float4 v) { s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w; };
#pragma unroll 4
    for (int r = lead; r < parts; r += 8) add(*reinterpret_cast<const float4*>(p + static_cast<int64_t>(r) * pitch + column));
    shared[lead][lane] = s;
    __syncthreads();
    if (lead > 0) return;
#pragma unroll
    for (int r = 1; r < 8; ++r) add(shared[r][lane]);
    const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (column + k < d) to.p[which][blockIdx.y * to.stride[which] + column + k] = v[k];
}

#endif  // RELAY_PASS

// ---------------------------------------------------------------- launching

// f(R) for the Ring with the fewest warps a row that holds one; none (false) where the CTA's
// warps do not.
template <typename T, int kInputs, int kParts = 1, typename F>
bool by_ring(int64_t d, F f) {
    using R = Ring<T, kParts, kInputs>;
    if (d <= R::kWide) {
        f(R());
        return true;
    }
    if constexpr (R::kWarps % (2 * kParts) == 0 && R::kWarps >= 2 * kParts) return by_ring<T, kInputs, 2 * kParts>(d, f);
    return false;
}

// Whether rows go through shared memory: where that is faster, by what was measured, old way and
// this one in us, 4 workers:
//   backward  [512 rows][1000] bf16  10.5 12.6, [1024][1000] 14.7 12.7, [16384][512] 58 37,
//             [8192][4096] 226 110, [8192][8192] 735 287, fp32 [8192][4096] 324 228
//   forward   [2048][4096] bf16 18.7 20.7, [4096][4096] 39 37, [8192][2048] 44 35,
//             [8192][4096] 70 62, fp32 [8192][4096] 114 116
template <typename T, int kInputs>
bool takes_ring(int32_t n, int64_t tokens, int64_t d) {
    const bool fits = by_ring<T, kInputs>(d, [](auto) {});
    return fits && (kInputs == 5 ? n * tokens * d >= 1 << 20 : n * tokens * d >= 1 << 24);
}

bool weight_fits(const float* p, int64_t stride) { return p != nullptr && aligned(p, 4) && stride >= 0; }

Weight weight_of(const float* p, int64_t stride, int32_t n, int64_t d) {
    return Weight{p, n > 1 ? stride : 0, d % 8 == 0 && aligned(p, 16) && (n == 1 || stride % 4 == 0)};
}

#if RELAY_PASS == 1

int64_t ring_ctas(int32_t n) { return 152 > n ? 152 / n : 1; }  // of a worker

#else

// Calls f(kParts, kStrips) for the backward pass, whose sums over the tokens take three
// times a strip's registers: one strip a warp as far as a CTA's 32 warps go.
template <typename F>
int by_back_width(int64_t pitch, F f) {
    if (pitch <= 256) return f(Hold<1, 1>());
    if (pitch <= 512) return f(Hold<2, 1>());
    if (pitch <= 1024) return f(Hold<4, 1>());
    if (pitch <= 2048) return f(Hold<8, 1>());
    if (pitch <= 4096) return f(Hold<16, 1>());
    if (pitch <= 8192) return f(Hold<32, 1>());
    if (pitch <= 16384) return f(Hold<32, 2>());
    return f(Hold<32, 4>());
}

// Rows of partial sums per worker, one per CTA: as many CTAs as are resident over all
// workers (two per SM where they have 8 warps), no more than take a token each; multiples
// where a thread would add up more than 256 rows in one chain.  The kernel of the aligned
// rows takes at least as many side by side.
int64_t block_partials(int32_t n, int64_t tokens, int64_t d) {
    const int64_t pitch = pitch_of(d), side = pitch <= 256 ? 8 : pitch <= 512 ? 4 : pitch <= 1024 ? 2 : 1;  // kRows
    const int64_t slots = pitch <= 2048 ? 304 : 152, fill = slots > n ? slots / n : 1, chain = fill * side * 256;
    const int64_t want = tokens > chain ? fill * ((tokens + chain - 1) / chain) : fill, most = (tokens + side - 1) / side;
    return most < want ? (most > 0 ? most : 1) : want;
}

// The same for the kernel of the aligned rows, one CTA per SM; never more than the above.
template <typename T, int kParts>
int64_t ring_partials(int32_t n, int64_t tokens, int64_t d) {
    const int64_t side = Ring<T, kParts, 5>::kGroups, fill = 152 > n ? 152 / n : 1, chain = fill * side * 256;
    const int64_t want = tokens > chain ? fill * ((tokens + chain - 1) / chain) : fill, most = (tokens + side - 1) / side;
    const int64_t parts = most < want ? (most > 0 ? most : 1) : want, room = block_partials(n, tokens, d);
    return parts < room ? parts : room;
}

template <typename T, int kParts, bool kWhole>
int launch_rows(const BlockBackwardArgs<T>& a, int64_t parts, int32_t n, cudaStream_t stream) {
    constexpr auto kernel = relay_block_norm_backward_rows_kernel<T, kParts, kWhole>;
    if (!allow_shared<kernel>(Ring<T, kParts, 5>::kShared)) return RELAY_ECUDA;
    kernel<<<dim3(static_cast<unsigned>(parts), n), 32 * Ring<T, kParts, 5>::kWarps, Ring<T, kParts, 5>::kShared, stream>>>(a);
    return status_of_launch();
}

bool gradient_fits(const float* p, int64_t stride, int32_t n, int64_t d) {
    return p != nullptr && aligned(p, 4) && (n == 1 || stride >= d);
}

#endif  // RELAY_PASS

}  // namespace

extern "C" {

#if RELAY_PASS == 1

int relay_block_norm(int32_t type, int32_t n, int64_t tokens, int64_t d, const relay_rows* x, const relay_rows* gate,
                     const relay_rows* residual, const float* post, int64_t post_stride, const float* pre, int64_t pre_stride,
                     const float* scale, int64_t scale_stride, float eps, const relay_rows* total, const relay_rows* y,
                     float* rstd, int8_t* codes, uint8_t* scales, relay_stream_t stream) {
    if (const int rc = check_shape(type, n, tokens, d)) return rc;
    if (d > RELAY_NORM_MAX_D) return RELAY_EUNSUPPORTED;
    if (!(eps > 0.0f) || !(eps < 1e30f) || !weight_fits(post, post_stride) || !weight_fits(pre, pre_stride) ||
        (scale != nullptr && !weight_fits(scale, scale_stride)))
        return RELAY_EINVAL;
    if (!rows_fit(x, type, n, tokens, d, false) || !rows_fit(residual, type, n, tokens, d, false) ||
        !rows_fit(y, type, n, tokens, d, true) || (gate != nullptr && !rows_fit(gate, type, n, tokens, d, false)) ||
        (total != nullptr && !rows_fit(total, type, n, tokens, d, true)))
        return RELAY_EINVAL;
    if (!aligned(rstd, 4) || (codes == nullptr) != (scales == nullptr)) return RELAY_EINVAL;
    if (codes != nullptr && !checkpoint_fits(codes, scales, tokens)) return RELAY_EINVAL;
    if (tokens == 0) return RELAY_OK;
    for (const relay_rows* in : {x, gate, residual, total})
        if (in != nullptr && y->data == in->data) return RELAY_EINVAL;
    if ((total != nullptr && gate != nullptr && total->data == gate->data) || crossed(total, x, n, tokens) ||
        crossed(total, residual, n, tokens))
        return RELAY_EINVAL;
    const bool vec = d % 8 == 0 && vectors(x, type, n, tokens) && vectors(gate, type, n, tokens) &&
                     vectors(residual, type, n, tokens) && vectors(total, type, n, tokens) && vectors(y, type, n, tokens);
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        const BlockArgs<T> a{view<const T>(x, n, tokens), view<const T>(gate, n, tokens), view<const T>(residual, n, tokens),
                             view<T>(total, n, tokens), view<T>(y, n, tokens), weight_of(post, post_stride, n, d),
                             weight_of(pre, pre_stride, n, d), weight_of(scale, scale_stride, n, d), eps, rstd, codes, scales,
                             static_cast<int32_t>(tokens), static_cast<int32_t>(d), static_cast<int32_t>(pitch_of(d))};
        if constexpr (sizeof(T) == 2) {
            if (vec && takes_ring<T, 3>(n, tokens, d)) {
                int rc = RELAY_OK;
                by_ring<T, 3>(d, [&](auto r) {
                    using R = decltype(r);
                    const auto go = [&](auto whole) {
                        constexpr auto kernel = relay_block_norm_rows_kernel<T, R::kParts, decltype(whole)::value>;
                        if (!allow_shared<kernel>(R::kShared)) return RELAY_ECUDA;
                        const dim3 grid(static_cast<unsigned>(ring_ctas(n)), static_cast<unsigned>(n));
                        kernel<<<grid, 32 * R::kWarps, R::kShared, stream>>>(a);
                        return status_of_launch();
                    };
                    rc = d > R::kWide - kQuads ? go(std::true_type()) : go(std::false_type());
                });
                return rc;
            }
        }
        return by_width(a.pitch, [&](auto hold) {
            constexpr int kParts = decltype(hold)::kParts, kStrips = decltype(hold)::kStrips;
            constexpr int kRows = kNormWarps<kParts> / kParts;
            const dim3 grid(static_cast<unsigned>((tokens + kRows - 1) / kRows), static_cast<unsigned>(n));
            (vec ? relay_block_norm_kernel<T, kVector, kParts, kStrips> : relay_block_norm_kernel<T, kDirect, kParts, kStrips>)
                <<<grid, 32 * kNormWarps<kParts>, 0, stream>>>(a);
            return status_of_launch();
        });
    });
}

#else

int64_t relay_block_norm_backward_workspace(int32_t n, int64_t tokens, int64_t d) {
    if (const int rc = check_shape(RELAY_FP32, n, tokens, d)) return rc;
    if (d > RELAY_NORM_MAX_D) return RELAY_EUNSUPPORTED;
    return 12 * n * block_partials(n, tokens, d) * pitch_of(d);
}

int relay_block_norm_backward(int32_t type, int32_t n, int64_t tokens, int64_t d, const relay_rows* dy,
                              const relay_rows* dtotal, const relay_rows* x, const relay_rows* gate,
                              const relay_rows* residual, const float* post, int64_t post_stride, const float* pre,
                              int64_t pre_stride, const float* scale, int64_t scale_stride, const float* rstd,
                              const int32_t* lengths, const relay_rows* dx, const relay_rows* dgate,
                              const relay_rows* dresidual, float* dpost, int64_t dpost_stride, float* dpre,
                              int64_t dpre_stride, float* dscale, int64_t dscale_stride, void* workspace,
                              int64_t workspace_bytes, relay_stream_t stream) {
    if (const int rc = check_shape(type, n, tokens, d)) return rc;
    if (d > RELAY_NORM_MAX_D) return RELAY_EUNSUPPORTED;
    if (!weight_fits(post, post_stride) || !weight_fits(pre, pre_stride) ||
        (scale != nullptr && !weight_fits(scale, scale_stride)))
        return RELAY_EINVAL;
    for (const relay_rows* in : {dy, x, residual})
        if (!rows_fit(in, type, n, tokens, d, false)) return RELAY_EINVAL;
    for (const relay_rows* in : {dtotal, gate})
        if (in != nullptr && !rows_fit(in, type, n, tokens, d, false)) return RELAY_EINVAL;
    if ((gate == nullptr) != (dgate == nullptr) || (scale == nullptr && dscale != nullptr)) return RELAY_EINVAL;
    if (!rows_fit(dx, type, n, tokens, d, true) || !rows_fit(dresidual, type, n, tokens, d, true) ||
        (dgate != nullptr && !rows_fit(dgate, type, n, tokens, d, true)))
        return RELAY_EINVAL;
    if (tokens > 0 && (rstd == nullptr || !aligned(rstd, 4))) return RELAY_EINVAL;
    if (!aligned(lengths, 4)) return RELAY_EINVAL;
    if (!gradient_fits(dpost, dpost_stride, n, d) || !gradient_fits(dpre, dpre_stride, n, d) ||
        (dscale != nullptr && !gradient_fits(dscale, dscale_stride, n, d)) || dpost == dpre || dpost == dscale || dpre == dscale)
        return RELAY_EINVAL;
    if (workspace == nullptr || !aligned(workspace, 16) ||
        workspace_bytes < relay_block_norm_backward_workspace(n, tokens, d))
        return RELAY_EINVAL;
    if (tokens > 0) {
        for (const relay_rows* out : {dx, dresidual, dgate})
            for (const relay_rows* in : {dy, dtotal, x, gate, residual})
                if (out != nullptr && in != nullptr && out->data == in->data) return RELAY_EINVAL;
        if (dx->data == dresidual->data || (dgate != nullptr && (dgate->data == dx->data || dgate->data == dresidual->data)))
            return RELAY_EINVAL;
    }
    bool vec = d % 8 == 0;
    for (const relay_rows* r : {dy, dtotal, x, gate, residual, dx, dgate, dresidual}) vec = vec && vectors(r, type, n, tokens);
    int parts = static_cast<int>(block_partials(n, tokens, d));
    const int rc = by_type(type, [&](auto t) {
        using T = decltype(t);
        const BlockBackwardArgs<T> a{
            view<const T>(dy, n, tokens), view<const T>(dtotal, n, tokens), view<const T>(x, n, tokens),
            view<const T>(gate, n, tokens), view<const T>(residual, n, tokens), view<T>(dx, n, tokens),
            view<T>(dgate, n, tokens), view<T>(dresidual, n, tokens), weight_of(post, post_stride, n, d),
            weight_of(pre, pre_stride, n, d), weight_of(scale, scale_stride, n, d), rstd, lengths,
            static_cast<float*>(workspace), static_cast<int32_t>(tokens), static_cast<int32_t>(d),
            static_cast<int32_t>(pitch_of(d))};
        if (vec && takes_ring<T, 5>(n, tokens, d)) {
            int rc = RELAY_OK;
            by_ring<T, 5>(d, [&](auto r) {
                constexpr int kParts = decltype(r)::kParts;
                parts = static_cast<int>(ring_partials<T, kParts>(n, tokens, d));
                rc = d > decltype(r)::kWide - kQuads ? launch_rows<T, kParts, true>(a, parts, n, stream)
                                                     : launch_rows<T, kParts, false>(a, parts, n, stream);
            });
            return rc;
        }
        return by_back_width(a.pitch, [&](auto hold) {
            constexpr int kParts = decltype(hold)::kParts, kStrips = decltype(hold)::kStrips;
            constexpr size_t kSmem = (kNormWarps<kParts> / kParts - 1) * kStrips * kParts * kStrip * sizeof(float);
            (vec ? relay_block_norm_backward_kernel<T, kVector, kParts, kStrips>
                 : relay_block_norm_backward_kernel<T, kDirect, kParts, kStrips>)
                <<<dim3(parts, n), 32 * kNormWarps<kParts>, kSmem, stream>>>(a);
            return status_of_launch();
        });
    });
    if (rc != RELAY_OK) return rc;
    const Sums to{{dpost, dpre, dscale}, {dpost_stride, dpre_stride, dscale_stride}};
    relay_block_norm_join_kernel<<<dim3(static_cast<unsigned>((d + 127) / 128), n, dscale == nullptr ? 2 : 3), 256, 0, stream>>>(
        static_cast<const float*>(workspace), parts, static_cast<int>(d), static_cast<int>(pitch_of(d)), to);
    return status_of_launch();
}

#endif

}  // extern "C"
