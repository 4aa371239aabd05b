// block_norm.cu -- the step from one block of a model to the next (relaylayers.h), forward
// and backward, on GB300 (sm_103a): the block's output is normalised, gated and joined to
// the residual, and the sum normalised for the next block,
//
//   m = x s_x w_post;  h = rho r + sigma(z) m;  y = h s_h w_pre
//
// All rows in and all rows out once, two sums over a row between them, so memory bounds it.
// kParts warps share a row, each with kStrips strips of 256 features (layers.cuh).
#include <type_traits>

#include "blackwell.cuh"
#include "layers.cuh"

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

// The lane's octet of a weight of any alignment.
__device__ __forceinline__ void load_octet(const Weight& w, int worker, int base, int lane, int left, float (&v)[8]) {
    const float* p = w.p + worker * w.stride + base;
    if (w.quads) {
        load_strip<kVector>(p, lane, left, v);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = 8 * lane + k < left ? p[8 * lane + k] : 0.0f;
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

// What a lane makes again of 8 features of a row: `x`, `z`, `r` come as x, gate and residual
// and leave as xhat, p and r; `w` and `rho` are w_post and rho (1 without).
template <typename T>
struct Octet {
    float xhat[8], p[8], q[8], m[8], r[8], hhat[8];
    __device__ __forceinline__ void make(const float (&w)[8], const float (&rho)[8], bool gated, float sx, float sh) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            xhat[k] *= sx;
            m[k] = xhat[k] * w[k];
            if (gated) {
                const Gate<T> g(p[k]);
                p[k] = g.at, q[k] = g.rest;
            } else {
                p[k] = 1.0f, q[k] = 0.0f;
            }
            hhat[k] = fmaf(rho[k], r[k], p[k] * m[k]) * sh;
        }
    }
    // Adds to the three sums and to dw_pre.
    __device__ __forceinline__ void add(const float (&dy)[8], const float (&pre)[8], const float (&over)[8], float sh,
                                        float (&sums)[3], float (&dpre)[8]) const {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float u = dy[k] * pre[k], a = p[k] * m[k];
            dpre[k] = fmaf(dy[k], hhat[k], dpre[k]);
            sums[0] = fmaf(u, hhat[k], sums[0]);
            sums[1] = fmaf(a, fmaf(sh, u, over[k]), sums[1]);
            sums[2] = fmaf(a, hhat[k], sums[2]);
        }
    }
    // The three gradients of the rows (dy becomes dx), and what w_post and rho get of them.
    __device__ __forceinline__ void leave(float (&dy)[8], const float (&pre)[8], const float (&over)[8], const float (&w)[8],
                                          const float (&rho)[8], float sx, float sh, float along, float along_x, float (&dz)[8],
                                          float (&dr)[8], float (&dpost)[8], float (&dscale)[8]) const {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float d = fmaf(sh, fmaf(dy[k], pre[k], -hhat[k] * along), over[k]), dp = d * p[k];
            dr[k] = rho[k] * d;
            dz[k] = dp * m[k] * q[k];
            dscale[k] = fmaf(d, r[k], dscale[k]);
            dpost[k] = fmaf(dp, xhat[k], dpost[k]);
            dy[k] = sx * fmaf(dp, w[k], -xhat[k] * along_x);
        }
    }
};

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

    float dpost[kStrips][8] = {}, dpre[kStrips][8] = {}, dscale[kStrips][8] = {};
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
        const auto remake = [&](int j, Octet<T>& o, float (&w)[8], float (&rho)[8], float (&pre)[8], float (&u)[8], float (&over)[8]) {
            const int base = base_of(j), left = counts ? a.d - base : 0;
            x[j].get(o.xhat);
            r[j].get(o.r);
            dy[j].get(u);
            dtotal[j].get(over);
            if (a.gate.p != nullptr) z[j].get(o.p);
            a.post.template load<kWay>(worker, base, lane, left, w, turn);
            a.pre.template load<kWay>(worker, base, lane, left, pre, turn);
            if (a.scale.p != nullptr) {
                a.scale.template load<kWay>(worker, base, lane, left, rho, turn);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) rho[k] = 1.0f;
            }
            o.make(w, rho, a.gate.p != nullptr, sx, sh);
        };
        float three[3] = {};
#pragma unroll
        for (int j = 0; j < kStrips; ++j) {
            Octet<T> o;
            float w[8], rho[8], pre[8], u[8], over[8];
            remake(j, o, w, rho, pre, u, over);
            o.add(u, pre, over, sh, three, dpre[j]);
        }
#pragma unroll
        for (int e = 0; e < 3; ++e) three[e] = row_sum<kParts>(three[e], shared[e], slot, part) / static_cast<float>(a.d);
        if (token >= a.tokens) continue;
        const float along = three[0], along_x = three[1] - sh * along * three[2];
#pragma unroll
        for (int j = 0; j < kStrips; ++j) {
            const int base = base_of(j), left = a.d - base;
            if (left <= 0) break;
            Octet<T> o;
            float w[8], rho[8], pre[8], u[8], over[8], dz[8], dr[8];
            if (counts) {
                remake(j, o, w, rho, pre, u, over);
                o.leave(u, pre, over, w, rho, sx, sh, along, along_x, dz, dr, dpost[j], dscale[j]);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) u[k] = dz[k] = dr[k] = 0.0f;
            }
            store_strip<kWay>(a.dx.row(worker, token) + base, lane, left, u);
            store_strip<kWay>(a.dresidual.row(worker, token) + base, lane, left, dr);
            if (a.dgate.p != nullptr) store_strip<kWay>(a.dgate.row(worker, token) + base, lane, left, dz);
        }
    }
    const auto leave = [&](float (&v)[kStrips][8], int which) {
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

// Aligned rows of up to 8192 features in 16 bits and 4096 in 32: rows come by bulk copies to
// shared memory, two a group of kParts warps, so that the next one is on its way while this
// one's two sweeps read it there, and registers are left for two strips' sums over the
// tokens.  The groups of a CTA take rows of their own and wait only for themselves.
template <typename T, int kParts>
struct Ring {
    static constexpr int kWarps = sizeof(T) == 2 ? 16 : 8, kGroups = kWarps / kParts, kStages = 2;
    static constexpr int kRow = kParts * 2 * kStrip * static_cast<int>(sizeof(T));  // bytes kept free for a row
    static constexpr int kStage = 5 * kRow;
    static constexpr bool kWeights = kParts <= 8;  // there is room for the three weights too
    static constexpr int kWide = kParts * 2 * kStrip;
    static constexpr int kRows = kGroups * kStages * kStage, kShared = kRows + (kWeights ? 3 * 4 * kWide : 0) + 16;
    static_assert(kShared <= 232448 - 2048, "shared memory of a CTA");
};

// A wait that runs out makes a group's results from there on NaN.
template <typename T, int kParts>
__global__ void __launch_bounds__(32 * Ring<T, kParts>::kWarps, 1) relay_block_norm_backward_rows_kernel(BlockBackwardArgs<T> a) {
    using R = Ring<T, kParts>;
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
    if (R::kWeights) {
        const Weight* from[3] = {&a.post, &a.pre, &a.scale};
#pragma unroll
        for (int e = 0; e < 3; ++e)
            for (int k = threadIdx.x; k < R::kWide; k += 32 * R::kWarps)
                weights[e * R::kWide + k] = k >= a.d ? 0.0f : from[e]->p == nullptr ? 1.0f : from[e]->p[worker * from[e]->stride + k];
    }
    __syncthreads();

    const int step = static_cast<int>(gridDim.x) * R::kGroups, begin = static_cast<int>(blockIdx.x) * R::kGroups + group;
    const uint32_t bytes = static_cast<uint32_t>(a.d) * sizeof(T);
    const bool brings = part == 0 && elected();
    uint8_t* mine = ring + group * (R::kStages * R::kStage);
    const auto bring = [&](int token, int s) {  // one thread of the group
        const uint32_t bar = shared_address(&bars[group][s]), to = shared_address(mine + s * R::kStage);
        barrier_expect(bar, bytes * (3 + gated + over_too));
        copy_row(to, a.x.row(worker, token), bytes, bar);
        copy_row(to + R::kRow, a.residual.row(worker, token), bytes, bar);
        copy_row(to + 2 * R::kRow, a.dy.row(worker, token), bytes, bar);
        if (gated) copy_row(to + 3 * R::kRow, a.gate.row(worker, token), bytes, bar);
        if (over_too) copy_row(to + 4 * R::kRow, a.dtotal.row(worker, token), bytes, bar);
    };
    if (brings) {
        if (begin < length) bring(begin, 0);
        if (begin + step < length) bring(begin + step, 1);
    }
    float dpost[2][8] = {}, dpre[2][8] = {}, dscale[2][8] = {};
    bool ok = true;
    int i = 0;
    for (int token = begin; token < length; token += step, ++i) {
        const int s = i % 2;
        const int64_t row = static_cast<int64_t>(worker) * a.tokens + token;
        float sx = a.rstd[row];
        const float sh = a.rstd[static_cast<int64_t>(n) * a.tokens + row];
        ok = ok && barrier_wait_warp(shared_address(&bars[group][s]), i / 2 & 1);
        if (!ok) sx = __int_as_float(0x7fffffff);
        const auto remake = [&](int j, Octet<T>& o, float (&w)[8], float (&rho)[8], float (&pre)[8], float (&u)[8], float (&over)[8]) {
            const int at = (part + kParts * j) * kStrip, left = a.d - at;
            const T* from = reinterpret_cast<const T*>(mine + s * R::kStage) + at;
            constexpr int kNext = R::kRow / static_cast<int>(sizeof(T));
            load_strip<kVector>(from, lane, left, o.xhat);
            load_strip<kVector>(from + kNext, lane, left, o.r);
            load_strip<kVector>(from + 2 * kNext, lane, left, u);
            if (gated) load_strip<kVector>(from + 3 * kNext, lane, left, o.p);
            load_strip<kVector>(from + 4 * kNext, lane, over_too ? left : 0, over);
            if constexpr (R::kWeights) {
                load_strip<kVector>(weights + at, lane, left, w);
                load_strip<kVector>(weights + R::kWide + at, lane, left, pre);
                load_strip<kVector>(weights + 2 * R::kWide + at, lane, left, rho);
            } else {
                load_octet(a.post, worker, at, lane, left, w);
                load_octet(a.pre, worker, at, lane, left, pre);
                if (scaled) load_octet(a.scale, worker, at, lane, left, rho);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (!scaled) rho[k] = 1.0f;
            }
            o.make(w, rho, gated, sx, sh);
        };
        float three[3] = {};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            Octet<T> o;
            float w[8], rho[8], pre[8], u[8], over[8];
            remake(j, o, w, rho, pre, u, over);
            o.add(u, pre, over, sh, three, dpre[j]);
        }
#pragma unroll
        for (int e = 0; e < 3; ++e)
#pragma unroll
            for (int m = 16; m > 0; m >>= 1) three[e] += __shfl_xor_sync(0xffffffffu, three[e], m);
        if constexpr (kParts > 1) {
            float(&sums)[kParts][3] = shared[i & 1][group];
            if (lane < 3) sums[part][lane] = lane == 0 ? three[0] : lane == 1 ? three[1] : three[2];
            asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(32 * kParts) : "memory");
#pragma unroll
            for (int e = 0; e < 3; ++e) {
                three[e] = 0.0f;
#pragma unroll
                for (int w = 0; w < kParts; ++w) three[e] += sums[w][e];
            }
        } else {
            __syncwarp();
        }
        // here every warp of the group is done with the row before this one
        if (brings && i > 0 && token + step < length) bring(token + step, s ^ 1);
        const float over_d = 1.0f / static_cast<float>(a.d), along = three[0] * over_d;
        const float along_x = three[1] * over_d - sh * along * (three[2] * over_d);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int at = (part + kParts * j) * kStrip, left = a.d - at;
            Octet<T> o;
            float w[8], rho[8], pre[8], u[8], over[8], dz[8], dr[8];
            remake(j, o, w, rho, pre, u, over);
            o.leave(u, pre, over, w, rho, sx, sh, along, along_x, dz, dr, dpost[j], dscale[j]);
            store_strip<kVector>(a.dx.row(worker, token) + at, lane, left, u);
            store_strip<kVector>(a.dresidual.row(worker, token) + at, lane, left, dr);
            if (gated) store_strip<kVector>(a.dgate.row(worker, token) + at, lane, left, dz);
        }
    }
    // padding
    for (int token = begin + i * step; token < a.tokens; token += step) {
        const float none[8] = {};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int at = (part + kParts * j) * kStrip, left = a.d - at;
            store_strip<kVector>(a.dx.row(worker, token) + at, lane, left, none);
            store_strip<kVector>(a.dresidual.row(worker, token) + at, lane, left, none);
            if (gated) store_strip<kVector>(a.dgate.row(worker, token) + at, lane, left, none);
        }
    }
    // the groups' sums in their order, through the ring's memory: [kGroups - 1][kWide]
    float* others = reinterpret_cast<float*>(ring);
    const auto leave = [&](float (&v)[2][8], int which) {
        if (R::kGroups > 1) {
            __syncthreads();
            if (group > 0) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    store_strip<kVector>(others + (group - 1) * R::kWide + (part + kParts * j) * kStrip, lane, kStrip, v[j]);
            }
            __syncthreads();
            if (group > 0) return;
            for (int g = 0; g < R::kGroups - 1; ++g)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float add[8];
                    load_strip<kVector>(others + g * R::kWide + (part + kParts * j) * kStrip, lane, kStrip, add);
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[j][k] += add[k];
                }
        }
        float* out = a.partial + ((static_cast<int64_t>(which) * n + worker) * gridDim.x + blockIdx.x) * a.pitch;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int at = (part + kParts * j) * kStrip;
            store_strip<kVector>(out + at, lane, a.pitch - at, v[j]);
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

// out[i][k] = sum_p partial[i][p][k]: a CTA sums 32 columns, 8 rows at a time.
__global__ void __launch_bounds__(256) relay_block_norm_join_kernel(const float* partial, int parts, int d, int pitch, Sums to) {
    __shared__ float shared[8][32];
    const int column = blockIdx.x * 32 + threadIdx.x % 32, lead = threadIdx.x / 32, which = blockIdx.z;
    if (to.p[which] == nullptr) return;
    const float* p = partial + (static_cast<int64_t>(which) * gridDim.y + blockIdx.y) * parts * pitch;
    float s = 0.0f;
    if (column < d)
        for (int r = lead; r < parts; r += 8) s += p[static_cast<int64_t>(r) * pitch + column];
    shared[lead][threadIdx.x % 32] = s;
    __syncthreads();
    if (lead > 0 || column >= d) return;
#pragma unroll
    for (int r = 1; r < 8; ++r) s += shared[r][threadIdx.x];
    to.p[which][blockIdx.y * to.stride[which] + column] = s;
}

// ---------------------------------------------------------------- launching

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
    const int64_t side = Ring<T, kParts>::kGroups, fill = 152 > n ? 152 / n : 1, chain = fill * side * 256;
    const int64_t want = tokens > chain ? fill * ((tokens + chain - 1) / chain) : fill, most = (tokens + side - 1) / side;
    const int64_t parts = most < want ? (most > 0 ? most : 1) : want, room = block_partials(n, tokens, d);
    return parts < room ? parts : room;
}

template <typename T, int kParts>
int launch_rows(const BlockBackwardArgs<T>& a, int64_t parts, int32_t n, cudaStream_t stream) {
    constexpr auto kernel = relay_block_norm_backward_rows_kernel<T, kParts>;
    if (!allow_shared<kernel>(Ring<T, kParts>::kShared)) return RELAY_ECUDA;
    kernel<<<dim3(static_cast<unsigned>(parts), n), 32 * Ring<T, kParts>::kWarps, Ring<T, kParts>::kShared, stream>>>(a);
    return status_of_launch();
}

// f(kParts) for the least that holds a row in two strips a warp.
template <typename F>
int by_ring(int64_t pitch, F f) {
    if (pitch <= 512) return f(std::integral_constant<int, 1>());
    if (pitch <= 1024) return f(std::integral_constant<int, 2>());
    if (pitch <= 2048) return f(std::integral_constant<int, 4>());
    if (pitch <= 4096) return f(std::integral_constant<int, 8>());
    return f(std::integral_constant<int, 16>());
}

bool weight_fits(const float* p, int64_t stride) { return p != nullptr && aligned(p, 4) && stride >= 0; }

bool gradient_fits(const float* p, int64_t stride, int32_t n, int64_t d) {
    return p != nullptr && aligned(p, 4) && (n == 1 || stride >= d);
}

Weight weight_of(const float* p, int64_t stride, int32_t n, int64_t d) {
    return Weight{p, n > 1 ? stride : 0, d % 8 == 0 && aligned(p, 16) && (n == 1 || stride % 4 == 0)};
}

}  // namespace

extern "C" {

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
    for (const relay_rows* out : {dx, dresidual, dgate})
        if ((out != nullptr || gate != nullptr || out != dgate) && !rows_fit(out, type, n, tokens, d, true)) return RELAY_EINVAL;
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
    const bool ring = vec && tokens > 0 && d <= (type == RELAY_FP32 ? 4096 : 8192);
    const int rc = by_type(type, [&](auto t) {
        using T = decltype(t);
        const BlockBackwardArgs<T> a{
            view<const T>(dy, n, tokens), view<const T>(dtotal, n, tokens), view<const T>(x, n, tokens),
            view<const T>(gate, n, tokens), view<const T>(residual, n, tokens), view<T>(dx, n, tokens),
            view<T>(dgate, n, tokens), view<T>(dresidual, n, tokens), weight_of(post, post_stride, n, d),
            weight_of(pre, pre_stride, n, d), weight_of(scale, scale_stride, n, d), rstd, lengths,
            static_cast<float*>(workspace), static_cast<int32_t>(tokens), static_cast<int32_t>(d),
            static_cast<int32_t>(pitch_of(d))};
        if (ring)
            return by_ring(a.pitch, [&](auto with) {
                constexpr int kParts = decltype(with)::value;
                if constexpr (kParts <= Ring<T, 1>::kWarps) {
                    parts = static_cast<int>(ring_partials<T, kParts>(n, tokens, d));
                    return launch_rows<T, kParts>(a, parts, n, stream);
                }
                return RELAY_EUNSUPPORTED;  // (not reached: `ring`)
            });
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
    relay_block_norm_join_kernel<<<dim3(static_cast<unsigned>((d + 31) / 32), n, dscale == nullptr ? 2 : 3), 256, 0, stream>>>(
        static_cast<const float*>(workspace), parts, static_cast<int>(d), static_cast<int>(pitch_of(d)), to);
    return status_of_launch();
}

}  // extern "C"
