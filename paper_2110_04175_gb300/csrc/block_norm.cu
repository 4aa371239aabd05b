// block_norm.cu -- the step from one block of a model to the next (relaylayers.h), forward
// and backward, on GB300 (sm_103a): the block's output is normalised, gated and joined to
// the residual, and the sum normalised for the next block,
//
//   m = x s_x w_post;  h = rho r + sigma(z) m;  y = h s_h w_pre
//
// All rows in and all rows out once, two sums over a row between them, so memory bounds it.
// kParts warps share a row, each with kStrips strips of 256 features (layers.cuh).
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
// with xhat = x s_x and hhat = h s_h made again from the rows.

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

template <typename T, Way kWay, int kParts, int kStrips>
__global__ void __launch_bounds__(32 * kNormWarps<kParts>, kNormWarps<kParts> > 8 ? 1 : 2)
relay_block_norm_backward_kernel(BlockBackwardArgs<T> a) {
    constexpr int kRows = kNormWarps<kParts> / kParts;
    __shared__ float shared[kNormWarps<kParts>];
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
        Piece<T, kWay> x[kStrips], z[kStrips], r[kStrips], dy[kStrips];
#pragma unroll
        for (int j = 0; j < kStrips; ++j) {
            const int base = base_of(j), left = counts ? a.d - base : 0;
            x[j].load(a.x.row(worker, token) + base, lane, left);
            if (a.gate.p != nullptr) z[j].load(a.gate.row(worker, token) + base, lane, left);
            r[j].load(a.residual.row(worker, token) + base, lane, left);
            dy[j].load(a.dy.row(worker, token) + base, lane, left);
        }
        // strip j's xhat, sigma(z) and the rest to 1, m, r, and hhat
        const auto remake = [&](int j, float (&xhat)[8], float (&p)[8], float (&q)[8], float (&m)[8], float (&res)[8],
                                float (&hhat)[8], float (&w)[8], float (&rho)[8]) {
            const int base = base_of(j), left = counts ? a.d - base : 0;
            x[j].get(xhat);
            a.post.template load<kWay>(worker, base, lane, left, w, turn);
            r[j].get(res);
            if (a.scale.p != nullptr) a.scale.template load<kWay>(worker, base, lane, left, rho, turn);
            if (a.gate.p != nullptr) z[j].get(p);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (a.scale.p == nullptr) rho[k] = 1.0f;
                xhat[k] *= sx;
                m[k] = xhat[k] * w[k];
                if (a.gate.p != nullptr) {
                    const Gate<T> g(p[k]);
                    p[k] = g.at, q[k] = g.rest;
                } else {
                    p[k] = 1.0f, q[k] = 0.0f;
                }
                hhat[k] = fmaf(rho[k], res[k], p[k] * m[k]) * sh;
            }
        };
        float along = 0.0f;
#pragma unroll
        for (int j = 0; j < kStrips; ++j) {
            const int base = base_of(j), left = counts ? a.d - base : 0;
            float xhat[8], p[8], q[8], m[8], res[8], hhat[8], w[8], rho[8], u[8], pre[8];
            remake(j, xhat, p, q, m, res, hhat, w, rho);
            dy[j].get(u);
            a.pre.template load<kWay>(worker, base, lane, left, pre, turn);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                dpre[j][k] = fmaf(u[k], hhat[k], dpre[j][k]);
                along = fmaf(u[k] * pre[k], hhat[k], along);
            }
        }
        along = row_sum<kParts>(along, shared, slot, part) / static_cast<float>(a.d);
        float along_x = 0.0f, dh[kStrips][8];
#pragma unroll
        for (int j = 0; j < kStrips; ++j) {
            const int base = base_of(j), left = counts ? a.d - base : 0;
            float xhat[8], p[8], q[8], m[8], res[8], hhat[8], w[8], rho[8], pre[8], over[8] = {}, dg[8], dr[8];
            remake(j, xhat, p, q, m, res, hhat, w, rho);
            dy[j].get(dh[j]);
            a.pre.template load<kWay>(worker, base, lane, left, pre, turn);
            if (a.dtotal.p != nullptr) load_strip<kWay>(a.dtotal.row(worker, token) + base, lane, left, over);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float d = fmaf(sh, dh[j][k] * pre[k] - hhat[k] * along, over[k]);
                dr[k] = counts ? rho[k] * d : 0.0f;
                dg[k] = counts ? d * m[k] * p[k] * q[k] : 0.0f;
                dscale[j][k] = fmaf(d, res[k], dscale[j][k]);
                dpost[j][k] = fmaf(d * p[k], xhat[k], dpost[j][k]);
                dh[j][k] = d * p[k] * w[k];
                along_x = fmaf(dh[j][k], xhat[k], along_x);
            }
            if (token < a.tokens) {
                store_strip<kWay>(a.dresidual.row(worker, token) + base, lane, a.d - base, dr);
                if (a.dgate.p != nullptr) store_strip<kWay>(a.dgate.row(worker, token) + base, lane, a.d - base, dg);
            }
        }
        along_x = row_sum<kParts>(along_x, shared, slot, part) / static_cast<float>(a.d);
        if (token < a.tokens) {
#pragma unroll
            for (int j = 0; j < kStrips; ++j) {
                float xhat[8];
                x[j].get(xhat);
#pragma unroll
                for (int k = 0; k < 8; ++k) dh[j][k] = counts ? sx * (dh[j][k] - xhat[k] * sx * along_x) : 0.0f;
                store_strip<kWay>(a.dx.row(worker, token) + base_of(j), lane, a.d - base_of(j), dh[j]);
            }
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
// workers, no more than there are tokens to take; multiples where a thread would add up
// more than 256 rows in one chain.
int64_t block_partials(int32_t n, int64_t tokens, int64_t d) {
    const int64_t pitch = pitch_of(d), side = pitch <= 256 ? 8 : pitch <= 512 ? 4 : pitch <= 1024 ? 2 : 1;  // kRows
    const int64_t slots = pitch <= 2048 ? 304 : 152, fill = slots > n ? slots / n : 1, chain = fill * side * 256;
    const int64_t want = tokens > chain ? fill * ((tokens + chain - 1) / chain) : fill, most = (tokens + side - 1) / side;
    return most < want ? (most > 0 ? most : 1) : want;
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
    const int parts = static_cast<int>(block_partials(n, tokens, d));
    const int rc = by_type(type, [&](auto t) {
        using T = decltype(t);
        const BlockBackwardArgs<T> a{
            view<const T>(dy, n, tokens), view<const T>(dtotal, n, tokens), view<const T>(x, n, tokens),
            view<const T>(gate, n, tokens), view<const T>(residual, n, tokens), view<T>(dx, n, tokens),
            view<T>(dgate, n, tokens), view<T>(dresidual, n, tokens), weight_of(post, post_stride, n, d),
            weight_of(pre, pre_stride, n, d), weight_of(scale, scale_stride, n, d), rstd, lengths,
            static_cast<float*>(workspace), static_cast<int32_t>(tokens), static_cast<int32_t>(d),
            static_cast<int32_t>(pitch_of(d))};
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
