// weight_grad.cu -- the weight gradient of a linear layer whose inputs were kept
// in 8 bits (relay_weight_grad of relaylayers.h) on GB300 (sm_103a):
//
//   dW_i[o][k] = scale_i[k] sum_t dy_i[t][o] xhat_i[t][k]
#include "layers.cuh"

namespace {

constexpr int kTile = 64, kDepth = 16;  // outputs and inputs of a CTA's tile; tokens per step

template <typename T>
struct WeightGradArgs {
    View<const T> dy;
    const int8_t* codes;
    const uint8_t* scales;
    const float* column_scale;
    int64_t column_scale_stride;
    const int32_t* lengths;
    float* dweight;
    int64_t worker_stride, row_stride;
    int32_t tokens, outputs, inputs, pitch;
};

// One CTA per 64 x 64 tile, 4 x 4 results a thread.
template <typename T>
__global__ void __launch_bounds__(256) relay_weight_grad_kernel(WeightGradArgs<T> a) {
    __shared__ float left[kDepth][kTile], right[kDepth][kTile];
    const int worker = blockIdx.z, o0 = blockIdx.y * kTile, k0 = blockIdx.x * kTile;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const int length = a.lengths == nullptr ? a.tokens : min(max(a.lengths[worker], 0), a.tokens);
    float acc[4][4] = {};
    for (int t0 = 0; t0 < length; t0 += kDepth) {
        for (int e = threadIdx.x; e < kDepth * kTile; e += 256) {
            const int t = t0 + e / kTile, c = e % kTile;
            float l = 0.0f, r = 0.0f;
            if (t < length) {
                if (o0 + c < a.outputs) l = widen(a.dy.row(worker, t)[o0 + c]);
                if (k0 + c < a.inputs) {
                    const int64_t row = static_cast<int64_t>(worker) * a.tokens + t;
                    r = static_cast<float>(a.codes[row * a.pitch + k0 + c]) *
                        scale_unit(a.scales[row * (a.pitch / kBlock) + (k0 + c) / kBlock]);
                }
            }
            left[e / kTile][c] = l;
            right[e / kTile][c] = r;
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < kDepth; ++t) {
            float l[4], r[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) l[i] = left[t][ty + 16 * i], r[i] = right[t][tx + 16 * i];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(l[i], r[j], acc[i][j]);
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int o = o0 + ty + 16 * i, k = k0 + tx + 16 * j;
            if (o >= a.outputs || k >= a.inputs) continue;
            const float s =
                a.column_scale == nullptr ? 1.0f : a.column_scale[worker * a.column_scale_stride + k];
            a.dweight[worker * a.worker_stride + o * a.row_stride + k] = acc[i][j] * s;
        }
}

}  // namespace

extern "C" {

int64_t relay_weight_grad_workspace(int32_t n, int64_t tokens, int64_t outputs, int64_t inputs) {
    if (const int rc = check_shape(RELAY_FP32, n, tokens, inputs)) return rc;
    if (const int rc = check_shape(RELAY_FP32, n, tokens, outputs)) return rc;
    return 0;
}

int relay_weight_grad(int32_t type, int32_t n, int64_t tokens, int64_t outputs, int64_t inputs, const relay_rows* dy,
                      const int8_t* codes, const uint8_t* scales, const float* column_scale,
                      int64_t column_scale_stride, const int32_t* lengths, float* dweight, int64_t worker_stride,
                      int64_t row_stride, void* workspace, int64_t workspace_bytes, relay_stream_t stream) {
    if (const int rc = check_shape(type, n, tokens, inputs)) return rc;
    if (const int rc = check_shape(type, n, tokens, outputs)) return rc;
    if (!rows_fit(dy, type, n, tokens, outputs, false) || !checkpoint_fits(codes, scales, tokens)) return RELAY_EINVAL;
    if (!aligned(column_scale, 4) || (column_scale != nullptr && column_scale_stride < 0) || !aligned(lengths, 4))
        return RELAY_EINVAL;
    const relay_rows out{dweight, worker_stride, row_stride};
    if (!rows_fit(&out, RELAY_FP32, n, outputs, inputs, true)) return RELAY_EINVAL;
    const int64_t need = relay_weight_grad_workspace(n, tokens, outputs, inputs);
    if (workspace_bytes < need || (need > 0 && (workspace == nullptr || !aligned(workspace, 16)))) return RELAY_EINVAL;
    const dim3 grid(static_cast<unsigned>((inputs + kTile - 1) / kTile),
                    static_cast<unsigned>((outputs + kTile - 1) / kTile), n);
    if (grid.y > 65535) return RELAY_EUNSUPPORTED;
    auto launch = [&](auto t) {
        using T = decltype(t);
        const WeightGradArgs<T> a{view<const T>(dy, n, tokens), codes, scales, column_scale,
                                  n > 1 ? column_scale_stride : 0, lengths, dweight, n > 1 ? worker_stride : 0,
                                  outputs > 1 ? row_stride : 0, static_cast<int32_t>(tokens),
                                  static_cast<int32_t>(outputs), static_cast<int32_t>(inputs),
                                  static_cast<int32_t>(pitch_of(inputs))};
        relay_weight_grad_kernel<T><<<grid, 256, 0, stream>>>(a);
        return status_of_launch();
    };
    return type == RELAY_BF16 ? launch(__nv_bfloat16()) : type == RELAY_FP16 ? launch(__half()) : launch(float());
}

}  // extern "C"
