// layer_kernels.cu -- the row-wise layer operators of relaylayers.h on GB300
// (sm_103a): the 8-bit checkpoint, the root-mean-square norm with the
// residual's addition, and the gated activation, forward and backward.
//
// All of them move rows and compute little, so memory bounds them.  A warp
// works on strips of 256 features (layers.cuh); what a row needs twice stays in
// registers between its two uses.  Measured in bf16, bytes moved against the
// 6.67 TB/s of a plain copy:
//   norm, residual, 8-bit output        [4][4096][4096]   93 us  6.5 TB/s
//   norm backward from 8 bits           [4][4096][4096]   84 us  5.6 TB/s
//   to 8 bits and back                  [4][4096][8192]  127 us  6.4 TB/s
//   gated, both inputs put away         [4][4096][8192]  163 us  6.6 TB/s
//   gated backward from 8 bits          [4][4096][8192]  190 us  6.4 TB/s
#include "layers.cuh"

namespace {

template <typename F>
int by_type(int32_t type, F f) {
    return type == RELAY_BF16 ? f(__nv_bfloat16()) : type == RELAY_FP16 ? f(__half()) : f(float());
}

// The warp's `turn` (layers.cuh) in a kernel of `warps` warps, if it is `used`.
#define WARP_TURN(warps, used)                                                  \
    __shared__ __align__(16) float turns[(used) ? (warps) : 1][(used) ? kStrip : 1]; \
    float* turn = turns[(used) ? threadIdx.x / 32 : 0]

// ------------------------------------------------------- element-wise kernels

constexpr int kWarps = 8;  // of an element-wise CTA

// A warp takes this many strips of a row at a time, all of them asked for first.
constexpr int kRun = 2;

struct Grid {
    int64_t rows;    // n tokens
    int32_t tokens;
    int32_t runs;    // of a row
    int32_t d, pitch;
    // what the whole grid's warps step over together, in workers, tokens and runs
    int32_t step_worker, step_token, step_run;
};

// Calls f(row, worker, token, first feature) for this warp's runs of strips: every
// (gridDim.x kWarps)-th one, found without a division past the first.
template <typename F>
__device__ __forceinline__ void each_run(const Grid& g, F f) {
    const int64_t first = static_cast<int64_t>(blockIdx.x) * kWarps + threadIdx.x / 32;
    int64_t row = first / g.runs;
    int run = static_cast<int>(first - row * g.runs), worker = static_cast<int>(row / g.tokens);
    int token = static_cast<int>(row - static_cast<int64_t>(worker) * g.tokens);
    while (row < g.rows) {
        f(row, worker, token, run * (kRun * kStrip));
        run += g.step_run;
        token += g.step_token;
        worker += g.step_worker;
        if (run >= g.runs) run -= g.runs, ++token;
        if (token >= g.tokens) token -= g.tokens, ++worker;
        row = static_cast<int64_t>(worker) * g.tokens + token;
    }
}

// To 8 bits: a block's 32 features are four lanes' octets, its largest magnitude two
// shuffles.  In 16 bits that is found two features at a time.  Bound by HBM.
template <typename T, Way kWay>
__global__ void __launch_bounds__(32 * kWarps)
relay_checkpoint_pack_kernel(Grid g, View<const T> x, int8_t* codes, uint8_t* scales) {
    WARP_TURN(kWarps, kWay == kDirect);
    const int lane = threadIdx.x % 32;
    each_run(g, [&](int64_t row, int worker, int token, int base) {
        Piece<T, kWay> p[kRun];
        const T* from = x.row(worker, token) + base;
#pragma unroll
        for (int j = 0; j < kRun; ++j) p[j].load(from + j * kStrip, lane, g.d - base - j * kStrip);
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            float v[8];
            p[j].get(v);
            put_strip<kWay>(codes + row * g.pitch, scales + row * (g.pitch / kBlock), base + j * kStrip, lane, g.pitch, v,
                            largest(p[j], v), turn);
        }
    });
}

// fp16 cannot hold all that 8 bits can: held at the largest finite magnitude.
template <typename T>
__device__ __forceinline__ float within(float v) { return v; }
template <>
__device__ __forceinline__ float within<__half>(float v) { return fabsf(v) > 65504.0f ? copysignf(65504.0f, v) : v; }

template <typename T, Way kWay>
__global__ void __launch_bounds__(32 * kWarps)
relay_checkpoint_unpack_kernel(Grid g, const int8_t* codes, const uint8_t* scales, View<T> out) {
    WARP_TURN(kWarps, kWay == kDirect);
    const int lane = threadIdx.x % 32;
    each_run(g, [&](int64_t row, int worker, int token, int base) {
        CodePiece p[kRun];
#pragma unroll
        for (int j = 0; j < kRun; ++j)
            p[j].load(codes + row * g.pitch, scales + row * (g.pitch / kBlock), base + j * kStrip, lane, g.pitch);
        T* to = out.row(worker, token) + base;
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            float v[8];
            p[j].template get<kWay>(v, lane, turn);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = within<T>(v[k]);
            store_strip<kWay>(to + j * kStrip, lane, g.d - base - j * kStrip, v);
        }
    });
}

// sigma(g) and 1 - sigma(g).  Rows of 16 bits take the hardware's exponential and reciprocal:
// with e = exp(-g), sigma(g) = 1 / (1 + e) is off by less than (3 + 2 |g|) 2^-23 relative, far
// below the rows' rounding.  It is made from e / 4: the reciprocal, 4 sigma(g), is then a normal
// number down to sigma(g) = 2^-128 (g = -88.7), about where exp(-g) ends in fp32; below, sigma(g)
// is 0.  (Holding e at 2^126 instead left g sigma(g) growing with |g|: -4 at bf16's lowest value.)
// The difference from 1 is off by 2^-23 and exactly 0 where sigma(g) is 1 (g > 17: the reciprocal
// of a power of two is exact), so g times it is off by 2e-6 at most.  fp32 rows take the exact
// ones, of exp(-|g|), in the order that the sign of g gives, both without cancellation.
template <typename T>
struct Sigmoid {
    float at, rest;
    __device__ __forceinline__ explicit Sigmoid(float g) {
        if constexpr (sizeof(T) == 2) {
            float e, r;
            asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fmaf(g, -1.44269504f, -2.0f)));
            asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(0.25f + e));
            at = 0.25f * r;
            rest = 1.0f - at;
        } else {
            const float e = expf(-fabsf(g)), r = 1.0f / (1.0f + e);
            at = g < 0.0f ? e * r : r;
            rest = g < 0.0f ? r : e * r;
        }
    }
};

// a = g sigma(g) u, and both inputs to 8 bits from the registers that they came to.  HBM
// and issue are close: with libm's exponential, divisions and one strip at a time it took
// 53 us for [1][4096][8192] with both checkpoints where it takes 44 us.
template <typename T, Way kWay>
__global__ void __launch_bounds__(32 * kWarps)
relay_gated_kernel(Grid g, View<const T> gate, View<const T> up, View<T> out, int8_t* gate_codes,
                   uint8_t* gate_scales, int8_t* up_codes, uint8_t* up_scales) {
    WARP_TURN(kWarps, kWay == kDirect);
    const int lane = threadIdx.x % 32;
    each_run(g, [&](int64_t row, int worker, int token, int base) {
        Piece<T, kWay> p[kRun], q[kRun];
        const T *from = gate.row(worker, token) + base, *from_up = up.row(worker, token) + base;
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            p[j].load(from + j * kStrip, lane, g.d - base - j * kStrip);
            q[j].load(from_up + j * kStrip, lane, g.d - base - j * kStrip);
        }
        const int64_t at = row * g.pitch, scale_at = row * (g.pitch / kBlock);
        T* to = out.row(worker, token) + base;
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            float a[8], b[8];
            p[j].get(a);
            q[j].get(b);
            if (gate_codes != nullptr)
                put_strip<kWay>(gate_codes + at, gate_scales + scale_at, base + j * kStrip, lane, g.pitch, a, largest(p[j], a), turn);
            if (up_codes != nullptr)
                put_strip<kWay>(up_codes + at, up_scales + scale_at, base + j * kStrip, lane, g.pitch, b, largest(q[j], b), turn);
#pragma unroll
            for (int k = 0; k < 8; ++k) a[k] = a[k] * Sigmoid<T>(a[k]).at * b[k];
            store_strip<kWay>(to + j * kStrip, lane, g.d - base - j * kStrip, a);
        }
    });
}

struct GatedSource {  // one of the two
    const int8_t *gate_codes, *up_codes;
    const uint8_t *gate_scales, *up_scales;
};

// du = da g sigma(g) and dg = da u (sigma(g) + g sigma(g) (1 - sigma(g))), and a again.  54 us for
// [1][4096][8192] from 8 bits and back to them (85 us one strip at a time).  Aligned 16-bit
// rows from 8 bits keep within the 64 registers that leave room for four CTAs per SM (with
// three, [4][4096][8192] takes 227 us, with four 190); the others get what they take anyway.
template <typename T, Way kWay, bool kEight>
constexpr int kGatedBackwardCtas = kWay == kVector && sizeof(T) == 2 ? (kEight ? 4 : 3) : sizeof(T) == 4 && kEight ? 3 : 2;

template <typename T, Way kWay, bool kEight>
__global__ void __launch_bounds__(32 * kWarps, (kGatedBackwardCtas<T, kWay, kEight>))
relay_gated_backward_kernel(Grid g, View<const T> dout, View<const T> gate, View<const T> up, GatedSource from,
                            View<T> dgate, View<T> dup, int8_t* out_codes, uint8_t* out_scales) {
    WARP_TURN(kWarps, kWay == kDirect);
    const int lane = threadIdx.x % 32;
    each_run(g, [&](int64_t row, int worker, int token, int base) {
        const int64_t at = row * g.pitch, scale_at = row * (g.pitch / kBlock);
        Piece<T, kWay> p[kRun], gp[kEight ? 1 : kRun], up_p[kEight ? 1 : kRun];
        CodePiece gq[kEight ? kRun : 1], uq[kEight ? kRun : 1];
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            const int first = base + j * kStrip;
            p[j].load(dout.row(worker, token) + first, lane, g.d - first);
            if constexpr (kEight) {
                gq[j].load(from.gate_codes + at, from.gate_scales + scale_at, first, lane, g.pitch);
                uq[j].load(from.up_codes + at, from.up_scales + scale_at, first, lane, g.pitch);
            } else {
                gp[j].load(gate.row(worker, token) + first, lane, g.d - first);
                up_p[j].load(up.row(worker, token) + first, lane, g.d - first);
            }
        }
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            const int first = base + j * kStrip, left = g.d - first;
            float da[8], a[8], b[8], dg[8];
            p[j].get(da);
            if constexpr (kEight) {
                gq[j].template get<kWay>(a, lane, turn);
                uq[j].template get<kWay>(b, lane, turn);
            } else {
                gp[j].get(a);
                up_p[j].get(b);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const Sigmoid<T> s(a[k]);
                const float silu = a[k] * s.at;
                a[k] = silu * b[k];
                dg[k] = fmaf(silu, s.rest, s.at) * b[k] * da[k];
                da[k] *= silu;
            }
            store_strip<kWay>(dgate.row(worker, token) + first, lane, left, dg);
            store_strip<kWay>(dup.row(worker, token) + first, lane, left, da);
            if (out_codes != nullptr) {
                // a block that reads as NaN does so past d too: those stay 0
                clear_past<kWay>(a, lane, left);
                put_strip<kWay>(out_codes + at, out_scales + scale_at, first, lane, g.pitch, a, kWay == kVector ? largest(a) : 0u, turn);
            }
        }
    });
}

// ----------------------------------------------------------------- the norm

template <typename T>
struct NormArgs {
    View<const T> x, residual;
    View<T> total, y;
    const float* weight;
    int64_t weight_stride;
    bool weight_quads;
    float eps;
    float* rstd;
    int8_t* codes;
    uint8_t* scales;
    int32_t tokens, d, pitch;
};

// The sum of v over the kParts warps of a row (each warp's lanes included), the
// same on all of them.  `slot`: the row's place in the CTA.  Called by all threads.
template <int kParts>
__device__ __forceinline__ float row_sum(float v, float* shared, int slot, int part) {
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
    if (kParts == 1) return v;
    __syncthreads();  // the last sum's readers are done
    if (threadIdx.x % 32 == 0) shared[slot * kParts + part] = v;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int p = 0; p < kParts; ++p) s += shared[slot * kParts + p];
    return s;
}

template <int kParts>
constexpr int kNormWarps = kParts > 8 ? kParts : 8;  // of a CTA

// Rows of which the norm's CTAs may stay and take one after the other, the next asked for
// before this one's sum and the weight in registers (kAhead): aligned 16-bit rows of up to
// 8192 features.  That pays where little moves per row or rows are wide, so it is done
// without a residual and past 4096 features.  Measured in us, one CTA a row and staying:
//   n T d = 2^26   [4][16384][1024]   [4][8192][2048]   [4][4096][4096]   [4][2048][8192]
//     y alone             63   50           64   50           61   49           74   59
//     and 8 bits          75   67           75   67           73   60           87   69
//     residual            84   86           84   85           83   87           97   89
//     and 8 bits          94   97           94   99           93  101          108   99
// At 2^23 features the two are within 12 % either way (with 8 bits staying is the slower one,
// without them the faster), at 2^20 staying is 4 to 13 % faster, but 15 to 20 % slower for rows of
// 256 features (2.7 and 2.3 us).  Rows of fp32 keep HBM as busy one CTA each.
template <typename T, Way kWay, int kStrips>
constexpr bool kMayStay = kWay == kVector && kStrips <= 2 && sizeof(T) == 2;

// CTAs per SM that the norm's registers have to leave room for.
template <int kParts, bool kAhead>
constexpr int kNormCtas = kParts > 16 ? 1 : kParts == 16 ? (kAhead ? 1 : 2) : (kAhead ? 3 : 5);

// kParts warps share a row, each with kStrips strips of it in registers: h is formed once,
// its squares summed over the CTA, and everything written from the registers, so that a
// row crosses the chip once.  Sums are fp32, at most 80 additions in a chain.  CTA (p, i)
// takes tokens p, p + gridDim.x, ... (kRows at a time) of worker i.
template <typename T, Way kWay, int kParts, int kStrips, bool kAhead>
__global__ void __launch_bounds__(32 * kNormWarps<kParts>, (kNormCtas<kParts, kAhead>))
relay_rms_norm_kernel(NormArgs<T> a) {
    constexpr int kRows = kNormWarps<kParts> / kParts;
    __shared__ float shared[kNormWarps<kParts>];
    WARP_TURN(kNormWarps<kParts>, true);  // kVector: for unaligned weights
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, slot = warp / kParts, part = warp % kParts;
    const int worker = blockIdx.y, step = static_cast<int>(gridDim.x) * kRows;
    const float* weight = a.weight + worker * a.weight_stride;
    const auto base_of = [&](int j) { return (part + kParts * j) * kStrip; };

    Piece<T, kWay> x[kAhead ? kStrips : 1], r[kAhead ? kStrips : 1];
    const auto ask_strip = [&](int token, int j, int to) {
        const int left = token < a.tokens ? a.d - base_of(j) : 0;
        x[to].load(a.x.row(worker, token) + base_of(j), lane, left);
        if (a.residual.p != nullptr) r[to].load(a.residual.row(worker, token) + base_of(j), lane, left);
    };
    const auto ask = [&](int token) {
#pragma unroll
        for (int j = 0; j < kStrips; ++j) ask_strip(token, j, kAhead ? j : 0);
    };
    float w[kAhead ? kStrips : 1][8];
    int first = static_cast<int>(blockIdx.x) * kRows;
    if (kAhead) {
        ask(first + slot);
#pragma unroll
        for (int j = 0; j < kStrips; ++j)
            load_weight<kWay>(weight + base_of(j), lane, a.d - base_of(j), a.weight_quads, w[kAhead ? j : 0], turn);
    }
    for (; first < a.tokens; first += step) {
        const int token = first + slot;
        const int64_t row = static_cast<int64_t>(worker) * a.tokens + token;
        float h[kStrips][8];
        float squares = 0.0f;
#pragma unroll
        for (int j = 0; j < kStrips; ++j) {
            if (!kAhead) ask_strip(token, j, 0);
            x[kAhead ? j : 0].get(h[j]);
            if (a.residual.p != nullptr) {
                float add[8];
                r[kAhead ? j : 0].get(add);
#pragma unroll
                for (int k = 0; k < 8; ++k) h[j][k] += add[k];
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) squares = fmaf(h[j][k], h[j][k], squares);
        }
        if (kAhead && first + step < a.tokens) ask(first + step + slot);
        squares = row_sum<kParts>(squares, shared, slot, part);
        if (token >= a.tokens) {
            if (!kAhead) break;
            continue;
        }
        const float rstd = 1.0f / sqrtf(squares / static_cast<float>(a.d) + a.eps);
        if (a.rstd != nullptr && part == 0 && lane == 0) a.rstd[row] = rstd;
#pragma unroll
        for (int j = 0; j < kStrips; ++j) {
            const int base = base_of(j), left = a.d - base;
            if (base >= a.pitch) break;
            if (a.total.p != nullptr) store_strip<kWay>(a.total.row(worker, token) + base, lane, left, h[j]);
#pragma unroll
            for (int k = 0; k < 8; ++k) h[j][k] *= rstd;
            clear_past<kWay>(h[j], lane, left);
            if (a.codes != nullptr)
                put_strip<kWay>(a.codes + row * a.pitch, a.scales + row * (a.pitch / kBlock), base, lane, a.pitch, h[j],
                                kWay == kVector ? largest(h[j]) : 0u, turn);
            float m[8];
            if (!kAhead) load_weight<kWay>(weight + base, lane, left, a.weight_quads, m, turn);
#pragma unroll
            for (int k = 0; k < 8; ++k) h[j][k] *= kAhead ? w[kAhead ? j : 0][k] : m[k];
            store_strip<kWay>(a.y.row(worker, token) + base, lane, left, h[j]);
        }
        if (!kAhead) break;  // one row each
    }
}

template <typename T>
struct NormBackwardArgs {
    View<const T> dy, dtotal, total;
    View<T> dx;
    const float* weight;
    int64_t weight_stride;
    bool weight_quads;
    const float* rstd;
    const int8_t* codes;
    const uint8_t* scales;
    const int32_t* lengths;
    float* partial;  // [n][gridDim.x][pitch]
    int32_t tokens, d, pitch;
};

// CTA (p, i) takes tokens p, p + gridDim.x, ... (kRows at a time) of worker i and
// leaves their sum of dy xhat in its row of `partial`.  Aligned rows of up to 8192
// features keep the weight in registers (kHold); they, and others that leave room, ask
// for the next row before this one's sum over the CTA (kAhead).  16-bit rows stay as they
// came from memory and are widened again after that sum; others, and those in 8 bits, whose
// recall costs more than the registers, are kept as fp32 (kKeep).  The widest rows are read
// twice (kTwice), the second time from the caches.  The two CTAs' 128 registers are not
// quite enough for fp32 rows from the sum (72 to 80 bytes a thread go to local memory,
// [4][4096][4096] 156 us, 0.77 of the copy rate), nor the 64 of the widest rows (130 to 350).
template <typename T, Way kWay, int kParts, int kStrips, bool kEight>
__global__ void __launch_bounds__(32 * kNormWarps<kParts>, kNormWarps<kParts> > 8 ? 1 : 2)
relay_rms_norm_backward_kernel(NormBackwardArgs<T> a) {
    constexpr int kRows = kNormWarps<kParts> / kParts;
    constexpr bool kTwice = kParts > 16, kHold = kWay == kVector && kStrips <= 2,
                   kKeep = !kTwice && (kEight || kWay == kDirect || sizeof(T) == 4),
                   kAhead = kHold || (kWay == kVector && !kTwice && !kKeep);
    __shared__ float shared[kNormWarps<kParts>];
    WARP_TURN(kNormWarps<kParts>, true);  // kVector: for unaligned weights
    extern __shared__ float sums[];  // kRows > 1: [kRows - 1][kStrips][kParts][256]
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, slot = warp / kParts, part = warp % kParts;
    const int worker = blockIdx.y;
    const int length = a.lengths == nullptr ? a.tokens : min(max(a.lengths[worker], 0), a.tokens);
    const float* weight = a.weight + worker * a.weight_stride;
    const auto base_of = [&](int j) { return (part + kParts * j) * kStrip; };

    struct Row {  // what a lane needs of a row, as it lies in memory
        Piece<T, kWay> dy[kStrips], total[kEight ? 1 : kStrips], dtotal[kHold ? kStrips : 1];
        CodePiece codes[kEight ? kStrips : 1];
        float rstd;
    };
    const auto ask_strip = [&](Row& r, int token, int j, int to) {
        const bool on = token < length;
        const int base = base_of(j), left = on ? a.d - base : 0;
        const int64_t row = static_cast<int64_t>(worker) * a.tokens + token;
        r.dy[to].load(a.dy.row(worker, token) + base, lane, left);
        if constexpr (kEight)
            r.codes[to].load(a.codes + row * a.pitch, a.scales + row * (a.pitch / kBlock), base, lane, on ? a.pitch : 0);
        else
            r.total[to].load(a.total.row(worker, token) + base, lane, left);
    };
    const auto ask = [&](Row& r, int token) {
        r.rstd = token < length ? a.rstd[static_cast<int64_t>(worker) * a.tokens + token] : 0.0f;
#pragma unroll
        for (int j = 0; j < kStrips; ++j) {
            ask_strip(r, token, j, j);
            if constexpr (kHold)
                if (a.dtotal.p != nullptr)
                    r.dtotal[j].load(a.dtotal.row(worker, token) + base_of(j), lane, token < length ? a.d - base_of(j) : 0);
        }
    };
    // dy and xhat of strip j, from `from` of the row
    const auto widen_strip = [&](const Row& r, int token, int j, int from, float (&dy)[8], float (&xhat)[8]) {
        r.dy[from].get(dy);
        if constexpr (kEight) {
            r.codes[from].template get<kWay>(xhat, lane, turn);
            clear_past<kWay>(xhat, lane, token < length ? a.d - base_of(j) : 0);
        } else {
            r.total[from].get(xhat);
#pragma unroll
            for (int k = 0; k < 8; ++k) xhat[k] *= r.rstd;
        }
    };

    float w[kHold ? kStrips : 1][8];
    if constexpr (kHold) {
#pragma unroll
        for (int j = 0; j < kStrips; ++j) load_weight<kWay>(weight + base_of(j), lane, a.d - base_of(j), a.weight_quads, w[j], turn);
    }
    // u = dy w and xhat of strip j; `before` gets each k's dy and xhat
    const auto weigh = [&](const Row& r, int token, int j, float (&u)[8], float (&xhat)[8], auto before) {
        widen_strip(r, token, j, kTwice ? 0 : j, u, xhat);
        float m[8];
        if constexpr (!kHold) load_weight<kWay>(weight + base_of(j), lane, a.d - base_of(j), a.weight_quads, m, turn);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            before(k, u[k], xhat[k]);
            u[k] *= kHold ? w[kHold ? j : 0][k] : m[k];
        }
    };
    float dw[kStrips][8] = {};
    const int step = static_cast<int>(gridDim.x) * kRows;
    Row next;
    int first = static_cast<int>(blockIdx.x) * kRows;
    if (kAhead) ask(next, first + slot);
    for (; first < a.tokens; first += step) {
        const int token = first + slot;
        Row r;
        if (kTwice)
            r.rstd = token < length ? a.rstd[static_cast<int64_t>(worker) * a.tokens + token] : 0.0f;
        else if (kAhead)
            r = next;
        else
            ask(r, token);
        float along = 0.0f;
        float us[kKeep ? kStrips : 1][8], xhats[kKeep ? kStrips : 1][8];
#pragma unroll
        for (int j = 0; j < kStrips; ++j) {
            if (kTwice) ask_strip(r, token, j, 0);
            float(&u)[8] = us[kKeep ? j : 0];
            float(&xhat)[8] = xhats[kKeep ? j : 0];
            weigh(r, token, j, u, xhat, [&](int k, float dy, float x) { dw[j][k] = fmaf(dy, x, dw[j][k]); });
#pragma unroll
            for (int k = 0; k < 8; ++k) along = fmaf(u[k], xhat[k], along);
        }
        if (kAhead && first + step < a.tokens) ask(next, first + step + slot);
        along = row_sum<kParts>(along, shared, slot, part) / static_cast<float>(a.d);
        if (token < a.tokens) {
#pragma unroll
            for (int j = 0; j < kStrips; ++j) {
                const int base = base_of(j), left = a.d - base;
                if (left <= 0) break;
                float dh[8] = {};
                // padding is 0 also where 0 times the weight is not: by a branch, or element by element
                // where that goes faster ([2][2048][16384] from 8 bits: 102 us and 97 us)
                const bool counts = token < length;
                if (!kHold || counts) {
                    if (kTwice) ask_strip(r, token, j, 0);
                    float(&u)[8] = us[kKeep ? j : 0];
                    float(&xhat)[8] = xhats[kKeep ? j : 0];
                    if constexpr (!kKeep) {
                        if constexpr (!kTwice) {
                            r.dy[j].forget();
                            r.total[j].forget();
                        }
                        weigh(r, token, j, u, xhat, [](int, float, float) {});
                    }
                    if (a.dtotal.p != nullptr) {
                        if constexpr (!kHold) r.dtotal[0].load(a.dtotal.row(worker, token) + base, lane, counts ? left : 0);
                        r.dtotal[kHold ? j : 0].get(dh);
                    }
#pragma unroll
                    for (int k = 0; k < 8; ++k) dh[k] = kHold || counts ? fmaf(r.rstd, u[k] - xhat[k] * along, dh[k]) : 0.0f;
                }
                store_strip<kWay>(a.dx.row(worker, token) + base, lane, left, dh);
            }
        }
    }
    if (kRows > 1) {  // the rows that went side by side, in their order
        if (slot > 0) {
#pragma unroll
            for (int j = 0; j < kStrips; ++j)
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    sums[(((slot - 1) * kStrips + j) * kParts + part) * kStrip + 32 * k + lane] = dw[j][k];
        }
        __syncthreads();
        if (slot > 0) return;
        for (int s = 0; s < kRows - 1; ++s)
#pragma unroll
            for (int j = 0; j < kStrips; ++j)
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    dw[j][k] += sums[((s * kStrips + j) * kParts + part) * kStrip + 32 * k + lane];
    }
    float* out = a.partial + (static_cast<int64_t>(worker) * gridDim.x + blockIdx.x) * a.pitch;
#pragma unroll
    for (int j = 0; j < kStrips; ++j)
        store_strip<kWay == kDirect ? kDirect : kVector>(out + base_of(j), lane, a.pitch - base_of(j), dw[j]);
}

// dweight[i][k] = sum_p partial[i][p][k]: a CTA sums 32 columns, 8 rows at a time.
__global__ void __launch_bounds__(256)
relay_norm_join_kernel(const float* partial, int parts, int d, int pitch, float* dweight, int64_t dweight_stride) {
    __shared__ float shared[8][32];
    const int column = blockIdx.x * 32 + threadIdx.x % 32, lead = threadIdx.x / 32;
    const float* p = partial + static_cast<int64_t>(blockIdx.y) * parts * pitch;
    float s = 0.0f;
    if (column < d)
        for (int r = lead; r < parts; r += 8) s += p[static_cast<int64_t>(r) * pitch + column];
    shared[lead][threadIdx.x % 32] = s;
    __syncthreads();
    if (lead > 0 || column >= d) return;
#pragma unroll
    for (int r = 1; r < 8; ++r) s += shared[r][threadIdx.x];
    dweight[blockIdx.y * dweight_stride + column] = s;
}

// ---------------------------------------------------------------- launching

// The runs of an activation (with its checkpoint's padding), and the CTAs that take
// them: 0 where there is no device.
Grid make_grid(int32_t n, int64_t tokens, int64_t d, bool checkpoint, int* ctas) {
    constexpr int64_t run = kStrip * kRun;
    const int64_t pitch = pitch_of(d), runs = ((checkpoint ? pitch : d) + run - 1) / run, rows = n * tokens;
    const int64_t want = (rows * runs + kWarps - 1) / kWarps, most = int64_t(32) * sm_count();
    *ctas = static_cast<int>(want < most ? want : most);
    const int64_t step = int64_t(*ctas) * kWarps, step_rows = step / runs;
    return Grid{rows,
                static_cast<int32_t>(tokens),
                static_cast<int32_t>(runs),
                static_cast<int32_t>(d),
                static_cast<int32_t>(pitch),
                static_cast<int32_t>(step_rows / tokens),
                static_cast<int32_t>(step_rows % tokens),
                static_cast<int32_t>(step % runs)};
}

// Calls f(kParts, kStrips) as constants for the smallest instance that holds a row.
template <int kParts_, int kStrips_>
struct Hold {
    static constexpr int kParts = kParts_, kStrips = kStrips_;
};

template <typename F>
int by_width(int64_t pitch, F f) {
    if (pitch <= 256) return f(Hold<1, 1>());
    if (pitch <= 512) return f(Hold<1, 2>());
    if (pitch <= 1024) return f(Hold<2, 2>());
    if (pitch <= 2048) return f(Hold<4, 2>());
    if (pitch <= 4096) return f(Hold<8, 2>());
    if (pitch <= 8192) return f(Hold<16, 2>());
    if (pitch <= 16384) return f(Hold<16, 4>());
    return f(Hold<32, 4>());
}

// Rows of partial sums per worker in the norm's backward pass, one per CTA: about two
// CTAs per SM over all workers and no more than there are tokens; whole multiples of
// that where a thread would otherwise add up more than 256 rows in one chain, which
// for products of random signs is off by 4e-7 ([160][4096][2304] in one chain per
// worker was off by 6.1e-7).
int64_t norm_partials(int32_t n, int64_t tokens, int64_t d) {
    const int64_t pitch = pitch_of(d), side = pitch <= 512 ? 8 : pitch <= 1024 ? 4 : pitch <= 2048 ? 2 : 1;  // kRows
    const int64_t fill = 304 / n, chain = fill * side * 256, want = tokens > chain ? fill * ((tokens + chain - 1) / chain) : fill;
    return tokens < want ? (tokens > 0 ? tokens : 1) : want;
}
static_assert(RELAY_MAX_N <= 304, "a CTA per worker");

}  // namespace

extern "C" {

int64_t relay_checkpoint_pitch(int64_t d) { return d < 1 || d > kMaxD ? RELAY_EINVAL : pitch_of(d); }

int relay_checkpoint_pack(int32_t type, int32_t n, int64_t tokens, int64_t d, const relay_rows* x, int8_t* codes,
                          uint8_t* scales, relay_stream_t stream) {
    if (const int rc = check_shape(type, n, tokens, d)) return rc;
    if (!rows_fit(x, type, n, tokens, d, false) || !checkpoint_fits(codes, scales, tokens)) return RELAY_EINVAL;
    if (tokens == 0) return RELAY_OK;
    const bool vec = d % 8 == 0 && vectors(x, type, n, tokens);
    int ctas;
    const Grid g = make_grid(n, tokens, d, true, &ctas);
    if (ctas == 0) return RELAY_ECUDA;
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        (vec ? relay_checkpoint_pack_kernel<T, kVector> : relay_checkpoint_pack_kernel<T, kDirect>)
            <<<ctas, 32 * kWarps, 0, stream>>>(g, view<const T>(x, n, tokens), codes, scales);
        return status_of_launch();
    });
}

int relay_checkpoint_unpack(int32_t type, int32_t n, int64_t tokens, int64_t d, const int8_t* codes,
                            const uint8_t* scales, const relay_rows* out, relay_stream_t stream) {
    if (const int rc = check_shape(type, n, tokens, d)) return rc;
    if (!rows_fit(out, type, n, tokens, d, true) || !checkpoint_fits(codes, scales, tokens)) return RELAY_EINVAL;
    if (tokens == 0) return RELAY_OK;
    const bool vec = d % 8 == 0 && vectors(out, type, n, tokens);
    int ctas;
    const Grid g = make_grid(n, tokens, d, false, &ctas);
    if (ctas == 0) return RELAY_ECUDA;
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        (vec ? relay_checkpoint_unpack_kernel<T, kVector> : relay_checkpoint_unpack_kernel<T, kDirect>)
            <<<ctas, 32 * kWarps, 0, stream>>>(g, codes, scales, view<T>(out, n, tokens));
        return status_of_launch();
    });
}

int relay_rms_norm(int32_t type, int32_t n, int64_t tokens, int64_t d, const relay_rows* x,
                   const relay_rows* residual, const float* weight, int64_t weight_stride, float eps,
                   const relay_rows* total, const relay_rows* y, float* rstd, int8_t* codes, uint8_t* scales,
                   relay_stream_t stream) {
    if (const int rc = check_shape(type, n, tokens, d)) return rc;
    if (d > RELAY_NORM_MAX_D) return RELAY_EUNSUPPORTED;
    if (!(eps > 0.0f) || !(eps < 1e30f) || weight == nullptr || !aligned(weight, 4) || weight_stride < 0)
        return RELAY_EINVAL;
    if (!rows_fit(x, type, n, tokens, d, false) || !rows_fit(y, type, n, tokens, d, true)) return RELAY_EINVAL;
    if (residual != nullptr && !rows_fit(residual, type, n, tokens, d, false)) return RELAY_EINVAL;
    if (total != nullptr && !rows_fit(total, type, n, tokens, d, true)) return RELAY_EINVAL;
    if (!aligned(rstd, 4) || (codes == nullptr) != (scales == nullptr)) return RELAY_EINVAL;
    if (codes != nullptr && !checkpoint_fits(codes, scales, tokens)) return RELAY_EINVAL;
    if (tokens == 0) return RELAY_OK;
    if (y->data == x->data || (residual != nullptr && y->data == residual->data) ||
        (total != nullptr && y->data == total->data))
        return RELAY_EINVAL;
    if (crossed(total, x, n, tokens) || crossed(total, residual, n, tokens)) return RELAY_EINVAL;
    const bool vec = d % 8 == 0 && vectors(x, type, n, tokens) && vectors(residual, type, n, tokens) &&
                     vectors(total, type, n, tokens) && vectors(y, type, n, tokens);
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        const NormArgs<T> a{view<const T>(x, n, tokens), view<const T>(residual, n, tokens),
                            view<T>(total, n, tokens), view<T>(y, n, tokens), weight, n > 1 ? weight_stride : 0,
                            d % 8 == 0 && aligned(weight, 16) && (n == 1 || weight_stride % 4 == 0), eps, rstd, codes, scales,
                            static_cast<int32_t>(tokens), static_cast<int32_t>(d),
                            static_cast<int32_t>(pitch_of(d))};
        return by_width(a.pitch, [&](auto hold) {
            constexpr int kParts = decltype(hold)::kParts, kStrips = decltype(hold)::kStrips;
            constexpr int kRows = kNormWarps<kParts> / kParts;
            // three CTAs per SM where they stay, over all workers, otherwise one for each row (or kRows of them)
            const int64_t all = (tokens + kRows - 1) / kRows, stay = 3 * 152 / n > 0 ? 3 * 152 / n : 1;
            constexpr bool kMay = kMayStay<T, kVector, kStrips>;
            const bool stays = kMay && vec && (residual == nullptr || a.pitch > 4096);
            const dim3 grid(static_cast<unsigned>(stays && stay < all ? stay : all), static_cast<unsigned>(n));
            (stays ? relay_rms_norm_kernel<T, kVector, kParts, kStrips, kMay>
             : vec ? relay_rms_norm_kernel<T, kVector, kParts, kStrips, false>
                   : relay_rms_norm_kernel<T, kDirect, kParts, kStrips, false>)
                <<<grid, 32 * kNormWarps<kParts>, 0, stream>>>(a);
            return status_of_launch();
        });
    });
}

int64_t relay_rms_norm_backward_workspace(int32_t n, int64_t tokens, int64_t d) {
    if (const int rc = check_shape(RELAY_FP32, n, tokens, d)) return rc;
    if (d > RELAY_NORM_MAX_D) return RELAY_EUNSUPPORTED;
    return 4 * n * norm_partials(n, tokens, d) * pitch_of(d);
}

int relay_rms_norm_backward(int32_t type, int32_t n, int64_t tokens, int64_t d, const relay_rows* dy,
                            const relay_rows* dtotal, const float* weight, int64_t weight_stride, const float* rstd,
                            const relay_rows* total, const int8_t* codes, const uint8_t* scales,
                            const int32_t* lengths, const relay_rows* dx, float* dweight, int64_t dweight_stride,
                            void* workspace, int64_t workspace_bytes, relay_stream_t stream) {
    if (const int rc = check_shape(type, n, tokens, d)) return rc;
    if (d > RELAY_NORM_MAX_D) return RELAY_EUNSUPPORTED;
    if (weight == nullptr || !aligned(weight, 4) || weight_stride < 0) return RELAY_EINVAL;
    if (!rows_fit(dy, type, n, tokens, d, false) || !rows_fit(dx, type, n, tokens, d, true)) return RELAY_EINVAL;
    if (dtotal != nullptr && !rows_fit(dtotal, type, n, tokens, d, false)) return RELAY_EINVAL;
    if (tokens > 0 && (rstd == nullptr || !aligned(rstd, 4))) return RELAY_EINVAL;
    const bool eight = codes != nullptr || scales != nullptr;
    if (eight ? total != nullptr || !checkpoint_fits(codes, scales, tokens)
              : tokens > 0 && !rows_fit(total, type, n, tokens, d, false))
        return RELAY_EINVAL;
    if (!aligned(lengths, 4)) return RELAY_EINVAL;
    if (dweight == nullptr || !aligned(dweight, 4) || (n > 1 && dweight_stride < d)) return RELAY_EINVAL;
    if (workspace == nullptr || !aligned(workspace, 16) ||
        workspace_bytes < relay_rms_norm_backward_workspace(n, tokens, d))
        return RELAY_EINVAL;
    if (tokens > 0 && (dx->data == dy->data || (dtotal != nullptr && dx->data == dtotal->data) ||
                       (!eight && dx->data == total->data)))
        return RELAY_EINVAL;
    const bool vec = d % 8 == 0 && vectors(dy, type, n, tokens) && vectors(dtotal, type, n, tokens) &&
                     vectors(eight ? nullptr : total, type, n, tokens) && vectors(dx, type, n, tokens);
    const int parts = static_cast<int>(norm_partials(n, tokens, d));
    const int rc = by_type(type, [&](auto t) {
        using T = decltype(t);
        const NormBackwardArgs<T> a{view<const T>(dy, n, tokens), view<const T>(dtotal, n, tokens),
                                    view<const T>(total, n, tokens), view<T>(dx, n, tokens), weight,
                                    n > 1 ? weight_stride : 0,
                                    d % 8 == 0 && aligned(weight, 16) && (n == 1 || weight_stride % 4 == 0), rstd, codes, scales,
                                    lengths, static_cast<float*>(workspace), static_cast<int32_t>(tokens),
                                    static_cast<int32_t>(d), static_cast<int32_t>(pitch_of(d))};
        // Unaligned 16-bit rows of up to 256 features from 8 bits go faster with the wider instance's two
        // strips where they come from HBM ([16][16384][201]: 153 against 162 us, [4][89240][94] with
        // dtotal 251 and 267), and slower where L2 holds them ([4][16384][201]: 38 against 29 us,
        // [4][2048][94] 9.2 and 7.8); fp32 rows and aligned ones always do better with one.
        const int64_t row_bytes = element_size(type) * d * (dtotal != nullptr ? 3 : 2) + pitch_of(d) * 33 / 32;
        const bool two = eight && !vec && type != RELAY_FP32 && n * tokens * row_bytes > 120000000;
        return by_width(two && a.pitch <= 256 ? 512 : a.pitch, [&](auto hold) {
            constexpr int kParts = decltype(hold)::kParts, kStrips = decltype(hold)::kStrips;
            constexpr size_t kSmem = (kNormWarps<kParts> / kParts - 1) * kStrips * kParts * kStrip * sizeof(float);
            (vec ? (eight ? relay_rms_norm_backward_kernel<T, kVector, kParts, kStrips, true>
                          : relay_rms_norm_backward_kernel<T, kVector, kParts, kStrips, false>)
                 : (eight ? relay_rms_norm_backward_kernel<T, kDirect, kParts, kStrips, true>
                          : relay_rms_norm_backward_kernel<T, kDirect, kParts, kStrips, false>))
                <<<dim3(parts, n), 32 * kNormWarps<kParts>, kSmem, stream>>>(a);
            return status_of_launch();
        });
    });
    if (rc != RELAY_OK) return rc;
    relay_norm_join_kernel<<<dim3(static_cast<unsigned>((d + 31) / 32), n), 256, 0, stream>>>(
        static_cast<const float*>(workspace), parts, static_cast<int>(d), static_cast<int>(pitch_of(d)), dweight,
        dweight_stride);
    return status_of_launch();
}

int relay_gated(int32_t type, int32_t n, int64_t tokens, int64_t d, const relay_rows* gate, const relay_rows* up,
                const relay_rows* out, int8_t* gate_codes, uint8_t* gate_scales, int8_t* up_codes,
                uint8_t* up_scales, relay_stream_t stream) {
    if (const int rc = check_shape(type, n, tokens, d)) return rc;
    if (!rows_fit(gate, type, n, tokens, d, false) || !rows_fit(up, type, n, tokens, d, false) ||
        !rows_fit(out, type, n, tokens, d, true))
        return RELAY_EINVAL;
    if ((gate_codes == nullptr) != (gate_scales == nullptr) || (up_codes == nullptr) != (up_scales == nullptr))
        return RELAY_EINVAL;
    if (gate_codes != nullptr && !checkpoint_fits(gate_codes, gate_scales, tokens)) return RELAY_EINVAL;
    if (up_codes != nullptr && !checkpoint_fits(up_codes, up_scales, tokens)) return RELAY_EINVAL;
    if (gate_codes != nullptr && (gate_codes == up_codes || gate_scales == up_scales)) return RELAY_EINVAL;
    if (tokens == 0) return RELAY_OK;
    if (out->data == gate->data || out->data == up->data) return RELAY_EINVAL;
    const bool vec = d % 8 == 0 && vectors(gate, type, n, tokens) && vectors(up, type, n, tokens) &&
                     vectors(out, type, n, tokens);
    int ctas;
    const Grid g = make_grid(n, tokens, d, gate_codes != nullptr || up_codes != nullptr, &ctas);
    if (ctas == 0) return RELAY_ECUDA;
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        (vec ? relay_gated_kernel<T, kVector> : relay_gated_kernel<T, kDirect>)<<<ctas, 32 * kWarps, 0, stream>>>(
            g, view<const T>(gate, n, tokens), view<const T>(up, n, tokens), view<T>(out, n, tokens), gate_codes,
            gate_scales, up_codes, up_scales);
        return status_of_launch();
    });
}

int relay_gated_backward(int32_t type, int32_t n, int64_t tokens, int64_t d, const relay_rows* dout,
                         const relay_rows* gate, const relay_rows* up, const int8_t* gate_codes,
                         const uint8_t* gate_scales, const int8_t* up_codes, const uint8_t* up_scales,
                         const relay_rows* dgate, const relay_rows* dup, int8_t* out_codes, uint8_t* out_scales,
                         relay_stream_t stream) {
    if (const int rc = check_shape(type, n, tokens, d)) return rc;
    if (!rows_fit(dout, type, n, tokens, d, false) || !rows_fit(dgate, type, n, tokens, d, true) ||
        !rows_fit(dup, type, n, tokens, d, true))
        return RELAY_EINVAL;
    const bool eight = gate_codes != nullptr || gate_scales != nullptr || up_codes != nullptr || up_scales != nullptr;
    if (eight ? gate != nullptr || up != nullptr || !checkpoint_fits(gate_codes, gate_scales, tokens) ||
                    !checkpoint_fits(up_codes, up_scales, tokens)
              : tokens > 0 && (!rows_fit(gate, type, n, tokens, d, false) || !rows_fit(up, type, n, tokens, d, false)))
        return RELAY_EINVAL;
    if ((out_codes == nullptr) != (out_scales == nullptr)) return RELAY_EINVAL;
    if (out_codes != nullptr && (!checkpoint_fits(out_codes, out_scales, tokens) || out_codes == gate_codes ||
                                 out_codes == up_codes || out_scales == gate_scales || out_scales == up_scales))
        return RELAY_EINVAL;
    if (tokens == 0) return RELAY_OK;
    for (const relay_rows* o : {dgate, dup})
        if (o->data == dout->data || (!eight && (o->data == gate->data || o->data == up->data))) return RELAY_EINVAL;
    if (dgate->data == dup->data) return RELAY_EINVAL;
    const bool vec = d % 8 == 0 && vectors(dout, type, n, tokens) && vectors(dgate, type, n, tokens) &&
                     vectors(dup, type, n, tokens) && vectors(eight ? nullptr : gate, type, n, tokens) &&
                     vectors(eight ? nullptr : up, type, n, tokens);
    int ctas;
    const Grid g = make_grid(n, tokens, d, out_codes != nullptr, &ctas);
    if (ctas == 0) return RELAY_ECUDA;
    const GatedSource from{gate_codes, up_codes, gate_scales, up_scales};
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        (vec ? (eight ? relay_gated_backward_kernel<T, kVector, true> : relay_gated_backward_kernel<T, kVector, false>)
             : (eight ? relay_gated_backward_kernel<T, kDirect, true> : relay_gated_backward_kernel<T, kDirect, false>))
            <<<ctas, 32 * kWarps, 0, stream>>>(g, view<const T>(dout, n, tokens),
                                               view<const T>(eight ? nullptr : gate, n, tokens),
                                               view<const T>(eight ? nullptr : up, n, tokens), from,
                                               view<T>(dgate, n, tokens), view<T>(dup, n, tokens), out_codes,
                                               out_scales);
        return status_of_launch();
    });
}

}  // extern "C"
