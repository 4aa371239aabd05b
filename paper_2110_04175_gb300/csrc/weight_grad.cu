// weight_grad.cu -- the weight gradient of a linear layer whose inputs were kept
// in 8 bits (relay_weight_grad of relaylayers.h) on GB300 (sm_103a):
//
//   dW_i[o][k] = scale_i[k] sum_t dy_i[t][o] xhat_i[t][k]
//
// A product of dy^T [outputs][tokens] by xhat [tokens][inputs] on the tensor
// cores, accumulated in fp32.  Tokens are the axis that is summed over and lie
// furthest apart in both operands, so both go to shared memory as they lie in
// memory, M and N fastest, 64 tokens at a time:
//   - xhat is recalled from its codes on the way: a code is a whole number of 7
//     bits and its scale a power of two, so the bf16 values are exact;
//   - dy in bf16 comes by TMA.  fp16 and fp32 (and rows that TMA cannot take) are
//     read by the warps that recall xhat and split into bf16 terms that add up to
//     them exactly, 8 bits each: 2 for fp16, 3 for fp32, one product each.
//
// A pair of CTAs makes a tile of 256 outputs x kN inputs (cta_group::2): each
// brings half of both operands, so that a code is recalled once for 256 outputs.
//
// The tensor cores cut off what an addition shifts out, so that a long sum in
// their accumulator drifts towards zero: 6.3e-6 of the result after 384 additions.
// So they sum 32 to 48 additions at a time, in one of two accumulators, and the
// warps that write the stages add the other one to registers, rounded to the
// nearest.
#include "blackwell.cuh"
#include "layers.cuh"

namespace {

constexpr int kM = 128;        // outputs of a CTA
constexpr int kDepth = 64;     // tokens of a stage
// Warps: 0 .. 7 write stages and add up the sums, 8 .. 11 issue products and copies
// (one of them is idle), 12 .. 15 write stages only.  The writers are teams of 4 that
// take stages in turn, so that one team's waits are the others' work.
constexpr int kAdders = 8, kIssuer = 8, kTeam = 4, kTeams = 3;
constexpr int kThreads = 32 * 16;
// 4 warpgroups are launched with 128 registers a thread: 2 x 176 + 64 + 96 = 4 x 128
constexpr int kAdderRegisters = 176, kIssuerRegisters = 64, kMakerRegisters = 96;
constexpr int kPanel = kDepth * 128;  // bytes of 64 outputs or inputs x kDepth tokens
constexpr int kSms = 152;

template <typename T>
constexpr int kTerms = sizeof(T) == 4 ? 3 : 2;  // bf16 terms of a value
template <>
constexpr int kTerms<__nv_bfloat16> = 1;

// Stages that the tensor cores sum before the sums are added up in registers.
template <typename T>
constexpr int kGroup = kTerms<T> == 1 ? 8 : 4;

template <typename T, int kN>
struct Stages {  // in a CTA
    static constexpr int kLeft = kTerms<T> * kM / 64 * kPanel, kBytes = kLeft + kN / 2 / 64 * kPanel;
    static constexpr int kCount = 196608 / kBytes < 4 ? 196608 / kBytes : 4;
    // stages of codes, as they lie in memory: they come well before they are needed
    static constexpr int kCodes = kN / 2 * kDepth;
    static constexpr int kAhead = kCount * kBytes + 8 * kCodes <= 196608 ? 8 : 4;
    static constexpr int kShared = kCount * kBytes + kAhead * kCodes + 1024 + 512;  // alignment, barriers
    static_assert(kShared <= 232448, "shared memory of a CTA");
};

template <typename T>
struct WeightGradArgs {
    View<const T> dy;
    bool dy_vectors;
    const int8_t* codes;
    const uint8_t* scales;
    const float* column_scale;
    int64_t column_scale_stride;
    const int32_t* lengths;
    float* out;  // dweight, or with several splits the partial sums [split][n][outputs][inputs]
    int64_t worker_stride, row_stride, split_stride;
    int32_t n, tokens, outputs, inputs, pitch, splits;
};

// ----------------------------------------------------------------- the stages

// Byte offset of 8 outputs (or inputs) from number 8 j on, of token t, in an
// operand: 16-byte pieces, swizzled within 128 bytes by the token.
__device__ __forceinline__ uint32_t piece(int j, int t) {
    return static_cast<uint32_t>(j / 8 * kPanel + t * 128 + ((j % 8) ^ (t % 8)) * 16);
}

__device__ __forceinline__ void put_shared(uint32_t at, uint4 v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w)
                 : "memory");
}

__device__ __forceinline__ uint32_t bits(__nv_bfloat162 v) { return *reinterpret_cast<uint32_t*>(&v); }
__device__ __forceinline__ __nv_bfloat162 pair(uint32_t v) { return *reinterpret_cast<__nv_bfloat162*>(&v); }

// Codes 2h and 2h + 1 of the word w times `unit` (twice the same bf16).  A byte b
// stands for (b & 127) - (b & 128); under the exponent of 128 the two parts are
// the bf16 values 128 + (b & 127) and 128 + (b & 128), whose difference is exact.
__device__ __forceinline__ uint32_t recall_pair(uint32_t w, int h, uint32_t unit) {
    const uint32_t p = __byte_perm(w, 0u, h ? 0x4342 : 0x4140);
    const uint32_t low = (p & 0x007f007fu) | 0x43004300u, sign = (p & 0x00800080u) | 0x43004300u;
    return bits(__hmul2(__hsub2(pair(low), pair(sign)), pair(unit)));
}

// A warp's part of a stage of kWide inputs of xhat: a lane recalls 8 codes of a
// token per pass.
template <int kWide>
struct Recall {
    static constexpr int kLanes = kWide / 8;                         // lanes of a token
    static constexpr int kRows = 32 / kLanes;                        // tokens of a pass
    static constexpr int kPasses = kDepth / (kRows * kTeam);
    static constexpr int kTokens = kRows * kPasses;                  // of the warp
    static_assert(kTokens * kTeam == kDepth && kTokens <= 32 && kWide <= 128, "a lane per token's scales");

    static constexpr int kScaled = 32 / kTokens;                     // of the team's stages: those whose scales a load brings

    // The stage's token that sub-row `sub` of the warp has in pass r.
    static __device__ __forceinline__ int token(int warp, int r, int sub) { return (r * kTeam + warp) * kRows + sub; }

    // Lane l's word of scales: those of token l % kTokens (in the order of passes) of
    // the team's stage l / kTokens from the given one on.  warp: in the team.
    static __device__ __forceinline__ uint32_t scales(const uint8_t* p, int64_t row0, int left, int k0, int pitch,
                                                      int warp, int lane) {
        const int i = lane % kTokens, t = lane / kTokens * (kTeams * kDepth) + token(warp, i / kRows, i % kRows);
        if (t >= left || k0 >= pitch) return 0x07070707u;
        const uint8_t* at = p + (row0 + t) * (pitch / kBlock) + k0 / kBlock;
        if constexpr (kWide == 128) return __ldg(reinterpret_cast<const uint32_t*>(at));
        return __ldg(reinterpret_cast<const uint16_t*>(at));
    }

    // `from`: the stage's codes; tokens from `left` on do not count.  scales: what scales()
    // gave, each byte at least 7, less 6; 249 says that the block is no number (`odd`: some
    // byte says so).  turn: the stage's place among those of the load.
    static __device__ __forceinline__ void make(uint32_t from, uint32_t to, uint32_t scales, bool odd, int turn,
                                                int left, int warp, int lane) {
        const int j = lane % kLanes, sub = lane / kLanes;
        const uint32_t pick = 0x4040u | (j / 4) * 0x0101u;  // this lane's byte, in both halves
        const uint32_t at = from + token(warp, 0, sub) * kWide + 8 * j, put = to + piece(j, token(warp, 0, sub));
        uint2 q[kPasses];
        uint32_t u[kPasses];
#pragma unroll
        for (int r = 0; r < kPasses; ++r) {
            asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];"
                         : "=r"(q[r].x), "=r"(q[r].y)
                         : "r"(at + r * (kTeam * kRows * kWide)));
            const uint32_t w = __shfl_sync(0xffffffffu, scales, turn * kTokens + r * kRows + sub);
            u[r] = __byte_perm(w, 0u, pick) << 7;
        }
        if (odd) {
#pragma unroll
            for (int r = 0; r < kPasses; ++r)
                if (u[r] == (249u << 7 | 249u << 23)) u[r] = 0x7fff7fffu;
        }
        if (left < kDepth) {
#pragma unroll
            for (int r = 0; r < kPasses; ++r)
                if (token(warp, r, sub) >= left) q[r] = make_uint2(0, 0), u[r] = 0;
        }
#pragma unroll
        for (int r = 0; r < kPasses; ++r)
            put_shared(put + r * (kTeam * kRows * 128),
                       make_uint4(recall_pair(q[r].x, 0, u[r]), recall_pair(q[r].x, 1, u[r]),
                                  recall_pair(q[r].y, 0, u[r]), recall_pair(q[r].y, 1, u[r])));
    }
};

// A warp's part of a stage of dy, read and split into bf16 terms: each term is
// what is left with all but 8 bits cut off, so that the terms add up exactly.
template <typename T>
__device__ __forceinline__ void split_rows(const WeightGradArgs<T>& a, int worker, int token0, int left, int o0,
                                           uint32_t to, int warp, int lane) {
    const int j = lane % 16, o = o0 + 8 * j;
#pragma unroll
    for (int r = 0; r < kDepth / (2 * kTeam); ++r) {
        const int t = (r * kTeam + warp) * 2 + lane / 16;
        float v[8] = {};
        if (t < left && o < a.outputs) {
            const T* p = a.dy.row(worker, token0 + t) + o;
            if (a.dy_vectors) {
                load_strip<true>(p, 0, 8, v);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (o + k < a.outputs) v[k] = widen(p[k]);
            }
        }
#pragma unroll
        for (int term = 0; term < kTerms<T>; ++term) {
            uint32_t w[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                uint32_t high = __float_as_uint(v[k]) & 0xffff0000u;
                if ((high & 0x7f800000u) == 0x7f800000u) {  // infinity or NaN: all in the first term
                    high = v[k] != v[k] ? 0x7fff0000u : high;
                    v[k] = 0.0f;
                } else {
                    v[k] -= __uint_as_float(high);
                }
                w[k] = high;
            }
            put_shared(to + term * (kM / 64 * kPanel) + piece(j, t),
                       make_uint4(__byte_perm(w[0], w[1], 0x7632), __byte_perm(w[2], w[3], 0x7632),
                                  __byte_perm(w[4], w[5], 0x7632), __byte_perm(w[6], w[7], 0x7632)));
        }
    }
}

// ----------------------------------------------------------------- the kernel

// A pair of CTAs per tile of 256 outputs x kN inputs and per split of the tokens.
// Warps 0 .. 7 write xhat (and dy, without TMA) into the stages, add up the sums
// and write them to memory; warp 8 of CTA 0 issues the products (that of CTA 1
// says when its half is ready); warps 9 and 10 issue the copies.  A wait that runs out ends the
// work on the tile, and its results are NaN.
template <typename T, bool kTma, int kN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
relay_weight_grad_kernel(const __grid_constant__ WeightGradArgs<T> a, const __grid_constant__ CUtensorMap dy_map,
                         const __grid_constant__ CUtensorMap codes_map) {
    using S = Stages<T, kN>;
    constexpr int kCount = S::kCount, kColumns = kN / 2;  // columns: of a warp, in the end
    extern __shared__ uint8_t raw[];
    const uint32_t stages = (shared_address(raw) + 1023u) & ~1023u;
    const uint32_t codes = stages + kCount * S::kBytes, bars = codes + S::kAhead * S::kCodes;
    // per stage: full (of codes recalled, of dy; on CTA 0 of the other CTA's half too) and free
    // again; per accumulator: summed by the tensor cores, and read; per stage of codes: there, and used
    const auto full = [&](int s) { return bars + 8 * s; };
    const auto freed = [&](int s) { return bars + 8 * (kCount + s); };
    const auto summed = [&](int b) { return bars + 8 * (2 * kCount + b); };
    const auto read = [&](int b) { return bars + 8 * (2 * kCount + 2 + b); };
    const auto fetched = [&](int s) { return bars + 8 * (2 * kCount + 4 + s); };
    const auto used = [&](int s) { return bars + 8 * (2 * kCount + 4 + S::kAhead + s); };
    const uint32_t tensor_at = bars + 8 * (2 * kCount + 4 + 2 * S::kAhead);
    __shared__ int stalled;

    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x / 32), 0), lane = threadIdx.x % 32;
    const uint32_t rank = cluster_rank();
    const int o0 = blockIdx.x * kM, k0 = blockIdx.y * kN;
    const int worker = blockIdx.z / a.splits, split = blockIdx.z % a.splits;
    const int length = a.lengths == nullptr ? a.tokens : min(max(a.lengths[worker], 0), a.tokens);
    // this split's stages of the tokens
    const int all = (length + kDepth - 1) / kDepth, each = (all + a.splits - 1) / a.splits;
    const int first = min(split * each, all), count = min(first + each, all) - first;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kCount; ++s) {
            barrier_init(full(s), kTeam + (kTma ? 1 : 0) + (rank == 0 ? 1 : 0));
            barrier_init(freed(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            barrier_init(summed(b), 1);
            barrier_init(read(b), kAdders);
        }
        for (int s = 0; s < S::kAhead; ++s) {
            barrier_init(fetched(s), 1);
            barrier_init(used(s), kTeam);
        }
        barriers_ready();
        stalled = 0;
    }
    if (warp == kIssuer) tensor_alloc<2 * kN>(tensor_at);
    tensor_fence_before();
    __syncthreads();
    cluster_sync();
    tensor_fence_after();
    uint32_t tensor;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(tensor) : "r"(tensor_at));

    bool ok = true;
    const int half = k0 + kN / 2 * static_cast<int>(rank);  // the inputs that this CTA recalls
    const int64_t row0 = static_cast<int64_t>(worker) * a.tokens + first * kDepth;
    // Writes the team's stages; after each calls after(i), and ends where that fails.
    const auto write_stages = [&](int team, auto after) {
        using R = Recall<kN / 2>;
        const int member = warp % kTeam;
        const auto load = [&](int i) {  // the scales of the team's R::kScaled stages from i on
            const int left = length - (first + i) * kDepth;
            return R::scales(a.scales, row0 + static_cast<int64_t>(i) * kDepth, left, half, a.pitch, member, lane);
        };
        uint32_t now = 0, next = load(team);
        bool odd = false;
        for (int i = team, turn = 0; i < count; i += kTeams) {
            const int s = i % kCount, f = i % S::kAhead, left = length - (first + i) * kDepth;
            if (turn == 0) {
                odd = __any_sync(0xffffffffu, __vcmpeq4(next, 0xffffffffu) != 0u);
                now = __vmaxu4(next, 0x07070707u) - 0x06060606u;
                next = load(i + kTeams * R::kScaled);
            }
            if (!barrier_wait(freed(s), (i / kCount & 1) ^ 1)) return false;
            if (!kTma)
                split_rows(a, worker, (first + i) * kDepth, left, o0, stages + s * S::kBytes, member, lane);
            if (!barrier_wait(fetched(f), i / S::kAhead & 1)) return false;
            R::make(codes + f * S::kCodes, stages + s * S::kBytes + S::kLeft, now, odd, turn, left, member, lane);
            fence_async();
            __syncwarp();
            if (lane == 0) {
                barrier_arrive(full(s));
                barrier_arrive(used(f));
            }
            turn = turn == R::kScaled - 1 ? 0 : turn + 1;
            if (!after(i)) return false;
        }
        return true;
    };
    if (warp < kAdders) {
        more_registers<kAdderRegisters>();
        // outputs 32 (warp % 4) + lane, inputs kColumns (warp / 4) ..
        float sum[kColumns] = {};
        int groups = 0;  // added up so far
        const auto add_group = [&] {
            const int b = groups & 1;
            if (!barrier_wait(summed(b), groups >> 1 & 1)) return false;
            tensor_fence_after();
            const uint32_t at =
                tensor + (static_cast<uint32_t>(32 * (warp % 4)) << 16) + b * kN + kColumns * (warp / 4);
#pragma unroll
            for (int c = 0; c < kColumns; c += 16) {
                float v[16];
                tensor_load(at + c, v);
#pragma unroll
                for (int e = 0; e < 16; ++e) sum[c + e] += v[e];
            }
            tensor_fence_before();
            __syncwarp();
            if (lane == 0) barrier_arrive(read(b));
            ++groups;
            return true;
        };
        ok = write_stages(warp / kTeam, [&](int i) {
            // stage i - kCount is done, and with it perhaps a whole group
            return i + 1 - kCount < (groups + 1) * kGroup<T> || add_group();
        });
        while (ok && groups * kGroup<T> < count) ok = add_group();
        if (!ok) stalled = 1;
        asm volatile("bar.sync 1, %0;" ::"n"(32 * kAdders) : "memory");  // all stages are read: their memory is free

        // through shared memory, so that a warp's stores are contiguous whatever the rows' alignment
        float* turn = reinterpret_cast<float*>(raw + (stages - shared_address(raw))) + warp * (32 * 33);
        float* out = a.out + split * a.split_stride + worker * a.worker_stride;
        const int o = o0 + 32 * (warp % 4);
#pragma unroll
        for (int c = 0; c < kColumns; c += 32) {
            const int k = k0 + kColumns * (warp / 4) + c + lane;
#pragma unroll
            for (int e = 0; e < 32; ++e) turn[lane * 33 + e] = sum[c + e];
            __syncwarp();
            if (k < a.inputs) {
                float scale = a.column_scale == nullptr || a.splits > 1
                                  ? 1.0f
                                  : a.column_scale[worker * a.column_scale_stride + k];
                if (stalled) scale = __int_as_float(0x7fffffff);
#pragma unroll 8
                for (int r = 0; r < 32; ++r)
                    if (o + r < a.outputs) out[(o + r) * a.row_stride + k] = turn[r * 33 + lane] * scale;
            }
            __syncwarp();
        }
    } else if (warp >= kIssuer + 4) {
        fewer_registers<kMakerRegisters>();
        ok = write_stages(2, [](int) { return true; });
    } else {
      fewer_registers<kIssuerRegisters>();
      if (warp == kIssuer) {
        for (int i = 0; i < count; ++i) {
            const int s = i % kCount, group = i / kGroup<T>, b = group & 1;
            const uint32_t left = stages + s * S::kBytes;
            if (i % kGroup<T> == 0 && group > 1 && !(ok = barrier_wait(read(b), (group >> 1 & 1) ^ 1))) break;
            if (!(ok = barrier_wait(full(s), i / kCount & 1))) break;
            const int from = length - (first + i) * kDepth;
            if (kTma && from < kDepth) {  // the copy brought the rows past the length too, whatever they hold
                for (int e = from * 8 + lane; e < kDepth * 8; e += 32)
                    for (int p = 0; p < kM / 64; ++p) put_shared(left + p * kPanel + e * 16, make_uint4(0, 0, 0, 0));
                fence_async();
                __syncwarp();
            }
            if (rank != 0) {
                if (elected()) barrier_arrive_there(in_cta(full(s), 0));
                continue;
            }
            tensor_fence_after();
            if (elected()) {
                const uint64_t dy = operand(left, kPanel, 1024), xhat = operand(left + S::kLeft, kPanel, 1024);
#pragma unroll
                for (int term = 0; term < kTerms<T>; ++term)
#pragma unroll
                    for (int k = 0; k < kDepth / 16; ++k)  // addresses count 16 bytes
                        product(tensor + b * kN, dy + (term * (kM / 64 * kPanel) + k * 2048) / 16, xhat + k * 2048 / 16,
                                kProductKind<2 * kM, kN>, i % kGroup<T> + term + k > 0);
                products_arrive(freed(s));
                if (i % kGroup<T> == kGroup<T> - 1 || i == count - 1) products_arrive(summed(b));
            }
            __syncwarp();
        }
      } else if (kTma && warp == kIssuer + 1 && elected()) {
        int sent = 0;
        for (; sent < count; ++sent) {
            const int s = sent % kCount;
            if (!(ok = barrier_wait(freed(s), (sent / kCount & 1) ^ 1))) break;
            barrier_expect(full(s), kM / 64 * kPanel);
            for (int p = 0; p < kM / 64; ++p)
                copy_box(stages + s * S::kBytes + p * kPanel, &dy_map, o0 + 64 * p, (first + sent) * kDepth, worker,
                         full(s));
        }
        for (int i = max(0, sent - kCount); i < sent; ++i)  // nothing is left in flight
            if (!barrier_wait(full(i % kCount), i / kCount & 1)) break;
      } else if (warp == kIssuer + 2 && elected()) {
        int sent = 0;
        for (; sent < count; ++sent) {
            const int f = sent % S::kAhead;
            if (!(ok = barrier_wait(used(f), (sent / S::kAhead & 1) ^ 1))) break;
            barrier_expect(fetched(f), S::kCodes);
            copy_box(codes + f * S::kCodes, &codes_map, half, static_cast<int>(row0) + sent * kDepth, fetched(f));
        }
        for (int i = max(0, sent - S::kAhead); i < sent; ++i)
            if (!barrier_wait(fetched(i % S::kAhead), i / S::kAhead & 1)) break;
      }
    }
    if (!ok) stalled = 1;
    __syncwarp();
    __syncthreads();
    cluster_sync();  // the other CTA is done with this one's memory too
    if (warp == kIssuer) tensor_free<2 * kN>(tensor);
}

// dweight = scale times the sum of the splits' partial sums, in their order.
__global__ void __launch_bounds__(256)
relay_weight_grad_join_kernel(const float* partial, int64_t split_stride, int splits, int outputs, int inputs,
                              const float* column_scale, int64_t column_scale_stride, float* dweight,
                              int64_t worker_stride, int64_t row_stride) {
    const int k = blockIdx.x * 256 + threadIdx.x, worker = blockIdx.z;
    if (k >= inputs) return;
    const float scale = column_scale == nullptr ? 1.0f : column_scale[worker * column_scale_stride + k];
    for (int o = blockIdx.y; o < outputs; o += gridDim.y) {
        const float* p = partial + (static_cast<int64_t>(worker) * outputs + o) * inputs + k;
        float s = p[0];
        for (int i = 1; i < splits; ++i) s += p[i * split_stride];
        dweight[worker * worker_stride + o * row_stride + k] = s * scale;
    }
}

// ---------------------------------------------------------------- launching

// Tiles of 256 outputs x `wide` inputs.
int64_t tile_count(int64_t n, int64_t outputs, int64_t inputs, int wide) {
    return n * ((outputs + 2 * kM - 1) / (2 * kM)) * ((inputs + wide - 1) / wide);
}

// Inputs of a tile: 256, or 128 where those would leave SMs idle.
int tile_inputs(int64_t n, int64_t outputs, int64_t inputs) {
    return tile_count(n, outputs, inputs, 256) >= kSms / 2 ? 256 : 128;
}

// Splits of the tokens: as many as there are pairs of SMs for, of at least 8 stages each.
int token_splits(int64_t n, int64_t tokens, int64_t outputs, int64_t inputs) {
    const int64_t tiles = tile_count(n, outputs, inputs, tile_inputs(n, outputs, inputs));
    const int64_t room = kSms / 2 / tiles, most = tokens / (8 * kDepth);
    const int64_t s = room < most ? room : most;
    return s > 1 ? static_cast<int>(s) : 1;
}

using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                            const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                            CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's cuTensorMapEncodeTiled, NULL where it has none.
Encode encoder() {
    static const Encode encode = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) !=
                cudaSuccess ||
            found != cudaDriverEntryPointSuccess) {
            (void)cudaGetLastError();
            f = nullptr;
        }
        return reinterpret_cast<Encode>(f);
    }();
    return encode;
}

// The map of dy for 64 x 64 boxes; false where TMA cannot take its rows.
bool map_rows(CUtensorMap* map, const View<const __nv_bfloat16>& dy, int32_t n, int64_t tokens, int64_t outputs) {
    if (tokens == 0 || (tokens > 1 && dy.ts < outputs) || (n > 1 && dy.ws < outputs)) return false;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(outputs), static_cast<cuuint64_t>(tokens),
                                static_cast<cuuint64_t>(n)};
    // an axis of one row or one worker is never walked: any stride will do
    const cuuint64_t row = tokens > 1 ? static_cast<cuuint64_t>(dy.ts) * 2 : (outputs * 2 + 15) / 16 * 16;
    const cuuint64_t strides[2] = {row, n > 1 ? static_cast<cuuint64_t>(dy.ws) * 2 : row};
    const cuuint32_t box[3] = {64, kDepth, 1}, steps[3] = {1, 1, 1};
    return encoder()(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<__nv_bfloat16*>(dy.p), dims, strides, box,
                     steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                     CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The map of the codes for boxes of 64 tokens x `wide` inputs.
bool map_codes(CUtensorMap* map, const int8_t* codes, int64_t rows, int64_t pitch, int wide) {
    if (rows == 0) return true;  // nothing is copied
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(pitch), static_cast<cuuint64_t>(rows)};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(pitch)};
    const cuuint32_t box[2] = {static_cast<cuuint32_t>(wide), kDepth}, steps[2] = {1, 1};
    return encoder()(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<int8_t*>(codes), dims, strides, box, steps,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Lets Kernel use its shared memory, once per device.
template <auto Kernel>
bool allow_shared(int bytes) {
    static std::atomic<bool> set[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return false;
    if (dev < 64 && set[dev].load()) return true;
    if (cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) {
        (void)cudaGetLastError();
        return false;
    }
    if (dev < 64) set[dev].store(true);
    return true;
}

template <typename T, bool kTma, int kN>
int launch(const WeightGradArgs<T>& a, const CUtensorMap& dy_map, cudaStream_t stream) {
    constexpr auto kernel = relay_weight_grad_kernel<T, kTma, kN>;
    constexpr int kShared = Stages<T, kN>::kShared;
    if (!allow_shared<kernel>(kShared)) return RELAY_ECUDA;
    CUtensorMap codes_map = {};
    if (!map_codes(&codes_map, a.codes, static_cast<int64_t>(a.n) * a.tokens, a.pitch, kN / 2)) return RELAY_ECUDA;
    const dim3 grid(static_cast<unsigned>((a.outputs + 2 * kM - 1) / (2 * kM) * 2),
                    static_cast<unsigned>((a.inputs + kN - 1) / kN), static_cast<unsigned>(a.n * a.splits));
    kernel<<<grid, kThreads, kShared, stream>>>(a, dy_map, codes_map);
    return status_of_launch();
}

}  // namespace

extern "C" {

int64_t relay_weight_grad_workspace(int32_t n, int64_t tokens, int64_t outputs, int64_t inputs) {
    if (const int rc = check_shape(RELAY_FP32, n, tokens, inputs)) return rc;
    if (const int rc = check_shape(RELAY_FP32, n, tokens, outputs)) return rc;
    if (inputs > RELAY_WEIGHT_GRAD_MAX_INPUTS) return RELAY_EUNSUPPORTED;
    const int splits = token_splits(n, tokens, outputs, inputs);
    return splits > 1 ? 4 * splits * n * outputs * inputs : 0;
}

int relay_weight_grad(int32_t type, int32_t n, int64_t tokens, int64_t outputs, int64_t inputs, const relay_rows* dy,
                      const int8_t* codes, const uint8_t* scales, const float* column_scale,
                      int64_t column_scale_stride, const int32_t* lengths, float* dweight, int64_t worker_stride,
                      int64_t row_stride, void* workspace, int64_t workspace_bytes, relay_stream_t stream) {
    if (const int rc = check_shape(type, n, tokens, inputs)) return rc;
    const int64_t need = relay_weight_grad_workspace(n, tokens, outputs, inputs);
    if (need < 0) return static_cast<int>(need);
    if (!rows_fit(dy, type, n, tokens, outputs, false) || !checkpoint_fits(codes, scales, tokens)) return RELAY_EINVAL;
    if (!aligned(column_scale, 4) || (column_scale != nullptr && column_scale_stride < 0) || !aligned(lengths, 4))
        return RELAY_EINVAL;
    const relay_rows out{dweight, worker_stride, row_stride};
    if (!rows_fit(&out, RELAY_FP32, n, outputs, inputs, true)) return RELAY_EINVAL;
    if (workspace_bytes < need || (need > 0 && (workspace == nullptr || !aligned(workspace, 16)))) return RELAY_EINVAL;
    if (encoder() == nullptr) return RELAY_ECUDA;
    const int splits = token_splits(n, tokens, outputs, inputs);
    float* partial = static_cast<float*>(workspace);
    const int64_t plane = outputs * inputs;
    const auto run = [&](auto t) {
        using T = decltype(t);
        const View<const T> rows = view<const T>(dy, n, tokens);
        const WeightGradArgs<T> a{rows, outputs % 8 == 0 && vectors(dy, type, n, tokens), codes, scales, column_scale,
                                  n > 1 ? column_scale_stride : 0, lengths, splits > 1 ? partial : dweight,
                                  splits > 1 ? plane : n > 1 ? worker_stride : 0,
                                  splits > 1 ? inputs : outputs > 1 ? row_stride : 0, splits > 1 ? n * plane : 0, n,
                                  static_cast<int32_t>(tokens), static_cast<int32_t>(outputs),
                                  static_cast<int32_t>(inputs), static_cast<int32_t>(pitch_of(inputs)), splits};
        CUtensorMap map = {};
        const bool wide = tile_inputs(n, outputs, inputs) == 256;
        if constexpr (sizeof(T) == 2 && kTerms<T> == 1) {
            if (vectors(dy, type, n, tokens) && map_rows(&map, rows, n, tokens, outputs))
                return wide ? launch<T, true, 256>(a, map, stream) : launch<T, true, 128>(a, map, stream);
        }
        return wide ? launch<T, false, 256>(a, map, stream) : launch<T, false, 128>(a, map, stream);
    };
    const int rc =
        type == RELAY_BF16 ? run(__nv_bfloat16()) : type == RELAY_FP16 ? run(__half()) : run(float());
    if (rc != RELAY_OK || splits == 1) return rc;
    const dim3 grid(static_cast<unsigned>((inputs + 255) / 256),
                    static_cast<unsigned>(outputs < 65535 ? outputs : 65535), static_cast<unsigned>(n));
    relay_weight_grad_join_kernel<<<grid, 256, 0, stream>>>(
        partial, n * plane, splits, static_cast<int>(outputs), static_cast<int>(inputs), column_scale,
        n > 1 ? column_scale_stride : 0, dweight, n > 1 ? worker_stride : 0, outputs > 1 ? row_stride : 0);
    return status_of_launch();
}

}  // extern "C"
