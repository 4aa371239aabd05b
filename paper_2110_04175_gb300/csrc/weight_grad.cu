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
//   - dy comes by TMA, as bf16.  fp16 and fp32 rows (and bf16 rows that TMA cannot
//     take) are written to the workspace first as bf16 terms that add up to them
//     exactly, 8 bits each: 2 for fp16, 3 for fp32, one product each.  (bf16 ends at
//     2^-133, so what fp32 numbers below 2^-110 have below that is left out.)
//
// A pair of CTAs makes a tile of 256 outputs x kN inputs (cta_group::2): each
// brings half of both operands, so that a code is recalled once for 256 outputs.
//
// The tensor cores cut off what an addition shifts out, so that a long sum in
// their accumulator drifts towards zero: 6.3e-6 of the result after 384 additions.
// So they sum 32 or 36 additions at a time, in one of two accumulators, while
// other warps add the other one to registers, rounded to the nearest: 4e-7 against
// 64 bits at 8192 tokens.
//
// Measured: 2 x [8192 tokens, 8192 outputs, 4096 inputs], 1.1 TFLOP, takes 0.70 ms in bf16 on
// its own (1570 TFLOP/s, 0.81 of what a library product of 8192^3 does in a burst), 1.44 ms in
// fp16 and 2.07 ms in fp32; back to back, when power holds the clock, 0.77, 1.56 and 2.24 ms.
// A stage of 64 tokens takes a pair 620 cycles where its products take 512: shared memory
// carries 80 KB per SM and stage.  Where tokens are few, the results' way to memory bounds it
// (16 x [2 tokens, 3114, 4416]: 218 us, 4.0 TB/s).
#include "blackwell.cuh"
#include "layers.cuh"

namespace {

constexpr int kM = 128;        // outputs of a CTA
constexpr int kDepth = 64;     // tokens of a stage
// Warps: 0 .. 7 add up the sums and write them to memory, 8 .. 11 issue products and
// copies (one of them is idle), 12 .. 23 write stages: three teams of 4 take them in
// turn, so that one team's waits are the others' work (two teams: 6 % slower).
constexpr int kAdders = 8, kIssuer = 8, kMaker = 12, kTeam = 4, kTeams = 3;
constexpr int kThreads = 32 * (kMaker + kTeam * kTeams);
// 6 warpgroups are launched with 80 registers a thread: 2 x 144 + 48 + 3 x 48 = 6 x 80
// (in tiles of 256 inputs, whose adders hold 128 sums, 118 bytes a thread go to local memory)
constexpr int kAdderRegisters = 144, kIssuerRegisters = 48, kMakerRegisters = 48;
constexpr int kPanel = kDepth * 128;  // bytes of 64 outputs or inputs x kDepth tokens
constexpr int kSms = 152;

// Stages that the tensor cores sum before the sums are added up in registers.
template <int kTerms>
constexpr int kGroup = kTerms == 1 ? 8 : kTerms == 2 ? 4 : 3;

// An adder's 32 rows x 32 columns on their way to memory, rows 144 bytes apart: whole
// lines of 128 bytes a row (16 columns at a time took 268 us for 16 x [3114][4416] results
// where this takes 213).  After them its columns' scales.
constexpr int kTurnRow = 36, kTurnTile = 32 * kTurnRow * 4, kTurn = kTurnTile + 128 * 4;

template <int kTerms, int kN>
struct Stages {  // in a CTA
    static constexpr int kLeft = kTerms * kM / 64 * kPanel, kBytes = kLeft + kN / 2 / 64 * kPanel;
    // stages of codes, as they lie in memory: they come well before they are needed
    static constexpr int kCodes = kN / 2 * kDepth;
    static constexpr int kRoom = 232448 - 1024 - 512 - kAdders * kTurn;  // less alignment, barriers
    static constexpr int kMost = (kRoom - 4 * kCodes) / kBytes, kCount = kMost < 4 ? kMost : 4;
    static constexpr int kFit = (kRoom - kCount * kBytes) / kCodes, kAhead = kFit < 8 ? kFit : 8;
    static constexpr int kShared = kCount * kBytes + kAhead * kCodes + kAdders * kTurn + 1024 + 512;
    static_assert(kShared <= 232448, "shared memory of a CTA");
    // Teams at work: no more than stages.  A wait for a phase passes too when the barrier is
    // two phases behind, so a team that meets stage i has to know that stage i - 2 kCount was
    // freed.  With as many stages as teams it has met the same barrier before.  With more
    // (kAsk) it has met that of stage i - kTeamsIn, whose freeing says nothing of another's
    // arrival: the codes of stage i are copied only when the role that copies dy, which waits
    // for every stage, has found stage i - kCount free, and a team waits for its codes first.
    // A wait for codes is safe where the team knows that stage i - kAhead got its own: that
    // stage was the team's, or is not after stage i - kTeamsIn - kCount, which the team has
    // seen freed (without kAsk: not after stage i - kCount).
    static constexpr int kTeamsIn = kCount < kTeams ? kCount : kTeams;
    static constexpr bool kAsk = kTeamsIn < kCount;
    static_assert(kCount >= 2 && kTeamsIn <= kCount && kAhead >= kCount, "phases of the barriers");
    static_assert(!kAsk || kAhead % kTeamsIn == 0 || kAhead >= kTeamsIn + kCount, "phases of the codes' barriers");
};

struct WeightGradArgs {
    const int8_t* codes;
    const uint8_t* scales;
    const float* column_scale;
    int64_t column_scale_stride;
    const int32_t* lengths;
    float* out;  // dweight, or with several splits the partial sums [split][n][outputs][inputs]
    int64_t worker_stride, row_stride, split_stride;
    bool out_quads;  // rows of `out` can be written 16 bytes at a time
    int32_t n, tokens, outputs, inputs, pitch, splits;
    int32_t tiles_o, tiles_k;  // of a worker and split: 256 outputs, kN inputs
    int32_t tiles;             // of all
};

// One tile of the work and the stages of tokens that it sums.
struct Tile {
    int o0, k0, worker, split, length, first, count;

    // Tiles are taken in bands of 8 x 256 outputs, so that those in work at a time share
    // rows of both operands.
    __device__ __forceinline__ Tile(const WeightGradArgs& a, int tile, int wide) {
        const int plane = a.tiles_o * a.tiles_k, z = tile / plane, at = tile - z * plane;
        const int band = at / (8 * a.tiles_k), in = at - band * 8 * a.tiles_k;
        const int rows = min(8, a.tiles_o - 8 * band);
        o0 = (8 * band + in % rows) * 2 * kM;
        k0 = in / rows * wide;
        worker = z / a.splits;
        split = z - worker * a.splits;
        length = a.lengths == nullptr ? a.tokens : min(max(a.lengths[worker], 0), a.tokens);
        const int all = (length + kDepth - 1) / kDepth, each = (all + a.splits - 1) / a.splits;
        first = min(split * each, all);
        count = min(first + each, all) - first;
    }
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

__device__ __forceinline__ float4 get_shared(uint32_t at) {
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at));
    return v;
}

__device__ __forceinline__ uint32_t bits(__nv_bfloat162 v) { return *reinterpret_cast<uint32_t*>(&v); }
__device__ __forceinline__ __nv_bfloat162 pair(uint32_t v) { return *reinterpret_cast<__nv_bfloat162*>(&v); }

// The bytes 0 and 2 of w as codes, times `unit` (twice the same bf16).  A byte b stands
// for (b & 127) - (b & 128); under the exponent of 128 the two parts are the bf16
// values 128 + (b & 127) and 128 + (b & 128), whose difference is exact.
__device__ __forceinline__ uint32_t recall_pair(uint32_t w, uint32_t unit) {
    const uint32_t low = (w & 0x007f007fu) | 0x43004300u, sign = (w & 0x00800080u) | 0x43004300u;
    return bits(__hmul2(__hsub2(pair(low), pair(sign)), pair(unit)));
}

// Inputs lie in the operand in the order 0 2 1 3 of each four, which is how two bytes
// of a word come to the halves of another; the sums are put back in order on their
// way to memory.
__device__ __forceinline__ uint4 recall(uint2 q, uint32_t unit) {
    return make_uint4(recall_pair(q.x, unit), recall_pair(q.x >> 8, unit), recall_pair(q.y, unit),
                      recall_pair(q.y >> 8, unit));
}

// The first stage of `team` from number `base` of all on, counted from there.
template <int kTeamsIn>
__device__ __forceinline__ int first_stage(int team, int base) {
    return (team + kTeamsIn - base % kTeamsIn) % kTeamsIn;
}

// A warp's part of a stage of kWide inputs of xhat: a lane recalls 8 codes of a
// token per pass.
template <int kWide, int kTeamsIn>
struct Recall {
    static constexpr int kLanes = kWide / 8;                         // lanes of a token
    static constexpr int kRows = 32 / kLanes;                        // tokens of a pass
    static constexpr int kPasses = kDepth / (kRows * kTeam);
    static constexpr int kTokens = kRows * kPasses;                  // of the warp
    static_assert(kTokens * kTeam == kDepth && kTokens <= 32 && kWide <= 128, "a lane per token's scales");

    static constexpr int kScaled = 32 / kTokens;                     // of the team's stages: those whose scales a load brings

    // The stage's token that sub-row `sub` of the warp has in pass r.
    static __device__ __forceinline__ int token(int warp, int r, int sub) { return (r * kTeam + warp) * kRows + sub; }

    // Lane l's word of scales is that of the warp's token l % kTokens (in the order of
    // passes) of the team's stage l / kTokens; warp: in the team.
    static __device__ __forceinline__ int scale_token(int warp, int lane) {
        const int i = lane % kTokens;
        return lane / kTokens * (kTeamsIn * kDepth) + token(warp, i / kRows, i % kRows);
    }
    static __device__ __forceinline__ uint32_t scales(const uint8_t* at) {
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
            put_shared(put + r * (kTeam * kRows * 128), recall(q[r], u[r]));
    }
};

// dy as bf16 terms [n][kTerms][tokens][width], width = outputs rounded up to a multiple
// of 8: each term is what is left with all but 8 bits cut off, so that the terms add up
// exactly (down to bf16's 2^-133).  Rows that do not count are 0.
template <typename T, int kTerms, Way kWay>
__global__ void __launch_bounds__(256)
relay_weight_grad_terms_kernel(View<const T> dy, const int32_t* lengths, __nv_bfloat16* to, int n, int tokens,
                               int outputs, int width) {
    const int lane = threadIdx.x % 32, strips = (outputs + kStrip - 1) / kStrip;
    const int64_t all = static_cast<int64_t>(n) * tokens * strips;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 8 + threadIdx.x / 32; i < all; i += static_cast<int64_t>(gridDim.x) * 8) {
        const int64_t row = i / strips;
        const int base = static_cast<int>(i - row * strips) * kStrip, worker = static_cast<int>(row / tokens);
        const int token = static_cast<int>(row - static_cast<int64_t>(worker) * tokens);
        float v[8];
        load_strip<kWay>(dy.row(worker, token) + base, lane,
                         lengths == nullptr || token < lengths[worker] ? outputs - base : 0, v);
#pragma unroll
        for (int term = 0; term < kTerms; ++term) {
            float high[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                high[k] = __uint_as_float(__float_as_uint(v[k]) & 0xffff0000u);
                if ((__float_as_uint(v[k]) & 0x7f800000u) == 0x7f800000u) {  // infinity or NaN: all in the first term
                    high[k] = v[k];
                    v[k] = 0.0f;
                } else {
                    v[k] -= high[k];
                }
            }
            store_strip<kWay>(to + ((static_cast<int64_t>(worker) * kTerms + term) * tokens + token) * width + base, lane,
                              width - base, high);
        }
    }
}

// ----------------------------------------------------------------- the kernel

// Pairs of CTAs take tiles of 256 outputs x kN inputs (of a worker, of a split of the
// tokens) one after the other: the next one's products run while the last one's sums
// go to memory.  A wait that runs out ends a pair's work, and its results from there
// on are NaN.
template <int kTerms, int kN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
relay_weight_grad_kernel(const __grid_constant__ WeightGradArgs a, const __grid_constant__ CUtensorMap dy_map,
                         const __grid_constant__ CUtensorMap codes_map) {
    using S = Stages<kTerms, kN>;
    constexpr int kCount = S::kCount;
    extern __shared__ uint8_t raw[];
    const uint32_t stages = (shared_address(raw) + 1023u) & ~1023u;
    const uint32_t codes = stages + kCount * S::kBytes, turns = codes + S::kAhead * S::kCodes;
    const uint32_t bars = turns + kAdders * kTurn;
    // per stage: full (of codes recalled, of dy; on CTA 0 of the other CTA's half too) and free
    // again; per accumulator: summed by the tensor cores, and read; per stage of codes: there, and used
    const auto full = [&](int s) { return bars + 8 * s; };
    const auto freed = [&](int s) { return bars + 8 * (kCount + s); };
    const auto summed = [&](int b) { return bars + 8 * (2 * kCount + b); };
    const auto read = [&](int b) { return bars + 8 * (2 * kCount + 2 + b); };
    const auto fetched = [&](int s) { return bars + 8 * (2 * kCount + 4 + s); };
    const auto used = [&](int s) { return bars + 8 * (2 * kCount + 4 + S::kAhead + s); };
    const uint32_t tensor_at = bars + 8 * (2 * kCount + 4 + 2 * S::kAhead);
    const uint32_t passed = tensor_at + 4;  // how many stages the copies of dy have found free

    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x / 32), 0), lane = threadIdx.x % 32;
    const int rank = static_cast<int>(cluster_rank());
    const int pair = blockIdx.x / 2, pairs = gridDim.x / 2;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kCount; ++s) {
            barrier_init(full(s), kTeam + 1 + (rank == 0 ? 1 : 0));
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
        count_store(passed, 0);
        barriers_ready();
    }
    if (warp == kIssuer) tensor_alloc<2 * kN>(tensor_at);
    tensor_fence_before();
    __syncthreads();
    cluster_sync();
    tensor_fence_after();
    uint32_t tensor;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(tensor) : "r"(tensor_at));

    if (warp < kAdders) {
        more_registers<kAdderRegisters>();
        constexpr int kColumns = kN / 2;
        const int row = 32 * (warp % 4), column = kColumns * (warp / 4);  // of the CTA's 128 x kN
        const uint32_t turn = turns + warp * kTurn;
        bool ok = true;
        int group = 0;  // of all that the pair has summed
        for (int tile = pair; tile < a.tiles; tile += pairs) {
            const Tile at(a, tile, kN);
            const int64_t o = at.o0 + kM * rank + row;  // this warp's first output and input
            const int k0 = at.k0 + column;
            for (int e = lane; e < kColumns; e += 32) {
                float m = 1.0f;
                if (a.column_scale != nullptr && a.splits == 1 && k0 + e < a.inputs)
                    m = a.column_scale[at.worker * a.column_scale_stride + k0 + e];
                asm volatile("st.shared.f32 [%0], %1;" ::"r"(turn + kTurnTile + 4 * e), "f"(m) : "memory");
            }
            float sum[kColumns] = {};
            for (int done = 0; done < at.count && ok; done += kGroup<kTerms>, ++group) {
                const int b = group & 1;
                if (!(ok = barrier_wait_warp(summed(b), group >> 1 & 1))) break;
                tensor_fence_after();
                const uint32_t from = tensor + (static_cast<uint32_t>(row) << 16) + b * kN + column;
#pragma unroll
                for (int c = 0; c < kColumns; c += 16) {
                    float v[16];
                    tensor_load(from + c, v);
#pragma unroll
                    for (int e = 0; e < 16; ++e) sum[c + e] += v[e];
                }
                tensor_fence_before();
                __syncwarp();
                if (lane == 0) barrier_arrive(read(b));
            }
            if (!ok) {
#pragma unroll
                for (int e = 0; e < kColumns; ++e) sum[e] = __int_as_float(0x7fffffff);
            }
            // through shared memory, so that a warp writes whole lines of each row
            float* out = a.out + at.split * a.split_stride + at.worker * a.worker_stride;
#pragma unroll
            for (int c = 0; c < kColumns; c += 32) {
                if (k0 + c >= a.inputs) break;
#pragma unroll
                for (int e = 0; e < 32; e += 4)
                    put_shared(turn + lane * (4 * kTurnRow) + 4 * e,
                               make_uint4(__float_as_uint(sum[c + e]), __float_as_uint(sum[c + e + 2]),
                                          __float_as_uint(sum[c + e + 1]), __float_as_uint(sum[c + e + 3])));
                __syncwarp();
                if (a.out_quads) {
                    const int k = k0 + c + 4 * (lane % 8);
                    const float4 m = get_shared(turn + kTurnTile + 4 * c + 16 * (lane % 8));
                    float* to = out + (o + lane / 8) * a.row_stride + k;
#pragma unroll
                    for (int r = lane / 8; r < 32; r += 4, to += 4 * a.row_stride) {
                        float4 v = get_shared(turn + r * (4 * kTurnRow) + 16 * (lane % 8));
                        v.x *= m.x, v.y *= m.y, v.z *= m.z, v.w *= m.w;
                        if (o + r < a.outputs && k < a.inputs) *reinterpret_cast<float4*>(to) = v;
                    }
                } else {
                    const int k = k0 + c + lane;
                    float m, v;
                    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(m) : "r"(turn + kTurnTile + 4 * (c + lane)));
                    float* to = out + o * a.row_stride + k;
#pragma unroll 8
                    for (int r = 0; r < 32; ++r, to += a.row_stride) {
                        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(turn + r * (4 * kTurnRow) + 4 * lane));
                        if (o + r < a.outputs && k < a.inputs) *to = v * m;
                    }
                }
                __syncwarp();
            }
        }
    } else if (warp < kMaker) {
        fewer_registers<kIssuerRegisters>();
        if (warp == kIssuer) {
            int i = 0, group = 0;  // of all that the pair has summed
            bool ok = true;
            for (int tile = pair; tile < a.tiles && ok; tile += pairs) {
                const Tile at(a, tile, kN);
                for (int n = 0; n < at.count; ++n, ++i) {
                    const int s = i % kCount, place = n % kGroup<kTerms>, b = group & 1;
                    const uint32_t left = stages + s * S::kBytes;
                    if (place == 0 && group > 1 && !(ok = barrier_wait_warp(read(b), (group >> 1 & 1) ^ 1))) break;
                    if (!(ok = barrier_wait_warp(full(s), i / kCount & 1))) break;
                    const int from = at.length - (at.first + n) * kDepth;
                    if (kTerms == 1 && from < kDepth) {  // the copy brought the rows past the length too, whatever they hold
                        for (int e = from * 8 + lane; e < kDepth * 8; e += 32)
                            for (int p = 0; p < kM / 64; ++p)
                                put_shared(left + p * kPanel + e * 16, make_uint4(0, 0, 0, 0));
                        fence_async();
                        __syncwarp();
                    }
                    const bool last = place == kGroup<kTerms> - 1 || n == at.count - 1;
                    if (rank != 0) {
                        if (elected()) barrier_arrive_there(in_cta(full(s), 0));
                    } else {
                        tensor_fence_after();
                        if (elected()) {
                            const uint64_t dy = operand(left, kPanel, 1024), xhat = operand(left + S::kLeft, kPanel, 1024);
#pragma unroll
                            for (int term = 0; term < kTerms; ++term)
#pragma unroll
                                for (int k = 0; k < kDepth / 16; ++k)  // addresses count 16 bytes
                                    product(tensor + b * kN, dy + (term * (kM / 64 * kPanel) + k * 2048) / 16,
                                            xhat + k * 2048 / 16, kProductKind<2 * kM, kN>, place + term + k > 0);
                            products_arrive(freed(s));
                            if (last) products_arrive(summed(b));
                        }
                        __syncwarp();
                    }
                    if (last) ++group;
                }
            }
        } else if (warp == kIssuer + 1 && elected()) {
            int i = 0;
            bool ok = true;
            for (int tile = pair; tile < a.tiles && ok; tile += pairs) {
                const Tile at(a, tile, kN);
                for (int n = 0; n < at.count; ++n, ++i) {
                    const int s = i % kCount;
                    if (!(ok = barrier_wait(freed(s), (i / kCount & 1) ^ 1))) break;
                    if (S::kAsk) count_store(passed, i + 1);
                    barrier_expect(full(s), S::kLeft);
                    for (int p = 0; p < S::kLeft / kPanel; ++p)
                        copy_box(stages + s * S::kBytes + p * kPanel, &dy_map, at.o0 + kM * rank + 64 * (p % (kM / 64)),
                                 (at.first + n) * kDepth, at.worker * kTerms + p / (kM / 64), full(s));
                }
            }
            // nothing is left in flight: no copy, and no arrival that the last stages' products
            // still send to this CTA
            for (int j = max(0, i - kCount); j < i; ++j)
                if (!barrier_wait(full(j % kCount), j / kCount & 1) || !barrier_wait(freed(j % kCount), j / kCount & 1))
                    break;
        } else if (warp == kIssuer + 2 && elected()) {
            int i = 0;
            bool ok = true;
            for (int tile = pair; tile < a.tiles && ok; tile += pairs) {
                const Tile at(a, tile, kN);
                const int row0 = at.worker * a.tokens + at.first * kDepth, half = at.k0 + kN / 2 * rank;
                for (int n = 0; n < at.count; ++n, ++i) {
                    const int f = i % S::kAhead;
                    if (!(ok = barrier_wait(used(f), (i / S::kAhead & 1) ^ 1))) break;
                    if (S::kAsk && !(ok = count_wait(passed, i - kCount + 1))) break;
                    barrier_expect(fetched(f), S::kCodes);
                    copy_box(codes + f * S::kCodes, &codes_map, half, row0 + n * kDepth, fetched(f));
                }
            }
            for (int j = max(0, i - S::kAhead); j < i; ++j)
                if (!barrier_wait(fetched(j % S::kAhead), j / S::kAhead & 1)) break;
        }
    } else {
        fewer_registers<kMakerRegisters>();
        using R = Recall<kN / 2, S::kTeamsIn>;
        const int team = (warp - kMaker) / kTeam, member = warp % kTeam;
        // The scales come one load of R::kScaled stages ahead, across tiles: `ahead` is where the
        // lane's next word is, `ahead_left` how many of the tile's tokens there are from its
        // stage on, `ahead_stages` how many stages.
        const int mine = R::scale_token(member, lane);
        const int64_t stride = int64_t(S::kTeamsIn) * R::kScaled * kDepth * (a.pitch / kBlock);
        const uint8_t* ahead = nullptr;
        int ahead_tile = pair - pairs, ahead_left = 0, ahead_stages = 0, ahead_base = 0, ahead_count = 0;
        uint32_t now = 0, next = 0;
        bool ok = true, odd = false;
        const auto load_next = [&] {
            while (ahead_stages <= 0) {
                ahead_tile += pairs;
                if (ahead_tile >= a.tiles) return 0u;
                const Tile at(a, ahead_tile, kN);
                ahead_base += ahead_count;
                ahead_count = at.count;
                const int n = first_stage<S::kTeamsIn>(team, ahead_base), k = at.k0 + kN / 2 * rank, t = (at.first + n) * kDepth;
                ahead_stages = at.count - n;
                ahead_left = k < a.pitch ? at.length - t : 0;
                ahead = a.scales + (static_cast<int64_t>(at.worker) * a.tokens + t + mine) * (a.pitch / kBlock) + k / kBlock;
            }
            const uint32_t w = mine < ahead_left ? R::scales(ahead) : 0x07070707u;
            ahead += stride;
            ahead_left -= S::kTeamsIn * R::kScaled * kDepth;
            ahead_stages -= S::kTeamsIn * R::kScaled;
            return w;
        };
        int base = 0;
        if (team < S::kTeamsIn) next = load_next();
        for (int tile = pair; tile < a.tiles && ok && team < S::kTeamsIn; tile += pairs) {
            const Tile at(a, tile, kN);
            int turn = 0;
            for (int n = first_stage<S::kTeamsIn>(team, base); n < at.count; n += S::kTeamsIn) {
                const int i = base + n, s = i % kCount, f = i % S::kAhead, left = at.length - (at.first + n) * kDepth;
                if (turn == 0) {
                    odd = __any_sync(0xffffffffu, __vcmpeq4(next, 0xffffffffu) != 0u);
                    now = __vmaxu4(next, 0x07070707u) - 0x06060606u;
                    next = load_next();
                }
                if (S::kAsk && !(ok = barrier_wait_warp(fetched(f), i / S::kAhead & 1))) break;
                if (!(ok = barrier_wait_warp(freed(s), (i / kCount & 1) ^ 1))) break;
                if (!S::kAsk && !(ok = barrier_wait_warp(fetched(f), i / S::kAhead & 1))) break;
                R::make(codes + f * S::kCodes, stages + s * S::kBytes + S::kLeft, now, odd, turn, left, member, lane);
                fence_async();
                __syncwarp();
                if (lane == 0) {
                    barrier_arrive(full(s));
                    barrier_arrive(used(f));
                }
                turn = turn == R::kScaled - 1 ? 0 : turn + 1;
            }
            base += at.count;
        }
    }
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

// How the work is cut: inputs of a tile, and splits of the tokens.
struct Cut {
    int wide, splits;
};

// No more splits than fill the pairs twice, of at least 4 stages each.
int64_t most_splits(int64_t tiles, int64_t stages) {
    const int64_t fill = (kSms + tiles - 1) / tiles, deep = stages / 4;
    const int64_t most = fill < deep ? fill : deep;
    return most > 1 ? most : 1;
}

// The cut that should take the least time, by what was measured.  A stage of a 256 x 256
// tile takes a pair 0.35 us with one term of dy and 0.36 us a term with more, one of
// 256 x 128 0.215 us and 0.185 us a term; a tile besides 6.7 and 3.5 us (its results' way
// to memory); splits a launch and the partial sums' way to memory and back.  Of 22 cuts
// tried by hand the choice was within 6 % of the best but once, 14 % (4 x [2048 tokens, 2048 outputs,
// 2048 inputs]: bf16 68 us in 256 and 76 us in 128, fp32 164 and 151 us;
// [8192, 512, 512]: bf16 53 us in one piece and 15 us in splits).
Cut best_cut(int terms, int64_t n, int64_t tokens, int64_t outputs, int64_t inputs) {
    const int64_t stages = (tokens + kDepth - 1) / kDepth, pairs = kSms / 2;
    const double results = 4e-6 / 5.0 * static_cast<double>(n * outputs * inputs);  // us at 5 TB/s
    Cut best{256, 1};
    double least = 0.0;
    for (const int wide : {256, 128}) {
        const int64_t tiles = tile_count(n, outputs, inputs, wide);
        const double stage = wide == 256 ? (terms == 1 ? 0.35 : 0.36 * terms) : (terms == 1 ? 0.215 : 0.185 * terms);
        const double tile = wide == 256 ? 6.7 : 3.5;
        for (int64_t splits = 1; splits <= most_splits(tiles, stages); ++splits) {
            const double rounds = static_cast<double>((tiles * splits + pairs - 1) / pairs);
            double us = rounds * (tile + stage * static_cast<double>((stages + splits - 1) / splits));
            if (splits > 1) us += 5.0 + results * static_cast<double>(2 * splits + 1);
            if ((wide == 256 && splits == 1) || us < least) least = us, best = Cut{wide, static_cast<int>(splits)};
        }
    }
    return best;
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

// The map of bf16 rows [planes][tokens][outputs] for boxes of 64 x 64.
bool map_rows(CUtensorMap* map, const void* rows, int64_t planes, int64_t tokens, int64_t outputs,
              int64_t plane_bytes, int64_t row_bytes) {
    if (tokens == 0) return true;  // nothing is copied
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(outputs), static_cast<cuuint64_t>(tokens),
                                static_cast<cuuint64_t>(planes)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(row_bytes), static_cast<cuuint64_t>(plane_bytes)};
    const cuuint32_t box[3] = {64, kDepth, 1}, steps[3] = {1, 1, 1};
    return encoder()(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(rows), dims, strides, box, steps,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Whether TMA takes the rows as they are: bf16, 16-byte steps, no row read twice.
bool direct(int32_t type, const relay_rows* dy, int32_t n, int64_t tokens, int64_t outputs) {
    constexpr int64_t kMost = int64_t(1) << 38;  // elements: a map's strides end at 2^40 bytes
    return type == RELAY_BF16 && dy != nullptr && vectors(dy, type, n, tokens) &&
           (tokens <= 1 || (dy->token_stride >= outputs && dy->token_stride < kMost)) &&
           (n == 1 || (dy->worker_stride >= outputs && dy->worker_stride < kMost));
}

int terms_of(int32_t type) { return type == RELAY_BF16 ? 1 : type == RELAY_FP16 ? 2 : 3; }
int64_t width_of(int64_t outputs) { return (outputs + 7) / 8 * 8; }

// Bytes of the workspace's two parts: dy's terms, and the splits' partial sums.
int64_t terms_bytes(int32_t type, const relay_rows* dy, int32_t n, int64_t tokens, int64_t outputs) {
    if (direct(type, dy, n, tokens, outputs)) return 0;
    return 2 * terms_of(type) * n * tokens * width_of(outputs);
}
int64_t partial_bytes(int64_t splits, int32_t n, int64_t outputs, int64_t inputs) {
    return splits > 1 ? 4 * splits * n * outputs * inputs : 0;
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

template <int kTerms, int kN>
int launch(WeightGradArgs a, const CUtensorMap& dy_map, cudaStream_t stream) {
    constexpr auto kernel = relay_weight_grad_kernel<kTerms, kN>;
    constexpr int kShared = Stages<kTerms, kN>::kShared;
    if (!allow_shared<kernel>(kShared)) return RELAY_ECUDA;
    CUtensorMap codes_map = {};
    if (!map_codes(&codes_map, a.codes, static_cast<int64_t>(a.n) * a.tokens, a.pitch, kN / 2)) return RELAY_ECUDA;
    const int64_t tiles = tile_count(a.n, a.outputs, a.inputs, kN) * a.splits;
    if (tiles > INT32_MAX - kSms) return RELAY_EUNSUPPORTED;
    a.tiles_o = (a.outputs + 2 * kM - 1) / (2 * kM);
    a.tiles_k = (a.inputs + kN - 1) / kN;
    a.tiles = static_cast<int32_t>(tiles);
    const int pairs = tiles < kSms / 2 ? static_cast<int>(tiles) : kSms / 2;
    kernel<<<2 * pairs, kThreads, kShared, stream>>>(a, dy_map, codes_map);
    return status_of_launch();
}

template <int kTerms>
int launch(const WeightGradArgs& a, const CUtensorMap& dy_map, int wide, cudaStream_t stream) {
    return wide == 256 ? launch<kTerms, 256>(a, dy_map, stream) : launch<kTerms, 128>(a, dy_map, stream);
}

template <typename T, int kTerms>
int write_terms(const relay_rows* dy, int32_t type, const int32_t* lengths, void* to, int32_t n, int64_t tokens,
                int64_t outputs, cudaStream_t stream) {
    const int64_t warps = n * tokens * ((outputs + kStrip - 1) / kStrip), most = 16 * kSms;
    const int ctas = static_cast<int>((warps + 7) / 8 < most ? (warps + 7) / 8 : most);
    const bool vec = outputs % 8 == 0 && vectors(dy, type, n, tokens);
    (vec ? relay_weight_grad_terms_kernel<T, kTerms, kVector> : relay_weight_grad_terms_kernel<T, kTerms, kDirect>)
        <<<ctas, 256, 0, stream>>>(view<const T>(dy, n, tokens), lengths, static_cast<__nv_bfloat16*>(to), n,
                                   static_cast<int>(tokens), static_cast<int>(outputs),
                                   static_cast<int>(width_of(outputs)));
    return status_of_launch();
}

}  // namespace

extern "C" {

int64_t relay_weight_grad_workspace(int32_t type, int32_t n, int64_t tokens, int64_t outputs, int64_t inputs,
                                    const relay_rows* dy) {
    if (const int rc = check_shape(type, n, tokens, inputs)) return rc;
    if (const int rc = check_shape(type, n, tokens, outputs)) return rc;
    if (inputs > RELAY_WEIGHT_GRAD_MAX_INPUTS) return RELAY_EUNSUPPORTED;
    // without dy, the most splits that any type and any smaller number of tokens may take
    const int64_t splits = dy == nullptr
                               ? most_splits(tile_count(n, outputs, inputs, 256), (tokens + kDepth - 1) / kDepth)
                               : best_cut(terms_of(type), n, tokens, outputs, inputs).splits;
    return terms_bytes(type, dy, n, tokens, outputs) + partial_bytes(splits, n, outputs, inputs);
}

int relay_weight_grad(int32_t type, int32_t n, int64_t tokens, int64_t outputs, int64_t inputs, const relay_rows* dy,
                      const int8_t* codes, const uint8_t* scales, const float* column_scale,
                      int64_t column_scale_stride, const int32_t* lengths, float* dweight, int64_t worker_stride,
                      int64_t row_stride, void* workspace, int64_t workspace_bytes, relay_stream_t stream) {
    if (const int rc = check_shape(type, n, tokens, inputs)) return rc;
    const int64_t need = relay_weight_grad_workspace(type, n, tokens, outputs, inputs, dy);
    if (need < 0) return static_cast<int>(need);
    if (!rows_fit(dy, type, n, tokens, outputs, false) || !checkpoint_fits(codes, scales, tokens)) return RELAY_EINVAL;
    if (!aligned(column_scale, 4) || (column_scale != nullptr && column_scale_stride < 0) || !aligned(lengths, 4))
        return RELAY_EINVAL;
    const relay_rows out{dweight, worker_stride, row_stride};
    if (!rows_fit(&out, RELAY_FP32, n, outputs, inputs, true)) return RELAY_EINVAL;
    if (workspace_bytes < need || (need > 0 && (workspace == nullptr || !aligned(workspace, 16)))) return RELAY_EINVAL;
    if (encoder() == nullptr) return RELAY_ECUDA;

    const int terms = terms_of(type);
    const Cut cut = best_cut(terms, n, tokens, outputs, inputs);
    const int64_t terms_size = terms_bytes(type, dy, n, tokens, outputs), plane = outputs * inputs;
    CUtensorMap map = {};
    if (terms_size == 0) {
        // an axis of one row or one worker is never walked: any stride will do
        const int64_t row = tokens > 1 ? dy->token_stride * 2 : width_of(outputs) * 2;
        if (!map_rows(&map, dy->data, n, tokens, outputs, n > 1 ? dy->worker_stride * 2 : row, row)) return RELAY_ECUDA;
    } else {
        const int64_t row = width_of(outputs) * 2;
        if (!map_rows(&map, workspace, n * terms, tokens, outputs, tokens * row, row)) return RELAY_ECUDA;
        const int rc = type == RELAY_BF16
                           ? write_terms<__nv_bfloat16, 1>(dy, type, lengths, workspace, n, tokens, outputs, stream)
                       : type == RELAY_FP16 ? write_terms<__half, 2>(dy, type, lengths, workspace, n, tokens, outputs, stream)
                                            : write_terms<float, 3>(dy, type, lengths, workspace, n, tokens, outputs, stream);
        if (rc != RELAY_OK) return rc;
    }
    float* partial = reinterpret_cast<float*>(static_cast<char*>(workspace) + terms_size);
    const bool split = cut.splits > 1;
    WeightGradArgs a{};
    a.codes = codes;
    a.scales = scales;
    a.column_scale = column_scale;
    a.column_scale_stride = n > 1 ? column_scale_stride : 0;
    a.lengths = lengths;
    a.out = split ? partial : dweight;
    a.worker_stride = split ? plane : n > 1 ? worker_stride : 0;
    a.row_stride = split ? inputs : outputs > 1 ? row_stride : 0;
    a.split_stride = split ? n * plane : 0;
    a.out_quads = inputs % 4 == 0 && aligned(a.out, 16) && a.worker_stride % 4 == 0 && a.row_stride % 4 == 0;
    a.n = n;
    a.tokens = static_cast<int32_t>(tokens);
    a.outputs = static_cast<int32_t>(outputs);
    a.inputs = static_cast<int32_t>(inputs);
    a.pitch = static_cast<int32_t>(pitch_of(inputs));
    a.splits = cut.splits;
    const int rc = terms == 1   ? launch<1>(a, map, cut.wide, stream)
                   : terms == 2 ? launch<2>(a, map, cut.wide, stream)
                                : launch<3>(a, map, cut.wide, stream);
    if (rc != RELAY_OK || !split) return rc;
    const dim3 grid(static_cast<unsigned>((inputs + 255) / 256),
                    static_cast<unsigned>(outputs < 65535 ? outputs : 65535), static_cast<unsigned>(n));
    relay_weight_grad_join_kernel<<<grid, 256, 0, stream>>>(
        partial, n * plane, cut.splits, static_cast<int>(outputs), static_cast<int>(inputs), column_scale,
        a.column_scale_stride, dweight, n > 1 ? worker_stride : 0, outputs > 1 ? row_stride : 0);
    return status_of_launch();
}

}  // extern "C"
