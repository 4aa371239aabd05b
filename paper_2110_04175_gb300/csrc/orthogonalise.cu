// orthogonalise.cu -- an update made orthogonal by Newton-Schulz steps (relay_orthogonalise
// of relaylayers.h) on GB300 (sm_103a):
//
//   x = u / (|u| + eps);  a step: g = x x^T,  x <- a x + (b g + c g g) x
//
// with the coefficients of the Muon optimiser (K. Jordan and others, 2024) and x as wide as it is
// high or wider (u or its transpose).  Three products a step, on the
// tensor cores, bound by them where matrices are large and by the way from product to product
// where they are small.
//
// A step multiplies small singular values by 3.4, five of them by 480, and what an operand
// is rounded by with them: bf16 operands would leave 1 % of noise.  So every operand is
// held as two fp16 terms, hi + lo, 22 to 23 bits, and a product is three of theirs (lo lo is
// below what an fp32 sum keeps).  Singular values stay within 1.21, b g + c g g within 2.9,
// and operands are held times 2^12: the terms of an element of 2^-10 still have all their
// bits, and nothing reaches fp16's 65504.
//
// A pair of CTAs makes a tile of 256 x kN (cta_group::2), each brings half of both operands
// by TMA; small matrices get tiles of one CTA, and those of up to 128 rows a whole step a launch.
// x x^T and g g are symmetric: tiles above the diagonal are copies.  The tensor
// cores cut off what an addition shifts out, so sums leave them every one to three stages for
// registers of other warps, as in the weight gradient.  Errors against 64 bits are 0.5 to 1.1
// times those of the same steps in plain fp32 (0.6 where k is thousands).
//
// Measured: 4 x [2048][8192] 4.4 ms on its own, 2.2 TFLOP as a count of the symmetric halves, 6.7
// in fp16 products (1530 TFLOP/s, 0.79 of what a library product of 8192^3 does in a burst), 4.8 to 4.9 back to
// back, when power holds the clock; 3 x [1537][1001] 344 us; 8 x [128][256] 52 us.
#include <cuda_fp16.h>

#include "blackwell.cuh"
#include "layers.cuh"

namespace {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kHeld = 4096.0f;  // operands are held times this

constexpr int kM = 128, kDepth = 64;  // rows of a CTA, and what a stage goes along the summed axis
constexpr int kAdders = 8, kIssuer = 8, kLoader = 9, kThreads = 32 * 12;
constexpr int kTurn = 32 * 128;  // bytes of an adder's 32 rows on their way from or to memory
// tiles of 256 columns: 3 warpgroups are launched with 168 registers a thread, 2 x 224 + 56 = 3 x 168
constexpr int kAdderRegisters = 224, kOtherRegisters = 56;
constexpr int kSms = 152;

// A kernel's shape: tiles of 128 kCtas x kN.
template <int kCtas_, int kN_>
struct Shape {
    static constexpr int kCtas = kCtas_, kN = kN_, kHigh = kM * kCtas;
    static constexpr int kRight = kN / kCtas;  // columns that a CTA brings
    static constexpr int kLeftTerm = kM * 128, kRightTerm = kRight * 128;  // bytes of a term of a stage
    static constexpr int kBytes = 2 * (kLeftTerm + kRightTerm);
    static constexpr int kFit = (232448 - 1024 - 256 - kAdders * kTurn) / kBytes, kCount = kFit < 4 ? kFit : 4;  // stages
    static constexpr int kShared = kCount * kBytes + kAdders * kTurn + 1024 + 256;
    static_assert(kCount >= 2 && kShared <= 232448 && kHigh % kN == 0, "shape of the tiles");
};

struct ProductArgs {
    const __half* c;  // what is added, times beta: [n][2][rows][pitch], or NULL
    __half* out;      // the same shape, or NULL, and
    float* final;     // fp32: element (i, j) at i row_stride + j column_stride
    int64_t worker_stride, row_stride, column_stride;
    float alpha, beta, scale;  // scale: of `final`
    int32_t n, rows, columns, depth, pitch;
    int32_t tiles_m, tiles_n, tiles;
    int32_t group;  // stages that the tensor cores sum
};

// The tile's place; kFlip: all tiles, otherwise those on and below the diagonal.
template <typename S, bool kFlip>
struct Tile {
    int worker, row, column;
    bool mirror;
    __device__ __forceinline__ Tile(const ProductArgs& a, int tile) {
        const int plane = a.tiles / a.n;
        worker = tile / plane;
        int at = tile - worker * plane, i, j;
        if (kFlip) {  // bands of 4 rows, so that those in work at a time share operands
            const int band = at / (4 * a.tiles_n), in = at - band * 4 * a.tiles_n, high = min(4, a.tiles_m - 4 * band);
            i = 4 * band + in % high;
            j = in / high;
            mirror = false;
        } else {
            constexpr int kWide = S::kHigh / S::kN;  // tiles across a diagonal block
            for (i = 0;; ++i) {
                const int across = min(kWide * (i + 1), a.tiles_n);
                if (at < across) break;
                at -= across;
            }
            j = at;
            mirror = j < kWide * i;
        }
        row = i * S::kHigh;
        column = j * S::kN;
    }
};

// Operand in shared memory whose fastest axis is K, 64 of it in rows of 128 bytes, in the
// 128-byte swizzle: groups of 8 rows are 1024 bytes apart.
__device__ __forceinline__ uint64_t operand_k(uint32_t at) {
    return static_cast<uint64_t>((at & 0x3FFFFu) >> 4) | uint64_t(1) << 16 | uint64_t(1024 >> 4) << 32 | uint64_t(1) << 46 |
           uint64_t(2) << 61;
}

// fp16 x fp16 to fp32; kFlip: the right operand has N fastest.
template <typename S, bool kFlip>
constexpr uint32_t kKind = 1u << 4 | uint32_t(kFlip) << 16 | uint32_t(S::kN / 8) << 17 | uint32_t(S::kHigh / 16) << 24;

// v as two terms, each rounded to fp16.
__device__ __forceinline__ void split(float v, __half& hi, __half& lo) {
    hi = __float2half_rn(v);
    lo = __float2half_rn(v - __half2float(hi));
}

// An adder's 32 rows of 128 bytes in shared memory, 16-byte pieces swizzled by the row: a lane has
// a row, memory is read and written row by row.  (With every lane at a row of its own in memory
// an access was 32 lines: 10 to 15 us a tile.)
struct Turn {
    uint32_t at;
    __device__ __forceinline__ uint32_t piece(int row, int q) const { return at + row * 128 + ((q ^ (row & 7)) << 4); }
    __device__ __forceinline__ void put(int row, int q, uint4 v) const {
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(piece(row, q)), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
    }
    __device__ __forceinline__ uint4 get(int row, int q) const {
        uint4 v;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(piece(row, q)) : "memory");
        return v;
    }
    __device__ __forceinline__ float number(int row, int k) const {  // fp32 number k of the row
        float v;
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(piece(row, k / 4) + k % 4 * 4) : "memory");
        return v;
    }
};

// What an adder's 32 rows x kColumns are, one row a lane, and the way between them and memory.  `rows`
// and `columns`: how many there are from the first on.

// Memory's order: kPieces lanes a row; whether piece p of a lane is there.
template <int kPieces>
__device__ __forceinline__ bool piece_of(int p, int lane, int rows, int columns, int& r, int& q) {
    r = (p * 32 + lane) / kPieces, q = (p * 32 + lane) % kPieces;
    return r < rows && 8 * q < columns;
}

template <int kColumns>
constexpr int kChunkOf = kColumns < 64 ? kColumns : 64;  // columns that go through `turn` together

// sum = start (hi + lo) of what lies at c and c + plane.
template <int kColumns>
__device__ __forceinline__ void bring_added(float (&sum)[kColumns], const Turn& turn, const __half* c, int64_t plane, int pitch,
                                            int rows, int columns, float start, int lane) {
    constexpr int kChunk = kChunkOf<kColumns>, kPieces = kChunk / 8;
#pragma unroll
    for (int j = 0; j < kColumns; j += kChunk) {
        uint4 part[2][kPieces];
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            int r, q;
            const bool there = piece_of<kPieces>(p, lane, rows, columns - j, r, q);
#pragma unroll
            for (int t = 0; t < 2; ++t)
                part[t][p] = there ? *reinterpret_cast<const uint4*>(c + t * plane + static_cast<int64_t>(r) * pitch + j + 8 * q)
                                   : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            __syncwarp();
#pragma unroll
            for (int p = 0; p < kPieces; ++p) turn.put((p * 32 + lane) / kPieces, (p * 32 + lane) % kPieces, part[t][p]);
            __syncwarp();
#pragma unroll
            for (int q = 0; q < kPieces; ++q) {
                const uint4 v = turn.get(lane, q);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float& to = sum[j + 8 * q + e];
                    const float part_of = __half2float(reinterpret_cast<const __half*>(&v)[e]);
                    to = t == 0 ? part_of : start * (to + part_of);
                }
            }
        }
    }
}

// 8 numbers as the term `t` of two.
__device__ __forceinline__ uint4 term_of(const float* v, int t) {
    uint4 w;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        __half hi, lo;
        split(v[e], hi, lo);
        reinterpret_cast<__half*>(&w)[e] = t == 0 ? hi : lo;
    }
    return w;
}

// The terms of `sum` to out and out + plane; `mirror`: their place above the diagonal, at the lane's
// row, or NULL.
template <int kColumns>
__device__ __forceinline__ void put_terms(const float (&sum)[kColumns], const Turn& turn, __half* out, int64_t plane, int pitch,
                                          int rows, int columns, __half* mirror, int lane) {
    constexpr int kChunk = kChunkOf<kColumns>, kPieces = kChunk / 8;
#pragma unroll
    for (int j = 0; j < kColumns; j += kChunk) {
        if (j >= columns) break;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            __syncwarp();
#pragma unroll
            for (int q = 0; q < kPieces; ++q) {
                const uint4 v = term_of(sum + j + 8 * q, t);
                turn.put(lane, q, v);
                if (mirror != nullptr && lane < rows) {
                    __half* over = mirror + t * plane + static_cast<int64_t>(j + 8 * q) * pitch;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (j + 8 * q + e < columns) over[e * pitch] = reinterpret_cast<const __half*>(&v)[e];
                }
            }
            __syncwarp();
#pragma unroll
            for (int p = 0; p < kPieces; ++p) {
                int r, q;
                if (piece_of<kPieces>(p, lane, rows, columns - j, r, q))
                    *reinterpret_cast<uint4*>(out + t * plane + static_cast<int64_t>(r) * pitch + j + 8 * q) = turn.get(r, q);
            }
        }
    }
}

// `sum` in fp32: element (i, j) at to + i row_stride + j column_stride, one of them 1.
template <int kColumns>
__device__ __forceinline__ void put_final(const float (&sum)[kColumns], const Turn& turn, float* to, int64_t row_stride,
                                          int64_t column_stride, int rows, int columns, int lane) {
    if (column_stride == 1) {
#pragma unroll
        for (int j = 0; j < kColumns; j += 32) {
            if (j >= columns) break;
            __syncwarp();
#pragma unroll
            for (int q = 0; q < 8; ++q)
                turn.put(lane, q, make_uint4(__float_as_uint(sum[j + 4 * q]), __float_as_uint(sum[j + 4 * q + 1]),
                                             __float_as_uint(sum[j + 4 * q + 2]), __float_as_uint(sum[j + 4 * q + 3])));
            __syncwarp();
            if (j + lane < columns)
#pragma unroll 8
                for (int r = 0; r < min(32, rows); ++r) to[r * row_stride + j + lane] = turn.number(r, lane);
        }
    } else if (lane < rows) {
#pragma unroll
        for (int j = 0; j < kColumns; ++j)
            if (j < columns) to[lane * row_stride + j * column_stride] = sum[j];
    }
}

// Adds an accumulator's part to the warp's sums.
template <int kColumns>
__device__ __forceinline__ void add_accumulator(float (&sum)[kColumns], uint32_t from) {
#pragma unroll
    for (int c = 0; c < kColumns; c += 16) {
        float v[16];
        tensor_load(from + c, v);
#pragma unroll
        for (int e = 0; e < 16; ++e) sum[c + e] += v[e];
    }
}

// out = alpha (left right) + beta c.  left [n][2][rows][depth]; right [n][2][columns][depth], or with kFlip
// [n][2][depth][columns].  A wait that runs out ends a pair's work, and its results from there on are
// NaN.
template <typename S, bool kFlip>
__global__ void __launch_bounds__(kThreads, 1)
relay_orthogonalise_kernel(const __grid_constant__ ProductArgs a, const __grid_constant__ CUtensorMap left_map,
                           const __grid_constant__ CUtensorMap right_map) {
    constexpr int kCtas = S::kCtas, kN = S::kN, kCount = S::kCount;
    extern __shared__ uint8_t raw[];
    const uint32_t stages = (shared_address(raw) + 1023u) & ~1023u;
    const uint32_t turns = stages + kCount * S::kBytes, bars = turns + kAdders * kTurn;
    // per stage: full (on CTA 0 of the other CTA's half too) and free again; per accumulator:
    // summed by the tensor cores, and read
    const auto full = [&](int s) { return bars + 8 * s; };
    const auto freed = [&](int s) { return bars + 8 * (kCount + s); };
    const auto summed = [&](int b) { return bars + 8 * (2 * kCount + b); };
    const auto read = [&](int b) { return bars + 8 * (2 * kCount + 2 + b); };
    const uint32_t tensor_at = bars + 8 * (2 * kCount + 4);

    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x / 32), 0), lane = threadIdx.x % 32;
    const int rank = kCtas == 2 ? static_cast<int>(cluster_rank()) : 0;
    const int pair = blockIdx.x / kCtas, pairs = gridDim.x / kCtas;
    const int count = (a.depth + kDepth - 1) / kDepth;  // stages of a tile

    if (threadIdx.x == 0) {
        for (int s = 0; s < kCount; ++s) {
            barrier_init(full(s), kCtas == 2 && rank == 0 ? 2 : 1);
            barrier_init(freed(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            barrier_init(summed(b), 1);
            barrier_init(read(b), kAdders);
        }
        barriers_ready();
    }
    if (warp == kIssuer) tensor_alloc<2 * kN, kCtas>(tensor_at);
    tensor_fence_before();
    __syncthreads();
    if (kCtas == 2) cluster_sync();
    tensor_fence_after();
    uint32_t tensor;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(tensor) : "r"(tensor_at));
    let_next_start();
    wait_for_previous();

    if (warp < kAdders) {
        if constexpr (kN == 256) more_registers<kAdderRegisters>();
        constexpr int kColumns = kN / 2;
        const int row = 32 * (warp % 4), column = kColumns * (warp / 4);  // of the CTA's 128 x kN
        const int64_t plane = static_cast<int64_t>(a.rows) * a.pitch;
        const Turn turn{turns + static_cast<uint32_t>(warp) * kTurn};
        bool ok = true;
        int group = 0;  // of all that the pair has summed
        for (int tile = pair; tile < a.tiles; tile += pairs) {
            const Tile<S, kFlip> at(a, tile);
            const int i0 = at.row + kM * rank + row, j0 = at.column + column, rows = a.rows - i0, columns = a.columns - j0;
            const int64_t first = static_cast<int64_t>(at.worker) * 2 * plane, base = first + static_cast<int64_t>(i0) * a.pitch + j0;
            // beta c is where the sum starts, so that it comes while the tensor cores are at work
            float sum[kColumns] = {};
            if (a.c != nullptr) bring_added(sum, turn, a.c + base, plane, a.pitch, rows, columns, a.beta / a.alpha, lane);
            for (int done = 0; done < count && ok; done += a.group, ++group) {
                const int b = group & 1;
                if (!(ok = barrier_wait_warp(summed(b), group >> 1 & 1))) break;
                tensor_fence_after();
                add_accumulator(sum, tensor + (static_cast<uint32_t>(row) << 16) + b * kN + column);
                tensor_fence_before();
                __syncwarp();
                if (lane == 0) barrier_arrive(read(b));
            }
            const float factor = !ok ? __int_as_float(0x7fffffff) : a.out != nullptr ? a.alpha : a.scale;
#pragma unroll
            for (int e = 0; e < kColumns; ++e) sum[e] *= factor;
            if (a.out != nullptr)
                put_terms(sum, turn, a.out + base, plane, a.pitch, rows, columns,
                          !kFlip && at.mirror ? a.out + first + static_cast<int64_t>(j0) * a.pitch + i0 + lane : nullptr, lane);
            else
                put_final(sum, turn, a.final + at.worker * a.worker_stride + i0 * a.row_stride + j0 * a.column_stride, a.row_stride,
                          a.column_stride, rows, columns, lane);
        }
    } else {
        if constexpr (kN == 256) fewer_registers<kOtherRegisters>();
        if (warp == kIssuer) {
            int i = 0, group = 0;  // of all that the pair has summed
            bool ok = true;
            for (int tile = pair; tile < a.tiles && ok; tile += pairs) {
                for (int n = 0; n < count; ++n, ++i) {
                    const int s = i % kCount, place = n % a.group, b = group & 1;
                    if (place == 0 && group > 1 && !(ok = barrier_wait_warp(read(b), (group >> 1 & 1) ^ 1))) break;
                    if (!(ok = barrier_wait_warp(full(s), i / kCount & 1))) break;
                    const bool last = place == a.group - 1 || n == count - 1;
                    if (rank != 0) {
                        if (elected()) barrier_arrive_there(in_cta(full(s), 0));
                    } else {
                        tensor_fence_after();
                        if (elected()) {
                            const uint32_t l = stages + s * S::kBytes, r = l + 2 * S::kLeftTerm;
                            constexpr uint32_t kNext = kFlip ? 16 * 128 / 16 : 2;  // 16 of K, in 16 bytes
    #pragma unroll
                            for (int t = 0; t < 3; ++t)  // lo hi, hi lo, hi hi: the small ones first
    #pragma unroll
                                for (int k = 0; k < kDepth / 16; ++k) {
                                    const uint32_t at_r = r + (t == 1 ? S::kRightTerm : 0);
                                    const uint64_t x = operand_k(l + (t == 0 ? S::kLeftTerm : 0)) + 2 * k;
                                    const uint64_t y = (kFlip ? operand(at_r, kDepth * 128, 1024) : operand_k(at_r)) + kNext * k;
                                    product<kCtas>(tensor + b * kN, x, y, kKind<S, kFlip>, place + k + t > 0);
                                }
                            products_arrive<kCtas>(freed(s));
                            if (last) products_arrive<kCtas>(summed(b));
                        }
                        __syncwarp();
                    }
                    if (last) ++group;
                }
            }
        } else if (warp == kLoader && elected()) {
            int i = 0;
            bool ok = true;
            for (int tile = pair; tile < a.tiles && ok; tile += pairs) {
                const Tile<S, kFlip> at(a, tile);
                for (int n = 0; n < count; ++n, ++i) {
                    const int s = i % kCount, k = n * kDepth;
                    if (!(ok = barrier_wait(freed(s), (i / kCount & 1) ^ 1))) break;
                    barrier_expect(full(s), S::kBytes);
                    const uint32_t l = stages + s * S::kBytes, r = l + 2 * S::kLeftTerm;
                    const int column = at.column + S::kRight * rank;
    #pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        copy_box(l + t * S::kLeftTerm, &left_map, k, at.row + kM * rank, 2 * at.worker + t, full(s));
                        if (!kFlip)
                            copy_box(r + t * S::kRightTerm, &right_map, k, column, 2 * at.worker + t, full(s));
                        else
    #pragma unroll
                            for (int p = 0; p < S::kRight / 64; ++p)
                                copy_box(r + t * S::kRightTerm + p * kDepth * 128, &right_map, column + 64 * p, k,
                                         2 * at.worker + t, full(s));
                    }
                }
            }
            // nothing is left in flight: no copy, and no arrival that the last stages' products still send to this CTA
            for (int j = max(0, i - kCount); j < i; ++j)
                if (!barrier_wait(full(j % kCount), j / kCount & 1) || !barrier_wait(freed(j % kCount), j / kCount & 1)) break;
        }
    }
    __syncwarp();
    __syncthreads();
    if (kCtas == 2) cluster_sync();  // the other CTA is done with this one's memory too
    if (warp == kIssuer) tensor_free<2 * kN, kCtas>(tensor);
}

// ------------------------------------------------------------------ a whole step
//
// Matrices of up to 128 rows: g is one tile, so each CTA makes it for itself, and b g + c g g from
// it without leaving the SM (the adders write both as operands to shared memory), and then its
// columns of x.  One launch a step instead of three, while the CTAs of all matrices run at once.

template <int kN>
struct Whole {
    static constexpr int kTerm = kM * 128, kStage = 2 * kTerm, kSlice = 2 * kN * 128;  // bytes: of 64 along the summed axis
    static constexpr int kCount = 4, kOperand = 4 * kTerm;  // stages; b g + c g g: two terms of two panels of 64 columns
    static constexpr int kShared = kCount * kStage + kOperand + kAdders * kTurn + 1024 + 256;
    static_assert(kSlice <= kStage && kShared <= 232448, "shared memory of a CTA");
};

struct StepArgs {
    const __half* x;  // [n][2][rows][pitch]
    __half* out;      // the same shape, or NULL, and
    float* final;     // as in ProductArgs
    int64_t worker_stride, row_stride, column_stride;
    float scale;
    int32_t rows, columns, pitch, slices;
};

template <int kN>
__global__ void __launch_bounds__(kThreads, 1)
relay_orthogonalise_step_kernel(const __grid_constant__ StepArgs a, const __grid_constant__ CUtensorMap rows_map,
                                const __grid_constant__ CUtensorMap slice_map) {
    using W = Whole<kN>;
    constexpr int kCount = W::kCount;
    constexpr uint32_t kSquare = 1u << 4 | uint32_t(128 / 8) << 17 | uint32_t(kM / 16) << 24;
    constexpr uint32_t kLast = 1u << 4 | 1u << 16 | uint32_t(kN / 8) << 17 | uint32_t(kM / 16) << 24;
    extern __shared__ uint8_t raw[];
    const uint32_t stages = (shared_address(raw) + 1023u) & ~1023u, operand_at = stages + kCount * W::kStage;
    const uint32_t turns = operand_at + W::kOperand, bars = turns + kAdders * kTurn;
    const auto full = [&](int s) { return bars + 8 * s; };
    const auto freed = [&](int s) { return bars + 8 * (kCount + s); };
    const auto summed = [&](int b) { return bars + 8 * (2 * kCount + b); };
    const auto read = [&](int b) { return bars + 8 * (2 * kCount + 2 + b); };
    const uint32_t ready = bars + 8 * (2 * kCount + 4), tensor_at = ready + 8;

    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x / 32), 0), lane = threadIdx.x % 32;
    const int worker = blockIdx.x / a.slices, slice = (blockIdx.x % a.slices) * kN;
    const int count = (a.columns + kDepth - 1) / kDepth, panels = (a.rows + kDepth - 1) / kDepth;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kCount; ++s) {
            barrier_init(full(s), 1);
            barrier_init(freed(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            barrier_init(summed(b), 1);
            barrier_init(read(b), kAdders);
        }
        barrier_init(ready, kAdders);
        barriers_ready();
    }
    if (warp == kIssuer) tensor_alloc<256, 1>(tensor_at);
    tensor_fence_before();
    __syncthreads();
    tensor_fence_after();
    uint32_t tensor;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(tensor) : "r"(tensor_at));
    let_next_start();
    wait_for_previous();

    if (warp < kAdders) {
        const int row = 32 * (warp % 4), half = warp / 4;
        const int64_t plane = static_cast<int64_t>(a.rows) * a.pitch;
        const Turn turn{turns + static_cast<uint32_t>(warp) * kTurn};
        bool ok = true;
        int group = 0;
        const auto sums = [&](auto& sum, int groups, int column) {
            for (int n = 0; n < groups && ok; ++n, ++group) {
                const int b = group & 1;
                if (!(ok = barrier_wait_warp(summed(b), group >> 1 & 1))) break;
                tensor_fence_after();
                add_accumulator(sum, tensor + (static_cast<uint32_t>(row) << 16) + b * 128 + column);
                tensor_fence_before();
                __syncwarp();
                if (lane == 0) barrier_arrive(read(b));
            }
        };
        // 64 columns of the lane's row as a panel of the operand
        const auto to_operand = [&](const float (&v)[64]) {
            const Turn panel{operand_at + half * W::kTerm};
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                panel.put(row + lane, q, term_of(v + 8 * q, 0));
                Turn{panel.at + 2 * W::kTerm}.put(row + lane, q, term_of(v + 8 * q, 1));
            }
            fence_async();
            __syncwarp();
            if (lane == 0) barrier_arrive(ready);
        };
        float g[64] = {};
        sums(g, count, 64 * half);
#pragma unroll
        for (int e = 0; e < 64; ++e) g[e] *= 1.0f / kHeld;
        to_operand(g);
#pragma unroll
        for (int e = 0; e < 64; ++e) g[e] *= kB * kHeld / kC;  // where the sum starts
        sums(g, panels, 64 * half);
#pragma unroll
        for (int e = 0; e < 64; ++e) g[e] *= kC / kHeld;
        to_operand(g);
        constexpr int kColumns = kN / 2;
        const int j0 = slice + kColumns * half, rows = a.rows - row, columns = a.columns - j0;
        const int64_t base = static_cast<int64_t>(worker) * 2 * plane + static_cast<int64_t>(row) * a.pitch + j0;
        float sum[kColumns];
        bring_added(sum, turn, a.x + base, plane, a.pitch, rows, columns, kA * kHeld, lane);
        sums(sum, panels, kColumns * half);
        const float factor = !ok ? __int_as_float(0x7fffffff) : a.out != nullptr ? 1.0f / kHeld : a.scale;
#pragma unroll
        for (int e = 0; e < kColumns; ++e) sum[e] *= factor;
        if (a.out != nullptr)
            put_terms(sum, turn, a.out + base, plane, a.pitch, rows, columns, static_cast<__half*>(nullptr), lane);
        else
            put_final(sum, turn, a.final + worker * a.worker_stride + row * a.row_stride + j0 * a.column_stride, a.row_stride,
                      a.column_stride, rows, columns, lane);
    } else if (warp == kIssuer) {
        int group = 0;
        bool ok = true;
        // one group: 64 along the summed axis, terms at `l` and l + lo_l, `r` and r + lo_r
        const auto multiply = [&](uint32_t l, uint32_t lo_l, uint32_t r, uint32_t lo_r, bool flip, int stage) {
            tensor_fence_after();
            if (elected()) {
#pragma unroll
                for (int t = 0; t < 3; ++t)  // lo hi, hi lo, hi hi: the small ones first
#pragma unroll
                    for (int k = 0; k < kDepth / 16; ++k) {
                        const uint32_t at_r = r + (t == 1 ? lo_r : 0);
                        const uint64_t x = operand_k(l + (t == 0 ? lo_l : 0)) + 2 * k;
                        const uint64_t y = flip ? operand(at_r, kDepth * 128, 1024) + 128 * k : operand_k(at_r) + 2 * k;
                        product<1>(tensor + (group & 1) * 128, x, y, flip ? kLast : kSquare, t + k > 0);
                    }
                if (stage >= 0) products_arrive<1>(freed(stage));
                products_arrive<1>(summed(group & 1));
            }
            __syncwarp();
            ++group;
        };
        const auto accumulator = [&] { return group <= 1 || barrier_wait_warp(read(group & 1), (group >> 1 & 1) ^ 1); };
        for (int i = 0; i < count && ok; ++i) {
            const uint32_t at = stages + i % kCount * W::kStage;
            if ((ok = accumulator() && barrier_wait_warp(full(i % kCount), i / kCount & 1))) multiply(at, W::kTerm, at, W::kTerm, false, i % kCount);
        }
        ok = ok && barrier_wait_warp(ready, 0);
        for (int p = 0; p < panels && ok; ++p) {
            const uint32_t at = operand_at + p * W::kTerm;
            if ((ok = accumulator())) multiply(at, 2 * W::kTerm, at, 2 * W::kTerm, false, -1);
        }
        ok = ok && barrier_wait_warp(ready, 1);
        for (int p = 0; p < panels && ok; ++p) {
            const int i = count + p, s = i % kCount;
            if ((ok = accumulator() && barrier_wait_warp(full(s), i / kCount & 1)))
                multiply(operand_at + p * W::kTerm, 2 * W::kTerm, stages + s * W::kStage, W::kSlice / 2, true, s);
        }
    } else if (warp == kLoader && elected()) {
        int i = 0;
        for (; i < count + panels; ++i) {
            const int s = i % kCount;
            const uint32_t at = stages + s * W::kStage;
            if (!barrier_wait(freed(s), (i / kCount & 1) ^ 1)) break;
            barrier_expect(full(s), i < count ? W::kStage : W::kSlice);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                if (i < count)
                    copy_box(at + t * W::kTerm, &rows_map, i * kDepth, 0, 2 * worker + t, full(s));
                else
#pragma unroll
                    for (int p = 0; p < kN / 64; ++p)
                        copy_box(at + t * (W::kSlice / 2) + p * kDepth * 128, &slice_map, slice + 64 * p, (i - count) * kDepth,
                                 2 * worker + t, full(s));
            }
        }
        // nothing is left in flight: no copy, and no arrival of the last products
        for (int j = max(0, i - kCount); j < i; ++j)
            if (!barrier_wait(full(j % kCount), j / kCount & 1) || !barrier_wait(freed(j % kCount), j / kCount & 1)) break;
    }
    __syncwarp();
    __syncthreads();
    if (warp == kIssuer) tensor_free<256, 1>(tensor);
}

// ------------------------------------------------------------------- the start

constexpr int kParts = 512;  // CTAs that sum a matrix's squares, at most

struct Update {
    const float* p;
    int64_t worker_stride, row_stride;
    int32_t rows, columns;
};

// sums[worker][part][3]: of the squares of values of middling size, of those above 2^40 times
// 2^-80 and of those below 2^-40 times 2^80, so that no sum leaves fp32.  (Values of one
// matrix rarely are of more than one kind.)
__global__ void __launch_bounds__(256) relay_orthogonalise_norm_kernel(Update u, float* sums) {
    __shared__ float shared[8][3];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, strips = (u.columns + kStrip - 1) / kStrip;
    const float* from = u.p + blockIdx.y * u.worker_stride;
    float s[3] = {};
    const int64_t all = static_cast<int64_t>(u.rows) * strips;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 8 + warp; i < all; i += static_cast<int64_t>(gridDim.x) * 8) {
        const int64_t row = i / strips;
        const int base = static_cast<int>(i - row * strips) * kStrip;
        float v[8], near = 0.0f;
        load_strip<kDirect>(from + row * u.row_stride + base, lane, u.columns - base, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float m = fabsf(v[k]);
            if (m > 0x1p40f)
                s[1] = fmaf(v[k] * 0x1p-80f, v[k] * 0x1p-80f, s[1]);
            else if (m < 0x1p-40f)
                s[2] = fmaf(v[k] * 0x1p80f, v[k] * 0x1p80f, s[2]);
            else
                near = fmaf(v[k], v[k], near);  // NaN too
        }
        s[0] += near;
    }
#pragma unroll
    for (int e = 0; e < 3; ++e) {
#pragma unroll
        for (int m = 16; m > 0; m >>= 1) s[e] += __shfl_xor_sync(0xffffffffu, s[e], m);
        if (lane == 0) shared[warp][e] = s[e];
    }
    __syncthreads();
    if (threadIdx.x < 3) {
        float t = 0.0f;
        for (int w = 0; w < 8; ++w) t += shared[w][threadIdx.x];
        sums[(static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x) * 3 + threadIdx.x] = t;
    }
}

// kHeld / (|u| + eps), called by all threads of a CTA; NaN where |u| is no number.  One warp adds
// the parts and one thread takes the root: 64-bit arithmetic is slow here (with every thread at
// it this took 180 us of a 268 MB start).
struct Factor {
    float lift, near;  // a power of two, 1 but where fp32 does not hold the factor (lengths below 2^-115)
    __device__ __forceinline__ float times(float v) const { return v * lift * near; }
};

__device__ Factor start_factor(const float* sums, int parts, float eps) {
    __shared__ Factor shared;
    if (threadIdx.x < 32) {
        double v = 0.0;
        for (int p = threadIdx.x; p < parts; p += 32) {
            const float* s = sums + (static_cast<int64_t>(blockIdx.y) * parts + p) * 3;
            v += s[0] + s[1] * 0x1p160 + s[2] * 0x1p-160;
        }
#pragma unroll
        for (int m = 16; m > 0; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
        if (threadIdx.x == 0) {
            const double length = sqrt(v), over = length + eps, f = over > 0.0 ? kHeld / over : 0.0;
            const double lift = f < 1e38 ? 1.0 : 0x1p64;
            shared = Factor{static_cast<float>(lift), length < 1e300 ? static_cast<float>(f / lift) : __int_as_float(0x7fffffff)};
        }
    }
    __syncthreads();
    return shared;
}

// x = u f as two terms, [n][2][rows][pitch]: a warp takes strips of 256 columns.
__global__ void __launch_bounds__(256)
relay_orthogonalise_start_kernel(Update u, const float* sums, int parts, float eps, __half* x, int pitch) {
    __shared__ __align__(16) float turns[8][kStrip];
    let_next_start();
    wait_for_previous();
    const Factor f = start_factor(sums, parts, eps);
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, strips = (u.columns + kStrip - 1) / kStrip;
    const float* from = u.p + blockIdx.y * u.worker_stride;
    const int64_t plane = static_cast<int64_t>(u.rows) * pitch, all = static_cast<int64_t>(u.rows) * strips;
    __half* to = x + static_cast<int64_t>(blockIdx.y) * 2 * plane;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 8 + warp; i < all; i += static_cast<int64_t>(gridDim.x) * 8) {
        const int64_t row = i / strips;
        const int base = static_cast<int>(i - row * strips) * kStrip;
        float v[8];
        load_strip<kDirect>(from + row * u.row_stride + base, lane, u.columns - base, v);
        to_octets(v, lane, turns[warp]);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = f.times(v[k]);
        store_strip<kVector>(to + row * pitch + base, lane, pitch - base, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] -= __half2float(__float2half_rn(v[k]));
        store_strip<kVector>(to + plane + row * pitch + base, lane, pitch - base, v);
    }
}

// The same of the transpose, x [n][2][columns][pitch]: a CTA takes squares of 64 x 64.
__global__ void __launch_bounds__(256)
relay_orthogonalise_turn_kernel(Update u, const float* sums, int parts, float eps, __half* x, int pitch) {
    __shared__ float square[64][65];
    let_next_start();
    wait_for_previous();
    const Factor f = start_factor(sums, parts, eps);
    const float* from = u.p + blockIdx.y * u.worker_stride;
    const int64_t plane = static_cast<int64_t>(u.columns) * pitch;
    __half* to = x + static_cast<int64_t>(blockIdx.y) * 2 * plane;
    const int across = (u.columns + 63) / 64, all = (u.rows + 63) / 64 * across, lead = threadIdx.x / 64, at = threadIdx.x % 64;
    for (int i = blockIdx.x; i < all; i += gridDim.x) {
        const int row = i / across * 64, column = i % across * 64;
        __syncthreads();
#pragma unroll 4
        for (int r = lead; r < 64; r += 4)
            square[r][at] = row + r < u.rows && column + at < u.columns ? from[(row + r) * u.row_stride + column + at] : 0.0f;
        __syncthreads();
#pragma unroll 4
        for (int c = lead; c < 64; c += 4) {
            if (column + c >= u.columns || row + at >= u.rows) continue;
            __half hi, lo;
            split(f.times(square[at][c]), hi, lo);
            __half* out = to + static_cast<int64_t>(column + c) * pitch + row + at;
            out[0] = hi, out[plane] = lo;
        }
    }
}

// ---------------------------------------------------------------- launching

int pitch_to(int64_t columns) { return static_cast<int>((columns + 15) / 16 * 16); }  // 32 bytes

// Two terms of n matrices for boxes of 64 columns x `high` rows.
bool map_terms(CUtensorMap* map, const __half* p, int64_t n, int64_t rows, int64_t columns, int high) {
    const cuuint64_t pitch = static_cast<cuuint64_t>(pitch_to(columns)) * 2;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(columns), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(2 * n)};
    const cuuint64_t strides[2] = {pitch, pitch * static_cast<cuuint64_t>(rows)};
    const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(high), 1}, steps[3] = {1, 1, 1};
    return encoder()(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<__half*>(p), dims, strides, box, steps,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Launches a kernel that starts before the one in front of it ends (wait_for_previous).
template <typename... Args, typename... Given>
int launch_early(void (*kernel)(Args...), dim3 grid, int threads, int shared, int cluster, cudaStream_t stream, Given... given) {
    cudaLaunchAttribute with[2] = {};
    with[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    with[0].val.programmaticStreamSerializationAllowed = 1;
    with[1].id = cudaLaunchAttributeClusterDimension;
    with[1].val.clusterDim.x = static_cast<unsigned>(cluster), with[1].val.clusterDim.y = 1, with[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t how = {};
    how.gridDim = grid, how.blockDim = dim3(static_cast<unsigned>(threads)), how.dynamicSmemBytes = static_cast<size_t>(shared);
    how.stream = stream, how.attrs = with, how.numAttrs = cluster > 1 ? 2 : 1;
    if (cudaLaunchKernelEx(&how, kernel, Args(given)...) == cudaSuccess) return RELAY_OK;
    (void)cudaGetLastError();
    return RELAY_ECUDA;
}

// Tiles of all matrices; kFlip: the whole, otherwise on and below the diagonal.
int64_t tile_count(int64_t n, int64_t rows, int64_t columns, int high, int wide, bool flip) {
    const int64_t down = (rows + high - 1) / high, across = (columns + wide - 1) / wide;
    if (flip) return n * down * across;
    int64_t tiles = 0;
    for (int64_t i = 0; i < down; ++i) tiles += high / wide * (i + 1) < across ? high / wide * (i + 1) : across;
    return n * tiles;
}

template <typename S, bool kFlip>
int launch(ProductArgs a, const __half* left, const __half* right, cudaStream_t stream) {
    constexpr auto kernel = relay_orthogonalise_kernel<S, kFlip>;
    if (!allow_shared<kernel>(S::kShared)) return RELAY_ECUDA;
    CUtensorMap left_map, right_map;
    if (!map_terms(&left_map, left, a.n, a.rows, a.depth, kM) ||
        !(kFlip ? map_terms(&right_map, right, a.n, a.depth, a.columns, kDepth)
                : map_terms(&right_map, right, a.n, a.columns, a.depth, S::kRight)))
        return RELAY_ECUDA;
    a.tiles_m = (a.rows + S::kHigh - 1) / S::kHigh;
    a.tiles_n = (a.columns + S::kN - 1) / S::kN;
    const int64_t tiles = tile_count(a.n, a.rows, a.columns, S::kHigh, S::kN, kFlip);
    if (tiles > INT32_MAX - kSms) return RELAY_EUNSUPPORTED;
    a.tiles = static_cast<int32_t>(tiles);
    const int64_t most = kSms / S::kCtas, pairs = tiles < most ? tiles : most;
    return launch_early(kernel, dim3(static_cast<unsigned>(S::kCtas * pairs)), kThreads, S::kShared, S::kCtas, stream, a, left_map,
                        right_map);
}

// The shape that should take the least time, by what was measured: rounds of tiles, each a
// time per stage and one for the tile.  Of three products at 15 sizes from [16][38] to
// 4 x [2048][8192] the choice is within 3 us of the best of the three shapes, or 5 %.
template <bool kFlip>
int launch(const ProductArgs& a, const __half* left, const __half* right, cudaStream_t stream) {
    const double stages = static_cast<double>((a.depth + kDepth - 1) / kDepth);
    const auto us = [&](int ctas, int wide, double stage, double tile) {
        const int64_t most = kSms / ctas;
        return static_cast<double>((tile_count(a.n, a.rows, a.columns, kM * ctas, wide, kFlip) + most - 1) / most) * (stage * stages + tile);
    };
    const double big = us(2, 256, 0.68, 9.0), middle = us(2, 128, 0.34, 5.0), small = us(1, 64, 0.48, 2.0);
    if (small <= middle && small <= big) return launch<Shape<1, 64>, kFlip>(a, left, right, stream);
    if (middle <= big) return launch<Shape<2, 128>, kFlip>(a, left, right, stream);
    return launch<Shape<2, 256>, kFlip>(a, left, right, stream);
}

template <int kN>
int launch_step(const StepArgs& a, int32_t n, cudaStream_t stream) {
    constexpr auto kernel = relay_orthogonalise_step_kernel<kN>;
    if (!allow_shared<kernel>(Whole<kN>::kShared)) return RELAY_ECUDA;
    CUtensorMap rows_map, slice_map;
    if (!map_terms(&rows_map, a.x, n, a.rows, a.columns, kM) || !map_terms(&slice_map, a.x, n, a.rows, a.columns, kDepth))
        return RELAY_ECUDA;
    return launch_early(kernel, dim3(static_cast<unsigned>(n * a.slices)), kThreads, Whole<kN>::kShared, 1, stream, a, rows_map, slice_map);
}

// Columns of a CTA where a step goes in one launch, 0 where it does not.
int whole_step(int64_t n, int64_t m, int64_t k) {
    if (m > kM) return 0;
    return n * ((k + 63) / 64) <= kSms ? 64 : n * ((k + 127) / 128) <= kSms ? 128 : 0;
}

// Stages that the tensor cores sum before the sums are added up in registers: 36 additions, or
// with one stage (its small products first) 4 of the large ones, where m is small: the
// cut is to one side and shows where sums are short otherwise.
int group_of(int64_t m) { return m <= 448 ? 1 : 3; }

// Where the workspace's parts begin, in bytes.
struct Parts {
    int64_t x, g, p, sums, size;
    Parts(int64_t n, int64_t m, int64_t k) {
        const int64_t wide = 4 * n * m * pitch_to(k), square = 4 * n * m * pitch_to(m);
        x = 0, g = 2 * wide, p = g + square, sums = p + square, size = sums + 12 * n * kParts;
    }
};

int check_matrices(int32_t n, int64_t rows, int64_t columns) {
    if (n < 1 || rows < 1 || columns < 1) return RELAY_EINVAL;
    if (n > RELAY_MAX_N || rows > RELAY_ORTHOGONALISE_MAX || columns > RELAY_ORTHOGONALISE_MAX) return RELAY_EUNSUPPORTED;
    return RELAY_OK;
}

int launch_start(const Update& u, bool tall, const float* sums, int parts, float eps, __half* x, int pitch, int32_t n,
                 cudaStream_t stream) {
    const int64_t ctas = tall ? ((u.rows + 63) / 64) * static_cast<int64_t>((u.columns + 63) / 64)
                              : (u.rows * static_cast<int64_t>((u.columns + kStrip - 1) / kStrip) + 7) / 8;
    const int64_t most = 8 * kSms > n ? 8 * kSms / n : 1;
    const dim3 grid(static_cast<unsigned>(ctas < most ? ctas : most), static_cast<unsigned>(n));
    return launch_early(tall ? relay_orthogonalise_turn_kernel : relay_orthogonalise_start_kernel, grid, 256, 0, 1,
                        stream, u, sums, parts, eps, x, pitch);
}

}  // namespace

extern "C" {

int64_t relay_orthogonalise_workspace(int32_t n, int64_t rows, int64_t columns) {
    if (const int rc = check_matrices(n, rows, columns)) return rc;
    return rows <= columns ? Parts(n, rows, columns).size : Parts(n, columns, rows).size;
}

int relay_orthogonalise(int32_t n, int64_t rows, int64_t columns, const float* update, int64_t worker_stride,
                        int64_t row_stride, int32_t steps, float eps, float scale, float* out, int64_t out_worker_stride,
                        int64_t out_row_stride, void* workspace, int64_t workspace_bytes, relay_stream_t stream) {
    if (const int rc = check_matrices(n, rows, columns)) return rc;
    const relay_rows in{const_cast<float*>(update), worker_stride, row_stride}, to{out, out_worker_stride, out_row_stride};
    if (!rows_fit(&in, RELAY_FP32, n, rows, columns, false) || !rows_fit(&to, RELAY_FP32, n, rows, columns, true) ||
        crossed(&in, &to, n, rows))
        return RELAY_EINVAL;
    if (steps < 1 || steps > RELAY_ORTHOGONALISE_MAX_STEPS || !(eps >= 0.0f) || !(eps < 1e30f) || !(scale > -1e30f) ||
        !(scale < 1e30f))
        return RELAY_EINVAL;
    if (workspace == nullptr || !aligned(workspace, 16) || workspace_bytes < relay_orthogonalise_workspace(n, rows, columns))
        return RELAY_EINVAL;
    if (encoder() == nullptr) return RELAY_ECUDA;

    const bool tall = rows > columns;
    const int64_t m = tall ? columns : rows, k = tall ? rows : columns;
    const Parts parts(n, m, k);
    char* base = static_cast<char*>(workspace);
    __half* x[2] = {reinterpret_cast<__half*>(base), reinterpret_cast<__half*>(base + parts.g / 2)};
    __half *g = reinterpret_cast<__half*>(base + parts.g), *p = reinterpret_cast<__half*>(base + parts.p);
    float* sums = reinterpret_cast<float*>(base + parts.sums);
    const Update u{update, n > 1 ? worker_stride : 0, rows > 1 ? row_stride : 0, static_cast<int32_t>(rows),
                   static_cast<int32_t>(columns)};
    // two strips a warp at least, eight CTAs per SM at most
    const int64_t warps = rows * ((columns + kStrip - 1) / kStrip), want = (warps + 15) / 16;
    const int64_t fit = 8 * kSms / n < 1 ? 1 : 8 * kSms / n < kParts ? 8 * kSms / n : kParts;
    const int cut = static_cast<int>(want < fit ? want : fit);
    relay_orthogonalise_norm_kernel<<<dim3(static_cast<unsigned>(cut), static_cast<unsigned>(n)), 256, 0, stream>>>(u, sums);
    if (const int rc = status_of_launch()) return rc;
    if (const int rc = launch_start(u, tall, sums, cut, eps, x[0], pitch_to(k), n, stream)) return rc;

    const int whole = whole_step(n, m, k);
    for (int step = 0; step < steps; ++step) {
        const __half* now = x[step & 1];
        const bool last = step == steps - 1;
        if (whole != 0) {
            StepArgs a{};
            a.x = now, a.rows = static_cast<int32_t>(m), a.columns = static_cast<int32_t>(k), a.pitch = pitch_to(k);
            a.slices = static_cast<int32_t>((k + whole - 1) / whole);
            if (last) {
                a.final = out, a.worker_stride = n > 1 ? out_worker_stride : 0, a.scale = scale / (kHeld * kHeld);
                a.row_stride = tall ? 1 : out_row_stride, a.column_stride = tall ? out_row_stride : 1;
            } else {
                a.out = x[(step & 1) ^ 1];
            }
            if (const int rc = whole == 64 ? launch_step<64>(a, n, stream) : launch_step<128>(a, n, stream)) return rc;
            continue;
        }
        ProductArgs a{};
        a.n = n, a.rows = static_cast<int32_t>(m);
        a.columns = static_cast<int32_t>(m), a.depth = static_cast<int32_t>(k), a.pitch = pitch_to(m);
        a.alpha = 1.0f / kHeld, a.out = g, a.group = group_of(m);
        if (const int rc = launch<false>(a, now, now, stream)) return rc;
        a.depth = static_cast<int32_t>(m);
        a.alpha = kC / kHeld, a.beta = kB, a.c = g, a.out = p;
        if (const int rc = launch<false>(a, g, g, stream)) return rc;
        a.columns = static_cast<int32_t>(k), a.pitch = pitch_to(k);
        a.alpha = 1.0f / kHeld, a.beta = kA, a.c = now, a.out = x[(step & 1) ^ 1];
        if (last) {
            a.scale = a.alpha * (scale / kHeld);
            a.out = nullptr, a.final = out, a.worker_stride = n > 1 ? out_worker_stride : 0;
            a.row_stride = tall ? 1 : out_row_stride, a.column_stride = tall ? out_row_stride : 1;
        }
        if (const int rc = launch<true>(a, p, now, stream)) return rc;
    }
    return RELAY_OK;
}

}  // extern "C"
