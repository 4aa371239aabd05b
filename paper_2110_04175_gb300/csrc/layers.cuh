// layers.cuh -- what the layer kernels (layer_kernels.cu, weight_grad.cu)
// share: the activation types, a warp's strip of 256 features, the 8-bit
// format of relaylayers.h, and the argument checks.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

#include "relaylayers.h"

namespace {

constexpr int kStrip = 256;     // features that a warp handles together: 8 per lane
constexpr int kBlock = 32;      // features that share a scale
constexpr int kPitch = 128;     // checkpoint rows are whole multiples of this
constexpr int64_t kMaxD = int64_t(1) << 24, kMaxRows = int64_t(1) << 30;

// -------------------------------------------------------------------- types

__device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float widen(__half v) { return __half2float(v); }
__device__ __forceinline__ float widen(float v) { return v; }

template <typename T>
__device__ __forceinline__ T narrow(float v);
template <>
__device__ __forceinline__ __nv_bfloat16 narrow(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half narrow(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ float narrow(float v) { return v; }

// A view [n][tokens][d] as the kernels get it (relay_rows).
template <typename T>
struct View {
    T* p;
    int64_t ws, ts;
    __device__ __forceinline__ T* row(int64_t worker, int64_t token) const { return p + worker * ws + token * ts; }
};

// ------------------------------------------------------- a strip of 256 features
//
// Two ways to hold a strip of a row (`left`: the row's features from the strip's first on):
//   kVector  lane l has features 8l .. 8l + 7, moved in 16-byte pieces: rows on 16-byte
//            boundaries, d a multiple of 8;
//   kDirect  lane l has features l, 32 + l, ..., 224 + l, moved element by element, each of
//            the warp's accesses one contiguous piece: any row.
// The 8-bit format is kept in octets whichever way the row goes: with kDirect its values
// change places in `turn`, 256 floats of shared memory of the warp's own.  (At
// [4][8380][1001] in bf16, the gated step with its checkpoints: 292 us with codes, scales
// and block maxima element by element, 179 us this way.)  All lanes of the warp call these
// together.
enum Way { kDirect, kVector };

template <Way kWay>
__device__ __forceinline__ int feature(int lane, int k) { return kWay == kDirect ? 32 * k + lane : 8 * lane + k; }

__device__ __forceinline__ void to_octets(float (&v)[8], int lane, float* turn) {
#pragma unroll
    for (int k = 0; k < 8; ++k) turn[32 * k + lane] = v[k];
    __syncwarp();
    const float4 a = reinterpret_cast<const float4*>(turn + 8 * lane)[0], b = reinterpret_cast<const float4*>(turn + 8 * lane)[1];
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    __syncwarp();
}

__device__ __forceinline__ void from_octets(float (&v)[8], int lane, float* turn) {
    reinterpret_cast<float4*>(turn + 8 * lane)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(turn + 8 * lane)[1] = make_float4(v[4], v[5], v[6], v[7]);
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = turn[32 * k + lane];
    __syncwarp();
}

template <typename T>
__device__ __forceinline__ void widen_octet(const T* e, float (&v)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = widen(e[k]);
}

// A lane's 8 features as they lie in memory, so that they can be asked for long before
// they are used.
template <typename T, Way kWay>
struct Piece {
    T e[8];
    __device__ __forceinline__ void load(const T* p, int lane, int left) {
#pragma unroll
        for (int k = 0; k < 8; ++k) e[k] = 32 * k + lane < left ? p[32 * k + lane] : T(0.0f);
    }
    __device__ __forceinline__ void get(float (&v)[8]) const { widen_octet(e, v); }
};
template <typename T>
struct Piece<T, kVector> {
    static constexpr int kWords = sizeof(T) / 2;
    uint4 w[kWords];
    __device__ __forceinline__ void load(const T* p, int lane, int left) {
#pragma unroll
        for (int h = 0; h < kWords; ++h)
            w[h] = 8 * lane < left ? reinterpret_cast<const uint4*>(p + 8 * lane)[h]
                                   : make_uint4(0, 0, 0, 0);  // +0 in every type
    }
    __device__ __forceinline__ void get(float (&v)[8]) const { widen_octet(reinterpret_cast<const T*>(w), v); }
    // Lets what was widened from here be widened again rather than kept.
    __device__ __forceinline__ void forget() {
#pragma unroll
        for (int h = 0; h < kWords; ++h) asm volatile("" : "+r"(w[h].x), "+r"(w[h].y), "+r"(w[h].z), "+r"(w[h].w));
    }
};

template <Way kWay, typename T>
__device__ __forceinline__ void load_strip(const T* p, int lane, int left, float (&v)[8]) {
    Piece<T, kWay> piece;
    piece.load(p, lane, left);
    piece.get(v);
}

template <Way kWay, typename T>
__device__ __forceinline__ void store_strip(T* p, int lane, int left, const float (&v)[8]) {
    if constexpr (kWay == kDirect) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (32 * k + lane < left) p[32 * k + lane] = narrow<T>(v[k]);
    } else {
        constexpr int kWords = sizeof(T) / 2;
        if (8 * lane >= left) return;
        uint4 w[kWords];
        T* e = reinterpret_cast<T*>(w);
#pragma unroll
        for (int k = 0; k < 8; ++k) e[k] = narrow<T>(v[k]);
#pragma unroll
        for (int h = 0; h < kWords; ++h) reinterpret_cast<uint4*>(p + 8 * lane)[h] = w[h];
    }
}

// fp32 weights of the strip; `quads`: on 16-byte boundaries, with whole octets.
template <Way kWay>
__device__ __forceinline__ void load_weight(const float* p, int lane, int left, bool quads, float (&v)[8], float* turn) {
    if (kWay == kVector && quads) {
        load_strip<kVector>(p, lane, left, v);
        return;
    }
    load_strip<kDirect>(p, lane, left, v);
    if (kWay == kVector) to_octets(v, lane, turn);
}

// v is 0 past the row's end, also where its block reads as NaN.
template <Way kWay>
__device__ __forceinline__ void clear_past(float (&v)[8], int lane, int left) {
    if (left >= kStrip) return;
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (feature<kWay>(lane, k) >= left) v[k] = 0.0f;
}

// ------------------------------------------------------------- the 8-bit format

// The scale byte of a block whose largest magnitude has the bits `most` (sign
// cleared; as integers, NaN > infinity > any number).  Adding 2^16 carries into
// the exponent exactly where the magnitude is 127.5/128 of the next power of two
// or more, where code 128 would be needed.
__device__ __forceinline__ uint32_t scale_byte(uint32_t most) {
    return min(255u, max(7u, (most + 0x10000u) >> 23));
}

// 2^(c - 133), NaN for c = 255.  Bytes below 7 are never written; they read as 7.
__device__ __forceinline__ float scale_unit(uint32_t c) {
    return c == 255u ? __int_as_float(0x7fffffff) : __uint_as_float((max(c, 7u) - 6u) << 23);
}

// v / 2^(c - 133) rounded to a whole number (ties to even), in the low byte: the
// product by a power of two is exact, and adding 1.5 2^23 leaves the integer in
// the low bits.
__device__ __forceinline__ uint32_t code_bits(float v, uint32_t c) {
    return __float_as_uint(fmaf(v, __uint_as_float((260u - c) << 23), 12582912.0f));
}

// Code number `k` of the word w, as fp32: the byte with its sign bit turned over
// is q + 128, put under the exponent of 2^23.
__device__ __forceinline__ float code_value(uint32_t w, int k) {
    return __uint_as_float(__byte_perm(w ^ 0x80808080u, 0x4B000000u, 0x7650u | k)) - 8388736.0f;
}

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// The largest magnitude among a lane's 8 features, as bits.
__device__ __forceinline__ uint32_t largest(const float (&v)[8]) {
    uint32_t most = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) most = max(most, magnitude(v[k]));
    return most;
}

// The same from 16-bit features as they lie in memory, two at a time: their bits
// without the sign order as their magnitudes do, NaN last.
template <typename T>
__device__ __forceinline__ uint32_t largest(const Piece<T, kVector>& p) {
    const uint4 w = p.w[0];
    const uint32_t m = __vmaxu2(__vmaxu2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu),
                                __vmaxu2(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu));
    const unsigned short most = static_cast<unsigned short>(max(m & 0xffffu, m >> 16));
    return magnitude(widen(*reinterpret_cast<const T*>(&most)));
}

// The same, by what is at hand (0 for kDirect, where put_strip finds it).
template <typename T, Way kWay>
__device__ __forceinline__ uint32_t largest(const Piece<T, kWay>& p, const float (&v)[8]) {
    if constexpr (kWay == kDirect)
        return 0u;
    else if constexpr (sizeof(T) == 2)
        return largest(p);
    else
        return largest(v);
}

// Puts the strip that starts at feature `base` of a row away; `codes` and `scales`
// are the row's.  v is 0 past d; most: the lane's largest() (found here for kDirect).
template <Way kWay>
__device__ __forceinline__ void put_strip(int8_t* codes, uint8_t* scales, int base, int lane, int pitch,
                                          const float (&values)[8], uint32_t most, float* turn) {
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = values[k];
    if (kWay == kDirect) {
        to_octets(v, lane, turn);
        most = largest(v);
    }
    most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
    most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
    const uint32_t c = scale_byte(most);
    if (base + 8 * lane >= pitch) return;
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t ab = __byte_perm(code_bits(v[4 * h], c), code_bits(v[4 * h + 1], c), 0x0040);
        const uint32_t cd = __byte_perm(code_bits(v[4 * h + 2], c), code_bits(v[4 * h + 3], c), 0x0040);
        w[h] = c == 255u ? 0u : __byte_perm(ab, cd, 0x5410);
    }
    *reinterpret_cast<uint2*>(codes + base + 8 * lane) = make_uint2(w[0], w[1]);
    if (lane % 4 == 0) scales[base / kBlock + lane / 4] = static_cast<uint8_t>(c);
}

// A lane's 8 codes and their scale as they lie in memory.
struct CodePiece {
    uint2 q;
    uint32_t c;
    __device__ __forceinline__ void load(const int8_t* codes, const uint8_t* scales, int base, int lane, int pitch) {
        q = make_uint2(0, 0);
        c = 7;
        if (base + 8 * lane < pitch) {
            q = *reinterpret_cast<const uint2*>(codes + base + 8 * lane);
            c = scales[base / kBlock + lane / 4];
        }
    }
    template <Way kWay>
    __device__ __forceinline__ void get(float (&v)[8], int lane, float* turn) const {
        const float unit = scale_unit(c);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = code_value(k < 4 ? q.x : q.y, k % 4) * unit;
        if (kWay == kDirect) from_octets(v, lane, turn);
    }
};

// ----------------------------------------------------------- argument checks

inline int64_t element_size(int32_t type) { return type == RELAY_FP32 ? 4 : 2; }

inline bool aligned(const void* p, int64_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// RELAY_OK or why (n, tokens, d) and the type are refused.
inline int check_shape(int32_t type, int32_t n, int64_t tokens, int64_t d) {
    if (type < RELAY_BF16 || type > RELAY_FP32 || n < 1 || tokens < 0 || d < 1) return RELAY_EINVAL;
    if (n > RELAY_MAX_N || tokens >= kMaxRows || tokens * n >= kMaxRows || d > kMaxD) return RELAY_EUNSUPPORTED;
    return RELAY_OK;
}

// Whether a view may be used (NULL is not a view).
inline bool rows_fit(const relay_rows* r, int32_t type, int32_t n, int64_t tokens, int64_t d, bool output) {
    if (r == nullptr || r->worker_stride < 0 || r->token_stride < 0) return false;
    if (tokens == 0) return true;
    if (r->data == nullptr || !aligned(r->data, element_size(type))) return false;
    if (!output) return true;
    const __int128 ws = r->worker_stride, ts = r->token_stride;
    const bool by_worker = (tokens == 1 || ts >= d) && (n == 1 || ws >= (tokens - 1) * ts + d);
    const bool by_token = (n == 1 || ws >= d) && (tokens == 1 || ts >= (n - 1) * ws + d);
    return by_worker || by_token;
}

inline bool checkpoint_fits(const void* codes, const void* scales, int64_t tokens) {
    return tokens == 0 || (codes != nullptr && scales != nullptr && aligned(codes, 16) && aligned(scales, 16));
}

// The view as a kernel gets it; strides that are never walked are 0.
template <typename T>
View<T> view(const relay_rows* r, int32_t n, int64_t tokens) {
    if (r == nullptr) return View<T>{nullptr, 0, 0};
    return View<T>{static_cast<T*>(r->data), n > 1 ? r->worker_stride : 0, tokens > 1 ? r->token_stride : 0};
}

// Whether two views start at the same place without being the same rows.
inline bool crossed(const relay_rows* a, const relay_rows* b, int32_t n, int64_t tokens) {
    return a != nullptr && b != nullptr && a->data == b->data &&
           ((n > 1 && a->worker_stride != b->worker_stride) || (tokens > 1 && a->token_stride != b->token_stride));
}

// Whether the rows can be moved 16 bytes at a time (true for NULL).
inline bool vectors(const relay_rows* r, int32_t type, int32_t n, int64_t tokens) {
    if (r == nullptr) return true;
    const int64_t e = element_size(type);
    return aligned(r->data, 16) && (n == 1 || r->worker_stride * e % 16 == 0) &&
           (tokens == 1 || r->token_stride * e % 16 == 0);
}

inline int64_t pitch_of(int64_t d) { return (d + kPitch - 1) / kPitch * kPitch; }

inline int status_of_launch() { return cudaGetLastError() == cudaSuccess ? RELAY_OK : RELAY_ECUDA; }

// SMs of the current device, 0 on a CUDA error (cleared).
inline int sm_count() {
    static std::atomic<int> cache[64];
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) {
        (void)cudaGetLastError();
        return 0;
    }
    if (dev < 64 && (sms = cache[dev].load()) > 0) return sms;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        (void)cudaGetLastError();
        return 0;
    }
    if (dev < 64) cache[dev].store(sms);
    return sms;
}

}  // namespace
