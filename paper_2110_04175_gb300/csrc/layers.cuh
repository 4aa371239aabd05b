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
// kVec: lane l holds features 8l .. 8l+7 of the strip and moves them in 16-byte
// pieces (d is a multiple of 8 then).  Otherwise lane l holds features l, 32 + l,
// ... 224 + l, so that every element-wise access of the warp is one contiguous
// piece whatever the rows' alignment, and a block of the 8-bit format is one
// element of every lane.  `left`: features of the row from the strip's first on.

template <bool kVec>
__device__ __forceinline__ int feature(int lane, int k) { return kVec ? 8 * lane + k : 32 * k + lane; }

// A lane's 8 features as they lie in memory, so that they can be asked for long before
// they are used.
template <typename T, bool kVec>
struct Piece {
    T e[8];
    __device__ __forceinline__ void load(const T* p, int lane, int left) {
#pragma unroll
        for (int k = 0; k < 8; ++k) e[k] = 32 * k + lane < left ? p[32 * k + lane] : T(0.0f);
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = widen(e[k]);
    }
};
template <typename T>
struct Piece<T, true> {
    static constexpr int kPer = 16 / sizeof(T);  // features of 16 bytes
    uint4 w[8 / kPer];
    __device__ __forceinline__ void load(const T* p, int lane, int left) {
#pragma unroll
        for (int h = 0; h < 8 / kPer; ++h)
            w[h] = 8 * lane < left ? *reinterpret_cast<const uint4*>(p + 8 * lane + h * kPer)
                                   : make_uint4(0, 0, 0, 0);  // +0 in every type
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
        for (int h = 0; h < 8 / kPer; ++h) {
            const T* e = reinterpret_cast<const T*>(&w[h]);
#pragma unroll
            for (int k = 0; k < kPer; ++k) v[h * kPer + k] = widen(e[k]);
        }
    }
};

template <bool kVec, typename T>
__device__ __forceinline__ void load_strip(const T* p, int lane, int left, float (&v)[8]) {
    Piece<T, kVec> piece;
    piece.load(p, lane, left);
    piece.get(v);
}

template <bool kVec, typename T>
__device__ __forceinline__ void store_strip(T* p, int lane, int left, const float (&v)[8]) {
    if constexpr (kVec) {
        if (8 * lane >= left) return;
        constexpr int kPer = 16 / sizeof(T);
#pragma unroll
        for (int h = 0; h < 8 / kPer; ++h) {
            uint4 w;
            T* e = reinterpret_cast<T*>(&w);
#pragma unroll
            for (int k = 0; k < kPer; ++k) e[k] = narrow<T>(v[h * kPer + k]);
            *reinterpret_cast<uint4*>(p + 8 * lane + h * kPer) = w;
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (32 * k + lane < left) p[32 * k + lane] = narrow<T>(v[k]);
    }
}

// fp32 weights at the same features; `quads`: their addresses are multiples of 16 bytes.
template <bool kVec>
__device__ __forceinline__ void load_weight(const float* p, int lane, int left, bool quads, float (&v)[8]) {
    if (kVec && quads) {
        load_strip<true>(p, lane, left, v);
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = feature<kVec>(lane, k) < left ? p[feature<kVec>(lane, k)] : 0.0f;
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
__device__ __forceinline__ uint32_t largest(const Piece<T, true>& p) {
    if constexpr (sizeof(T) == 2) {
        const uint4 w = p.w[0];
        const uint32_t m = __vmaxu2(__vmaxu2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu),
                                    __vmaxu2(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu));
        const unsigned short most = static_cast<unsigned short>(max(m & 0xffffu, m >> 16));
        return magnitude(widen(*reinterpret_cast<const T*>(&most)));
    } else {
        float v[8];
        p.get(v);
        return largest(v);
    }
}

// Puts the strip that starts at feature `base` of a row away; `codes` and `scales`
// are the row's.  v is 0 past d; most: largest() of the lane's (unused without kVec).
// All lanes of the warp take part.
template <bool kVec>
__device__ __forceinline__ void put_strip(int8_t* codes, uint8_t* scales, int base, int lane, int pitch,
                                          const float (&v)[8], uint32_t most) {
    if constexpr (kVec) {
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
    } else {
        uint32_t mine = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t c = scale_byte(__reduce_max_sync(0xffffffffu, magnitude(v[k])));
            if (lane == k) mine = c;
            if (base + 32 * k < pitch)
                codes[base + 32 * k + lane] = c == 255u ? 0 : static_cast<int8_t>(code_bits(v[k], c) & 0xffu);
        }
        if (lane < 8 && base + 32 * lane < pitch) scales[base / kBlock + lane] = static_cast<uint8_t>(mine);
    }
}

template <bool kVec>
__device__ __forceinline__ void put_strip(int8_t* codes, uint8_t* scales, int base, int lane, int pitch,
                                          const float (&v)[8]) {
    put_strip<kVec>(codes, scales, base, lane, pitch, v, kVec ? largest(v) : 0u);
}

// A lane's 8 codes and their scales as they lie in memory.
template <bool kVec>
struct CodePiece {
    int8_t q[8];
    uint8_t c[8];
    __device__ __forceinline__ void load(const int8_t* codes, const uint8_t* scales, int base, int lane, int pitch) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            q[k] = 0;
            c[k] = 7;
            if (base + 32 * k < pitch) {
                q[k] = codes[base + 32 * k + lane];
                c[k] = scales[base / kBlock + k];
            }
        }
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = static_cast<float>(q[k]) * scale_unit(c[k]);
    }
};
template <>
struct CodePiece<true> {
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
    __device__ __forceinline__ void get(float (&v)[8]) const {
        const float unit = scale_unit(c);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = code_value(k < 4 ? q.x : q.y, k % 4) * unit;
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
