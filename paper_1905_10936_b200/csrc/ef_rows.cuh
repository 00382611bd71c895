// Shared by the operators that work on rows of a matrix (norm, checkpoints, activation, policy
// loss): element types, how a warp owns a 256-column segment of a row, and the 8-bit checkpoint
// code.  Internal; the interface is include/ef.h.
#pragma once

#include "ef_internal.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace efr {

using efk::kFull;

constexpr int kGroup = EF_CHECKPOINT_GROUP;      // columns that share a scale
constexpr int kSeg = 256;                        // columns of a segment: one warp, eight per lane
constexpr int kSegGroups = kSeg / kGroup;
static_assert(kSegGroups == 2, "the code below reduces two groups per segment");

// ---- element types -----------------------------------------------------------------------------
template <class T> struct Elem;
template <> struct Elem<float> {
    static __device__ __forceinline__ float up(float v) { return v; }
    static __device__ __forceinline__ float down(float v) { return v; }
};
template <> struct Elem<__nv_bfloat16> {
    static constexpr bool kEndsAt65504 = false;
    static __device__ __forceinline__ float up(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 down(float v) { return __float2bfloat16_rn(v); }
    static __device__ __forceinline__ float2 up2(unsigned v) {
        return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
    }
    static __device__ __forceinline__ unsigned down2(float a, float b) {
        const __nv_bfloat162 r = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const unsigned*>(&r);
    }
};
template <> struct Elem<__half> {
    static constexpr bool kEndsAt65504 = true;
    static __device__ __forceinline__ float up(__half v) { return __half2float(v); }
    static __device__ __forceinline__ __half down(float v) { return __float2half_rn(v); }
    static __device__ __forceinline__ float2 up2(unsigned v) { return __half22float2(*reinterpret_cast<__half2*>(&v)); }
    static __device__ __forceinline__ unsigned down2(float a, float b) {
        const __half2 r = __floats2half2_rn(a, b);
        return *reinterpret_cast<const unsigned*>(&r);
    }
};

// ---- which columns of a segment a lane owns ----------------------------------------------------
// Eight values per lane.  Where every pointer, row stride and row length of a call allows 16-byte accesses,
// 16-bit types own eight neighbours (one 16-byte access; a checkpoint group is half the warp) and
// fp32 twice four (two accesses; group 0 is the first four of every lane, group 1 the rest).
// Otherwise a lane owns every 32nd column: each access is one element wide and still coalesced
// over the warp, so ragged rows cost issue slots (8 accesses instead of 1 or 2) but no extra sectors.
template <class T, bool ALIGNED>
struct Own {
    static constexpr bool kHalf = ALIGNED && sizeof(T) == 2;
    static constexpr bool kQuad = ALIGNED && sizeof(T) == 4;
    static constexpr int kRun = kHalf ? 8 : (kQuad ? 4 : 1);         // neighbours per access
    static __host__ __device__ __forceinline__ constexpr int col(int lane, int k) {
        return kHalf ? 8 * lane + k : (kQuad ? 128 * (k >> 2) + 4 * lane + (k & 3) : lane + 32 * k);
    }
};

// Elements before row `row` of a matrix whose rows are ld apart: one widening multiplication.
__device__ __forceinline__ size_t before(unsigned row, unsigned ld) { return (size_t)row * ld; }

// ---- pairs ---------------------------------------------------------------------------------------
// These kernels would be bound by instruction issue before HBM (6 bytes per element leave about 30
// issue slots for it): values are kept in pairs and fp32 arithmetic uses the two-wide instructions.
using V8 = float2[4];                            // a lane's eight values, value k = element k & 1 of pair k >> 1

__device__ __forceinline__ unsigned long long bits2(float2 a) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a.x), "f"(a.y));
    return r;
}
__device__ __forceinline__ float2 pair2(unsigned long long r) {
    float2 a;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a.x), "=f"(a.y) : "l"(r));
    return a;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits2(a)), "l"(bits2(b)));
    return pair2(r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits2(a)), "l"(bits2(b)));
    return pair2(r);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(bits2(a)), "l"(bits2(b)), "l"(bits2(c)));
    return pair2(r);
}
__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp_approx(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float2 exp2_2(float2 v) { return make_float2(exp2_approx(v.x), exp2_approx(v.y)); }
__device__ __forceinline__ float2 rcp2(float2 v) { return make_float2(rcp_approx(v.x), rcp_approx(v.y)); }
// Largest of three, NaN if one is.
__device__ __forceinline__ float max_nan(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// Start of every kernel of these operators, before its first access to global memory.  All are
// launched with programmatic stream serialization and wait here for the kernel before them on the
// stream; none signals early, so a caller's kernel that follows sees what it always saw.  (Signalling
// at the start of each kernel gained at most 1 us on the smallest calls and cost 3 us on the
// GELU forward and backward at 8192 x 4096.)
__device__ __forceinline__ void enter() { efk::pdl_wait(); }
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}

// Everything but parameters is used once.
template <class U> __device__ __forceinline__ U load_once(const U* p) { return __ldcs(p); }
template <class U> __device__ __forceinline__ void store_once(U* p, U v) { __stcs(p, v); }

// ---- loads and stores of a segment ---------------------------------------------------------------
// ALIGNED also means that the number of columns is a multiple of a 16-byte access: an access lies
// inside the row or outside, and past the row's end it is predicated off.  (Single elements behind the last whole
// access would put a branch around each load; waiting there for one after the other cost 30 % at 20000 x 1000.)
template <class T> struct Raw8 { uint4 q[sizeof(T) == 2 ? 1 : 2]; };

// Loads this lane's eight values of the segment that starts at column s; columns >= C read as 0.
// The values stay in their type until up8 (so that several loads are in flight in few registers).
template <class T, bool ALIGNED>
__device__ __forceinline__ void load_raw(const T* __restrict__ row, int s, int lane, int C, Raw8<T>& r) {
    using O = Own<T, ALIGNED>;
    if constexpr (ALIGNED) {
#pragma unroll
        for (int k = 0; k < 8; k += O::kRun) {
            const int c = s + O::col(lane, k);
            r.q[k / O::kRun] = make_uint4(0u, 0u, 0u, 0u);
            if (c < C) r.q[k / O::kRun] = load_once(reinterpret_cast<const uint4*>(row + c));
        }
    } else {
        T* const e = reinterpret_cast<T*>(r.q);
        const T* const p = row + s + lane;
        if (s + kSeg <= C) {
#pragma unroll
            for (int k = 0; k < 8; ++k) e[k] = load_once(p + 32 * k);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) e[k] = s + lane + 32 * k < C ? load_once(p + 32 * k) : Elem<T>::down(0.f);
        }
    }
}

template <class T>
__device__ __forceinline__ void up8(const Raw8<T>& r, V8& v) {
    if constexpr (sizeof(T) == 2) {
        const unsigned w[4] = {r.q[0].x, r.q[0].y, r.q[0].z, r.q[0].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = Elem<T>::up2(w[k]);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float* f = reinterpret_cast<const float*>(r.q) + 2 * k;
            v[k] = make_float2(f[0], f[1]);
        }
    }
}

// fp32 parameters (weights) in the ownership of type T; read by every row, so cached normally.
template <class T, bool ALIGNED>
__device__ __forceinline__ void load_param8(const float* __restrict__ p, int s, int lane, int C, V8& v) {
    using O = Own<T, ALIGNED>;
    if constexpr (ALIGNED) {
#pragma unroll
        for (int k = 0; k < 8; k += 4) {
            const int c = s + O::col(lane, k);
            float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
            if (c < C) w = __ldg(reinterpret_cast<const float4*>(p + c));
            v[k / 2] = make_float2(w.x, w.y);
            v[k / 2 + 1] = make_float2(w.z, w.w);
        }
    } else {
        float* const f = reinterpret_cast<float*>(v);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int c = s + O::col(lane, k);
            f[k] = c < C ? __ldg(p + c) : 0.f;
        }
    }
}

template <class T, bool ALIGNED>
__device__ __forceinline__ void store8(T* __restrict__ row, int s, int lane, int C, const V8& v) {
    using O = Own<T, ALIGNED>;
    if constexpr (ALIGNED) {
#pragma unroll
        for (int k = 0; k < 8; k += O::kRun) {
            const int c = s + O::col(lane, k);
            uint4 q;
            if constexpr (sizeof(T) == 2)
                q = make_uint4(Elem<T>::down2(v[0].x, v[0].y), Elem<T>::down2(v[1].x, v[1].y),
                               Elem<T>::down2(v[2].x, v[2].y), Elem<T>::down2(v[3].x, v[3].y));
            else
                q = make_uint4(__float_as_uint(v[k / 2].x), __float_as_uint(v[k / 2].y), __float_as_uint(v[k / 2 + 1].x),
                               __float_as_uint(v[k / 2 + 1].y));
            if (c < C) store_once(reinterpret_cast<uint4*>(row + c), q);
        }
    } else {
        const float* const f = reinterpret_cast<const float*>(v);
        T* const p = row + s + lane;
        if (s + kSeg <= C) {
#pragma unroll
            for (int k = 0; k < 8; ++k) store_once(p + 32 * k, Elem<T>::down(f[k]));
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) if (s + lane + 32 * k < C) store_once(p + 32 * k, Elem<T>::down(f[k]));
        }
    }
}

// Sets the values of columns >= C to 0.
template <class T, bool ALIGNED>
__device__ __forceinline__ void clear_behind(V8& v, int s, int lane, int C) {
    float* const f = reinterpret_cast<float*>(v);
#pragma unroll
    for (int k = 0; k < 8; ++k) if (s + Own<T, ALIGNED>::col(lane, k) >= C) f[k] = 0.f;
}

// ---- the 8-bit checkpoint ----------------------------------------------------------------------
// A group's scale is the smallest power of two s with max|x| <= 127 s, its codes are
// rint(x / s) in [-127, 127].  With a power of two, x / s and code * s are exact: the codes do not
// depend on how the division is done, and code * s (seven significant bits) is exact in bf16 and
// fp32, so every reader sees the same value, the tensor cores' bf16 operands included.  The price is up
// to one bit of resolution (half a bit on average) against s = max|x| / 127.
//
// 127 = 1.984375 * 2^6: adding 0x01ffff to the bits of max|x| carries into the exponent exactly
// when its mantissa is above 1.984375, so the sum's exponent minus 6 is that of s.  A group of
// zeros gets s = 0; one that holds a NaN, an infinity or a value above 127 * 2^121 (within 0.8 %
// of fp32's largest, where the code's value could overflow) gets s = NaN and decodes to NaN.
// (1 / s needs neither case: a zero has code 0 by any finite factor, and codes under NaN say nothing.)
// fp16 ends at 65504, and from scale 1024 on the nearest code of a value just below may stand for 65536, which every fp16 output
// would turn into an infinity.  So in a matrix of fp16, a value that is finite there gets the last code that is, too.
constexpr unsigned kLargestCoded = ((127u + 6u + 121u) << 23) | 0x7e0000u;     // bits of 127 * 2^121

struct Scale { float s, inv; };

__device__ __forceinline__ Scale group_scale(unsigned amax_bits) {
    const int e = max((int)((amax_bits + 0x01ffffu - (6u << 23)) & 0xff800000u), 1 << 23);   // at least 2^-126
    Scale r;
    r.inv = __uint_as_float((254u << 23) - (unsigned)e);
    r.s = __uint_as_float(amax_bits == 0u ? 0u : (amax_bits > kLargestCoded ? 0x7fc00000u : (unsigned)e));
    return r;
}

// Scales of the segment's two groups: of this lane's first four values, and of its last four.
struct Scale2 { Scale lo, hi; };
template <class T, bool ALIGNED>
__device__ __forceinline__ Scale2 segment_scales(const V8& v, int lane) {
    // integer order of the bits = magnitude order, NaN on top
    Scale2 r;
    const float a = max_nan(fabsf(v[0].x), fabsf(v[0].y), fabsf(v[1].x));
    if constexpr (Own<T, ALIGNED>::kHalf) {              // a group is half the warp
        const float b = max_nan(max_nan(a, fabsf(v[1].y), fabsf(v[2].x)), fabsf(v[2].y), fabsf(v[3].x));
        const unsigned m = __float_as_uint(max_nan(b, fabsf(v[3].y)));
        const unsigned g0 = __reduce_max_sync(kFull, lane < 16 ? m : 0u), g1 = __reduce_max_sync(kFull, lane < 16 ? 0u : m);
        r.lo = r.hi = group_scale(lane < 16 ? g0 : g1);
    } else {
        const float b = max_nan(fabsf(v[2].x), fabsf(v[2].y), fabsf(v[3].x));
        r.lo = group_scale(__reduce_max_sync(kFull, __float_as_uint(max_nan(a, fabsf(v[1].y)))));
        r.hi = group_scale(__reduce_max_sync(kFull, __float_as_uint(max_nan(b, fabsf(v[3].y)))));
    }
    return r;
}

// Replaces v by the values its checkpoint stands for, and writes codes and scales of the segment.
// codes: the row's codes (pitch = EF_CHECKPOINT_PITCH(C), 16-byte aligned rows; columns C..pitch-1
// are written as 0); scales: the row's scales.  Columns >= C of v must be 0.  Whole warp.
// rint by adding 1.5 * 2^23: the sum's low byte is the code, and taking the constant off again
// leaves the code as a number.
template <class T, bool ALIGNED>
__device__ __forceinline__ void encode8(V8& v, int s, int lane, int pitch, int groups,
                                        signed char* __restrict__ codes, float* __restrict__ scales) {
    using O = Own<T, ALIGNED>;
    constexpr float kMagic = 12582912.f;
    const Scale2 sc = segment_scales<T, ALIGNED>(v, lane);
    const int g = s / kGroup;
    if constexpr (O::kHalf) {
        if ((lane & 15) == 0 && g + (lane >> 4) < groups) scales[g + (lane >> 4)] = sc.lo.s;
    } else {
        if (lane < 2 && g + lane < groups) scales[g + lane] = lane == 0 ? sc.lo.s : sc.hi.s;
    }
    unsigned f[8];
    bool near_end = false;
    if constexpr (sizeof(T) == 2) near_end = Elem<T>::kEndsAt65504 && fmaxf(sc.lo.s, sc.hi.s) >= 1024.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const Scale& q = k < 2 ? sc.lo : sc.hi;
        float2 y = fma2(v[k], both(q.inv), both(kMagic));
        if constexpr (sizeof(T) == 2) {
            if (near_end) {                      // 65520 is the first value that rounds to an infinity
                if (fabsf(v[k].x) < 65520.f && fabsf((y.x - kMagic) * q.s) >= 65520.f) y.x -= copysignf(1.f, v[k].x);
                if (fabsf(v[k].y) < 65520.f && fabsf((y.y - kMagic) * q.s) >= 65520.f) y.y -= copysignf(1.f, v[k].y);
            }
        }
        f[2 * k] = __float_as_uint(y.x);
        f[2 * k + 1] = __float_as_uint(y.y);
        v[k] = mul2(add2(y, both(-kMagic)), both(q.s));
    }
    if constexpr (ALIGNED) {
        unsigned w[2];
#pragma unroll
        for (int j = 0; j < 2; ++j)
            w[j] = __byte_perm(__byte_perm(f[4 * j], f[4 * j + 1], 0x0040),
                               __byte_perm(f[4 * j + 2], f[4 * j + 3], 0x0040), 0x5410);
        const int c = s + O::col(lane, 0);
        if constexpr (O::kHalf) {
            if (c < pitch) store_once(reinterpret_cast<uint2*>(codes + c), make_uint2(w[0], w[1]));
        } else {
            if (c < pitch) store_once(reinterpret_cast<unsigned*>(codes + c), w[0]);
            if (c + 128 < pitch) store_once(reinterpret_cast<unsigned*>(codes + c + 128), w[1]);
        }
    } else {
        signed char* const p = codes + s + lane;
        if (s + kSeg <= pitch) {
#pragma unroll
            for (int k = 0; k < 8; ++k) store_once(p + 32 * k, (signed char)(f[k] & 0xffu));
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) if (s + lane + 32 * k < pitch) store_once(p + 32 * k, (signed char)(f[k] & 0xffu));
        }
    }
}

// This lane's eight codes of a segment as they lie in memory (columns >= C: 0), and the scales of
// its first and last four values.
struct RawCodes { unsigned w[2]; float s[2]; };

template <class T, bool ALIGNED>
__device__ __forceinline__ void load_codes(const signed char* __restrict__ codes, const float* __restrict__ scales,
                                           int s, int lane, int C, int pitch, int groups, RawCodes& r) {
    using O = Own<T, ALIGNED>;
    const int g = s / kGroup;
    if constexpr (ALIGNED) {
        const int c = s + O::col(lane, 0);
        if constexpr (O::kHalf) {
            const uint2 q = c < pitch ? load_once(reinterpret_cast<const uint2*>(codes + c)) : make_uint2(0u, 0u);
            r.w[0] = q.x; r.w[1] = q.y;
        } else {
            r.w[0] = c < pitch ? load_once(reinterpret_cast<const unsigned*>(codes + c)) : 0u;
            r.w[1] = c + 128 < pitch ? load_once(reinterpret_cast<const unsigned*>(codes + c + 128)) : 0u;
        }
    } else {
        const signed char* const p = codes + s + lane;
        unsigned b[8];
        if (s + kSeg <= pitch) {
#pragma unroll
            for (int k = 0; k < 8; ++k) b[k] = (unsigned)(unsigned char)load_once(p + 32 * k);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) b[k] = s + lane + 32 * k < pitch ? (unsigned)(unsigned char)load_once(p + 32 * k) : 0u;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
            r.w[j] = __byte_perm(__byte_perm(b[4 * j], b[4 * j + 1], 0x0040),
                                 __byte_perm(b[4 * j + 2], b[4 * j + 3], 0x0040), 0x5410);
    }
    if constexpr (O::kHalf) {
        const int gg = g + (lane >> 4);
        r.s[0] = r.s[1] = gg < groups ? __ldg(scales + gg) : 0.f;
    } else {
        r.s[0] = __ldg(scales + g);
        r.s[1] = g + 1 < groups ? __ldg(scales + g + 1) : 0.f;
    }
}

// code * s: the byte (biased to 0..255) becomes the low mantissa byte of 2^23 + code + 128.
__device__ __forceinline__ void decode8(const RawCodes& r, V8& v) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const unsigned b = r.w[k >> 1] ^ 0x80808080u;
        const int at = (k & 1) * 2;
        const float2 y = make_float2(__uint_as_float(__byte_perm(b, 0x4b000000u, 0x7440 + at)),
                                     __uint_as_float(__byte_perm(b, 0x4b000000u, 0x7441 + at)));
        v[k] = mul2(add2(y, both(-8388736.f)), both(r.s[k >> 1]));
    }
}

}  // namespace efr

namespace efh {

// ---- host side ---------------------------------------------------------------------------------
inline size_t type_size(int32_t t) { return t == EF_TYPE_F32 ? 4 : 2; }
inline bool type_ok(int32_t t) { return t == EF_TYPE_F32 || t == EF_TYPE_BF16 || t == EF_TYPE_F16; }

// A matrix argument: elements of type t, rows ld elements apart.  A null pointer is an absent
// argument and allows everything.
struct Mat { const void* p; int64_t ld; int32_t type; };
inline bool natural(const Mat& m) { return ((uintptr_t)m.p & (type_size(m.type) - 1)) == 0; }
inline bool vectors16(const Mat& m, int64_t c) {
    return m.p == nullptr ||
           (aligned16(m.p) && (size_t)m.ld * type_size(m.type) % 16 == 0 && (size_t)c * type_size(m.type) % 16 == 0);
}

// Rows and strides are counted in 32 bits on the device (offsets in 64).
inline bool fits31(int64_t v) { return v <= 0x7fffffffLL; }

// Compute capability 10.x, asked once per device.
inline int check_device() {
    static signed char known[64] = {};
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return EF_ERR_CUDA;
    if (dev < 0 || dev >= 64) return EF_ERR_UNSUPPORTED_DEVICE;
    if (known[dev] == 0) {
        int major = 0;
        if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) return EF_ERR_CUDA;
        known[dev] = major == 10 ? 1 : -1;
    }
    return known[dev] > 0 ? EF_OK : EF_ERR_UNSUPPORTED_DEVICE;
}

// Launches a kernel that begins with efr::enter() (clusters of `cluster` CTAs, or as the kernel says where 0).
template <typename... KArgs, typename... Args>
inline int launch(void (*kernel)(KArgs...), dim3 grid, unsigned block, size_t smem, cudaStream_t st, unsigned cluster,
                  Args&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...) == cudaSuccess ? EF_OK : EF_ERR_CUDA;
}

// Calls f with a value of the element type that t names.
template <class F>
inline int with_type(int32_t t, F&& f) {
    if (t == EF_TYPE_F32) return f(float{});
    if (t == EF_TYPE_BF16) return f(__nv_bfloat16{});
    return f(__half{});
}

constexpr int kSMs = 148;

}  // namespace efh
