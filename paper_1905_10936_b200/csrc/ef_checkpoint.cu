// 8-bit activation checkpoints, and the activation between two linear layers that keeps its input
// as one: save, load, activation forward and backward.
//
//   save       (codes, scales) = Q8(x)                  load   x^ = codes * scale
//   forward    z^ = Q8(z) kept;  a = act(z^)            (or a = act(z) where nothing is kept)
//              with a checkpoint of the output: a := values of Q8(a)
//   backward   dz = da * act'(z^)
//
// act is GELU in its tanh form, z sigmoid(2 sqrt(2/pi) (z + 0.044715 z^3)) (the same function,
// with one exponential), or SwiGLU over rows [g | u]: g sigmoid(g) u.  The forward pass uses the
// values that the checkpoint stands for, so the backward pass differentiates exactly what was computed.
//
// Everything is elementwise but the groups' maxima, which stay inside a warp: a warp owns a
// 256-column segment of a row (two scale groups), one read and one write per element, no shared
// memory and no barrier.  8192 x 4096 bf16: GELU backward 33 us, 78 % of the copy rate; forward with
// both checkpoints 42 us, 75 %: the two quantisations and the activation take 240 instructions per segment and issue
// is 71 % busy.  Rows that do not allow 16-byte accesses (4099 x 2731 fp16, SwiGLU backward: 28 us, 48 %) are
// bound by the number of accesses: one per element and code.
#include "ef_rows.cuh"

#include <algorithm>

namespace {

using namespace efr;
using efh::Mat;

constexpr int kBlock = 256;
constexpr int kBlockWarps = kBlock / 32;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kGeluA = 1.5957691216057308f;                    // 2 sqrt(2/pi)
constexpr float kGeluB = 1.5957691216057308f * 0.044715f;

struct RowsArgs {
    const void* in; void* out;                   // z or da / a or dz (x / values for save and load)
    signed char* codes; float* scales;           // checkpoint of x or z (read by load and backward)
    signed char* out_codes; float* out_scales;   // checkpoint of a
    unsigned ld_in, ld_out;
    int C, pitch, groups, segs;
    unsigned items;                              // n * segs
};

// A warp's walk over segments, row-major with a stride of all warps of the grid.
struct Walk {
    unsigned idx, row, seg, stride, drow, dseg;
    __device__ __forceinline__ explicit Walk(const RowsArgs& a) {
        stride = gridDim.x * kBlockWarps;
        idx = blockIdx.x * kBlockWarps + (threadIdx.x >> 5);
        row = idx / (unsigned)a.segs; seg = idx - row * (unsigned)a.segs;
        drow = stride / (unsigned)a.segs; dseg = stride - drow * (unsigned)a.segs;
    }
    __device__ __forceinline__ bool in(const RowsArgs& a) const { return idx < a.items; }
    __device__ __forceinline__ int col() const { return (int)seg * kSeg; }
    __device__ __forceinline__ void next(const RowsArgs& a) {
        idx += stride; row += drow; seg += dseg;
        if (seg >= (unsigned)a.segs) { seg -= (unsigned)a.segs; ++row; }
    }
};

// Runs op over the segments of this warp (Op::kCtas CTAs per SM, as registers allow).  op.load fetches a segment into op's registers, op.take
// turns them into values, op.work does the rest; the next segment is fetched between the two, so that a warp's
// loads are in flight while it computes and stores.
template <class Op>
__device__ __forceinline__ void over_segments(const RowsArgs& a, Op& op) {
    Walk w(a);
    if (!w.in(a)) return;
    op.load(w.row, w.col());
    for (;;) {
        const unsigned row = w.row;
        const int s = w.col();
        op.take();
        w.next(a);
        const bool more = w.in(a);
        if (more) op.load(w.row, w.col());
        op.work(row, s);
        if (!more) return;
    }
}

template <class T, bool ALIGNED>
struct Save {
    static constexpr int kCtas = 5;
    const RowsArgs& a; const int lane;
    Raw8<T> raw; V8 v;
    __device__ __forceinline__ void load(unsigned row, int s) {
        load_raw<T, ALIGNED>(static_cast<const T*>(a.in) + before(row, a.ld_in), s, lane, a.C, raw);
    }
    __device__ __forceinline__ void take() { up8<T>(raw, v); }
    __device__ __forceinline__ void work(unsigned row, int s) {
        encode8<T, ALIGNED>(v, s, lane, a.pitch, a.groups, a.codes + before(row, a.pitch), a.scales + before(row, a.groups));
    }
};
template <class T, bool ALIGNED>
struct Load {
    static constexpr int kCtas = 5;
    const RowsArgs& a; const int lane;
    RawCodes raw; V8 v;
    __device__ __forceinline__ void load(unsigned row, int s) {
        load_codes<T, ALIGNED>(a.codes + before(row, a.pitch), a.scales + before(row, a.groups), s, lane, a.C, a.pitch, a.groups, raw);
    }
    __device__ __forceinline__ void take() { decode8(raw, v); }
    __device__ __forceinline__ void work(unsigned row, int s) {
        store8<T, ALIGNED>(static_cast<T*>(a.out) + before(row, a.ld_out), s, lane, a.C, v);
    }
};

// s = sigmoid(v) and 1 - s, v = 2 sqrt(2/pi) (z + 0.044715 z^3); zz = z * z.  Exponential and reciprocal are the hardware's
// approximations.  Outputs of 16 bits round away what they and the difference 1 - s leave (2 to 20 units of 2^-24).  fp32 outputs
// would show it, 1 - s most of all, which the slope multiplies by up to 20: there the smaller of the two comes from exp(-|v|) <= 1
// and the larger is the difference (a and dz of 2000 x 1604: 2.3e-8 and 5.0e-8 from 64 bits in the 2-norm, elementary fp32
// operations 2.5e-8 and 7.3e-8, the short form 3.6e-8 and 1.7e-7).
struct Gate { float2 s, rest; };
template <class T>
__device__ __forceinline__ Gate gelu_gate(float2 z, float2 zz) {
    if constexpr (sizeof(T) == 4) {
        const float2 v = mul2(z, fma2(zz, both(kGeluB), both(kGeluA)));
        const float2 q = exp2_2(mul2(make_float2(fabsf(v.x), fabsf(v.y)), both(-kLog2e)));
        const float2 small = mul2(q, rcp2(add2(both(1.f), q))), large = fma2(small, both(-1.f), both(1.f));
        return Gate{make_float2(v.x >= 0.f ? large.x : small.x, v.y >= 0.f ? large.y : small.y),
                    make_float2(v.x >= 0.f ? small.x : large.x, v.y >= 0.f ? small.y : large.y)};
    } else {
        const float2 t = mul2(z, fma2(zz, both(-kLog2e * kGeluB), both(-kLog2e * kGeluA)));
        const float2 s = rcp2(add2(both(1.f), exp2_2(t)));
        return Gate{s, fma2(s, both(-1.f), both(1.f))};
    }
}
// z^2 stops at 2^100, where the slope has long been 0 or 1: an infinity would meet the 0 of z s (1 - s).
template <class T>
__device__ __forceinline__ float2 gelu_slope(float2 z) {
    constexpr float kFar = 1.2676506e30f;
    float2 zz = mul2(z, z);
    zz = make_float2(fminf(zz.x, kFar), fminf(zz.y, kFar));
    const Gate g = gelu_gate<T>(z, zz);
    return fma2(mul2(mul2(z, g.s), g.rest), fma2(zz, both(3.f * kGeluB), both(kGeluA)), g.s);
}
__device__ __forceinline__ float2 sigmoid(float2 g) { return rcp2(add2(both(1.f), exp2_2(mul2(g, both(-kLog2e))))); }

// Row n of z is [z] (GELU) or [g | u] (SwiGLU), the checkpoint's rows are n, or 2n (g) and 2n + 1 (u).
template <int KIND> constexpr int kParts = KIND == EF_ACT_SWIGLU ? 2 : 1;

template <class T, bool ALIGNED, int KIND>
struct Forward {
    static constexpr int P = kParts<KIND>, kCtas = 6 - P;
    const RowsArgs& a; const int lane;
    Raw8<T> raw[P]; V8 z[P];
    __device__ __forceinline__ void load(unsigned row, int s) {
        const T* const p = static_cast<const T*>(a.in) + before(row, a.ld_in);
#pragma unroll
        for (int i = 0; i < P; ++i) load_raw<T, ALIGNED>(p + i * a.C, s, lane, a.C, raw[i]);
    }
    __device__ __forceinline__ void take() {
#pragma unroll
        for (int i = 0; i < P; ++i) up8<T>(raw[i], z[i]);
    }
    __device__ __forceinline__ void work(unsigned row, int s) {
        if (a.codes) {
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const unsigned r = row * P + i;
                encode8<T, ALIGNED>(z[i], s, lane, a.pitch, a.groups, a.codes + before(r, a.pitch), a.scales + before(r, a.groups));
            }
        }
        V8 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if constexpr (KIND == EF_ACT_GELU) v[k] = mul2(z[0][k], gelu_gate<T>(z[0][k], mul2(z[0][k], z[0][k])).s);
            else v[k] = mul2(mul2(z[0][k], sigmoid(z[0][k])), z[P - 1][k]);
        }
        if (s + kSeg > a.C) clear_behind<T, ALIGNED>(v, s, lane, a.C);           // a NaN scale must not reach the padding's codes
        if (a.out_codes)
            encode8<T, ALIGNED>(v, s, lane, a.pitch, a.groups, a.out_codes + before(row, a.pitch), a.out_scales + before(row, a.groups));
        if (a.out) store8<T, ALIGNED>(static_cast<T*>(a.out) + before(row, a.ld_out), s, lane, a.C, v);
    }
};

template <class T, bool ALIGNED, int KIND>
struct Backward {
    static constexpr int P = kParts<KIND>, kCtas = 6 - P;
    const RowsArgs& a; const int lane;
    Raw8<T> raw; RawCodes codes[P]; V8 da, z[P];
    __device__ __forceinline__ void load(unsigned row, int s) {
        load_raw<T, ALIGNED>(static_cast<const T*>(a.in) + before(row, a.ld_in), s, lane, a.C, raw);
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const unsigned r = row * P + i;
            load_codes<T, ALIGNED>(a.codes + before(r, a.pitch), a.scales + before(r, a.groups), s, lane, a.C, a.pitch, a.groups, codes[i]);
        }
    }
    __device__ __forceinline__ void take() {
        up8<T>(raw, da);
#pragma unroll
        for (int i = 0; i < P; ++i) decode8(codes[i], z[i]);
    }
    __device__ __forceinline__ void work(unsigned row, int s) {
        V8 d[P];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if constexpr (KIND == EF_ACT_GELU) {
                d[0][k] = mul2(da[k], gelu_slope<T>(z[0][k]));
            } else {
                const float2 g = z[0][k], sg = sigmoid(g), das = mul2(da[k], sg);
                const float2 rest = fma2(sg, both(-1.f), both(1.f));
                d[0][k] = mul2(mul2(das, z[P - 1][k]), fma2(g, rest, both(1.f)));
                d[P - 1][k] = mul2(das, g);
            }
        }
        T* const o = static_cast<T*>(a.out) + before(row, a.ld_out);
#pragma unroll
        for (int i = 0; i < P; ++i) store8<T, ALIGNED>(o + i * a.C, s, lane, a.C, d[i]);
    }
};

template <class Op>
__global__ void __launch_bounds__(kBlock, Op::kCtas) ef_segments_kernel(const RowsArgs a) {
    enter();
    Op op{a, (int)(threadIdx.x & 31)};
    over_segments(a, op);
}

template <class Op>
int launch_segments(const RowsArgs& a, cudaStream_t st) {
    const unsigned need = (a.items + kBlockWarps - 1) / kBlockWarps;
    return efh::launch(ef_segments_kernel<Op>, std::min<unsigned>(need, efh::kSMs * Op::kCtas), kBlock, 0, st, 0, a);
}

// Sizes and the parts of the arguments that all four calls share.  Fills a.
int rows_args(RowsArgs& a, int64_t n, int64_t c) {
    if (n < 0 || c < 1) return EF_ERR_INVALID_ARG;
    if (c > (int64_t)1 << 30) return EF_ERR_TOO_LARGE;
    const int64_t segs = (c + kSeg - 1) / kSeg;
    if (n > (((int64_t)1 << 31) - 1) / segs) return EF_ERR_TOO_LARGE;
    a = RowsArgs{};
    a.C = (int)c; a.segs = (int)segs; a.items = (unsigned)(n * segs);
    a.pitch = (int)EF_CHECKPOINT_PITCH(c); a.groups = (int)EF_CHECKPOINT_GROUPS(c);
    return EF_OK;
}

int check_mats(const Mat* m, int count, const void* codes, const void* out_codes) {
    for (int i = 0; i < count; ++i) if (!efh::fits31(m[i].ld)) return EF_ERR_TOO_LARGE;
    for (int i = 0; i < count; ++i) if (!efh::natural(m[i])) return EF_ERR_ALIGNMENT;
    return efh::aligned16(codes) && efh::aligned16(out_codes) ? EF_OK : EF_ERR_ALIGNMENT;
}

}  // namespace

extern "C" {

int ef_checkpoint_save(int32_t type, int64_t n, int64_t c, const void* x, int64_t ldx, int8_t* codes, float* scales,
                       void* cuda_stream) {
    EF_API_RANGE();
    RowsArgs a;
    if (!efh::type_ok(type) || ldx < c) return EF_ERR_INVALID_ARG;
    if (const int rc = rows_args(a, n, c)) return rc;
    if (n == 0) return EF_OK;
    if (!x || !codes || !scales) return EF_ERR_INVALID_ARG;
    const Mat ms[] = {{x, ldx, type}, {scales, 0, EF_TYPE_F32}};
    if (const int rc = check_mats(ms, 2, codes, nullptr)) return rc;
    if (const int rc = efh::check_device()) return rc;
    a.in = x; a.ld_in = (unsigned)ldx; a.codes = (signed char*)codes; a.scales = scales;
    return efh::with_type(type, [&](auto t) {
        using T = decltype(t);
        cudaStream_t st = (cudaStream_t)cuda_stream;
        return efh::vectors16(ms[0], c) ? launch_segments<Save<T, true>>(a, st) : launch_segments<Save<T, false>>(a, st);
    });
}

int ef_checkpoint_load(int32_t type, int64_t n, int64_t c, const int8_t* codes, const float* scales, void* x,
                       int64_t ldx, void* cuda_stream) {
    EF_API_RANGE();
    RowsArgs a;
    if (!efh::type_ok(type) || ldx < c) return EF_ERR_INVALID_ARG;
    if (const int rc = rows_args(a, n, c)) return rc;
    if (n == 0) return EF_OK;
    if (!x || !codes || !scales) return EF_ERR_INVALID_ARG;
    const Mat ms[] = {{x, ldx, type}, {scales, 0, EF_TYPE_F32}};
    if (const int rc = check_mats(ms, 2, codes, nullptr)) return rc;
    if (const int rc = efh::check_device()) return rc;
    a.out = x; a.ld_out = (unsigned)ldx; a.codes = (signed char*)codes; a.scales = const_cast<float*>(scales);
    return efh::with_type(type, [&](auto t) {
        using T = decltype(t);
        cudaStream_t st = (cudaStream_t)cuda_stream;
        return efh::vectors16(ms[0], c) ? launch_segments<Load<T, true>>(a, st) : launch_segments<Load<T, false>>(a, st);
    });
}

int ef_activation_forward(int32_t type, int32_t kind, int64_t n, int64_t c, const void* z, int64_t ldz, void* out,
                          int64_t ldo, int8_t* z_codes, float* z_scales, int8_t* a_codes, float* a_scales,
                          void* cuda_stream) {
    EF_API_RANGE();
    RowsArgs a;
    if (!efh::type_ok(type) || (kind != EF_ACT_GELU && kind != EF_ACT_SWIGLU)) return EF_ERR_INVALID_ARG;
    const int parts = kind == EF_ACT_SWIGLU ? 2 : 1;
    if (const int rc = rows_args(a, n, c)) return rc;
    if (ldz < parts * c || (out && ldo < c) || !z_codes != !z_scales || !a_codes != !a_scales)
        return EF_ERR_INVALID_ARG;
    if (n == 0) return EF_OK;
    if (!z || (!out && !a_codes)) return EF_ERR_INVALID_ARG;
    const Mat ms[] = {{z, ldz, type}, {out, ldo, type}, {z_scales, 0, EF_TYPE_F32}, {a_scales, 0, EF_TYPE_F32}};
    if (const int rc = check_mats(ms, 4, z_codes, a_codes)) return rc;
    if (const int rc = efh::check_device()) return rc;
    const bool aligned = efh::vectors16(ms[0], c) && efh::vectors16(ms[1], c);
    a.in = z; a.ld_in = (unsigned)ldz; a.out = out; a.ld_out = (unsigned)ldo;
    a.codes = (signed char*)z_codes; a.scales = z_scales; a.out_codes = (signed char*)a_codes; a.out_scales = a_scales;
    return efh::with_type(type, [&](auto t) {
        using T = decltype(t);
        cudaStream_t st = (cudaStream_t)cuda_stream;
        if (kind == EF_ACT_GELU)
            return aligned ? launch_segments<Forward<T, true, EF_ACT_GELU>>(a, st) : launch_segments<Forward<T, false, EF_ACT_GELU>>(a, st);
        return aligned ? launch_segments<Forward<T, true, EF_ACT_SWIGLU>>(a, st) : launch_segments<Forward<T, false, EF_ACT_SWIGLU>>(a, st);
    });
}

int ef_activation_backward(int32_t type, int32_t kind, int64_t n, int64_t c, const void* da, int64_t ldda,
                           const int8_t* z_codes, const float* z_scales, void* dz, int64_t lddz, void* cuda_stream) {
    EF_API_RANGE();
    RowsArgs a;
    if (!efh::type_ok(type) || (kind != EF_ACT_GELU && kind != EF_ACT_SWIGLU)) return EF_ERR_INVALID_ARG;
    const int parts = kind == EF_ACT_SWIGLU ? 2 : 1;
    if (const int rc = rows_args(a, n, c)) return rc;
    if (ldda < c || lddz < parts * c) return EF_ERR_INVALID_ARG;
    if (n == 0) return EF_OK;
    if (!da || !z_codes || !z_scales || !dz) return EF_ERR_INVALID_ARG;
    const Mat ms[] = {{da, ldda, type}, {dz, lddz, type}, {z_scales, 0, EF_TYPE_F32}};
    if (const int rc = check_mats(ms, 3, z_codes, nullptr)) return rc;
    if (const int rc = efh::check_device()) return rc;
    const bool aligned = efh::vectors16(ms[0], c) && efh::vectors16(ms[1], c);
    a.in = da; a.ld_in = (unsigned)ldda; a.out = dz; a.ld_out = (unsigned)lddz;
    a.codes = (signed char*)z_codes; a.scales = const_cast<float*>(z_scales);
    return efh::with_type(type, [&](auto t) {
        using T = decltype(t);
        cudaStream_t st = (cudaStream_t)cuda_stream;
        if (kind == EF_ACT_GELU)
            return aligned ? launch_segments<Backward<T, true, EF_ACT_GELU>>(a, st) : launch_segments<Backward<T, false, EF_ACT_GELU>>(a, st);
        return aligned ? launch_segments<Backward<T, true, EF_ACT_SWIGLU>>(a, st) : launch_segments<Backward<T, false, EF_ACT_SWIGLU>>(a, st);
    });
}

}  // extern "C"
