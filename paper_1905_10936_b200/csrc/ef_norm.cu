// Root-mean-square norm of rows with the residual's addition and an output in 8 bits, and its gradient.
//
//   forward    h = x + r;  rstd = 1 / sqrt(mean_c(h^2) + eps);  y = h * rstd * w
//              with a checkpoint: codes and scales of y, and y := the values they stand for
//   backward   n = h * rstd;  u = w * dy;  dx = rstd * (u - n * mean_c(u n)) + dh;  dw = sum_rows dy * n
//
// Both are bound by HBM: the forward pass reads x and r and writes h, y and the codes once, the
// backward pass reads dy, h (or its codes) and dh and writes dx once.  A row stays in the
// registers of the W warps that own it, VPT segments of 256 columns each, between its reduction
// and its use, so nothing is read twice.  Sums are fp32 in a fixed order.
// 16384 x 1024 bf16 forward with residual and codes: 26.1 us, 89 % of the copy rate; 8192 x 4096 bf16
// backward with dh: 51 us, 80 %, 5 of them for the sum of the CTAs' parts of dw.
#include "ef_rows.cuh"

#include <algorithm>

namespace {

using namespace efr;
using efh::Mat;

constexpr int kBlock = 256;
constexpr int kMaxCols = 16 * 4 * kSeg;          // 16 warps of 4 segments

// Sum of v over the W warps that share a row; every thread gets it.  s: W floats of the row's
// group, used alternately (parity) so that one barrier per call suffices.
template <int W>
__device__ __forceinline__ float row_sum(float v, float* s, int parity, int group, int warp, int lane) {
    v = warp_sum(v);
    if constexpr (W > 1) {
        s += parity * W;
        if (lane == 0) s[warp] = v;
        asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(W * 32) : "memory");
        v = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) v += s[i];
    }
    return v;
}

// Threads of a CTA: as many rows as 256 threads hold, one at least.
template <int W> constexpr int kRowsPerCta = W * 32 > kBlock ? 1 : kBlock / (W * 32);
template <int W> constexpr int kCtaThreads = kRowsPerCta<W> * W * 32;

struct ForwardArgs {
    const void* x; const void* r; const float* w;
    void* h; void* y; float* rstd; signed char* codes; float* scales;
    unsigned n, ldx, ldr, ldh, ldy;
    int C, pitch, groups;
    double eps, inv_c;                   // the last step of rstd in 64 bits: one rounding after the sum's own
};

// Both passes walk over rows with all CTAs of the grid resident, and load the next row's values, in
// their type, before this row's sum is waited for: with a row's reduction between its loads and its
// stores and nothing else in flight, 20000 x 1000 bf16 rows took 37.9 us forward instead of 30.4.
template <class T, int VPT> struct ForwardRow { Raw8<T> x[VPT], r[VPT]; };
template <class T, bool ALIGNED, int W, int VPT>
__device__ __forceinline__ void load_row(const ForwardArgs& a, unsigned row, int warp, int lane, ForwardRow<T, VPT>& v) {
    const T* const x = static_cast<const T*>(a.x) + before(row, a.ldx);
    const T* const r = static_cast<const T*>(a.r) + before(row, a.ldr);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int s = (i * W + warp) * kSeg;
        if (s >= a.C) break;
        load_raw<T, ALIGNED>(x, s, lane, a.C, v.x[i]);
        if (a.r) load_raw<T, ALIGNED>(r, s, lane, a.C, v.r[i]);
    }
}

// Threads per SM, measured at n c = 2e7: 16-bit rows of six warps and more want 1536 of them (40 registers; 5120
// columns: 28.2 us, with 1024 threads 35.4), shorter ones 1024 (1024 columns: 28.4 us, with 1536 31.3), fp32 rows 1024.
template <class T, bool ALIGNED, int W, int VPT>
constexpr int kForwardCtas = VPT > 2 ? 1 : VPT > 1 ? (sizeof(T) == 2 ? 2 : 1)
                             : (W == 1 ? 1280 : W == 3 ? 768 : W < 6 || sizeof(T) == 4 ? 1024 : ALIGNED ? 1536 : 1280) / kCtaThreads<W>;

template <class T, bool ALIGNED, int W, int VPT>
__global__ void __launch_bounds__(kCtaThreads<W>, kForwardCtas<T, ALIGNED, W, VPT>) ef_rmsnorm_forward_kernel(const ForwardArgs a) {
    constexpr int kRows = kRowsPerCta<W>;
    __shared__ float s_part[kRows][2 * W];
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, group = wid / W, warp = wid % W;
    const unsigned step = gridDim.x * kRows;
    unsigned row = blockIdx.x * kRows + group;
    if (row >= a.n) return;
    enter();
    ForwardRow<T, VPT> next;
    load_row<T, ALIGNED, W, VPT>(a, row, warp, lane, next);
    int parity = 0;
    for (; row < a.n; row += step) {
        V8 h[VPT];
        float2 ss2 = both(0.f);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            if ((i * W + warp) * kSeg >= a.C) break;
            up8<T>(next.x[i], h[i]);
            if (a.r) {
                V8 r;
                up8<T>(next.r[i], r);
#pragma unroll
                for (int k = 0; k < 4; ++k) h[i][k] = add2(h[i][k], r[k]);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) ss2 = fma2(h[i][k], h[i][k], ss2);
        }
        if (row + step < a.n) load_row<T, ALIGNED, W, VPT>(a, row + step, warp, lane, next);
        if (a.h) {
            T* const o = static_cast<T*>(a.h) + before(row, a.ldh);
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                if ((i * W + warp) * kSeg >= a.C) break;
                store8<T, ALIGNED>(o, (i * W + warp) * kSeg, lane, a.C, h[i]);
            }
        }
        const float ss = row_sum<W>(ss2.x + ss2.y, s_part[group], parity, group, warp, lane);
        parity ^= 1;
        const float rstd = (float)rsqrt(fma((double)ss, a.inv_c, a.eps));
        if (warp == 0 && lane == 0) a.rstd[row] = rstd;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int s = (i * W + warp) * kSeg;
            if (s >= a.C) break;
            V8 w;
            load_param8<T, ALIGNED>(a.w, s, lane, a.C, w);
#pragma unroll
            for (int k = 0; k < 4; ++k) h[i][k] = mul2(mul2(h[i][k], both(rstd)), w[k]);
            if (a.codes && s + kSeg > a.C)       // 0 times a rstd that is not finite must not reach the padding's codes
                clear_behind<T, ALIGNED>(h[i], s, lane, a.C);
            if (a.codes)
                encode8<T, ALIGNED>(h[i], s, lane, a.pitch, a.groups, a.codes + before(row, a.pitch),
                                    a.scales + before(row, a.groups));
            if (a.y) store8<T, ALIGNED>(static_cast<T*>(a.y) + before(row, a.ldy), s, lane, a.C, h[i]);
        }
    }
}

struct BackwardArgs {
    const void* dy; const void* h; const signed char* codes; const float* scales;
    const void* dh; const float* w; const float* rstd;
    void* dx; float* partial;            // [gridDim.x][C] sums of dy * n over the CTA's rows
    unsigned n, lddy, ldh, lddh, lddx;
    int C, pitch, groups;
    float inv_c;
};

// Each thread keeps the sums for dw of the columns that it owns in registers over all its rows.
template <class T, int VPT> struct BackwardRow {
    Raw8<T> dy[VPT], h[VPT], dh[VPT];
    RawCodes codes[VPT];
    float rstd;
};
template <class T, bool ALIGNED, int W, int VPT, bool CODES>
__device__ __forceinline__ void load_row(const BackwardArgs& a, unsigned row, int warp, int lane, BackwardRow<T, VPT>& r) {
    const T* const dy = static_cast<const T*>(a.dy) + before(row, a.lddy);
    const T* const h = static_cast<const T*>(a.h) + before(row, a.ldh);
    const T* const dh = static_cast<const T*>(a.dh) + before(row, a.lddh);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int s = (i * W + warp) * kSeg;
        if (s >= a.C) break;
        load_raw<T, ALIGNED>(dy, s, lane, a.C, r.dy[i]);
        if constexpr (CODES)
            load_codes<T, ALIGNED>(a.codes + before(row, a.pitch), a.scales + before(row, a.groups), s, lane, a.C, a.pitch, a.groups,
                                   r.codes[i]);
        else load_raw<T, ALIGNED>(h, s, lane, a.C, r.h[i]);
        if (a.dh) load_raw<T, ALIGNED>(dh, s, lane, a.C, r.dh[i]);
    }
    r.rstd = __ldg(a.rstd + row);
}

// CTAs per SM, measured at n c = 2e7: 16-bit rows of up to four warps 4 (1024 columns: 31.4 us, with three CTAs
// 34.8), of 12 and 16 warps 2; fp32 rows hold twice the registers in flight and want about half as many threads.
template <class T, int W, int VPT>
constexpr int kBackwardCtas = VPT > 1 ? 1
                              : sizeof(T) == 4 ? (W == 6 ? 3 : W == 16 ? 1 : 2)
                              : W == 6 ? 5 : W >= 24 ? 1 : W >= 12 ? 2 : 4;

template <class T, bool ALIGNED, int W, int VPT, bool CODES>
__global__ void __launch_bounds__(kCtaThreads<W>, kBackwardCtas<T, W, VPT>) ef_rmsnorm_backward_kernel(const BackwardArgs a) {
    constexpr int kRows = kRowsPerCta<W>;
    __shared__ float s_part[kRows][2 * W];
    extern __shared__ float s_dw[];                      // [W * VPT * kSeg] when rows share a CTA
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, group = wid / W, warp = wid % W;
    V8 dw[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) dw[i][k] = both(0.f);
    enter();
    int parity = 0;
    BackwardRow<T, VPT> next;
    const unsigned step = gridDim.x * kRows;
    unsigned row = blockIdx.x * kRows + group;
    if (row < a.n) load_row<T, ALIGNED, W, VPT, CODES>(a, row, warp, lane, next);
    for (; row < a.n; row += step) {
        const float rstd = next.rstd;
        V8 n[VPT], u[VPT], dh[VPT];
        float2 dot2 = both(0.f);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int s = (i * W + warp) * kSeg;
            if (s >= a.C) break;
            V8 dy, w;
            up8<T>(next.dy[i], dy);
            if constexpr (CODES) decode8(next.codes[i], n[i]);
            else up8<T>(next.h[i], n[i]);
            if (a.dh) up8<T>(next.dh[i], dh[i]);
            load_param8<T, ALIGNED>(a.w, s, lane, a.C, w);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                n[i][k] = mul2(n[i][k], both(rstd));
                dw[i][k] = fma2(dy[k], n[i][k], dw[i][k]);
                u[i][k] = mul2(dy[k], w[k]);
                dot2 = fma2(u[i][k], n[i][k], dot2);
            }
        }
        if (row + step < a.n) load_row<T, ALIGNED, W, VPT, CODES>(a, row + step, warp, lane, next);
        const float mean = row_sum<W>(dot2.x + dot2.y, s_part[group], parity, group, warp, lane) * a.inv_c;
        parity ^= 1;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int s = (i * W + warp) * kSeg;
            if (s >= a.C) break;
            V8 o;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                o[k] = mul2(fma2(n[i][k], both(-mean), u[i][k]), both(rstd));
                if (a.dh) o[k] = add2(o[k], dh[i][k]);
            }
            store8<T, ALIGNED>(static_cast<T*>(a.dx) + before(row, a.lddx), s, lane, a.C, o);
        }
    }
    // the rows of a CTA are added in a fixed order, group after group
    float* out = a.partial + (long long)blockIdx.x * a.C;
    float* const f = reinterpret_cast<float*>(dw);
    if constexpr (kRows > 1) {
        for (int g = 0; g < kRows; ++g) {
            if (group == g) {
#pragma unroll
                for (int i = 0; i < VPT; ++i)
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const int c = (i * W + warp) * kSeg + 32 * k + lane;     // a place per value, free of conflicts
                        s_dw[c] = g == 0 ? f[8 * i + k] : s_dw[c] + f[8 * i + k];
                    }
            }
            __syncthreads();
        }
        if (group == 0) {
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int k = 0; k < 8; ++k) f[8 * i + k] = s_dw[(i * W + warp) * kSeg + 32 * k + lane];
        }
    }
    if (group == 0) {
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int c = (i * W + warp) * kSeg + Own<T, ALIGNED>::col(lane, k);
                if (c < a.C) out[c] = f[8 * i + k];
            }
    }
}

// dw[c] = sum over the CTAs' partial sums: 16 columns per CTA, 64 threads along the sum.
constexpr int kSumCols = 16, kSumRows = 64;
__global__ void __launch_bounds__(kSumCols * kSumRows) ef_rmsnorm_weight_kernel(const float* __restrict__ partial, int parts,
                                                                                int C, float* __restrict__ dw) {
    __shared__ float s[kSumCols][kSumRows + 1];
    enter();
    const int tx = threadIdx.x % kSumCols, ty = threadIdx.x / kSumCols, c = blockIdx.x * kSumCols + tx;
    float v = 0.f;
    if (c < C) {
#pragma unroll 8
        for (int p = ty; p < parts; p += kSumRows) v += partial[(long long)p * C + c];
    }
    s[tx][ty] = v;
    __syncthreads();
    const int col = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (col < kSumCols) {
        v = warp_sum(s[col][lane] + s[col][lane + 32]);
        if (lane == 0 && blockIdx.x * kSumCols + col < C) dw[blockIdx.x * kSumCols + col] = v;
    }
}

// Shapes (warps per row, segments per warp): one segment per warp as far as 16 warps reach.  A row that
// leaves warps idle costs its time all the same, so there are shapes between the powers of two.  The backward
// pass of 16-bit rows keeps to one segment per warp up to 8192 columns: 5001 (one element per access) 85 us
// instead of 128 at n c = 2e7, 5120 39.2 instead of 41.1.
template <class T, bool BACKWARD, class F>
int with_shape(int64_t C, F&& f) {
    using std::integral_constant;
#define EF_SHAPE(W, V) if (C <= (W) * (V) * kSeg) return f(integral_constant<int, W>{}, integral_constant<int, V>{})
    EF_SHAPE(1, 1);
    EF_SHAPE(2, 1);
    EF_SHAPE(3, 1);
    EF_SHAPE(4, 1);
    EF_SHAPE(6, 1);
    EF_SHAPE(8, 1);
    EF_SHAPE(12, 1);
    EF_SHAPE(16, 1);
    if constexpr (BACKWARD && sizeof(T) == 2) {
        EF_SHAPE(24, 1);
        EF_SHAPE(32, 1);
    } else {
        EF_SHAPE(12, 2);
        EF_SHAPE(16, 2);
    }
    return f(integral_constant<int, 16>{}, integral_constant<int, 4>{});
#undef EF_SHAPE
}

// CTAs of the backward pass, each of which leaves one partial sum of dw in the workspace.
constexpr int kMaxParts = efh::kSMs * 5;
constexpr int kRowsPerPart = 2;                  // rows of a group at least, where there are enough
int backward_parts(int64_t n, int rows_per_cta, int ctas_per_sm) {
    const int64_t want = (n + (int64_t)rows_per_cta * kRowsPerPart - 1) / ((int64_t)rows_per_cta * kRowsPerPart);
    return (int)std::max<int64_t>(1, std::min<int64_t>({want, (int64_t)efh::kSMs * ctas_per_sm, kMaxParts}));
}

}  // namespace

extern "C" {

int ef_rmsnorm_forward(int32_t type, int64_t n, int64_t c, const void* x, int64_t ldx, const void* r, int64_t ldr,
                       const float* w, float eps, void* h, int64_t ldh, void* y, int64_t ldy, float* rstd,
                       int8_t* codes, float* scales, void* cuda_stream) {
    EF_API_RANGE();
    if (!efh::type_ok(type) || n < 0 || c < 1 || !(eps >= 0.f) || !(eps < INFINITY)) return EF_ERR_INVALID_ARG;
    if (c > kMaxCols || !efh::fits31(n) || !efh::fits31(ldx) || !efh::fits31(ldr) || !efh::fits31(ldh) || !efh::fits31(ldy))
        return EF_ERR_TOO_LARGE;
    if (ldx < c || (r && ldr < c) || (h && ldh < c) || (y && ldy < c) || !codes != !scales) return EF_ERR_INVALID_ARG;
    if (n == 0) return EF_OK;
    if (!x || !w || !rstd || (!y && !codes)) return EF_ERR_INVALID_ARG;
    const Mat ms[] = {{x, ldx, type}, {r, ldr, type}, {h, ldh, type}, {y, ldy, type},
                      {w, 0, EF_TYPE_F32}, {rstd, 0, EF_TYPE_F32}, {scales, 0, EF_TYPE_F32}};
    for (const Mat& m : ms) if (!efh::natural(m)) return EF_ERR_ALIGNMENT;
    if (!efh::aligned16(codes)) return EF_ERR_ALIGNMENT;
    if (const int rc = efh::check_device()) return rc;
    bool aligned = true;
    for (int i = 0; i < 5; ++i) aligned = aligned && efh::vectors16(ms[i], c);
    ForwardArgs a;
    a.x = x; a.r = r; a.w = w; a.h = h; a.y = y; a.rstd = rstd; a.codes = (signed char*)codes; a.scales = scales;
    a.n = (unsigned)n; a.ldx = (unsigned)ldx; a.ldr = (unsigned)ldr; a.ldh = (unsigned)ldh; a.ldy = (unsigned)ldy;
    a.C = (int)c; a.pitch = (int)EF_CHECKPOINT_PITCH(c); a.groups = (int)EF_CHECKPOINT_GROUPS(c);
    a.eps = (double)eps; a.inv_c = 1.0 / (double)c;
    return efh::with_type(type, [&](auto t) {
        using T = decltype(t);
        return with_shape<T, false>(c, [&](auto w_, auto v_) {
            constexpr int W = decltype(w_)::value, V = decltype(v_)::value;
            constexpr int rows = kRowsPerCta<W>;
            auto go = [&](auto vectors) {
                constexpr bool A = decltype(vectors)::value;
                const int64_t grid = std::min<int64_t>((n + rows - 1) / rows, efh::kSMs * kForwardCtas<T, A, W, V>);
                return efh::launch(ef_rmsnorm_forward_kernel<T, A, W, V>, (unsigned)grid, kCtaThreads<W>, 0,
                                   (cudaStream_t)cuda_stream, 0, a);
            };
            return aligned ? go(std::true_type{}) : go(std::false_type{});
        });
    });
}

int ef_rmsnorm_backward_workspace_bytes(int64_t n, int64_t c, size_t* bytes) {
    if (!bytes || n < 0 || c < 1) return EF_ERR_INVALID_ARG;
    if (c > kMaxCols) return EF_ERR_TOO_LARGE;
    *bytes = (size_t)std::min<int64_t>(std::max<int64_t>(n, 1), kMaxParts) * (size_t)c * sizeof(float);
    return EF_OK;
}

int ef_rmsnorm_backward(int32_t type, int64_t n, int64_t c, const void* dy, int64_t lddy, const void* h, int64_t ldh,
                        const int8_t* h_codes, const float* h_scales, const float* w, const float* rstd,
                        const void* dh, int64_t lddh, void* dx, int64_t lddx, float* dw, void* workspace,
                        size_t workspace_bytes, void* cuda_stream) {
    EF_API_RANGE();
    size_t need = 0;
    if (!efh::type_ok(type)) return EF_ERR_INVALID_ARG;
    if (const int rc = ef_rmsnorm_backward_workspace_bytes(n, c, &need)) return rc;
    if (!efh::fits31(n) || !efh::fits31(lddy) || !efh::fits31(ldh) || !efh::fits31(lddh) || !efh::fits31(lddx))
        return EF_ERR_TOO_LARGE;
    if (!dw || lddy < c || lddx < c || (h && ldh < c) || (dh && lddh < c) || !h_codes != !h_scales)
        return EF_ERR_INVALID_ARG;
    const Mat ms[] = {{dy, lddy, type}, {h, ldh, type}, {dh, lddh, type}, {dx, lddx, type}, {w, 0, EF_TYPE_F32},
                      {rstd, 0, EF_TYPE_F32}, {dw, 0, EF_TYPE_F32}, {h_scales, 0, EF_TYPE_F32}};
    for (const Mat& m : ms) if (!efh::natural(m)) return EF_ERR_ALIGNMENT;
    if (!efh::aligned16(h_codes)) return EF_ERR_ALIGNMENT;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (n == 0) {                                        // no rows: the sum over rows is zero
        if (const int rc = efh::check_device()) return rc;
        return cudaMemsetAsync(dw, 0, (size_t)c * sizeof(float), st) == cudaSuccess ? EF_OK : EF_ERR_CUDA;
    }
    if (!dy || !h == !h_codes || !w || !rstd || !dx) return EF_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < need) return EF_ERR_WORKSPACE;
    if (!efh::aligned16(workspace)) return EF_ERR_ALIGNMENT;
    if (const int rc = efh::check_device()) return rc;
    bool aligned = true;
    for (int i = 0; i < 5; ++i) aligned = aligned && efh::vectors16(ms[i], c);
    BackwardArgs a;
    a.dy = dy; a.h = h; a.codes = (const signed char*)h_codes; a.scales = h_scales; a.dh = dh; a.w = w; a.rstd = rstd;
    a.dx = dx; a.partial = (float*)workspace;
    a.n = (unsigned)n; a.lddy = (unsigned)lddy; a.ldh = (unsigned)ldh; a.lddh = (unsigned)lddh; a.lddx = (unsigned)lddx;
    a.C = (int)c; a.pitch = (int)EF_CHECKPOINT_PITCH(c); a.groups = (int)EF_CHECKPOINT_GROUPS(c);
    a.inv_c = 1.f / (float)c;
    return efh::with_type(type, [&](auto t) {
        using T = decltype(t);
        return with_shape<T, true>(c, [&](auto w_, auto v_) {
            constexpr int W = decltype(w_)::value, V = decltype(v_)::value;
            constexpr int rows = kRowsPerCta<W>;
            const int parts = backward_parts(n, rows, kBackwardCtas<T, W, V>);
            const size_t smem = rows > 1 ? (size_t)W * V * kSeg * sizeof(float) : 0;
            auto go = [&](auto codes) {
                constexpr bool K = decltype(codes)::value;
                return efh::launch(aligned ? ef_rmsnorm_backward_kernel<T, true, W, V, K> : ef_rmsnorm_backward_kernel<T, false, W, V, K>,
                                   parts, kCtaThreads<W>, smem, st, 0, a);
            };
            if (const int rc = a.codes ? go(std::true_type{}) : go(std::false_type{})) return rc;
            return efh::launch(ef_rmsnorm_weight_kernel, (unsigned)((c + kSumCols - 1) / kSumCols), kSumCols * kSumRows, 0, st, 0,
                               (const float*)a.partial, parts, a.C, dw);
        });
    });
}

}  // extern "C"
