// Clipped policy loss with a KL term on a vocabulary's logits, and its gradient, in one pass.
//
//   logp_n  = x_{n,t} / T - log sum_j exp(x_{n,j} / T)              (t = target of token n)
//   ratio   = exp(logp - old);   gap = ref - logp
//   l_n     = -min(ratio A, clip(ratio, 1 - lo, 1 + hi) A) + beta (exp(gap) - gap - 1)
//   loss    = sum_n w_n l_n
//   dx_{n,j} = w_n / T * dl_n/dlogp * ([j = t] - p_{n,j}),
//   dl/dlogp = (ratio A <= clip A ? -ratio A : 0) + beta (1 - exp(gap))
//
// The gradient's coefficient depends on its own row only, so a row can be read once, kept, and its
// gradient written as soon as the row's sum is known: HBM sees one read and one write of the
// logits, which bounds the kernel.  A row (50257 bf16 logits: 98 KB) does not fit registers; it is staged in
// shared memory by bulk copies (16-byte aligned interior; at most 15 bytes at each end go through registers, so
// rows may start anywhere).  The first pass over it keeps a running maximum and sum, the second recomputes the exponentials.
// Rows of weight 0 are not read.  A group of warps handles a row:
//   - long rows: 8 warps, one row per CTA, two or three CTAs per SM, so that one loads while another computes and
//     writes.  Where there are more rows than that, CTAs walk over them and load the next while they write one
//     (ef_policy_rows_kernel).  Else the row comes in eight chunks that enter the first pass as they arrive; beyond
//     104 KB, or where rows are few, a cluster of CTAs shares it and exchanges (maximum, sum) through distributed
//     shared memory.  (Clusters of four 25 KB slices for 50257 bf16 logits, the same memory per SM, took
//     188 us instead of 145 at 4096 rows: they start and end together.)
//   - short rows: 1 or 4 warps, which walk over rows and load the next one while they work on this one
//     (16000 x 1001 bf16: 28 us; as rows of their own CTA 74; floor 9).  What bounds them is the chain of each row, with few in flight.
// 4096 x 50257 bf16, 15 % of the rows masked: 138 us for 762 MB, 84 % of the copy rate; two rows of 98 KB on an SM do not
// always cover one another's sums (8192 x 32000, three rows: 91 %).
// A device-side wait that runs out is the last of its CTA (or thread): copies in flight land, and rows not finished become NaN.
#include "ef_rows.cuh"

#include <algorithm>
#include <cmath>

namespace {

using namespace efr;
using efh::Mat;

constexpr int kMaxChunks = 8;                    // bulk copies (and mbarriers) per slice of a long row
constexpr int kMaxCluster = 8;
constexpr int kSliceUnit = 64;                   // slices start at multiples of 64 logits: same phase mod 16 bytes as the row
constexpr int kMaxSliceBytes = 200 * 1024, kMaxSmem = kMaxSliceBytes + 1024;
constexpr int kAloneBytes = 104 * 1024;          // slices of a row that leave room for another one on the SM
constexpr int kShortBytes[2] = {5 * 1024, 24 * 1024};            // longest rows of 1 and of 4 warps
constexpr double kLog2e = 1.4426950408889634074;
constexpr float kLowest = -3.402823466e38f;

// log2(e) / T as hi + lo, lo > 0 (so that an infinite distance stays infinite).  hi alone is up to
// 2^-25 off, which times a typical exponent of ten shifts the log-probabilities of all tokens alike by 1e-7;
// the loss is a sum over tokens of both signs and shows that.  The gradient's own rounding does not need lo.
struct Factor { float hi, lo; };
__device__ __forceinline__ float exp_of(float d, Factor k) { return exp2_approx(fmaf(d, k.lo, d * k.hi)); }
__device__ __forceinline__ float2 exp_of(float2 d, Factor k) { return exp2_2(fma2(d, both(k.lo), mul2(d, both(k.hi)))); }

struct PolicyArgs {
    const void* x; long long ldx;
    const long long* target;
    const float *old_logp, *adv, *weight, *ref;      // null for log-probabilities only (ref also: no KL term)
    float *logp, *token;
    void* grad; long long ldg;
    long long n;
    int C, slice;                                    // slice: logits per CTA of the cluster
    float lo, hi, beta, inv_t;
    double inv_t64;
    Factor k;
    int wait_limit;
};

struct MaxSum { float m, s; };
// m: largest logit so far (at least the lowest finite value, so that m - m is never inf - inf);
// s: sum of exp((x - m) / T).
__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b, Factor k) {
    MaxSum r;
    r.m = fmaxf(a.m, b.m);
    r.s = a.s * exp_of(a.m - r.m, k) + b.s * exp_of(b.m - r.m, k);
    return r;
}
__device__ __forceinline__ MaxSum join_warp(MaxSum v, Factor k) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        MaxSum u;
        u.m = __shfl_xor_sync(kFull, v.m, o);
        u.s = __shfl_xor_sync(kFull, v.s, o);
        v = join(v, u, k);
    }
    return v;
}

template <class T> constexpr int kVec = 16 / (int)sizeof(T);
template <class T> using VecPairs = float2[kVec<T> / 2];
template <class T>
__device__ __forceinline__ void up_vec(uint4 q, VecPairs<T>& v) {
    const unsigned w[4] = {q.x, q.y, q.z, q.w};
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = Elem<T>::up2(w[i]);
    } else {
        v[0] = make_float2(__uint_as_float(w[0]), __uint_as_float(w[1]));
        v[1] = make_float2(__uint_as_float(w[2]), __uint_as_float(w[3]));
    }
}
template <class T>
__device__ __forceinline__ uint4 down_vec(const VecPairs<T>& v) {
    if constexpr (sizeof(T) == 2)
        return make_uint4(Elem<T>::down2(v[0].x, v[0].y), Elem<T>::down2(v[1].x, v[1].y),
                          Elem<T>::down2(v[2].x, v[2].y), Elem<T>::down2(v[3].x, v[3].y));
    else
        return make_uint4(__float_as_uint(v[0].x), __float_as_uint(v[0].y), __float_as_uint(v[1].x), __float_as_uint(v[1].y));
}
// Running maximum and (two-wide) sum of a thread.
struct Running {
    float m; float2 s;
    __device__ __forceinline__ void raise(float top, Factor k) {
        if (top > m) {
            s = mul2(s, both(exp_of(m - top, k)));
            m = top;
        }
    }
    template <int N>
    __device__ __forceinline__ float top_of(const float2 (&v)[N]) {
        float t = fmaxf(v[0].x, v[0].y);
#pragma unroll
        for (int i = 1; i < N; ++i) t = fmaxf(fmaxf(t, v[i].x), v[i].y);
        return t;
    }
    template <int N>
    __device__ __forceinline__ void add(const float2 (&v)[N], Factor k) {
#pragma unroll
        for (int i = 0; i < N; ++i) s = add2(s, exp_of(add2(v[i], both(-m)), k));
    }
};

__device__ __forceinline__ unsigned cluster_size() { unsigned v; asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(v)); return v; }
__device__ __forceinline__ unsigned cluster_rank() { unsigned v; asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(v)); return v; }
__device__ __forceinline__ void cluster_started() { asm volatile("barrier.cluster.arrive.relaxed.aligned;"); }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void store_cluster(void* local, unsigned rank, MaxSum v) {
    unsigned addr;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(efk::smem_u32(local)), "r"(rank));
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(addr), "f"(v.m), "f"(v.s) : "memory");
}

// GW warps per row.  kLongWarps: long rows (one slot, kMaxChunks copies); 1, 4: two slots of one copy each.
constexpr int kLongWarps = 8;
template <int GW> struct Shape {
    static constexpr bool kLong = GW == kLongWarps;
    static constexpr int kBlock = kLong ? GW * 32 : 256, kGroups = kBlock / 32 / GW, kLanes = GW * 32;
    static constexpr int kSlots = kLong ? 1 : 2, kChunks = kLong ? kMaxChunks : 1;
    static constexpr int kCtas = kLong ? 3 : GW == 1 ? 4 : 3;     // per SM, as shared memory allows
};
// Bytes of one slot: the row's (or slice's) logits and room for its phase.
__host__ __device__ constexpr int slot_bytes(int len, int size) { return (len * size + 31) / 16 * 16; }

// A row's slice and where its logits lie: j < head and j >= tail by plain loads, the vectors between by bulk copy.
template <class T>
struct Slice {
    const T* x;
    int phase, head, vecs, tail;
    __device__ __forceinline__ Slice(const T* p, int len) : x(p) {
        phase = (int)((uintptr_t)p & 15u);
        head = min(len, ((16 - phase) & 15) / (int)sizeof(T));
        vecs = (len - head) / kVec<T>;
        tail = head + vecs * kVec<T>;
    }
};
// What is known of a row besides its vectors; fetched together with them.
template <class T> struct RowHead { long long t; float xt, old_logp, adv, ref; T edge; };

// A row's log-probability, loss and the factor of its gradient.  In 64 bits up to the ratio and the gap: logp's own
// rounding (5e-7 at -10) would show in the loss, where tokens of both signs nearly cancel.
struct Outcome { float logp, token, coef; };
template <class T>
__device__ __forceinline__ Outcome outcome_of(const PolicyArgs& a, MaxSum all, float w, const RowHead<T>& head) {
    const float nan = __uint_as_float(0x7fc00000u);
    const bool t_ok = head.t >= 0 && head.t < a.C;
    const double logp = t_ok ? (double)(head.xt - all.m) * a.inv_t64 - log((double)all.s) : (double)nan;
    float token = 0.f, coef = 0.f;
    if (a.old_logp) {
        const float ratio = expf((float)(logp - (double)head.old_logp)), straight = ratio * head.adv;
        const float clipped = fminf(fmaxf(ratio, 1.f - a.lo), 1.f + a.hi) * head.adv;
        const bool taken = !(straight > clipped);                // also where a side is NaN, which the bounds would drop
        token = -(taken ? straight : clipped);
        coef = taken ? -straight : 0.f;
        if (a.ref) {
            const float gap = (float)((double)head.ref - logp), e = expm1f(gap);
            token = fmaf(a.beta, e - gap, token);
            coef = fmaf(-a.beta, e, coef);
        }
        token *= w;
        coef *= w * a.inv_t;
    }
    return Outcome{(float)logp, token, coef};
}

template <int GW>
__device__ __forceinline__ void group_barrier(int group) {
    if constexpr (GW == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(GW * 32) : "memory");
}

template <class T, int GW>
__global__ void __launch_bounds__(Shape<GW>::kBlock, Shape<GW>::kCtas) ef_policy_kernel(const PolicyArgs a) {
    using S = Shape<GW>;
    constexpr int V = kVec<T>, kLanes = S::kLanes;
    extern __shared__ __align__(16) unsigned char s_rows[];      // [group][slot][slot_bytes]
    __shared__ unsigned long long s_bar[S::kGroups][S::kSlots][S::kChunks];
    __shared__ MaxSum s_warp[S::kGroups][GW], s_peer[kMaxCluster];
    __shared__ float s_out[S::kGroups][3];                       // maximum, -coef / sum, coef
    const unsigned cs = S::kLong ? cluster_size() : 1u, rank = S::kLong ? cluster_rank() : 0u;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, group = warp / GW, gw = warp % GW;
    const int tid = (int)threadIdx.x % kLanes;                   // within the group
    const int c0 = (int)rank * a.slice, len = max(0, min(a.slice, a.C - c0));
    const int slot_size = slot_bytes(a.slice, (int)sizeof(T));
    unsigned char* const slots = s_rows + group * S::kSlots * slot_size;
    if (tid == 0) {
        for (int i = 0; i < S::kSlots; ++i)
            for (int c = 0; c < S::kChunks; ++c) efk::mbar_init(&s_bar[group][i][c], 1);
        efk::mbar_fence_init();
    }
    group_barrier<GW>(group);
    enter();

    const Factor k = a.k;
    const float nan = __uint_as_float(0x7fc00000u);
    const long long step = (long long)(gridDim.x / cs) * S::kGroups;
    auto slice_of = [&](long long n) { return Slice<T>(static_cast<const T*>(a.x) + n * a.ldx + c0, len); };
    auto weight_of = [&](long long n) { return n < a.n ? (a.weight ? __ldg(a.weight + n) : 1.f) : 0.f; };
    // vectors per thread and chunk
    auto per_chunk_of = [&](int vecs) {
        return S::kChunks == 1 ? vecs : max(1, ((vecs + kLanes - 1) / kLanes + S::kChunks - 1) / S::kChunks) * kLanes;
    };
    auto edge_of = [&](const Slice<T>& sl) {                     // this thread's logit of the ends, or -1
        const int j = tid < sl.head ? tid : sl.tail + (tid - sl.head);
        return j < len && (tid < sl.head || j >= sl.tail) ? j : -1;
    };
    // A wait that runs out is this thread's last: its group's later rows are NaN, since the parities that it would wait
    // for no longer say which copy has landed.  (A long row is its CTA's only one, and has a barrier per chunk.)
    bool ok = true;
    unsigned in_flight = 0u;                                     // parities of the copies then on their way
    RowHead<T> next;
    auto fetch = [&](long long n, int slot) {
        const Slice<T> sl = slice_of(n);
        if (tid == 0 && ok) {
            T* const row = reinterpret_cast<T*>(slots + slot * slot_size + sl.phase);
            const int per = per_chunk_of(sl.vecs);
            efk::fence_proxy_async();                            // the slot was last read through ordinary loads
            for (int c = 0, at = 0; at < sl.vecs; ++c, at += per) {
                const unsigned bytes = (unsigned)min(per, sl.vecs - at) * 16u;
                efk::mbar_expect_tx(&s_bar[group][slot][c], bytes);
                efk::bulk_load(row + sl.head + at * V, sl.x + sl.head + at * V, bytes, &s_bar[group][slot][c]);
            }
        }
        const int e = edge_of(sl);
        next.edge = e >= 0 ? sl.x[e] : Elem<T>::down(0.f);
        next.t = a.target[n];
        next.xt = next.t >= 0 && next.t < a.C ? Elem<T>::up(static_cast<const T*>(a.x)[n * a.ldx + next.t]) : 0.f;
        if (a.old_logp) {
            next.old_logp = __ldg(a.old_logp + n);
            next.adv = __ldg(a.adv + n);
            next.ref = a.ref ? __ldg(a.ref + n) : 0.f;
        }
    };

    long long n = (long long)(blockIdx.x / cs) * S::kGroups + group;
    if (n >= a.n) return;
    float w = weight_of(n), w_next = weight_of(n + step);
    if (w != 0.f) fetch(n, 0);
    unsigned arrived = 0u;                                       // parity of each slot's next copy
    for (int it = 0; n < a.n; n += step, ++it) {
        const int slot = S::kSlots == 1 ? 0 : it & 1;
        const RowHead<T> head = next;
        const float w_after = weight_of(n + 2 * step);
        if constexpr (S::kSlots == 2) {
            if (w_next != 0.f) fetch(n + step, slot ^ 1);
        }
        T* const g = a.grad ? static_cast<T*>(a.grad) + n * a.ldg + c0 : nullptr;
        if (w == 0.f) {                                          // the whole cluster takes this way
            if (g) {
                const int first = min(len, (int)((16u - ((uintptr_t)g & 15u)) & 15u) / (int)sizeof(T));
                const int vecs = (len - first) / V;
                for (int j = tid; j < first; j += kLanes) g[j] = Elem<T>::down(0.f);
                for (int i = tid; i < vecs; i += kLanes)
                    store_once(reinterpret_cast<uint4*>(g + first) + i, make_uint4(0u, 0u, 0u, 0u));
                for (int j = first + vecs * V + tid; j < len; j += kLanes) g[j] = Elem<T>::down(0.f);
            }
            if (tid == 0 && rank == 0) {
                a.logp[n] = 0.f;
                if (a.token) a.token[n] = 0.f;
            }
        } else {
            const Slice<T> sl = slice_of(n);
            const T* const row = reinterpret_cast<const T*>(slots + slot * slot_size + sl.phase);
            const uint4* const sv = reinterpret_cast<const uint4*>(row + sl.head);
            const int edge = edge_of(sl), per = per_chunk_of(sl.vecs);
            if (cs > 1) cluster_started();                       // this CTA runs: its s_peer may be written
            Running run = {kLowest, both(0.f)};
            if (edge >= 0) {
                run.raise(Elem<T>::up(head.edge), k);
                run.s.x += exp_of(Elem<T>::up(head.edge) - run.m, k);
            }
            for (int c = 0, at = 0; at < sl.vecs; ++c, at += per) {
                if (S::kLong || ok) {
                    const bool landed = efk::mbar_wait_bounded(&s_bar[group][slot][c], arrived >> slot & 1u, a.wait_limit);
                    if (!landed && !S::kLong) in_flight = arrived ^ (w_next != 0.f && slice_of(n + step).vecs > 0 ? 0u : 1u << (slot ^ 1));
                    ok = landed && ok;
                }
                const int end = min(sl.vecs, at + per);
                int i = at + tid;
                for (; i + kLanes < end; i += 2 * kLanes) {
                    VecPairs<T> v, u;
                    up_vec<T>(sv[i], v);
                    up_vec<T>(sv[i + kLanes], u);
                    run.raise(fmaxf(run.top_of(v), run.top_of(u)), k);
                    run.add(v, k);
                    run.add(u, k);
                }
                if (i < end) {
                    VecPairs<T> v;
                    up_vec<T>(sv[i], v);
                    run.raise(run.top_of(v), k);
                    run.add(v, k);
                }
            }
            if (sl.vecs > 0) arrived ^= 1u << slot;
            MaxSum all = {run.m, run.s.x + run.s.y};
            if (!ok) all.s = nan;
            all = join_warp(all, k);
            if constexpr (GW > 1) {
                if (lane == 0) s_warp[group][gw] = all;
                group_barrier<GW>(group);
            }
            // the first warp joins the warps and CTAs and works out the coefficient for the others
            float scale = 0.f, coef = 0.f;
            if (cs > 1) cluster_wait();
            if (gw == 0) {
                if constexpr (GW > 1) {
                    all = s_warp[group][lane % GW];
#pragma unroll
                    for (int o = GW / 2; o > 0; o >>= 1) {
                        MaxSum u;
                        u.m = __shfl_xor_sync(kFull, all.m, o);
                        u.s = __shfl_xor_sync(kFull, all.s, o);
                        all = join(all, u, k);
                    }
                }
                if (cs > 1 && lane < (int)cs) store_cluster(&s_peer[rank], (unsigned)lane, all);
            }
            if (cs > 1) { cluster_arrive(); cluster_wait(); }
            if (gw == 0) {
                if (cs > 1) {
                    all = s_peer[0];
                    for (unsigned r = 1; r < cs; ++r) all = join(all, s_peer[r], k);
                }
                const Outcome o = outcome_of(a, all, w, head);
                coef = o.coef;
                if (lane == 0 && rank == 0) {
                    a.logp[n] = o.logp;
                    if (a.token) a.token[n] = o.token;
                }
                scale = -coef / all.s;
                if (GW > 1 && lane == 0) { s_out[group][0] = all.m; s_out[group][1] = scale; s_out[group][2] = coef; }
            }
            if constexpr (GW > 1) {
                group_barrier<GW>(group);
                all.m = s_out[group][0]; scale = s_out[group][1]; coef = s_out[group][2];
            }
            __syncwarp();                                        // the gradient may lie over logits that other lanes read
            if (g) {
                const float m = all.m;
                const int tl = head.t >= c0 && head.t < c0 + len ? (int)(head.t - c0) : -1;
                auto slope = [&](float v, int j) { return fmaf(exp2_approx((v - m) * k.hi), scale, j == tl ? coef : 0.f); };
                if ((int)((uintptr_t)g & 15u) == sl.phase) {
                    uint4* const gv = reinterpret_cast<uint4*>(g + sl.head);
#pragma unroll 2
                    for (int i = tid; i < sl.vecs; i += kLanes) {
                        VecPairs<T> v;
                        up_vec<T>(sv[i], v);
#pragma unroll
                        for (int q = 0; q < V / 2; ++q)
                            v[q] = mul2(exp2_2(mul2(add2(v[q], both(-m)), both(k.hi))), both(scale));
                        store_once(gv + i, down_vec<T>(v));
                    }
                    // the target's own term, by the thread that wrote its vector
                    if (tl >= sl.head && tl < sl.tail && (tl - sl.head) / V % kLanes == tid)
                        g[tl] = Elem<T>::down(slope(head.xt, tl));
                } else {                                         // rows of another phase: element by element
                    for (int j = sl.head + tid; j < sl.tail; j += kLanes) g[j] = Elem<T>::down(slope(Elem<T>::up(row[j]), j));
                }
                if (edge >= 0) g[edge] = Elem<T>::down(slope(Elem<T>::up(head.edge), edge));
            }
        }
        if (n + step < a.n) {
            group_barrier<GW>(group);                            // the slot, s_warp and s_peer may be written again
            if constexpr (S::kSlots == 1) {
                if (w_next != 0.f) fetch(n + step, 0);
            }
        }
        w = w_next;
        w_next = w_after;
    }
    if (tid == 0 && !ok) {                                       // copies on their way land before the CTA ends
        if constexpr (S::kLong) {
            const int vecs = slice_of((long long)(blockIdx.x / cs)).vecs, per = per_chunk_of(vecs);
            for (int c = 0, at = 0; at < vecs; ++c, at += per) efk::mbar_wait_bounded(&s_bar[group][0][c], 0u);
        } else {
            for (int i = 0; i < 2; ++i) efk::mbar_wait_bounded(&s_bar[group][i][0], in_flight >> i & 1u);
        }
    }
}

// Long rows, many of them: resident CTAs, each of one loading warp and eight that compute.  While a row's gradient is
// written, the loading warp refills each half of the row with the next one's as soon as all warps are done with it, so
// reads and writes of HBM run side by side inside each CTA.  It also fetches the row's scalars and ends, which cost the
// others two dependent accesses.  The next row is the one of a CTA of the grid that has not started yet and now
// never will (cluster launch control), so masked rows leave no CTA idle.
// 4096 x 50257 bf16, 15 % masked: 138 us, one row per CTA 151; 8192 x 32000: 163 and 180 us; 8192 x 16001 fp16: 97 and 114.
// Four chunks per row took 139 us and seven 146: each costs a wait.  Sixteen warps: 146.
__device__ __forceinline__ void ask_for_cta(uint4* answer, unsigned long long* bar) {
    efk::mbar_expect_tx(bar, 16);
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];"
                 ::"r"(efk::smem_u32(answer)), "r"(efk::smem_u32(bar)) : "memory");
}
// The CTA that was taken from the grid, or -1: none was left, after which no request may follow.
__device__ __forceinline__ int taken_cta(const uint4* answer) {
    int v;
    asm volatile("{\n\t.reg .b128 a;\n\t.reg .pred p;\n\tld.shared.b128 a, [%1];\n\tmov.b32 %0, -1;\n\t"
                 "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, a;\n\t"
                 "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %0, a;\n\t}"
                 : "=r"(v) : "r"(efk::smem_u32(answer)) : "memory");
    return v;
}
__device__ __forceinline__ void mbar_arrive(unsigned long long* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(efk::smem_u32(bar)) : "memory");
}
// A barrier of a long row's warps; true where any of them says so.
__device__ __forceinline__ bool any_of_warps(bool v) {
    unsigned r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((unsigned)v), "n"(kLongWarps * 32) : "memory");
    return r != 0u;
}

constexpr int kRowsThreads = (kLongWarps + 1) * 32;
constexpr int kHalves = 2;                       // chunks per row

template <class T>
__global__ void __launch_bounds__(kRowsThreads, 3) ef_policy_rows_kernel(const PolicyArgs a) {
    constexpr int V = kVec<T>, GW = kLongWarps, kLanes = GW * 32;
    extern __shared__ __align__(16) unsigned char s_rows[];      // the row's vectors
    __shared__ unsigned long long s_full[kHalves], s_free[kHalves], s_known[2], s_read[2], s_answered;
    __shared__ uint4 s_answer;
    struct Row { long long n; float w; RowHead<T> head; T edge[2 * V]; };
    __shared__ Row s_row[2];
    __shared__ MaxSum s_warp[GW];
    __shared__ float s_out[3];                                   // maximum, -coef / sum, coef
    // For a wait that ran out: s_stop ends the CTA's work, the rest says what it leaves.
    __shared__ unsigned s_stop, s_sent, s_phase;                 // chunks that a copy was sent to, and its phase's parity
    __shared__ int s_count, s_done, s_asked;                     // rows taken, rows finished, parity of an answer to come or -1
    __shared__ long long s_taken[4];                             // the rows taken last, by their number
    const int tid = (int)threadIdx.x, lane = tid & 31, gw = tid >> 5, len = a.C;
    if (tid == 0) {
        s_stop = 0u;
        for (int c = 0; c < kHalves; ++c) { efk::mbar_init(&s_full[c], 1); efk::mbar_init(&s_free[c], GW); }
        for (int b = 0; b < 2; ++b) { efk::mbar_init(&s_known[b], 1); efk::mbar_init(&s_read[b], GW); }
        efk::mbar_init(&s_answered, 1);
        efk::mbar_fence_init();
    }
    __syncthreads();
    enter();

    // Vectors per chunk, the same for every row, so that a chunk can be refilled while later ones are still read.
    const int per = max(1, ((len / V + kLanes - 1) / kLanes + kHalves - 1) / kHalves) * kLanes;
    auto slice_of = [&](long long n) { return Slice<T>(static_cast<const T*>(a.x) + n * a.ldx, len); };
    auto chunks_of = [&](const Slice<T>& sl) { return (sl.vecs + per - 1) / per; };
    // The first wait that runs out stops the CTA: it loads and takes no more rows, and no later wait relies on a parity.
    // (A row that was taken and not finished becomes NaN, see the end.)
    volatile unsigned* const stop = &s_stop;
    auto wait = [&](unsigned long long* bar, unsigned parity) {
        for (int i = 0; i < a.wait_limit; ++i) {
            if (efk::mbar_try_wait(bar, parity)) return true;
            if (*stop != 0u) return false;
        }
        *stop = 1u;
        return false;
    };

    if (gw == GW) {                                              // the loading warp
        long long n = blockIdx.x;
        bool ok = true, asked = false;
        unsigned freed = 0u;                                     // parity of each chunk's next release
        unsigned sent = 0u, phase = 0u;                          // chunks filled at least once, parity of the last time
        int used = 0;                                            // chunks that hold a row
        int it = 0;
        auto all_wait = [&](unsigned long long* bar, unsigned parity) { return __all_sync(kFull, wait(bar, parity)) != 0; };
        for (;; ++it) {
            Row& row = s_row[it & 1];
            const bool end = n >= a.n;
            if (!end && lane == 0) s_taken[it & 3] = n;
            const float w = end ? 0.f : a.weight ? __ldg(a.weight + n) : 1.f;
            const Slice<T> sl = slice_of(n);
            const int chunks = chunks_of(sl);
            auto load = [&]() {
                for (int c = 0; c < max(used, chunks); ++c) {
                    ok = ok && (c >= used || all_wait(&s_free[c], freed >> c & 1u));
                    if (!ok) return;
                    if (c >= chunks) continue;
                    if (sent >> c & 1u) phase ^= 1u << c;
                    sent |= 1u << c;
                    if (lane == 0) {
                        const unsigned bytes = (unsigned)min(per, sl.vecs - c * per) * 16u;
                        efk::fence_proxy_async();                // the chunk was last read through ordinary loads
                        efk::mbar_expect_tx(&s_full[c], bytes);
                        efk::bulk_load(s_rows + c * per * 16, sl.x + sl.head + c * per * V, bytes, &s_full[c]);
                    }
                }
                freed ^= (1u << used) - 1u;
            };
            if (!end && w != 0.f && used == 0) load();
            RowHead<T> h = {};
            T edge = Elem<T>::down(0.f);
            if (!end && w != 0.f) {
                const int j = lane < sl.head ? lane : sl.tail + (lane - sl.head);
                if (j < len && (lane < sl.head || j >= sl.tail)) edge = sl.x[j];
                h.t = a.target[n];
                if (a.old_logp) {
                    h.old_logp = __ldg(a.old_logp + n);
                    h.adv = __ldg(a.adv + n);
                    h.ref = a.ref ? __ldg(a.ref + n) : 0.f;
                }
                h.xt = h.t >= 0 && h.t < len ? Elem<T>::up(sl.x[h.t]) : 0.f;
            }
            if (it >= 2) ok = ok && all_wait(&s_read[it & 1], (it >> 1) + 1 & 1);
            if (!ok) break;
            if (lane == 0) { row.n = end ? -1 : n; row.w = w; row.head = h; }
            if (lane < 2 * V) row.edge[lane] = edge;
            __syncwarp();
            if (lane == 0) mbar_arrive(&s_known[it & 1]);
            if (end) break;
            if (w != 0.f) {
                if (used != 0) load();
                used = chunks;
            }
            if (!ok) break;
            if (lane == 0) {
                efk::fence_proxy_async();                        // the last answer was read through an ordinary load, by this lane
                ask_for_cta(&s_answer, &s_answered);
            }
            asked = true;
            ok = all_wait(&s_answered, it & 1);
            if (!ok) break;
            asked = false;
            int cta = -1;
            if (lane == 0) cta = taken_cta(&s_answer);
            cta = __shfl_sync(kFull, cta, 0);
            n = cta < 0 ? a.n : cta;
        }
        if (lane == 0) { s_count = n >= a.n ? it : it + 1; s_sent = sent; s_phase = phase; s_asked = asked ? it & 1 : -1; }
    } else {
        const Factor k = a.k;
        unsigned arrived = 0u;                                       // parity of each chunk's next copy
        int it = 0;
        for (;; ++it) {
            const Row& row = s_row[it & 1];
            if (any_of_warps(!wait(&s_known[it & 1], it >> 1 & 1)) || row.n < 0) break;
            const long long n = row.n;
            const float w = row.w;
            const RowHead<T> head = row.head;
            const Slice<T> sl = slice_of(n);
            const int ends = len - (sl.tail - sl.head);              // logits outside of the vectors
            const int edge = tid >= ends ? -1 : tid < sl.head ? tid : sl.tail + (tid - sl.head);
            const T edge_value = row.edge[tid & (2 * V - 1)];
            __syncwarp();
            if (lane == 0) mbar_arrive(&s_read[it & 1]);
            T* const g = a.grad ? static_cast<T*>(a.grad) + n * a.ldg : nullptr;
            if (w == 0.f) {
                if (g) {
                    const int first = min(len, (int)((16u - ((uintptr_t)g & 15u)) & 15u) / (int)sizeof(T));
                    const int vecs = (len - first) / V;
                    for (int j = tid; j < first; j += kLanes) g[j] = Elem<T>::down(0.f);
                    for (int i = tid; i < vecs; i += kLanes)
                        store_once(reinterpret_cast<uint4*>(g + first) + i, make_uint4(0u, 0u, 0u, 0u));
                    for (int j = first + vecs * V + tid; j < len; j += kLanes) g[j] = Elem<T>::down(0.f);
                }
                if (tid == 0) {
                    a.logp[n] = 0.f;
                    if (a.token) a.token[n] = 0.f;
                }
                continue;
            }
            const uint4* const sv = reinterpret_cast<const uint4*>(s_rows);
            const int chunks = chunks_of(sl);
            auto release = [&](int c) {                              // this warp is done with chunk c
                __syncwarp();
                if (lane == 0) mbar_arrive(&s_free[c]);
            };
            Running run = {kLowest, both(0.f)};
            bool ok = true;
            for (int c = 0; c < chunks; ++c) {
                ok = ok && wait(&s_full[c], arrived >> c & 1u);
                const int end = min(sl.vecs, (c + 1) * per);
                int i = c * per + tid;
                for (; i + kLanes < end; i += 2 * kLanes) {
                    VecPairs<T> v, u;
                    up_vec<T>(sv[i], v);
                    up_vec<T>(sv[i + kLanes], u);
                    run.raise(fmaxf(run.top_of(v), run.top_of(u)), k);
                    run.add(v, k);
                    run.add(u, k);
                }
                if (i < end) {
                    VecPairs<T> v;
                    up_vec<T>(sv[i], v);
                    run.raise(run.top_of(v), k);
                    run.add(v, k);
                }
                if (!g) release(c);
            }
            arrived ^= (1u << chunks) - 1u;
            if (edge >= 0) {
                run.raise(Elem<T>::up(edge_value), k);
                run.s.x += exp_of(Elem<T>::up(edge_value) - run.m, k);
            }
            MaxSum all = {run.m, run.s.x + run.s.y};
            all = join_warp(all, k);
            if (lane == 0) s_warp[gw] = all;
            if (any_of_warps(!ok)) break;
            if (gw == 0) {
                all = s_warp[lane % GW];
    #pragma unroll
                for (int o = GW / 2; o > 0; o >>= 1) {
                    MaxSum u;
                    u.m = __shfl_xor_sync(kFull, all.m, o);
                    u.s = __shfl_xor_sync(kFull, all.s, o);
                    all = join(all, u, k);
                }
                const Outcome o = outcome_of(a, all, w, head);
                if (lane == 0) {
                    a.logp[n] = o.logp;
                    if (a.token) a.token[n] = o.token;
                    s_out[0] = all.m; s_out[1] = -o.coef / all.s; s_out[2] = o.coef;
                }
            }
            group_barrier<GW>(0);
            if (!g) continue;
            const float m = s_out[0], scale = s_out[1], coef = s_out[2];
            const int tl = head.t >= 0 && head.t < len ? (int)head.t : -1;
            auto slope = [&](float v, int j) { return fmaf(exp2_approx((v - m) * k.hi), scale, j == tl ? coef : 0.f); };
            if ((int)((uintptr_t)g & 15u) == sl.phase) {
                uint4* const gv = reinterpret_cast<uint4*>(g + sl.head);
                for (int c = 0; c < chunks; ++c) {
                    const int end = min(sl.vecs, (c + 1) * per);
    #pragma unroll 2
                    for (int i = c * per + tid; i < end; i += kLanes) {
                        VecPairs<T> v;
                        up_vec<T>(sv[i], v);
    #pragma unroll
                        for (int q = 0; q < V / 2; ++q)
                            v[q] = mul2(exp2_2(mul2(add2(v[q], both(-m)), both(k.hi))), both(scale));
                        store_once(gv + i, down_vec<T>(v));
                    }
                    release(c);
                }
                // the target's own term, by the thread that wrote its vector
                if (tl >= sl.head && tl < sl.tail && (tl - sl.head) / V % kLanes == tid)
                    g[tl] = Elem<T>::down(slope(head.xt, tl));
            } else {                                                 // rows of another phase: element by element
                const T* const inner = reinterpret_cast<const T*>(sv);
                for (int j = sl.head + tid; j < sl.tail; j += kLanes) g[j] = Elem<T>::down(slope(Elem<T>::up(inner[j - sl.head]), j));
                for (int c = 0; c < chunks; ++c) release(c);
            }
            if (edge >= 0) g[edge] = Elem<T>::down(slope(Elem<T>::up(edge_value), edge));
        }
        if (tid == 0) s_done = it;
    }

    __syncthreads();
    if (*stop == 0u) return;
    // A wait ran out.  The copies and the answer that are on their way land first (waited for as long again); then every row
    // that this CTA took and did not finish becomes NaN, masked ones too, and with them the loss.
    if (tid == 0) {
        for (int c = 0; c < kHalves; ++c) if (s_sent >> c & 1u) efk::mbar_wait_bounded(&s_full[c], s_phase >> c & 1u);
        if (s_asked >= 0) {
            const bool answered = efk::mbar_wait_bounded(&s_answered, (unsigned)s_asked);
            const int cta = answered ? taken_cta(&s_answer) : -1;
            if (cta >= 0) s_taken[s_count++ & 3] = cta;
            if (!answered) s_done = min(s_done, s_count - 1);    // a row may be lost
        }
    }
    __syncthreads();
    const float nan = __uint_as_float(0x7fc00000u);
    for (int i = s_done; i < s_count; ++i) {
        const long long n = s_taken[i & 3];
        if (tid == 0) {
            a.logp[n] = nan;
            if (a.token) a.token[n] = nan;
        }
        if (a.grad)
            for (int j = tid; j < len; j += kRowsThreads) static_cast<T*>(a.grad)[n * a.ldg + j] = Elem<T>::down(nan);
    }
}

// loss = sum of the tokens' weighted losses, in a fixed order.
constexpr int kSumThreads = 1024;
__global__ void __launch_bounds__(kSumThreads) ef_policy_sum_kernel(const float* __restrict__ token, long long n,
                                                                    float* __restrict__ loss) {
    __shared__ double s[kSumThreads / 32];
    enter();
    double v = 0.0;
    for (long long i = threadIdx.x; i < n; i += kSumThreads) v += (double)token[i];
    v = efk::warp_sum(v);
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    if (threadIdx.x < 32) {
        v = efk::warp_sum(s[threadIdx.x]);
        if (threadIdx.x == 0) *loss = (float)v;
    }
}

// CTAs per row: slices of at most 104 KB, two CTAs of which share an SM; with few rows the row is
// spread further, down to 4 KB per CTA.
int cluster_of(int64_t n, int64_t row_bytes) {
    int cs = 1;
    while (cs < kMaxCluster && (row_bytes + cs - 1) / cs > kAloneBytes) cs *= 2;
    while (cs < kMaxCluster && n * cs < efh::kSMs && row_bytes / (2 * cs) >= 4096) cs *= 2;
    return cs;
}

template <class K>
int raise_smem(K kernel, bool (&raised)[64]) {
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return EF_ERR_CUDA;
    if (raised[dev]) return EF_OK;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem) != cudaSuccess) return EF_ERR_CUDA;
    raised[dev] = true;
    return EF_OK;
}

template <class T>
int launch_rows(PolicyArgs& a, cudaStream_t st) {
    static bool raised[64] = {};
    if (const int rc = raise_smem(ef_policy_rows_kernel<T>, raised)) return rc;
    return efh::launch(ef_policy_rows_kernel<T>, (unsigned)a.n, kRowsThreads, (size_t)a.C * sizeof(T) / 16 * 16, st, 0, a);
}

template <class T, int GW>
int launch_policy(PolicyArgs& a, cudaStream_t st) {
    using S = Shape<GW>;
    int cs = 1;
    a.slice = a.C;
    if (S::kLong) {
        cs = cluster_of(a.n, (int64_t)a.C * (int64_t)sizeof(T));
        a.slice = std::min<int>(a.C, ((a.C + cs - 1) / cs + kSliceUnit - 1) / kSliceUnit * kSliceUnit);
    }
    const size_t smem = (size_t)S::kGroups * S::kSlots * slot_bytes(a.slice, (int)sizeof(T));
    if (smem > kMaxSmem) return EF_ERR_TOO_LARGE;
    if (a.n > 0x7fffffffLL / cs) return EF_ERR_TOO_LARGE;
    static bool raised[64] = {};
    if (const int rc = raise_smem(ef_policy_kernel<T, GW>, raised)) return rc;
    // long rows: one per cluster, so that masked rows leave no CTA idle; short ones: resident CTAs walk over them
    const int64_t resident = efh::kSMs * std::min<int64_t>(S::kCtas, 224 * 1024 / (smem + 1024));
    const int64_t ctas = S::kLong ? a.n * cs : std::min<int64_t>((a.n + S::kGroups - 1) / S::kGroups, resident);
    return efh::launch(ef_policy_kernel<T, GW>, (unsigned)ctas, S::kBlock, smem, st, S::kLong ? (unsigned)cs : 0, a);
}

int launch(int32_t type, PolicyArgs& a, cudaStream_t st) {
    return efh::with_type(type, [&](auto t) {
        using T = decltype(t);
        const int64_t bytes = (int64_t)a.C * (int64_t)sizeof(T);
        if (bytes <= kShortBytes[0]) return launch_policy<T, 1>(a, st);
        if (bytes <= kShortBytes[1] && a.n > 2 * efh::kSMs) return launch_policy<T, 4>(a, st);
        // Up to two rows per SM there is no next row to load early (300 x 50257 bf16: resident CTAs 20 us, a CTA per row 19.7).
        // With few rows more a CTA per row is still ahead (400 x 50257: 26.8 and 29.2 us, 900 x 20001: 22.9 and 26.0), with many far behind.
        if (bytes <= kAloneBytes && a.n > 2 * efh::kSMs && a.n <= 0x7fffffff) return launch_rows<T>(a, st);
        return launch_policy<T, kLongWarps>(a, st);
    });
}

// The temperature's parts of the arguments; false where there are none.
bool set_temperature(PolicyArgs& a, float temperature) {
    if (!(temperature > 0.f) || !std::isfinite(1.f / temperature)) return false;
    const double k = kLog2e / (double)temperature;
    a.inv_t64 = 1.0 / (double)temperature;
    a.inv_t = (float)a.inv_t64;
    a.k.hi = (float)k;
    if ((double)a.k.hi >= k) a.k.hi = std::nextafter(a.k.hi, 0.f);
    a.k.lo = (float)(k - (double)a.k.hi);
    return std::isfinite(a.k.hi) && a.k.lo > 0.f;
}

int check_logits(int32_t type, int64_t n, int64_t c, const void* x, int64_t ldx, const int64_t* target, const float* logp) {
    if (!efh::type_ok(type) || n < 0 || c < 1 || ldx < c) return EF_ERR_INVALID_ARG;
    if (c > (int64_t)kMaxCluster * kMaxSliceBytes / (int64_t)efh::type_size(type)) return EF_ERR_TOO_LARGE;
    if (n == 0) return EF_OK;
    if (!x || !target || !logp) return EF_ERR_INVALID_ARG;
    if (!efh::natural(Mat{x, ldx, type}) || ((uintptr_t)target & 7u) || ((uintptr_t)logp & 3u)) return EF_ERR_ALIGNMENT;
    return EF_OK;
}

}  // namespace

extern "C" {

int ef_token_logprob(int32_t type, int64_t n, int64_t c, const void* logits, int64_t ldx, const int64_t* targets,
                     float temperature, float* logp, void* cuda_stream) {
    EF_API_RANGE();
    if (const int rc = check_logits(type, n, c, logits, ldx, targets, logp)) return rc;
    PolicyArgs a = {};
    if (!set_temperature(a, temperature)) return EF_ERR_INVALID_ARG;
    if (n == 0) return EF_OK;
    if (const int rc = efh::check_device()) return rc;
    a.x = logits; a.ldx = ldx; a.target = (const long long*)targets; a.logp = logp;
    a.n = n; a.C = (int)c; a.wait_limit = efh::wait_limit();
    return launch(type, a, (cudaStream_t)cuda_stream);
}

int ef_policy_loss(int32_t type, int64_t n, int64_t c, const void* logits, int64_t ldx, const int64_t* targets,
                   const float* old_logp, const float* advantages, const float* weights, const float* ref_logp,
                   float clip_low, float clip_high, float beta, float temperature, float* loss, float* logp,
                   float* token_loss, void* grad, int64_t ldg, void* cuda_stream) {
    EF_API_RANGE();
    if (const int rc = check_logits(type, n, c, logits, ldx, targets, logp)) return rc;
    PolicyArgs a = {};
    if (!set_temperature(a, temperature) || !(clip_low >= 0.f) || !(clip_high >= 0.f) ||
        !std::isfinite(beta) || !loss || (grad && ldg < c))
        return EF_ERR_INVALID_ARG;
    if (((uintptr_t)loss & 3u)) return EF_ERR_ALIGNMENT;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (n == 0) {
        if (const int rc = efh::check_device()) return rc;
        return cudaMemsetAsync(loss, 0, sizeof(float), st) == cudaSuccess ? EF_OK : EF_ERR_CUDA;
    }
    if (!old_logp || !advantages || !weights || !token_loss) return EF_ERR_INVALID_ARG;
    for (const void* p : {(const void*)old_logp, (const void*)advantages, (const void*)weights, (const void*)ref_logp,
                          (const void*)token_loss})
        if ((uintptr_t)p & 3u) return EF_ERR_ALIGNMENT;
    if (!efh::natural(Mat{grad, ldg, type})) return EF_ERR_ALIGNMENT;
    if (const int rc = efh::check_device()) return rc;
    a.x = logits; a.ldx = ldx; a.target = (const long long*)targets; a.old_logp = old_logp; a.adv = advantages;
    a.weight = weights; a.ref = ref_logp; a.logp = logp; a.token = token_loss; a.grad = grad; a.ldg = ldg;
    a.n = n; a.C = (int)c; a.lo = clip_low; a.hi = clip_high; a.beta = beta;
    a.wait_limit = efh::wait_limit();
    if (const int rc = launch(type, a, st)) return rc;
    return efh::launch(ef_policy_sum_kernel, 1, kSumThreads, 0, st, 0, (const float*)token_loss, (long long)n, loss);
}

}  // extern "C"
