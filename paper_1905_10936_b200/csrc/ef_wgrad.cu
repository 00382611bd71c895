// Weight gradient of a linear layer from the 8-bit checkpoint of its input:
//
//   dW[c, j] (+)= sum_n X^[n, c] * dY[n, j],      X^ = codes * scales (one scale per row and 128 columns)
//
// 2 n c j operations on the fifth-generation tensor cores (tcgen05, bf16 operands, fp32 accumulators in
// tensor memory).  A pair of CTAs (cta_group::2) makes 256 x N of dW; each holds 128 of the rows,
// exactly one scale group of X^, and half of the columns of dY.
//
// Both operands lie with the summed index n outermost, so both enter the tensor core "MN-major":
// a stage holds 64 tokens, each 64 columns of an operand as rows of 128 bytes in the 128-byte swizzle.
// dY is brought there by TMA.  The codes come by TMA as they are into a ring of their own; 16 warps in two
// groups that take the stages in turn make code * scale of them and store it with the same swizzle.
// code * scale has seven significant bits, so the bf16 operand is exact, and the product is that of the
// checkpoint's values without another rounding.
//
// The tensor core cuts its running sum at each step instead of rounding it: after 8192 tokens in one
// accumulator dW was 4.3e-6 off (2-norm), ten times an fp32 product.  So an accumulator runs over
// kSpan stages only; there are two, and while one runs the convert warps add the other into fp32
// registers: 2.1e-7 off (8192 x 384 x 640; fp32 products of the same 1e-7 to 5e-7).
//
// 8192 tokens, 1024 x 4096: 60 to 61 us, 1130 TFLOP/s; cuBLAS on operands that are bf16 already 45 us.  What bounds it is the
// convert warps' work beside the matrix instructions (without the conversion 52 us; 16 times 128 x 256
// sums in 64 registers each leave them 96 registers at 18 warps).  Steps on the way: CTAs by themselves, 128 x 256,
// 120 us; pairs, with a release at cluster scope for each stage of the second CTA, 149, without it
// 107; a single lane that walks the
// issuing loop, 75, the whole warp together with one elected lane, 68; codes read from global memory by the convert warps, whose
// fence before each hand-over waits for loads under way, 68 to 72, by TMA and scales in batches, 60.
//
// Device-side waits are bounded and have one answer per warp.  One that runs out makes the tile NaN; the load warp waits for its
// copies, and the issuing warp for its matrix instructions, before the pair parts and frees its accumulators.
//
// dY of 16-byte aligned bf16 rows is read as it is.  Other types and strides are first rewritten
// as bf16 rows in the workspace: fp16 as the sum of two bf16 values (exact: 11 bits), fp32 as the sum of
// three (exact: 24 bits), and the token loop runs over the terms one after the other.
//
// With few tiles the tokens are split over several pairs, whose partial sums go through the
// workspace and are added in a fixed order by a second kernel; few sums per pair are stored faster than many
// (300 tokens, 1024 x 1024: 7.5 us in 256 x 128 tiles, 9.9 in 256 x 256), so the tile's width is chosen too.
#include "ef_rows.cuh"

#include <algorithm>
#include <cuda.h>

namespace {

using namespace efr;
using efh::Mat;

constexpr int kTileM = 128;                      // rows of dW per CTA: one scale group
constexpr int kTileK = 64;                       // tokens per stage
constexpr int kChunkBytes = kTileK * 128;        // 64 columns x 64 tokens of bf16
constexpr int kStages = 6, kRawStages = 4;
constexpr int kRawBytes = kTileK * kTileM;       // codes of a stage
static_assert(kStages == 6 && kRawStages == 4, "a round of the convert loop goes over both rings");
constexpr int kMmaWarp = 0, kLoadWarp = 1, kFirstConvert = 2;
constexpr int kGroupWarps = 8;                   // a group of convert warps: eight tokens per warp
constexpr int kConvertWarps = 2 * kGroupWarps;   // also add up the accumulators and store the result
constexpr int kThreadsW = (kFirstConvert + kConvertWarps) * 32;
constexpr int kSpan = 18;                        // stages per accumulator
constexpr int kLag = kStages;                    // stages produced before the previous accumulator is collected: done by then
constexpr int kMaxSplits = 32;

struct WgradArgs {
    const float* scales;
    long long n;                                 // tokens
    int C, J, groups;
    int blocks_n;                                // stages per term: ceil(n / 64)
    int blocks;                                  // stages in all: terms * blocks_n
    int splits;
    float* out; long long ldo;                   // dW, or the partial sums [split][C][J] in the workspace
    int accumulate, wait_limit;
};

// ---- tcgen05 -----------------------------------------------------------------------------------
__device__ __forceinline__ void tmem_alloc(unsigned* dst, unsigned cols) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(efk::smem_u32(dst)), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(unsigned addr, unsigned cols) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols));
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void mma_f16(unsigned d, unsigned long long a, unsigned long long b, unsigned idesc, bool add) {
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
                 " tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((unsigned)add) : "memory");
}
// Arrives at the barrier of this offset in both CTAs once all matrix instructions so far are done.
__device__ __forceinline__ void mma_commit(unsigned long long* bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(efk::smem_u32(bar)), "h"((unsigned short)3) : "memory");
}
// 16 accumulator columns of this warp's 32 rows, added to acc.
__device__ __forceinline__ void tmem_add16(unsigned addr, float* acc) {
    unsigned r[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] += __uint_as_float(r[i]);
}
// Shared-memory operand, MN-major in the 128-byte swizzle: 64-column chunks kChunkBytes apart,
// groups of eight tokens 1024 bytes apart.
__device__ __forceinline__ unsigned long long operand(unsigned smem) {
    unsigned long long d = (unsigned long long)((smem & 0x3ffffu) >> 4);
    d |= (unsigned long long)(kChunkBytes >> 4) << 16;
    d |= (unsigned long long)(1024 >> 4) << 32;
    d |= 1ull << 46;                             // descriptor version of this architecture
    d |= 2ull << 61;                             // 128-byte swizzle
    return d;
}
// bf16 x bf16 -> fp32, both operands MN-major, 256 x N over the pair
template <int N>
constexpr unsigned kMmaShape = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((unsigned)(N >> 3) << 17) |
                               ((unsigned)(2 * kTileM >> 4) << 24);
__device__ __forceinline__ bool elect_one() {
    unsigned r;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(r));
    return r != 0u;
}
__device__ __forceinline__ void mbar_arrive(unsigned long long* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(efk::smem_u32(bar)) : "memory");
}
// A bounded wait of a whole warp, with the same answer in all lanes: what follows a wait that ran out has barriers in it.
__device__ __forceinline__ bool wait_warp(unsigned long long* bar, unsigned parity, int limit) {
    for (int i = 0; i < limit; ++i)
        if (__all_sync(kFull, efk::mbar_try_wait(bar, parity))) return true;
    return false;
}
// Arrives at the barrier of this offset in the pair's first CTA.
__device__ __forceinline__ void mbar_arrive_leader(unsigned long long* bar) {
    asm volatile("{\n .reg .b32 a;\n mapa.shared::cluster.u32 a, %0, 0;\n"
                 " mbarrier.arrive.shared::cluster.b64 _, [a];\n}" ::"r"(efk::smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void tma_load(void* dst, const CUtensorMap* map, int x, int y, unsigned long long* bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(efk::smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(efk::smem_u32(bar)) : "memory");
}

// Two codes (bytes 0 and 2 of w) as bf16 times s.  A byte in two's complement is
// (b & 127) - (b & 128); in bf16, 0x4300 | (b & 127) is 128 + (b & 127) and 0x4300 | (b & 128) is 128
// or 256, so their difference, exact, is the code.
__device__ __forceinline__ unsigned code_pair(unsigned w, __nv_bfloat162 s) {
    const unsigned lo = (w & 0x007f007fu) | 0x43004300u, sg = (w & 0x00800080u) | 0x43004300u;
    const __nv_bfloat162 v = __hmul2_rn(__hsub2_rn(*reinterpret_cast<const __nv_bfloat162*>(&lo),
                                                   *reinterpret_cast<const __nv_bfloat162*>(&sg)), s);
    return *reinterpret_cast<const unsigned*>(&v);
}
// Eight codes; in each four, the columns come in the order 0, 2, 1, 3 (no byte is moved for it), and
// the rows of the result are put back in order where they are stored.
__device__ __forceinline__ uint4 code_octet(unsigned a, unsigned b, __nv_bfloat162 s) {
    return make_uint4(code_pair(a, s), code_pair(a >> 8, s), code_pair(b, s), code_pair(b >> 8, s));
}
__device__ __forceinline__ int column_of(int m) { return (m & ~3) | ((m & 1) << 1) | ((m >> 1) & 1); }

template <int N> constexpr int kStageBytes = kTileM * 128 + N / 2 * 128;
template <int N> constexpr size_t kWgradSmem = (size_t)kStages * kStageBytes<N> + kRawStages * kRawBytes + 1024;

// A pair of CTAs: 256 x N of dW over a range of stages.  Per CTA, warps 2-17 convert codes, add up
// the accumulators and store the result; warp 1 issues the TMA loads; warp 0 issues the matrix
// instructions in the first CTA and tells the first CTA of full stages in the second.
template <int N>
__global__ void __launch_bounds__(kThreadsW, 1) __cluster_dims__(2, 1, 1)
ef_wgrad_kernel(const WgradArgs a, const __grid_constant__ CUtensorMap codes, const __grid_constant__ CUtensorMap dy) {
    extern __shared__ unsigned char s_raw[];
    // full: operand A of the stage (and in the first CTA, both operands of the second's); dy: operand B, by TMA
    __shared__ unsigned long long s_full[kStages], s_dy[kStages], s_empty[kStages], s_raw_full[kRawStages], s_raw_empty[kRawStages];
    __shared__ unsigned long long s_acc_full[2], s_acc_empty[2], s_drained;
    __shared__ unsigned s_tmem, s_failed;
    unsigned char* const stage0 = s_raw + ((1024u - (efk::smem_u32(s_raw) & 1023u)) & 1023u);
    unsigned char* const raw0 = stage0 + kStages * kStageBytes<N>;
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(kFull, tid >> 5, 0);
    const int rank = blockIdx.x & 1, pair = blockIdx.x >> 1;
    const int tiles_i = (a.C + 2 * kTileM - 1) / (2 * kTileM), tiles_j = (a.J + N - 1) / N;
    const int tile = pair % (tiles_i * tiles_j), split = pair / (tiles_i * tiles_j);
    const int i0 = (tile % tiles_i * 2 + rank) * kTileM, j0 = tile / tiles_i * N;
    // this split's stages
    const int b0 = (int)((long long)a.blocks * split / a.splits), b1 = (int)((long long)a.blocks * (split + 1) / a.splits);
    const int total = b1 - b0, spans = (total + kSpan - 1) / kSpan;
    if (tid == kLoadWarp * 32) {
        for (int s = 0; s < kStages; ++s) {
            // the convert warps, and in the first CTA the second's full stage
            efk::mbar_init(&s_full[s], kGroupWarps + (rank == 0));
            efk::mbar_init(&s_dy[s], 1);
            efk::mbar_init(&s_empty[s], 1);
        }
        for (int s = 0; s < kRawStages; ++s) {
            efk::mbar_init(&s_raw_full[s], 1);
            efk::mbar_init(&s_raw_empty[s], kGroupWarps);
        }
        for (int i = 0; i < 2; ++i) {
            efk::mbar_init(&s_acc_full[i], 1);
            efk::mbar_init(&s_acc_empty[i], 2 * kConvertWarps);
        }
        efk::mbar_init(&s_drained, 1);
        efk::mbar_fence_init();
        s_failed = 0u;
    }
    __syncthreads();
    // The other CTA's barriers may be reached once it has arrived here too; until then the loads and the
    // first stages get under way.
    cluster_arrive();
    enter();

    if (warp >= kFirstConvert) {
        const int cw = warp - kFirstConvert;
        constexpr int kCols = N / 4;             // accumulator columns of this warp: four warps share 32 rows
        unsigned acc_at = ((unsigned)((warp & 3) * 32) << 16) + (unsigned)((cw >> 2) * kCols);
        float acc[kCols];
#pragma unroll
        for (int i = 0; i < kCols; ++i) acc[i] = 0.f;
        bool ok = true;
        int span = 0;                            // next accumulator run to collect
        auto collect = [&] {
            const int buf = span & 1;
            if (span == 0) {                     // the accumulators' address is there, and so is the other CTA
                asm volatile("bar.sync 2, %0;" ::"n"((kConvertWarps + 1) * 32) : "memory");
                acc_at += s_tmem;
                cluster_wait();
            }
            ok = ok && wait_warp(&s_acc_full[buf], (unsigned)(span >> 1) & 1u, a.wait_limit);
            fence_after();
#pragma unroll
            for (int c = 0; c < kCols; c += 16) tmem_add16(acc_at + (unsigned)(buf * N + c), acc + c);
            fence_before();
            __syncwarp();
            if (span + 2 < spans && lane == 0) mbar_arrive_leader(&s_acc_empty[buf]);
            ++span;
        };
        // thread: token k = 8 * (warp in group) + lane / 4 of the stage, 16 codes of each 64-column chunk.
        // Odd tokens take the chunks in the other order: eight lanes then read, and write, different banks.
        const int group = cw / kGroupWarps, k = cw % kGroupWarps * 8 + (lane >> 2), v = lane & 3;
        // Scales: a lane loads the one of its token for every fourth stage of the group, four stages at a time and a
        // batch ahead (a load still under way would hold up each stage's fence).
        const float* const scales = a.scales + (i0 < a.C ? i0 / kTileM : 0);
        auto batch = [&](int first) {
            const int t = first + 2 * v;
            const long long n = (long long)((b0 + t) % a.blocks_n) * kTileK + k;     // a term's first tokens follow the last ones
            return t < total && n < a.n ? __ldg(scales + n * a.groups) : 0.f;
        };
        const unsigned x = (unsigned)(k & 7), odd = x & 1u;
        const unsigned u0 = (unsigned)(k * 128) + (((2 * v) ^ x) << 4), u1 = (unsigned)(k * 128) + (((2 * v + 1) ^ x) << 4);
        const unsigned char* const from0 = raw0 + group * kRawBytes + k * kTileM + 16 * v + odd * 64;
        const unsigned char* const from1 = raw0 + group * kRawBytes + k * kTileM + 16 * v + (odd ^ 1u) * 64;
        unsigned char* const to0 = stage0 + group * kStageBytes<N> + odd * kChunkBytes;
        unsigned char* const to1 = stage0 + group * kStageBytes<N> + (odd ^ 1u) * kChunkBytes;
        float sc = batch(group), sc_next = batch(group + 8);
        int turn = 0, until = kSpan + kLag;      // until: stages of this group before the next run is collected
        unsigned raw_parity = 0u;
        // six stages of the group: every slot of both rings (the first pass over the stages finds them empty)
        for (int t0 = group; ok && t0 < total; t0 += 12) {
#pragma unroll
            for (int i = 0; i < 6; ++i) {
                if (t0 + 2 * i >= total) break;
                const int s = i % 3 * 2, rs = i % 2 * 2;
                ok = ok && wait_warp(&s_raw_full[group + rs], raw_parity ^ (unsigned)(i / 2 & 1), a.wait_limit);
                const uint4 q0 = *reinterpret_cast<const uint4*>(from0 + rs * kRawBytes);
                const uint4 q1 = *reinterpret_cast<const uint4*>(from1 + rs * kRawBytes);
                const __nv_bfloat162 s2 = __float2bfloat162_rn(__shfl_sync(kFull, sc, (lane & ~3) | turn));
                ok = ok && wait_warp(&s_empty[group + s], i < 3 ? 1u : 0u, a.wait_limit);
                if (!ok) break;
                *reinterpret_cast<uint4*>(to0 + s * kStageBytes<N> + u0) = code_octet(q0.x, q0.y, s2);
                *reinterpret_cast<uint4*>(to0 + s * kStageBytes<N> + u1) = code_octet(q0.z, q0.w, s2);
                *reinterpret_cast<uint4*>(to1 + s * kStageBytes<N> + u0) = code_octet(q1.x, q1.y, s2);
                *reinterpret_cast<uint4*>(to1 + s * kStageBytes<N> + u1) = code_octet(q1.z, q1.w, s2);
                efk::fence_proxy_async();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&s_full[group + s]);
                    mbar_arrive(&s_raw_empty[group + rs]);
                }
                if (++turn == 4) {
                    turn = 0;
                    sc = sc_next;
                    sc_next = batch(t0 + 2 * i + 10);
                }
                if (i % 3 == 2 && (until -= 6) == 0) { collect(); until = kSpan; }
            }
            raw_parity ^= 1u;
        }
        while (span < spans) collect();
        if (!ok) s_failed = 1u;
        cluster_arrive();                        // nothing more reaches for the other CTA
        // result: 32 columns at a time through shared memory, so that a warp stores whole lines.
        // All matrix instructions are done (the last run was collected), so the stages are free.
        asm volatile("bar.sync 1, %0;" ::"n"(kConvertWarps * 32) : "memory");
        // a warp's 32 x 32 floats, 16-byte units of row r in the order of their number xor (r & 7)
        float4* const buf = reinterpret_cast<float4*>(stage0) + cw * 256;
        const int row0 = i0 + (warp & 3) * 32;
        const bool parts = a.splits > 1, add = a.accumulate != 0 && !parts;
        const long long ldo = parts ? a.J : a.ldo;
        float* const out = a.out + (parts ? (long long)split * a.C * a.J : 0);
        const bool vectors = (ldo & 3) == 0 && (a.J & 3) == 0 && ((uintptr_t)out & 15u) == 0;
#pragma unroll
        for (int c = 0; c < kCols; c += 32) {
            __syncwarp();
#pragma unroll
            for (int u = 0; u < 8; ++u)
                buf[lane * 8 + (u ^ (lane & 7))] = make_float4(acc[c + 4 * u], acc[c + 4 * u + 1], acc[c + 4 * u + 2], acc[c + 4 * u + 3]);
            __syncwarp();
            const int col0 = j0 + (cw >> 2) * kCols + c, u = lane & 7, j = col0 + 4 * u;
            float* const o = out + j;
            if (vectors) {
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    const int m = 4 * t + (lane >> 3), row = row0 + column_of(m);
                    float4 q = buf[m * 8 + (u ^ (m & 7))];
                    if (row < a.C && j < a.J) {
                        float4* const p = reinterpret_cast<float4*>(o + row * ldo);
                        if (add) {
                            const float4 w = *p;
                            q = make_float4(q.x + w.x, q.y + w.y, q.z + w.z, q.w + w.w);
                        }
                        *p = q;
                    }
                }
            } else if (col0 + lane < a.J) {      // rows that 16-byte stores do not fit: a column per lane
                const float* const f = reinterpret_cast<const float*>(buf);
#pragma unroll 8
                for (int t = 0; t < 32; ++t) {
                    const int row = row0 + column_of(t);
                    float* const p = out + row * ldo + col0 + lane;
                    const float val = f[t * 32 + (((lane >> 2) ^ (t & 7)) << 2) + (lane & 3)];
                    if (row < a.C) *p = add ? *p + val : val;
                }
            }
        }
        if (s_failed != 0u) {                    // a wait ran out: what this warp has stored becomes NaN
            __syncwarp();
            for (int c = lane; c < kCols; c += 32) {
                const int j = j0 + (cw >> 2) * kCols + c;
                for (int r = 0; r < 32; ++r)
                    if (row0 + r < a.C && j < a.J) out[(long long)(row0 + r) * ldo + j] = __uint_as_float(0x7fc00000u);
            }
        }
    } else if (warp == kLoadWarp) {
        const bool one = elect_one();
        int s = 0, rs = 0, block = b0 % a.blocks_n;
        unsigned parity = 1u, raw_parity = 1u;
        int raw_sent = 0, dy_sent = 0;           // stages under way
        for (int t = 0; t < total; ++t) {
            if (!wait_warp(&s_raw_empty[rs], raw_parity, a.wait_limit)) { s_failed = 1u; break; }
            ++raw_sent;
            if (one) {
                efk::mbar_expect_tx(&s_raw_full[rs], kRawBytes);
                tma_load(raw0 + rs * kRawBytes, &codes, i0, block * kTileK, &s_raw_full[rs]);
            }
            if (!wait_warp(&s_empty[s], parity, a.wait_limit)) { s_failed = 1u; break; }
            ++dy_sent;
            unsigned char* const dst = stage0 + s * kStageBytes<N> + kTileM * 128;
            if (one) {
                efk::mbar_expect_tx(&s_dy[s], N / 2 * 128);
#pragma unroll
                for (int c = 0; c < N / 128; ++c)
                    tma_load(dst + c * kChunkBytes, &dy, j0 + rank * (N / 2) + 64 * c, (b0 + t) * kTileK, &s_dy[s]);
            }
            if (++s == kStages) { s = 0; parity ^= 1u; }
            if (++rs == kRawStages) { rs = 0; raw_parity ^= 1u; }
            if (++block == a.blocks_n) block = 0;
        }
        __syncwarp();
        // No copy is under way when the CTA ends, also where the loop was left early: the last one of each slot lands.
        for (int i = max(0, raw_sent - kRawStages); i < raw_sent; ++i)
            wait_warp(&s_raw_full[i % kRawStages], (unsigned)(i / kRawStages) & 1u, efk::kMbarWaitLimit);
        for (int i = max(0, dy_sent - kStages); i < dy_sent; ++i)
            wait_warp(&s_dy[i % kStages], (unsigned)(i / kStages) & 1u, efk::kMbarWaitLimit);
        cluster_wait();
        cluster_arrive();
    } else if (rank != 0) {
        tmem_alloc(&s_tmem, 2 * N);
        asm volatile("bar.arrive 2, %0;" ::"n"((kConvertWarps + 1) * 32) : "memory");
        cluster_wait();
        const bool one = elect_one();
        int s = 0;
        unsigned parity = 0u;
        for (int t = 0; t < total; ++t) {
            if (!wait_warp(&s_full[s], parity, a.wait_limit) || !wait_warp(&s_dy[s], parity, a.wait_limit)) { s_failed = 1u; break; }
            if (one) mbar_arrive_leader(&s_full[s]);
            if (++s == kStages) { s = 0; parity ^= 1u; }
        }
        __syncwarp();
        cluster_arrive();
    } else {
        tmem_alloc(&s_tmem, 2 * N);
        asm volatile("bar.arrive 2, %0;" ::"n"((kConvertWarps + 1) * 32) : "memory");
        __syncwarp();
        const unsigned tmem = __shfl_sync(kFull, s_tmem, 0);
        cluster_wait();
        // One thread's latency per stage bounds the pair.  The warp stays together and its values are
        // the same for all lanes, one elected thread issues (68 us; a single lane walking the loop 75).
        const bool one = elect_one();
        const unsigned long long first = operand(efk::smem_u32(stage0));
        int s = 0, at = 0, span = 0;             // at: stage of the span
        unsigned parity = 0u;
        unsigned long long da = first;
        for (int t = 0; t < total; ++t) {
            bool ok = wait_warp(&s_dy[s], parity, a.wait_limit) && wait_warp(&s_full[s], parity, a.wait_limit);
            if (at == 0) ok = ok && wait_warp(&s_acc_empty[span & 1], ((unsigned)(span >> 1) & 1u) ^ 1u, a.wait_limit);
            if (!ok) { s_failed = 1u; break; }
            fence_after();
            const unsigned d = tmem + (unsigned)((span & 1) * N);
            const bool last = at == kSpan - 1 || t == total - 1;
            if (one) {
#pragma unroll
                for (int kk = 0; kk < kTileK / 16; ++kk)
                    mma_f16(d, da + kk * (2048 >> 4), da + (kTileM * 128 >> 4) + kk * (2048 >> 4), kMmaShape<N>,
                            at > 0 || kk > 0);
                if (t + kStages < total) mma_commit(&s_empty[s]);      // no arrivals that nobody waits for
                if (last) mma_commit(&s_acc_full[span & 1]);
            }
            ++at;
            if (last) { at = 0; ++span; }
            da += kStageBytes<N> >> 4;
            if (++s == kStages) { s = 0; parity ^= 1u; da = first; }
        }
        __syncwarp();
        // Nor is a matrix instruction, which reads both CTAs' stages and writes both CTAs' accumulators.
        if (one) mma_commit(&s_drained);
        wait_warp(&s_drained, 0u, efk::kMbarWaitLimit);
        cluster_arrive();
    }
    // No CTA leaves, and none frees its accumulators, while the other may still reach them.
    fence_before();
    __syncthreads();
    cluster_wait();
    if (warp == kMmaWarp) {
        fence_after();
        tmem_free(s_tmem, 2 * N);
    }
}

// dW (+)= sum over the splits, in order.  A CTA takes 1024 columns of a row.
__global__ void __launch_bounds__(256) ef_wgrad_join_kernel(const float* __restrict__ part, int splits, int C, int J,
                                                            float* __restrict__ out, long long ldo, int accumulate) {
    enter();
    const long long total = (long long)C * J, row = blockIdx.x;
    const float* const p = part + row * J;
    float* const o = out + row * ldo;
    const int j0 = blockIdx.y * 1024 + threadIdx.x;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = 0; s < splits; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) if (j0 + 256 * i < J) v[i] += p[s * total + j0 + 256 * i];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (j0 + 256 * i < J) o[j0 + 256 * i] = accumulate ? o[j0 + 256 * i] + v[i] : v[i];
}

// dY as `terms` stacked bf16 matrices [terms * rows_pad][pitch] whose sum it is, the smallest first (the running sum is cut at
// each step: small terms on top of a large sum put 64 fp32 tokens 3.9e-7 off in the 2-norm, below it 5.7e-8); rows and
// columns past the end are 0.  A warp per 256-column segment.
template <class T, bool ALIGNED, int TERMS>
__global__ void __launch_bounds__(256) ef_wgrad_terms_kernel(const T* __restrict__ dy, long long ld, long long n, int J,
                                                             long long rows_pad, int pitch, __nv_bfloat16* __restrict__ out) {
    using O = Own<T, ALIGNED>;
    const int lane = threadIdx.x & 31, segs = (pitch + kSeg - 1) / kSeg;
    const long long item = (long long)blockIdx.x * 8 + (threadIdx.x >> 5), row = item / segs;
    if (row >= rows_pad) return;
    enter();
    const int s = (int)(item - row * segs) * kSeg;
    V8 v = {both(0.f), both(0.f), both(0.f), both(0.f)};
    if (row < n) {
        Raw8<T> raw;
        load_raw<T, ALIGNED>(dy + row * ld, s, lane, J, raw);
        up8<T>(raw, v);
    }
    float* const f = reinterpret_cast<float*>(v);
#pragma unroll
    for (int t = 0; t < TERMS; ++t) {
        __nv_bfloat16* const o = out + ((TERMS - 1 - t) * rows_pad + row) * pitch;
        __align__(16) __nv_bfloat16 h[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            h[k] = __float2bfloat16_rz(f[k]);              // cut, so that 8 bits go to each term and none overflows
            const float g = __bfloat162float(h[k]);
            f[k] = f[k] == g ? 0.f : f[k] - g;             // also of an infinity
        }
        if constexpr (O::kHalf) {
            const int c = s + O::col(lane, 0);
            if (c < pitch) *reinterpret_cast<uint4*>(o + c) = *reinterpret_cast<const uint4*>(h);
        } else if constexpr (O::kQuad) {
#pragma unroll
            for (int k = 0; k < 8; k += 4) {
                const int c = s + O::col(lane, k);
                if (c < pitch) *reinterpret_cast<uint2*>(o + c) = *reinterpret_cast<const uint2*>(h + k);
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int c = s + O::col(lane, k);
                if (c < pitch) o[c] = h[k];
            }
        }
    }
}

// ---- host --------------------------------------------------------------------------------------
struct Plan {
    int tile_n = 0, splits = 1, terms = 1;
    int64_t tiles = 0, blocks_n = 0, blocks = 0, rows_pad = 0, pitch_j = 0;
    size_t off_terms = 0, total = 0;
};

constexpr int kPairs = efh::kSMs / 2;
constexpr double kStageNs[2] = {420, 500}, kTileNs[2] = {4200, 5800};          // of 256 x 128 and 256 x 256

Plan plan_of(int32_t type, int64_t n, int64_t c, int64_t j, bool direct) {
    Plan p;
    p.terms = type == EF_TYPE_F32 ? 3 : (type == EF_TYPE_F16 ? 2 : 1);
    p.blocks_n = (n + kTileK - 1) / kTileK;
    p.blocks = p.blocks_n * p.terms;
    // Tile width and splits by what they are expected to cost, in ns: a pair takes kStageNs per stage and kTileNs
    // around them (set-up, first loads, and storing 128 x N sums per CTA at about 25 bytes a clock),
    // the join reads the partial sums from L2.
    double best = 0;
    for (const int tn : {256, 128}) {
        const int64_t tiles = (c + 2 * kTileM - 1) / (2 * kTileM) * ((j + tn - 1) / tn);
        const int64_t most = std::max<int64_t>(1, std::min<int64_t>({kMaxSplits, p.blocks / 4, kPairs / std::max<int64_t>(1, tiles)}));
        for (int64_t s = 1; s <= most; ++s) {
            const double waves = (double)((tiles * s + kPairs - 1) / kPairs);
            const double cost = waves * ((double)((p.blocks + s - 1) / s) * kStageNs[tn == 256] + kTileNs[tn == 256]) +
                                (s > 1 ? 2500. + (double)s * (double)(c * j) / 1000. : 0.);
            if (best == 0 || cost < best) {
                best = cost;
                p.tile_n = tn; p.splits = (int)s; p.tiles = tiles;
            }
        }
    }
    size_t o = 0;
    if (p.splits > 1) o += efh::align_up((size_t)p.splits * (size_t)c * (size_t)j * sizeof(float));
    p.off_terms = o;
    p.rows_pad = p.blocks_n * kTileK;
    p.pitch_j = (j + 7) / 8 * 8;
    if (!direct) o += efh::align_up((size_t)p.terms * (size_t)p.rows_pad * (size_t)p.pitch_j * 2);
    p.total = o;
    return p;
}

bool reads_direct(int32_t type, const void* dy, int64_t ldy) {
    return type == EF_TYPE_BF16 && efh::aligned16(dy) && ldy % 8 == 0 && ldy < (int64_t)1 << 39;      // TMA strides: below 2^40 bytes
}

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled() {
    static EncodeTiled f = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r) != cudaSuccess ||
            r != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return f;
}

// Map of a matrix of rows x cols elements, rows stride bytes apart, read in boxes of kTileK rows x box columns;
// what lies outside reads as 0.
bool encode_map(CUtensorMap* map, CUtensorMapDataType type, const void* p, int64_t cols, int64_t rows, int64_t stride,
                unsigned box, CUtensorMapSwizzle swizzle) {
    const EncodeTiled encode = encode_tiled();
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride};
    const cuuint32_t boxes[2] = {box, kTileK}, steps[2] = {1, 1};
    return encode && encode(map, type, 2, const_cast<void*>(p), dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int N>
int launch_wgrad(const WgradArgs& a, const CUtensorMap& codes, const CUtensorMap& dy, int64_t grid, cudaStream_t st) {
    static bool raised[64] = {};
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return EF_ERR_CUDA;
    if (!raised[dev]) {
        if (cudaFuncSetAttribute(ef_wgrad_kernel<N>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kWgradSmem<N>) !=
            cudaSuccess)
            return EF_ERR_CUDA;
        raised[dev] = true;
    }
    return efh::launch(ef_wgrad_kernel<N>, (unsigned)grid, kThreadsW, kWgradSmem<N>, st, 0, a, codes, dy);
}

}  // namespace

extern "C" {

int ef_checkpoint_weight_grad_workspace_bytes(int32_t type, int64_t n, int64_t c, int64_t j, const void* dy,
                                              int64_t lddy, size_t* bytes) {
    if (!bytes || !efh::type_ok(type) || n < 0 || c < 1 || j < 1 || lddy < j) return EF_ERR_INVALID_ARG;
    if (n > (int64_t)1 << 31 || c > (int64_t)1 << 24 || j > (int64_t)1 << 24) return EF_ERR_TOO_LARGE;
    *bytes = plan_of(type, n, c, j, reads_direct(type, dy, lddy)).total;
    return EF_OK;
}

int ef_checkpoint_weight_grad(int32_t type, int64_t n, int64_t c, int64_t j, const int8_t* codes, const float* scales,
                              const void* dy, int64_t lddy, float* dw, int64_t lddw, int32_t accumulate, void* workspace,
                              size_t workspace_bytes, void* cuda_stream) {
    EF_API_RANGE();
    size_t need = 0;
    if (const int rc = ef_checkpoint_weight_grad_workspace_bytes(type, n, c, j, dy, lddy, &need)) return rc;
    if (!dw || lddw < j) return EF_ERR_INVALID_ARG;
    if ((uintptr_t)dw & 3u) return EF_ERR_ALIGNMENT;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (n == 0) {                                        // the empty sum
        if (const int rc = efh::check_device()) return rc;
        if (accumulate) return EF_OK;
        return cudaMemset2DAsync(dw, (size_t)lddw * 4, 0, (size_t)j * 4, (size_t)c, st) == cudaSuccess ? EF_OK : EF_ERR_CUDA;
    }
    if (!codes || !scales || !dy) return EF_ERR_INVALID_ARG;
    const bool direct = reads_direct(type, dy, lddy);
    const Plan p = plan_of(type, n, c, j, direct);
    if (need && (!workspace || workspace_bytes < need)) return EF_ERR_WORKSPACE;
    if (!efh::natural(Mat{dy, lddy, type}) || !efh::aligned16(codes) || ((uintptr_t)scales & 3u) ||
        ((uintptr_t)workspace & (efh::kAlign - 1)))
        return EF_ERR_ALIGNMENT;
    if (p.blocks > 0x7fffffff / kTileK || p.tiles * p.splits > 0x3fffffff) return EF_ERR_TOO_LARGE;
    if (const int rc = efh::check_device()) return rc;
    const void* src = dy;
    int64_t ld = lddy, rows = n;
    if (!direct) {
        __nv_bfloat16* t = reinterpret_cast<__nv_bfloat16*>((char*)workspace + p.off_terms);
        const int64_t items = p.rows_pad * ((p.pitch_j + kSeg - 1) / kSeg);
        if (items / 8 >= 0x7fffffff) return EF_ERR_TOO_LARGE;
        const bool aligned = efh::vectors16(Mat{dy, lddy, type}, j);
        auto go = [&](auto value, auto terms) {
            using T = decltype(value);
            constexpr int K = decltype(terms)::value;
            const unsigned grid = (unsigned)((items + 7) / 8);
            return efh::launch(aligned ? ef_wgrad_terms_kernel<T, true, K> : ef_wgrad_terms_kernel<T, false, K>, grid, 256, 0, st, 0,
                               (const T*)dy, (long long)lddy, (long long)n, (int)j, (long long)p.rows_pad, (int)p.pitch_j, t);
        };
        if (const int rc = type == EF_TYPE_F32   ? go(float{}, std::integral_constant<int, 3>{})
                           : type == EF_TYPE_F16 ? go(__half{}, std::integral_constant<int, 2>{})
                                                 : go(__nv_bfloat16{}, std::integral_constant<int, 1>{}))
            return rc;
        src = t;
        ld = p.pitch_j;
        rows = p.rows_pad * p.terms;
    }
    const int64_t pitch = EF_CHECKPOINT_PITCH(c);
    CUtensorMap map_codes, map_dy;
    if (!encode_map(&map_codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, codes, pitch, n, pitch, kTileM, CU_TENSOR_MAP_SWIZZLE_NONE) ||
        !encode_map(&map_dy, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, src, j, rows, ld * 2, 64, CU_TENSOR_MAP_SWIZZLE_128B))
        return EF_ERR_CUDA;

    WgradArgs a = {};
    a.scales = scales; a.n = n; a.C = (int)c; a.J = (int)j;
    a.groups = (int)EF_CHECKPOINT_GROUPS(c);
    a.blocks_n = (int)p.blocks_n; a.blocks = (int)p.blocks; a.splits = p.splits;
    a.out = p.splits > 1 ? (float*)workspace : dw;
    a.ldo = lddw; a.accumulate = accumulate != 0; a.wait_limit = efh::wait_limit();
    const int64_t grid = 2 * p.tiles * p.splits;
    if (const int rc = p.tile_n == 256 ? launch_wgrad<256>(a, map_codes, map_dy, grid, st)
                                                 : launch_wgrad<128>(a, map_codes, map_dy, grid, st)) return rc;
    if (p.splits > 1) {
        return efh::launch(ef_wgrad_join_kernel, dim3((unsigned)c, (unsigned)((j + 1023) / 1024)), 256, 0, st, 0,
                           (const float*)workspace, p.splits, (int)c, (int)j, dw, (long long)lddw, a.accumulate);
    }
    return EF_OK;
}

}  // extern "C"
