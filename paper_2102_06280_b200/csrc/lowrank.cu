// Low-rank adapters of many workers beside one shared projection (dbw_lowrank_forward, dbw_lowrank_backward).
//
//   forward    hidden = x A_w^T                     y  = x W^T + bias + scale hidden B_w
//   backward   u = scale dy B_w^T                   dx = dy W + u A_w        dA_w = u^T x        dB_w = scale hidden^T dy
//
// in three kinds of kernel: `shrink` (a long row times the worker's factor: hidden and u), `outer` (the factors' gradients) and
// the projection, whose tiles take the adapter's share along as further steps of their k loop.  All three multiply 16-bit
// operands on the tensor cores.  x, dy and W are bf16 as they are; an fp32 value v enters as pieces that are bf16 numbers,
//   v = h + m + l + rest,  h = bf16(v), m = bf16(v - h), l = bf16(v - h - m),  |rest| <= 2^-27 |v|
// (each difference is exact), so its product with a bf16 value is the fp32 one up to 2^-27.  Where the result is fp32 (hidden, u, dA, dB) the pieces are
// of 2^24 v: unscaled, l would fall below the smallest bf16 number for |v| < 2^-110.  From 2^104 on the scaled v, or a sum, is infinite or NaN, as it
// is where an operand is: such a result is summed again on the CUDA cores, in fp32 from the values as they are.
#include <cuda_bf16.h>

#include <algorithm>

#include "common.cuh"
#include "rows.cuh"
#include "tc_ptx.cuh"

namespace dbw {

namespace {

typedef __nv_bfloat16 bf16;
using namespace ptx;

constexpr int BM = 128, BK = 64;  // rows of an operand tile, and its depth: 128 bytes, one swizzled row
constexpr uint32_t kSpinLimit = 1u << 24;

// The two halves of dependent_begin().  A kernel that allocates tensor memory waits for the kernel before it first (so it holds none that
// that kernel may still need), and lets the next one take its places only after all its blocks have theirs.  All is read by plain loads (rows.cuh).
__device__ __forceinline__ void dependent_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void prefetch_map(const CUtensorMap* m) { asm volatile("prefetch.tensormap [%0];" ::"l"(m) : "memory"); }
__device__ __forceinline__ void dependents_may_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ----------------------------------------------------------------------------- pieces, and the 16 x 8 x 16 product of a warp
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// The first `n` pieces of two neighbours, packed.
template <int n>
__device__ __forceinline__ void pieces(float a, float b, uint32_t (&p)[n]) {
#pragma unroll
    for (int i = 0; i < n; ++i) {
        p[i] = pack2(a, b);
        a -= __uint_as_float(p[i] << 16);
        b -= __uint_as_float(p[i] & 0xffff0000u);
    }
}
constexpr float kScale = 16777216.f, kUnscale = 1.f / kScale;
__device__ __forceinline__ bool finite(float x) { return fabsf(x) < INFINITY; }
// Sum of f_k v_k over k < width (a multiple of 8; both begin at multiples of 16 bytes).  A warp.  NaN stays NaN: it goes no further then, here and below
// (8192 rows, 4096 <- 4096, rank 64, all workers diverged: 5.8 ms for the backward pass, 11.4 with sums to the end).
__device__ __noinline__ float dot_again(const float* f, const bf16* v, int width) {
    float sum = 0.f;
    for (int k0 = 0; k0 < width && !__any_sync(0xffffffffu, sum != sum); k0 += 256) {
        const int k = k0 + 8 * (threadIdx.x & 31);
        if (k >= width) continue;
        const uint4 u = *reinterpret_cast<const uint4*>(v + k);
        const uint32_t b[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 x = *reinterpret_cast<const float2*>(f + k + 2 * e);
            sum = fmaf(x.x, __uint_as_float(b[e] << 16), sum);
            sum = fmaf(x.y, __uint_as_float(b[e] & 0xffff0000u), sum);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    return sum;
}
// Sum of c_t v_t over n rows, one value of each.  A thread (its neighbours in a warp take the next v).
__device__ __noinline__ float column_again(const float* c, int rank, const bf16* v, long long ld_v, int n) {
    float sum = 0.f;
    for (int t0 = 0; t0 < n && sum == sum; t0 += 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int t = t0 + i;
            if (t < n) sum = fmaf(c[(size_t)t * rank], __bfloat162float(v[(size_t)t * ld_v]), sum);
        }
    }
    return sum;
}

// d += a b, a 16 x 16 (row major) and b 16 x 8 (column major) of bf16.  Lane l holds of a the values at rows l/4 (registers 0 and 2) and l/4 + 8
// (1 and 3), k 2(l%4) and the one behind it (0 and 1; 8 further: 2 and 3); of b those at column l/4 and the same k; of d rows l/4
// and l/4 + 8, columns 2(l%4) and the one behind it.  The k of a product are summed, so any order of them will do, the same in a and b.
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t map_to_block(uint32_t smem_addr, uint32_t rank) {  // the same place in block `rank` of the cluster
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void store_to(uint32_t cluster_addr, float v) { asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(cluster_addr), "f"(v) : "memory"); }
__device__ __forceinline__ void store_to(uint32_t cluster_addr, float a, float b, float c, float d) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(cluster_addr), "f"(a), "f"(b), "f"(c), "f"(d) : "memory");
}
// The sum, in the order of the blocks, of the floats that the `n` (2 to 8) blocks of the cluster have at this place of their shared memory.  The
// loads are on their way together: one after another they take 0.2 us each.
__device__ __forceinline__ float sum_of_cluster(const float* p, int n) {
    float v[8];
#pragma unroll
    for (int s = 0; s < 8; ++s)
        if (s < n) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[s]) : "r"(map_to_block(smem_u32(p), s)) : "memory");
    float sum = v[0];
#pragma unroll
    for (int s = 1; s < 8; ++s)
        if (s < n) sum += v[s];
    return sum;
}

// ----------------------------------------------------------------------------- shrink, few rows to a worker
// c_t = factor (F_w v_t) for the rows t of worker w: F_w [rank][width] fp32 at f_off of the worker's row of X, v_t bf16.
//
// A block takes 16 rows of one worker.  Its eight warps share the width in steps of 32 by turns (a block reads 512 bytes of every row
// per turn) and keep sums of all its rows x rank; the warps' sums, and those of the blocks of a cluster (which split the width where
// there are few rows), are added in a fixed order.  Of 32 consecutive k a lane takes the eight at 8 (lane % 4), 16 bytes of a row and 32 of the
// factor straight from global memory into the operands' registers (the order of k is free), and forms the factor's pieces there.
//
// What bounds it is reading the factors, and with so little of them the way there and the joining of the sums: 100 rows of 52 workers, width 4096,
// rank 16 (13.6 MB of factors, 2.1 us of the memory): 14 us.
constexpr int kShrinkWarps = 8, kShrinkThreads = 32 * kShrinkWarps;
__host__ __device__ constexpr size_t shrink_smem(int nt) { return (size_t)(kShrinkWarps / 2) * nt * 128 * sizeof(float); }

template <int NT>
__global__ void __launch_bounds__(kShrinkThreads) shrink_kernel(RowGroups g, const float* X, long long ld, long long f_off, int rank, int width,
                                                                const bf16* v, long long ld_v, float factor, float* out, int splits) {
    dependent_begin();
    extern __shared__ float part[];  // [kShrinkWarps / 2][NT * 4 * 32]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, q = lane & 3, row = lane >> 2;
    const int tile = blockIdx.x / splits, split = blockIdx.x % splits;  // split: this block's place in its cluster
    if (blockIdx.x == 0) check_groups(g);
    int2 range;
    const int w = find_tile(g, 16, tile, range);
    if (w < 0) return;  // the whole cluster
    const float* F = X + (size_t)w * ld + f_off;
    // this block's share of the factor on its way to L2 at once: turn by turn, a block waited for memory in each (16 ranks of 1024 values: 10 us)
    {
        const int turns = (width + kShrinkWarps * 32 - 1) / (kShrinkWarps * 32);  // of 1 KB of a row
        for (int e = threadIdx.x; e < rank * turns * 8; e += kShrinkThreads) {
            const int j = e / (turns * 8), line = e % (turns * 8), k = line * 32;
            if (line / 8 % splits == split && k < width) prefetch_l2(F + (size_t)j * width + k);
        }
    }

    float acc[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][e] = 0.f;
    const bf16* at[2];  // this lane's rows
#pragma unroll
    for (int i = 0; i < 2; ++i) at[i] = v + (size_t)min(range.x + 8 * i + row, range.y - 1) * ld_v;  // (behind the last: the last again, not stored)
    const uint4 none = make_uint4(0u, 0u, 0u, 0u);
    auto load = [&](int k, uint4 (&a)[2]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) a[i] = k < width ? *reinterpret_cast<const uint4*>(at[i] + k) : none;
    };
    const int stride = splits * kShrinkWarps * 32;
    int k = (split * kShrinkWarps + warp) * 32 + 8 * q;
    const int k_end = (width + 31) / 32 * 32 + 8 * q;  // the same number of turns for all lanes of a warp
    uint4 now[2], next[2];
    load(k, now);
    for (; k < k_end; k += stride) {
        load(k + stride, next);
        float4 f[NT][2];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const bool in = 8 * j + row < rank && k < width;
            const float4* p = reinterpret_cast<const float4*>(F + (size_t)(8 * j + row) * width + k);
            f[j][0] = in ? *p : make_float4(0.f, 0.f, 0.f, 0.f);
            f[j][1] = in ? p[1] : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            float sum[4] = {0.f, 0.f, 0.f, 0.f};  // of this turn: what the MMAs add up is truncated, so it goes no further than 32 k
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const float4 x = f[j][half];
                uint32_t b0[3], b1[3];
                pieces(kScale * x.x, kScale * x.y, b0);
                pieces(kScale * x.z, kScale * x.w, b1);
                const uint4 lo = now[0], hi = now[1];
                const uint32_t a[4] = {half ? lo.z : lo.x, half ? hi.z : hi.x, half ? lo.w : lo.y, half ? hi.w : hi.y};
#pragma unroll
                for (int p = 2; p >= 0; --p) mma(sum, a, b0[p], b1[p]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[j][e] += sum[e];
        }
        now[0] = next[0];
        now[1] = next[1];
    }

    // the warps' sums, halved three times, then the cluster's
    constexpr int SIZE = NT * 128;
#pragma unroll
    for (int live = kShrinkWarps / 2; live >= 1; live /= 2) {
        if (warp >= live && warp < 2 * live)
#pragma unroll
            for (int i = 0; i < NT * 4; ++i) part[(warp - live) * SIZE + i * 32 + lane] = (&acc[0][0])[i];
        __syncthreads();
        if (warp < live)
#pragma unroll
            for (int i = 0; i < NT * 4; ++i) (&acc[0][0])[i] += part[warp * SIZE + i * 32 + lane];
        __syncthreads();
    }
    if (splits > 1) {
        if (warp == 0)
#pragma unroll
            for (int i = 0; i < NT * 4; ++i) part[i * 32 + lane] = (&acc[0][0])[i];
        cluster_sync();
        if (split == 0 && warp == 0)
#pragma unroll
            for (int i = 0; i < NT * 4; ++i) (&acc[0][0])[i] = sum_of_cluster(part + i * 32 + lane, splits);
        cluster_sync();
    }
    if (split != 0) return;
    bool odd = false;
    if (warp == 0) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int t = range.x + row + (e >> 1) * 8, r = 8 * j + 2 * q + (e & 1);
                if (t >= range.y || r >= rank) continue;
                if (finite(acc[j][e])) out[(size_t)t * rank + r] = factor * (kUnscale * acc[j][e]);
                else odd = true;
                part[(e >> 1) * (8 * NT * 8) + row * (8 * NT) + r] = acc[j][e];  // [16][8 NT]
            }
    }
    if (!__syncthreads_or(odd)) return;
    for (int e = warp; e < (range.y - range.x) * rank; e += kShrinkWarps) {
        const int t = e / rank, r = e % rank;
        if (finite(part[t * (8 * NT) + r])) continue;
        const float sum = dot_again(F + (size_t)r * width, v + (size_t)(range.x + t) * ld_v, width);
        if (lane == 0) out[(size_t)(range.x + t) * rank + r] = factor * sum;
    }
}

// ----------------------------------------------------------------------------- shrink and outer: what they share
// Both are products of few columns (3 R: the pieces of an fp32 operand side by side, R = rank rounded up to 16) with a 128-row
// operand that is read once, so what bounds them is that reading.  Warp 0 of a block brings the bf16 operand by TMA, one thread of warp 1
// issues the MMAs (cta_group::1, M = 128, N = 3 R), the others read the fp32 operand, form its pieces in shared memory (128-byte
// swizzle) and add up the accumulators: those of h, m and l are columns of their own.  Tensor-memory sums are truncated, not
// rounded, at every MMA (K = 784: -5e-7 of a sum), so the k loop is cut into runs of at most kRun stages, which go to the sets of accumulators
// by turns; who forms pieces moves a run's sums to registers, added there with rounding, before it fills the first stage of the run that
// takes the set next (the MMAs of the runs between are under way meanwhile, and nobody waits).  Sums of one sign, rank 64: 2.3e-7 short at any length
// (with runs as long as the sets allow: 131072 values 3.4e-4, 40000 rows 6.9e-5); 8192 rows, 4096 <- 4096, rank 64: 377 us for the backward pass (370).
// Forming pieces is a chain of loads, roundings, shared-memory writes and a fence, so the warps are four groups and a group fills
// every fourth stage by itself, the one slot of the ring that is its own (all of them on one stage after another: 8192 rows, 4096 wide,
// rank 64: shrink 39 us, outer 57).
constexpr int kFillGroups = 4;
constexpr int kRun = 8;  // stages: 32 MMAs, 512 k
__host__ __device__ constexpr int fill_warps(int R) { return R <= 16 ? 8 : 16; }
__host__ __device__ constexpr int thin_threads(int R) { return 64 + 32 * fill_warps(R); }
__host__ __device__ constexpr int thin_columns(int R) { return R <= 16 ? 256 : 512; }  // of tensor memory: two blocks an SM, or one
__host__ __device__ constexpr int thin_a_stages(int R) { return R <= 16 ? 4 : R <= 32 ? 8 : 7; }  // copies on their way: 64 KB an SM did not cover their latency
__host__ __device__ constexpr int thin_set(int R) { return (3 * R + 31) / 32 * 32; }    // columns of one set
__host__ __device__ constexpr int thin_sets(int R) { return thin_columns(R) / thin_set(R); }
__host__ __device__ constexpr int thin_b_bytes(int R) { return (3 * R + 63) / 64 * 8192; }  // one stage of pieces: 3 R rows of 64 k, or 64 k rows of 3 R
__host__ __device__ constexpr size_t thin_ring(int R) { return (size_t)thin_a_stages(R) * (BM * BK * 2) + (size_t)kFillGroups * thin_b_bytes(R); }
__host__ __device__ constexpr size_t thin_smem(int R) { return thin_ring(R) + 1024 /*alignment*/ + 384 /*barriers*/; }
// kind::f16, D fp32, A and B bf16, M = 128, N = 3 R; bits 15 and 16: A and B MN-major
__host__ __device__ constexpr uint32_t thin_idesc(int R, bool mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (mn ? 3u << 15 : 0u) | ((uint32_t)(3 * R >> 3) << 17) | ((uint32_t)(BM >> 4) << 24);
}
// Three pieces of 2^24 times eight values.
__device__ __forceinline__ void split8(const float4& x, const float4& y, uint4 (&p)[3]) {
    uint32_t a[3], b[3], c[3], d[3];
    pieces(kScale * x.x, kScale * x.y, a);
    pieces(kScale * x.z, kScale * x.w, b);
    pieces(kScale * y.x, kScale * y.y, c);
    pieces(kScale * y.z, kScale * y.w, d);
#pragma unroll
    for (int i = 0; i < 3; ++i) p[i] = make_uint4(a[i], b[i], c[i], d[i]);
}

// A block's shared memory, barriers and tensor memory.
template <int R>
struct Thin {
    static constexpr int STAGES = kFillGroups, A_STAGES = thin_a_stages(R), A_BYTES = BM * BK * 2, B_BYTES = thin_b_bytes(R), SET = thin_set(R), SETS = thin_sets(R);
    static constexpr int FILL_WARPS = fill_warps(R), GROUP_THREADS = 32 * FILL_WARPS / kFillGroups, THREADS = thin_threads(R);
    uint8_t *a, *b;
    // of a stage: its copy is there and has been read, its pieces are there and have been read; of a set: its sums are there, and have been read
    uint64_t *landed, *used, *filled, *empty, *done, *drained, *shutdown;
    static_assert((2 * A_STAGES + 2 * STAGES + 2 * SETS + 1) * 8 + 8 <= 384 && R / 16 <= FILL_WARPS / 4, "room for the barriers; a warp has 16 columns of sums at most");
    volatile uint32_t* abort;
    uint32_t tmem, *status;

    __device__ __forceinline__ void setup(uint8_t* raw, uint32_t* status_word) {
        uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
        a = smem;
        b = smem + A_STAGES * A_BYTES;
        landed = reinterpret_cast<uint64_t*>(smem + thin_ring(R));
        used = landed + A_STAGES;
        filled = used + A_STAGES;
        empty = filled + STAGES;
        done = empty + STAGES;
        drained = done + SETS;
        shutdown = drained + SETS;
        uint32_t* slot = reinterpret_cast<uint32_t*>(shutdown + 1);
        abort = slot + 1;
        status = status_word;
        if (threadIdx.x == 0) {
            *abort = 0u;
            for (int s = 0; s < A_STAGES; ++s) {
                mbar_init(&landed[s], 1);
                mbar_init(&used[s], 1);
            }
            for (int s = 0; s < STAGES; ++s) {
                mbar_init(&filled[s], FILL_WARPS / kFillGroups);
                mbar_init(&empty[s], 1);
            }
            for (int s = 0; s < SETS; ++s) {
                mbar_init(&done[s], 1);
                mbar_init(&drained[s], FILL_WARPS);
            }
            mbar_init(shutdown, 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        if (threadIdx.x >> 5 == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(thin_columns(R)) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
        tmem = *slot;
    }
    // The end, a barrier: returns whether `p` holds for any thread.
    __device__ __forceinline__ bool finish(bool p = false) {
        ptx::tc_fence_before();
        p = __syncthreads_or(p);
        if (threadIdx.x >> 5 == 1) {
            ptx::tc_fence_after();
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(thin_columns(R)) : "memory");
        }
        return p;
    }
    __device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity) const {
        return ptx::mbar_try_wait<false>(bar, parity) || ptx::mbar_wait_bounded<false>(bar, parity, kSpinLimit, 0, abort, status);
    }
    __device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity, unsigned pause_ns) const {
        bool ok = true;
        if ((threadIdx.x & 31) == 0) ok = ptx::mbar_wait_bounded<false>(bar, parity, kSpinLimit / 4, pause_ns, abort, status);
        return __all_sync(0xffffffffu, ok);
    }
    static __device__ __forceinline__ int run_of(int n) { return min(kRun, (n + SETS - 1) / SETS); }  // stages of a run, of n in all
    // The MMAs of `n` stages, from ring position `it` and run number `rt` on.  One thread.
    template <bool MN>
    __device__ __forceinline__ bool multiply(int it, int& rt, int n) const {
        const uint64_t da = MN ? mnmajor_sw128_desc(smem_u32(a), 8192) : kmajor_sw128_desc(smem_u32(a));
        const uint64_t db = MN ? mnmajor_sw128_desc(smem_u32(b), 8192) : kmajor_sw128_desc(smem_u32(b));
        constexpr uint64_t STEP = (MN ? 16 * 128 : 16 * 2) / 16;  // 16 further along k: 16 rows of 128 bytes, or 32 bytes inside the swizzle atom
        const int run = run_of(n);
        for (int i = 0, in_set = 0, set = 0; i < n; ++i, ++it) {
            const int sa = it % A_STAGES, s = it % STAGES;
            if (in_set == 0) {
                set = rt % SETS;
                if (rt >= SETS && !wait(&drained[set], ((rt / SETS) - 1) & 1)) return false;
            }
            if (!wait(&landed[sa], (it / A_STAGES) & 1) || !wait(&filled[s], (it / STAGES) & 1)) return false;
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < BK / 16; ++k)
                tc_mma_bf16(tmem + set * SET, da + (uint64_t)(sa * (A_BYTES / 16)) + k * STEP, db + (uint64_t)(s * (B_BYTES / 16)) + k * STEP, thin_idesc(R, MN), in_set > 0 || k > 0);
            tc_commit(&empty[s]);
            tc_commit(&used[sa]);
            if (++in_set == run || i == n - 1) {
                tc_commit(&done[set]);
                in_set = 0;
                ++rt;
            }
        }
        return true;
    }
    // Adds the sums of run `rt` to v: columns [16 g, 16 g + 16) of the operand that was split, g being the warp's number in its lane quarter (none
    // behind the last).  A warp that forms pieces, all lanes; false: a wait ran out.
    __device__ __forceinline__ bool drain(int rt, float (&v)[16]) const {
        const int set = rt % SETS, g = (int)(threadIdx.x >> 5) - 2 >> 2;
        if (!wait_warp(&done[set], (rt / SETS) & 1, 64)) return false;
        ptx::tc_fence_after();
        if (g < R / 16) {
            const uint32_t at = tmem + ((threadIdx.x >> 5 & 3u) << 21) + set * SET + 16 * g;
            uint32_t r[16];
            float sum[16];
            tc_ld16(at + 2 * R, r);
#pragma unroll
            for (int j = 0; j < 16; ++j) sum[j] = __uint_as_float(r[j]);
            tc_ld16(at + R, r);
#pragma unroll
            for (int j = 0; j < 16; ++j) sum[j] += __uint_as_float(r[j]);
            tc_ld16(at, r);
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] += sum[j] + __uint_as_float(r[j]);
        }
        ptx::tc_fence_before();
        __syncwarp();
        if ((threadIdx.x & 31) == 0) ptx::mbar_arrive(&drained[set]);
        return true;
    }
};

// Shutdown of the copying thread after an expired wait: the copies still in flight have landed before the block leaves.
template <int R>
__device__ __forceinline__ void land(const Thin<R>& x, int issued) {
    for (int j = max(0, issued - Thin<R>::A_STAGES); j < issued; ++j) ptx::mbar_wait_quiet<false>(&x.landed[j % Thin<R>::A_STAGES], (j / Thin<R>::A_STAGES) & 1, 1u << 20);
}

// ----------------------------------------------------------------------------- shrink, many rows
// c_t = factor (F_w v_t) as above, 128 rows of one worker to a block (rows of others may come along in its copies: every row of the product
// is its own, theirs are not stored).  The blocks of a cluster share the width.
// 8192 rows, 4096 wide, rank 16: 20 us (67 MB of rows, 10.2 us of the memory; 3.4 TB/s); rank 64: 34 us, where forming the pieces is as long.
template <int R>
__global__ void __launch_bounds__(thin_threads(R)) shrink_tc_kernel(const __grid_constant__ CUtensorMap map_v, RowGroups g, const float* X, long long ld, long long f_off,
                                                                 int rank, int width, const bf16* rows_v, long long ld_v, float factor, float* out, int splits) {
    using T = Thin<R>;
    extern __shared__ uint8_t raw[];
    if (threadIdx.x == 0) prefetch_map(&map_v);
    dependent_wait();
    if (blockIdx.x == 0) check_groups(g);
    int2 range;
    const int w = find_tile(g, BM, blockIdx.x / splits, range);
    if (w < 0) return;  // the whole cluster
    T x;
    x.setup(raw, g.status);
    dependents_may_start();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, split = blockIdx.x % splits;
    const float* F = X + (size_t)w * ld + f_off;
    const int all = (width + BK - 1) / BK, kb0 = (int)((long long)all * split / splits), n = (int)((long long)all * (split + 1) / splits) - kb0;
    bool live = true;
    float v[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = 0.f;
    if (warp == 0) {
        if (lane == 0) {
            int i = 0;
            for (; i < n && live; ++i) {
                const int s = i % T::A_STAGES;
                if (i >= T::A_STAGES && !x.wait(&x.used[s], ((i / T::A_STAGES) - 1) & 1)) {
                    live = false;
                    break;
                }
                ptx::mbar_expect_tx(&x.landed[s], T::A_BYTES);
                tma_load_2d(x.a + s * T::A_BYTES, &map_v, (kb0 + i) * BK, range.x, &x.landed[s]);
            }
            if (!live) land(x, i);
        }
    } else if (warp == 1) {
        int rt = 0;
        if (lane == 0 && !x.template multiply<false>(0, rt, n)) {
            tc_commit(x.shutdown);
            ptx::mbar_wait_quiet<false>(x.shutdown, 0, 1u << 20);
        }
    } else {
        const int group = (warp - 2) % kFillGroups, tid = (warp - 2) / kFillGroups * 32 + lane;
        constexpr int PER = R * 8 / T::GROUP_THREADS;  // pieces of 8 k of a thread
        float4 f[PER][2];
        auto load = [&](int i, int e) {
            const int at = tid + e * T::GROUP_THREADS, j = at >> 3, k = (kb0 + i) * BK + 8 * (at & 7);
            const bool in = i < n && j < rank && k < width;
            const float4* p = reinterpret_cast<const float4*>(F + (size_t)j * width + k);
            f[e][0] = in ? *p : make_float4(0.f, 0.f, 0.f, 0.f);
            f[e][1] = in ? p[1] : make_float4(0.f, 0.f, 0.f, 0.f);
        };
#pragma unroll
        for (int e = 0; e < PER; ++e) load(group, e);
        const int run = T::run_of(n);
        int rt = 0;
        for (int i = group; i < n; i += kFillGroups) {
            const int s = i % T::STAGES;
            for (; live && i >= (rt + T::SETS) * run; ++rt) live = x.drain(rt, v);
            if (live && i >= T::STAGES) live = x.wait_warp(&x.empty[s], ((i / T::STAGES) - 1) & 1, 32);
            if (!live) break;
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                const int at = tid + e * T::GROUP_THREADS, j = at >> 3, k8 = at & 7;
                uint4 p[3];
                split8(f[e][0], f[e][1], p);
                load(i + kFillGroups, e);
#pragma unroll
                for (int q = 0; q < 3; ++q) {
                    const int row = q * R + j;
                    *reinterpret_cast<uint4*>(x.b + s * T::B_BYTES + row * 128 + ((k8 ^ (row & 7)) * 16)) = p[q];
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&x.filled[s]);
        }
        for (; live && rt * run < n; ++rt) live = x.drain(rt, v);
    }
    // ---- sums: every block of the cluster gets its share of the rows from all of them, over the ring, adds it up and writes it ----
    // (loads from the other blocks instead, one behind the other, took 8 us of 35 at rank 64)
    __syncthreads();
    if (splits > 1) cluster_sync();  // every MMA of the cluster has been waited for: nobody reads a ring
    constexpr int PITCH = R + 4;     // four floats a lane at this pitch meet all banks
    float* sums = reinterpret_cast<float*>(x.a);  // [splits][share][PITCH]
    const int share = BM / splits;
    if (warp >= 2) {
        const int row = (warp & 3) * 32 + lane;
        const uint32_t to = map_to_block(smem_u32(sums + (split * share + row % share) * PITCH), row / share);
        const int group = (warp - 2) >> 2;
        if (group < R / 16)
#pragma unroll
            for (int j = 0; j < 16; j += 4) store_to(to + (16 * group + j) * 4, v[j], v[j + 1], v[j + 2], v[j + 3]);
    }
    if (splits > 1) cluster_sync();
    else __syncthreads();
    auto sum_of = [&](int i, int j) {
        float sum = sums[i * PITCH + j];
        for (int k = 1; k < splits; ++k) sum += sums[(k * share + i) * PITCH + j];
        return sum;
    };
    bool odd = false;
    const int first = range.x + split * share;
    for (int e = threadIdx.x; e < share * R; e += T::THREADS) {
        const int i = e / R, j = e % R;
        if (first + i >= range.y || j >= rank) continue;
        const float sum = sum_of(i, j);
        if (finite(sum)) out[(size_t)(first + i) * rank + j] = factor * (kUnscale * sum);
        else odd = true;
    }
    if (x.finish(odd))
        for (int e = warp; e < min(share, range.y - first) * rank; e += T::THREADS / 32) {
            const int i = e / rank, j = e % rank;
            if (finite(sum_of(i, j))) continue;
            const float sum = dot_again(F + (size_t)j * width, rows_v + (size_t)(first + i) * ld_v, width);
            if (lane == 0) out[(size_t)(first + i) * rank + j] = factor * sum;
        }
}

// ----------------------------------------------------------------------------- outer
// dF_w = factor sum_t c_t v_t^T over the rows t of worker w, for every worker (zeros without rows), fp32 into G; both factors in one launch.
//
// An item is 128 columns of one factor of one worker: v's rows are the MMA's k, 64 to a stage, v's columns its 128 rows (MN-major, no
// transposition anywhere), the pieces of c its columns.  Rows behind the worker's last are zeros in c and, since they
// may hold anything, are made zeros in v's last stage too.  Where there are fewer items than SMs the blocks of a cluster share an item's rows
// and add their sums in a fixed order; otherwise a block walks items.
// Both factors of a projection 4096 -> 4096, 8192 rows, rank 64: 69 us (134 MB of rows, 20.5 us of the memory; forming the pieces of
// c anew for every 128 columns is what it spends the rest on).  With a launch for each factor, backwards of little work took 5 to 8 us more.
struct OuterJobs {  // of the one factor, and of the other
    long long f_off[2];
    int width[2];
    float factor[2];
    const float* c[2];
    const bf16* v[2];
    long long ld_v[2];
};
template <int R>
__global__ void __launch_bounds__(thin_threads(R)) outer_tc_kernel(const __grid_constant__ CUtensorMap map_0, const __grid_constant__ CUtensorMap map_1, RowGroups g, float* G,
                                                                long long ld, int rank, const __grid_constant__ OuterJobs jobs, int splits) {
    using T = Thin<R>;
    extern __shared__ uint8_t raw[];
    T x;
    if (threadIdx.x == 0 && g.rows > 0) {
        prefetch_map(&map_0);
        prefetch_map(&map_1);
    }
    dependent_wait();
    x.setup(raw, g.status);
    dependents_may_start();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, split = blockIdx.x % splits, first = blockIdx.x / splits, stride = gridDim.x / splits;
    const int parts_0 = (jobs.width[0] + BM - 1) / BM, parts = parts_0 + (jobs.width[1] + BM - 1) / BM, items = g.N * parts;  // of one worker: both factors' columns
    auto job_of = [&](int item) { return item % parts >= parts_0 ? 1 : 0; };
    auto column_of = [&](int item) { return (item % parts - (item % parts >= parts_0 ? parts_0 : 0)) * BM; };
    // of an item: its rows, and how many stages of them are this block's (number split, split + splits, ...)
    auto stages = [&](const int2& r) {
        const int all = (r.y - r.x + BK - 1) / BK;
        return all > split ? (all - split + splits - 1) / splits : 0;
    };
    int it = 0, rt = 0;
    bool live = true;
    float v[16];
    if (warp == 0) {
        if (lane == 0) {
            for (int item = first; item < items && live; item += stride) {
                const int2 r = rows_of(g, item / parts);
                const int n = stages(r), col0 = column_of(item);
                const CUtensorMap* map = job_of(item) ? &map_1 : &map_0;
                for (int i = 0; i < n; ++i, ++it) {
                    const int s = it % T::A_STAGES;
                    if (it >= T::A_STAGES && !x.wait(&x.used[s], ((it / T::A_STAGES) - 1) & 1)) {
                        live = false;
                        break;
                    }
                    ptx::mbar_expect_tx(&x.landed[s], T::A_BYTES);
#pragma unroll
                    for (int h = 0; h < 2; ++h) tma_load_2d(x.a + s * T::A_BYTES + h * 8192, map, col0 + 64 * h, r.x + (split + i * splits) * BK, &x.landed[s]);
                }
            }
            if (!live) land(x, it);
        }
    } else if (warp == 1) {
        if (lane == 0) {
            for (int item = first; item < items && live; item += stride) {
                const int n = stages(rows_of(g, item / parts));
                live = x.template multiply<true>(it, rt, n);
                it += n;
            }
            if (!live) {
                tc_commit(x.shutdown);
                ptx::mbar_wait_quiet<false>(x.shutdown, 0, 1u << 20);
            }
        }
    } else {
        const int group = (warp - 2) % kFillGroups, tid = (warp - 2) / kFillGroups * 32 + lane;
        constexpr int PER = BK * R / 8 / T::GROUP_THREADS;  // pieces of 8 values of a thread
        const bool wide = (rank & 3) == 0;
        for (int item = first; item < items && live; item += stride) {
            const int w = item / parts, col0 = column_of(item), job = job_of(item), width = jobs.width[job];
            const float* c = jobs.c[job];
            const int2 r = rows_of(g, w);
            const int n = stages(r);
            float4 f[PER][2];
            auto load = [&](int i, int e) {
                const int at = tid + e * T::GROUP_THREADS, t = r.x + (split + i * splits) * BK + at / (R / 8), j = 8 * (at % (R / 8));
                const bool in = i < n && t < r.y;
                const float* p = c + (size_t)t * rank + j;
                if (wide) {
                    f[e][0] = in && j < rank ? *reinterpret_cast<const float4*>(p) : make_float4(0.f, 0.f, 0.f, 0.f);
                    f[e][1] = in && j + 4 < rank ? *(reinterpret_cast<const float4*>(p) + 1) : make_float4(0.f, 0.f, 0.f, 0.f);
                } else {
                    float v[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = in && j + k < rank ? p[k] : 0.f;
                    f[e][0] = make_float4(v[0], v[1], v[2], v[3]);
                    f[e][1] = make_float4(v[4], v[5], v[6], v[7]);
                }
            };
            const int mine = (group - it % kFillGroups + kFillGroups) % kFillGroups;  // the group's first stage of this item
            const int run = T::run_of(n);
            int drained = 0;  // runs of this item
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = 0.f;
#pragma unroll
            for (int e = 0; e < PER; ++e) load(mine, e);
            for (int i = mine; i < n; i += kFillGroups) {
                const int at_ring = it + i, s = at_ring % T::STAGES;
                for (; live && i >= (drained + T::SETS) * run; ++drained) live = x.drain(rt++, v);
                if (live && at_ring >= T::STAGES) live = x.wait_warp(&x.empty[s], ((at_ring / T::STAGES) - 1) & 1, 32);
                if (!live) break;
#pragma unroll
                for (int e = 0; e < PER; ++e) {
                    const int at = tid + e * T::GROUP_THREADS, t = at / (R / 8), j = 8 * (at % (R / 8));
                    uint4 p[3];
                    split8(f[e][0], f[e][1], p);
                    load(i + kFillGroups, e);
#pragma unroll
                    for (int q = 0; q < 3; ++q) {
                        const int col = q * R + j;
                        *reinterpret_cast<uint4*>(x.b + s * T::B_BYTES + (col >> 6) * 8192 + t * 128 + (((col >> 3 & 7) ^ (t & 7)) * 16)) = p[q];
                    }
                }
                const int rows = r.y - (r.x + (split + i * splits) * BK);  // in this stage
                if (rows < BK) {
                    const int sa = at_ring % T::A_STAGES;
                    live = x.wait_warp(&x.landed[sa], (at_ring / T::A_STAGES) & 1, 32);
                    if (!live) break;
                    for (int e = tid; e < (BK - rows) * 16; e += T::GROUP_THREADS)
                        *reinterpret_cast<uint4*>(x.a + sa * T::A_BYTES + (e & 1) * 8192 + (rows + (e >> 4)) * 128 + (e >> 1 & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&x.filled[s]);
            }
            it += n;
            for (; live && drained * run < n; ++drained) live = x.drain(rt++, v);
            if (!live || splits > 1) break;
            const int col = col0 + (warp & 3) * 32 + lane, j0 = 16 * ((warp - 2) >> 2);
            float* to = G + (size_t)w * ld + jobs.f_off[job] + (size_t)j0 * width + col;
            float none = 0.f;  // NaN as soon as a sum is not finite
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                none = fmaf(0.f, v[j], none);
                if (j0 + j < rank && col < width) to[(size_t)j * width] = jobs.factor[job] * (kUnscale * v[j]);
            }
            if (none != 0.f && col < width) {
                uint32_t odd = 0;
#pragma unroll
                for (int j = 0; j < 16; ++j) odd |= j0 + j < rank && !finite(v[j]) ? 1u << j : 0u;
                for (; odd; odd &= odd - 1) {
                    const int j = __ffs(odd) - 1;
                    to[(size_t)j * width] = jobs.factor[job] * column_again(c + (size_t)r.x * rank + j0 + j, rank, jobs.v[job] + (size_t)r.x * jobs.ld_v[job] + col, jobs.ld_v[job], r.y - r.x);
                }
            }
            __syncwarp();
        }
    }
    if (splits > 1) {  // one item for each cluster: every block gets its share of the factor's rows from all, over the ring, adds it up and writes it
        __syncwarp();
        cluster_sync();  // every MMA of the cluster has been waited for: nobody reads a ring
        float* sums = reinterpret_cast<float*>(x.a);  // [splits][share][BM]
        const int share = R / splits;
        if (warp >= 2) {
            const int col = (warp & 3) * 32 + lane, group = (warp - 2) >> 2;
            if (group < R / 16)
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const int r = 16 * group + j;
                    store_to(map_to_block(smem_u32(sums + (split * share + r % share) * BM + col), r / share), v[j]);
                }
        }
        cluster_sync();
        const int w = first / parts, col0 = column_of(first), job = job_of(first), width = jobs.width[job];
        for (int e = threadIdx.x; e < share * BM; e += T::THREADS) {
            const int i = e / BM, k = e % BM, r = split * share + i;
            if (r >= rank || col0 + k >= width) continue;
            float sum = sums[e];
            for (int j = 1; j < splits; ++j) sum += sums[j * share * BM + e];
            if (finite(sum)) {
                sum *= kUnscale;
            } else {
                const int2 own = rows_of(g, w);
                sum = column_again(jobs.c[job] + (size_t)own.x * rank + r, rank, jobs.v[job] + (size_t)own.x * jobs.ld_v[job] + col0 + k, jobs.ld_v[job], own.y - own.x);
            }
            G[(size_t)w * ld + jobs.f_off[job] + (size_t)r * width + col0 + k] = jobs.factor[job] * sum;
        }
    }
    x.finish();
}

// ----------------------------------------------------------------------------- projection
// y_t = W v_t (K-major W [n][k]) or W^T v_t (BMN: W [k][n]) + bias + factor F_w^T c_t, bf16.
//
// Persistent and warp-specialised, in pairs of blocks (tcgen05 cta_group::2): a pair owns tiles of 256 rows x BN columns, each block
// 128 of the rows and, as an operand, half of the columns, so that a step of the k loop brings (128 + BN / 2) x 64 values into each.
// Warp 0 streams tiles of v and W by TMA through a ring of STAGES slots (128-byte swizzle, no multicast; the copies of both blocks
// are counted on the leader's barriers), one thread of the leader's warp 1 issues the MMAs into one of two accumulators in tensor
// memory, warps 2 to 9 drain the finished one.  (8192 rows, 4096 -> 4096: 128 x 256 tiles of single blocks, 48 KB a step for the same products, 293 us;
// in pairs 193 to 212 us with rank 16, by the board, 1.3 to 1.43 PFLOP/s.  No unit is full: tensor cores active 67 % of the cycles, L2 at 40 % of its rate, memory
// at 9 %; that fewer bytes a step made it faster says that it waits for the tiles on their way from L2.)
//
// A tile's rows are the batch's, whosever they are.  The adapters join as further slots, spread over the k loop: for every worker
// with rows in the tile, warps 2 to 9 fill slots with the pieces of factor x c_t (zeros in the rows of others) and of the worker's factor,
//     k:            [0, R)        [R, 2R)      [2R, 3R)         R = rank rounded up to 16
//     rows:         h of c        l of c       h of c           (v = h + l + rest, |rest| <= 2^-17 |v|)
//     columns:      h of F        h of F       l of F
// while the MMAs of the slots before run.  What is left out, l l and the rests, is below 2^-16 of a product; y has 8 bits.  The sums in
// tensor memory stay there over the whole k loop and are truncated at every MMA: of one sign, 8e-8 of the sum for 16 k, 2e-5 at K = 4096 (y's
// half step: 2e-3).
// An infinite or NaN value of one worker's factor must not reach the rows of another through 0 x inf, and of one value's pieces it would make NaN where
// the product is infinite: a value of F, or of factor x c, that is not finite or rounds to infinity enters as zero, and the epilogue adds its products to the
// rows they belong to on the CUDA cores, in fp32.
constexpr int kProjectThreads = 320, kDrainWarps = 8, kDrainThreads = 32 * kDrainWarps;
__host__ __device__ constexpr int project_stages(int bn) { return bn == 256 ? 6 : 8; }
__host__ __device__ constexpr size_t project_stage(int bn) { return (size_t)(BM + bn / 2) * BK * 2; }
__host__ __device__ constexpr size_t project_smem(int bn) { return project_stages(bn) * project_stage(bn) + 1024 /*alignment*/ + 512 /*barriers*/; }

struct ProjectArgs {
    RowGroups g;
    const float* X;      // the workers' rows; F_w [rank][N] at f_off
    long long ld, f_off;
    int rank, N, K;
    float factor;
    const float* c;      // [rows][rank]
    const float* bias;   // [N] or null
    bf16* y;
    long long ld_y;
};

// Bounded waits that share one abort word per block, raised in both blocks of the pair: after one that ran out all return at once.
struct Waits {
    volatile uint32_t* abort;
    uint32_t peer_abort;
    uint32_t* status;
    __device__ __forceinline__ bool operator()(uint64_t* bar, uint32_t parity) const {
        if (ptx::mbar_try_wait<true>(bar, parity)) return true;  // (most often it is complete: nothing else on the MMAs' path)
        if (ptx::mbar_wait_bounded<true>(bar, parity, kSpinLimit, 0, abort, status)) return true;
        asm volatile("st.relaxed.cluster.shared::cluster.u32 [%0], %1;" ::"r"(peer_abort), "r"(1u) : "memory");
        return false;
    }
    // For a whole warp, off the critical path: one lane polls, with pauses (polls take shared-memory cycles from the MMAs' operands).
    __device__ __forceinline__ bool warp(uint64_t* bar, uint32_t parity, unsigned pause_ns) const {
        bool ok = true;
        if ((threadIdx.x & 31) == 0) {
            ok = ptx::mbar_wait_bounded<true>(bar, parity, kSpinLimit / 4, pause_ns, abort, status);
            if (!ok) asm volatile("st.relaxed.cluster.shared::cluster.u32 [%0], %1;" ::"r"(peer_abort), "r"(1u) : "memory");
        }
        return __all_sync(0xffffffffu, ok);
    }
};
// kind::f16, D fp32, A and B bf16, M = 256 (two blocks), N = bn; bit 16: B is MN-major
__host__ __device__ constexpr uint32_t idesc_for(int bn, bool b_mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(bn >> 3) << 17) | ((uint32_t)(2 * BM >> 4) << 24);
}

// The first worker from `w` on with a row before `end`, or -1.  All lanes of a warp, the same arguments.
__device__ __forceinline__ int next_worker(const RowGroups& g, int w, int end) {
    const int lane = threadIdx.x & 31;
    for (; w < g.N; w += 32) {
        const int2 r = w + lane < g.N ? rows_of(g, w + lane) : make_int2(end, end);
        const unsigned some = __ballot_sync(0xffffffffu, r.x < end && r.y > r.x);
        if (some) return w + __ffs(some) - 1;
        if (__any_sync(0xffffffffu, r.x >= end)) break;
    }
    return -1;
}
// The workers with rows in [t0, end), one after another.  All lanes of a warp, the same arguments.  Up to 32 workers are looked at at once.
struct TileWorkers {
    uint32_t mask;  // N <= 32: those that are left
    int next;       // N > 32: the next one, or -1
    __device__ __forceinline__ TileWorkers(const RowGroups& g, int t0, int end) {
        const int lane = threadIdx.x & 31;
        if (g.N <= 32) {
            const int2 r = lane < g.N ? rows_of(g, lane) : make_int2(end, end);
            mask = __ballot_sync(0xffffffffu, r.x < end && r.y > max(r.x, t0));
            next = -1;
        } else {
            mask = 0u;
            next = next_worker(g, max(0, worker_of_row(g, t0)), end);
        }
    }
    __device__ __forceinline__ int count(const RowGroups& g, int end) const {
        if (g.N <= 32) return __popc(mask);
        int n = 0;
        for (int w = next; w >= 0; w = next_worker(g, w + 1, end)) ++n;
        return n;
    }
    __device__ __forceinline__ int take(const RowGroups& g, int end) {  // -1 behind the last
        int w = next;
        if (g.N <= 32) {
            w = __ffs(mask) - 1;
            mask &= mask - 1u;
        } else if (next >= 0) {
            next = next_worker(g, next + 1, end);
        }
        return w;
    }
};

// Whether it holds for any thread of the eight warps that drain; a barrier for them.
__device__ __forceinline__ bool any_of_drain(bool mine) {
    uint32_t any;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %1, 0;\n\tbarrier.red.or.pred p, 1, %2, q;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(any) : "r"((uint32_t)mine), "n"(kDrainThreads) : "memory");
    return any != 0;
}

// Whether f is finite and rounds to a finite bf16 number.
__device__ __forceinline__ bool fits(float f) { return fabsf(f) < 0x1.ffp127f; }
__device__ __forceinline__ float larger(float a, float b) {  // of the magnitudes; NaN if one is
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(fabsf(a)), "f"(fabsf(b)));
    return d;
}
// Makes the values that do not fit 0; returns whether there were any.  (One comparison of the largest of them: with masks for every value and piece
// backward_ragged took 45.8 us instead of 43.7.)
template <int n>
__device__ __forceinline__ bool without_infinities(float4 (&v)[n][2]) {
    float most = 0.f;
#pragma unroll
    for (int x = 0; x < n; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y) most = larger(larger(most, v[x][y].x), larger(v[x][y].y, larger(v[x][y].z, v[x][y].w)));
    if (fits(most)) return false;
#pragma unroll
    for (int x = 0; x < n; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            float4& u = v[x][y];
            u = make_float4(fits(u.x) ? u.x : 0.f, fits(u.y) ? u.y : 0.f, fits(u.z) ? u.z : 0.f, fits(u.w) ? u.w : 0.f);
        }
    return true;
}
// Eight values as a piece: h, or l.  (A value below 2^-116 is held to 2^-134, half the smallest bf16 number: times the other factor that is nothing to
// a bf16 y unless that is 2^100 and more.)
__device__ __forceinline__ uint4 piece8(const float4 (&v)[2], bool low) {
    const float f[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
    uint32_t o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        uint32_t p[2];
        pieces(f[2 * e], f[2 * e + 1], p);
        o[e] = low ? p[1] : p[0];
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
}

template <int BN, bool BMN>
__global__ void __launch_bounds__(kProjectThreads, 1)
project_kernel(const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ ProjectArgs a) {
    constexpr int STAGES = project_stages(BN), BH = BN / 2, A_BYTES = BM * BK * 2, B_BYTES = BH * BK * 2;
    constexpr uint32_t IDESC = idesc_for(BN, BMN), IDESC_MN = idesc_for(BN, true);
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* tiles_a = smem;
    uint8_t* tiles_b = smem + STAGES * A_BYTES;
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + STAGES * (A_BYTES + B_BYTES));
    uint64_t* empty = full + STAGES;
    uint64_t* grant = empty + STAGES;  // a slot is free for the pieces of an adapter (who fills them does not see every use of a slot)
    uint64_t* acc_full = grant + STAGES;
    uint64_t* acc_empty = acc_full + 2;
    uint64_t* drain = acc_empty + 2;  // shutdown after an expired wait: completion of the MMAs issued so far
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
    volatile uint32_t* abort = tmem_slot + 1;
    volatile uint32_t* odd_flag = tmem_slot + 2;  // [3], a tile's by turns: its factors hold values that are not finite
    volatile uint32_t* odd_rows = tmem_slot + 5;  // [3], its c, of this block's rows

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();  // 0 = leader of the pair
    if (threadIdx.x == 0) {
        prefetch_map(&map_v);
        prefetch_map(&map_w);
    }
    if (threadIdx.x == 0) {
        *abort = 0u;
        for (int e = 0; e < 3; ++e) odd_flag[e] = odd_rows[e] = 0u;
        mbar_init(drain, 1);
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(&full[s], 2);  // (the leader's) its copies' arrival and one more, or one for each block's pieces
            mbar_init(&empty[s], 1);
            mbar_init(&grant[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&acc_full[b], 1);
            mbar_init(&acc_empty[b], 2 * kDrainWarps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(2 * BN) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    const Waits wait{abort, map_to_block(smem_u32((const void*)abort), rank ^ 1u), a.g.status};
    // The kernel before this one is one of this file: it writes c or G, everything before it was complete when it let this one start, and it has all its
    // tensor memory.  So only who reads c (and writes y) waits for it.
    dependents_may_start();

    const int first = row_bound(a.g, 0), last = row_bound(a.g, a.g.N);
    const int tiles_n = (a.N + BN - 1) / BN, n_tiles = (max(0, last - first) + 2 * BM - 1) / (2 * BM) * tiles_n;
    const int pair = blockIdx.x / 2, pairs = gridDim.x / 2;
    const int num_kb = (a.K + BK - 1) / BK;
    const int R = (a.rank + 15) / 16 * 16, steps = 3 * R / 16, blocks = (steps + 3) / 4;  // of one worker: k 16 at a time, and ring slots
    // Of a tile's n slots, `extra` are an adapter's, spread evenly: the place of number e.
    auto place = [](int e, int extra, int n) { return e < extra ? ((e + 1) * n + extra - 1) / extra - 1 : n; };

    if (warp == 0) {
        int it = 0;  // ring slots up to here
        uint32_t copies = 0, copy_phase = 0;  // slots that were last copied to, and the parity of that use
        bool live = true;
        for (int tile = pair; tile < n_tiles && live; tile += pairs) {
            const int n0 = (tile % tiles_n) * BN + (int)rank * BH, t0 = first + (tile / tiles_n) * 2 * BM;
            const int extra = blocks * TileWorkers(a.g, t0, min(last, t0 + 2 * BM)).count(a.g, min(last, t0 + 2 * BM)), n = num_kb + extra;
            if (lane == 0) {
                int kb = 0, e = 0, next = place(0, extra, n);
                for (int i = 0; i < n; ++i) {
                    const int j = it + i, s = j % STAGES;
                    if (j >= STAGES && !wait(&empty[s], ((j / STAGES) - 1) & 1)) {
                        live = false;
                        break;
                    }
                    if (i == next) {
                        next = place(++e, extra, n);
                        copies &= ~(1u << s);
                        mbar_arrive(&grant[s]);
                        continue;
                    }
                    copies |= 1u << s;
                    copy_phase = (copy_phase & ~(1u << s)) | (((uint32_t)(j / STAGES) & 1u) << s);
                    if (rank == 0) {
                        mbar_expect_tx(&full[s], 2 * (A_BYTES + B_BYTES));
                        mbar_arrive(&full[s]);
                    }
                    const uint32_t bar = map_to_block(smem_u32(&full[s]), 0);
                    tma_load_2d_pair(tiles_a + s * A_BYTES, &map_v, kb * BK, t0 + (int)rank * BM, bar);
                    if (!BMN) {
                        tma_load_2d_pair(tiles_b + s * B_BYTES, &map_w, kb * BK, n0, bar);
                    } else {
#pragma unroll
                        for (int c = 0; c < BH / 64; ++c) tma_load_2d_pair(tiles_b + s * B_BYTES + c * 8192, &map_w, n0 + c * 64, kb * BK, bar);
                    }
                    ++kb;
                }
            }
            live = __shfl_sync(0xffffffffu, live, 0);
            it += n;
        }
        // after an expired wait: the copies still in flight (the leader counts those of both), the last of each slot at most, have landed before
        // the pair meets at the end
        if (rank == 0 && lane == 0 && *abort)
            for (int s = 0; s < STAGES; ++s)
                if (copies & (1u << s)) mbar_wait_quiet<true>(&full[s], (copy_phase >> s) & 1, 1u << 20);
    } else if (warp == 1) {
        if (rank == 0) {
            const uint64_t desc_a = kmajor_sw128_desc(smem_u32(tiles_a)), desc_mn = mnmajor_sw128_desc(smem_u32(tiles_b), 8192);
            const uint64_t desc_b = BMN ? desc_mn : kmajor_sw128_desc(smem_u32(tiles_b));
            int it = 0, lt = 0;
            bool live = true;
            for (int tile = pair; tile < n_tiles && live; tile += pairs, ++lt) {
                const int t0 = first + (tile / tiles_n) * 2 * BM, buf = lt & 1;
                const int extra = blocks * TileWorkers(a.g, t0, min(last, t0 + 2 * BM)).count(a.g, min(last, t0 + 2 * BM)), n = num_kb + extra;
                if (lane == 0) {
                    if (lt >= 2 && !wait(&acc_empty[buf], ((lt / 2) - 1) & 1)) live = false;
                    tc_fence_after();
                    const uint32_t d = tmem_base + (uint32_t)(buf * BN);
                    int e = 0, next = place(0, extra, n);
                    for (int i = 0; i < n; ++i) {
                        const int j = it + i, s = j % STAGES;
                        if (!wait(&full[s], (j / STAGES) & 1)) {
                            live = false;
                            break;
                        }
                        tc_fence_after();
                        const uint64_t da = desc_a + (uint64_t)(s * (A_BYTES / 16)), db = (i == next ? desc_mn : desc_b) + (uint64_t)(s * (B_BYTES / 16));
                        // 16 further along k: 32 bytes inside the swizzle atom (K-major) or 16 rows of 128 bytes (MN-major)
                        constexpr uint64_t STEP = (BMN ? 16 * 128 : 16 * 2) / 16, STEP_MN = 16 * 128 / 16;
                        if (i != next) {
#pragma unroll
                            for (int k = 0; k < BK / 16; ++k) tc_mma_bf16_pair(d, da + (uint64_t)(k * 2), db + k * STEP, IDESC, i > 0 || k > 0);
                        } else {  // an adapter's
                            const int ks = min(4, steps - 4 * (e % blocks));
                            for (int k = 0; k < ks; ++k) tc_mma_bf16_pair(d, da + (uint64_t)(k * 2), db + k * STEP_MN, IDESC_MN, i > 0 || k > 0);
                            next = place(++e, extra, n);
                        }
                        tc_commit_pair(&empty[s]);  // frees the slot once these MMAs have read it
                    }
                    if (live) tc_commit_pair(&acc_full[buf]);
                    else {  // shutdown after an expired wait: the MMAs issued so far are complete before tensor memory is freed
                        tc_commit_pair(drain);
                        mbar_wait_quiet<true>(drain, 0, 1u << 20);
                    }
                }
                live = __shfl_sync(0xffffffffu, live, 0);
                it += n;
            }
        }
    } else {
        const int tid = threadIdx.x - 64, quarter = warp & 3, half = (warp - 2) >> 2;
        int it = 0, lt = 0;
        uint32_t granted = 0;  // the parity of each slot's next grant
        bool live = true, dead = false;
        const bool wide = (a.rank & 3) == 0;
        dependent_wait();
        float4 raw_c[4][2], raw_f[BH / 32][2];
        int w = -1, b = 0;                               // whose piece it is, and which
        TileWorkers tile_workers(a.g, last, last);       // of the tile that is loaded
        auto load = [&](int tile) {
            const int own_t = first + (tile / tiles_n) * 2 * BM + (int)rank * BM, own_n = (tile % tiles_n) * BN + (int)rank * BH, end = min(last, first + (tile / tiles_n + 1) * 2 * BM);
            const int2 own = rows_of(a.g, w);
            const float* F = a.X + (size_t)w * a.ld + a.f_off;
            const int kc = 64 * b + 8 * (tid & 7), j0 = kc - (kc >= R ? R : 0) - (kc >= 2 * R ? R : 0);
#pragma unroll
            for (int x = 0; x < 4; ++x) {  // rows: 128 x 8 pieces of 8 k
                const int t = own_t + (tid >> 3) + 32 * x;
                const bool mine = kc < 3 * R && t >= own.x && t < min(own.y, end);
                const float* p = a.c + (size_t)t * a.rank + j0;
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (mine && wide) {
                        if (j0 + 4 * y < a.rank) v = *(reinterpret_cast<const float4*>(p) + y);
                    } else if (mine) {
                        if (j0 + 4 * y < a.rank) v.x = p[4 * y];
                        if (j0 + 4 * y + 1 < a.rank) v.y = p[4 * y + 1];
                        if (j0 + 4 * y + 2 < a.rank) v.z = p[4 * y + 2];
                        if (j0 + 4 * y + 3 < a.rank) v.w = p[4 * y + 3];
                    }
                    raw_c[x][y] = v;
                }
            }
#pragma unroll
            for (int x = 0; x < BH / 32; ++x) {  // columns: 64 k x BH / 8 pieces
                const int kk = 64 * b + tid / (BH / 8) + x * (kDrainThreads * 8 / BH), col = own_n + 8 * (tid % (BH / 8));
                const int j = kk - (kk >= R ? R : 0) - (kk >= 2 * R ? R : 0);
                const bool in = kk < 3 * R && j < a.rank && col < a.N;
                const float4* p = reinterpret_cast<const float4*>(F + (size_t)j * a.N + col);
                raw_f[x][0] = in ? *p : make_float4(0.f, 0.f, 0.f, 0.f);
                raw_f[x][1] = in ? p[1] : make_float4(0.f, 0.f, 0.f, 0.f);
            }
        };
        int tile_extra = 0;
        auto enter = [&](int tile) {  // the first piece of a tile
            if (tile >= n_tiles) return;
            const int t0 = first + (tile / tiles_n) * 2 * BM, end = min(last, t0 + 2 * BM);
            tile_workers = TileWorkers(a.g, t0, end);
            tile_extra = blocks * tile_workers.count(a.g, end);
            w = tile_workers.take(a.g, end);
            b = 0;
            if (w >= 0) load(tile);
        };
        enter(pair);
        for (int tile = pair; tile < n_tiles && live; tile += pairs, ++lt) {
            const int n0 = (tile % tiles_n) * BN, t0 = first + (tile / tiles_n) * 2 * BM, end = min(last, t0 + 2 * BM), buf = lt & 1;
            const int own_t = t0 + (int)rank * BM;  // this block's rows
            const int extra = tile_extra, n = num_kb + extra;
            volatile uint32_t* odd = odd_flag + lt % 3;
            if (tid == 0) odd_flag[(lt + 1) % 3] = odd_rows[(lt + 1) % 3] = 0u;  // its last readers are behind the barrier of the tile before
            // ---- the adapters' ring slots: the values of the next one are on their way while one is written ----
            for (int e = 0; w >= 0 && live; ++e) {
                const int s = (it + place(e, extra, n)) % STAGES;
                uint4 pa[4], pb[BH / 32];
                const int kc = 64 * b + 8 * (tid & 7);
#pragma unroll
                for (int x = 0; x < 4; ++x)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        float4& u = raw_c[x][y];
                        u = make_float4(a.factor * u.x, a.factor * u.y, a.factor * u.z, a.factor * u.w);
                    }
                const bool bad_row = without_infinities(raw_c), bad = without_infinities(raw_f);
#pragma unroll
                for (int x = 0; x < 4; ++x) pa[x] = piece8(raw_c[x], kc >= R && kc < 2 * R);
#pragma unroll
                for (int x = 0; x < BH / 32; ++x) pb[x] = piece8(raw_f[x], 64 * b + tid / (BH / 8) + x * (kDrainThreads * 8 / BH) >= 2 * R);
                if (++b == blocks) {
                    b = 0;
                    w = tile_workers.take(a.g, end);
                }
                if (w >= 0) load(tile);
                if (bad_row) odd_rows[lt % 3] = 1u;
                if (bad) {
                    *odd = 1u;  // in both blocks: each has rows of every column
                    asm volatile("st.relaxed.cluster.shared::cluster.u32 [%0], %1;" ::"r"(map_to_block(smem_u32((const void*)odd), rank ^ 1u)), "r"(1u) : "memory");
                }
                const bool ready = wait.warp(&grant[s], (granted >> s) & 1u, 32);
                granted ^= 1u << s;
                if (ready) {
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int m = (tid >> 3) + 32 * x;
                        *reinterpret_cast<uint4*>(tiles_a + s * A_BYTES + m * 128 + (((tid & 7) ^ (m & 7)) * 16)) = pa[x];
                    }
#pragma unroll
                    for (int x = 0; x < BH / 32; ++x) {
                        const int k = tid / (BH / 8) + x * (kDrainThreads * 8 / BH), n8 = tid % (BH / 8);
                        *reinterpret_cast<uint4*>(tiles_b + s * B_BYTES + (n8 >> 3) * 8192 + k * 128 + (((n8 & 7) ^ (k & 7)) * 16)) = pb[x];
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                live = !any_of_drain(!ready || dead);  // one answer for all eight warps: they leave together
                if (live && tid == 0) mbar_arrive_cluster(map_to_block(smem_u32(&full[s]), 0));
            }
            it += n;
            enter(tile + pairs);
            // ---- the accumulator ----
            if (!live) break;
            const bool ready = wait.warp(&acc_full[buf], (lt / 2) & 1, 128);
            if (!ready) {  // a wait ran out: nothing to drain, and at the next barrier everybody leaves
                dead = true;
                continue;
            }
            tc_fence_after();
            const int t = own_t + quarter * 32 + lane;
            const bool odd_f = *odd != 0u, odd_c = odd_rows[lt % 3] != 0u;
            for (int c = half * (BN / 64); c < (half + 1) * (BN / 64); ++c) {
                const int nb = n0 + c * 32;
                if (nb >= a.N) break;
                float bias[32];
                if (a.bias)
#pragma unroll
                    for (int j = 0; j < 32; ++j) bias[j] = nb + j < a.N ? a.bias[nb + j] : 0.f;
                uint32_t r[32];
                tc_ld32(tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * BN + c * 32), r);
                float v[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]);
                if (a.bias)
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] += bias[j];
                if (odd_f || odd_c) {
                    TileWorkers again(a.g, t0, end);
                    for (int w = again.take(a.g, end); w >= 0; w = again.take(a.g, end)) {
                        const int2 own = rows_of(a.g, w);
                        if (t < own.x || t >= min(own.y, end)) continue;
                        for (int j = 0; j < a.rank; ++j) {
                            const float* F = a.X + (size_t)w * a.ld + a.f_off + (size_t)j * a.N + nb;
                            const float ct = a.factor * a.c[(size_t)t * a.rank + j];
                            const bool whole = !fits(ct);  // it entered as 0: all of its products are missing
                            if (!whole && !odd_f) continue;
#pragma unroll
                            for (int x = 0; x < 32; ++x)
                                if (nb + x < a.N && (whole || !fits(F[x]))) v[x] = fmaf(ct, F[x], v[x]);
                        }
                    }
                    __syncwarp();
                }
                if (t < end) {
                    bf16* dst = a.y + (size_t)t * a.ld_y + nb;
#pragma unroll
                    for (int j = 0; j < 32; j += 8)
                        if (nb + j < a.N)
                            *reinterpret_cast<uint4*>(dst + j) = make_uint4(pack2(v[j], v[j + 1]), pack2(v[j + 2], v[j + 3]), pack2(v[j + 4], v[j + 5]), pack2(v[j + 6], v[j + 7]));
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(map_to_block(smem_u32(&acc_empty[buf]), 0));
        }
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();  // neither block's shared or tensor memory goes while the other uses it
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(2 * BN) : "memory");
    }
}

// ----------------------------------------------------------------------------- projection, few rows to a worker
// The same product where a worker has a handful of rows or one: a decoding step.  What bounds it is reading W and the factors.
//
// An item is 128 outputs x TOK rows: W's rows are the MMA's 128, the batch's rows its columns, and the blocks of a cluster share the k loop.
// Warp 0 streams tiles by TMA, one thread of warp 1 issues the MMAs.  Meanwhile warps 2 to 9 compute the adapters' share on the CUDA cores in
// fp32, each for rows of its own, a lane for four neighbouring outputs: the factors are read 512 bytes at a time.  Then every block gets
// its share of the rows' sums from all blocks of the cluster, adds them to the adapters' in a fixed order and writes them.
// (With the adapters as slots of a k loop, one worker after another: 100 rows of 52 workers, 4096 -> 4096: 155 us; here 25 us.  The copies and
// products are done long before the adapters' share, the exchange of sums and the writing, some 4 us each, one after another with a block an SM.)
constexpr int kServeThreads = 320;
__host__ __device__ constexpr size_t serve_stage(int tok) { return (size_t)(BM + tok) * BK * 2; }
__host__ __device__ constexpr int serve_stages(int tok) { return tok >= 128 ? 6 : tok >= 64 ? 8 : 10; }
__host__ __device__ constexpr size_t serve_ring(int tok) {
    const size_t ring = serve_stages(tok) * serve_stage(tok), sums = (size_t)tok * BM * 4;
    return ring > sums ? ring : sums;
}
__host__ __device__ constexpr size_t serve_smem(int tok) { return serve_ring(tok) + 1024 /*alignment*/ + 256 /*barriers*/ + tok * 4; }

template <int TOK, bool BMN>
__global__ void __launch_bounds__(kServeThreads, 1)
serve_kernel(const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ ProjectArgs a, int splits) {
    constexpr int STAGES = serve_stages(TOK), W_BYTES = BM * BK * 2, V_BYTES = TOK * BK * 2, COLUMNS = TOK < 32 ? 32 : TOK;
    constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | ((BMN ? 1u : 0u) << 15) | ((uint32_t)(TOK >> 3) << 17) | ((uint32_t)(BM >> 4) << 24);
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* tiles_w = smem;
    uint8_t* tiles_v = smem + STAGES * W_BYTES;
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + serve_ring(TOK));
    uint64_t* empty = full + STAGES;
    uint64_t* done = empty + STAGES;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(done + 1);
    volatile uint32_t* abort = tmem_slot + 1;
    int* who = reinterpret_cast<int*>(smem + serve_ring(TOK) + 256);  // [TOK] the rows' workers

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        prefetch_map(&map_v);
        prefetch_map(&map_w);
        *abort = 0u;
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        mbar_init(done, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(COLUMNS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    dependents_may_start();
    const uint32_t tmem = *tmem_slot;
    auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_try_wait<false>(bar, parity) || mbar_wait_bounded<false>(bar, parity, kSpinLimit, 0, abort, a.g.status); };

    // The kernel before this one only writes c (its own waiting done, everything before it is complete): who reads no c need not wait for it.
    const int first = row_bound(a.g, 0), last = row_bound(a.g, a.g.N);
    const int split = blockIdx.x % splits, tiles_n = (a.N + BM - 1) / BM, item = blockIdx.x / splits, n0 = item % tiles_n * BM, t0 = first + item / tiles_n * TOK;
    const int rows = min(TOK, last - t0);  // (none: the whole cluster has nothing to do, and goes on without)
    const int all = (a.K + BK - 1) / BK, kb0 = (int)((long long)all * split / splits), n = rows > 0 ? (int)((long long)all * (split + 1) / splits) - kb0 : 0;
    const int share = TOK / splits, share_bits = __ffs(share) - 1;  // rows that this block finishes, a power of two
    constexpr int MINE = TOK / 8;
    float4 low[MINE];
    bool live = true;
    if (warp == 0) {
        if (lane == 0) {
            int i = 0;
            for (; i < n; ++i) {
                const int s = i % STAGES;
                if (i >= STAGES && !wait(&empty[s], ((i / STAGES) - 1) & 1)) {
                    for (int j = i - STAGES; j < i; ++j) mbar_wait_quiet<false>(&full[j % STAGES], (j / STAGES) & 1, 1u << 20);  // in flight still
                    break;
                }
                mbar_expect_tx(&full[s], W_BYTES + V_BYTES);
                if (!BMN) {
                    tma_load_2d(tiles_w + s * W_BYTES, &map_w, (kb0 + i) * BK, n0, &full[s]);
                } else {
#pragma unroll
                    for (int c = 0; c < 2; ++c) tma_load_2d(tiles_w + s * W_BYTES + c * 8192, &map_w, n0 + 64 * c, (kb0 + i) * BK, &full[s]);
                }
                tma_load_2d(tiles_v + s * V_BYTES, &map_v, (kb0 + i) * BK, t0, &full[s]);
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            const uint64_t dw = BMN ? mnmajor_sw128_desc(smem_u32(tiles_w), 8192) : kmajor_sw128_desc(smem_u32(tiles_w)), dv = kmajor_sw128_desc(smem_u32(tiles_v));
            constexpr uint64_t STEP = (BMN ? 16 * 128 : 16 * 2) / 16;
            for (int i = 0; i < n; ++i) {
                const int s = i % STAGES;
                if (!wait(&full[s], (i / STAGES) & 1)) break;
                tc_fence_after();
#pragma unroll
                for (int k = 0; k < BK / 16; ++k) tc_mma_bf16(tmem, dw + (uint64_t)(s * (W_BYTES / 16)) + k * STEP, dv + (uint64_t)(s * (V_BYTES / 16)) + (uint64_t)(k * 2), IDESC, i > 0 || k > 0);
                tc_commit(&empty[s]);
            }
            tc_commit(done);  // (after an expired wait too: what was issued is complete before tensor memory is freed)
            mbar_wait_quiet<false>(done, 0, 1u << 20);
        }
    } else {
        for (int t = threadIdx.x - 64; t < rows; t += 256) {  // how many boundaries are <= t, by halves
            int lo = 0, hi = a.g.N + 1;
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (a.g.rowstart[mid] <= t0 + t) lo = mid + 1;
                else hi = mid;
            }
            who[t] = lo - 1 < a.g.N ? lo - 1 : -1;
        }
        asm volatile("bar.sync 1, 256;" ::: "memory");
        const int n4 = n0 + 4 * lane;
        // the factors' lines on their way to L2 while c is computed
        if (n4 < a.N && (lane & 7) == 0)
            for (int i = 0; i < MINE; ++i) {
                const int t = split * share + warp - 2 + 8 * i;
                if (8 * i + warp - 2 >= share || t >= rows || who[t] < 0) break;
                const float* F = a.X + (size_t)who[t] * a.ld + a.f_off + n4;
                for (int j = 0; j < a.rank; ++j) prefetch_l2(F + (size_t)j * a.N);
            }
        dependent_wait();  // c is there
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            low[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            const int t = split * share + warp - 2 + 8 * i;
            if (8 * i + warp - 2 >= share || t >= rows || n4 >= a.N) continue;
            const int w = who[t];
            if (w < 0) continue;
            const float* F = a.X + (size_t)w * a.ld + a.f_off + n4;
            const float* c = a.c + (size_t)(t0 + t) * a.rank;
            float4 sum = low[i];
            auto add = [&](float ct, const float4& f) { sum = make_float4(fmaf(ct, f.x, sum.x), fmaf(ct, f.y, sum.y), fmaf(ct, f.z, sum.z), fmaf(ct, f.w, sum.w)); };
            int j = 0;
            for (; j + 16 <= a.rank; j += 16) {  // sixteen loads on their way
                float4 f[16];
                float ct[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    f[e] = *reinterpret_cast<const float4*>(F + (size_t)(j + e) * a.N);
                    ct[e] = a.factor * c[j + e];
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) add(ct[e], f[e]);
            }
#pragma unroll 4
            for (; j < a.rank; ++j) add(a.factor * c[j], *reinterpret_cast<const float4*>(F + (size_t)j * a.N));
            low[i] = sum;
        }
        if (n > 0) {
            if (lane == 0) live = mbar_wait_bounded<false>(done, 0, kSpinLimit / 4, 64, abort, a.g.status);
            live = __all_sync(0xffffffffu, live);
        }
        tc_fence_after();
    }
    __syncthreads();
    if (splits > 1) cluster_sync();  // every MMA of the cluster has been waited for: nobody reads a ring
    float* sums = reinterpret_cast<float*>(smem);  // [splits][share][BM]
    if (warp >= 2 && n > 0 && live) {
        const int quarter = warp & 3;
        const uint32_t mine = smem_u32(sums + split * share * BM + quarter * 32 + lane);
#pragma unroll
        for (int g = 0; g < TOK / 16; ++g) {
            if ((g & 1) != (warp - 2) >> 2) continue;
            uint32_t r[16];
            tc_ld16(tmem + ((uint32_t)quarter << 21) + 16 * g, r);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int t = 16 * g + j;
                store_to(map_to_block(mine + ((t & (share - 1)) * BM) * 4, t >> share_bits), __uint_as_float(r[j]));
            }
        }
    }
    if (splits > 1) cluster_sync();
    else __syncthreads();
    if (warp >= 2) {
        const int n4 = n0 + 4 * lane;
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            const int at = 8 * i + warp - 2, t = split * share + at;
            if (at >= share || t >= rows || n4 >= a.N || who[t] < 0) continue;
            float4 sum = a.bias ? make_float4(a.bias[n4], a.bias[n4 + 1], a.bias[n4 + 2], a.bias[n4 + 3]) : make_float4(0.f, 0.f, 0.f, 0.f);
            for (int s = 0; s < splits; ++s) {
                const float4 v = *reinterpret_cast<const float4*>(sums + (s * share + at) * BM + 4 * lane);
                sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
            }
            *reinterpret_cast<uint2*>(a.y + (size_t)(t0 + t) * a.ld_y + n4) =
                make_uint2(pack2(sum.x + low[i].x, sum.y + low[i].y), pack2(sum.z + low[i].z, sum.w + low[i].w));
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(COLUMNS) : "memory");
    }
}

// ----------------------------------------------------------------------------- host side
// [outer][inner] bf16, rows `pitch` elements apart, in boxes of box_outer x 64 with the 128-byte swizzle; zeros outside.
int make_map(CUtensorMap* m, const void* p, int64_t inner, int64_t outer, int64_t pitch, int box_outer) {
    const EncodeTiledFn encode = encode_tiled_fn();
    if (!encode) return DBW_ERR_CUDA;
    const cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)outer}, strides[1] = {(cuuint64_t)pitch * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)box_outer}, step[2] = {1, 1};
    const CUresult r = encode(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? DBW_OK : DBW_ERR_CUDA;
}

template <class K>
int allow_smem(K kernel, size_t bytes, PerDeviceOnce& once, int device) {
    return once.run(device, [&]() -> int {
        DBW_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
        return DBW_OK;
    });
}

template <int BN, bool BMN>
int launch_project_as(dbw_handle* h, const ProjectArgs& a, const void* W, const void* v, int64_t ld_v, cudaStream_t s) {
    static PerDeviceOnce once;
    CUtensorMap map_v, map_w;
    int rc;
    if ((rc = allow_smem(project_kernel<BN, BMN>, project_smem(BN), once, h->device)) || (rc = make_map(&map_v, v, a.K, a.g.rows, ld_v, BM)) ||
        (rc = BMN ? make_map(&map_w, W, a.N, a.K, a.N, 64) : make_map(&map_w, W, a.K, a.N, a.K, BN / 2)))
        return rc;
    const int tiles = (a.g.rows + 2 * BM - 1) / (2 * BM) * ((a.N + BN - 1) / BN);
    launch_clusters(project_kernel<BN, BMN>, 2 * std::min(tiles, h->sm_count / 2), kProjectThreads, 2, project_smem(BN), s, map_v, map_w, a);
    DBW_LAUNCHED();
    return DBW_OK;
}
template <int TOK, bool BMN>
int launch_serve_as(dbw_handle* h, const ProjectArgs& a, const void* W, const void* v, int64_t ld_v, cudaStream_t s) {
    static PerDeviceOnce once;
    CUtensorMap map_v, map_w;
    int rc;
    if ((rc = allow_smem(serve_kernel<TOK, BMN>, serve_smem(TOK), once, h->device)) || (rc = make_map(&map_v, v, a.K, a.g.rows, ld_v, TOK)) ||
        (rc = BMN ? make_map(&map_w, W, a.N, a.K, a.N, 64) : make_map(&map_w, W, a.K, a.N, a.K, BM)))
        return rc;
    const int items = (a.N + BM - 1) / BM * ((a.g.rows + TOK - 1) / TOK);
    int splits = 1;
    while (splits < 8 && 2 * splits * items <= h->sm_count + h->sm_count / 4 && a.K >= 2 * splits * BK) splits *= 2;
    launch_clusters(serve_kernel<TOK, BMN>, items * splits, kServeThreads, splits, serve_smem(TOK), s, map_v, map_w, a, splits);
    DBW_LAUNCHED();
    return DBW_OK;
}
template <bool BMN>
int launch_project(dbw_handle* h, const ProjectArgs& a, const void* W, const void* v, int64_t ld_v, cudaStream_t s) {
    // Serving's kernel splits the k loop over a cluster.  It takes the rows where a worker has few (each tile's workers would cost project's tensor cores a
    // product with each factor), and where project's tiles would leave most SMs idle over a long k loop: items of 128 rows and columns, their k loops split
    // in up to 8, that fit the SMs at once, and no more of them unsplit than half of the SMs (312 rows of 12 workers, 992 -> 248 at rank 64: 22.4 us here,
    // 65.0 there; 363 rows, 2200 -> 448 at rank 32: 17.0 and 25.6.  7781 rows, 192 -> 176, are 122 items that cannot be split: 44.5 here, 31.1 there; with
    // three times the SMs, 2319 rows of 29 workers, 280 -> 768 at rank 64, took 75 here and 44 there).  Also where the items fit the SMs and the workers
    // of a tile of project (256 rows) come to more than ten slots of its k loop, which take it 2.6 us each (the passes of 1551 rows of 59 workers, backward
    // 1408 <- 968 at rank 32, 21 slots: 93 us here, 119 there; 1271 rows of 50 workers, 2504 -> 208 at rank 16, 11 slots: 43 and 56; 546 rows of 16 workers,
    // backward 2816 <- 400 at rank 8, 9 slots: 48 and 41).
    const int64_t columns = (a.N + BM - 1) / BM, items = columns * ((a.g.rows + 127) / 128), splits = std::max(1, std::min(8, a.K / (2 * BK)));
    const int64_t slots = (256 * (int64_t)a.g.N / a.g.rows + 1) * ((3 * ((a.rank + 15) / 16) + 3) / 4);  // (rows > 0)
    if (a.g.rows <= 16 * (int64_t)a.g.N || a.g.rows <= 128 || (items * splits <= h->sm_count && items <= h->sm_count / 2) || (items <= h->sm_count && slots > 10)) {
        // Rows of an item: all up to 128, fewer where the items, their k loops split, do not fill the SMs (the rows that a block finishes are what it
        // spends its time on: 67 rows of 2 workers, backward 656 <- 1520, 18.4 us with a halving that may exceed the SMs and 23.1 without it).
        int tok = a.g.rows <= 16 ? 16 : a.g.rows <= 32 ? 32 : a.g.rows <= 64 ? 64 : 128;
        while (tok > 16 && columns * ((a.g.rows + tok - 1) / tok) * splits < h->sm_count) tok /= 2;
        return tok == 16   ? launch_serve_as<16, BMN>(h, a, W, v, ld_v, s)
               : tok == 32 ? launch_serve_as<32, BMN>(h, a, W, v, ld_v, s)
               : tok == 64 ? launch_serve_as<64, BMN>(h, a, W, v, ld_v, s)
                           : launch_serve_as<128, BMN>(h, a, W, v, ld_v, s);
    }
    // Columns of a tile: 256 where that fills the SMs, else 128.
    const int rows = (a.g.rows + 2 * BM - 1) / (2 * BM), pairs = h->sm_count / 2;
    auto turns = [&](int bn) { return (int64_t)((rows * ((a.N + bn - 1) / bn) + pairs - 1) / pairs) * bn; };
    return turns(128) < turns(256) ? launch_project_as<128, BMN>(h, a, W, v, ld_v, s) : launch_project_as<256, BMN>(h, a, W, v, ld_v, s);
}

template <int NT>
int launch_shrink_few(dbw_handle* h, const RowGroups& g, const float* X, int64_t f_off, int rank, int width, const void* v, int64_t ld_v, float factor, float* out, cudaStream_t s) {
    static PerDeviceOnce once;
    const int rc = allow_smem(shrink_kernel<NT>, shrink_smem(NT), once, h->device);
    if (rc) return rc;
    const int tiles = g.rows / 16 + std::min(g.N, g.rows);
    int splits = 1;
    while (splits < 8 && 2 * splits * std::min(g.N, g.rows) <= 2 * h->sm_count && width >= 512 * splits) splits *= 2;
    launch_clusters(shrink_kernel<NT>, tiles * splits, kShrinkThreads, splits, shrink_smem(NT), s, g, X, h->ld, f_off, rank, width, (const bf16*)v, ld_v, factor, out, splits);
    DBW_LAUNCHED();
    return DBW_OK;
}
template <int R>
int launch_shrink_tc(dbw_handle* h, const RowGroups& g, const float* X, int64_t f_off, int rank, int width, const void* v, int64_t ld_v, float factor, float* out, cudaStream_t s) {
    static PerDeviceOnce once;
    CUtensorMap map;
    int rc;
    if ((rc = allow_smem(shrink_tc_kernel<R>, thin_smem(R), once, h->device)) || (rc = make_map(&map, v, width, g.rows, ld_v, BM))) return rc;
    const int tiles = g.rows / BM + std::min(g.N, g.rows), room = h->sm_count * (thin_columns(R) == 256 ? 2 : 1);
    int splits = 1;
    while (splits < 8 && 2 * splits * (g.rows / BM) <= room && width >= 4 * BK * splits) splits *= 2;
    launch_clusters(shrink_tc_kernel<R>, tiles * splits, thin_threads(R), splits, thin_smem(R), s, map, g, X, h->ld, f_off, rank, width, (const bf16*)v, ld_v, factor, out, splits);
    DBW_LAUNCHED();
    return DBW_OK;
}
int launch_shrink(dbw_handle* h, const RowGroups& g, const float* X, int64_t f_off, int rank, int width, const void* v, int64_t ld_v, float factor, float* out, cudaStream_t s) {
    if (g.rows <= 16 * (int64_t)g.N)  // a worker's rows fill no more than 16
        return rank <= 8    ? launch_shrink_few<1>(h, g, X, f_off, rank, width, v, ld_v, factor, out, s)
               : rank <= 16 ? launch_shrink_few<2>(h, g, X, f_off, rank, width, v, ld_v, factor, out, s)
               : rank <= 32 ? launch_shrink_few<4>(h, g, X, f_off, rank, width, v, ld_v, factor, out, s)
                            : launch_shrink_few<8>(h, g, X, f_off, rank, width, v, ld_v, factor, out, s);
    return rank <= 16   ? launch_shrink_tc<16>(h, g, X, f_off, rank, width, v, ld_v, factor, out, s)
           : rank <= 32 ? launch_shrink_tc<32>(h, g, X, f_off, rank, width, v, ld_v, factor, out, s)
           : rank <= 48 ? launch_shrink_tc<48>(h, g, X, f_off, rank, width, v, ld_v, factor, out, s)
                        : launch_shrink_tc<64>(h, g, X, f_off, rank, width, v, ld_v, factor, out, s);
}

struct OuterSide {  // one factor's gradient: v [rows][width], c [rows][rank]
    int64_t f_off;
    int width;
    const void* v;
    int64_t ld_v;
    float factor;
    const float* c;
};
template <int R>
int launch_outer_as(dbw_handle* h, const RowGroups& g, float* G, int rank, const OuterSide& a, const OuterSide& b, cudaStream_t s) {
    static PerDeviceOnce once;
    CUtensorMap map_a{}, map_b{};
    int rc;
    // without rows nothing is copied, and there may be nothing to make a map of
    if ((rc = allow_smem(outer_tc_kernel<R>, thin_smem(R), once, h->device)) ||
        (g.rows > 0 && ((rc = make_map(&map_a, a.v, a.width, g.rows, a.ld_v, BK)) || (rc = make_map(&map_b, b.v, b.width, g.rows, b.ld_v, BK)))))
        return rc;
    const OuterJobs jobs{{a.f_off, b.f_off}, {a.width, b.width}, {a.factor, b.factor}, {a.c, b.c}, {(const bf16*)a.v, (const bf16*)b.v}, {a.ld_v, b.ld_v}};
    const int64_t items = (int64_t)g.N * ((a.width + BM - 1) / BM + (b.width + BM - 1) / BM), room = h->sm_count * (thin_columns(R) == 256 ? 2 : 1);
    int splits = 1;
    while (splits < 8 && 2 * splits * items <= room && (int64_t)g.rows >= 2 * (int64_t)g.N * splits * BK) splits *= 2;
    const int64_t clusters = splits > 1 ? items : std::min(items, room);
    launch_clusters(outer_tc_kernel<R>, (unsigned)(clusters * splits), thin_threads(R), splits, thin_smem(R), s, map_a, map_b, g, G, h->ld, rank, jobs, splits);
    DBW_LAUNCHED();
    return DBW_OK;
}
int launch_outer(dbw_handle* h, const RowGroups& g, float* G, int rank, const OuterSide& a, const OuterSide& b, cudaStream_t s) {
    return rank <= 16   ? launch_outer_as<16>(h, g, G, rank, a, b, s)
           : rank <= 32 ? launch_outer_as<32>(h, g, G, rank, a, b, s)
           : rank <= 48 ? launch_outer_as<48>(h, g, G, rank, a, b, s)
                        : launch_outer_as<64>(h, g, G, rank, a, b, s);
}

}  // namespace

int launch_lowrank_forward(dbw_handle* h, const dbw_lowrank_desc& a, float scale, const float* X, const void* W, const float* bias, const void* x,
                           int64_t ld_x, const int32_t* rowstart, int32_t rows, void* y, int64_t ld_y, float* hidden, cudaStream_t s) {
    if (rows == 0) return launch_check_groups(h, rowstart, rows, s);
    const RowGroups g{rowstart, h->N, rows, h->d_status};
    const int rc = launch_shrink(h, g, X, a.a_off, a.rank, a.in, x, ld_x, 1.f, hidden, s);
    if (rc) return rc;
    return launch_project<false>(h, {g, X, h->ld, a.b_off, a.rank, a.out, a.in, scale, hidden, bias, (bf16*)y, ld_y}, W, x, ld_x, s);
}

int launch_lowrank_backward(dbw_handle* h, const dbw_lowrank_desc& a, float scale, const float* X, const void* W, const void* x, int64_t ld_x,
                            const float* hidden, const void* dy, int64_t ld_dy, const int32_t* rowstart, int32_t rows, float* G, float* d_hidden, void* dx,
                            int64_t ld_dx, cudaStream_t s) {
    const RowGroups g{rowstart, h->N, rows, h->d_status};
    int rc;
    if ((rc = rows > 0 ? launch_shrink(h, g, X, a.b_off, a.rank, a.out, dy, ld_dy, scale, d_hidden, s) : launch_check_groups(h, rowstart, rows, s))) return rc;
    if ((rc = launch_outer(h, g, G, a.rank, {a.b_off, a.out, dy, ld_dy, scale, hidden}, {a.a_off, a.in, x, ld_x, 1.f, d_hidden}, s))) return rc;
    if (!dx || rows == 0) return DBW_OK;
    return launch_project<true>(h, {g, X, h->ld, a.a_off, a.rank, a.in, a.out, 1.f, d_hidden, nullptr, (bf16*)dx, ld_dx}, W, dy, ld_dy, s);
}

}  // namespace dbw
