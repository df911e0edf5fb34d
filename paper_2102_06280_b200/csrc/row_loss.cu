// Losses over a vocabulary with their gradients: distillation from a teacher's top logits, and the clipped policy objective
// (dbw_distill, dbw_policy_loss).
//
// Both need of a row's logits z the softmax q at temperature tau, and a few of its values.  With c = log2(e) / tau, m the row's maximum and
// S = sum of 2^(c (z - m)) the gradient is
//     d_v = f 2^(c (z_v - m)),  f = weight x (tau for distillation, -slope / tau for the policy loss) / S,
// to which the few places of the teacher's entries or of the action then add their own share, rounded once.  What bounds them is the
// logits in and the gradient out.
//
// A row may begin anywhere: it is cut into pieces of 16 bytes from its first multiple of 16 bytes on; the values before and behind
// them ("loose", 14 at most) are taken one by one.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "common.cuh"
#include "rows.cuh"
#include "tc_ptx.cuh"

namespace dbw {

namespace {

constexpr int kThreads = 256;

struct LossArgs {
    RowGroups g;
    const void* logits;
    long long ld;
    int vocab;
    const float* row_weight;
    float* row_loss;
    void* d_logits;
    long long ld_d;
    double tau, over_tau;
    // distillation
    const int32_t* top_idx;
    const float* top_logit;
    int top;
    // policy
    const int32_t* action;
    const float *old_logp, *ref_logp, *advantage;
    float* logp;
    float low, high, kl;  // the ratio's bounds, and the KL term's factor
};

enum { DISTILL = 0, POLICY = 1 };

// ----------------------------------------------------------------------------- values of 16 bytes
template <class T>
struct Vec {  // 16-bit types: eight values
    static constexpr int n = 8;
    static __device__ __forceinline__ void load(uint4 u, float (&v)[8]) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) unpack(w[e], v[2 * e], v[2 * e + 1]);
    }
    static __device__ __forceinline__ uint4 store(const float (&v)[8]) { return make_uint4(pack(v[0], v[1]), pack(v[2], v[3]), pack(v[4], v[5]), pack(v[6], v[7])); }
    static __device__ __forceinline__ void unpack(uint32_t w, float& lo, float& hi);
    static __device__ __forceinline__ uint32_t pack(float lo, float hi);
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b);  // of both halves; a NaN yields to a number
    static __device__ __forceinline__ float most(uint4 u) {
        float lo, hi;
        unpack(larger(larger(u.x, u.y), larger(u.z, u.w)), lo, hi);
        return fmaxf(lo, hi);
    }
};
template <>
__device__ __forceinline__ uint32_t Vec<__nv_bfloat16>::larger(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
template <>
__device__ __forceinline__ uint32_t Vec<__half>::larger(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("max.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
template <>
__device__ __forceinline__ void Vec<__nv_bfloat16>::unpack(uint32_t w, float& lo, float& hi) {
    lo = __uint_as_float(w << 16);
    hi = __uint_as_float(w & 0xffff0000u);
}
template <>
__device__ __forceinline__ uint32_t Vec<__nv_bfloat16>::pack(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <>
__device__ __forceinline__ void Vec<__half>::unpack(uint32_t w, float& lo, float& hi) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    lo = f.x;
    hi = f.y;
}
template <>
__device__ __forceinline__ uint32_t Vec<__half>::pack(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <>
struct Vec<float> {
    static constexpr int n = 4;
    static __device__ __forceinline__ void load(uint4 u, float (&v)[4]) {
        v[0] = __uint_as_float(u.x); v[1] = __uint_as_float(u.y); v[2] = __uint_as_float(u.z); v[3] = __uint_as_float(u.w);
    }
    static __device__ __forceinline__ float most(uint4 u) { return fmaxf(fmaxf(__uint_as_float(u.x), __uint_as_float(u.y)), fmaxf(__uint_as_float(u.z), __uint_as_float(u.w))); }
    static __device__ __forceinline__ uint4 store(const float (&v)[4]) {
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
};

__device__ __forceinline__ float exp2_fast(float x) {  // 2^x to 2^-22, 0 below 2^-126
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Two fp32 values in one register pair, for one instruction.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair(float lo, float hi) {
    f32x2 d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
    return d;
}
__device__ __forceinline__ void unpair(f32x2 d, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(d)); }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}

// 2^(c (z - m)) as 2^(c z - c m), one multiply-add: c m (`cm`) is rounded once and the same in every power of a maximum m, so that its rounding
// cancels in q; in log S it is taken back (log_sum).  That holds while the rounding is small: below 2^24 it is at most 1, a factor of two in every
// power.  So maxima are kept at or above -limit(c), and a row whose maximum is not within the limits (huge logits, a tiny temperature, a row masked
// throughout with -inf or the type's lowest value) is summed again by power_beyond, the difference first: that can take a value from neither end.
__device__ __forceinline__ float limit_of(float c) { return fminf(16777216.f / c, 1e38f); }
__device__ __forceinline__ float power(float z, float cm, float c) { return exp2_fast(fmaf(z, c, -cm)); }
__device__ __forceinline__ f32x2 power2(float lo, float hi, f32x2 minus_cm, f32x2 c) {
    unpair(fma2(pair(lo, hi), c, minus_cm), lo, hi);
    return pair(exp2_fast(lo), exp2_fast(hi));
}
__device__ __forceinline__ float power_beyond(float z, float m, float c) { return exp2_fast((z - m) * c); }  // (of an infinite m: NaN)

// Maximum of z, and the sum of 2^(c (z - max)); a NaN lies in the sum.
struct Softmax {
    float m, s;
    __device__ __forceinline__ void raise(float to, float c) {  // to >= m
        s *= exp2_fast(__fmul_rn(m, c) - __fmul_rn(to, c));
        m = to;
    }
};
__device__ __forceinline__ Softmax join_warp(Softmax x, float c) {
    float to = x.m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) to = fmaxf(to, __shfl_xor_sync(0xffffffffu, to, o));
    x.raise(to, c);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x.s += __shfl_xor_sync(0xffffffffu, x.s, o);
    return x;
}
// log of the sum, S >= 1/2 (a row's largest term is 1), to 2^-25 and better: the exponent's share is exact in 64 bits, the rest is below 0.35
__device__ __forceinline__ double log_of(float s) {
    if (!(s < INFINITY)) return (double)s;
    int e = (int)(__float_as_uint(s) >> 23) - 127;
    float f = __uint_as_float((__float_as_uint(s) & 0x7fffffu) | 0x3f800000u);
    if (f > 1.41421354f) {
        f *= 0.5f;
        ++e;
    }
    return s > 0.f ? (double)e * 0.6931471805599453 + (double)logf(f) : (s == 0.f ? -(double)INFINITY : (double)s);
}
// log of the sum of e^((z - m) / tau): without the rounding of c m
__device__ __forceinline__ double log_sum(const Softmax& x, float c, bool far) {
    return log_of(x.s) - (far ? 0.0 : 0.6931471805599453 * (double)fmaf(x.m, c, -__fmul_rn(x.m, c)));
}
// e^x - 1 - x, by its series where the difference would cancel
__device__ __forceinline__ float beyond_linear(float x) {
    if (x == INFINITY) return x;
    if (fabsf(x) > 0.5f) return expm1f(x) - x;
    float t = 1.f / 40320.f;
    t = fmaf(t, x, 1.f / 5040.f);
    t = fmaf(t, x, 1.f / 720.f);
    t = fmaf(t, x, 1.f / 120.f);
    t = fmaf(t, x, 1.f / 24.f);
    t = fmaf(t, x, 1.f / 6.f);
    t = fmaf(t, x, 0.5f);
    return t * x * x;
}

// ----------------------------------------------------------------------------- a row's cut, and what is asked of it
template <class T>
struct Cut {
    int head, pieces, loose;  // values before the first piece, pieces, values outside of them
    __device__ __forceinline__ Cut(const T* z, int V) {
        head = min(V, (int)(((16u - ((uintptr_t)z & 15u)) & 15u) / sizeof(T)));
        pieces = (V - head) / Vec<T>::n;
        loose = V - pieces * Vec<T>::n;
    }
    __device__ __forceinline__ int loose_at(int i) const { return i < head ? i : i + pieces * Vec<T>::n; }
    __device__ __forceinline__ int piece_of(int v) const { return v < head || v >= head + pieces * Vec<T>::n ? -1 : (v - head) / Vec<T>::n; }
};

// Row t's weight: the caller's, or 1 / rows of its worker (0 where a malformed rowstart gives it none).  All lanes of a warp.
__device__ __forceinline__ float weight_of(const LossArgs& a, int t) {
    if (a.row_weight) return a.row_weight[t];
    const int w = worker_of_row(a.g, t);
    if (w < 0) return 0.f;
    const int2 own = rows_of(a.g, w);
    return own.y > own.x ? 1.f / (float)(own.y - own.x) : 0.f;
}

// The teacher's side of a row, by one warp: lane l has entries l, l + 32, ... (v < 0: none), their logits t and the row's own z there.  In 64 bits: an
// error of p counts as often as the logits lie apart.
//     loss = tau^2 (cross + (m - z_ref) / tau + log S),  cross = sum_j p_j (log p_j - (z_j - z_ref) / tau),
// z_ref being the largest of the z_j, so that nothing cancels where all of them are large.
template <int PER>
struct Teacher {
    double cross;
    float z_ref;
    float p[PER];
    __device__ __forceinline__ Teacher(const int (&v)[PER], const float (&t)[PER], const float (&z)[PER], double over_tau) {
        float most = -INFINITY, ref = -INFINITY;
#pragma unroll
        for (int k = 0; k < PER; ++k)
            if (v[k] >= 0) {
                most = fmaxf(most, t[k]);
                ref = fmaxf(ref, z[k]);
            }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
            ref = fmaxf(ref, __shfl_xor_sync(0xffffffffu, ref, o));
        }
        z_ref = ref == -INFINITY ? 0.f : ref;
        double mass = 0.0, e[PER];
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            e[k] = v[k] >= 0 ? exp(((double)t[k] - (double)most) * over_tau) : 0.0;
            mass += e[k];
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mass += __shfl_xor_sync(0xffffffffu, mass, o);
        const double over_mass = 1.0 / mass, log_mass = log_of((float)mass);  // mass >= 1: the largest entry's share is 1
        cross = 0.0;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            p[k] = (float)(e[k] * over_mass);
            if (e[k] != 0.0) cross += e[k] * over_mass * ((((double)t[k] - (double)most) - ((double)z[k] - (double)z_ref)) * over_tau - log_mass);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) cross += __shfl_xor_sync(0xffffffffu, cross, o);
    }
    static __device__ __forceinline__ float loss(double cross, float z_ref, const Softmax& x, const LossArgs& a, float c, bool far) {
        return (float)(a.tau * a.tau * (cross + ((double)x.m - (double)z_ref) * a.over_tau + log_sum(x, c, far)));
    }
};

struct Policy {
    float logp, loss, slope;  // slope: d loss / d logp
    __device__ __forceinline__ Policy(const LossArgs& a, float z, float old, float ref, float adv, const Softmax& x, float c, bool far) {
        const double lp = ((double)z - (double)x.m) * a.over_tau - log_sum(x, c, far);
        const float ratio = expf((float)(lp - (double)old)), open = ratio * adv, held = fminf(fmaxf(ratio, a.low), a.high) * adv;
        logp = (float)lp;
        loss = -(held < open ? held : open);
        slope = held < open ? 0.f : -open;
        if (a.kl != 0.f) {
            const float far = (float)((double)ref - lp);
            loss = fmaf(a.kl, beyond_linear(far), loss);
            slope = fmaf(-a.kl, expm1f(far), slope);
        }
    }
};

// The gradient's factor f times the power e of a logit z.  An infinite f (a slope beyond fp32: a ratio or a KL term of more than 2^128) leaves a logit
// of -inf without a gradient; times another power that has become 0 it is NaN, the product being anything.
__device__ __forceinline__ bool infinite(float f) { return fabsf(f) == INFINITY; }
__device__ __forceinline__ float share(float f, float e, float z) { return z == -INFINITY && infinite(f) ? 0.f : f * e; }
// The action's own: slope (1 - e / S), f = -slope / S; an infinite one stays where q < 1 (and is NaN at 1, as above).
__device__ __forceinline__ float action_share(float slope, float f, float e, float S) { return infinite(slope) && e < S ? slope : slope + f * e; }

// What L2 keeps: logits that are read a second time stay; their second reading and the gradient are the first to leave.
__device__ __forceinline__ uint64_t keep_policy() {
    uint64_t p;
    asm("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(p));
    return p;
}
__device__ __forceinline__ uint64_t leave_policy() {
    uint64_t p;
    asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
    return p;
}
// One piece of the gradient; where z and d do not break into the same pieces, value by value.
template <class T>
__device__ __forceinline__ void put(T* d, int at, bool alike, const float (&g)[Vec<T>::n], uint64_t policy) {
    if (alike) {
        const uint4 u = Vec<T>::store(g);
        asm volatile("st.global.L2::cache_hint.v4.b32 [%0], {%1, %2, %3, %4}, %5;" ::"l"(d + at), "r"(u.x), "r"(u.y), "r"(u.z), "r"(u.w), "l"(policy) : "memory");
    } else
    {
#pragma unroll
        for (int e = 0; e < Vec<T>::n; ++e) d[at + e] = T(g[e]);
    }
}

// The sum of a piece's powers, and its gradient.
template <class T>
__device__ __forceinline__ void add_piece(const uint4& u, float cm, float c, f32x2 (&sums)[2]) {
    float f[Vec<T>::n];
    Vec<T>::load(u, f);
#pragma unroll
    for (int e = 0; e < Vec<T>::n; e += 2) sums[e / 2 & 1] = add2(sums[e / 2 & 1], power2(f[e], f[e + 1], pair(-cm, -cm), pair(c, c)));
}
__device__ __forceinline__ float total(const f32x2 (&sums)[2]) {
    float lo, hi;
    unpair(add2(sums[0], sums[1]), lo, hi);
    return lo + hi;
}
template <class T>
__device__ __forceinline__ void grade_piece(const uint4& u, float cm, float c, float f, float (&g)[Vec<T>::n]) {
    Vec<T>::load(u, g);
#pragma unroll
    for (int e = 0; e < Vec<T>::n; e += 2) unpair(mul2(power2(g[e], g[e + 1], pair(-cm, -cm), pair(c, c)), pair(f, f)), g[e], g[e + 1]);
}

// ----------------------------------------------------------------------------- short rows
// A warp per row, the row in its registers: HELD pieces a lane, 4 KB a row.
constexpr int HELD = 8;
template <class T, int KIND>
__global__ void __launch_bounds__(kThreads) short_row_kernel(const __grid_constant__ LossArgs a) {
    dependent_begin();
    constexpr int ROWS = kThreads / 32, ENTRIES = KIND == DISTILL ? DBW_DISTILL_MAX_TOP : 1, PER = (ENTRIES + 31) / 32, VN = Vec<T>::n;
    __shared__ int entry_v[ROWS][ENTRIES];
    __shared__ float entry_p[ROWS][ENTRIES];
    const int slot = threadIdx.x / 32, lane = threadIdx.x & 31;
    if (blockIdx.x == 0) check_groups(a.g);
    const int t = row_bound(a.g, 0) + blockIdx.x * ROWS + slot;
    if (t >= row_bound(a.g, a.g.N)) return;
    const float weight = weight_of(a, t);
    const T* z = (const T*)a.logits + (size_t)t * a.ld;
    T* d = a.d_logits ? (T*)a.d_logits + (size_t)t * a.ld_d : nullptr;
    const int V = a.vocab;
    const Cut<T> cut(z, V);
    const bool alike = (((uintptr_t)z ^ (uintptr_t)d) & 15u) == 0;

    int v[PER], n = 0;
    float et[PER], ez[PER];
    bool live = weight != 0.f;
    if (KIND == DISTILL) {
        n = live ? a.top : 0;
        bool some = false;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int j = 32 * k + lane;
            v[k] = -1;
            et[k] = ez[k] = 0.f;
            if (j < n) {
                v[k] = a.top_idx[(size_t)t * a.top + j];
                et[k] = a.top_logit[(size_t)t * a.top + j];
                if (v[k] < -1 || v[k] >= V) {
                    atomicOr(a.g.status, DBW_STATUS_BAD_INDEX);
                    v[k] = -1;
                }
                if (v[k] >= 0) ez[k] = (float)z[v[k]];
                entry_v[slot][j] = v[k];
            }
            some |= v[k] >= 0;
        }
        live = __any_sync(0xffffffffu, some);
    } else if (live) {
        v[0] = a.action[t];
        live = v[0] >= 0 && v[0] < V;
        if (live) ez[0] = (float)z[v[0]];
        else if (lane == 0) atomicOr(a.g.status, DBW_STATUS_BAD_INDEX);
    }
    if (!live) {
        if (lane == 0) {
            a.row_loss[t] = 0.f;
            if (KIND == POLICY && a.logp) a.logp[t] = 0.f;
        }
        if (d && alike) {
            for (int i = lane; i < cut.pieces; i += 32) *reinterpret_cast<uint4*>(d + cut.head + i * VN) = make_uint4(0, 0, 0, 0);
            if (lane < cut.loose) d[cut.loose_at(lane)] = T(0.f);
        } else if (d) {
            for (int i = lane; i < V; i += 32) d[i] = T(0.f);
        }
        return;
    }

    const float c = (float)(1.4426950408889634 * a.over_tau);
    uint4 held[HELD];
#pragma unroll
    for (int k = 0; k < HELD; ++k)
        if (lane + 32 * k < cut.pieces) held[k] = *reinterpret_cast<const uint4*>(z + cut.head + (lane + 32 * k) * VN);
    const float loose = lane < cut.loose ? (float)z[cut.loose_at(lane)] : -INFINITY;
    const float limit = limit_of(c);
    Softmax x{fmaxf(-limit, loose), 0.f};
#pragma unroll
    for (int k = 0; k < HELD; ++k)
        if (lane + 32 * k < cut.pieces) x.m = fmaxf(x.m, Vec<T>::most(held[k]));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x.m = fmaxf(x.m, __shfl_xor_sync(0xffffffffu, x.m, o));
    const bool far = !(fabsf(x.m) < limit);
    float cm = __fmul_rn(x.m, c);
    if (!far) {
        f32x2 sums[2] = {pair(0.f, 0.f), pair(0.f, 0.f)};
#pragma unroll
        for (int k = 0; k < HELD; ++k)
            if (lane + 32 * k < cut.pieces) add_piece<T>(held[k], cm, c, sums);
        x.s = total(sums);
        if (lane < cut.loose) x.s += power(loose, cm, c);
    } else {
        x.m = -INFINITY;
        for (int i = lane; i < V; i += 32) x.m = fmaxf(x.m, (float)z[i]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) x.m = fmaxf(x.m, __shfl_xor_sync(0xffffffffu, x.m, o));
        for (int i = lane; i < V; i += 32) x.s += power_beyond((float)z[i], x.m, c);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x.s += __shfl_xor_sync(0xffffffffu, x.s, o);
    const float m = x.m;
    auto at_row = [&](float z) { return far ? power_beyond(z, m, c) : power(z, cm, c); };

    float f, slope = 0.f, p[PER];
    if (KIND == POLICY) {
        const Policy r(a, ez[0], a.old_logp[t], a.kl != 0.f ? a.ref_logp[t] : 0.f, a.advantage[t], x, c, far);
        if (lane == 0) {
            a.row_loss[t] = r.loss;
            if (a.logp) a.logp[t] = r.logp;
        }
        slope = r.slope * weight * (float)a.over_tau;
        f = -slope / x.s;
    } else {
        const Teacher<PER> teacher(v, et, ez, a.over_tau);
        if (lane == 0) a.row_loss[t] = Teacher<PER>::loss(teacher.cross, teacher.z_ref, x, a, c, far);
        f = weight * (float)a.tau / x.s;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            p[k] = teacher.p[k];
            if (32 * k + lane < n) entry_p[slot][32 * k + lane] = p[k];
        }
    }
    if (!d) return;
    __syncwarp();  // the gradient may replace the logits: all that is wanted of them has been read
    const uint64_t leave = leave_policy();
    const bool slow = far || infinite(f);
#pragma unroll
    for (int k = 0; k < HELD; ++k) {
        if (lane + 32 * k >= cut.pieces) continue;
        float g[VN];
        if (slow) {
            Vec<T>::load(held[k], g);
#pragma unroll
            for (int e = 0; e < VN; ++e) g[e] = share(f, at_row(g[e]), g[e]);
        } else {
            grade_piece<T>(held[k], cm, c, f, g);
        }
        put(d, cut.head + (lane + 32 * k) * VN, alike, g, leave);
    }
    if (lane < cut.loose) d[cut.loose_at(lane)] = T(share(f, at_row(loose), loose));
    __syncwarp();
    if (KIND == POLICY) {
        if (lane == 0) d[v[0]] = T(action_share(slope, f, at_row(ez[0]), x.s));
    } else {
        const float scale = weight * (float)a.tau;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            if (v[k] < 0) continue;
            float sum = 0.f;  // of every entry of this index
            for (int i = 0; i < n; ++i)
                if (entry_v[slot][i] == v[k]) sum += entry_p[slot][i];
            d[v[k]] = T(fmaf(-scale, sum, share(f, at_row(ez[k]), ez[k])));
        }
    }
}

// ----------------------------------------------------------------------------- long rows
// A block per row: G threads that work, and a warp that meanwhile collects what is asked of the row (the teacher's softmax, the action's
// numbers) and in the end adds it.  The row is read twice, for maximum and sum and for the gradient, the second time from L2, where
// the rows of all blocks have room.  Every thread streams its pieces through AHEAD buffers of its own in shared memory (cp.async; nobody
// else reads them, so no barrier is involved), into the second pass while the sums are joined.
//
// 4096 rows of bf16 values: 128000 a row, policy loss: 432 us, 4.9 TB/s; 131072, distillation with a teacher's 64 entries: 451 us, 4.8 TB/s.  Neither
// memory (60 % of its peak, half of it written) nor the exponentials (two a value: 72 and 65 % of what their pipe can do) is full: a row's phases, and
// memory that turns from reading to writing, leave some of both.
//
// What was slower, 4096 rows of 128000: a row in the registers of a cluster's blocks, 750 us (nothing overlaps a row's phases);
// a row in a ring of bulk copies of one or two blocks an SM over clusters of two or four, 744 us and more (the exchange of sums, and
// phases that wait for the slowest block); this with blocks that stay and take every 296th row, 460 us (half of them are done after 310, the
// others after 390), and with blocks that take rows over by cluster launch control, 525 us.
template <int G>
struct Stream {
    static constexpr int AHEAD = 4, PER = 2;  // steps, pieces of a thread in one
    static constexpr int BLOCKS = G == 512 ? 2 : G == 256 ? 4 : 8;  // an SM
};

struct RowInfo {
    int asked;   // something is asked of the row
    float z, old, ref, adv;  // policy
    float loose[16];
};

template <int G>
__host__ __device__ constexpr size_t stream_smem() { return (size_t)Stream<G>::AHEAD * Stream<G>::PER * G * 16; }

template <class T, int KIND, int G>
__global__ void __launch_bounds__(G + 32, Stream<G>::BLOCKS) long_row_kernel(const __grid_constant__ LossArgs a) {
    constexpr int VN = Vec<T>::n, WARPS = G / 32, PER = KIND == DISTILL ? DBW_DISTILL_MAX_TOP / 32 : 1, AHEAD = Stream<G>::AHEAD, P = Stream<G>::PER;
    extern __shared__ uint4 buffers[];  // [AHEAD][P][G]
    __shared__ RowInfo info;
    __shared__ float part_m[3][WARPS], part_s[3][WARPS];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    dependent_begin();
    if (blockIdx.x == 0) check_groups(a.g);
    const int t = row_bound(a.g, 0) + blockIdx.x, V = a.vocab;
    if (t >= row_bound(a.g, a.g.N)) return;
    const T* z = (const T*)a.logits + (size_t)t * a.ld;
    T* d = a.d_logits ? (T*)a.d_logits + (size_t)t * a.ld_d : nullptr;
    const Cut<T> cut(z, V);
    const bool helper = warp == WARPS, alike = (((uintptr_t)z ^ (uintptr_t)d) & 15u) == 0;
    auto nothing = [&]() {  // loss and gradient 0
        if (helper) {
            if (lane == 0) {
                a.row_loss[t] = 0.f;
                if (KIND == POLICY && a.logp) a.logp[t] = 0.f;
            }
        } else if (d && alike) {
            for (int i = tid; i < cut.pieces; i += G) *reinterpret_cast<uint4*>(d + cut.head + (size_t)i * VN) = make_uint4(0, 0, 0, 0);
            if (tid < cut.loose) d[cut.loose_at(tid)] = T(0.f);
        } else if (d) {
            for (int i = tid; i < V; i += G) d[i] = T(0.f);
        }
    };
    const float weight = weight_of(a, t);
    if (weight == 0.f) {
        nothing();
        return;
    }
    const float c = (float)(1.4426950408889634 * a.over_tau), limit = limit_of(c);

    // ---- what is asked of the row; maximum and sum ----
    Softmax x{-limit, 0.f};
    int v[PER];
    float ez[PER], ep[PER];  // of the helper's lanes: the entries' logits and p (of every entry of the index), or the action
    double cross = 0.0;
    float z_ref = 0.f;
    // the workers' stream: this thread's next copies, and how many pieces the row has from there on
    const int passes = d ? 2 : 1;
    const uint64_t keep = keep_policy(), leave = leave_policy();
    const uint4* const z_begin = reinterpret_cast<const uint4*>(z + cut.head) + tid;
    const uint4* ahead_z = z_begin;
    int ahead_left = cut.pieces - tid, ahead_pass = 0;
    uint64_t ahead_policy = passes == 2 ? keep : leave;
    uint32_t buffer = ptx::smem_u32(buffers + tid);  // this thread's place in the oldest step
    const uint32_t buffers_end = buffer + AHEAD * P * G * 16;
    auto copy_next = [&]() {
        if (ahead_pass < passes) {
#pragma unroll
            for (int e = 0; e < P; ++e)
                if (e * G < ahead_left)
                    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(buffer + e * G * 16), "l"(ahead_z + e * G), "l"(ahead_policy) : "memory");
            ahead_z += P * G;
            ahead_left -= P * G;
            if (ahead_left + tid <= 0) {  // (the same for all workers)
                ++ahead_pass;
                ahead_z = z_begin;
                ahead_left = cut.pieces - tid;
                ahead_policy = leave;
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        buffer += P * G * 16;
        if (buffer == buffers_end) buffer -= AHEAD * P * G * 16;
    };
    auto next = [&](uint4 (&u)[P]) {  // this thread's next pieces, and the copies of others into their place
        asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD - 1) : "memory");
#pragma unroll
        for (int e = 0; e < P; ++e)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(u[e].x), "=r"(u[e].y), "=r"(u[e].z), "=r"(u[e].w) : "r"(buffer + e * G * 16) : "memory");
        copy_next();
    };
    const int whole = cut.pieces / (P * G), rest = cut.pieces - whole * P * G;  // steps in which every thread has P pieces, and what is left
    const int last_pieces = rest > tid ? (rest - tid + G - 1) / G : 0;
    if (helper) {
        bool asked = true;
        if (KIND == DISTILL) {
            bool some = false;
            float et[PER];
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int j = 32 * i + lane;
                v[i] = -1;
                et[i] = ez[i] = ep[i] = 0.f;
                if (j < a.top) {
                    v[i] = a.top_idx[(size_t)t * a.top + j];
                    et[i] = a.top_logit[(size_t)t * a.top + j];
                    if (v[i] < -1 || v[i] >= V) {
                        atomicOr(a.g.status, DBW_STATUS_BAD_INDEX);
                        v[i] = -1;
                    }
                    if (v[i] >= 0) ez[i] = (float)z[v[i]];
                }
                some |= v[i] >= 0;
            }
            asked = __any_sync(0xffffffffu, some);
            if (asked) {
                const Teacher<PER> teacher(v, et, ez, a.over_tau);
                cross = teacher.cross;
                z_ref = teacher.z_ref;
                for (int j = 0; j < a.top; ++j) {  // every lane's entries against entry j
                    int vj = 0;
                    float pj = 0.f;
#pragma unroll
                    for (int i = 0; i < PER; ++i)
                        if (j >> 5 == i) {
                            vj = __shfl_sync(0xffffffffu, v[i], j & 31);
                            pj = __shfl_sync(0xffffffffu, teacher.p[i], j & 31);
                        }
#pragma unroll
                    for (int e = 0; e < PER; ++e) ep[e] += v[e] == vj ? pj : 0.f;
                }
            }
        } else {
            v[0] = a.action[t];
            asked = v[0] >= 0 && v[0] < V;
            if (asked) ez[0] = (float)z[v[0]];
            else if (lane == 0) atomicOr(a.g.status, DBW_STATUS_BAD_INDEX);
            if (lane == 0) {
                info.z = asked ? ez[0] : 0.f;
                info.old = a.old_logp[t];
                info.ref = a.kl != 0.f ? a.ref_logp[t] : 0.f;
                info.adv = a.advantage[t];
            }
        }
        if (lane == 0) info.asked = asked;
        // the loose values: this warp's share of the sum
        const float y = lane < cut.loose ? (float)z[cut.loose_at(lane)] : -INFINITY;
        if (lane < 16) info.loose[lane] = y;
        x.m = fmaxf(x.m, y);
        x.s = lane < cut.loose ? power(y, __fmul_rn(x.m, c), c) : 0.f;
        x = join_warp(x, c);
    } else {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) copy_next();
        float own_cm = __fmul_rn(-limit, c);
        f32x2 sums[2] = {pair(0.f, 0.f), pair(0.f, 0.f)};
        auto add = [&](const uint4 (&u)[P], int pieces) {  // this thread's first `pieces` of them
            float most = x.m;
#pragma unroll
            for (int e = 0; e < P; ++e)
                if (e < pieces) most = fmaxf(most, Vec<T>::most(u[e]));
            if (most > x.m) {  // seldom after the first ones
                x.m = most;
                const float cm = __fmul_rn(most, c), by = exp2_fast(own_cm - cm);
                own_cm = cm;
                sums[0] = mul2(sums[0], pair(by, by));
                sums[1] = mul2(sums[1], pair(by, by));
            }
#pragma unroll
            for (int e = 0; e < P; ++e)
                if (e < pieces) add_piece<T>(u[e], own_cm, c, sums);
        };
        uint4 u[P];
        for (int i = 0; i < whole; ++i) {
            next(u);
            add(u, P);
        }
        if (rest) {
            next(u);
            if (last_pieces) add(u, last_pieces);
        }
        x.s = total(sums);
        x = join_warp(x, c);
        if (lane == 0) {
            part_m[0][warp] = x.m;
            part_s[0][warp] = x.s;
        }
    }
    __shared__ float loose_m, loose_s;
    if (helper && lane == 0) {
        loose_m = x.m;
        loose_s = x.s;
    }
    __syncthreads();
    x = join_warp(lane < WARPS ? Softmax{part_m[0][lane], part_s[0][lane]} : lane == WARPS ? Softmax{loose_m, loose_s} : Softmax{-limit, 0.f}, c);
    const bool far = !(fabsf(x.m) < limit);
    if (far) {  // (the same for the whole block)
        x = {-INFINITY, 0.f};
        if (!helper)
            for (int i = tid; i < V; i += G) x.m = fmaxf(x.m, (float)z[i]);
        for (int step = 1; step < 3; ++step) {  // the maximum, then the sum
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                x.m = fmaxf(x.m, __shfl_xor_sync(0xffffffffu, x.m, o));
                x.s += __shfl_xor_sync(0xffffffffu, x.s, o);
            }
            if (!helper && lane == 0) {
                part_m[step][warp] = x.m;
                part_s[step][warp] = x.s;
            }
            __syncthreads();
            x = lane < WARPS ? Softmax{part_m[step][lane], part_s[step][lane]} : Softmax{-INFINITY, 0.f};
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                x.m = fmaxf(x.m, __shfl_xor_sync(0xffffffffu, x.m, o));
                x.s += __shfl_xor_sync(0xffffffffu, x.s, o);
            }
            if (step == 1 && !helper)
                for (int i = tid; i < V; i += G) x.s += power_beyond((float)z[i], x.m, c);
        }
    }
    const float m = x.m, cm = __fmul_rn(m, c);
    auto at_row = [&](float y) { return far ? power_beyond(y, m, c) : power(y, cm, c); };
    if (!info.asked) {
        if (!helper) asm volatile("cp.async.wait_all;" ::: "memory");
        if (d && far) __syncthreads();  // (everybody has read what the far path reads)
        nothing();
        return;
    }

    // ---- the gradient's factor ----
    float f, slope = 0.f;
    if (KIND == POLICY) {
        const Policy r(a, info.z, info.old, info.ref, info.adv, x, c, far);
        if (helper && lane == 0) {
            a.row_loss[t] = r.loss;
            if (a.logp) a.logp[t] = r.logp;
        }
        slope = r.slope * weight * (float)a.over_tau;
        f = -slope / x.s;
    } else {
        if (helper && lane == 0) a.row_loss[t] = Teacher<PER>::loss(cross, z_ref, x, a, c, far);
        f = weight * (float)a.tau / x.s;
    }
    if (!d) {
        if (!helper) asm volatile("cp.async.wait_all;" ::: "memory");
        return;
    }

    // ---- gradient; the few places that get more than that when everybody's values are there ----
    if (!helper) {
        T* out = d + cut.head + tid * VN;
        auto write = [&](const uint4 (&u)[P], int pieces) {
#pragma unroll
            for (int e = 0; e < P; ++e) {
                if (e >= pieces) break;
                float g[VN];
                grade_piece<T>(u[e], cm, c, f, g);
                put(out + e * G * VN, 0, alike, g, leave);
            }
            out += P * G * VN;
        };
        if (!far && !infinite(f)) {
            uint4 u[P];
            for (int i = 0; i < whole; ++i) {
                next(u);
                write(u, P);
            }
            if (rest) {
                next(u);
                write(u, last_pieces);
            }
        } else {
            for (int i = cut.head + tid; i < cut.head + cut.pieces * VN; i += G) {
                const float y = (float)z[i];
                d[i] = T(share(f, at_row(y), y));
            }
        }
        if (tid < cut.loose) d[cut.loose_at(tid)] = T(share(f, at_row(info.loose[tid]), info.loose[tid]));
        asm volatile("cp.async.wait_all;" ::: "memory");
        asm volatile("bar.arrive 1, %0;" ::"n"(G + 32) : "memory");
    } else {
        asm volatile("bar.sync 1, %0;" ::"n"(G + 32) : "memory");
        if (KIND == POLICY) {
            if (lane == 0) d[v[0]] = T(action_share(slope, f, at_row(ez[0]), x.s));
        } else {
            const float scale = weight * (float)a.tau;
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (v[i] >= 0) d[v[i]] = T(fmaf(-scale, ep[i], share(f, at_row(ez[i]), ez[i])));
        }
    }
}

__global__ void __launch_bounds__(kThreads) check_groups_kernel(RowGroups g) {
    dependent_begin();
    check_groups(g);
}

// loss[w] = sum of weight x row_loss over the worker's rows, in an order that depends on their number alone.  A block per worker.
__global__ void __launch_bounds__(kThreads) worker_loss_kernel(RowGroups g, const float* row_weight, const float* row_loss, float* loss) {
    dependent_begin();
    __shared__ double part[kThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int2 own = rows_of(g, blockIdx.x);
    double sum = 0.0;
    for (int t = own.x + threadIdx.x; t < own.y; t += kThreads) {
        const float w = row_weight ? row_weight[t] : 1.f;
        if (w != 0.f) sum += (double)w * (double)row_loss[t];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) part[warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        sum = 0.0;
        for (int k = 0; k < kThreads / 32; ++k) sum += part[k];
        if (!row_weight && own.y > own.x) sum /= (double)(own.y - own.x);
        loss[blockIdx.x] = (float)sum;
    }
}

template <class T, int KIND, int G>
int launch_long(dbw_handle* h, const LossArgs& a, cudaStream_t s) {
    static PerDeviceOnce once;
    const int rc = once.run(h->device, [&]() -> int {
        DBW_CUDA(cudaFuncSetAttribute(long_row_kernel<T, KIND, G>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)stream_smem<G>()));
        return DBW_OK;
    });
    if (rc) return rc;
    launch(long_row_kernel<T, KIND, G>, a.g.rows, G + 32, stream_smem<G>(), s, a);
    DBW_LAUNCHED();
    return DBW_OK;
}

template <class T, int KIND>
int launch_rows(dbw_handle* h, const LossArgs& a, float* loss, cudaStream_t s) {
    if (a.g.rows == 0) {
        const int rc = launch_check_groups(h, a.g.rowstart, 0, s);
        if (rc) return rc;
    } else {
        // A warp where a row fits its registers; else a block of 128, 256 or 512 threads, by the bytes of a row (us, 128 / 256 / 512: rows of
        // 26 KB 175 / 231 / -, 62 KB 53 / 47 / 51, 98 KB - / 91 / 95, 250 KB - / 473 / 430).
        const int64_t bytes = (int64_t)a.vocab * sizeof(T);
        int rc = DBW_OK;
        if (bytes <= 32 * HELD * 16) {
            launch(short_row_kernel<T, KIND>, (a.g.rows + kThreads / 32 - 1) / (kThreads / 32), kThreads, 0, s, a);
            DBW_LAUNCHED();
        } else if (bytes <= 32 * 1024) {
            rc = launch_long<T, KIND, 128>(h, a, s);
        } else if (bytes <= 112 * 1024) {
            rc = launch_long<T, KIND, 256>(h, a, s);
        } else {
            rc = launch_long<T, KIND, 512>(h, a, s);
        }
        if (rc) return rc;
    }
    if (loss) {
        launch(worker_loss_kernel, a.g.N, kThreads, 0, s, a.g, a.row_weight, (const float*)a.row_loss, loss);
        DBW_LAUNCHED();
    }
    return DBW_OK;
}

template <int KIND>
int launch_type(dbw_handle* h, const LossArgs& a, int type, float* loss, cudaStream_t s) {
    return type == DBW_TYPE_F32 ? launch_rows<float, KIND>(h, a, loss, s)
                                : type == DBW_TYPE_BF16 ? launch_rows<__nv_bfloat16, KIND>(h, a, loss, s) : launch_rows<__half, KIND>(h, a, loss, s);
}

}  // namespace

int launch_check_groups(dbw_handle* h, const int32_t* rowstart, int32_t rows, cudaStream_t s) {
    launch(check_groups_kernel, 1, kThreads, 0, s, RowGroups{rowstart, h->N, rows, h->d_status});
    DBW_LAUNCHED();
    return DBW_OK;
}

int launch_distill(dbw_handle* h, const RowLoss& r, const int32_t* top_idx, const float* top_logit, int top, cudaStream_t s) {
    LossArgs a{{r.rowstart, h->N, r.rows, h->d_status}, r.logits, r.ld, r.vocab, r.row_weight, r.row_loss, r.d_logits, r.ld_d, (double)r.temperature, 1.0 / (double)r.temperature};
    a.top_idx = top_idx;
    a.top_logit = top_logit;
    a.top = top;
    return launch_type<DISTILL>(h, a, r.type, r.loss, s);
}

int launch_policy_loss(dbw_handle* h, const RowLoss& r, const int32_t* action, const float* old_logp, const float* ref_logp, const float* advantage,
                       float clip_low, float clip_high, float kl_coef, float* logp, cudaStream_t s) {
    LossArgs a{{r.rowstart, h->N, r.rows, h->d_status}, r.logits, r.ld, r.vocab, r.row_weight, r.row_loss, r.d_logits, r.ld_d, (double)r.temperature, 1.0 / (double)r.temperature};
    a.action = action;
    a.old_logp = old_logp;
    a.ref_logp = ref_logp;
    a.advantage = advantage;
    a.logp = logp;
    a.low = (float)(1.0 - (double)clip_low);
    a.high = (float)(1.0 + (double)clip_high);
    a.kl = kl_coef;
    return launch_type<POLICY>(h, a, r.type, r.loss, s);
}

}  // namespace dbw
