// Distillation from a teacher's lists. For a row of student scores z (N
// entities) and a teacher's list of k (entity a_j, score t_j), at temperature
// tau:
//   p = softmax(t / tau) over the list,  q = softmax(z / tau) over the entities
//   loss   = tau^2 sum_j p_j (log p_j - log q_{a_j})
//   grad_i = w tau (q_i - sum_{j: a_j = i} p_j)
// with w the row's weight. The list's share of the gradient touches k entries,
// so the row is one softmax: a maximum, a sum, and one product per entry.
#include <algorithm>

#include "row_ops.hpp"

namespace kgq {

namespace {

constexpr int DT = 1024;               // threads per row
constexpr int DW = DT / 64;
constexpr int kHash = 2 * kMaxK;       // slots of the list's entities

// exp(d / tau) for d <= 0 by its power of two: d log2(e) / tau = n + r, both
// of it from d itself, so that the error is the one of exp2 and of d's
// rounding, however far d lies. chi = log2(e) / tau, clo its rounding error
// over chi. -inf gives 0, NaN stays.
__device__ __forceinline__ float exp_of(float d, float chi, float clo)
{
    const float n = fmaxf(rintf(d * chi), -0x1p20f);
    const float r = fmaf(n, clo, fmaf(d, chi, -n));
    return ldexpf(__builtin_amdgcn_exp2f(r), (int)n);
}

struct DistillLds {
    int32_t key[kHash];
    unsigned long long sum[kHash];
    float fbuf[DW];
    double dbuf[DW];
    double dbuf2[DW];
    int any;
};

}  // namespace

// One workgroup per row.
template <typename T>
__global__ __launch_bounds__(DT) void k_distill(DistillArgs a, float chi, float clo)
{
    __shared__ DistillLds L;
    const int tid = threadIdx.x;
    const int64_t b = blockIdx.x;
    const T* z = reinterpret_cast<const T*>(a.scores) + b * a.ld;
    T* g = a.grad ? reinterpret_cast<T*>(a.grad) + b * a.ld_grad : nullptr;

    for (int i = tid; i < kHash; i += DT) {
        L.key[i] = -1;
        L.sum[i] = 0ull;
    }
    if (tid == 0) L.any = 0;
    __syncthreads();

    // the teacher's list, one entry per thread
    const double inv_tau = 1.0 / (double)a.tau;
    int32_t id = -1;
    float t = -INFINITY, zj = 0.f;
    if (tid < a.k) {
        id = a.idx[b * a.k + tid];
        t = a.teacher[b * a.k + tid];
        if (id >= a.N || id < -1) {
            if (a.flag) atomicOr(a.flag, kErrRange);
            id = -1;
        }
        if (id >= 0) {
            zj = row_value(z[id]);
            if (!(t == -INFINITY)) L.any = 1;          // (a NaN is a target: it makes the row NaN)
        } else {
            t = -INFINITY;
        }
    }
    const float tmax = block_reduce<DW>(t, L.fbuf, OpMax());
    const bool empty = L.any == 0;
    double e = 0.0;
    if (id >= 0) e = tmax == INFINITY ? (t == INFINITY ? 1.0 : t != t ? (double)t : 0.0) : exp(((double)t - (double)tmax) * inv_tau);
    if (t == -INFINITY) e = 0.0;
    const double zt = block_reduce<DW>(e, L.dbuf, OpSum());
    const double p = e / zt;

    // the row's maximum and sum
    float m = -INFINITY;
    for (int64_t i = tid; i < a.N; i += DT) m = fmaxf(m, row_value(z[i]));
    __syncthreads();
    m = block_reduce<DW>(m, L.fbuf, OpMax());
    float s = 0.f;
    for (int64_t i = tid; i < a.N; i += DT) s += exp_of(row_value(z[i]) - m, chi, clo);
    const double Z = block_reduce<DW>((double)s, L.dbuf2, OpSum());

    if (a.loss) {
        double l = 0.0;
        if (p > 0.0 || p != p) {
            const double logp = (tmax == INFINITY ? 0.0 : ((double)t - (double)tmax) * inv_tau) - log(zt);
            const double logq = ((double)zj - (double)m) * inv_tau - log(Z);
            l = p * (logp - logq);
        }
        __syncthreads();
        l = block_reduce<DW>(l, L.dbuf, OpSum());
        if (tid == 0) a.loss[b] = empty ? 0.f : (float)(l * (double)a.tau * (double)a.tau);
    }
    if (!g) return;

    const float w = a.weight ? a.weight[b] : 1.f;
    // a row without a target, or without weight, has no gradient
    if (empty || w == 0.f) {
        for (int64_t i = tid; i < a.N; i += DT) g[i] = row_element<T>(0.f);
        return;
    }
    // entries of one entity add up, in fixed point, so that their order does
    // not matter; the thread that opened the entity's slot writes its entry
    int slot = -1;
    if (id >= 0 && zt == zt) {
        const unsigned long long fixed = (unsigned long long)(p * 0x1p62);
        int at = (int)(((uint32_t)id * 2654435769u) >> 21);
        for (;;) {
            const int32_t was = atomicCAS(&L.key[at], -1, id);
            if (was == -1) slot = at;
            if (was == -1 || was == id) break;
            at = (at + 1) & (kHash - 1);
        }
        atomicAdd(&L.sum[at], fixed);
    }
    const double wt = (double)w * (double)a.tau;
    const float f = (float)(zt == zt ? wt / Z : zt);
    for (int64_t i = tid; i < a.N; i += DT) g[i] = row_element<T>(exp_of(row_value(z[i]) - m, chi, clo) * f);
    __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
    __syncthreads();
    if (slot >= 0) {
        const double q = (double)exp_of(zj - m, chi, clo) / Z;
        g[id] = row_element<T>((float)(wt * (q - (double)L.sum[slot] * 0x1p-62)));
    }
}

void launch_distill(const DistillArgs& a, hipStream_t s)
{
    const double c = 1.4426950408889634074 / (double)a.tau;
    const float chi = (float)c;
    const float clo = (float)((c - (double)chi) / c);
    if (a.dtype == KGQ_BF16)
        hipLaunchKernelGGL(k_distill<uint16_t>, dim3(a.batch), dim3(DT), 0, s, a, chi, clo);
    else
        hipLaunchKernelGGL(k_distill<float>, dim3(a.batch), dim3(DT), 0, s, a, chi, clo);
}

}  // namespace kgq
