// Distillation from a teacher's lists. For a row of student scores z (N
// entities) and a teacher's list of k (entity a_j, score t_j), at temperature
// tau:
//   p = softmax(t / tau) over the list,  q = softmax(z / tau) over the entities
//   loss   = tau^2 sum_j p_j (log p_j - log q_{a_j})
//   grad_i = w tau (q_i - sum_{j: a_j = i} p_j)
// with w the row's weight. The list's share of the gradient touches k entries,
// so the row is one softmax: a maximum, a sum, and one product per entry. One
// workgroup takes a row; up to 65,536 scores stay in registers from the load to
// the store, so that the row is read once and written once.
#include <algorithm>

#include "row_ops.hpp"

namespace kgq {

namespace {

constexpr int kHash = 2 * kMaxK;       // slots of the list's entities at most

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

template <int DW>
struct DistillLds {
    int32_t key[kHash];
    unsigned long long sum[kHash];
    float top[DW], list_top[DW];
    int any[DW];
    double sum_exp[DW], list_sum[DW], loss[DW];
};

// V elements at p.
template <typename T, int V>
struct Elements {
    typedef T vec __attribute__((ext_vector_type(V), aligned(sizeof(T))));
};
// The same 16 bytes as words, and element e of them.
template <typename T>
struct Words;
template <>
struct Words<float> {
    typedef uint32_t vec __attribute__((ext_vector_type(4), aligned(4)));
};
template <>
struct Words<uint16_t> {
    typedef uint32_t vec __attribute__((ext_vector_type(4), aligned(2)));
};
template <typename T, typename W>
__device__ __forceinline__ float word_value(const W& w, int e)
{
    if (sizeof(T) == 4) return __uint_as_float(w[e]);
    return __uint_as_float(e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
}

}  // namespace

// One workgroup per row. NV > 0: the row's scores in registers, NV vectors of
// 16 bytes a thread and the row's end beside them; their exponentials take the
// scores' place, or (KEEP false, bfloat16: half the registers, and twice the
// rows in flight) are computed again for the gradient. NV = 0: the row is read
// twice. Three barriers: behind the maxima, the sums, and the row's stores.
// Bound by memory where rows are many: 2,048 rows of 63,361, K = 100: 237 us a
// call among others (243 as profiled), 4.4 TB/s read and written (a plain copy of
// the scores 195 us: it has no barrier between its loads and its stores, and more
// than one row a compute unit to fill the gaps). 1,024 in bfloat16, K = 1,000: 98
// us (95), 2.6 TB/s, where the exponentials, two a score, take as long as the
// bytes. 509 rows of 14,505: 15 us (15.8), 4.0 TB/s. 32 rows of 1,000: 6 us as
// profiled, the latency of the three barriers. The loss alone of 2,048 rows: 150
// us, 3.5 TB/s read; 500 rows of 200,000, read twice: 250 us.
template <typename T, int DT, int NV, bool KEEP, int WAVES>
__global__ __launch_bounds__(DT, WAVES) void k_distill(DistillArgs a, float chi, float clo, int slots)
{
    constexpr int V = RowVec<T>::n, DW = DT / 64, PER = kMaxK / DT;
    typedef typename Elements<T, V>::vec vec;
    __shared__ DistillLds<DW> L;
    const int tid = threadIdx.x, wave = tid >> 6;
    const int64_t b = blockIdx.x, N = a.N;
    const T* z = reinterpret_cast<const T*>(a.scores) + b * a.ld;
    T* g = a.grad ? reinterpret_cast<T*>(a.grad) + b * a.ld_grad : nullptr;

    // the teacher's list, PER entries a thread at most
    int32_t id[PER];
    float t[PER], zj[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int j = k * DT + tid;
        id[k] = j < a.k ? a.idx[b * a.k + j] : -1;
        t[k] = j < a.k ? a.teacher[b * a.k + j] : -INFINITY;
    }
    // the row: whole vectors (those past the end load the last whole one and
    // count as -inf), and the last elements, one by one, in one thread
    const int64_t whole = N / V;
    const bool last = tid == (int)(whole % DT);
    typename Words<T>::vec raw[NV > 0 ? NV : 1];
    float x[NV > 0 && KEEP ? NV : 1][V], tail[V];
    if constexpr (NV > 0) {
        if (whole > 0) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
                raw[j] = *reinterpret_cast<const typename Words<T>::vec*>(z + min((int64_t)(j * DT + tid), whole - 1) * V);
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) tail[e] = last && whole * V + e < N ? row_value(z[whole * V + e]) : -INFINITY;

    for (int i = tid; i < slots; i += DT) {
        L.key[i] = -1;
        L.sum[i] = 0ull;
    }
    float tmax = -INFINITY;
    bool any = false;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        if (id[k] >= N || id[k] < -1) {
            if (a.flag) atomicOr(a.flag, kErrRange);
            id[k] = -1;
        }
        zj[k] = 0.f;
        if (id[k] >= 0) {
            zj[k] = row_value(z[id[k]]);
            any |= !(t[k] == -INFINITY);               // (a NaN is a target: it makes the row NaN)
        } else {
            t[k] = -INFINITY;
        }
        tmax = fmaxf(tmax, t[k]);
    }
    // the maxima
    auto value = [&](int j, int e) __attribute__((always_inline)) {
        return (int64_t)(j * DT + tid) < whole ? word_value<T>(raw[j], e) : -INFINITY;
    };
    float m = -INFINITY, part = 0.f;
    if constexpr (NV > 0) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float y = value(j, e);
                if (KEEP) x[j][e] = y;
                m = fmaxf(m, y);
            }
#pragma unroll
        for (int e = 0; e < V; ++e) m = fmaxf(m, tail[e]);
    } else {
        // (and each thread's sum relative to its own)
        auto add = [&](const float (&y)[V]) __attribute__((always_inline)) {
            float top = y[0];
#pragma unroll
            for (int e = 1; e < V; ++e) top = fmaxf(top, y[e]);
            if (top > m) {
                part *= exp_of(m - top, chi, clo);
                m = top;
            }
#pragma unroll
            for (int e = 0; e < V; ++e) part += y[e] == -INFINITY ? 0.f : exp_of(y[e] - m, chi, clo);
        };
#pragma unroll 4
        for (int64_t i = tid; i < whole; i += DT) {
            const vec r = *reinterpret_cast<const vec*>(z + i * V);
            float y[V];
#pragma unroll
            for (int e = 0; e < V; ++e) y[e] = row_value((T)r[e]);
            add(y);
        }
        add(tail);
    }
    const float mine = m;
    m = wave_reduce(m, OpMax());
    tmax = wave_reduce(tmax, OpMax());
    any = __builtin_amdgcn_ballot_w64(any) != 0;
    if ((tid & 63) == 0) {
        L.top[wave] = m;
        L.list_top[wave] = tmax;
        L.any[wave] = any;
    }
    __syncthreads();
    bool empty = true;
#pragma unroll
    for (int w = 0; w < DW; ++w) {
        m = fmaxf(m, L.top[w]);
        tmax = fmaxf(tmax, L.list_top[w]);
        empty &= !L.any[w];
    }
    // (what was computed of the scores is not to be kept, where they are)
    auto again = [&]() __attribute__((always_inline)) {
        if constexpr (NV > 0 && !KEEP) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    uint32_t u = raw[j][k];
                    asm volatile("" : "+v"(u));
                    raw[j][k] = u;
                }
        }
    };
    // the sums
    double p[PER], zt = 0.0, Z = 0.0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        p[k] = 0.0;
        if (id[k] >= 0 && !(t[k] == -INFINITY))
            p[k] = tmax == INFINITY ? (t[k] == INFINITY ? 1.0 : t[k] != t[k] ? (double)t[k] : 0.0)
                                    : exp(((double)t[k] - (double)tmax) * a.inv_tau);
        zt += p[k];
    }
    if constexpr (NV > 0) {
        float s[V] = {};
        again();
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float y = exp_of((KEEP ? x[j][e] : value(j, e)) - m, chi, clo);
                if (KEEP) x[j][e] = y;
                s[e] += y;
            }
        // (a row of -inf alone is NaN: so is every difference from its maximum)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            tail[e] = exp_of(tail[e] - m, chi, clo);
            Z += (double)(s[e] + tail[e]);
        }
    } else {
        // (NaN where a score is: the factor must not hide it)
        Z = part == 0.f && m > -INFINITY ? 0.0 : (double)(part * exp_of(mine - m, chi, clo));
#pragma unroll
        for (int e = 0; e < V; ++e) tail[e] = exp_of(tail[e] - m, chi, clo);
    }
    Z = wave_reduce(Z, OpSum());
    zt = wave_reduce(zt, OpSum());
    if ((tid & 63) == 0) {
        L.sum_exp[wave] = Z;
        L.list_sum[wave] = zt;
    }
    __syncthreads();
    Z = zt = 0.0;
#pragma unroll
    for (int w = 0; w < DW; ++w) {
        Z += L.sum_exp[w];
        zt += L.list_sum[w];
    }
    double l = 0.0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        p[k] /= zt;
        if (a.loss && (p[k] > 0.0 || p[k] != p[k])) {
            const double logp = (tmax == INFINITY ? 0.0 : ((double)t[k] - (double)tmax) * a.inv_tau) - log(zt);
            const double logq = ((double)zj[k] - (double)m) * a.inv_tau - log(Z);
            l += p[k] * (logp - logq);
        }
    }
    if (a.loss) {
        l = wave_reduce(l, OpSum());
        if ((tid & 63) == 0) L.loss[wave] = l;
    }

    const float w = a.weight ? a.weight[b] : 1.f;
    // (a factor beyond float32 makes the whole row NaN, not some entries
    // infinite and the masked ones NaN)
    const double product = (double)w * a.tau, wt = fabs(product) <= 3.4028234664e38 ? product : __builtin_nan("");
    // a row without a target, or without weight, has no gradient
    const bool zero = empty || w == 0.f;
    const float f = zero ? 0.f : (float)(zt == zt ? wt / Z : zt);
    // entries of one entity add up, in fixed point, so that their order does
    // not matter; the thread that opened the entity's slot writes its entry
    int slot[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        slot[k] = -1;
        if (g && id[k] >= 0 && zt == zt && !zero) {
            const unsigned long long fixed = (unsigned long long)(p[k] * 0x1p62);
            uint32_t at = ((uint32_t)id[k] * 2654435769u) >> 16 & (uint32_t)(slots - 1);
            for (;;) {
                const int32_t was = atomicCAS(&L.key[at], -1, id[k]);
                if (was == -1) slot[k] = (int)at;
                if (was == -1 || was == id[k]) break;
                at = (at + 1) & (uint32_t)(slots - 1);
            }
            atomicAdd(&L.sum[at], fixed);
        }
    }
    auto store = [&](int64_t i, const float (&y)[V]) __attribute__((always_inline)) {
        vec r;
#pragma unroll
        for (int e = 0; e < V; ++e) r[e] = row_element<T>(zero ? 0.f : y[e] * f);
        *reinterpret_cast<vec*>(g + i * V) = r;
    };
    if (g) {
        again();
        if constexpr (NV > 0) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float y[V];
#pragma unroll
                for (int e = 0; e < V; ++e) y[e] = KEEP ? x[j][e] : exp_of(value(j, e) - m, chi, clo);
                if ((int64_t)(j * DT + tid) < whole) store(j * DT + tid, y);
            }
        } else {
#pragma unroll 4
            for (int64_t i = tid; i < whole; i += DT) {
                const vec r = *reinterpret_cast<const vec*>(z + i * V);
                float y[V];
#pragma unroll
                for (int e = 0; e < V; ++e) y[e] = exp_of(row_value((T)r[e]) - m, chi, clo);
                store(i, y);
            }
        }
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (last && whole * V + e < N) g[whole * V + e] = row_element<T>(zero ? 0.f : tail[e] * f);
    }
    // the entries of the list, behind the row's own
    __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
    __syncthreads();
    if (a.loss && tid == 0) {
        l = 0.0;
#pragma unroll
        for (int v = 0; v < DW; ++v) l += L.loss[v];
        a.loss[b] = empty ? 0.f : (float)(l * a.tau * a.tau);
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        if (slot[k] >= 0) {
            const double q = (double)exp_of(zj[k] - m, chi, clo) / Z;
            g[id[k]] = row_element<T>((float)(wt * (q - (double)L.sum[slot[k]] * 0x1p-62)));
        }
    }
}

namespace {

template <typename T>
void launch(const DistillArgs& a, hipStream_t s)
{
    const double c = 1.4426950408889634074 / a.tau;
    const float chi = (float)c;
    const float clo = chi > 0.f && chi < INFINITY ? (float)((c - (double)chi) / c) : 0.f;
    int slots = 64;
    while (slots < 2 * a.k) slots <<= 1;
    constexpr int V = RowVec<T>::n;
    auto go = [&](auto kernel, int threads) {
        hipLaunchKernelGGL(kernel, dim3(a.batch), dim3(threads), 0, s, a, chi, clo, slots);
    };
    // The row in registers where it fits, several rows to a compute unit where
    // the scores are few: 16 a thread up to 4,096 (2,048 rows of 4,000: 21 us, 35
    // with 32 a thread), 32 up to 16,384 (of 14,505: 45 us, 109 with 128), 128 up
    // to 65,536 (of 63,361: 237 us, 327 read twice; one row: 15 and 22). Of
    // bfloat16, two rows fit a compute unit if the exponentials are computed
    // twice: slower up to two rows a compute unit (one row 20 us, 15 kept; 512:
    // 42 and 41), faster behind (2,048: 152 and 176).
    if (a.N <= 4096) {
        go(k_distill<T, 256, 16 / V, true, 4>, 256);
    } else if (a.N <= 16384) {
        go(k_distill<T, 512, 32 / V, true, 4>, 512);
    } else if (a.N <= 65536) {
        if constexpr (sizeof(T) == 2) {
            if (a.batch > 512) return go(k_distill<T, 512, 128 / V, false, 4>, 512);
        }
        go(k_distill<T, 512, 128 / V, true, 2>, 512);
    } else {
        go(k_distill<T, 1024, 0, false, 4>, 1024);
    }
}

}  // namespace

void launch_distill(const DistillArgs& a, hipStream_t s)
{
    if (a.dtype == KGQ_BF16) launch<uint16_t>(a, s);
    else launch<float>(a, s);
}

}  // namespace kgq
