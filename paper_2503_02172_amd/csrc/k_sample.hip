// Drawing entities from score rows, from given random numbers. For a row x of
// N scores and its settings (temperature T, top-k k, top-p p, min-p m):
//   M = max x,  w_i = exp((x_i - M) / T)                (NaN and -inf: 0)
//   first cut   the first k entities in the ranking order (score descending,
//               index ascending)
//   second cut  the shortest prefix of these, in that order, that holds at
//               least p of their weight
//   third cut   those of them with w_i >= m
//   a draw u    the first entity, by index, at which the running sum of what
//               is left exceeds u times its total
// A draw compares sums over the row, so a relative error e of them moves about
// N e of the draws: weights and sums are doubles.
//
// Both cuts along the ranking order are one: a composite (order-preserving key
// of the score, inverted index) above which everything is kept. It is found
// from histograms over ever narrower ranges: first over the distance from M in
// equal steps (scores spread evenly over them), then over the composites of the
// bin that holds the cut, until what is left fits the sort buffer. Counts and
// weights are added with integer atomics (weights in fixed point relative to
// their bin's largest), so the sums do not depend on their order.
#include <algorithm>

#include "row_ops.hpp"

namespace kgq {

namespace {

constexpr int SW = kSampleThreads / 64;
constexpr int kBins = 2048;
constexpr int kSort = 2048;                  // entries that the last step sorts
constexpr int kMaxChunks = 4096;             // partial sums of a row in index order

// 2^t for t <= 0 in doubles, 0 below 2^-1022 and for NaN: Taylor's series of
// 2^r, |r| <= 1/2, cut off below 2^-53 of the value.
__device__ __forceinline__ double pow2d(double t)
{
    t = fmax(t, -1100.0);                    // (a NaN goes here too)
    const double n = rint(t);
    const double r = (t - n) * 0.693147180559945309417;
    double y = 1.0 / 479001600.0;
    y = fma(y, r, 1.0 / 39916800.0);
    y = fma(y, r, 1.0 / 3628800.0);
    y = fma(y, r, 1.0 / 362880.0);
    y = fma(y, r, 1.0 / 40320.0);
    y = fma(y, r, 1.0 / 5040.0);
    y = fma(y, r, 1.0 / 720.0);
    y = fma(y, r, 1.0 / 120.0);
    y = fma(y, r, 1.0 / 24.0);
    y = fma(y, r, 1.0 / 6.0);
    y = fma(y, r, 0.5);
    y = fma(y, r, 1.0);
    y = fma(y, r, 1.0);
    return ldexp(y, (int)n);
}

// A row's weights. Where the maximum is +inf, the infinite scores share the
// weight.
struct RowWeight {
    float M;
    double c;                                // log2(e) / T
    __device__ __forceinline__ double exponent(float x) const
    {
        if (M == INFINITY) return x == INFINITY ? 0.0 : -INFINITY;
        return ((double)x - (double)M) * c;
    }
    __device__ __forceinline__ double operator()(float x) const { return pow2d(exponent(x)); }
};

__device__ __forceinline__ uint64_t ranking(float x, uint32_t i)
{
    return ((uint64_t)score_key(x) << 32) | (uint32_t)~i;
}
__device__ __forceinline__ float ranking_score(uint64_t c)
{
    const uint32_t key = (uint32_t)(c >> 32);
    return __uint_as_float((key & 0x80000000u) ? (key & 0x7FFFFFFFu) : ~key);
}

struct SampleLds {
    union {
        struct {
            uint32_t count[kBins];
            unsigned long long mass[kBins];
        } h;
        struct {
            uint64_t c[kSort];
            double w[kSort];
        } s;
        double chunk[kMaxChunks];
    };
    float fbuf[SW];
    double dbuf[SW];
    uint32_t ubuf[SW];
    unsigned long long lo, hi;
    uint32_t n;
    int bin;
    double above;
    uint32_t ahead;
};

// What a cut looks for along the ranking order: the entry number `count`, or
// the first entry at which the running weight reaches `mass`.
struct CutGoal {
    bool by_mass;
    uint32_t count;
    double mass;
};

// Inclusive running sum over the workgroup in thread order, and the total.
template <typename V>
__device__ __forceinline__ V block_scan(V x, V* buf, V* total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const V o = __shfl_up(x, d, 64);
        if (lane >= d) x += o;
    }
    __syncthreads();
    if (lane == 63) buf[wave] = x;
    __syncthreads();
    V before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < SW; ++w) {
        if (w < wave) before += buf[w];
        all += buf[w];
    }
    *total = all;
    return before + x;
}

// The bin of the histogram at which the goal is met, and what the bins before
// it hold (added to *count / *mass). weight_of: what a bin's fixed-point sum
// is counted in. false: the goal lies behind every bin (the last bin with an
// entry is then taken).
template <typename W>
__device__ __forceinline__ void find_bin(SampleLds& L, const CutGoal& goal, W weight_of, uint32_t* count, double* mass)
{
    constexpr int per = kBins / kSampleThreads;
    const int tid = threadIdx.x;
    uint32_t c[per], csum = 0;
    double m[per], msum = 0.0;
#pragma unroll
    for (int j = 0; j < per; ++j) {
        c[j] = L.h.count[tid * per + j];
        m[j] = goal.by_mass ? (double)L.h.mass[tid * per + j] * weight_of(tid * per + j) : 0.0;
        csum += c[j];
        msum += m[j];
    }
    uint32_t call;
    double mall = 0.0;
    uint32_t cb = block_scan(csum, L.ubuf, &call) - csum;
    double mb = 0.0;
    if (goal.by_mass) mb = block_scan(msum, L.dbuf, &mall) - msum;
    if (tid == 0) L.bin = kBins;
    __syncthreads();
    // the first bin at which the goal is met, or else the last with an entry
    int met = kBins, last = -1;
    uint32_t c_at = 0, c_last = 0;
    double m_at = 0.0, m_last = 0.0;
#pragma unroll
    for (int j = 0; j < per; ++j) {
        if (c[j]) {
            const bool ok = goal.by_mass ? *mass + (mb + m[j]) >= goal.mass : *count + cb + c[j] >= goal.count;
            if (ok && met == kBins) {
                met = tid * per + j;
                c_at = cb;
                m_at = mb;
            }
            last = tid * per + j;
            c_last = cb;
            m_last = mb;
        }
        cb += c[j];
        mb += m[j];
    }
    if (met < kBins) atomicMin(&L.bin, met);
    __syncthreads();
    const bool found = L.bin < kBins;
    __syncthreads();
    if (!found) {
        if (tid == 0) L.bin = -1;
        __syncthreads();
        if (last >= 0) atomicMax(&L.bin, last);
        __syncthreads();
    }
    const int bin = L.bin;
    if (found ? met == bin : last == bin) {
        L.ahead = found ? c_at : c_last;
        L.above = found ? m_at : m_last;
    }
    __syncthreads();
    *count += L.ahead;
    *mass += L.above;
}

// The composite of the last entry that a cut keeps, among the entries with a
// composite of at least `floor` (the cut before). range: distances from M that
// the first histogram spans; entries further off count as one bin.
template <typename T>
__device__ uint64_t find_cut(SampleLds& L, const T* row, int64_t N, const RowWeight& wt, const CutGoal goal,
                             uint64_t floor, float range)
{
    const int tid = threadIdx.x;
    const int bits = 62 - (64 - __builtin_clzll((unsigned long long)N));
    const double unit = ldexp(1.0, bits);
    const float step = range < INFINITY ? range / (float)(kBins - 1) : 0.f;
    const float inv = step > 0.f ? 1.0f / step : 0.f;
    uint32_t count = 0;
    double mass = 0.0;
    unsigned long long lo = floor, hi = ~0ull;
    auto bin_of = [&](float x) {
        const float v = (wt.M - x) * inv;        // 0 and up; NaN (infinite M, or a step of 0) to bin 0
        return v < (float)(kBins - 1) ? max((int)v, 0) : v >= (float)(kBins - 1) ? kBins - 1 : 0;
    };
    for (int level = 0;; ++level) {
        // histogram over [lo, hi]
        for (int i = tid; i < kBins; i += kSampleThreads) {
            L.h.count[i] = 0;
            L.h.mass[i] = 0;
        }
        __syncthreads();
        const int shift = level == 0 ? 0 : max(0, 64 - __builtin_clzll((hi - lo) | 1ull) - 11);
        const double top = level == 0 ? 0.0 : wt.exponent(ranking_score(hi));
        auto scale_of = [&](int bin) { return level == 0 ? fmax((double)bin * (double)step * -wt.c, -1100.0) : top; };
        // (an entry whose distance was rounded up into its bin may weigh a
        // little more than the bin's scale: there is a bit of room for that)
        auto value_bin = [&](float x, unsigned long long c) {
            return level == 0 ? bin_of(x) : (int)((hi - c) >> shift);
        };
        for (int64_t i = tid; i < N; i += kSampleThreads) {
            const float x = row_value(row[i]);
            if (!(x > -INFINITY)) continue;
            const unsigned long long c = ranking(x, (uint32_t)i);
            if (c < lo || c > hi) continue;
            const int bin = value_bin(x, c);
            atomicAdd(&L.h.count[bin], 1u);
            if (goal.by_mass)
                atomicAdd(&L.h.mass[bin], (unsigned long long)(pow2d(fmin(wt.exponent(x) - scale_of(bin), 0.5)) * unit));
        }
        __syncthreads();
        find_bin(L, goal, [&](int bin) { return pow2d(scale_of(bin)) / unit; }, &count, &mass);
        const int bin = L.bin;
        const uint32_t in_bin = L.h.count[bin];
        __syncthreads();
        // the composites in that bin
        if (tid == 0) {
            L.lo = ~0ull;
            L.hi = 0ull;
            L.n = 0;
        }
        __syncthreads();
        const bool take = in_bin <= (uint32_t)kSort;
        unsigned long long mine_lo = ~0ull, mine_hi = 0ull;
        for (int64_t i = tid; i < N; i += kSampleThreads) {
            const float x = row_value(row[i]);
            if (!(x > -INFINITY)) continue;
            const unsigned long long c = ranking(x, (uint32_t)i);
            if (c < lo || c > hi || value_bin(x, c) != bin) continue;
            mine_lo = min(mine_lo, c);
            mine_hi = max(mine_hi, c);
            if (take) L.s.c[atomicAdd(&L.n, 1u)] = c;
        }
        if (!take) {
            if (mine_lo != ~0ull) {
                atomicMin(&L.lo, mine_lo);
                atomicMax(&L.hi, mine_hi);
            }
            __syncthreads();
            lo = L.lo;
            hi = L.hi;
            __syncthreads();
            continue;
        }
        // sorted descending, summed in that order
        int P = 2;
        while (P < (int)in_bin) P <<= 1;
        for (int i = (int)in_bin + tid; i < P; i += kSampleThreads) L.s.c[i] = 0ull;
        __syncthreads();
        for (int size = 2; size <= P; size <<= 1) {
            for (int stride = size >> 1; stride > 0; stride >>= 1) {
                for (int p = tid; p < P / 2; p += kSampleThreads) {
                    const int a = 2 * p - (p & (stride - 1));
                    const uint64_t ca = L.s.c[a], cb = L.s.c[a + stride];
                    const bool down = (a & size) == 0;
                    if (down ? ca < cb : ca > cb) {
                        L.s.c[a] = cb;
                        L.s.c[a + stride] = ca;
                    }
                }
                __syncthreads();
            }
        }
        constexpr int per = kSort / kSampleThreads;
        double w[per], sum = 0.0;
#pragma unroll
        for (int j = 0; j < per; ++j) {
            const int i = tid * per + j;
            w[j] = i < (int)in_bin ? wt(ranking_score(L.s.c[i])) : 0.0;
            sum += w[j];
        }
        double all;
        double before = block_scan(sum, L.dbuf, &all) - sum;
        if (tid == 0) L.n = in_bin - 1;          // (what rounding leaves short of the goal: the last one)
        __syncthreads();
#pragma unroll
        for (int j = 0; j < per; ++j) {
            before += w[j];
            const int i = tid * per + j;
            const bool ok = goal.by_mass ? mass + before >= goal.mass : count + i + 1 >= goal.count;
            if (i < (int)in_bin && ok) atomicMin(&L.n, (uint32_t)i);
        }
        __syncthreads();
        const uint64_t cut = L.s.c[L.n];
        __syncthreads();
        return cut;
    }
}

}  // namespace

// One workgroup per row.
template <typename T>
__global__ __launch_bounds__(kSampleThreads) void k_sample(SampleArgs a)
{
    __shared__ SampleLds L;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t b = blockIdx.x;
    const int64_t N = a.N;
    const T* row = reinterpret_cast<const T*>(a.scores) + b * a.ld;
    const float temperature = a.temperature_rows ? a.temperature_rows[b] : a.temperature;
    const int32_t top_k = a.top_k_rows ? a.top_k_rows[b] : a.top_k;
    const float top_p = a.top_p_rows ? a.top_p_rows[b] : a.top_p;
    const float min_p = a.min_p_rows ? a.min_p_rows[b] : a.min_p;
    const float* u = a.u + b * a.S;
    int32_t* out = a.idx + b * a.S;
    float* logp = a.logp ? a.logp + b * a.S : nullptr;

    const bool bad = !(temperature >= 0.f && temperature < INFINITY) || top_k < 0 || !(top_p > 0.f) ||
                     !(min_p >= 0.f && min_p <= 1.f);
    if (bad && a.flag && tid == 0) atomicOr(a.flag, kErrSettings);

    float M = -INFINITY;
    for (int64_t i = tid; i < N; i += kSampleThreads) M = fmaxf(M, row_value(row[i]));
    M = block_reduce<SW>(M, L.fbuf, OpMax());
    if (bad || M == -INFINITY) {                 // nothing to draw from
        for (int s = tid; s < a.S; s += kSampleThreads) {
            out[s] = -1;
            if (logp) logp[s] = __builtin_nanf("");
        }
        return;
    }
    if (temperature == 0.f || top_k == 1) {      // the first in ranking order
        if (tid == 0) L.n = ~0u;
        __syncthreads();
        for (int64_t i = tid; i < N; i += kSampleThreads)
            if (row_value(row[i]) == M) {
                atomicMin(&L.n, (uint32_t)i);
                break;
            }
        __syncthreads();
        for (int s = tid; s < a.S; s += kSampleThreads) {
            out[s] = (int32_t)L.n;
            if (logp) logp[s] = 0.f;
        }
        return;
    }
    const RowWeight wt{M, 1.4426950408889634074 / (double)temperature};

    uint64_t cut = 0;
    double total;
    const bool by_count = top_k > 0 && top_k < N;
    if (by_count) {
        float lowest = M;
        for (int64_t i = tid; i < N; i += kSampleThreads) {
            const float x = row_value(row[i]);
            if (x > -INFINITY && x < lowest) lowest = x;
        }
        __syncthreads();
        lowest = -block_reduce<SW>(-lowest, L.fbuf, OpMax());
        cut = find_cut(L, row, N, wt, CutGoal{false, (uint32_t)top_k, 0.0}, 0ull, M - lowest);
    }
    if (top_p < 1.f) {
        // the weight that p is a share of
        double sum = 0.0;
        for (int64_t i = tid; i < N; i += kSampleThreads) {
            const float x = row_value(row[i]);
            if (ranking(x, (uint32_t)i) >= cut) sum += wt(x);
        }
        __syncthreads();
        sum = block_reduce<SW>(sum, L.dbuf, OpSum());
        __syncthreads();
        // entries with less than (1 - p) / N of the largest weight lie behind the cut
        const double far = (log((double)N) - log(1.0 - (double)top_p) + 1.0) * (double)temperature;
        const uint64_t c = find_cut(L, row, N, wt, CutGoal{true, 0u, (double)top_p * sum}, cut, (float)fmin(far, 3e38));
        cut = max(cut, c);
    }

    // running sums of what is kept, chunk by chunk in index order
    auto kept = [&](float x, int64_t i) {
        if (!(x > -INFINITY) || ranking(x, (uint32_t)i) < cut) return 0.0;
        const double w = wt(x);
        return w >= (double)min_p ? w : 0.0;
    };
    int64_t len = 64;
    while ((N + len - 1) / len > kMaxChunks) len <<= 1;
    const int n_chunks = (int)((N + len - 1) / len);
    __syncthreads();
    for (int c = wave; c < n_chunks; c += SW) {
        double sum = 0.0;
        const int64_t end = min(N, (c + 1) * len);
        for (int64_t i = c * len + lane; i < end; i += 64) sum += kept(row_value(row[i]), i);
        sum = wave_reduce(sum, OpSum());
        if (lane == 0) L.chunk[c] = sum;
    }
    __syncthreads();
    {
        constexpr int per = kMaxChunks / kSampleThreads;
        double s[per], sum = 0.0, all;
#pragma unroll
        for (int j = 0; j < per; ++j) {
            const int c = tid * per + j;
            s[j] = c < n_chunks ? L.chunk[c] : 0.0;
            sum += s[j];
        }
        double run = block_scan(sum, L.dbuf, &all) - sum;
#pragma unroll
        for (int j = 0; j < per; ++j) {
            run += s[j];
            if (tid * per + j < n_chunks) L.chunk[tid * per + j] = run;
        }
        total = all;
    }
    __syncthreads();

    // one draw per wavefront
    for (int s = wave; s < a.S; s += SW) {
        const float uf = u[s];
        const double target = (uf >= 0.f ? fmin((double)uf, 1.0) : 0.0) * total;
        int lo = 0, hi = n_chunks;               // the first chunk whose running sum exceeds the target
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (L.chunk[mid] > target) hi = mid;
            else lo = mid + 1;
        }
        if (lo == n_chunks) {                    // (u = 1) the last chunk that holds something
            hi = n_chunks - 1;
            lo = 0;
            const double last = L.chunk[n_chunks - 1];
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (L.chunk[mid] >= last) hi = mid;
                else lo = mid + 1;
            }
        }
        const double rest = target - (lo ? L.chunk[lo - 1] : 0.0);
        double run = 0.0, w = 0.0;
        int64_t pick = -1, last = -1;
        double w_last = 0.0;
        const int64_t end = min(N, (lo + 1) * len);
        for (int64_t i0 = lo * len; i0 < end && pick < 0; i0 += 64) {
            const int64_t i = i0 + lane;
            w = i < end ? kept(row_value(row[i]), i) : 0.0;
            double c = w;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const double o = __shfl_up(c, d, 64);
                if (lane >= d) c += o;
            }
            c += run;
            const uint64_t over = __builtin_amdgcn_ballot_w64(c > rest && w > 0.0);
            const uint64_t some = __builtin_amdgcn_ballot_w64(w > 0.0);
            if (over) {
                const int l = __builtin_ctzll(over);
                pick = i0 + l;
                w = __shfl(w, l, 64);
            } else if (some) {
                const int l = 63 - __builtin_clzll(some);
                last = i0 + l;
                w_last = __shfl(w, l, 64);
            }
            run = __shfl(c, 63, 64);
        }
        if (pick < 0) {                          // rounding: the chunk's last
            pick = last;
            w = w_last;
        }
        if (lane == 0) {
            out[s] = (int32_t)pick;
            if (logp) logp[s] = (float)log(w / total);
        }
    }
}

void launch_sample(const SampleArgs& a, hipStream_t s)
{
    if (a.dtype == KGQ_BF16)
        hipLaunchKernelGGL(k_sample<uint16_t>, dim3(a.batch), dim3(kSampleThreads), 0, s, a);
    else
        hipLaunchKernelGGL(k_sample<float>, dim3(a.batch), dim3(kSampleThreads), 0, s, a);
}

}  // namespace kgq
