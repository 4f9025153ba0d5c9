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
// Without cuts (k_sample_sums, k_sample_draw) the row is read once, by as many
// wavefronts as it has pieces of 1,024 scores: the weights' sums of every 64
// scores, relative to the piece's largest. The draws then search these sums and
// read again only the 64 scores that each of them ends in.
//
// With cuts (k_sample_rows) one workgroup holds the row in registers, up to
// 65,536 scores. Both cuts along the ranking order are one: a composite
// (order-preserving key of the score, inverted index) from which on everything
// is kept. A histogram of the distances from M counts where it lies: for top-k
// in one bin, for top-p in the few bins around the place at which the counts,
// times the weight at each bin's middle, reach p. One pass in doubles then sums
// the row, what lies before those bins, and lists what lies in them; the list,
// sorted, gives the cut exactly, or says that it lies elsewhere. Such rows are
// left to a second launch (k_sample_far), which narrows the range down by
// histogram after histogram, counts and fixed-point weights added with integer
// atomics, whose order does not matter.
#include <algorithm>
#include <type_traits>

#include "row_ops.hpp"

namespace kgq {

namespace {

constexpr int kBins = 2048;
constexpr int kSort = 2048;                  // entries that are sorted for a cut
constexpr int kRun = 16;                     // lanes per draw, and per 64 scores
constexpr int kPiece = 1024;                 // scores of a row per wavefront, without cuts
constexpr int kMaxPieces = 8192;             // of a row (their running sums lie in LDS)

// 2^t for t <= 0 in doubles, 0 below 2^-1074 and for NaN. On |r| <= 1/2 the
// polynomial interpolates 2^r at Chebyshev's points; it is off by 3e-16.
__device__ __forceinline__ double pow2d(double t)
{
    t = fmax(t, -1100.0);                    // (a NaN goes here too)
    const double n = rint(t);
    const double r = t - n;
    double y = 7.072585949269223e-09;
    y = fma(y, r, 1.0208690299958306e-07);
    y = fma(y, r, 1.321544258792169e-06);
    y = fma(y, r, 1.5252657260200837e-05);
    y = fma(y, r, 0.0001540353044173605);
    y = fma(y, r, 0.0013333558230164974);
    y = fma(y, r, 0.009618129107606888);
    y = fma(y, r, 0.05550410866444772);
    y = fma(y, r, 0.24022650695910097);
    y = fma(y, r, 0.69314718055995);
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

// THREADS per row; CHUNKS running sums of the row in index order.
template <int THREADS, int CHUNKS>
struct SampleLds {
    static constexpr int waves = THREADS / 64;
    union {
        struct {
            uint32_t count[kBins];
            unsigned long long mass[kBins];
        } h;
        struct {
            uint64_t c[kSort];
            unsigned long long extra[CHUNKS];
        } s;
    };
    double chunk[CHUNKS];
    float fbuf[waves];
    double dbuf[waves], dbuf2[waves];
    uint32_t ubuf[waves];
    unsigned long long lo, hi;
    uint32_t n;
    int bin, last;
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
template <int WAVES, typename V>
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
    for (int w = 0; w < WAVES; ++w) {
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
template <int THREADS, int CHUNKS, typename W>
__device__ __forceinline__ void find_bin(SampleLds<THREADS, CHUNKS>& L, const CutGoal& goal, W weight_of, uint32_t* count,
                                         double* mass)
{
    constexpr int per = kBins / THREADS, SW = THREADS / 64;
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
    uint32_t cb = block_scan<SW>(csum, L.ubuf, &call) - csum;
    double mb = 0.0;
    if (goal.by_mass) mb = block_scan<SW>(msum, L.dbuf, &mall) - msum;
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

// The composites L.s.c[0 .. n), sorted descending.
template <int THREADS, int CHUNKS>
__device__ __forceinline__ void sort_list(SampleLds<THREADS, CHUNKS>& L, int n)
{
    const int tid = threadIdx.x;
    int P = 2;
    while (P < n) P <<= 1;
    for (int i = n + tid; i < P; i += THREADS) L.s.c[i] = 0ull;
    __syncthreads();
    for (int size = 2; size <= P; size <<= 1) {
        for (int stride = size >> 1; stride > 0; stride >>= 1) {
            for (int p = tid; p < P / 2; p += THREADS) {
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
}

// Sorts the list L.s.c[0 .. n), n <= kSort, and finds the entry of it at which
// the goal is met, behind `count` entries of weight `mass`; n if it is not.
template <int THREADS, int CHUNKS>
__device__ __forceinline__ uint32_t sorted_cut(SampleLds<THREADS, CHUNKS>& L, int n, const RowWeight& wt,
                                               const CutGoal& goal, uint32_t count, double mass)
{
    constexpr int per = kSort / THREADS;
    const int tid = threadIdx.x;
    sort_list(L, n);
    if (!goal.by_mass) return goal.count - count - 1 < (uint32_t)n ? goal.count - count - 1 : (uint32_t)n;
    double w[per], sum = 0.0, all;
#pragma unroll
    for (int j = 0; j < per; ++j) {
        const int i = tid * per + j;
        w[j] = i < n ? wt(ranking_score(L.s.c[i])) : 0.0;
        sum += w[j];
    }
    double before = block_scan<THREADS / 64>(sum, L.dbuf, &all) - sum;
    if (tid == 0) L.n = (uint32_t)n;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < per; ++j) {
        before += w[j];
        const int i = tid * per + j;
        if (i < n && mass + before >= goal.mass) atomicMin(&L.n, (uint32_t)i);
    }
    __syncthreads();
    return L.n;
}

// The composite of the last entry that a cut keeps, among the entries with a
// composite of at least `floor` (the cut before). range: distances from M that
// the first histogram spans; entries further off count as one bin.
template <int THREADS, int CHUNKS, typename T>
__device__ __forceinline__ uint64_t find_cut(SampleLds<THREADS, CHUNKS>& L, const T* row, int64_t N, const RowWeight& wt,
                                             const CutGoal& goal, uint64_t floor, float range)
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
        for (int i = tid; i < kBins; i += THREADS) {
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
        for (int64_t i = tid; i < N; i += THREADS) {
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
        for (int64_t i = tid; i < N; i += THREADS) {
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
        __syncthreads();
        const uint32_t at = sorted_cut(L, (int)in_bin, wt, goal, count, mass);
        const uint64_t cut = L.s.c[at == in_bin ? in_bin - 1 : at];   // (short of the goal by rounding: the last one)
        __syncthreads();
        return cut;
    }
}

// Four scores from element i (a multiple of 4) on, -inf past the row's end.
// Without a branch: a vector that reaches past the end is loaded from the
// row's last four (a row below four: element by element) and shifted by end4,
// so that loads of several vectors stay in flight together.
template <typename T>
struct Four {
    typedef T vec __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    vec v;
    __device__ __forceinline__ void load(const T* row, int64_t i, int64_t N)
    {
        if (N >= 4) {
            v = *reinterpret_cast<const vec*>(row + min(i, N - 4));
        } else {
            v[0] = row[0];
            v[1] = row[N > 1 ? 1 : 0];
            v[2] = v[3] = row[N - 1];
        }
    }
    __device__ __forceinline__ void get(float (&x)[4]) const
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = row_value((T)v[e]);
    }
};
__device__ __forceinline__ void end4(float (&x)[4], int64_t i, int64_t N)
{
    const int over = (int)min(i + 4 - N, (int64_t)4);
    if (over <= 0) return;
    if (N >= 4) {
        x[0] = over == 1 ? x[1] : over == 2 ? x[2] : over == 3 ? x[3] : -INFINITY;
        x[1] = over == 1 ? x[2] : over == 2 ? x[3] : -INFINITY;
        x[2] = over == 1 ? x[3] : -INFINITY;
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e) x[e] = e < 4 - over ? x[e] : -INFINITY;
    }
    x[3] = -INFINITY;
}
template <typename T>
__device__ __forceinline__ void load4(const T* row, int64_t i, int64_t N, float (&x)[4])
{
    Four<T> f;
    f.load(row, i, N);
    f.get(x);
    end4(x, i, N);
}

// Sum over 16 neighbouring lanes, the same in each.
__device__ __forceinline__ double sum16(double x)
{
    auto step = [&](auto ctrl) {
        const uint64_t u = __builtin_bit_cast(uint64_t, x);
        const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, decltype(ctrl)::value, 0xF, 0xF, false);
        const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(u >> 32), decltype(ctrl)::value, 0xF, 0xF, false);
        x += __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
    };
    step(std::integral_constant<int, 0xB1>());       // neighbours
    step(std::integral_constant<int, 0x4E>());       // pairs
    step(std::integral_constant<int, 0x141>());      // half rows mirrored
    step(std::integral_constant<int, 0x140>());      // rows mirrored
    return x;
}

__device__ __forceinline__ double scan16(double x)
{
    const int lane = threadIdx.x & (kRun - 1);
#pragma unroll
    for (int d = 1; d < kRun; d <<= 1) {
        const double o = __shfl_up(x, d, kRun);
        if (lane >= d) x += o;
    }
    return x;
}

// A predicate's lanes among the 16 of a draw.
__device__ __forceinline__ uint32_t ballot16(bool b)
{
    return (uint32_t)(__builtin_amdgcn_ballot_w64(b) >> (threadIdx.x & 48)) & 0xFFFFu;
}

// The first of run[0 .. n), ascending, above the target (n: none), by 16 lanes.
__device__ __forceinline__ int search16(const double* run, int n, double target)
{
    const int lane = threadIdx.x & (kRun - 1);
    int lo = 0, hi = n;
    while (lo < hi) {
        const int step = (hi - lo + kRun - 1) / kRun;
        const int at = lo + lane * step;
        const int k = __popc(ballot16(at < hi && !(run[at < hi ? at : lo] > target)));
        if (k == 0) return lo;
        hi = min(hi, lo + k * step);
        lo = lo + (k - 1) * step + 1;
    }
    return lo;
}

// Where a draw of a row ends: 16 lanes over the scores [i0, end), of which
// weigh(x, i) is what is kept. The first element at which the running sum
// exceeds rest, or the last one with a weight. w: its weight.
template <typename T, typename W>
__device__ __forceinline__ int64_t pick16(const T* row, int64_t N, int64_t i0, int64_t end, double rest, W weigh, double* w)
{
    const int lane = threadIdx.x & (kRun - 1);
    double run = 0.0, w_pick = 0.0;
    int64_t pick = -1;
    for (; i0 < end; i0 += 4 * kRun) {
        const int64_t i = i0 + lane * 4;
        float x[4];
        double v[4], sum = 0.0;
        load4(row, i, N, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = weigh(x[e], i + e);
            sum += v[e];
        }
        const double incl = run + scan16(sum);
        const uint32_t some = ballot16(sum > 0.0), over = ballot16(sum > 0.0 && incl > rest);
        // (no lane over yet: the last one with a weight, in case there is no other)
        const int l = over ? __builtin_ctz(over) : some ? 31 - __builtin_clz(some) : -1;
        if (l >= 0) {
            double before = __shfl_up(incl, 1, kRun);
            if (lane == 0) before = run;
            int at = 0;
            bool found = false;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (v[e] > 0.0 && !found) {
                    at = e;
                    before += v[e];
                    found = over && before > rest;
                }
            }
            pick = i0 + l * 4 + __shfl(at, l, kRun);
            w_pick = __shfl(at == 0 ? v[0] : at == 1 ? v[1] : at == 2 ? v[2] : v[3], l, kRun);
        }
        if (over) break;
        run = __shfl(incl, kRun - 1, kRun);
    }
    *w = w_pick;
    return pick;
}

__device__ __forceinline__ double draw_share(float u) { return u >= 0.f ? fmin((double)u, 1.0) : 0.0; }

// A row's settings.
struct RowSettings {
    float temperature, top_p, min_p;
    int32_t top_k;
    __device__ __forceinline__ RowSettings(const SampleArgs& a, int64_t b)
        : temperature(a.temperature_rows ? a.temperature_rows[b] : a.temperature),
          top_p(a.top_p_rows ? a.top_p_rows[b] : a.top_p),
          min_p(a.min_p_rows ? a.min_p_rows[b] : a.min_p),
          top_k(a.top_k_rows ? a.top_k_rows[b] : a.top_k)
    {
    }
    __device__ __forceinline__ bool bad() const
    {
        return !(temperature >= 0.f && temperature < INFINITY) || top_k < 0 || !(top_p > 0.f) ||
               !(min_p >= 0.f && min_p <= 1.f);
    }
    __device__ __forceinline__ double c() const { return 1.4426950408889634074 / (double)temperature; }
};

}  // namespace

// ---- without cuts -------------------------------------------------------------

// A row's pieces: the largest score of each and, relative to it, the weights'
// sums of its 16 chunks.
struct SamplePieces {
    double* sums;                            // [batch x pieces x 16]
    float* best;                             // [batch x pieces]
    int pieces;
};

template <typename T>
__global__ __launch_bounds__(256) void k_sample_sums(SampleArgs a, SamplePieces q)
{
    const int lane = threadIdx.x & 63;
    const int64_t wave = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t b = wave / q.pieces, piece = wave % q.pieces;
    if (b >= a.batch) return;
    const T* row = reinterpret_cast<const T*>(a.scores) + b * a.ld;
    Four<T> f[4];
    float x[4][4], best = -INFINITY;
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j].load(row, piece * kPiece + j * 256 + lane * 4, a.N);
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j].get(x[j]);
    if ((piece + 1) * kPiece > a.N) {
#pragma unroll
        for (int j = 0; j < 4; ++j) end4(x[j], piece * kPiece + j * 256 + lane * 4, a.N);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) best = fmaxf(best, x[j][e]);
    best = wave_reduce(best, OpMax());
    const RowWeight wt{best, RowSettings(a, b).c()};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const double s = sum16((wt(x[j][0]) + wt(x[j][1])) + (wt(x[j][2]) + wt(x[j][3])));
        if ((lane & (kRun - 1)) == 0) q.sums[wave * 16 + j * 4 + lane / kRun] = s;
    }
    if (lane == 0) q.best[wave] = best;
}

template <typename T>
__global__ __launch_bounds__(256) void k_sample_draw(SampleArgs a, SamplePieces q)
{
    extern __shared__ double run[];                  // [pieces]
    __shared__ float fbuf[4];
    __shared__ double dbuf[4];
    __shared__ uint32_t first;
    const int tid = threadIdx.x, lane = tid & (kRun - 1);
    const int64_t b = blockIdx.x, N = a.N;
    const T* row = reinterpret_cast<const T*>(a.scores) + b * a.ld;
    const float* best = q.best + b * q.pieces;
    const double* sums = q.sums + b * q.pieces * 16;
    int32_t* out = a.idx + b * a.S;
    float* logp = a.logp ? a.logp + b * a.S : nullptr;
    const RowSettings set(a, b);
    if (set.bad() && a.flag && tid == 0) atomicOr(a.flag, kErrSettings);
    float M = -INFINITY;
    for (int i = tid; i < q.pieces; i += 256) M = fmaxf(M, best[i]);
    M = block_reduce<4>(M, fbuf, OpMax());
    if (set.bad() || M == -INFINITY) {               // nothing to draw from
        for (int s = tid; s < a.S; s += 256) {
            out[s] = -1;
            if (logp) logp[s] = __builtin_nanf("");
        }
        return;
    }
    if (set.temperature == 0.f) {                    // the first of the best
        if (tid == 0) first = ~0u;
        __syncthreads();
        for (int i = tid; i < q.pieces; i += 256)
            if (best[i] == M) {
                atomicMin(&first, (uint32_t)i);
                break;
            }
        __syncthreads();
        const int64_t i0 = (int64_t)first * kPiece;
        __syncthreads();
        if (tid == 0) first = ~0u;
        __syncthreads();
        for (int64_t i = i0 + tid; i < min(N, i0 + kPiece); i += 256)
            if (row_value(row[i]) == M) {
                atomicMin(&first, (uint32_t)i);
                break;
            }
        __syncthreads();
        for (int s = tid; s < a.S; s += 256) {
            out[s] = (int32_t)first;
            if (logp) logp[s] = 0.f;
        }
        return;
    }
    const RowWeight wt{M, set.c()};
    // running sums over the pieces: a thread's share of them, then the threads'
    const int per = (q.pieces + 255) / 256;
    double sum = 0.0, total;
    for (int j = 0; j < per; ++j) {
        const int i = tid * per + j;
        if (i < q.pieces) {
            double s = 0.0;
#pragma unroll
            for (int e = 0; e < 16; ++e) s += sums[(int64_t)i * 16 + e];
            sum += s * wt(best[i]);
            run[i] = sum;
        }
    }
    const double before = block_scan<4>(sum, dbuf, &total) - sum;
    for (int j = 0; j < per; ++j)
        if (tid * per + j < q.pieces) run[tid * per + j] += before;
    __syncthreads();
    total = run[q.pieces - 1];
    for (int s = tid / kRun; s < a.S; s += 256 / kRun) {
        const double target = draw_share(a.u[b * a.S + s]) * total;
        int piece = search16(run, q.pieces, target);
        if (piece == q.pieces) {                     // (u = 1) the last one that holds something
            piece = q.pieces - 1;
            while (piece > 0 && run[piece - 1] == total) --piece;
        }
        const float top = best[piece];
        const double scale = wt(top);
        double rest = (target - (piece ? run[piece - 1] : 0.0)) / scale;
        // its chunks
        const double mine = sums[(int64_t)piece * 16 + lane];
        const double incl = scan16(mine);
        const uint32_t some = ballot16(mine > 0.0), over = ballot16(mine > 0.0 && incl > rest);
        const int c = over ? __builtin_ctz(over) : 31 - __builtin_clz(some | 1u);
        const double ahead = __shfl(incl - mine, c, kRun);
        rest -= ahead;
        const int64_t i0 = (int64_t)piece * kPiece + c * 64;
        const RowWeight in_piece{top, wt.c};
        double w;
        const int64_t i = pick16(row, N, i0, i0 + 64, rest, [&](float x, int64_t) { return in_piece(x); }, &w);
        if (lane == 0) {
            out[s] = (int32_t)i;
            if (logp) logp[s] = (float)log(w * scale / total);
        }
    }
}

// ---- with cuts ------------------------------------------------------------------

namespace {

constexpr int kPending = -2;                 // in a row's first index: k_sample_rows left the row to k_sample_far

// A row with nothing to draw from.
template <int THREADS>
__device__ __forceinline__ void draw_nothing(const SampleArgs& a, int64_t b)
{
    for (int s = threadIdx.x; s < a.S; s += THREADS) {
        a.idx[b * a.S + s] = -1;
        if (a.logp) a.logp[b * a.S + s] = __builtin_nanf("");
    }
}

// Draws from the entities at and behind `cut` of weight min_p and up, given
// their sums of n_chunks chunks of len scores, which become running sums.
template <int THREADS, int CHUNKS, typename T>
__device__ __forceinline__ void draw_kept(SampleLds<THREADS, CHUNKS>& L, const SampleArgs& a, int64_t b, const T* row,
                                          const RowWeight& wt, uint64_t cut, double min_p, int n_chunks, int64_t len)
{
    constexpr int per = (CHUNKS + THREADS - 1) / THREADS;
    const int tid = threadIdx.x;
    const int64_t N = a.N;
    __syncthreads();
    double s[per], sum = 0.0, total;
#pragma unroll
    for (int j = 0; j < per; ++j) {
        const int c = tid * per + j;
        s[j] = c < n_chunks ? L.chunk[c] : 0.0;
        sum += s[j];
    }
    double run = block_scan<THREADS / 64>(sum, L.dbuf, &total) - sum;
#pragma unroll
    for (int j = 0; j < per; ++j) {
        run += s[j];
        if (tid * per + j < n_chunks) L.chunk[tid * per + j] = run;
    }
    __syncthreads();
    total = L.chunk[n_chunks - 1];
    for (int s = tid / kRun; s < a.S; s += THREADS / kRun) {
        const double target = draw_share(a.u[b * a.S + s]) * total;
        int c = search16(L.chunk, n_chunks, target);
        if (c == n_chunks) {                         // (u = 1) the last one that holds something
            c = n_chunks - 1;
            while (c > 0 && L.chunk[c - 1] == total) --c;
        }
        double w;
        const int64_t i = pick16(row, N, c * len, min(N, (c + 1) * len), target - (c ? L.chunk[c - 1] : 0.0),
                                 [&](float x, int64_t at) {
                                     if (!(x > -INFINITY) || ranking(x, (uint32_t)at) < cut) return 0.0;
                                     const double v = wt(x);
                                     return v >= min_p ? v : 0.0;
                                 },
                                 &w);
        if ((tid & (kRun - 1)) == 0) {
            a.idx[b * a.S + s] = (int32_t)i;
            if (a.logp) a.logp[b * a.S + s] = (float)log(w / total);
        }
    }
}

}  // namespace

// One workgroup per row. NV > 0: the row's scores in registers, NV vectors of
// four a thread, element (j THREADS + thread) 4 + e; NV = 0: read again in each
// pass.
template <typename T, int THREADS, int NV, int CHUNKS>
__global__ __launch_bounds__(THREADS) void k_sample_rows(SampleArgs a)
{
    constexpr int SW = THREADS / 64;
    __shared__ SampleLds<THREADS, CHUNKS> L;
    const int tid = threadIdx.x;
    const int64_t b = blockIdx.x;
    const int64_t N = a.N;
    const T* row = reinterpret_cast<const T*>(a.scores) + b * a.ld;
    const RowSettings set(a, b);
    if (set.bad() && a.flag && tid == 0) atomicOr(a.flag, kErrSettings);

    // (held[e][j]: the passes loop over j, a uniform register index; unrolled,
    // they would not fit the instruction cache)
    typedef float Held __attribute__((ext_vector_type(NV > 0 ? NV : 1)));
    Held held[4];
    if constexpr (NV > 0) {
        if (N >= 4) {
            Four<T> f[NV];
#pragma unroll
            for (int j = 0; j < NV; ++j) f[j].load(row, (int64_t)(j * THREADS + tid) * 4, N);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float x[4];
                f[j].get(x);
                const bool past = (int64_t)(j * THREADS + tid) * 4 + 4 > N;
#pragma unroll
                for (int e = 0; e < 4; ++e) held[e][j] = past ? -INFINITY : x[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) held[e] = -INFINITY;
        }
        // the last vector, where it is not whole
        if (N % 4 && tid == (int)(N / 4) % THREADS) {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < (int)(N % 4)) held[e][(int)(N / 4) / THREADS] = row_value(row[N / 4 * 4 + e]);
        }
    }
    // f(first element, four scores), the same number of times in every thread
    auto each = [&](auto f) {
        if constexpr (NV > 0) {
#pragma unroll 1
            for (int j = 0; j < NV; ++j) {
                const float x[4] = {held[0][j], held[1][j], held[2][j], held[3][j]};
                f((int64_t)(j * THREADS + tid) * 4, x);
            }
        } else {
            // four vectors ahead
            float x[4][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) load4(row, (int64_t)(j * THREADS + tid) * 4, N, x[j]);
#pragma unroll 1
            for (int64_t i0 = 0; i0 < N; i0 += 4 * THREADS) {
                f(i0 + tid * 4, x[0]);
#pragma unroll
                for (int j = 0; j < 3; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[j][e] = x[j + 1][e];
                load4(row, i0 + (int64_t)(4 * THREADS + tid) * 4, N, x[3]);
            }
        }
    };
    float mine = -INFINITY;
    if constexpr (NV > 0) {
#pragma unroll
        for (int j = 0; j < NV; ++j) mine = fmaxf(mine, fmaxf(fmaxf(held[0][j], held[1][j]), fmaxf(held[2][j], held[3][j])));
    } else {
        each([&](int64_t, const float (&x)[4]) { mine = fmaxf(mine, fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]))); });
    }
    const float M = block_reduce<SW>(mine, L.fbuf, OpMax());
    if (set.bad() || M == -INFINITY) {
        draw_nothing<THREADS>(a, b);
        return;
    }
    if (set.temperature == 0.f || set.top_k == 1) {  // the first in ranking order
        if (tid == 0) L.n = ~0u;
        __syncthreads();
        uint32_t first = ~0u;
        each([&](int64_t i, const float (&x)[4]) {
#pragma unroll
            for (int e = 3; e >= 0; --e)
                if (x[e] == M) first = min(first, (uint32_t)(i + e));
        });
        if (first != ~0u) atomicMin(&L.n, first);
        __syncthreads();
        for (int s = tid; s < a.S; s += THREADS) {
            a.idx[b * a.S + s] = (int32_t)L.n;
            if (a.logp) a.logp[b * a.S + s] = 0.f;
        }
        return;
    }
    const RowWeight wt{M, set.c()};
    const double min_p = (double)set.min_p;
    uint64_t cut = 0;                                // what is kept: composites from here on

    // Histogram of the distances from M over `range`, of what is kept so far.
    float inv = 0.f, step = 0.f;
    auto bin_of = [&](float x) {
        const float v = (M - x) * inv;
        return v < (float)(kBins - 1) ? (int)v : kBins - 1;
    };
    auto histogram = [&](float range) {
        step = range / (float)(kBins - 1);
        inv = 1.0f / step;
        for (int i = tid; i < kBins; i += THREADS) L.h.count[i] = 0;
        __syncthreads();
        each([&](int64_t i, const float (&x)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (x[e] > -INFINITY && (!cut || ranking(x[e], (uint32_t)(i + e)) >= cut))
                    atomicAdd(&L.h.count[bin_of(x[e])], 1u);
        });
        __syncthreads();
    };
    constexpr float kNormal = 1.1754944e-38f * kBins;   // ranges whose steps have an inverse
    auto leave = [&]() {
        if (tid == 0) a.idx[b * a.S] = kPending;
    };

    if (set.top_k > 0 && set.top_k < N) {
        // the k-th score is at least the smallest of the threads' largest ones
        // where k threads have one, and the smallest score always
        float low = -INFINITY;
        if (set.top_k <= THREADS && N >= 4 * THREADS) {
            __syncthreads();
            low = -block_reduce<SW>(-mine, L.fbuf, OpMax());
        }
        if (low == -INFINITY) {
            low = M;
            each([&](int64_t, const float (&x)[4]) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (x[e] > -INFINITY) low = fminf(low, x[e]);
            });
            __syncthreads();
            low = -block_reduce<SW>(-low, L.fbuf, OpMax());
        }
        const CutGoal goal{false, (uint32_t)set.top_k, 0.0};
        const float range = (M - low) * 1.0001f;
        if (!(range > kNormal && range < INFINITY)) return leave();
        histogram(range);
        uint32_t count = 0;
        double none = 0.0;
        find_bin(L, goal, [](int) { return 0.0; }, &count, &none);
        const int bin = L.bin;
        const uint32_t in_bin = L.h.count[bin];
        if (in_bin > (uint32_t)kSort || goal.count > count + in_bin) return leave();
        if (tid == 0) L.n = 0;
        __syncthreads();
        each([&](int64_t i, const float (&x)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (x[e] > -INFINITY && bin_of(x[e]) == bin)
                    L.s.c[atomicAdd(&L.n, 1u)] = ranking(x[e], (uint32_t)(i + e));
        });
        __syncthreads();
        sort_list(L, (int)in_bin);
        cut = L.s.c[goal.count - count - 1];
        __syncthreads();
    }

    // the bins that top-p's cut lies in, by the counts
    const bool by_mass = set.top_p < 1.f;
    int from = kBins, to = kBins;
    if (by_mass) {
        // entries further off than this hold less than a 1,000th of 1 - p together
        const float range = (logf((float)N) - logf(1.f - set.top_p) + 8.f) * set.temperature;
        if (!(M < INFINITY && range > kNormal && range < INFINITY)) return leave();
        histogram(range);
        constexpr int per = kBins / THREADS;
        double m[per], sum = 0.0, all;
        uint32_t c[per];
#pragma unroll
        for (int j = 0; j < per; ++j) {
            c[j] = L.h.count[tid * per + j];
            m[j] = c[j] ? (double)c[j] * pow2d(-((double)(tid * per + j) + 0.5) * (double)step * wt.c) : 0.0;
            sum += m[j];
        }
        double run = block_scan<SW>(sum, L.dbuf, &all) - sum;
        const double margin = fmin(1e-3, 0.5 - 0.5 * (double)set.top_p);
        if (tid == 0) {
            L.bin = kBins;
            L.last = kBins;
            L.n = 0;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < per; ++j) {
            run += m[j];
            if (c[j] && run >= ((double)set.top_p - margin) * all) atomicMin(&L.bin, tid * per + j);
            if (c[j] && run >= ((double)set.top_p + margin) * all) atomicMin(&L.last, tid * per + j);
        }
        for (int i = tid; i < CHUNKS; i += THREADS) L.s.extra[i] = 0ull;
        __syncthreads();
        from = L.bin;
        to = L.last;
    }

    // One pass in doubles: sums in index order, the total, and for top-p what
    // lies before the bins and the list of what lies in them.
    int64_t len = 64;
    while ((N + len - 1) / len > CHUNKS) len <<= 1;
    const int n_chunks = (int)((N + len - 1) / len);
    double z = 0.0, above = 0.0;
    auto four = [&](int64_t i, const float (&x)[4]) {
        double sum = 0.0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            double w = x[e] > -INFINITY ? wt(x[e]) : 0.0;
            if (cut) w = ranking(x[e], (uint32_t)(i + e)) >= cut ? w : 0.0;
            const double keep = w >= min_p ? w : 0.0;
            if (by_mass) {
                const int bin = bin_of(x[e]);
                z += w;
                above += bin < from ? w : 0.0;
                sum += bin < from ? keep : 0.0;
                if (bin >= from && bin <= to && w > 0.0) {
                    const uint32_t at = atomicAdd(&L.n, 1u);
                    if (at < (uint32_t)kSort) L.s.c[at] = ranking(x[e], (uint32_t)(i + e));
                }
            } else {
                sum += keep;
            }
        }
        return sum;
    };
    if (NV > 0 || len == 64) {
        each([&](int64_t i, const float (&x)[4]) {
            const double s = sum16(four(i, x));
            if ((tid & (kRun - 1)) == 0 && i < N) L.chunk[i / 64] = s;
        });
    } else {
        for (int c = tid / 64; c < n_chunks; c += SW) {
            double s = 0.0;
            for (int64_t i = c * len + (tid & 63) * 4; i < (c + 1) * len; i += 256) {
                float x[4];
                load4(row, i, N, x);
                s += four(i, x);
            }
            s = wave_reduce(s, OpSum());
            if ((tid & 63) == 0) L.chunk[c] = s;
        }
    }
    if (by_mass) {
        z = block_reduce<SW>(z, L.dbuf, OpSum());
        above = block_reduce<SW>(above, L.dbuf2, OpSum());
        const CutGoal goal{true, 0u, (double)set.top_p * z};
        const uint32_t n = L.n;
        __syncthreads();
        if (n == 0 || n > (uint32_t)kSort || !(above < goal.mass)) return leave();
        const uint32_t at = sorted_cut(L, (int)n, wt, goal, 0u, above);
        if (at == n) return leave();
        cut = L.s.c[at];
        // what is kept of the list goes to its chunks, in fixed point relative
        // to its largest weight
        const double top = wt(ranking_score(L.s.c[0])), unit = 0x1p50 / top;
        for (int i = tid; i <= (int)at; i += THREADS) {
            const uint64_t c = L.s.c[i];
            const double w = wt(ranking_score(c));
            if (w >= min_p) atomicAdd(&L.s.extra[(uint32_t)~c / len], (unsigned long long)(w * unit));
        }
        __syncthreads();
        for (int i = tid; i < n_chunks; i += THREADS)
            if (L.s.extra[i]) L.chunk[i] += (double)L.s.extra[i] * (top * 0x1p-50);
    }
    draw_kept(L, a, b, row, wt, cut, min_p, n_chunks, len);
}

// The rows that k_sample_rows left: infinite scores, more equal or nearly
// equal scores around a cut than it sorts, a cut it did not find. One
// workgroup per row, which is read once for each step of the search.
template <typename T>
__global__ __launch_bounds__(1024) void k_sample_far(SampleArgs a)
{
    constexpr int THREADS = 1024, SW = THREADS / 64, CHUNKS = 4096;
    __shared__ SampleLds<THREADS, CHUNKS> L;
    const int tid = threadIdx.x;
    const int64_t b = blockIdx.x, N = a.N;
    if (a.idx[b * a.S] != kPending) return;
    const T* row = reinterpret_cast<const T*>(a.scores) + b * a.ld;
    const RowSettings set(a, b);
    float M = -INFINITY, low = INFINITY;
    for (int64_t i = tid; i < N; i += THREADS) {
        const float x = row_value(row[i]);
        M = fmaxf(M, x);
        if (x > -INFINITY) low = fminf(low, x);
    }
    M = block_reduce<SW>(M, L.fbuf, OpMax());
    __syncthreads();
    low = -block_reduce<SW>(-low, L.fbuf, OpMax());
    __syncthreads();
    const RowWeight wt{M, set.c()};
    uint64_t cut = 0;
    // (both cuts in one loop: the search is long code)
    for (int turn = 0; turn < 2; ++turn) {
        CutGoal goal{turn == 1, (uint32_t)set.top_k, 0.0};
        float range = M - low;
        if (turn == 0 ? !(set.top_k > 0 && set.top_k < N) : !(set.top_p < 1.f)) continue;
        if (turn == 1) {
            // the weight that p is a share of
            double sum = 0.0;
            for (int64_t i = tid; i < N; i += THREADS) {
                const float x = row_value(row[i]);
                if (x > -INFINITY && ranking(x, (uint32_t)i) >= cut) sum += wt(x);
            }
            sum = block_reduce<SW>(sum, L.dbuf, OpSum());
            __syncthreads();
            goal.mass = (double)set.top_p * sum;
            // entries with less than (1 - p) / N of the largest weight lie behind the cut
            range = fminf((logf((float)N) - logf(1.f - set.top_p) + 1.f) * set.temperature, 1e38f);
        }
        cut = max(cut, find_cut(L, row, N, wt, goal, cut, range));
    }
    int64_t len = 64;
    while ((N + len - 1) / len > CHUNKS) len <<= 1;
    const int n_chunks = (int)((N + len - 1) / len);
    __syncthreads();
    for (int c = tid / 64; c < n_chunks; c += SW) {
        double sum = 0.0;
        const int64_t end = min(N, (c + 1) * len);
        for (int64_t i = c * len + (tid & 63); i < end; i += 64) {
            const float x = row_value(row[i]);
            const double w = x > -INFINITY && ranking(x, (uint32_t)i) >= cut ? wt(x) : 0.0;
            sum += w >= (double)set.min_p ? w : 0.0;
        }
        sum = wave_reduce(sum, OpSum());
        if ((tid & 63) == 0) L.chunk[c] = sum;
    }
    draw_kept(L, a, b, row, wt, cut, (double)set.min_p, n_chunks, len);
}

namespace {

int64_t pieces_of(int64_t N) { return (N + kPiece - 1) / kPiece; }

template <typename T>
void launch(const SampleArgs& a, hipStream_t s)
{
    const bool cuts = a.top_k_rows || a.top_p_rows || a.min_p_rows || (a.top_k > 0 && a.top_k < a.N) || a.top_p < 1.f ||
                      a.min_p > 0.f;
    if (!cuts && pieces_of(a.N) <= kMaxPieces) {
        const int pieces = (int)pieces_of(a.N);
        double* sums = reinterpret_cast<double*>(a.ws);
        const SamplePieces q{sums, reinterpret_cast<float*>(sums + (int64_t)a.batch * pieces * 16), pieces};
        hipLaunchKernelGGL(k_sample_sums<T>, dim3((uint32_t)(((int64_t)a.batch * pieces + 3) / 4)), dim3(256), 0, s, a, q);
        hipLaunchKernelGGL(k_sample_draw<T>, dim3(a.batch), dim3(256), pieces * sizeof(double), s, a, q);
        return;
    }
    // the row in registers where it fits; short rows four or more to a compute
    // unit, the others one or two
    auto go = [&](auto kernel, int threads) {
        hipLaunchKernelGGL(kernel, dim3(a.batch), dim3(threads), 0, s, a);
        hipLaunchKernelGGL(k_sample_far<T>, dim3(a.batch), dim3(1024), 0, s, a);
    };
    if (a.N <= 4096) go(k_sample_rows<T, 256, 4, 64>, 256);
    else if (a.N <= 16384) go(k_sample_rows<T, 1024, 4, 256>, 1024);
    else if (a.N <= 65536) go(k_sample_rows<T, 1024, 16, 1024>, 1024);
    else go(k_sample_rows<T, 1024, 0, 4096>, 1024);
}

}  // namespace

int64_t sample_workspace(int64_t batch, int64_t N)
{
    if (pieces_of(N) > kMaxPieces) return 0;
    return batch * pieces_of(N) * (int64_t)(16 * sizeof(double) + sizeof(float));
}

void launch_sample(const SampleArgs& a, hipStream_t s)
{
    if (a.dtype == KGQ_BF16) launch<uint16_t>(a, s);
    else launch<float>(a, s);
}

}  // namespace kgq
