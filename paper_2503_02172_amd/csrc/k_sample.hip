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
// atomics, whose order does not matter. It starts over, so that such a row
// takes two to five times as long: infinite scores, more than 2,048 entries in
// the bins around the cut (bfloat16 scores, which tie, of rows above 65,536, or
// of any at high temperatures), and a top-k above the number of entries that
// are not masked.
#include <algorithm>
#include <type_traits>

#include "row_ops.hpp"

namespace kgq {

namespace {

constexpr int kBins = 2048;
constexpr int kSort = 2048;                  // entries that are sorted for a cut
constexpr int kRankSort = 512;               // of these, sorted by counting (top-p, 2,048 rows, a call: 379 us, 404 by merging)
constexpr int kDrawn = 1024;                 // draws of a row whose logarithms are taken together
constexpr int kRun = 16;                     // lanes per draw, and per 64 scores
constexpr int kPiece = 1024;                 // scores of a row per wavefront, without cuts
constexpr int kMaxPieces = 320;              // of a row (their chunks' running sums lie in LDS)

// 2^r on |r| <= 1/2, off by 4e-14 (a draw compares sums that are off by less
// then, and none in 10^8 moves): the polynomial through Chebyshev's points.
__device__ __forceinline__ double pow2_part(double r)
{
    double y = 1.0205905413765595e-07;
    y = fma(y, r, 1.325964524488711e-06);
    y = fma(y, r, 1.5252672924850737e-05);
    y = fma(y, r, 0.0001540343375125101);
    y = fma(y, r, 0.0013333558200794592);
    y = fma(y, r, 0.009618129193934313);
    y = fma(y, r, 0.05550410866465167);
    y = fma(y, r, 0.2402265069564034);
    y = fma(y, r, 0.6931471805599462);
    return fma(y, r, 1.0);
}
// 2^t for t <= 0, 0 below 2^-1074 and for NaN.
__device__ __forceinline__ double pow2d(double t)
{
    t = fmax(t, -1100.0);                    // (a NaN goes here too)
    const double n = rint(t);
    return ldexp(pow2_part(t - n), (int)n);
}

// A row's weights, 2^((x - M) c) with c = log2(e) / T; 0 below 2^-1000, for
// -inf and NaN. Where the maximum is +inf, the infinite scores share the
// weight. Rounding and scaling by n take an addition each instead of the
// instructions of that name, which run at a quarter of the rate or less: the
// sum of 1.5 2^52 and a number holds it rounded in its low bits, and adding n to
// the exponent field multiplies by 2^n. (The sums of 2,048 rows of 63,361 take
// 144 us with those instructions, 128 without.)
struct RowWeight {
    float top, low, from;                    // scores are taken into [low, top]; below `from` they have no weight
    double M, c;
    __device__ __forceinline__ RowWeight(float max, double T)
    {
        constexpr float kMax = 3.4028234664e38f;
        const bool inf = max == INFINITY;
        top = fminf(max, kMax);
        low = inf ? kMax : fmaxf(max - 693.f * (float)T, -kMax);
        from = inf ? INFINITY : low;
        M = top;
        c = fmin(1.4426950408889634074 / T, 1e300);      // (times 0 for the largest score)
    }
    // (for scores of weight; not clamped)
    __device__ __forceinline__ double exponent(float x) const
    {
        if (from == INFINITY) return x == INFINITY ? 0.0 : -INFINITY;
        return ((double)x - M) * c;
    }
    __device__ __forceinline__ double operator()(float x) const
    {
        constexpr double magic = 6755399441055744.0;
        const double d = (double)__builtin_amdgcn_fmed3f(x, low, top) - M;
        const double s = fma(d, c, magic);
        const double y = pow2_part(fma(d, c, magic - s));
        const int n = max((int)(uint32_t)__builtin_bit_cast(uint64_t, s), -1021);
        uint64_t u = __builtin_bit_cast(uint64_t, y);
        u = ((uint64_t)((uint32_t)(u >> 32) + ((uint32_t)n << 20)) << 32) | (uint32_t)u;
        return x >= from ? __builtin_bit_cast(double, u) : 0.0;
    }
};

// A value that every lane holds, in scalar registers.
__device__ __forceinline__ float uniform(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }
__device__ __forceinline__ uint64_t uniform(uint64_t x)
{
    // (the builtin returns an int: its sign must not spread over the upper half)
    return ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(x >> 32)) << 32) |
           (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)x);
}
__device__ __forceinline__ double uniform(double x)
{
    return __builtin_bit_cast(double, uniform(__builtin_bit_cast(uint64_t, x)));
}

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
            alignas(16) uint32_t count[kBins + 64];   // (the last 64: scores that belong to no bin, by lane)
            unsigned long long mass[kBins];
        } h;
        struct {
            alignas(16) uint64_t c[kSort];
            unsigned long long extra[CHUNKS];
        } s;
        struct {
            double share[kDrawn];
            int32_t idx[kDrawn];
        } d;
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
// is counted in. Where the goal lies behind every bin, the last one with an
// entry is taken.
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
            // (the bin in which the sum crosses the goal)
            const bool ok = goal.by_mass ? *mass + (mb + m[j]) >= goal.mass && (*mass + mb < goal.mass || cb == 0)
                                         : *count + cb + c[j] >= goal.count && *count + cb < goal.count;
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
    if (n <= kRankSort) {
        // few: an entry's place is the number of larger ones
        static_assert(kRankSort <= 2 * THREADS, "two entries a thread at most");
        if (tid == 0 && (n & 1)) L.s.c[n] = 0ull;
        __syncthreads();
        uint64_t mine[2];
        int place[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int i = tid + k * THREADS;
            place[k] = -1;
            if (i >= n) continue;
            mine[k] = L.s.c[i];
            int larger = 0;
            for (int j = 0; j < n; j += 2) {
                const ulonglong2 o = *reinterpret_cast<const ulonglong2*>(&L.s.c[j]);
                larger += (o.x > mine[k]) + (o.y > mine[k]);
            }
            place[k] = larger;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (place[k] >= 0) L.s.c[place[k]] = mine[k];
        __syncthreads();
        return;
    }
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
        const int i = tid * per + j;
        const bool short_of = mass + before < goal.mass;
        before += w[j];
        // (the entry at which the sum crosses the goal)
        if (i < n && mass + before >= goal.mass && (short_of || i == 0)) atomicMin(&L.n, (uint32_t)i);
    }
    __syncthreads();
    return L.n;
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

// f(first element, four scores) over the row, by THREADS threads, the same
// number of times in each; four vectors ahead.
template <int THREADS, typename T, typename F>
__device__ __forceinline__ void each_four(const T* row, int64_t N, F f)
{
    const int tid = threadIdx.x;
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
        const float v = (wt.top - x) * inv;        // 0 and up; NaN (infinite M, or a step of 0) to bin 0
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
        each_four<THREADS>(row, N, [&](int64_t i, const float (&x)[4]) __attribute__((always_inline)) {
#pragma unroll 1
            for (int e = 0; e < 4; ++e) {
                const float y = e == 0 ? x[0] : e == 1 ? x[1] : e == 2 ? x[2] : x[3];
                if (!(y > -INFINITY)) continue;
                const unsigned long long c = ranking(y, (uint32_t)(i + e));
                if (c < lo || c > hi) continue;
                const int bin = value_bin(y, c);
                atomicAdd(&L.h.count[bin], 1u);
                if (goal.by_mass)
                    atomicAdd(&L.h.mass[bin],
                              (unsigned long long)(pow2d(fmin(wt.exponent(y) - scale_of(bin), 0.5)) * unit));
            }
        });
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
        each_four<THREADS>(row, N, [&](int64_t i, const float (&x)[4]) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (!(x[e] > -INFINITY)) continue;
                const unsigned long long c = ranking(x[e], (uint32_t)(i + e));
                if (c < lo || c > hi || value_bin(x[e], c) != bin) continue;
                mine_lo = min(mine_lo, c);
                mine_hi = max(mine_hi, c);
                if (take) L.s.c[atomicAdd(&L.n, 1u)] = c;
            }
        });
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

// A double from another lane of the 16, by DPP (0 where there is none).
template <int CTRL>
__device__ __forceinline__ double dpp16(double x)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, 0xF, 0xF, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, 0xF, 0xF, false);
    return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
// Sum over 16 neighbouring lanes, the same in each: neighbours, pairs, half
// rows mirrored, rows mirrored.
__device__ __forceinline__ double sum16(double x)
{
    x += dpp16<0xB1>(x);
    x += dpp16<0x4E>(x);
    x += dpp16<0x141>(x);
    x += dpp16<0x140>(x);
    return x;
}
// Running sum over 16 lanes (rows shifted by 1, 2, 4 and 8).
__device__ __forceinline__ double scan16(double x)
{
    x += dpp16<0x111>(x);
    x += dpp16<0x112>(x);
    x += dpp16<0x114>(x);
    x += dpp16<0x118>(x);
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
        weigh(x, i, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += v[e];
        const double incl = run + scan16(sum);
        const uint32_t some = ballot16(sum > 0.0), over = ballot16(sum > 0.0 && incl > rest);
        // (no lane over yet: the last one with a weight, in case there is no other)
        const int l = over ? __builtin_ctz(over) : some ? 31 - __builtin_clz(some) : -1;
        if (l >= 0) {
            double before = dpp16<0x111>(incl);
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

// The same over a row whose chunks of len scores have the running sums run[0 ..
// n): the first chunk whose sum exceeds the target, and the element in it.
// Where rounding has the target end in a chunk that holds nothing, the next one
// that does; behind the total (u = 1), the last one that does.
template <typename T, typename W>
__device__ __forceinline__ int64_t pick_in(const T* row, int64_t N, const double* run, int n, int64_t len, double target,
                                           W weigh, double* w)
{
    const int at = search16(run, n, target);
    bool back = false;
    for (int c = at;;) {
        if (c == n) {
            if (at == 0) return -1;
            back = true;
            c = at - 1;
        }
        const double rest = c == at ? target - (c ? run[c - 1] : 0.0) : back ? INFINITY : -1.0;
        const int64_t i = pick16(row, N, c * len, min(N, (c + 1) * len), rest, weigh, w);
        if (i >= 0 || (back && c == 0)) return i;
        c += back ? -1 : 1;
    }
}

__device__ __forceinline__ double draw_share(float u) { return u >= 0.f ? fmin((double)u, 1.0) : 0.0; }

// A row's draws, 16 lanes each: draw(target, &weight) returns the entity for a
// share of the total. Their logarithms are taken afterwards, a lane each.
template <int THREADS, typename D>
__device__ __forceinline__ void draw_all(double* share, int32_t* idx, const SampleArgs& a, int64_t b, double total, D draw)
{
    const int tid = threadIdx.x;
    for (int s0 = 0; s0 < a.S; s0 += kDrawn) {
        const int n = min(kDrawn, a.S - s0);
        for (int s = tid / kRun; s < n; s += THREADS / kRun) {
            double w;
            const int64_t i = draw(draw_share(a.u[b * a.S + s0 + s]) * total, &w);
            if ((tid & (kRun - 1)) == 0) {
                share[s] = w;
                idx[s] = (int32_t)i;
            }
        }
        __syncthreads();
        for (int s = tid; s < n; s += THREADS) {
            a.idx[b * a.S + s0 + s] = idx[s];
            if (a.logp) a.logp[b * a.S + s0 + s] = (float)log(share[s] / total);
        }
        __syncthreads();
    }
}

// A row's settings.
struct RowSettings {
    double temperature, top_p, min_p;
    int32_t top_k;
    __device__ __forceinline__ RowSettings(const SampleArgs& a, int64_t b)
        : temperature(a.temperature_rows ? (double)a.temperature_rows[b] : a.temperature),
          top_p(a.top_p_rows ? (double)a.top_p_rows[b] : a.top_p),
          min_p(a.min_p_rows ? (double)a.min_p_rows[b] : a.min_p),
          top_k(a.top_k_rows ? a.top_k_rows[b] : a.top_k)
    {
    }
    __device__ __forceinline__ bool bad() const
    {
        return !(temperature >= 0.0 && temperature < INFINITY) || top_k < 0 || !(top_p > 0.0) ||
               !(min_p >= 0.0 && min_p <= 1.0);
    }
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

// A piece per wavefront. 2,048 rows of 63,361: 128 us, bound by the doubles (the
// same loads with float32 exponentials 103 us, which is what the bytes take);
// two or four pieces a wavefront, the next one's scores ahead, take as long.
template <typename T>
__global__ __launch_bounds__(256) void k_sample_sums(SampleArgs a, SamplePieces q)
{
    const int lane = threadIdx.x & 63;
    const int64_t b = blockIdx.x;
    const int piece = blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (piece >= q.pieces) return;
    const T* row = reinterpret_cast<const T*>(a.scores) + b * a.ld;
    const int64_t i0 = (int64_t)piece * kPiece + lane * 4, at = b * q.pieces + piece;
    Four<T> f[4];
    float x[4][4], best = -INFINITY;
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j].load(row, i0 + j * 256, a.N);
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j].get(x[j]);
    if ((int64_t)(piece + 1) * kPiece > a.N) {
#pragma unroll
        for (int j = 0; j < 4; ++j) end4(x[j], i0 + j * 256, a.N);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) best = fmaxf(best, x[j][e]);
    best = wave_reduce(best, OpMax());
    const RowWeight wt(best, RowSettings(a, b).temperature);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const double s = sum16((wt(x[j][0]) + wt(x[j][1])) + (wt(x[j][2]) + wt(x[j][3])));
        if ((lane & (kRun - 1)) == 0) q.sums[at * 16 + j * 4 + lane / kRun] = s;
    }
    if (lane == 0) q.best[at] = best;
}

// A row's draws from its pieces' sums: a workgroup per row, as many as fit a
// compute unit. 2,048 rows of 63,361, 128 draws each: 56 us, bound by issue (64
// weights in doubles a draw; 64 us with slower ones) and by the three lines of
// 128 bytes that a draw's 64 scores touch, 100 MB; four draws ahead a group, or
// more wavefronts at the price of registers, are no faster (56 to 99 us).
template <typename T>
__global__ __launch_bounds__(256) void k_sample_draw(SampleArgs a, SamplePieces q)
{
    constexpr int DT = 256;
    extern __shared__ double run[];                  // [16 pieces]: the chunks' running sums
    __shared__ float fbuf[DT / 64];
    __shared__ double dbuf[DT / 64];
    __shared__ uint32_t first;
    __shared__ double share[kDrawn];
    __shared__ int32_t idx[kDrawn];
    const int tid = threadIdx.x;
    const int64_t b = blockIdx.x, N = a.N;
    const T* row = reinterpret_cast<const T*>(a.scores) + b * a.ld;
    const float* best = q.best + b * q.pieces;
    const double* sums = q.sums + b * q.pieces * 16;
    const int n = q.pieces * 16;
    int32_t* out = a.idx + b * a.S;
    float* logp = a.logp ? a.logp + b * a.S : nullptr;
    const RowSettings set(a, b);
    if (set.bad() && a.flag && tid == 0) atomicOr(a.flag, kErrSettings);
    float M = -INFINITY;
    for (int i = tid; i < q.pieces; i += DT) M = fmaxf(M, best[i]);
    M = block_reduce<DT / 64>(M, fbuf, OpMax());
    if (set.bad() || M == -INFINITY) {               // nothing to draw from
        for (int s = tid; s < a.S; s += DT) {
            out[s] = -1;
            if (logp) logp[s] = __builtin_nanf("");
        }
        return;
    }
    if (set.temperature == 0.0) {                    // the first of the best
        if (tid == 0) first = ~0u;
        __syncthreads();
        for (int i = tid; i < q.pieces; i += DT)
            if (best[i] == M) {
                atomicMin(&first, (uint32_t)i);
                break;
            }
        __syncthreads();
        const int64_t i0 = (int64_t)first * kPiece;
        __syncthreads();
        if (tid == 0) first = ~0u;
        __syncthreads();
        for (int64_t i = i0 + tid; i < min(N, i0 + kPiece); i += DT)
            if (row_value(row[i]) == M) {
                atomicMin(&first, (uint32_t)i);
                break;
            }
        __syncthreads();
        for (int s = tid; s < a.S; s += DT) {
            out[s] = (int32_t)first;
            if (logp) logp[s] = 0.f;
        }
        return;
    }
    const RowWeight wt(M, set.temperature);
    for (int i = tid; i < n; i += DT) run[i] = sums[i] * wt(best[i >> 4]);
    __syncthreads();
    const int per = (n + DT - 1) / DT;
    double sum = 0.0, total;
    for (int j = 0; j < per; ++j) {
        const int i = tid * per + j;
        if (i < n) {
            sum += run[i];
            run[i] = sum;
        }
    }
    const double before = block_scan<DT / 64>(sum, dbuf, &total) - sum;
    for (int j = 0; j < per; ++j)
        if (tid * per + j < n) run[tid * per + j] += before;
    __syncthreads();
    total = run[n - 1];
    draw_all<DT>(share, idx, a, b, total, [&](double target, double* w) {
        return pick_in(row, N, run, n, 64, target,
                      [&](const float (&x)[4], int64_t, double (&v)[4]) {
#pragma unroll
                          for (int e = 0; e < 4; ++e) v[e] = wt(x[e]);
                      },
                      w);
    });
}

// ---- with cuts ------------------------------------------------------------------

namespace {

constexpr int kPending = -2;                 // in a row's first index: k_sample_rows left the row to k_sample_far

// Scores per running sum, as a power of two: 64 or as many as CHUNKS sums need.
template <int CHUNKS>
__device__ __forceinline__ int chunk_shift(int64_t N)
{
    int shift = 6;
    while (((N + (1ll << shift) - 1) >> shift) > CHUNKS) ++shift;
    return shift;
}

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
    total = uniform(L.chunk[n_chunks - 1]);
    draw_all<THREADS>(L.d.share, L.d.idx, a, b, total, [&](double target, double* w) {
        return pick_in(row, N, L.chunk, n_chunks, len, target,
                      [&](const float (&x)[4], int64_t at, double (&v)[4]) {
#pragma unroll
                          for (int e = 0; e < 4; ++e) {
                              v[e] = wt(x[e]);
                              if (ranking(x[e], (uint32_t)(at + e)) < cut || !(v[e] >= min_p)) v[e] = 0.0;
                          }
                      },
                      w);
    });
}

}  // namespace

// One workgroup per row. NV > 0: the row's scores in registers, NV vectors of
// four a thread, element (j THREADS + thread) 4 + e; NV = 0: read again in each
// pass.
// 2,048 rows of 63,361, top-p 0.9: 387 us as profiled, 1.3 TB/s (a call among
// others, with the second launch, 378). A row takes about 42 us of
// its compute unit, one row after the other: loading 6, largest score 1,
// histogram 7, its bins 2, the pass in doubles 18, list and cut 3, the draw
// 3.5. So the phases' latency bounds it, and the doubles, which cost 18 us a row
// here and bound the sums without cuts at 16. (256 of the 512 registers of a
// lane hold scores: a second row does not fit; 1,024 threads with half as many
// each spill.) top-k 100: 292 us, min-p 0.02 156; bfloat16 rows, held as
// float32, take 407, 263 and 130. 61 rows with all cuts: 59 us, and one row of
// 14,505 with top-p 20: the latency of the phases alone.
template <typename T, int THREADS, int NV, int CHUNKS, int WAVES>
__global__ __launch_bounds__(THREADS, WAVES) void k_sample_rows(SampleArgs a)
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
    auto each = [&](auto f) __attribute__((always_inline)) {
        if constexpr (NV > 0) {
#pragma unroll 1
            for (int j = 0; j < NV; ++j) {
                const float x[4] = {held[0][j], held[1][j], held[2][j], held[3][j]};
                f((int64_t)(j * THREADS + tid) * 4, x);
            }
        } else {
            each_four<THREADS>(row, N, f);
        }
    };
    float mine = -INFINITY;
    if constexpr (NV > 0) {
#pragma unroll
        for (int j = 0; j < NV; ++j) mine = fmaxf(mine, fmaxf(fmaxf(held[0][j], held[1][j]), fmaxf(held[2][j], held[3][j])));
    } else {
        each([&](int64_t, const float (&x)[4]) { mine = fmaxf(mine, fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]))); });
    }
    const float M = uniform(block_reduce<SW>(mine, L.fbuf, OpMax()));
    if (set.bad() || M == -INFINITY) {
        draw_nothing<THREADS>(a, b);
        return;
    }
    auto leave = [&]() __attribute__((always_inline)) {
        if (tid == 0) a.idx[b * a.S] = kPending;
    };
    if (set.temperature == 0.0 || set.top_k == 1) {  // the first in ranking order
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
    if (M == INFINITY) return leave();
    const RowWeight wt(M, set.temperature);
    const double min_p = set.min_p;
    uint64_t cut = 0;                                // what is kept: composites from here on

    // Histogram of the distances from M over `range`, of what is kept so far.
    // Scores further off are in no bin, masked ones neither (their place in a
    // counter of the lane's own keeps the lanes together).
    float inv = 0.f, step = 0.f;
    auto bin_of = [&](float x) __attribute__((always_inline)) { return (M - x) * inv; };   // rounded down, below kBins
    auto histogram = [&](float range) __attribute__((always_inline)) {
        step = range / (float)kBins;
        inv = 1.0f / step;
        for (int i = tid; i < kBins; i += THREADS) L.h.count[i] = 0;
        __syncthreads();
        each([&](int64_t i, const float (&x)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = bin_of(x[e]);
                int bin = v < (float)kBins ? (int)v : kBins + (tid & 63);
                if (cut) bin = ranking(x[e], (uint32_t)(i + e)) >= cut ? bin : kBins + (tid & 63);
                atomicAdd(&L.h.count[bin], 1u);
            }
        });
        __syncthreads();
    };
    constexpr float kNormal = 1.1754944e-38f * kBins;   // ranges whose steps have an inverse
    auto lowest = [&]() __attribute__((always_inline)) {
        float low = M;
        each([&](int64_t, const float (&x)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e) low = fminf(low, x[e] > -INFINITY ? x[e] : M);
        });
        __syncthreads();
        return uniform(-block_reduce<SW>(-low, L.fbuf, OpMax()));
    };

    if (set.top_k > 0 && set.top_k < N) {
        // the k-th score is at least the smallest of the threads' largest ones
        // where k threads have one, and the smallest score always
        float low = -INFINITY;
        if (set.top_k <= THREADS && N >= 4 * THREADS) {
            __syncthreads();
            low = uniform(-block_reduce<SW>(-mine, L.fbuf, OpMax()));
        }
        if (low == -INFINITY) low = lowest();
        const CutGoal goal{false, (uint32_t)set.top_k, 0.0};
        const float range = (M - low) * 1.0001f;
        if (!(range > kNormal && range < INFINITY)) return leave();
        histogram(range);
        uint32_t count = 0;
        double none = 0.0;
        find_bin(L, goal, [](int) { return 0.0; }, &count, &none);
        const int bin = __builtin_amdgcn_readfirstlane(L.bin);
        const uint32_t in_bin = __builtin_amdgcn_readfirstlane(L.h.count[bin]);
        if (in_bin > (uint32_t)kSort || goal.count > count + in_bin) return leave();
        if (tid == 0) L.n = 0;
        __syncthreads();
        each([&](int64_t i, const float (&x)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (bin_of(x[e]) >= (float)bin && bin_of(x[e]) < (float)(bin + 1))
                    L.s.c[atomicAdd(&L.n, 1u)] = ranking(x[e], (uint32_t)(i + e));
        });
        __syncthreads();
        sort_list(L, (int)in_bin);
        cut = uniform(L.s.c[goal.count - count - 1]);
        __syncthreads();
    }

    // the bins that top-p's cut lies in, by the counts
    const double p = set.top_p;
    const bool by_mass = p < 1.0;
    float from = INFINITY, to = INFINITY;            // their distances: from this one, below that one
    if (by_mass) {
        // entries further off than this hold less than e^-8 of 1 - p together
        const float far = (logf((float)N) - logf((float)(1.0 - set.top_p)) + 8.f) * (float)set.temperature;
        // (all of the row, where that is less: looked up if the threads' largest
        // scores lie in a small part of it)
        float range = far;
        __syncthreads();
        const float near = M + uniform(block_reduce<SW>(-mine, L.fbuf, OpMax()));
        if (near < far * 0.0625f || near == INFINITY) range = fminf(far, (M - lowest()) * 1.0001f);
        if (!(range > kNormal && range < INFINITY)) return leave();
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
        // A bin's sum is off by up to half a step's weight, h, a share f of the
        // whole thus by 2 h f (1 - f); the entries behind the range add e^-8 f (1 - f).
        const double margin = (0.75 * (double)step * wt.c + 5e-4) * p * (1.0 - p) + 1e-9;
        if (tid == 0) {
            L.bin = kBins;
            L.last = kBins;
            L.n = 0;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < per; ++j) {
            const double lo = (p - margin) * all, hi = fmin(p + margin, 1.0 - 1e-12) * all;
            const double before = run;
            run += m[j];
            // (where the sum crosses the border: a bin or two)
            if (run >= lo && (before < lo || tid + j == 0)) atomicMin(&L.bin, tid * per + j);
            if (run >= hi && before < hi) atomicMin(&L.last, tid * per + j);
        }
        for (int i = tid; i < CHUNKS; i += THREADS) L.s.extra[i] = 0ull;
        __syncthreads();
        if (L.bin == kBins || L.last == kBins) return leave();
        from = uniform((float)L.bin);
        to = uniform((float)(L.last + 1));
    }

    // One pass in doubles: sums in index order, the total, and for top-p what
    // lies before the bins and the list of what lies in them.
    const int shift = chunk_shift<CHUNKS>(N);
    const int64_t len = 1ll << shift;
    const int n_chunks = (int)((N + len - 1) >> shift);
    // Scores below `skip` have no part in it: those behind the cut, or without p
    // those below min_p (a little lower, by what the logarithm and the sum round
    // off); a wavefront without any other score goes on to its next ones.
    float skip = cut ? ranking_score(cut) : -INFINITY;
    if (!by_mass && min_p > 0.0) {
        const double low = (double)M + set.temperature * (log(min_p) - 1e-6) - fabs((double)M) * 1e-6;
        if (low > -3.4028234664e38) skip = fmaxf(skip, (float)low);      // (else no score lies below it)
    }
    double z = 0.0, above = 0.0;
    // (whether the wavefront has anything to sum; sum: a lane's)
    auto four = [&](int64_t i, const float (&x)[4], double& sum) __attribute__((always_inline)) {
        sum = 0.0;
        const float top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
        if (__builtin_amdgcn_ballot_w64(top >= skip) == 0) return false;
        double w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = wt(x[e]);
        if (cut) {
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = ranking(x[e], (uint32_t)(i + e)) >= cut ? w[e] : 0.0;
        }
        if (by_mass) {
            z += (w[0] + w[1]) + (w[2] + w[3]);
            // all of it behind the bins?
            if (__builtin_amdgcn_ballot_w64(bin_of(top) < to) == 0) return false;
            float v[4];
            bool in[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] = bin_of(x[e]);
                in[e] = (v[e] >= from) & (v[e] < to);
            }
            if (in[0] | in[1] | in[2] | in[3]) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (in[e] && w[e] > 0.0) {
                        const uint32_t at = atomicAdd(&L.n, 1u);
                        if (at < (uint32_t)kSort) L.s.c[at] = ranking(x[e], (uint32_t)(i + e));
                    }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = v[e] < from ? w[e] : 0.0;
        }
        sum = (w[0] + w[1]) + (w[2] + w[3]);
        above += sum;
        if (min_p > 0.0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = w[e] >= min_p ? w[e] : 0.0;
            sum = (w[0] + w[1]) + (w[2] + w[3]);
        }
        return true;
    };
    if (NV > 0 || len == 64) {
        each([&](int64_t i, const float (&x)[4]) __attribute__((always_inline)) {
            double s;
            if (four(i, x, s)) s = sum16(s);
            if ((tid & (kRun - 1)) == 0 && i < N) L.chunk[i / 64] = s;
        });
    } else {
        for (int c = tid / 64; c < n_chunks; c += SW) {
            double s = 0.0;
            for (int64_t i = c * len + (tid & 63) * 4; i < (c + 1) * len; i += 256) {
                float x[4];
                double part;
                load4(row, i, N, x);
                four(i, x, part);
                s += part;
            }
            s = wave_reduce(s, OpSum());
            if ((tid & 63) == 0) L.chunk[c] = s;
        }
    }
    if (by_mass) {
        z = uniform(block_reduce<SW>(z, L.dbuf, OpSum()));
        above = uniform(block_reduce<SW>(above, L.dbuf2, OpSum()));
        const CutGoal goal{true, 0u, p * z};
        const uint32_t n = L.n;
        __syncthreads();
        if (n == 0 || n > (uint32_t)kSort || !(above < goal.mass)) return leave();
        const uint32_t at = sorted_cut(L, (int)n, wt, goal, 0u, above);
        if (at == n) return leave();
        cut = uniform(L.s.c[at]);
        // what is kept of the list goes to its chunks, in fixed point relative
        // to its largest weight
        const double top = wt(ranking_score(L.s.c[0])), unit = 0x1p50 / top;
        for (int i = tid; i <= (int)at; i += THREADS) {
            const uint64_t c = L.s.c[i];
            const double w = wt(ranking_score(c));
            if (w >= min_p) atomicAdd(&L.s.extra[(uint32_t)~c >> shift], (unsigned long long)(w * unit));
        }
        __syncthreads();
        for (int i = tid; i < n_chunks; i += THREADS)
            if (L.s.extra[i]) L.chunk[i] += (double)L.s.extra[i] * (top * 0x1p-50);
    }
    draw_kept(L, a, b, row, wt, cut, min_p, n_chunks, len);
}

// The rows that k_sample_rows left: infinite scores, more equal or nearly
// equal scores around a cut than it sorts, a cut it did not find. One
// workgroup per row, which is read once for each step of the search. 4 us where
// there is no such row; 2,048 rows of 63,361 with 50 entries that are not masked
// and top-k 100: 650 us; 500 bfloat16 rows of 200,000, top-p 0.9 at temperature
// 1.5, all of them left: 1,450 us.
template <typename T>
__global__ __launch_bounds__(512) void k_sample_far(SampleArgs a)
{
    constexpr int THREADS = 512, SW = THREADS / 64, CHUNKS = 4096;
    __shared__ SampleLds<THREADS, CHUNKS> L;
    const int tid = threadIdx.x;
    const int64_t b = blockIdx.x, N = a.N;
    if (a.idx[b * a.S] != kPending) return;
    const T* row = reinterpret_cast<const T*>(a.scores) + b * a.ld;
    const RowSettings set(a, b);
    float M = -INFINITY, low = INFINITY;
    each_four<THREADS>(row, N, [&](int64_t, const float (&x)[4]) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            M = fmaxf(M, x[e]);
            low = fminf(low, x[e] > -INFINITY ? x[e] : INFINITY);
        }
    });
    M = block_reduce<SW>(M, L.fbuf, OpMax());
    __syncthreads();
    low = -block_reduce<SW>(-low, L.fbuf, OpMax());
    __syncthreads();
    const RowWeight wt(M, set.temperature);
    uint64_t cut = 0;
    // (both cuts in one loop: the search is long code)
    for (int turn = 0; turn < 2; ++turn) {
        CutGoal goal{turn == 1, (uint32_t)set.top_k, 0.0};
        float range = M - low;
        if (turn == 0 ? !(set.top_k > 0 && set.top_k < N) : !(set.top_p < 1.0)) continue;
        if (turn == 1) {
            // the weight that p is a share of
            double sum = 0.0;
            each_four<THREADS>(row, N, [&](int64_t i, const float (&x)[4]) __attribute__((always_inline)) {
#pragma unroll
                for (int e = 0; e < 4; ++e) sum += ranking(x[e], (uint32_t)(i + e)) >= cut ? wt(x[e]) : 0.0;
            });
            sum = block_reduce<SW>(sum, L.dbuf, OpSum());
            __syncthreads();
            goal.mass = set.top_p * sum;
            // entries with less than (1 - p) / N of the largest weight lie behind the cut
            range = fminf((logf((float)N) - logf((float)(1.0 - set.top_p)) + 1.f) * (float)set.temperature, 1e38f);
        }
        cut = max(cut, find_cut(L, row, N, wt, goal, cut, range));
    }
    const int shift = chunk_shift<CHUNKS>(N);
    const int64_t len = 1ll << shift;
    const int n_chunks = (int)((N + len - 1) >> shift);
    __syncthreads();
    auto four = [&](int64_t i, const float (&x)[4]) __attribute__((always_inline)) {
        double sum = 0.0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const double w = ranking(x[e], (uint32_t)(i + e)) >= cut ? wt(x[e]) : 0.0;
            sum += w >= set.min_p ? w : 0.0;
        }
        return sum;
    };
    if (len == 64) {
        each_four<THREADS>(row, N, [&](int64_t i, const float (&x)[4]) __attribute__((always_inline)) {
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
    draw_kept(L, a, b, row, wt, cut, set.min_p, n_chunks, len);
}

namespace {

int64_t pieces_of(int64_t N) { return (N + kPiece - 1) / kPiece; }

template <typename T>
void launch(const SampleArgs& a, hipStream_t s)
{
    const bool cuts = a.top_k_rows || a.top_p_rows || a.min_p_rows || (a.top_k > 0 && a.top_k < a.N) || a.top_p < 1.0 ||
                      a.min_p > 0.0;
    // (2,048 rows of 63,361 without cuts, 4 draws each: 142 us so, 246 by
    // k_sample_rows; of 1,000: 17 and 24; one row of 63,361: 11 and 26)
    if (!cuts && pieces_of(a.N) <= kMaxPieces) {
        const int pieces = (int)pieces_of(a.N);
        double* sums = reinterpret_cast<double*>(a.ws);
        const SamplePieces q{sums, reinterpret_cast<float*>(sums + (int64_t)a.batch * pieces * 16), pieces};
        hipLaunchKernelGGL(k_sample_sums<T>, dim3(a.batch, (pieces + 3) / 4), dim3(256), 0, s, a, q);
        hipLaunchKernelGGL(k_sample_draw<T>, dim3(a.batch), dim3(256), pieces * 16 * sizeof(double), s, a, q);
        return;
    }
    // The row in registers where it fits: 16 scores a thread of 256 up to 4,096
    // (top-p, 2,048 rows of 4,000: 47 us, 104 with 32 a thread of 512; one row:
    // 16 and 23); up to 16,384, 16 of 1,024 where every row has a compute unit
    // (one row of 14,505: 22 us, top-k 19; with 32 of 512 23.5 and 24), else 32 of
    // 512, two or more rows to a unit (2,048 rows: 115 us, 165 and with 128 of
    // 512 304); 128 of 512 up to 65,536 (of 63,361: 379 us, 467 read again in each
    // pass; one row: 37 and 44).
    auto go = [&](auto kernel, int threads) {
        hipLaunchKernelGGL(kernel, dim3(a.batch), dim3(threads), 0, s, a);
        hipLaunchKernelGGL(k_sample_far<T>, dim3(a.batch), dim3(512), 0, s, a);
    };
    if (a.N <= 4096) go(k_sample_rows<T, 256, 4, 64, 4>, 256);
    else if (a.N <= 16384 && a.batch <= 256) go(k_sample_rows<T, 1024, 4, 256, 4>, 1024);
    else if (a.N <= 16384) go(k_sample_rows<T, 512, 8, 256, 4>, 512);
    else if (a.N <= 65536) go(k_sample_rows<T, 512, 32, 1024, 2>, 512);
    else go(k_sample_rows<T, 1024, 0, 4096, 4>, 1024);
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
