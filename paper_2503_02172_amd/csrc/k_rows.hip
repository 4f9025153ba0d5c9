// Rows of an embedding table by id, scaled, and the gradient of that with
// respect to the table:
//   out[t] = scale table[id_t]                          (id -1: zeros)
//   dT[v]  = (accumulate ? dT[v] : 0) + scale sum_{t: id_t = v} g[t]
// The gradient's sums run in float32 over the tokens of an id in a fixed
// order: the tokens are sorted by id first, stably, so a result does not
// depend on timing. The sorted tokens are cut into chunks of equal length,
// whatever their ids, so that an id with many tokens is summed by many
// wavefronts: a run of one id that lies inside a chunk goes to the table, a
// piece of a run that continues in another chunk to the workspace, and a last
// launch adds such pieces in chunk order. Few tokens take one launch, which
// compares their ids instead of sorting them.
#include <algorithm>

#include "row_ops.hpp"

namespace kgq {

namespace {

constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortBlocks = 128;             // blocks of a pass at most
constexpr int kFew = 2048;                   // tokens whose gradient takes one launch
constexpr int kFewWaves = 8;
constexpr int kFewAlone = 9;                 // tokens of an id that one wavefront adds
constexpr int kFewSplit = 64;                // workgroups of a token at most
constexpr int kJoinWaves = 16;
constexpr int kJoinAhead = 16;               // pieces in flight per wavefront
constexpr int kJoinAlone = 32;               // pieces of a run that one wavefront adds
constexpr int kAhead = 8;                    // gradient rows in flight per group
constexpr int kFillRows = 16;                // table rows per wavefront that are looked up for zeros

}  // namespace

// Elements at p and the row's end `left` columns on (more or fewer than V).
template <int V, typename T>
__device__ __forceinline__ void load_columns(const T* p, int left, float (&x)[V])
{
    typedef T vec __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    if (left >= V) {
        const vec v = *reinterpret_cast<const vec*>(p);
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = row_value((T)v[j]);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = j < left ? row_value(p[j]) : 0.f;
    }
}
// p[j] = scale x[j] (+ p[j])
template <int V, bool STREAM = false, typename O>
__device__ __forceinline__ void store_columns(O* p, int left, const float (&x)[V], float scale, bool accumulate)
{
    typedef O vec __attribute__((ext_vector_type(V), aligned(sizeof(O))));
    if (left >= V) {
        vec old = {}, y;
        if (accumulate) old = *reinterpret_cast<const vec*>(p);
#pragma unroll
        for (int j = 0; j < V; ++j)
            y[j] = row_element<O>(accumulate ? x[j] * scale + row_value((O)old[j]) : x[j] * scale);
        if (STREAM) __builtin_nontemporal_store(y, reinterpret_cast<vec*>(p));
        else *reinterpret_cast<vec*>(p) = y;
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j < left) p[j] = row_element<O>(accumulate ? x[j] * scale + row_value(p[j]) : x[j] * scale);
    }
}

// ---- lookup -----------------------------------------------------------------

// A workgroup takes `per` tokens, whose rows of `vecs` vectors of V elements
// lie one after the other over its threads: U vectors a thread, all of them
// loaded before the first is stored. inv = 2^32 / vecs rounded up: a quotient
// below 2^32 / vecs by one multiplication. 262,144 rows of 400 bfloat16 values to
// float32: 75 us, 5.6 TB/s of stores (a fill of the output 62); what it reads
// stays in the caches. 61 rows: 3 us, a launch.
template <typename T, typename O, int U>
__global__ __launch_bounds__(256) void k_embed_rows(EmbedArgs a, int per, int vecs, uint32_t inv)
{
    constexpr int V = sizeof(T) == 2 && sizeof(O) == 2 ? 8 : 4;
    const int64_t t0 = (int64_t)blockIdx.x * per;
    const T* table = reinterpret_cast<const T*>(a.table);
    O* out = reinterpret_cast<O*>(a.out);
    for (int j0 = threadIdx.x; j0 < per * vecs; j0 += U * 256) {
        float x[U][V];
        int64_t t[U];
        int c[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = j0 + u * 256;
            const int r = per == 1 ? 0 : vecs == 1 ? j : (int)__umulhi((uint32_t)j, inv);
            t[u] = t0 + r;
            c[u] = (j - r * vecs) * V;
            if (j >= per * vecs || t[u] >= a.n) t[u] = -1;
            const int32_t id = t[u] >= 0 ? a.ids[t[u]] : -1;
            if (id >= 0 && id < a.rows) {
                load_columns<V>(table + (int64_t)id * a.ld + c[u], a.d - c[u], x[u]);
            } else {
                if (id != -1 && a.flag) atomicOr(a.flag, kErrRange);
#pragma unroll
                for (int i = 0; i < V; ++i) x[u][i] = 0.f;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (t[u] >= 0) store_columns<V, (U > 1)>(out + t[u] * a.ld_out + c[u], a.d - c[u], x[u], a.scale, false);
    }
}

namespace {

template <typename T, typename O>
void launch_embed(const EmbedArgs& a, hipStream_t s)
{
    constexpr int V = sizeof(T) == 2 && sizeof(O) == 2 ? 8 : 4;
    const int vecs = (a.d + V - 1) / V;
    // four vectors a thread, stored past the caches, where that still leaves two
    // workgroups a compute unit (262,144 rows of 400 float32: 88 us, 172 with one;
    // 40,000: 17 and 20); one where latency counts (61 rows: 4.8 us, 5.1 with
    // four)
    const bool many = (int64_t)a.n * vecs >= (int64_t)512 * 1024;
    // (a launch has fewer than 2^32 threads)
    const int per = std::max({1, (many ? 1024 : 256) / vecs, (int)(((int64_t)a.n + (1 << 23) - 1) >> 23)});
    const uint32_t inv = (uint32_t)(((1ull << 32) + vecs - 1) / vecs);
    const dim3 grid((uint32_t)(((int64_t)a.n + per - 1) / per));
    if (many) hipLaunchKernelGGL((k_embed_rows<T, O, 4>), grid, dim3(256), 0, s, a, per, vecs, inv);
    else hipLaunchKernelGGL((k_embed_rows<T, O, 1>), grid, dim3(256), 0, s, a, per, vecs, inv);
}

}  // namespace

void launch_embed_rows(const EmbedArgs& a, hipStream_t s)
{
    if (a.dtype == KGQ_F32 && a.out_dtype == KGQ_F32) launch_embed<float, float>(a, s);
    else if (a.dtype == KGQ_F32) launch_embed<float, uint16_t>(a, s);
    else if (a.out_dtype == KGQ_F32) launch_embed<uint16_t, float>(a, s);
    else launch_embed<uint16_t, uint16_t>(a, s);
}

// ---- gradient of few tokens ---------------------------------------------------

// One launch. A workgroup takes a token and some blocks of 64 x 16 bytes of
// columns: it looks through all ids for its own, leaves it to the token before
// if there is one with the same id, and otherwise adds the rows of all of them
// in token order. Up to kFewAlone of them, a wavefront adds all of a block; more,
// each adds a share of them, and the shares are added in order. The workgroups
// behind the tokens' write zeros to the rows whose number they do not find among
// the ids. 1,536 tokens of 400 to 14,505 rows: 10.6 us, in a chain of calls 12
// (10 without the zeros' 23 MB): the latency of a launch, the ids, the rows and
// one exchange. As many wavefronts as keep the hottest ids short: with four 15
// us, with 16, of which most only look for the ids, 17.
template <typename T, typename O>
__global__ __launch_bounds__(64 * kFewWaves) void k_grad_few(EmbedGradArgs a, int blocks, int split)
{
    constexpr int V = RowVec<T>::n, AHEAD = 32 / V, THREADS = 64 * kFewWaves;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int token_groups = a.n * split;
    if ((int)blockIdx.x >= token_groups) {
        constexpr int VO = RowVec<O>::n, PER = 64, ROWS = PER / kFewWaves;
        __shared__ unsigned long long used;
        const int64_t step = (int64_t)(gridDim.x - token_groups) * PER;
        for (int64_t v0 = (int64_t)(blockIdx.x - token_groups) * PER; v0 < a.rows; v0 += step) {
            __syncthreads();
            if (tid == 0) used = 0ull;
            __syncthreads();
            for (int i = tid; i < a.n; i += THREADS) {
                const int64_t at = a.ids[i] - v0;
                if (at >= 0 && at < PER) atomicOr(&used, 1ull << at);
            }
            __syncthreads();
            const uint64_t mine = used >> (wave * ROWS);
            for (int r = 0; r < ROWS; ++r) {
                const int64_t v = v0 + wave * ROWS + r;
                if (v >= a.rows) break;
                if (mine >> r & 1) continue;
                const float zero[VO] = {};
                for (int c = lane * VO; c < a.d; c += 64 * VO)
                    store_columns<VO, true>(reinterpret_cast<O*>(a.out) + v * a.ld_out + c, a.d - c, zero, 1.f, false);
            }
        }
        return;
    }
    __shared__ uint64_t same[kFew / 64];             // the tokens with this id, as bits
    __shared__ uint16_t list[kFew];                  // and as a list
    __shared__ float share[kFewWaves][64 * V];
    const int t = blockIdx.x / split, block0 = blockIdx.x % split;   // (blocks block0, block0 + split, ...)
    const int32_t id = a.ids[t];
    if (id < 0 || id >= a.rows) {
        if (id != -1 && a.flag && tid == 0) atomicOr(a.flag, kErrRange);
        return;
    }
    const T* g = reinterpret_cast<const T*>(a.grad);
    O* out = reinterpret_cast<O*>(a.out) + (int64_t)id * a.ld_out;
    // (the token's own row meanwhile)
    int col = ((block0 + wave * split) * 64 + lane) * V;
    float sum[V];
    load_columns<V>(g + t * a.ld + col, a.d - col, sum);
    const int words = (a.n + 63) / 64;
    for (int w = wave; w < words; w += kFewWaves) {
        const int i = w * 64 + lane;
        const uint64_t m = __builtin_amdgcn_ballot_w64(i < a.n && a.ids[min(i, a.n - 1)] == id);
        if (lane == 0) same[w] = m;
    }
    __syncthreads();
    const uint64_t m = lane < words ? same[lane] : 0ull;
    const uint64_t before_t = lane < t / 64 ? m : lane == t / 64 ? m & ((1ull << (t & 63)) - 1) : 0ull;
    if (__builtin_amdgcn_ballot_w64(before_t != 0)) return;
    int upto = __popcll(m);                          // running count of the tokens in the words up to this lane's
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(upto, d, 64);
        if (lane >= d) upto += o;
    }
    const int total = __builtin_amdgcn_readlane(upto, 63);
    if (total > 1) {
        const int from = upto - __popcll(m);
        for (int w = wave; w < words; w += kFewWaves) {
            const uint64_t mw = same[w];
            const int at = __shfl(from, w, 64) + __popcll(mw & ((1ull << lane) - 1));
            if (mw >> lane & 1) list[at] = (uint16_t)(w * 64 + lane);
        }
        __syncthreads();
    }
    auto add = [&](int lo, int hi) __attribute__((always_inline)) {
        for (int i0 = lo; i0 < hi; i0 += AHEAD) {
            float x[AHEAD][V];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int64_t token = __builtin_amdgcn_readfirstlane((int)list[min(i0 + u, hi - 1)]);
                load_columns<V>(g + token * a.ld + col, a.d - col, x[u]);
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
#pragma unroll
                for (int j = 0; j < V; ++j) sum[j] += i0 + u < hi ? x[u][j] : 0.f;
        }
    };
    if (total <= kFewAlone) {
        for (int k = wave; block0 + k * split < blocks; k += kFewWaves) {
            col = ((block0 + k * split) * 64 + lane) * V;
            if (k != wave) load_columns<V>(g + t * a.ld + col, a.d - col, sum);
            add(1, total);
            store_columns<V, true>(out + col, a.d - col, sum, a.scale, a.accumulate != 0);
        }
        return;
    }
    const int per = (total + kFewWaves - 1) / kFewWaves, lo = min(total, wave * per), hi = min(total, lo + per);
    for (int block = block0; block < blocks; block += split) {
        col = (block * 64 + lane) * V;
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] = 0.f;
        add(lo, hi);
#pragma unroll
        for (int j = 0; j < V; ++j) share[wave][lane * V + j] = sum[j];
        __syncthreads();
        if (wave == 0) {
            for (int w = 1; w < kFewWaves; ++w)
#pragma unroll
                for (int j = 0; j < V; ++j) sum[j] += share[w][lane * V + j];
            store_columns<V, true>(out + col, a.d - col, sum, a.scale, a.accumulate != 0);
        }
        __syncthreads();
    }
}

// ---- tokens sorted by id ----------------------------------------------------

// A token's key: its id, or `rows` (behind every row) for what is no row.
__device__ __forceinline__ uint32_t token_key(const EmbedGradArgs& a, int64_t i)
{
    const int32_t id = a.ids[i];
    if (id >= 0 && id < a.rows) return (uint32_t)id;
    if (id != -1 && a.flag) atomicOr(a.flag, kErrRange);
    return (uint32_t)a.rows;
}

// Least significant digit first, 8 bits a pass, two launches a
// pass. Block b takes the positions [b * span, (b + 1) * span) tile by tile
// (one position per thread); hist[b * 256 + digit] is the number of its keys
// with that digit. The first pass reads the ids themselves. 262,144 tokens: 4.8
// us to count and 10.7 to place a pass, bound by latency (a block has two tiles:
// more blocks would each have more histograms to read).
__global__ __launch_bounds__(kSortThreads) void k_sort_count(EmbedGradArgs a, const int32_t* keys, int shift, int first,
                                                             int64_t span, uint32_t* hist)
{
    __shared__ uint32_t count[256];
    const int tid = threadIdx.x;
    if (tid < 256) count[tid] = 0;
    __syncthreads();
    const int64_t lo = blockIdx.x * span, hi = min((int64_t)a.n, lo + span);
    for (int64_t i = lo + tid; i < hi; i += kSortThreads)
        atomicAdd(&count[((first ? token_key(a, i) : (uint32_t)keys[i]) >> shift) & 255], 1u);
    __syncthreads();
    if (tid < 256) hist[(int64_t)blockIdx.x * 256 + tid] = count[tid];
}

__global__ __launch_bounds__(kSortThreads) void k_sort_place(EmbedGradArgs a, const int32_t* keys, const int32_t* tokens,
                                                             int shift, int first, int64_t span, const uint32_t* hist,
                                                             int32_t* keys_out, int32_t* tokens_out)
{
    __shared__ uint32_t base[256];                   // where the block's next key of a digit goes
    __shared__ uint32_t waves[kSortWaves][256];      // a tile's keys of a digit, by wavefront
    __shared__ uint4 part[2][kSortWaves][64];        // by wavefront: keys of four digits a lane
    __shared__ uint32_t scan[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    {
        // each digit's keys, and those in the blocks before this one: a
        // wavefront per block's histogram, 8 loads at most, all in flight
        uint4 all4 = make_uint4(0, 0, 0, 0), before4 = all4;
#pragma unroll
        for (int k = 0; k < kSortBlocks / kSortWaves; ++k) {
            const int b = k * kSortWaves + wave;
            if (b < (int)gridDim.x) {
                const uint4 h = reinterpret_cast<const uint4*>(hist)[(int64_t)b * 64 + lane];
                const uint32_t take = b < (int)blockIdx.x ? ~0u : 0u;
                all4.x += h.x;
                all4.y += h.y;
                all4.z += h.z;
                all4.w += h.w;
                before4.x += h.x & take;
                before4.y += h.y & take;
                before4.z += h.z & take;
                before4.w += h.w & take;
            }
        }
        part[0][wave][lane] = all4;
        part[1][wave][lane] = before4;
        __syncthreads();
        uint32_t x = 0, all = 0, before = 0;
        if (tid < 256) {
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) {
                all += reinterpret_cast<const uint32_t*>(part[0][w])[tid];
                before += reinterpret_cast<const uint32_t*>(part[1][w])[tid];
            }
            x = all;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const uint32_t o = __shfl_up(x, d, 64);
                if (lane >= d) x += o;
            }
            if (lane == 63) scan[wave] = x;
        }
        __syncthreads();
        if (tid < 256) {
            for (int w = 0; w < wave; ++w) x += scan[w];
            base[tid] = x - all + before;
        }
    }
    const int64_t lo = blockIdx.x * span, hi = min((int64_t)a.n, lo + span);
    for (int64_t i0 = lo; i0 < hi; i0 += kSortThreads) {
        const int64_t i = i0 + tid;
        const bool in = i < hi;
        const uint32_t key = in ? (first ? token_key(a, i) : (uint32_t)keys[i]) : 0u;
        const int32_t token = in ? (first ? (int32_t)i : tokens[i]) : 0;
        const uint32_t digit = (key >> shift) & 255;
        // the lanes with the same digit
        uint64_t same = __builtin_amdgcn_ballot_w64(in);
#pragma unroll
        for (int bit = 0; bit < 8; ++bit) {
            const uint64_t has = __builtin_amdgcn_ballot_w64((digit >> bit) & 1);
            same &= (digit >> bit) & 1 ? has : ~has;
        }
        const uint32_t rank = __popcll(same & ((1ull << lane) - 1));
#pragma unroll
        for (int w = 0; w < kSortWaves; w += kSortThreads / 256) waves[w + (tid >> 8)][tid & 255] = 0;
        __syncthreads();
        if (in && rank == 0) waves[wave][digit] = (uint32_t)__popcll(same);
        __syncthreads();
        // by wavefront: where its first key of a digit goes
        if (tid < 256) {
            uint32_t at = base[tid];
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) {
                const uint32_t c = waves[w][tid];
                waves[w][tid] = at;
                at += c;
            }
            base[tid] = at;
        }
        __syncthreads();
        if (in) {
            const uint32_t at = waves[wave][digit] + rank;
            keys_out[at] = (int32_t)key;
            tokens_out[at] = token;
        }
        __syncthreads();
    }
}

// ---- gradient ---------------------------------------------------------------

// How the sorted tokens are cut: groups of `lanes` lanes (a power of two) take
// a chunk and a block of lanes * 16 bytes of columns each.
struct GradCut {
    int lanes, blocks;                               // lanes per group, column blocks
    int chunk, chunks;                               // tokens per chunk, chunks
};

// First position in keys[0 .. n) with a key of at least v.
__device__ __forceinline__ int lower_bound(const int32_t* keys, int n, uint32_t v)
{
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = lo + ((hi - lo) >> 1);
        if ((uint32_t)keys[mid] < v) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

// The first `sum_blocks` workgroups sum chunks; the others write zeros to the
// rows without a token. piece: two rows of sums per chunk, of the run that
// came from the chunk before and of the run that leaves into the next.
// 262,144 tokens of 400 to 63,361 rows: 111 us, 4.8 TB/s of 419 MB read, 101
// written and 13 of pieces, the rate of a copy: each token's row is read once,
// wherever it lies.
template <typename T, typename O, bool WIDE>
__global__ __launch_bounds__(256) void k_grad_chunks(EmbedGradArgs a, GradCut cut, int sum_blocks, const int32_t* keys,
                                                     const int32_t* tokens, float* piece)
{
    constexpr int V = RowVec<T>::n;
    if ((int)blockIdx.x >= sum_blocks) {
        const int lane = threadIdx.x & 63;
        const int64_t waves = (int64_t)(gridDim.x - sum_blocks) * 4;
        for (int64_t w = (int64_t)(blockIdx.x - sum_blocks) * 4 + (threadIdx.x >> 6); w * kFillRows < a.rows; w += waves) {
            const int64_t v = w * kFillRows + lane;
            bool empty = false;
            if (lane < kFillRows && v < a.rows) {
                const int at = lower_bound(keys, a.n, (uint32_t)v);
                empty = at == a.n || (int64_t)keys[at] != v;
            }
            for (uint64_t rest = __builtin_amdgcn_ballot_w64(empty); rest; rest &= rest - 1) {
                O* row = reinterpret_cast<O*>(a.out) + (w * kFillRows + __builtin_ctzll(rest)) * a.ld_out;
                constexpr int VO = RowVec<O>::n;
                for (int c = lane * VO; c < a.d; c += 64 * VO) {
                    const float zero[VO] = {};
                    store_columns<VO, true>(row + c, a.d - c, zero, 1.f, false);
                }
            }
        }
        return;
    }
    int64_t group = ((int64_t)blockIdx.x * 256 + threadIdx.x) / cut.lanes;
    if (WIDE) group = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t chunk = group / cut.blocks;
    const int col = ((int)(group % cut.blocks) * cut.lanes + (threadIdx.x & (cut.lanes - 1))) * V;
    const int left = a.d - col;                      // (up to 0 in a row's last lanes, which then only keep up)
    if (chunk >= cut.chunks) return;
    const int lo = (int)(chunk * cut.chunk), hi = (int)min((int64_t)a.n, (chunk + 1) * cut.chunk);
    const T* g = reinterpret_cast<const T*>(a.grad) + col;
    O* out = reinterpret_cast<O*>(a.out) + col;
    uint32_t run = (uint32_t)keys[lo];
    const uint32_t ahead_of = (uint32_t)keys[max(lo - 1, 0)], behind = (uint32_t)keys[min(hi, a.n - 1)];
    bool from_before = lo > 0 && ahead_of == run;
    float sum[V] = {};
    auto flush = [&](bool leaves) {
        if ((int64_t)run < a.rows) {
            if (from_before || leaves) {
                store_columns<V>(piece + (2 * chunk + (from_before ? 0 : 1)) * a.d + col, left, sum, 1.f, false);
            } else {
                store_columns<V, true>(out + (int64_t)run * a.ld_out, left, sum, a.scale, a.accumulate != 0);
            }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] = 0.f;
        from_before = false;
    };
    // a whole wavefront per group: its chunk's keys and tokens in one load, then
    // from lane to scalar register
    uint32_t keys_ahead = 0, tokens_ahead = 0;
    const int count = hi - lo;                       // (positions are counted from lo: hi may be the largest int)
    if (WIDE && (int)(threadIdx.x & 63) < count) {
        keys_ahead = (uint32_t)keys[lo + (threadIdx.x & 63)];
        tokens_ahead = (uint32_t)tokens[lo + (threadIdx.x & 63)];
    }
    for (int i0 = 0; i0 < count; i0 += kAhead) {
        float x[kAhead][V];
        uint32_t key[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int i = min(i0 + u, count - 1);
            int64_t token;
            if (WIDE) {
                key[u] = __builtin_amdgcn_readlane(keys_ahead, i);
                token = __builtin_amdgcn_readlane(tokens_ahead, i);
            } else {
                key[u] = (uint32_t)keys[lo + i];
                token = tokens[lo + i];
            }
            // (rows of tokens without an id are not read)
            if ((int64_t)key[u] < a.rows) load_columns<V>(g + token * a.ld, left, x[u]);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i0 + u >= count) break;
            if (key[u] != run) {
                flush(false);
                run = key[u];
            }
            if ((int64_t)run < a.rows) {
#pragma unroll
                for (int j = 0; j < V; ++j) sum[j] += x[u][j];
            }
        }
    }
    flush(hi < a.n && behind == run);
}

// Pieces [lo, hi) of a run behind its first one, 256 columns: added to sum.
__device__ __forceinline__ void add_pieces(const float* rest, int d, int lo, int hi, int col, int left, float (&sum)[4])
{
    for (int i = lo; i < hi; i += kJoinAhead) {
        float x[kJoinAhead][4];
#pragma unroll
        for (int u = 0; u < kJoinAhead; ++u)
            load_columns<4>(rest + (int64_t)2 * min(i + u, hi - 1) * d + col, left, x[u]);
#pragma unroll
        for (int u = 0; u < kJoinAhead; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[j] += i + u < hi ? x[u][j] : 0.f;
    }
}

// The runs that start in one chunk and continue in the next: the sum of their
// pieces in chunk order. A wavefront looks at one chunk and adds a run of few
// pieces by itself; the workgroup then takes the longer runs of its 16 chunks
// together (each wavefront a share of the pieces, the shares added in order).
// 262,144 tokens, log-uniform ids: 13 us (the whole call 157; 200 if the
// workgroup takes every run); 2,500 tokens 8 us, 64 of one run 6: a chain of
// four loads.
template <typename O>
__global__ __launch_bounds__(64 * kJoinWaves) void k_grad_join(EmbedGradArgs a, GradCut cut, const int32_t* keys,
                                                               const float* piece)
{
    constexpr int V = 4;
    __shared__ float share[kJoinWaves][64 * V];
    __shared__ int pieces[kJoinWaves];               // of a run for the workgroup, or 0
    __shared__ uint32_t ids[kJoinWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * kJoinWaves + wave;
    int n = 0;                                       // pieces in the chunks behind c
    uint32_t run = 0;
    if (c + 1 < cut.chunks) {
        const int64_t next = (c + 1) * cut.chunk;    // (chunks but the last one are whole)
        // (every key that the usual run asks for, in one go)
        auto head = [&](int64_t k) { return (uint32_t)keys[min(k + lane, (int64_t)cut.chunks - 1) * cut.chunk]; };
        run = (uint32_t)keys[next - 1];
        const uint32_t after = (uint32_t)keys[next], first = (uint32_t)keys[next - cut.chunk];
        const uint32_t ahead = (uint32_t)keys[max(next - cut.chunk - 1, (int64_t)0)];
        uint32_t heads = head(c + 1);
        // (not if it came from the chunk before)
        bool mine = after == run && (int64_t)run < a.rows && !(c > 0 && first == run && ahead == run);
        // the chunks behind c that begin with it, 64 at a look
        for (int64_t k = c + 1; mine; heads = head(k)) {
            const uint64_t miss = __builtin_amdgcn_ballot_w64(!(k + lane < cut.chunks && heads == run));
            n += miss ? __builtin_ctzll(miss) : 64;
            mine = miss == 0;
            k += 64;
        }
    }
    if (lane == 0) {
        pieces[wave] = n > kJoinAlone ? n : 0;
        ids[wave] = run;
    }
    if (n > 0 && n <= kJoinAlone) {
        O* out = reinterpret_cast<O*>(a.out) + (int64_t)run * a.ld_out;
        for (int col = lane * V; col < a.d; col += 64 * V) {
            float sum[V];
            load_columns<V>(piece + (2 * c + 1) * a.d + col, a.d - col, sum);
            add_pieces(piece + 2 * (c + 1) * a.d, a.d, 0, n, col, a.d - col, sum);
            store_columns<V>(out + col, a.d - col, sum, a.scale, a.accumulate != 0);
        }
    }
    __syncthreads();
    for (int r = 0; r < kJoinWaves; ++r) {
        n = pieces[r];
        if (n == 0) continue;
        const int64_t cr = (int64_t)blockIdx.x * kJoinWaves + r;
        const int per = (n + kJoinWaves - 1) / kJoinWaves;
        const int lo = min(n, wave * per), hi = min(n, lo + per);
        O* out = reinterpret_cast<O*>(a.out) + (int64_t)ids[r] * a.ld_out;
        for (int col0 = 0; col0 < a.d; col0 += 64 * V) {
            const int col = col0 + lane * V, left = a.d - col;
            float sum[V] = {};
            if (left > 0) {
                if (wave == 0) load_columns<V>(piece + (2 * cr + 1) * a.d + col, left, sum);
                add_pieces(piece + 2 * (cr + 1) * a.d, a.d, lo, hi, col, left, sum);
            }
#pragma unroll
            for (int j = 0; j < V; ++j) share[wave][lane * V + j] = sum[j];
            __syncthreads();
            if (wave == 0 && left > 0) {
                for (int w = 1; w < kJoinWaves; ++w)
#pragma unroll
                    for (int j = 0; j < V; ++j) sum[j] += share[w][lane * V + j];
                store_columns<V>(out + col, left, sum, a.scale, a.accumulate != 0);
            }
            __syncthreads();
        }
    }
}

namespace {

int64_t align256(int64_t bytes) { return (bytes + 255) / 256 * 256; }

// Blocks of a sort pass, each over a run of whole tiles: few enough that every
// block sums the histograms of all.
int sort_blocks(int64_t n)
{
    return (int)std::max<int64_t>(1, std::min<int64_t>(kSortBlocks, (n + kSortThreads - 1) / kSortThreads));
}

// Groups of just enough lanes for a row, 16 bytes a lane, and chunks that give
// the chip some 16 wavefronts a compute unit: 8 to 64 tokens (5,000 tokens of
// 400: 31 us with 8, 49 with 64; 262,144: 157 us with 64, 225 with 8; longer ones
// would save pieces, one or two rows a chunk, that are few beside 64 already).
// vec: elements of 16 bytes of the gradient's type; the workspace, which is
// asked for without it, holds the pieces of either type's cut.
GradCut grad_cut(int64_t n, int d, int vec)
{
    GradCut c;
    c.lanes = 1;
    while (c.lanes < 64 && c.lanes * vec < d) c.lanes <<= 1;
    c.blocks = (d + c.lanes * vec - 1) / (c.lanes * vec);
    c.chunk = 8;
    while (c.chunk < 64 && n * c.blocks * c.lanes / c.chunk > (int64_t)256 * 16 * 64) c.chunk <<= 1;
    c.chunks = (int)((n + c.chunk - 1) / c.chunk);
    return c;
}

template <typename T, typename O>
void launch_grad(const EmbedGradArgs& a, const int32_t* keys, const int32_t* tokens, float* piece, hipStream_t s)
{
    const GradCut cut = grad_cut(a.n, a.d, RowVec<T>::n);
    const int64_t sum_blocks = ((int64_t)cut.chunks * cut.blocks * cut.lanes + 255) / 256;
    const int64_t fill_blocks =
        a.accumulate ? 0 : std::min<int64_t>((a.rows + 4 * kFillRows - 1) / (4 * kFillRows), 1 << 18);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((uint32_t)(sum_blocks + fill_blocks)), dim3(256), 0, s, a, cut,
                           (int)sum_blocks, keys, tokens, piece);
    };
    if (sum_blocks + fill_blocks > 0) {
        if (cut.lanes == 64) go(k_grad_chunks<T, O, true>);
        else go(k_grad_chunks<T, O, false>);
    }
    if (cut.chunks > 1)
        hipLaunchKernelGGL(k_grad_join<O>, dim3((cut.chunks - 1 + kJoinWaves - 1) / kJoinWaves), dim3(64 * kJoinWaves), 0, s, a, cut, keys, piece);
}

}  // namespace

int64_t embed_grad_workspace(int64_t n, int d)
{
    const int64_t pieces = std::max(grad_cut(n, d, RowVec<float>::n).chunks, grad_cut(n, d, RowVec<uint16_t>::n).chunks);
    return 4 * align256(n * 4) + align256((int64_t)256 * sort_blocks(n) * 4) + align256(2 * pieces * d * 4);
}

namespace {

template <typename T, typename O>
void launch_all(const EmbedGradArgs& a, hipStream_t s)
{
    // One launch instead of six or more: a call takes 11 us for 1,536 tokens of
    // 400 and 28 sorted, 61: 10 (the host's) and 24, 2,500: 17 and 29, 4,096: 26
    // and 30. But ids with
    // hundreds of tokens take longer than sorted (1,536 of one id: 57 us and 30),
    // and longer the more tokens: hence no more than kFew.
    if (a.n <= kFew) {
        const int blocks = (a.d + 64 * RowVec<T>::n - 1) / (64 * RowVec<T>::n);
        const int64_t fill = a.accumulate ? 0 : std::min<int64_t>((a.rows + 63) / 64, 1 << 18);
        // two blocks of columns a workgroup: an id with every token of 2,048 of
        // 2,000 columns takes 94 us so, 302 with all in one (no two alike: 47, 32)
        const int split = std::min((blocks + 1) / 2, kFewSplit);
        if (a.n + fill > 0)
            hipLaunchKernelGGL((k_grad_few<T, O>), dim3((uint32_t)(a.n * split + fill)), dim3(64 * kFewWaves), 0, s, a,
                               blocks, split);
        return;
    }
    char* ws = reinterpret_cast<char*>(a.ws);
    int32_t* buf[4];
    for (auto& b : buf) {
        b = reinterpret_cast<int32_t*>(ws);
        ws += align256((int64_t)a.n * 4);
    }
    const int sorters = sort_blocks(a.n);
    uint32_t* hist = reinterpret_cast<uint32_t*>(ws);
    float* piece = reinterpret_cast<float*>(ws + align256((int64_t)256 * sorters * 4));
    const int32_t *keys = buf[0], *tokens = buf[1];
    const int64_t tiles = ((int64_t)a.n + kSortThreads - 1) / kSortThreads;
    const int64_t span = (tiles + sorters - 1) / sorters * kSortThreads;
    int side = 0;
    for (int shift = 0; shift == 0 || (a.rows >> shift) > 0; shift += 8) {
        int32_t *ko = buf[side], *to = buf[side + 1];
        hipLaunchKernelGGL(k_sort_count, dim3(sorters), dim3(kSortThreads), 0, s, a, keys, shift, shift == 0, span, hist);
        hipLaunchKernelGGL(k_sort_place, dim3(sorters), dim3(kSortThreads), 0, s, a, keys, tokens, shift, shift == 0,
                           span, hist, ko, to);
        keys = ko;
        tokens = to;
        side ^= 2;
    }
    launch_grad<T, O>(a, keys, tokens, piece, s);
}

}  // namespace

void launch_embed_grad(const EmbedGradArgs& a, hipStream_t s)
{
    if (a.dtype == KGQ_F32 && a.out_dtype == KGQ_F32) launch_all<float, float>(a, s);
    else if (a.dtype == KGQ_F32) launch_all<float, uint16_t>(a, s);
    else if (a.out_dtype == KGQ_F32) launch_all<uint16_t, float>(a, s);
    else launch_all<uint16_t, uint16_t>(a, s);
}

}  // namespace kgq
