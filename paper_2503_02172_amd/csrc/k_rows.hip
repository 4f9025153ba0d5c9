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
// launch adds such pieces in chunk order.
#include <algorithm>

#include "row_ops.hpp"

namespace kgq {

namespace {

constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortParts = kSortThreads / 256;
constexpr int kSortShort = 4096;             // tokens that the counting sort takes
constexpr int kJoinWaves = 8;
constexpr int kAhead = 8;                    // gradient rows in flight per group
constexpr int kFillRows = 16;                // table rows per wavefront that are looked up for zeros

}  // namespace

// ---- lookup -----------------------------------------------------------------

template <typename T, typename O>
__global__ __launch_bounds__(256) void k_embed_rows(EmbedArgs a)
{
    const int64_t total = (int64_t)a.n * a.d;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t t = i / a.d, c = i % a.d;
        const int32_t id = a.ids[t];
        const bool ok = id >= 0 && id < a.rows;
        if (!ok && id != -1 && a.flag) atomicOr(a.flag, kErrRange);
        const float x = ok ? a.scale * row_value(reinterpret_cast<const T*>(a.table)[id * a.ld + c]) : 0.f;
        reinterpret_cast<O*>(a.out)[t * a.ld_out + c] = row_element<O>(x);
    }
}

void launch_embed_rows(const EmbedArgs& a, hipStream_t s)
{
    const int64_t blocks = std::min<int64_t>(((int64_t)a.n * a.d + 255) / 256, 8192);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((uint32_t)blocks), dim3(256), 0, s, a); };
    if (a.dtype == KGQ_F32 && a.out_dtype == KGQ_F32) go(k_embed_rows<float, float>);
    else if (a.dtype == KGQ_F32) go(k_embed_rows<float, uint16_t>);
    else if (a.out_dtype == KGQ_F32) go(k_embed_rows<uint16_t, float>);
    else go(k_embed_rows<uint16_t, uint16_t>);
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

// Few tokens: a token's place is the number of tokens with a smaller key, or
// the same key and earlier. One launch; n^2 comparisons, spread over the chip
// (64 tokens per workgroup, each wavefront against a quarter of all).
__global__ __launch_bounds__(256) void k_sort_short(EmbedGradArgs a, int32_t* keys_out, int32_t* tokens_out)
{
    __shared__ alignas(16) uint32_t key[kSortShort];
    __shared__ uint32_t before[4][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n4 = (a.n + 15) / 16 * 16;
    for (int i = tid; i < n4; i += 256) key[i] = i < a.n ? token_key(a, i) : ~0u;
    __syncthreads();
    const int t = blockIdx.x * 64 + lane;
    const uint32_t mine = t < a.n ? key[t] : 0u;
    uint32_t count = 0;
    const int part = n4 / 4, lo = wave * part;
#pragma unroll 4
    for (int j = lo; j < lo + part; j += 4) {
        const uint4 k = *reinterpret_cast<const uint4*>(&key[j]);
        count += (k.x < mine || (k.x == mine && j < t)) + (k.y < mine || (k.y == mine && j + 1 < t)) +
                 (k.z < mine || (k.z == mine && j + 2 < t)) + (k.w < mine || (k.w == mine && j + 3 < t));
    }
    before[wave][lane] = count;
    __syncthreads();
    if (wave == 0 && t < a.n) {
        const uint32_t at = before[0][lane] + before[1][lane] + before[2][lane] + before[3][lane];
        keys_out[at] = (int32_t)mine;
        tokens_out[at] = t;
    }
}

// Many tokens: least significant digit first, 8 bits a pass, two launches a
// pass. Block b takes the positions [b * span, (b + 1) * span) tile by tile
// (one position per thread); hist[b * 256 + digit] is the number of its keys
// with that digit. The first pass reads the ids themselves.
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
    __shared__ uint32_t part[2][kSortParts][256];
    __shared__ uint32_t scan[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    {
        // each digit's keys, and those in the blocks before this one
        const int digit = tid & 255, q = tid >> 8;
        uint32_t all = 0, before = 0;
#pragma unroll 8
        for (int b = q; b < (int)gridDim.x; b += kSortParts) {
            const uint32_t h = hist[(int64_t)b * 256 + digit];
            all += h;
            before += b < (int)blockIdx.x ? h : 0u;
        }
        part[0][q][digit] = all;
        part[1][q][digit] = before;
        __syncthreads();
        uint32_t x = 0;
        if (tid < 256) {
            all = before = 0;
#pragma unroll
            for (int p = 0; p < kSortParts; ++p) {
                all += part[0][p][tid];
                before += part[1][p][tid];
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
        for (int w = 0; w < kSortWaves; w += kSortParts) waves[w + (tid >> 8)][tid & 255] = 0;
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

// n elements at p, from a row whose columns from p on number `left` (more or
// fewer than n).
template <typename T>
__device__ __forceinline__ void load_columns(const T* p, int left, float (&x)[RowVec<T>::n])
{
    constexpr int V = RowVec<T>::n;
    if (left >= V) {
        const typename RowVec<T>::type v = *reinterpret_cast<const typename RowVec<T>::type*>(p);
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = row_value((T)v[j]);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = j < left ? row_value(p[j]) : 0.f;
    }
}
template <int V, typename O>
__device__ __forceinline__ void store_row(O* p, int left, const float (&x)[V], float scale, bool accumulate)
{
    typedef O vec __attribute__((ext_vector_type(V), aligned(sizeof(O))));
    if (left >= V) {
        vec old = {}, y;
        if (accumulate) old = *reinterpret_cast<const vec*>(p);
#pragma unroll
        for (int j = 0; j < V; ++j)
            y[j] = row_element<O>(accumulate ? x[j] * scale + row_value((O)old[j]) : x[j] * scale);
        *reinterpret_cast<vec*>(p) = y;
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j < left) p[j] = row_element<O>(accumulate ? x[j] * scale + row_value(p[j]) : x[j] * scale);
    }
}
template <int V>
__device__ __forceinline__ void store_piece(float* p, int left, const float (&x)[V])
{
    typedef float vec __attribute__((ext_vector_type(V), aligned(4)));
    if (left >= V) {
        vec y;
#pragma unroll
        for (int j = 0; j < V; ++j) y[j] = x[j];
        *reinterpret_cast<vec*>(p) = y;
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j < left) p[j] = x[j];
    }
}

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
template <typename T, typename O>
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
                    store_row<VO>(row + c, a.d - c, zero, 1.f, false);
                }
            }
        }
        return;
    }
    const int64_t group = ((int64_t)blockIdx.x * 256 + threadIdx.x) / cut.lanes;
    const int64_t chunk = group / cut.blocks;
    const int col = ((int)(group % cut.blocks) * cut.lanes + (threadIdx.x & (cut.lanes - 1))) * V;
    const int left = a.d - col;
    if (chunk >= cut.chunks || left <= 0) return;
    const int lo = (int)(chunk * cut.chunk), hi = (int)min((int64_t)a.n, (chunk + 1) * cut.chunk);
    const T* g = reinterpret_cast<const T*>(a.grad) + col;
    O* out = reinterpret_cast<O*>(a.out) + col;
    uint32_t run = (uint32_t)keys[lo];
    bool from_before = lo > 0 && (uint32_t)keys[lo - 1] == run;
    float sum[V] = {};
    auto flush = [&](bool leaves) {
        if ((int64_t)run < a.rows) {
            if (from_before || leaves) {
                store_piece<V>(piece + (2 * chunk + (from_before ? 0 : 1)) * a.d + col, left, sum);
            } else {
                store_row<V>(out + (int64_t)run * a.ld_out, left, sum, a.scale, a.accumulate != 0);
            }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] = 0.f;
        from_before = false;
    };
    for (int i0 = lo; i0 < hi; i0 += kAhead) {
        float x[kAhead][V];
        uint32_t key[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int i = min(i0 + u, hi - 1);
            key[u] = (uint32_t)keys[i];
            // (rows of tokens without an id are not read)
            if ((int64_t)key[u] < a.rows) load_columns(g + (int64_t)tokens[i] * a.ld, left, x[u]);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i0 + u >= hi) break;
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
    flush(hi < a.n && (uint32_t)keys[hi] == run);
}

// Block c: if a run starts in chunk c and continues in the next, the sum of
// its pieces in chunk order (each wavefront adds a share of them, the shares
// are added in order).
template <typename O>
__global__ __launch_bounds__(64 * kJoinWaves) void k_grad_join(EmbedGradArgs a, GradCut cut, const int32_t* keys,
                                                               const float* piece)
{
    constexpr int V = 4;
    __shared__ float share[kJoinWaves][64 * V];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = blockIdx.x;
    const int64_t next = (c + 1) * cut.chunk;        // (chunks but the last one are whole)
    const uint32_t run = (uint32_t)keys[next - 1];
    if ((uint32_t)keys[next] != run || (int64_t)run >= a.rows) return;
    // did it come from the chunk before?
    if (c > 0 && (uint32_t)keys[next - cut.chunk] == run && (uint32_t)keys[next - cut.chunk - 1] == run) return;
    const int end = lower_bound(keys, a.n, run + 1);
    const int n = (int)((end - 1) / cut.chunk - c);  // pieces in the chunks behind this one
    const int per = (n + kJoinWaves - 1) / kJoinWaves;
    const int lo = min(n, wave * per), hi = min(n, lo + per);
    const float* first = piece + (2 * c + 1) * a.d;  // the run's start
    const float* rest = piece + 2 * (c + 1) * a.d;   // its piece in the next chunk; the others 2 rows on each
    O* out = reinterpret_cast<O*>(a.out) + (int64_t)run * a.ld_out;
    for (int col0 = 0; col0 < a.d; col0 += 64 * V) {
        const int col = col0 + lane * V, left = a.d - col;
        float sum[V] = {};
        if (left > 0) {
            if (wave == 0) load_columns(first + col, left, sum);
            int i = lo;
            for (; i + kAhead <= hi; i += kAhead) {
                float x[kAhead][V];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) load_columns(rest + (int64_t)2 * (i + u) * a.d + col, left, x[u]);
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
#pragma unroll
                    for (int j = 0; j < V; ++j) sum[j] += x[u][j];
            }
            for (; i < hi; ++i) {
                float x[V];
                load_columns(rest + (int64_t)2 * i * a.d + col, left, x);
#pragma unroll
                for (int j = 0; j < V; ++j) sum[j] += x[j];
            }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) share[wave][lane * V + j] = sum[j];
        __syncthreads();
        if (wave == 0 && left > 0) {
            for (int w = 1; w < kJoinWaves; ++w)
#pragma unroll
                for (int j = 0; j < V; ++j) sum[j] += share[w][lane * V + j];
            store_row<V>(out + col, left, sum, a.scale, a.accumulate != 0);
        }
        __syncthreads();
    }
}

namespace {

int64_t align256(int64_t bytes) { return (bytes + 255) / 256 * 256; }

// Blocks of a sort pass, each over a run of whole tiles: at most 256, so that
// summing the blocks' histograms stays small beside the pass.
int sort_blocks(int64_t n)
{
    return (int)std::max<int64_t>(1, std::min<int64_t>(256, (n + kSortThreads - 1) / kSortThreads));
}

// Groups of just enough lanes for a row, 16 bytes a lane, and chunks that give
// the chip some 16 wavefronts a compute unit: 8 to 64 tokens (longer ones
// would save pieces, one or two rows a chunk, that are few beside 64 already).
// The element size is the smaller of the two types', so that the workspace
// holds either.
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
    if (sum_blocks + fill_blocks > 0)
        hipLaunchKernelGGL((k_grad_chunks<T, O>), dim3((uint32_t)(sum_blocks + fill_blocks)), dim3(256), 0, s, a, cut,
                           (int)sum_blocks, keys, tokens, piece);
    if (cut.chunks > 1)
        hipLaunchKernelGGL(k_grad_join<O>, dim3(cut.chunks - 1), dim3(64 * kJoinWaves), 0, s, a, cut, keys, piece);
}

}  // namespace

int64_t embed_grad_workspace(int64_t n, int d)
{
    const int64_t pieces = std::max(grad_cut(n, d, RowVec<float>::n).chunks, grad_cut(n, d, RowVec<uint16_t>::n).chunks);
    return 4 * align256(n * 4) + align256((int64_t)256 * sort_blocks(n) * 4) + align256(2 * pieces * d * 4);
}

void launch_embed_grad(const EmbedGradArgs& a, hipStream_t s)
{
    char* ws = reinterpret_cast<char*>(a.ws);
    int32_t* buf[4];
    for (auto& b : buf) {
        b = reinterpret_cast<int32_t*>(ws);
        ws += align256((int64_t)a.n * 4);
    }
    const int blocks = sort_blocks(a.n);
    uint32_t* hist = reinterpret_cast<uint32_t*>(ws);
    float* piece = reinterpret_cast<float*>(ws + align256((int64_t)256 * blocks * 4));
    const int32_t *keys = buf[0], *tokens = buf[1];
    if (a.n > kSortShort) {
        const int64_t tiles = ((int64_t)a.n + kSortThreads - 1) / kSortThreads;
        const int64_t span = (tiles + blocks - 1) / blocks * kSortThreads;
        int side = 0;
        for (int shift = 0; shift == 0 || (a.rows >> shift) > 0; shift += 8) {
            int32_t *ko = buf[side], *to = buf[side + 1];
            hipLaunchKernelGGL(k_sort_count, dim3(blocks), dim3(kSortThreads), 0, s, a, keys, shift, shift == 0, span,
                               hist);
            hipLaunchKernelGGL(k_sort_place, dim3(blocks), dim3(kSortThreads), 0, s, a, keys, tokens, shift,
                               shift == 0, span, hist, ko, to);
            keys = ko;
            tokens = to;
            side ^= 2;
        }
    } else if (a.n > 0) {
        hipLaunchKernelGGL(k_sort_short, dim3((a.n + 63) / 64), dim3(256), 0, s, a, buf[0], buf[1]);
    }
    if (a.dtype == KGQ_F32 && a.out_dtype == KGQ_F32) launch_grad<float, float>(a, keys, tokens, piece, s);
    else if (a.dtype == KGQ_F32) launch_grad<float, uint16_t>(a, keys, tokens, piece, s);
    else if (a.out_dtype == KGQ_F32) launch_grad<uint16_t, float>(a, keys, tokens, piece, s);
    else launch_grad<uint16_t, uint16_t>(a, keys, tokens, piece, s);
}

}  // namespace kgq
