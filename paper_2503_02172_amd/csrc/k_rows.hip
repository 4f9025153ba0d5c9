// Rows of an embedding table by id, scaled, and the gradient of that with
// respect to the table:
//   out[t] = scale table[id_t]                          (id -1: zeros)
//   dT[v]  = (accumulate ? dT[v] : 0) + scale sum_{t: id_t = v} g[t]
// The gradient's sums run in float32 over the tokens of an id in a fixed
// order: the tokens are sorted by id first, stably (least significant digit
// first, 8 bits a pass), so a result does not depend on timing.
#include <algorithm>

#include "row_ops.hpp"

namespace kgq {

namespace {

constexpr int kSortThreads = 256;
constexpr int kSortWaves = kSortThreads / 64;

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

// A pass over 8 bits of the keys. Block b takes the positions
// [b * span, (b + 1) * span) tile by tile (256 positions, one per thread);
// hist[digit * blocks + b] is the number of its keys with that digit. The
// first pass reads the ids themselves (key `rows`, behind every row, for what
// is no row), the others the pass before.
__device__ __forceinline__ uint32_t sort_key(const EmbedGradArgs& a, const int32_t* keys, int64_t i, bool first)
{
    if (!first) return (uint32_t)keys[i];
    const int32_t id = a.ids[i];
    if (id >= 0 && id < a.rows) return (uint32_t)id;
    if (id != -1 && a.flag) atomicOr(a.flag, kErrRange);
    return (uint32_t)a.rows;
}

__global__ __launch_bounds__(kSortThreads) void k_sort_count(EmbedGradArgs a, const int32_t* keys, int shift, int first,
                                                             int64_t span, uint32_t* hist)
{
    __shared__ uint32_t count[256];
    const int tid = threadIdx.x;
    count[tid] = 0;
    __syncthreads();
    const int64_t lo = blockIdx.x * span, hi = min((int64_t)a.n, lo + span);
    for (int64_t i = lo + tid; i < hi; i += kSortThreads)
        atomicAdd(&count[(sort_key(a, keys, i, first) >> shift) & 255], 1u);
    __syncthreads();
    hist[(int64_t)tid * gridDim.x + blockIdx.x] = count[tid];
}

__global__ __launch_bounds__(kSortThreads) void k_sort_place(EmbedGradArgs a, const int32_t* keys, const int32_t* tokens,
                                                             int shift, int first, int64_t span, const uint32_t* hist,
                                                             int32_t* keys_out, int32_t* tokens_out)
{
    __shared__ uint32_t base[256];                   // where the block's next key of a digit goes
    __shared__ uint32_t waves[kSortWaves][256];      // a tile's keys of a digit, by wavefront
    __shared__ uint32_t scan[kSortWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int blocks = gridDim.x;
    {
        // digit tid: all its keys, and those in the blocks before this one
        uint32_t all = 0, before = 0;
        for (int b = 0; b < blocks; ++b) {
            const uint32_t h = hist[(int64_t)tid * blocks + b];
            if (b < (int)blockIdx.x) before += h;
            all += h;
        }
        uint32_t x = all;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t o = __shfl_up(x, d, 64);
            if (lane >= d) x += o;
        }
        if (lane == 63) scan[wave] = x;
        __syncthreads();
        for (int w = 0; w < wave; ++w) x += scan[w];
        base[tid] = x - all + before;
    }
    const int64_t lo = blockIdx.x * span, hi = min((int64_t)a.n, lo + span);
    for (int64_t i0 = lo; i0 < hi; i0 += kSortThreads) {
        const int64_t i = i0 + tid;
        const bool in = i < hi;
        const uint32_t key = in ? sort_key(a, keys, i, first) : 0u;
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
        for (int w = 0; w < kSortWaves; ++w) waves[w][tid] = 0;
        __syncthreads();
        if (in && rank == 0) waves[wave][digit] = (uint32_t)__popcll(same);
        __syncthreads();
        if (in) {
            uint32_t at = base[digit] + rank;
            for (int w = 0; w < wave; ++w) at += waves[w][digit];
            keys_out[at] = (int32_t)key;
            tokens_out[at] = token;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) base[tid] += waves[w][tid];
        __syncthreads();
    }
}

// ---- gradient ---------------------------------------------------------------

// First position in keys[0 .. n) with a key of at least v, by a whole wavefront.
__device__ __forceinline__ int64_t wave_lower_bound(const int32_t* keys, int64_t n, int64_t v)
{
    const int lane = threadIdx.x & 63;
    int64_t lo = 0, hi = n;                          // the answer lies in [lo, hi]
    while (lo < hi) {
        const int64_t step = (hi - lo + 63) / 64;
        const int64_t at = lo + lane * step;
        const bool below = at < hi && (int64_t)keys[at] < v;
        const int k = __popcll(__builtin_amdgcn_ballot_w64(below));
        if (k == 0) return lo;
        const int64_t from = lo + (k - 1) * step + 1;
        hi = min(hi, lo + k * step);
        lo = from;
    }
    return lo;
}

// One wavefront per row of the table.
template <typename T, typename O>
__global__ __launch_bounds__(256) void k_embed_grad(EmbedGradArgs a, const int32_t* keys, const int32_t* tokens)
{
    const int lane = threadIdx.x & 63;
    for (int64_t v = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); v < a.rows; v += (int64_t)gridDim.x * 4) {
        const int64_t lo = wave_lower_bound(keys, a.n, v), hi = wave_lower_bound(keys, a.n, v + 1);
        if (lo == hi && a.accumulate) continue;
        O* out = reinterpret_cast<O*>(a.out) + v * a.ld_out;
        for (int c = lane; c < a.d; c += 64) {
            float sum = 0.f;
            for (int64_t i = lo; i < hi; ++i)
                sum += row_value(reinterpret_cast<const T*>(a.grad)[(int64_t)tokens[i] * a.ld + c]);
            sum *= a.scale;
            if (a.accumulate) sum += row_value(out[c]);
            out[c] = row_element<O>(sum);
        }
    }
}

namespace {

int64_t align256(int64_t bytes) { return (bytes + 255) / 256 * 256; }

// Blocks of a sort pass, each over a run of whole tiles: at most 256, so that
// summing the blocks' histograms stays small beside the pass.
int sort_blocks(int64_t n) { return (int)std::max<int64_t>(1, std::min<int64_t>(256, (n + 4095) / 4096)); }

}  // namespace

int64_t embed_grad_workspace(int64_t n)
{
    return 4 * align256(n * 4) + align256((int64_t)256 * sort_blocks(n) * 4);
}

void launch_embed_grad(const EmbedGradArgs& a, hipStream_t s)
{
    char* ws = reinterpret_cast<char*>(a.ws);
    int32_t* buf[4];
    for (auto& b : buf) {
        b = reinterpret_cast<int32_t*>(ws);
        ws += align256((int64_t)a.n * 4);
    }
    uint32_t* hist = reinterpret_cast<uint32_t*>(ws);
    const int blocks = sort_blocks(a.n);
    const int64_t tiles = (a.n + kSortThreads - 1) / kSortThreads;
    const int64_t span = (tiles + blocks - 1) / blocks * kSortThreads;
    const int32_t *keys = nullptr, *tokens = nullptr;
    int side = 0;
    for (int shift = 0; shift == 0 || (a.rows >> shift) > 0; shift += 8) {
        int32_t *ko = buf[side], *to = buf[side + 1];
        hipLaunchKernelGGL(k_sort_count, dim3(blocks), dim3(kSortThreads), 0, s, a, keys, shift, shift == 0, span, hist);
        hipLaunchKernelGGL(k_sort_place, dim3(blocks), dim3(kSortThreads), 0, s, a, keys, tokens, shift, shift == 0, span,
                           hist, ko, to);
        keys = ko;
        tokens = to;
        side ^= 2;
    }
    const dim3 grid((uint32_t)std::min<int64_t>((a.rows + 3) / 4, 1 << 20));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a, keys, tokens); };
    if (a.dtype == KGQ_F32 && a.out_dtype == KGQ_F32) go(k_embed_grad<float, float>);
    else if (a.dtype == KGQ_F32) go(k_embed_grad<float, uint16_t>);
    else if (a.out_dtype == KGQ_F32) go(k_embed_grad<uint16_t, float>);
    else go(k_embed_grad<uint16_t, uint16_t>);
}

}  // namespace kgq
