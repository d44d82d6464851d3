// Gradient of the embedding's table: dW[v] = scale sum over the tokens k of id v of dy[k].
//
// The tokens are sorted by id (a stable counting sort, digit by digit, from the least; few
// tokens by counting for each what comes before it), so that a row's tokens lie side by side in
// the order of their positions and their sum has the same bits on every call.  Then a workgroup
// takes a window of sorted tokens and walks it with its columns in registers: what begins and
// ends in the window is stored, what crosses a border goes to the workspace (at most one run
// enters and one leaves a window), and a last launch adds those, window by window.
//
// Rows without a token are zeros.  The sort's launches are short and leave the GPU idle, so each
// has further workgroups that store their share of zeros to all of dW; rows with tokens
// are stored again.
//
// Bound by memory: n rows of dy are read, V rows of dW written and the rows with tokens once
// more, beside launches of a few microseconds each.  65536 tokens of bfloat16 x 2048 with a
// table of 50000 rows, 16600 of them met: 66 us the sort and the zeros (6.2 TB/s), 125 the runs,
// 12 the joins; added to what is there (no zeros, the rows with tokens read too) 215 us in all, from
// float32 rows 247 written and 244 added.  Other ways that were built for the zeros: a fill of its own before the sort,
// 228 us in all against 203; only the rows without a token, which the sums' launch looks up
// among the sorted keys, 196, with a search in every row of it; the same from a bit per row that
// the sort sets, 344 (many tokens of few rows meet in an atomic).
#include "embed.hpp"

#include "block_ops.hpp"

namespace lh {
namespace {

constexpr int kSortBlock = 1024;
constexpr int kSortWaves = kSortBlock / kWave;
constexpr int kMaxBits = 9, kMaxDigits = 1 << kMaxBits;
constexpr int kSmall = 8192;  // tokens that are placed by counting, all keys in LDS
constexpr int kFillBlocks = 2048;  // workgroups that store zeros beside a launch's own, at most

// The sort key of an id: ids outside the table come last and take no part.
__device__ __forceinline__ uint32_t key_of(int id, uint32_t V)
{
    return uint32_t(id) < V ? uint32_t(id) : V;
}

// A launch's share of the zeros of dW (p = NULL: none), which the workgroups from `first` on store.
struct Zeros {
    float* p;
    int64_t count;
};
__device__ __forceinline__ void store_zeros(const Zeros& z, int64_t first)
{
    // whole pieces from the first 16-byte border on
    const int64_t head0 = (16 - (reinterpret_cast<uintptr_t>(z.p) & 15)) / 4 & 3;
    const int64_t head = head0 < z.count ? head0 : z.count;
    const int64_t body = (z.count - head) / 4 * 4;
    const int64_t step = (int64_t(gridDim.x) - first) * blockDim.x * 4;
    float4* p = reinterpret_cast<float4*>(z.p + head);
    for (int64_t i = ((int64_t(blockIdx.x) - first) * blockDim.x + threadIdx.x) * 4; i < body; i += step)
        p[i / 4] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (int64_t(blockIdx.x) == first) {
        if (threadIdx.x < head) z.p[threadIdx.x] = 0.f;
        if (threadIdx.x < z.count - head - body) z.p[head + body + threadIdx.x] = 0.f;
    }
}

// The stable ranks of one digit among a workgroup's 1024 tokens.  A wavefront finds the
// lanes that share a lane's digit bit by bit; its first of them counts for all.
// counts [wavefronts, digits] must be zero; it is left with the tokens of each digit before
// each wavefront's, and the digit's total in totals.
__device__ __forceinline__ uint32_t rank_in_block(uint32_t digit, int bits, bool live,
                                                  uint16_t (*counts)[kMaxDigits], uint32_t* totals)
{
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    uint64_t same = __ballot(live);
    for (int i = 0; i < bits; ++i) {
        const uint64_t ones = __ballot(digit >> i & 1);
        same &= digit >> i & 1 ? ones : ~ones;
    }
    const uint32_t before = __popcll(same & ((uint64_t(1) << lane) - 1));
    if (live && before == 0) counts[wave][digit] = uint16_t(__popcll(same));
    __syncthreads();
    for (int d = threadIdx.x; d < 1 << bits; d += kSortBlock) {
        uint32_t n = 0;
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = counts[w][d];
            counts[w][d] = uint16_t(n);
            n += c;
        }
        totals[d] = n;
    }
    __syncthreads();
    return before + (live ? counts[wave][digit] : 0);
}

// Exclusive sums of up to kMaxDigits values, in place, by the first wavefront.
__device__ __forceinline__ void exclusive_sum(uint32_t* v, int n)
{
    if (threadIdx.x < kWave) {
        const int lane = threadIdx.x;
        uint32_t base = 0;
        for (int i = 0; i < n; i += kWave) {
            const uint32_t x = i + lane < n ? v[i + lane] : 0;
            uint32_t s = x;
            for (int o = 1; o < kWave; o *= 2) {
                const uint32_t y = __shfl_up(s, o, kWave);
                if (lane >= o) s += y;
            }
            if (i + lane < n) v[i + lane] = base + s - x;
            base += __shfl(s, kWave - 1, kWave);
        }
    }
    __syncthreads();
}

__device__ __forceinline__ void clear_counts(uint16_t (*counts)[kMaxDigits])
{
    uint32_t* p = reinterpret_cast<uint32_t*>(counts);
    for (int i = threadIdx.x; i < kSortWaves * kMaxDigits / 2; i += kSortBlock) p[i] = 0;
    __syncthreads();
}

// Few tokens in one launch: a token's place is the number of tokens that come before it, those of
// lower keys and those of its own at lower positions.  Each wavefront counts for two tokens, over
// all keys in LDS: a compare with a scalar and a count of its bits, 64 keys at a time.
constexpr int kRankEach = 2, kRankTokens = kSortWaves * kRankEach;

__global__ __launch_bounds__(kSortBlock) void rank_kernel(const int* __restrict__ ids, int n, uint32_t V,
                                                          uint32_t* __restrict__ keys, uint32_t* __restrict__ rows,
                                                          Zeros zeros)
{
    const int own = (n + kRankTokens - 1) / kRankTokens;
    if (int(blockIdx.x) >= own) {
        store_zeros(zeros, own);
        return;
    }
    __shared__ __align__(16) uint32_t key[kSmall];
    constexpr int kChunk = kWave * 4;  // keys of a wavefront's load
    const int chunks = (n + kChunk - 1) / kChunk;
    for (int i = threadIdx.x; i < chunks * kChunk; i += kSortBlock) key[i] = i < n ? key_of(ids[i], V) : ~0u;
    __syncthreads();
    const int lane = threadIdx.x % kWave;
    const int i0 = blockIdx.x * kRankTokens + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) * kRankEach;
    if (i0 >= n) return;
    uint32_t mine[kRankEach], place[kRankEach] = {};
#pragma unroll
    for (int t = 0; t < kRankEach; ++t) mine[t] = __builtin_amdgcn_readfirstlane(int(key[i0 + t < n ? i0 + t : n - 1]));
    // (the two tokens lie in one chunk: equal keys count in the chunks before it, not in those after)
    const int home = i0 / kChunk;
    for (int c = 0; c < chunks; ++c) {
        const uint4 k4 = *reinterpret_cast<const uint4*>(key + c * kChunk + lane * 4);
        const uint32_t k[4] = {k4.x, k4.y, k4.z, k4.w};
        if (c == home) {
#pragma unroll
            for (int t = 0; t < kRankEach; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    place[t] += __popcll(__ballot(k[e] < mine[t] + (c * kChunk + lane * 4 + e < i0 + t ? 1 : 0)));
        } else {
#pragma unroll
            for (int t = 0; t < kRankEach; ++t) {
                const uint32_t below = mine[t] + (c < home ? 1 : 0);
#pragma unroll
                for (int e = 0; e < 4; ++e) place[t] += __popcll(__ballot(k[e] < below));
            }
        }
    }
#pragma unroll
    for (int t = 0; t < kRankEach; ++t)
        if (lane == t && i0 + t < n) {
            keys[place[t]] = mine[t];
            rows[place[t]] = i0 + t;
        }
}

// Tokens of each value of a digit in each tile: counts [tiles, digits].  FIRST: the keys are the
// ids.  (Counting the next digit where the one before is placed, by atomics on the tiles' counts,
// takes 8 us more than this launch: a few values are most of them.)
template <bool FIRST>
__global__ __launch_bounds__(kSortBlock) void sort_count_kernel(
    const uint32_t* __restrict__ keys, int64_t n, uint32_t V, int shift, int bits, int64_t tile,
    int64_t tiles, uint32_t* __restrict__ counts, Zeros zeros)
{
    if (int64_t(blockIdx.x) >= tiles) {
        store_zeros(zeros, tiles);
        return;
    }
    __shared__ uint32_t total[kMaxDigits];
    const uint32_t mask = (1u << bits) - 1;
    for (int d = threadIdx.x; d <= int(mask); d += kSortBlock) total[d] = 0;
    __syncthreads();
    const int64_t i0 = blockIdx.x * tile, i1 = i0 + tile < n ? i0 + tile : n;
    for (int64_t i = i0 + threadIdx.x; i < i1; i += kSortBlock) {
        const uint32_t k = FIRST ? key_of(int(keys[i]), V) : keys[i];
        atomicAdd(&total[k >> shift & mask], 1u);
    }
    __syncthreads();
    for (int d = threadIdx.x; d <= int(mask); d += kSortBlock)
        counts[blockIdx.x * int64_t(mask + 1) + d] = total[d];
}

// Places the tokens by one digit (FIRST: of the ids themselves).
template <bool FIRST>
__global__ __launch_bounds__(kSortBlock) void sort_place_kernel(
    const uint32_t* __restrict__ keys, const uint32_t* __restrict__ rows, int64_t n, uint32_t V,
    int shift, int bits, int64_t tile, int64_t tiles, const uint32_t* __restrict__ counts,
    uint32_t* __restrict__ keys_out, uint32_t* __restrict__ rows_out, Zeros zeros)
{
    if (int64_t(blockIdx.x) >= tiles) {
        store_zeros(zeros, tiles);
        return;
    }
    __shared__ uint16_t in_wave[kSortWaves][kMaxDigits];
    __shared__ uint32_t totals[kMaxDigits], first[kMaxDigits], mine[kMaxDigits];
    const uint32_t mask = (1u << bits) - 1;
    // a digit's first place in this tile: all tokens of lower digits, and its own in tiles before;
    // as many threads to a digit as there are
    for (int d = threadIdx.x; d <= int(mask); d += kSortBlock) first[d] = mine[d] = 0;
    __syncthreads();
    const int d0 = threadIdx.x & int(mask), parts = kSortBlock >> bits;
    uint32_t all = 0, before = 0;
#pragma unroll 8
    for (int64_t t = threadIdx.x >> bits; t < tiles; t += parts) {
        const uint32_t c = counts[t * (mask + 1) + d0];
        before += t < int64_t(blockIdx.x) ? c : 0;
        all += c;
    }
    atomicAdd(&first[d0], all);
    atomicAdd(&mine[d0], before);
    __syncthreads();
    exclusive_sum(first, int(mask) + 1);
    for (int d = threadIdx.x; d <= int(mask); d += kSortBlock) first[d] += mine[d];
    const int64_t i1 = int64_t(blockIdx.x + 1) * tile < n ? int64_t(blockIdx.x + 1) * tile : n;
    for (int64_t i0 = blockIdx.x * tile; i0 < i1; i0 += kSortBlock) {
        const int64_t i = i0 + threadIdx.x;
        const bool live = i < i1;
        clear_counts(in_wave);
        uint32_t x = live ? keys[i] : 0;
        if (FIRST) x = key_of(int(x), V);
        const uint32_t d = x >> shift & mask;
        const uint32_t rank = rank_in_block(d, bits, live, in_wave, totals);
        if (live) {
            const uint32_t to = first[d] + rank;
            keys_out[to] = x;
            rows_out[to] = FIRST ? uint32_t(i) : rows[i];
        }
        __syncthreads();
        for (int j = threadIdx.x; j <= int(mask); j += kSortBlock) first[j] += totals[j];
        __syncthreads();
    }
}

constexpr int kSumBlock = 256;

// V sums to p, in pieces of 16 bytes.
template <int V>
__device__ __forceinline__ void put_sums(float* p, const float (&v)[V])
{
    if constexpr (V == 1) {
        *p = v[0];
    } else {
#pragma unroll
        for (int i = 0; i < V / 4; ++i) {
            const float x[4] = {v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
            put<4>(p + 4 * i, x);
        }
    }
}

// A window's tokens, run by run.  part [windows, 2, D]: the sum of the run that entered the
// window (0) and of the one that leaves it and began in it (1).
template <typename T, int V>
__global__ __launch_bounds__(kSumBlock) void runs_kernel(
    const T* __restrict__ dy, const uint32_t* __restrict__ keys, const uint32_t* __restrict__ rows,
    int64_t n, uint32_t rows_of_table, int64_t D, int window, float scale, bool accumulate,
    float* __restrict__ dW, float* __restrict__ part)
{
    const int64_t blocks = (D + kSumBlock * V - 1) / (kSumBlock * V);
    const int64_t w = blockIdx.x / blocks;
    // (A piece that would pass the row's end starts before it, one past it repeats the last: lanes
    // store the same bits to the same place, but where they add to what is there, which only the
    // lane that owns a value may.  No lane ends early: the window's ids lie in all of them.)
    const int64_t c0 = (blockIdx.x % blocks * kSumBlock + threadIdx.x) * V;
    const int64_t c = c0 + V <= D ? c0 : D - V;
    const int twice = int(c0 - c < V ? c0 - c : V);
    const int64_t p0 = w * window, p1 = p0 + window < n ? p0 + window : n;
    // The window's ids and rows lie in the lanes of each wavefront (a window is 64 tokens or
    // fewer): loaded one by one as scalars, each would be waited for before the next is asked for.
    // The tokens that take part come first; where runs end is a bit for each token.
    const int lane = threadIdx.x % kWave, tokens = int(p1 - p0);
    const int64_t mine = lane < tokens ? p0 + lane : p1 - 1;
    const uint32_t my_key = keys[mine], my_row = rows[mine];
    const uint32_t entered = p0 > 0 ? keys[p0 - 1] : ~0u, leaves = p1 < n ? keys[p1] : ~0u;
    const int valid = __popcll(__ballot(lane < tokens && my_key < rows_of_table));
    if (valid == 0) return;
    const uint32_t next_key = __shfl_down(my_key, 1, kWave);
    const uint64_t ends = __ballot(lane < valid && (lane + 1 == valid || next_key != my_key));
    bool in_run = uint32_t(__builtin_amdgcn_readlane(int(my_key), 0)) == entered;  // of a token before the window
    float acc[V] = {};
    auto close = [&](int q) {  // the run that ends with token q
        const uint32_t key = uint32_t(__builtin_amdgcn_readlane(int(my_key), q));
        const bool leaving = q + 1 == tokens && key == leaves, partial = in_run || leaving;
        float* out = partial ? part + (w * 2 + (in_run ? 0 : 1)) * D + c : dW + int64_t(key) * D + c;
        const float factor = partial ? 1.f : scale;
        if (accumulate && !partial) {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (j >= twice) out[j] += acc[j] * factor;
        } else {
            float sum[V];
#pragma unroll
            for (int j = 0; j < V; ++j) sum[j] = acc[j] * factor;
            put_sums<V>(out, sum);
        }
        in_run = false;
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = 0.f;
    };
    // the rows of the next tokens are in flight while those before are added
    constexpr int kAhead = 8;
    Raw<T, V> raw[kAhead];
    auto load = [&](int q) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const uint32_t row = uint32_t(__builtin_amdgcn_readlane(int(my_row), q + i < valid ? q + i : valid - 1));
            raw[i] = load_raw<V>(dy + int64_t(row) * D + c);
        }
    };
    load(0);
    for (int q = 0; q < valid; q += kAhead) {
        float v[kAhead][V];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            expand<V, T>(raw[i], v[i]);
            // (waited for here: past a store, a wait for them would be one for the store too)
#pragma unroll
            for (int j = 0; j < V; ++j) asm volatile("" : "+v"(v[i][j]));
        }
        if (q + kAhead < valid) load(q + kAhead);
        const uint32_t here = uint32_t(ends >> q) & ((1u << kAhead) - 1);
        if (here == 0) {  // in the middle of a run
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) acc[j] += v[i][j];
        } else {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (q + i >= valid) return;
#pragma unroll
                for (int j = 0; j < V; ++j) acc[j] += v[i][j];
                if (here >> i & 1) close(q + i);
            }
        }
    }
}

// Runs that cross windows, each by the workgroups of the window that it begins in.  The lanes
// count the windows that it reaches (their first tokens are of the run), and four wavefronts
// to the same columns take them in turn: the longest run of a batch is one of many windows.
constexpr int kJoinParts = 4;

template <int V>
__global__ __launch_bounds__(kSumBlock * kJoinParts) void joins_kernel(
    const uint32_t* __restrict__ keys, int64_t n, uint32_t rows_of_table, int64_t D, int window,
    float scale, bool accumulate, float* __restrict__ dW, const float* __restrict__ part)
{
    __shared__ float red[kJoinParts - 1][V][kSumBlock];
    const int64_t blocks = (D + kSumBlock * V - 1) / (kSumBlock * V);
    const int64_t w = blockIdx.x / blocks;
    const int column = threadIdx.x % kSumBlock, turn = threadIdx.x / kSumBlock, lane = threadIdx.x % kWave;
    const int64_t p0 = w * window, p1 = p0 + window;
    if (p1 >= n) return;
    const uint32_t key = keys[p1 - 1];
    if (key >= rows_of_table || keys[p1] != key) return;           // nothing leaves
    if (keys[p0] == key && p0 > 0 && keys[p0 - 1] == key) return;  // it began before
    const int64_t c0 = (blockIdx.x % blocks * kSumBlock + column) * V;
    const int64_t c = c0 + V <= D ? c0 : D - V;
    auto get = [&](int64_t slot, float(&v)[V]) { expand<V, float>(load_raw<V>(part + slot * D + c), v); };
    const int64_t windows = (n + window - 1) / window;
    int64_t end = w + 1;
    for (uint64_t more = ~uint64_t(0); more == ~uint64_t(0);) {
        more = __ballot(end + lane < windows && keys[(end + lane) * window] == key);
        end += more == ~uint64_t(0) ? kWave : __builtin_ctzll(~more);
    }
    float acc[V] = {};
    if (turn == 0) get(w * 2 + 1, acc);
    constexpr int kAhead = 8;
    for (int64_t j = w + 1 + turn; j < end; j += kJoinParts * kAhead) {
        float v[kAhead][V];
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            get((j + i * kJoinParts < end ? j + i * kJoinParts : j) * 2, v[i]);
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (j + i * kJoinParts < end) {
#pragma unroll
                for (int l = 0; l < V; ++l) acc[l] += v[i][l];
            }
    }
    if (turn > 0) {
#pragma unroll
        for (int l = 0; l < V; ++l) red[turn - 1][l][column] = acc[l];
    }
    __syncthreads();
    if (turn > 0 || c0 >= D) return;
#pragma unroll
    for (int l = 0; l < V; ++l) {
        for (int i = 0; i < kJoinParts - 1; ++i) acc[l] += red[i][l][column];
        acc[l] *= scale;
    }
    float* out = dW + int64_t(key) * D + c;
    if (accumulate) {
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (k >= int(c0 - c)) out[k] += acc[k];
    } else {
        put_sums<V>(out, acc);
    }
}

size_t aligned(size_t n) { return (n + 255) / 256 * 256; }

template <typename T>
hipError_t launch_runs(const T* dy, const uint32_t* keys, const uint32_t* rows, int64_t n, int64_t V,
                       int64_t D, const EmbedGradPlan& p, float scale, bool accumulate, float* dW,
                       float* part, hipStream_t stream)
{
    auto launch = [&](auto wide) {
        constexpr int v = decltype(wide)::value;
        const int64_t blocks = p.windows * ((D + kSumBlock * v - 1) / (kSumBlock * v));
        hipLaunchKernelGGL((runs_kernel<T, v>), dim3(uint32_t(blocks)), dim3(kSumBlock), 0, stream, dy, keys, rows, n,
                           uint32_t(V), D, int(p.window), scale, accumulate, dW, part);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        hipLaunchKernelGGL((joins_kernel<v>), dim3(uint32_t(blocks)), dim3(kSumBlock * kJoinParts), 0, stream, keys, n, uint32_t(V),
                           D, int(p.window), scale, accumulate, dW, part);
        return hipGetLastError();
    };
    if (D < 4) return launch(std::integral_constant<int, 1>());
    return launch(std::integral_constant<int, 4>());
}

}  // namespace

EmbedGradPlan embed_grad_plan(int64_t n, int64_t V, int64_t D)
{
    EmbedGradPlan p{};
    // 64 tokens, one to a lane; of few tokens 16, so that more workgroups share them.  The number of
    // tokens alone decides: 8193 to 16384 of them, up to 1024 columns wide, are fewer workgroups than
    // CUs.  (65536 tokens x 2048: runs and joins 124 + 13 us with windows of 64, 120 + 27 with 32,
    // 120 + 46 with 16)
    p.window = n <= 8192 ? 16 : kWave;
    p.windows = (n + p.window - 1) / p.window;
    int bits = 1;  // of the keys 0 .. V
    while (V >> bits) ++bits;
    p.passes = (bits + kMaxBits - 1) / kMaxBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    if (n > kSmall) {
        // at most 128 tiles, over whose counts every tile sums
        p.tile = ((n + 127) / 128 + kSortBlock - 1) / kSortBlock * kSortBlock;
        p.tiles = (n + p.tile - 1) / p.tile;
    }
    size_t at = 0;
    for (int i = 0; i < 2; ++i) {
        p.off_keys[i] = at, at += aligned(4 * size_t(n));
        p.off_rows[i] = at, at += aligned(4 * size_t(n));
    }
    p.off_counts = at, at += aligned(4 * size_t(p.tiles) << p.bits);
    p.off_part = at, at += 8 * size_t(p.windows) * D;
    p.ws_bytes = n > 0 ? at : 0;
    return p;
}

int64_t embed_grad_threads(int64_t n, int64_t V, int64_t D)
{
    const EmbedGradPlan p = embed_grad_plan(n, V, D);
    const int64_t columns = kSumBlock * (D < 4 ? 1 : 4);
    const int64_t sum = p.windows * ((D + columns - 1) / columns) * kSumBlock * kJoinParts;
    const int64_t sort = (p.tiles + kSmall / kRankTokens + kFillBlocks) * kSortBlock;
    return sum > sort ? sum : sort;
}

hipError_t launch_embed_grad(const void* dy, const int32_t* ids, int64_t n, int64_t V, int64_t D,
                             bool bf16_io, float scale, bool accumulate, float* dW, void* workspace,
                             hipStream_t stream)
{
    const EmbedGradPlan p = embed_grad_plan(n, V, D);
    char* ws = static_cast<char*>(workspace);
    uint32_t* keys[2] = {reinterpret_cast<uint32_t*>(ws + p.off_keys[0]), reinterpret_cast<uint32_t*>(ws + p.off_keys[1])};
    uint32_t* rows[2] = {reinterpret_cast<uint32_t*>(ws + p.off_rows[0]), reinterpret_cast<uint32_t*>(ws + p.off_rows[1])};
    float* part = reinterpret_cast<float*>(ws + p.off_part);
    hipError_t e;
    int at = 0;  // where the sorted tokens are
    // each sorting launch's share of the zeros, 16 KiB to a workgroup at least
    const int launches = p.tiles > 0 ? 2 * p.passes : 1;
    int launch = 0;
    auto share = [&] {
        const int64_t all = accumulate ? 0 : V * D, i = launch++;
        const int64_t from = all / launches * i, to = i + 1 < launches ? all / launches * (i + 1) : all;
        return Zeros{dW + from, to - from};
    };
    auto grid = [](int64_t sorting, const Zeros& z) {
        const int64_t n = (z.count + 4095) / 4096;
        return dim3(uint32_t(sorting + (n < kFillBlocks ? n : kFillBlocks)));
    };
    const dim3 block(kSortBlock);
    if (p.tiles == 0) {
        const Zeros z = share();
        if (n == 0 && z.count == 0) return hipSuccess;
        hipLaunchKernelGGL(rank_kernel, grid((n + kRankTokens - 1) / kRankTokens, z), block, 0, stream, ids, int(n),
                           uint32_t(V), keys[0], rows[0], z);
        if ((e = hipGetLastError()) != hipSuccess || n == 0) return e;
    } else {
        uint32_t* counts = reinterpret_cast<uint32_t*>(ws + p.off_counts);
        for (int i = 0; i < p.passes; ++i) {
            const int to = i & 1, shift = i * p.bits;
            const Zeros z0 = share(), z1 = share();
            if (i == 0) {
                const uint32_t* in = reinterpret_cast<const uint32_t*>(ids);
                hipLaunchKernelGGL((sort_count_kernel<true>), grid(p.tiles, z0), block, 0, stream, in, n, uint32_t(V),
                                   shift, p.bits, p.tile, p.tiles, counts, z0);
                if ((e = hipGetLastError()) != hipSuccess) return e;
                hipLaunchKernelGGL((sort_place_kernel<true>), grid(p.tiles, z1), block, 0, stream, in,
                                   static_cast<const uint32_t*>(nullptr), n, uint32_t(V), shift, p.bits, p.tile,
                                   p.tiles, counts, keys[to], rows[to], z1);
            } else {
                hipLaunchKernelGGL((sort_count_kernel<false>), grid(p.tiles, z0), block, 0, stream, keys[at], n,
                                   uint32_t(V), shift, p.bits, p.tile, p.tiles, counts, z0);
                if ((e = hipGetLastError()) != hipSuccess) return e;
                hipLaunchKernelGGL((sort_place_kernel<false>), grid(p.tiles, z1), block, 0, stream, keys[at], rows[at],
                                   n, uint32_t(V), shift, p.bits, p.tile, p.tiles, counts, keys[to], rows[to], z1);
            }
            if ((e = hipGetLastError()) != hipSuccess) return e;
            at = to;
        }
    }
    return bf16_io ? launch_runs(static_cast<const bf16*>(dy), keys[at], rows[at], n, V, D, p, scale, accumulate,
                                 dW, part, stream)
                   : launch_runs(static_cast<const float*>(dy), keys[at], rows[at], n, V, D, p, scale, accumulate,
                                 dW, part, stream);
}

}  // namespace lh
