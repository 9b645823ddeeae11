// hsadmm_embedding / hsadmm_embedding_gradient / hsadmm_dropout: what a language model's tokens pass on their way into the network.
// Part of the single translation unit built from hsadmm.hip (included there, in order).
#ifndef KERNELS_TOKENS_HPP
#define KERNELS_TOKENS_HPP
#include "hsadmm_device.hpp"
#include "kernels_training.hpp"
#include "kernels_loss.hpp"

namespace {

// ------------------------------------------------------------------ embedding

// out[i] = scale W[id_i], zeros for an id outside [0, V).  `lanes` threads (a power of two) share a row.  Bound by HBM: 32768 tokens x
// 2048, bf16, 262 MB in 50 us (5.3 TB/s; tokens that are named often come from the caches).
template <int T>
__global__ __launch_bounds__(kBlock) void embedding_rows(const typename ElemOf<T>::type* __restrict__ W, int32_t V, int cols,
                                                         const void* __restrict__ ids, int wide, int64_t n, float scale,
                                                         typename ElemOf<T>::type* __restrict__ out, int64_t ld, int lanes)
{
    typedef typename ElemOf<T>::type E;
    constexpr int m = Wide<T>::n;
    const int each = kBlock / lanes;
    for (int64_t i = (int64_t)blockIdx.x * each + threadIdx.x / lanes; i < n; i += (int64_t)gridDim.x * each) {
        const int64_t id = index_at(ids, wide != 0, i);
        const bool has = id >= 0 && id < V;
        const E* from = W + (has ? id * cols : 0);
        for (int c = (threadIdx.x & (lanes - 1)) * m; c < cols; c += lanes * m) {
            typename Wide<T>::vec x = {};
            if (has) {
                x = load_piece<T>(from + c, cols - c);
#pragma unroll
                for (int e = 0; e < m; ++e) x[e] = (E)((float)x[e] * scale);
            }
            store_piece<T>(out + i * ld + c, x, cols - c);
        }
    }
}

// ------------------------------------------------------------------ tokens in order

// Positions sorted by their token, tokens that are equal in the order of their positions: radix sort from the lowest digit, of up to
// kDigitBits bits each.  Ids outside [0, V) become V and so come last.  A workgroup takes a tile of positions, a wave of it adjacent
// ones, kSortAtOnce for each lane at a time, whose loads are in flight together; lanes with equal digits find each other by ballots, so places depend on the ids alone.
typedef float v4f_at2 __attribute__((ext_vector_type(4), aligned(2)));
constexpr int kDigitBits = 9;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kSortAtOnce = 8;
constexpr int kSortMost = 4096;         // positions that one workgroup sorts in one launch; more: tiles of kSortTile or, of more
constexpr int kSortTile = 2048;         // than kSortTiles of them, of as many powers of two as make that many
constexpr int kSortTiles = 64;

// Rows without a token become zero while the tokens are sorted, which keeps a few compute units busy: each launch of the sort clears a
// part of the rows with workgroups of its own.  (Rows that a workgroup each looks up in the sorted list, and writes
// zeros to: 195 us for 131072 x 2048 in bf16, where the list names 11000, after a sort of 49; so 111 together with the sort, 4.8 TB/s.)
struct Clear {
    char* rows;
    int64_t pieces;             // of 16 bytes
    int rest;                   // bytes behind them
    int turns;                  // launches
};

// The share of the `which`-th of `of` workgroups in a launch.
__device__ void clear_rows(const Clear& a, int turn, int which, int of)
{
    const int64_t from = a.pieces * turn / a.turns, to = a.pieces * (turn + 1) / a.turns;
    for (int64_t i = from + (int64_t)which * blockDim.x + threadIdx.x; i < to; i += (int64_t)of * blockDim.x)
        *reinterpret_cast<v4f_at2*>(a.rows + 16 * i) = v4f_at2{0.f, 0.f, 0.f, 0.f};
    if (turn == a.turns - 1 && which == 0 && (int)threadIdx.x * 2 < a.rest)
        reinterpret_cast<uint16_t*>(a.rows + 16 * a.pieces)[threadIdx.x] = 0;
}

struct SortArgs {
    const void* ids;
    int wide;
    int32_t n, V;
    int32_t* key[2];
    int32_t* pos[2];
    uint32_t* counts;           // [digit][tile], several tiles only
    int tile, tiles;
    int bits, passes;
    Clear clear;
};

// The lanes (of those that are active) with this lane's digit: for each bit those that agree in it.
__device__ __forceinline__ unsigned long long same_digit(int digit, int bits, bool active)
{
    const unsigned long long all = __ballot(active);
    uint32_t lo = (uint32_t)all, hi = (uint32_t)(all >> 32);
    for (int b = 0; b < bits; ++b) {
        const unsigned long long set = __ballot((digit >> b) & 1);
        const uint32_t own = (uint32_t)-((digit >> b) & 1);
        lo &= ~((uint32_t)set ^ own);
        hi &= ~((uint32_t)(set >> 32) ^ own);
    }
    return (unsigned long long)hi << 32 | lo;
}

__device__ __forceinline__ int32_t sort_key(const SortArgs& a, int pass, int64_t i)
{
    if (pass > 0) return a.key[(pass - 1) & 1][i];
    const int64_t id = index_at(a.ids, a.wide != 0, i);
    return id >= 0 && id < a.V ? (int32_t)id : a.V;
}

struct SortShared {
    uint32_t count[kScanWaves][kDigits];
    uint32_t sums[kScanWaves];
};

// A wave's part of a tile.
struct SortPart {
    int64_t from, to;
    __device__ __forceinline__ SortPart(const SortArgs& a, int tile)
    {
        const int64_t begin = (int64_t)tile * a.tile, end = min((int64_t)a.n, begin + a.tile);
        const int each = (int)((end - begin + kScanBlock - 1) / kScanBlock) * kWave;
        from = begin + (int64_t)(threadIdx.x / kWave) * each;
        to = min(end, from + each);
    }
};

// Counts the digits of a tile, wave by wave.
__device__ void sort_count(const SortArgs& a, int pass, int tile, SortShared& s)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, shift = pass * a.bits, mask = (1 << a.bits) - 1;
    for (int d = lane; d < kDigits; d += kWave) s.count[wave][d] = 0;
    __syncthreads();
    const SortPart part(a, tile);
    for (int64_t i0 = part.from + lane; i0 - lane < part.to; i0 += kSortAtOnce * kWave) {
        int32_t key[kSortAtOnce];
#pragma unroll
        for (int u = 0; u < kSortAtOnce; ++u) key[u] = i0 + u * kWave < part.to ? sort_key(a, pass, i0 + u * kWave) : 0;
#pragma unroll
        for (int u = 0; u < kSortAtOnce; ++u) {
            if (i0 + u * kWave < part.to) atomicAdd(&s.count[wave][(key[u] >> shift) & mask], 1u);
        }
    }
    __syncthreads();
}

// Moves a tile's positions to their places.  s.count: where each wave's next of a digit goes.
__device__ void sort_move(const SortArgs& a, int pass, int tile, SortShared& s)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, shift = pass * a.bits, mask = (1 << a.bits) - 1;
    const SortPart part(a, tile);
    for (int64_t i0 = part.from + lane; i0 - lane < part.to; i0 += kSortAtOnce * kWave) {
        int32_t key[kSortAtOnce], pos[kSortAtOnce];
        uint32_t at[kSortAtOnce], behind[kSortAtOnce];
        int first[kSortAtOnce];
#pragma unroll
        for (int u = 0; u < kSortAtOnce; ++u) {
            const int64_t i = i0 + u * kWave;
            key[u] = i < part.to ? sort_key(a, pass, i) : 0;
            pos[u] = i < part.to && pass > 0 ? a.pos[(pass - 1) & 1][i] : (int32_t)i;
        }
#pragma unroll
        for (int u = 0; u < kSortAtOnce; ++u) {
            const bool active = i0 + u * kWave < part.to;
            const int d = (key[u] >> shift) & mask;
            const unsigned long long same = same_digit(d, a.bits, active);
            first[u] = active ? __ffsll((long long)same) - 1 : lane;
            behind[u] = (uint32_t)__popcll(same & ((1ull << lane) - 1));
            at[u] = 0;
            if (active && first[u] == lane) at[u] = atomicAdd(&s.count[wave][d], (uint32_t)__popcll(same));
        }
#pragma unroll
        for (int u = 0; u < kSortAtOnce; ++u) {
            const uint32_t to = __shfl(at[u], first[u], kWave) + behind[u];
            if (i0 + u * kWave < part.to) {
                a.key[pass & 1][to] = key[u];
                a.pos[pass & 1][to] = pos[u];
            }
        }
    }
    __syncthreads();
}

// s.count from counts to places: behind the digits below, then the waves before.  `start`: the tile's places of its digits, or null
// (a single tile).
__device__ void sort_places(SortShared& s, const uint32_t* start, int stride)
{
    const int d = threadIdx.x, lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    uint32_t own[kScanWaves], all = 0;
    const uint32_t begin = start && d < kDigits ? start[(int64_t)d * stride] : 0;
#pragma unroll
    for (int w = 0; w < kScanWaves; ++w) {
        own[w] = d < kDigits ? s.count[w][d] : 0;
        all += own[w];
    }
    uint32_t at = begin;
    if (!start) {
        uint32_t upto = all;
        for (int o = 1; o < kWave; o <<= 1) {
            const uint32_t x = __shfl_up(upto, o, kWave);
            if (lane >= o) upto += x;
        }
        if (lane == kWave - 1) s.sums[wave] = upto;
        __syncthreads();
        at = upto - all;
        for (int w = 0; w < wave; ++w) at += s.sums[w];
    }
    if (d < kDigits)
#pragma unroll
        for (int w = 0; w < kScanWaves; ++w) {
            s.count[w][d] = at;
            at += own[w];
        }
    __syncthreads();
}

// A single tile: all passes in one workgroup, the first.  Positions and their tokens stay in registers and pass through LDS from digit
// to digit (through memory: 18.6 us for 777 positions and two digits, so 13.6 with the clearing of 80 MB beside it).
struct SortedTile {
    int32_t key[kSortMost];
    uint16_t pos[kSortMost];
};

__global__ __launch_bounds__(kScanBlock) void token_sort(SortArgs a)
{
    __shared__ SortShared s;
    __shared__ SortedTile moved;
    if (blockIdx.x > 0) return clear_rows(a.clear, 0, blockIdx.x - 1, gridDim.x - 1);
    constexpr int kOwn = kSortMost / kScanBlock;
    static_assert(kSortMost <= 1 << 16, "positions of 16 bits");
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, mask = (1 << a.bits) - 1;
    const SortPart part(a, 0);
    int32_t key[kOwn];
    uint32_t pos[kOwn];
    bool active[kOwn];
#pragma unroll
    for (int u = 0; u < kOwn; ++u) {
        const int64_t i = part.from + u * kWave + lane;
        active[u] = i < part.to;
        key[u] = active[u] ? sort_key(a, 0, i) : 0;
        pos[u] = (uint32_t)i;
    }
    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = pass * a.bits;
        for (int d = lane; d < kDigits; d += kWave) s.count[wave][d] = 0;
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kOwn; ++u)
            if (active[u]) atomicAdd(&s.count[wave][(key[u] >> shift) & mask], 1u);
        __syncthreads();
        sort_places(s, nullptr, 0);
        const bool last = pass == a.passes - 1;
#pragma unroll
        for (int u = 0; u < kOwn; ++u) {
            const int d = (key[u] >> shift) & mask;
            const unsigned long long same = same_digit(d, a.bits, active[u]);
            const int first = active[u] ? __ffsll((long long)same) - 1 : lane;
            uint32_t at = 0;
            if (active[u] && first == lane) at = atomicAdd(&s.count[wave][d], (uint32_t)__popcll(same));
            at = __shfl(at, first, kWave) + (uint32_t)__popcll(same & ((1ull << lane) - 1));
            if (!active[u]) continue;
            if (last) {
                a.key[pass & 1][at] = key[u];
                a.pos[pass & 1][at] = (int32_t)pos[u];
            } else {
                moved.key[at] = key[u];
                moved.pos[at] = (uint16_t)pos[u];
            }
        }
        if (last) break;
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kOwn; ++u) {
            if (!active[u]) continue;
            const int i = (int)part.from + u * kWave + lane;
            key[u] = moved.key[i];
            pos[u] = moved.pos[i];
        }
        // (the next digit's counts are cleared behind a barrier that all of this has passed)
    }
}

// Several tiles, a pass in three launches: digits of every tile, their places, the move.
__global__ __launch_bounds__(kScanBlock) void token_count(SortArgs a, int pass)
{
    __shared__ SortShared s;
    if ((int)blockIdx.x >= a.tiles) return clear_rows(a.clear, 3 * pass, blockIdx.x - a.tiles, gridDim.x - a.tiles);
    sort_count(a, pass, blockIdx.x, s);
    for (int d = threadIdx.x; d < kDigits; d += kScanBlock) {
        uint32_t all = 0;
        for (int w = 0; w < kScanWaves; ++w) all += s.count[w][d];
        a.counts[(int64_t)d * a.tiles + blockIdx.x] = all;
    }
}

// (a thread takes adjacent counts, all of them at once)
__global__ __launch_bounds__(kScanBlock) void token_scan(SortArgs a, int pass)
{
    if (blockIdx.x > 0) return clear_rows(a.clear, 3 * pass + 1, blockIdx.x - 1, gridDim.x - 1);
    uint32_t* counts = a.counts;
    const int n = a.tiles << a.bits;
    constexpr int kMost = kDigits * kSortTiles / kScanBlock;
    __shared__ uint32_t sums[kScanWaves];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int each = (n + kScanBlock - 1) / kScanBlock, first = threadIdx.x * each;
    uint32_t own[kMost], all = 0;
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        if (i >= each) { own[i] = 0; continue; }        // (the same for all threads)
        const uint32_t c = counts[min(first + i, n - 1)];
        own[i] = first + i < n ? c : 0;
        all += own[i];
    }
    uint32_t upto = all;
    for (int o = 1; o < kWave; o <<= 1) {
        const uint32_t x = __shfl_up(upto, o, kWave);
        if (lane >= o) upto += x;
    }
    if (lane == kWave - 1) sums[wave] = upto;
    __syncthreads();
    uint32_t at = upto - all;
    for (int w = 0; w < wave; ++w) at += sums[w];
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        if (i < each && first + i < n) counts[first + i] = at;
        at += own[i];
    }
}

__global__ __launch_bounds__(kScanBlock) void token_move(SortArgs a, int pass)
{
    __shared__ SortShared s;
    if ((int)blockIdx.x >= a.tiles) return clear_rows(a.clear, 3 * pass + 2, blockIdx.x - a.tiles, gridDim.x - a.tiles);
    sort_count(a, pass, blockIdx.x, s);
    sort_places(s, a.counts + blockIdx.x, a.tiles);
    sort_move(a, pass, blockIdx.x, s);
}

// ------------------------------------------------------------------ gradient of the embedding

// dW[v] = scale times the sum of dY over v's tokens, in the order of their positions; in fp32, rounded once.  (Rows without a token
// are cleared beside the sort.)  A token with more than `part` positions is summed in parts first, those of the sorted list's stretches of `part`: a stretch holds the end of at most one
// such token and the beginning of at most one (or the whole stretch is one's), so it has two rows of sums: [2 b] for the token of its
// first position, [2 b + 1] for another that begins in it.
struct EmbedGradArgs {
    const int32_t* key;
    const int32_t* pos;
    int32_t n, V;
    int part;
    const void* dY;
    int64_t ld;
    int cols;
    float* sums;        // [2 stretches][pitch]
    int64_t pitch;
    void* G;
    float scale;
    int add;
    int shares;         // workgroups that share a stretch's, or some places', columns
};

// First place in the sorted list whose token is at least v, by a whole wave: it looks at 64 places at a time.
__device__ __forceinline__ int lower_bound_wave(const int32_t* __restrict__ key, int n, int32_t v)
{
    const int lane = threadIdx.x & (kWave - 1);
    int lo = 0, hi = n;
    while (lo < hi) {
        const int step = (hi - lo + kWave - 1) / kWave;
        const int64_t at = lo + (int64_t)(lane + 1) * step - 1;        // (the last one is hi - 1 or behind it)
        const int below = __popcll(__ballot(at < hi && key[at < hi ? at : hi - 1] < v));
        const int64_t end = lo + (int64_t)(below + 1) * step - 1;
        lo = (int)min((int64_t)hi, lo + (int64_t)below * step);
        hi = (int)min((int64_t)hi, end);
    }
    return lo;
}

// x += the rows of dY whose numbers are in lanes first to first + n - 1 of pos, K pieces of 16 bytes at the columns c[0 .. K); AT_ONCE
// rows in flight.  (The pieces are whole and all of them are read, also by lanes that have none to write: with a branch every load
// is waited for where it stands.)
template <int T, int K, int AT_ONCE>
__device__ __forceinline__ void add_rows(const EmbedGradArgs& a, int32_t pos, int first, int n, const int (&c)[K], float (&x)[K][Wide<T>::n])
{
    typedef typename ElemOf<T>::type E;
    const E* dY = static_cast<const E*>(a.dY);
    const auto add = [&](auto count, int at) {
        constexpr int kCount = decltype(count)::value;
        typename Wide<T>::vec y[kCount][K];
#pragma unroll
        for (int u = 0; u < kCount; ++u) {
            const E* row = dY + (int64_t)__builtin_amdgcn_readlane(pos, at + u) * a.ld;
#pragma unroll
            for (int k = 0; k < K; ++k) y[u][k] = *reinterpret_cast<const typename Wide<T>::any*>(row + c[k]);
        }
#pragma unroll
        for (int u = 0; u < kCount; ++u)
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int e = 0; e < Wide<T>::n; ++e) x[k][e] += (float)y[u][k][e];
    };
    int u = first;
    const int end = first + n;
    for (; u + AT_ONCE <= end; u += AT_ONCE) add(std::integral_constant<int, AT_ONCE>{}, u);
    if constexpr (AT_ONCE > 4)
        for (; u + 4 <= end; u += 4) add(std::integral_constant<int, 4>{}, u);
    if constexpr (AT_ONCE > 2)
        if (u + 2 <= end) { add(std::integral_constant<int, 2>{}, u); u += 2; }
    if (u < end) add(std::integral_constant<int, 1>{}, u);
}

// Sums over rows that are shorter than a piece: one column of the places [from, to).
template <int T>
__device__ __forceinline__ float add_column(const EmbedGradArgs& a, int from, int to, int c)
{
    float x = 0.f;
    for (int t = from; t < to; ++t) x += (float)static_cast<const typename ElemOf<T>::type*>(a.dY)[(int64_t)a.pos[t] * a.ld + c];
    return x;
}

// The stretches' sums.  Rows of at least a piece: a lane whose piece would pass the end of the row takes the row's last one instead
// and forms some columns a second time, from the same terms in the same order.
template <int T>
__global__ __launch_bounds__(kBlock) void embedding_parts(EmbedGradArgs a)
{
    constexpr int m = Wide<T>::n;
    __shared__ int bound[4];
    const int64_t b = blockIdx.x / a.shares;
    const int share = blockIdx.x % a.shares;
    const int from = (int)(b * a.part), to = (int)min((int64_t)a.n, (b + 1) * a.part), wave = threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1);
    // the extent of the tokens of the first and the last position
    {
        const int at = lower_bound_wave(a.key, a.n, a.key[wave < 2 ? from : to - 1] + (wave & 1));
        if (lane == 0) bound[wave] = at;
    }
    __syncthreads();
    const bool first = a.key[from] < a.V && bound[1] - bound[0] > a.part;
    const bool last = a.key[to - 1] < a.V && bound[3] - bound[2] > a.part && bound[2] != bound[0];
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if (!(which ? last : first)) continue;
        const int f = which ? bound[2] : from, t = which ? to : min(to, bound[1]);
        float* sums = a.sums + (2 * b + which) * a.pitch;
        if (a.cols < m) {
            if (share == 0 && (int)threadIdx.x < a.cols) sums[threadIdx.x] = add_column<T>(a, f, t, threadIdx.x);
            continue;
        }
        for (int64_t c0 = ((int64_t)share * kWaves + wave) * kWave * m; c0 < a.cols; c0 += (int64_t)a.shares * kBlock * m) {
            const int64_t at = c0 + lane * m;
            const int c[1] = {(int)min(at, (int64_t)a.cols - m)};
            float x[1][m] = {};
            for (int i = f; i < t; i += kWave) {
                const int n = min(kWave, t - i);
                add_rows<T, 1, 16>(a, a.pos[i + min(lane, n - 1)], 0, n, c, x);
            }
            if (at < a.cols)
#pragma unroll
                for (int e = 0; e < m; ++e) sums[c[0] + e] = x[0][e];
        }
    }
}

// The rows of dW that have tokens.  A wave takes kPlacesOfWave places of the sorted list and the tokens whose positions begin there; it
// has the keys and positions of the 64 places from its first on in its lanes, so most tokens' rows are loaded as soon as those are
// there.  kAcross pieces of 16 bytes a lane of up to four rows are in flight at once.  Bound by latency (keys, first rows, and the
// stretches' sums of a token of many positions, one after the other): 32768 positions x 2048 in bf16, 134 MB read and 45 written, in
// 47 us, behind 27 for the stretches.  Columns not shared among workgroups 54, for 11961 positions x 3854 over 87 rows, fp32, 89 for 15.
constexpr int kPlacesOfWave = 4;
constexpr int kAcross = 2;

template <int T>
__global__ __launch_bounds__(kBlock) void embedding_gradient(EmbedGradArgs a)
{
    typedef typename ElemOf<T>::type E;
    typedef typename Wide<T>::vec V;
    typedef typename Wide<T>::any A;
    constexpr int m = Wide<T>::n;
    const int lane = threadIdx.x & (kWave - 1);
    const int share = blockIdx.x % a.shares;
    const int64_t first = ((int64_t)(blockIdx.x / a.shares) * kWaves + threadIdx.x / kWave) * kPlacesOfWave;
    if (first >= a.n) return;
    const int64_t place = min(first + lane, (int64_t)a.n - 1);
    const int32_t key = first + lane < a.n ? a.key[place] : a.V;       // (behind the last place: no token)
    const int32_t pos = a.pos[place];
    const int32_t ahead = first > 0 ? a.key[first - 1] : -1, up = __shfl_up(key, 1, kWave);
    const int32_t before = lane == 0 ? ahead : up;
    const unsigned long long ends = __ballot(key != before), begins = ends & __ballot(key < a.V);
    for (int i = 0; i < kPlacesOfWave; ++i) {
        if (!((begins >> i) & 1)) continue;
        const int32_t v = __builtin_amdgcn_readlane(key, i);
        const unsigned long long later = i < kWave - 1 ? ends >> (i + 1) : 0;
        // how many positions the token has (all of them among the 64, or to be looked for)
        const int from = (int)first + i;
        const int n = later ? __ffsll((long long)later) : lower_bound_wave(a.key, a.n, v + 1) - from;
        const bool many = n > a.part;
        // a token with many positions: its stretches, of which the first holds it as the second one if it begins inside
        const int64_t b0 = from / a.part, b1 = (from + n - 1) / a.part;
        const int64_t inside = b0 * a.part != from ? 1 : 0;
        E* row = static_cast<E*>(a.G) + (int64_t)v * a.cols;
        if (a.cols < m) {
            if (share == 0 && lane < a.cols) {
                float x = 0.f;
                if (!many) x = add_column<T>(a, from, from + n, lane);
                else
                    for (int64_t b = b0; b <= b1; ++b) x += a.sums[(2 * b + (b == b0 ? inside : 0)) * a.pitch + lane];
                row[lane] = (E)(a.add ? x * a.scale + (float)row[lane] : x * a.scale);
            }
            continue;
        }
        for (int64_t c0 = (int64_t)share * kAcross * kWave * m; c0 < a.cols; c0 += (int64_t)a.shares * kAcross * kWave * m) {
            float x[kAcross][m] = {};
            int c[kAcross];
            bool on[kAcross];
            V g[kAcross];
#pragma unroll
            for (int k = 0; k < kAcross; ++k) {
                const int64_t at = c0 + (k * kWave + lane) * m;
                on[k] = at < a.cols;
                c[k] = (int)min(at, (int64_t)a.cols - m);
            }
            if (a.add)
#pragma unroll
                for (int k = 0; k < kAcross; ++k) g[k] = *reinterpret_cast<const A*>(row + c[k]);
            if (many) {
                constexpr int kAtOnce = 4;
                for (int64_t b = b0; b <= b1; b += kAtOnce) {
                    v4f y[kAtOnce][kAcross][m / 4];
#pragma unroll
                    for (int u = 0; u < kAtOnce; ++u) {
                        const int64_t at = min(b + u, b1);
                        const float* sums = a.sums + (2 * at + (at == b0 ? inside : 0)) * a.pitch;
#pragma unroll
                        for (int k = 0; k < kAcross; ++k)
#pragma unroll
                            for (int e = 0; e < m / 4; ++e) y[u][k][e] = ld4u(sums + c[k] + 4 * e);
                    }
#pragma unroll
                    for (int u = 0; u < kAtOnce; ++u)
                        if (b + u <= b1)
#pragma unroll
                            for (int k = 0; k < kAcross; ++k)
#pragma unroll
                                for (int e = 0; e < m; ++e) x[k][e] += y[u][k][e / 4][e % 4];
                }
            } else if (i + n <= kWave) {
                add_rows<T, kAcross, 4>(a, pos, i, n, c, x);
            } else {
                for (int t = 0; t < n; t += kWave) {
                    const int some = min(kWave, n - t);
                    add_rows<T, kAcross, 4>(a, a.pos[from + t + min(lane, some - 1)], 0, some, c, x);
                }
            }
#pragma unroll
            for (int k = 0; k < kAcross; ++k)
                if (on[k]) {
                    V y;
#pragma unroll
                    for (int e = 0; e < m; ++e) y[e] = (E)(a.add ? x[k][e] * a.scale + (float)g[k][e] : x[k][e] * a.scale);
                    const int skip = (int)(c0 + (k * kWave + lane) * m - c[k]);
                    if (!a.add || skip == 0) {
                        *reinterpret_cast<A*>(row + c[k]) = y;
                    } else {
                        // (columns that another piece adds to as well: their sums may have been written already when g was read)
#pragma unroll
                        for (int e = 1; e < m; ++e)
                            if (e >= skip) row[c[k] + e] = y[e];
                    }
                }
        }
    }
}

// ------------------------------------------------------------------ dropout

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): four words from a counter of four
// and a key of two.
__device__ __forceinline__ void philox(uint64_t group, uint64_t call, uint64_t seed, uint32_t (&w)[4])
{
    uint32_t c0 = (uint32_t)group, c1 = (uint32_t)(group >> 32), c2 = (uint32_t)call, c3 = (uint32_t)(call >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    w[0] = c0; w[1] = c1; w[2] = c2; w[3] = c3;
}

// A thread has a group of eight elements, one counter's numbers.  Bound by HBM: 16384 x 4096 in bf16 with a residual, 403 MB in 68 us
// (5.9 TB/s).
struct DropoutArgs {
    const void* X;
    const void* R;              // residual, or null
    void* Y;
    int64_t ldx, ldr, ldy;
    int64_t n, cols;            // elements, and those of a row
    uint32_t least;             // the smallest 16 bits that keep an element
    float scale;
    uint64_t seed, call;
    const uint64_t* call_dev;   // takes the place of call, or null
};

constexpr int kDropout = 8;     // elements that share a counter

template <int T, bool RES>
__global__ __launch_bounds__(kBlock) void dropout_kernel(DropoutArgs a)
{
    typedef typename ElemOf<T>::type E;
    const int64_t groups = (a.n + kDropout - 1) / kDropout;
    const uint64_t call = a.call_dev ? *a.call_dev : a.call;
    for (int64_t g = (int64_t)blockIdx.x * kBlock + threadIdx.x; g < groups; g += (int64_t)gridDim.x * kBlock) {
        uint32_t w[4];
        philox((uint64_t)g, call, a.seed, w);
        const int64_t i = g * kDropout;
        int64_t row, col;
        if (a.cols == a.n) { row = 0; col = i; }
        else if (a.n <= 0xffffffffll) { row = (uint32_t)i / (uint32_t)a.cols; col = i - row * a.cols; }
        else { row = i / a.cols; col = i - row * a.cols; }
        const E* x = static_cast<const E*>(a.X) + row * a.ldx + col;
        const E* r = RES ? static_cast<const E*>(a.R) + row * a.ldr + col : nullptr;
        E* y = static_cast<E*>(a.Y) + row * a.ldy + col;
        // (what is dropped is zero whatever it held)
        const auto one = [&](int j, float v, float res) {
            const float kept = ((w[j >> 1] >> (16 * (j & 1))) & 0xffffu) >= a.least ? v * a.scale : 0.f;
            return RES ? kept + res : kept;
        };
        if (col + kDropout <= a.cols) {
            // (the group lies in one row, at any element's address)
            constexpr int kPieces = kDropout / Wide<T>::n;
            typedef typename Wide<T>::vec V;
            typedef typename Wide<T>::any A;
            V vx[kPieces], vr[kPieces];
#pragma unroll
            for (int p = 0; p < kPieces; ++p) {
                vx[p] = __builtin_nontemporal_load(reinterpret_cast<const A*>(x) + p);
                if (RES) vr[p] = __builtin_nontemporal_load(reinterpret_cast<const A*>(r) + p);
            }
#pragma unroll
            for (int p = 0; p < kPieces; ++p) {
                V out;
#pragma unroll
                for (int e = 0; e < Wide<T>::n; ++e) out[e] = (E)one(p * Wide<T>::n + e, (float)vx[p][e], RES ? (float)vr[p][e] : 0.f);
                __builtin_nontemporal_store(out, reinterpret_cast<A*>(y) + p);
            }
        } else {
#pragma unroll
            for (int j = 0; j < kDropout; ++j) {
                if (i + j >= a.n) break;
                *y = (E)one(j, (float)*x, RES ? (float)*r : 0.f);
                ++x; ++y;
                if (RES) ++r;
                if (++col == a.cols) {
                    col = 0;
                    x += a.ldx - a.cols;
                    y += a.ldy - a.cols;
                    if (RES) r += a.ldr - a.cols;
                }
            }
        }
    }
}

}  // namespace
#endif
