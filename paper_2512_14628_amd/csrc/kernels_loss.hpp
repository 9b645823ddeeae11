// hsadmm_softmax_loss: softmax cross entropy of a linear layer's products, and its gradients, in pieces of the vocabulary.
// Part of the single translation unit built from hsadmm.hip (included there, in order).
//
// With l = x W^T (N rows that have a target, V classes, D inputs) and y the rows' labels,
//     loss_n = log(sum_v exp(l_nv)) - l_{n,y_n};   P = softmax(l) - onehot(y);   dX = g P W;   dW = g P^T X.
// Three products of 2 N V D operations; the logits are held for one piece of the vocabulary at a time (hsadmm.hip: the pieces), so
// those of all pieces but the last are formed a second time when their gradients are.
#ifndef KERNELS_LOSS_HPP
#define KERNELS_LOSS_HPP
#include "hsadmm_device.hpp"
#include "kernels_training.hpp"
#include "loss_plan.hpp"

namespace {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

typedef __bf16 v8bf_at2 __attribute__((ext_vector_type(8), aligned(2)));      // at any element's address
typedef _Float16 v8h_at2 __attribute__((ext_vector_type(8), aligned(2)));

template <int T> struct Wide { typedef v4f vec; typedef v4f_at4 any; static constexpr int n = 4; };        // 16 bytes of elements
template <> struct Wide<HSADMM_TYPE_BF16> { typedef v8bf vec; typedef v8bf_at2 any; static constexpr int n = 8; };
template <> struct Wide<HSADMM_TYPE_F16> { typedef v8h vec; typedef v8h_at2 any; static constexpr int n = 8; };

// 16 bytes of a row from p on, of which `left` elements belong to the row (zeros behind them).  Rows may start at any element: an
// access of 16 bytes that is aligned to its elements only costs a wave a cache line more.
template <int T>
__device__ __forceinline__ typename Wide<T>::vec load_piece(const typename ElemOf<T>::type* p, int left)
{
    if (left >= Wide<T>::n) return *reinterpret_cast<const typename Wide<T>::any*>(p);
    typename Wide<T>::vec v = {};
#pragma unroll
    for (int i = 0; i < Wide<T>::n; ++i)
        if (i < left) v[i] = p[i];
    return v;
}
template <int T>
__device__ __forceinline__ void store_piece(typename ElemOf<T>::type* p, typename Wide<T>::vec v, int left)
{
    if (left >= Wide<T>::n) {
        *reinterpret_cast<typename Wide<T>::any*>(p) = v;
        return;
    }
#pragma unroll
    for (int i = 0; i < Wide<T>::n; ++i)
        if (i < left) p[i] = v[i];
}

__device__ __forceinline__ int64_t index_at(const void* p, bool wide, int64_t i)
{
    return wide ? static_cast<const int64_t*>(p)[i] : (int64_t)static_cast<const int32_t*>(p)[i];
}

// ------------------------------------------------------------------ rows that have a target

constexpr int kZeroPage = 256;          // bytes of zeros that stand for what lies outside an operand

struct LossHead {
    int32_t count;                      // rows that have a target
    float factor;                       // what gradients are multiplied by
    int32_t pad[62];
    unsigned char zeros[kZeroPage];
};
static_assert(sizeof(LossHead) == kLossHeadBytes, "LossHead layout");

struct LossRows {
    LossHead* head;
    int32_t* row;        // [count] the original row of a held one, ascending
    int32_t* label;      // [count]
    int32_t* place;      // [N] the held row of an original one, or -1
};

// Lists the rows whose label lies in [0, V), in order (one workgroup, four labels a thread at a time), and settles the rows that have
// none.  Bound by the loads' latency: 8192 labels in 7.6 us (10.5 with one label a thread at a time).
__global__ __launch_bounds__(kScanBlock) void loss_targets(const void* __restrict__ labels, int wide, int64_t n, int32_t V, double scale,
                                                           int mean, LossRows r, float* __restrict__ loss, float* __restrict__ lse)
{
    constexpr int kAtOnce = 4;
    __shared__ int32_t sums[2][kAtOnce][kScanWaves];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    int32_t before = 0;
    int turn = 0;
    for (int64_t i0 = 0; i0 < n; i0 += kAtOnce * kScanBlock, turn ^= 1) {
        int64_t y[kAtOnce];
        unsigned long long all[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int64_t i = i0 + u * kScanBlock + threadIdx.x;
            y[u] = i < n ? index_at(labels, wide != 0, i) : -1;
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            all[u] = __ballot(y[u] >= 0 && y[u] < V);
            if (lane == 0) sums[turn][u][wave] = __popcll(all[u]);
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            int32_t at = before;
            for (int w = 0; w < kScanWaves; ++w) {
                const int32_t s = sums[turn][u][w];
                before += s;
                if (w < wave) at += s;
            }
            at += __popcll(all[u] & ((1ull << lane) - 1));
            const int64_t i = i0 + u * kScanBlock + threadIdx.x;
            if (i >= n) continue;
            const bool has = (all[u] >> lane) & 1;
            r.place[i] = has ? at : -1;
            if (has) {
                r.row[at] = (int32_t)i;
                r.label[at] = (int32_t)y[u];
            } else {
                if (loss) loss[i] = 0.f;
                if (lse) lse[i] = 0.f;
            }
        }
    }
    if (threadIdx.x == 0) {
        r.head->count = before;
        r.head->factor = (float)(mean ? scale / (double)max(before, 1) : scale);
    }
    if (threadIdx.x < kZeroPage / 4) reinterpret_cast<float*>(r.head->zeros)[threadIdx.x] = 0.f;
}

// Both for up to kFewLabels rows, in one launch: every workgroup reads all labels, so a row knows its place by itself, and copies it there
// if it has a target.  `lanes` threads (a wave or four) share a row.  Bound by the loads' latency: 32 rows of 64 in 3.6 us, 256 of 2048
// fp32 elements in 4.9, 1537 of 1441 in half precision in 7.0; two launches 2.4 + 2.7, 2.2 + 3.6, 5.1 + 5.1 and 1 to 2 between them.
constexpr int kFewLabels = 2048;
template <int T>
__global__ __launch_bounds__(kBlock) void loss_few(const void* __restrict__ labels, int wide, int n, int32_t V, double scale, int mean,
                                                   LossRows r, float* __restrict__ loss, float* __restrict__ lse,
                                                   const typename ElemOf<T>::type* __restrict__ src, int64_t ld, int cols,
                                                   typename ElemOf<T>::type* __restrict__ dst, int pitch, int lanes)
{
    constexpr int kEach = kFewLabels / kBlock, kWords = kFewLabels / kWave, m = Wide<T>::n;
    static_assert(kWords <= kWave, "a lane per word");
    __shared__ unsigned long long target[kWords];           // bit i % 64 of word i / 64: row i has one
    const int lane = threadIdx.x % kWave;
    int64_t y[kEach];
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
        const int i = u * kBlock + (int)threadIdx.x;
        y[u] = i < n ? index_at(labels, wide != 0, i) : -1;
    }
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
        const unsigned long long all = __ballot(y[u] >= 0 && y[u] < V);
        if (lane == 0) target[(u * kBlock + (int)threadIdx.x) / kWave] = all;
    }
    __syncthreads();
    const int i = (int)blockIdx.x * (kBlock / lanes) + (int)threadIdx.x / lanes;       // one row a wave
    const unsigned long long own = lane < kWords ? target[lane] : 0;
    const int word = i / kWave;
    int count = __popcll(own), at = lane < word ? count : lane == word ? __popcll(own & ((1ull << (i % kWave)) - 1)) : 0;
    for (int o = kWave / 2; o > 0; o >>= 1) {
        count += __shfl_xor(count, o, kWave);
        at += __shfl_xor(at, o, kWave);
    }
    if (blockIdx.x == 0) {
        if (threadIdx.x == 0) {
            r.head->count = count;
            r.head->factor = (float)(mean ? scale / (double)max(count, 1) : scale);
        }
        if (threadIdx.x < kZeroPage / 4) reinterpret_cast<float*>(r.head->zeros)[threadIdx.x] = 0.f;
    }
    if (i >= n) return;
    const bool has = (target[word] >> (i % kWave)) & 1;
    if (threadIdx.x % lanes == 0) {
        r.place[i] = has ? at : -1;
        if (has) {
            r.row[at] = i;
            r.label[at] = (int32_t)index_at(labels, wide != 0, i);
        } else {
            if (loss) loss[i] = 0.f;
            if (lse) lse[i] = 0.f;
        }
    }
    if (!has) return;
    for (int c = (threadIdx.x & (lanes - 1)) * m; c < pitch; c += lanes * m)
        *reinterpret_cast<typename Wide<T>::vec*>(dst + (int64_t)at * pitch + c) = load_piece<T>(src + i * ld + c, cols - c);
}

// Copies rows of `cols` elements that lie ld apart to rows of `pitch` (a multiple of kInputCols), zeros behind the last column.  LIST:
// the rows of the list (those that have a target: what the others hold, NaN included, is not looked at again).  The products then
// load whole 16-byte pieces and know no strides.  `lanes` threads (a wave or four) share a row.
template <int T, bool LIST>
__global__ __launch_bounds__(kBlock) void loss_rows(const typename ElemOf<T>::type* __restrict__ src, int64_t ld, int64_t rows, int cols,
                                                    LossRows r, typename ElemOf<T>::type* __restrict__ dst, int pitch, int lanes)
{
    constexpr int n = Wide<T>::n;
    const int64_t j = (int64_t)blockIdx.x * (kBlock / lanes) + threadIdx.x / lanes;
    if (j >= (LIST ? (int64_t)r.head->count : rows)) return;
    const typename ElemOf<T>::type* from = src + (LIST ? (int64_t)r.row[j] : j) * ld;
    for (int c = (threadIdx.x & (lanes - 1)) * n; c < pitch; c += lanes * n)
        *reinterpret_cast<typename Wide<T>::vec*>(dst + j * pitch + c) = load_piece<T>(from + c, cols - c);
}

// ------------------------------------------------------------------ products

// One operand of a product, as a matrix of `mn` by `k` valid elements.  Held by rows of k (KMAJOR false: element (i, k) at
// at[i ld + k]) or by rows of mn (at[k ld + i]).  Rows are whole 16-byte pieces, and so are the valid ones.
struct Operand {
    const void* at;
    int64_t ld;
    int64_t mn, k;
};

// kSums: the product itself in fp32, in parts of the k axis that somebody adds up (the inputs' gradients; logits of small calls).
enum LossProduct { kLogits = 0, kLogitGrads, kSums, kWeightGrads };

struct ProductArgs {
    Operand p, q;               // p: the output's adjacent index, q: its rows
    const LossHead* head;
    int tiles_p, tiles_q;       // tiles of the output
    int splits;                 // parts of the k axis (kSums)
    int64_t k_part;             // length of a part, a multiple of the tile's
    int64_t rest;               // 0, or bytes from q to what its rounding has left, which is multiplied as well
    // kLogits, kLogitGrads
    int32_t v0, V;              // first class of the piece, all classes
    const int32_t* label;
    float* picked;              // [rows] the label's logit
    float2* slab;               // [rows][slabs]: largest logit and sum of exponentials of a slab of classes
    int64_t slabs;
    void* held;                 // [rows][ld], classes from keep0 on, or null.  kLogits: fp32 logits, or in 16 bits the exponentials of
                                // what is left of them when their slab's largest is taken off; kLogitGrads: their gradients
    int32_t keep0;
    int64_t ld;
    const float2* stat;         // [rows] largest logit, 1 / sum
    const float* own;           // [rows] gradient of the label's logit
    const int32_t* rounded;     // [rows] the label of a row whose own gradient's rounding leaves something, else -1; or null: nothing is added
    // kSums: [splits][rows][ld]; kWeightGrads: rows of ld elements, part of an arena
    float* sums;
    int64_t sum_part;
    void* out;
    int add;                    // to what is there
};

// Gradients of the logits in half precision are held times 2^15: they lie in [-1, 1], and half of the softmax of a large vocabulary
// would fall below 2^-14, where half precision loses bits.  (bfloat16 has fp32's range.)
template <int T> constexpr float grad_unit() { return T == HSADMM_TYPE_F16 ? 32768.f : 1.f; }
constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// A tile of an operand lies in LDS as pieces of 16 bytes, kTileK bytes of k by B of mn, in the order in which the lanes of a wave
// load them (global_load_lds puts a wave's 64 pieces one behind the other), so bank conflicts are avoided by which piece a
// lane loads.  Rows of k (128 bytes, 8 pieces): piece c of row i at place c ^ (i / 2 mod 8), so the 16 rows that a quarter wave reads
// one piece of lie in 16 places of a 256-byte span.  Rows of mn: the pieces of row k move by `turn(k)` (rows of a multiple of 256
// bytes would put the four to eight rows that one read touches on the same banks).
constexpr int kTileK = 128;

template <int T, int B, bool KMAJOR> struct TilePart {
    typedef typename ElemOf<T>::type E;
    static constexpr int kPiece = Wide<T>::n;                       // elements of a piece
    static constexpr int kK = kTileK / (int)sizeof(E);              // length of the tile along k
    static constexpr int kPieces = B * kTileK / 16;
    static constexpr int kRow = KMAJOR ? B / kPiece : 8;            // pieces of a row
    static constexpr int kBytes = B * kTileK;

    static __device__ __forceinline__ int turn(int row)
    {
        if constexpr (!KMAJOR) return (row >> 1) & 7;
        else if constexpr (sizeof(E) == 4) return kRow >= 16 ? ((row >> 2) & 1) << 3 : 0;
        else return kRow >= 16 ? (row & 3) << 2 : kRow == 8 ? ((row >> 1) & 1) << 2 : 0;
    }
};

// 16 bytes from each lane's address to LDS, the wave's pieces one behind the other from `to` on.  Written out, since the compiler has
// every transposing read of LDS wait for all loads to LDS that it knows of, also those to places that are not read: whoever uses
// this waits by itself (tile_barrier), and once more before the workgroup ends.
__device__ __forceinline__ void load_to_lds(const void* from, const char* to)
{
    const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)to);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(at), "v"(from) : "m0");
}

// Where a lane's pieces of an operand's tiles come from.  Rows (or pieces) behind the operand's last one are read from a valid place
// instead: whatever they hold goes to outputs that nobody stores.  What lies behind the end of k comes from the page of zeros.
template <int T, int B, bool KMAJOR, int THREADS>
struct TileSource {
    typedef TilePart<T, B, KMAJOR> L;
    static constexpr int kLoads = L::kPieces / THREADS;
    static_assert(L::kPieces % THREADS == 0 && (THREADS / L::kRow) % 16 == 0 || KMAJOR, "whole loads; every load of a lane the same piece of its row");
    const char* from[kLoads];
    int64_t step;               // bytes from a tile to the next one
    int k;                      // of the lane's first element, in the tile
    __device__ __forceinline__ TileSource(const Operand& o, int64_t mn0, int64_t k0)
    {
        constexpr int size = sizeof(typename L::E);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int slot = i * THREADS + threadIdx.x;
            const int row = slot / L::kRow, piece = (slot % L::kRow) ^ L::turn(row);
            const int64_t mn = KMAJOR ? mn0 + piece * L::kPiece : min(mn0 + row, o.mn - 1);
            const int64_t at = KMAJOR ? (k0 + row) * o.ld + (mn < o.mn ? mn : 0) : mn * o.ld + k0 + piece * L::kPiece;
            from[i] = static_cast<const char*>(o.at) + at * size;
            if (i == 0) k = KMAJOR ? row : piece * L::kPiece;
        }
        step = KMAJOR ? (int64_t)L::kK * o.ld * size : kTileK;
    }
    // Load i of the tile that lies `offset` bytes behind the first one and has `left` of k left, to its place in LDS.
    __device__ __forceinline__ void load(int i, int64_t offset, int left, const unsigned char* zeros, char* lds) const
    {
        const void* at = (KMAJOR ? k + i * (THREADS / L::kRow) : k) < left ? static_cast<const void*>(from[i] + offset) : zeros;
        load_to_lds(at, lds + (i * THREADS + (threadIdx.x & ~(kWave - 1))) * 16);
    }
};

// Waits until no more than N loads of this wave are on their way and its LDS reads are back, then for the other waves.
template <int N>
__device__ __forceinline__ void tile_barrier()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// What a lane feeds the matrix unit with for 32 rows of mn and one step of k (two pieces): its row is lane % 32, its k are
// the piece of its half of the wave.
template <int T, int B, bool KMAJOR>
__device__ __forceinline__ typename Wide<T>::vec read_tile(const char* lds, int mn0, int step)
{
    typedef TilePart<T, B, KMAJOR> L;
    typedef typename Wide<T>::vec V;
    const int lane = threadIdx.x & (kWave - 1), half = lane >> 5;
    if constexpr (!KMAJOR) {
        const int row = mn0 + (lane & 31);
        return *reinterpret_cast<const V*>(lds + (row * 8 + ((2 * step + half) ^ L::turn(row))) * 16);
    } else if constexpr (T == HSADMM_TYPE_F32) {
        const int mn = mn0 + (lane & 31);
        V v;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int row = 8 * step + 4 * half + j;
            v[j] = *reinterpret_cast<const float*>(lds + (row * L::kRow + ((mn >> 2) ^ L::turn(row))) * 16 + (mn & 3) * 4);
        }
        return v;
    } else {
        // a transposing read: of 16 lanes, lane t brings four elements of mn at k = t / 4, and takes four k of the mn that is t
        v4s part[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int row = 16 * step + 8 * half + 4 * j + ((lane & 15) >> 2);
            const int mn = mn0 + (lane & 16) + 4 * (lane & 3);
            part[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) v4s*)(lds + (row * L::kRow + ((mn >> 3) ^ L::turn(row))) * 16 + (mn & 4) * 2));
        }
        V v;
        __builtin_memcpy(&v, part, 16);
        return v;
    }
}

template <int T>
__device__ __forceinline__ v16f multiply(typename Wide<T>::vec a, typename Wide<T>::vec b, v16f c)
{
    if constexpr (T == HSADMM_TYPE_BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    else if constexpr (T == HSADMM_TYPE_F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    else {
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
        return c;
    }
}

// A tile of BP by BQ of one product per workgroup of WP by WQ waves.  Lane l of a wave holds, of every 32 by 32 of its part, row
// q = l % 32 and 16 of the p.  A turn is a tile of k, four steps of the matrix units; while a step is multiplied the next one's operands
// are read from LDS.  LDS has five places for operands' tiles, taken in the order p, q, p, q, ...: two are read, three are on
// their way.  One barrier a turn, before its last step: the next turn's tiles have arrived, and this turn's are read, so their
// places take the q of the turn after the next and the p of the one behind that.  Loads and LDS reads stand between the products.
//
// Bound by the matrix units at the clock that their power leaves (8192 x 4096 x 65536 in bf16: 1.65 GHz, busy 67 to 71 % of the cycles):
// 8192 x 4096 x 32768 in bf16,
// logits 1205 TFLOP/s, inputs' gradients 1230, weights' 1190 (a library's plain products of these sizes 1353, 1250, 1115).  Two whole
// turns in LDS, each loaded in one go at its predecessor's beginning: 889, 896, 902; the same without loads 1248, 1596, 1439, without
// products 1019, 1421, 1407, so the two hardly overlapped.  Four waves of 128 x 128 instead of eight of 128 x 64: 963, 1175, 1132.
// In fp32, 256 x 2048 x 1000 (tiles of 64, four to eight parts): 14.5 us each, 72 TFLOP/s.
template <int T, int BP, int BQ, int WP, int WQ, bool PMAJOR, bool QMAJOR, int WHAT>
__global__ __launch_bounds__(WP * WQ * kWave) void loss_product(ProductArgs a)
{
    typedef typename ElemOf<T>::type E;
    typedef typename Wide<T>::vec V;
    typedef TilePart<T, BP, PMAJOR> LP;
    typedef TilePart<T, BQ, QMAJOR> LQ;
    constexpr int kThreads = WP * WQ * kWave, TP = BP / WP / 32, TQ = BQ / WQ / 32, kSteps = 4;
    constexpr int kPlaces = 5, kPlace = LP::kBytes > LQ::kBytes ? LP::kBytes : LQ::kBytes;
    __shared__ __align__(16) char lds[kPlaces * kPlace];

    // Workgroups go round the eight dies; a die takes adjacent tiles, 8 of q by as many p, so its cache holds what they share.  Tiles of
    // rows that have no target are none of them.
    const int count = a.head->count;
    if (WHAT != kWeightGrads) a.tiles_q = min(a.tiles_q, (count + BQ - 1) / BQ);
    const int64_t tiles = (int64_t)a.tiles_p * a.tiles_q;
    int64_t t = blockIdx.x;
    {
        const int64_t all = tiles * a.splits, each = (all + 7) / 8, die = t % 8;
        if (t / 8 >= each) return;
        t = die * each + t / 8;
        if (t >= all) return;
    }
    const int part = (int)(t / tiles);
    t -= part * tiles;
    constexpr int kBand = 8;
    const int64_t band = t / ((int64_t)kBand * a.tiles_p);
    const int in_band = (int)min((int64_t)kBand, a.tiles_q - band * kBand);
    t -= band * kBand * a.tiles_p;
    const int64_t q0 = (band * kBand + t % in_band) * BQ, p0 = t / in_band * BP;

    // (rows behind the last one with a target hold anything: as rows of the output nobody reads them, along k they are left out)
    if (WHAT == kWeightGrads) a.p.k = a.q.k = count;
    int64_t k_end = a.p.k;
    const int64_t k_begin = (int64_t)part * a.k_part;
    k_end = min(k_end, k_begin + a.k_part);

    const int wave = threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1), half = lane >> 5;
    const int wp = wave / WQ * (BP / WP), wq = wave % WQ * (BQ / WQ);
    v16f acc[TP][TQ];
#pragma unroll
    for (int i = 0; i < TP; ++i)
#pragma unroll
        for (int j = 0; j < TQ; ++j) acc[i][j] = v16f{};

    const int once = max(0, (int)((k_end - k_begin + LP::kK - 1) / LP::kK)), turns = a.rest ? 2 * once : once;
    const TileSource<T, BP, PMAJOR, kThreads> from_p(a.p, p0, k_begin);
    const TileSource<T, BQ, QMAJOR, kThreads> from_q(a.q, q0, k_begin);
    constexpr int kLoadsP = from_p.kLoads, kLoadsQ = from_q.kLoads;
    const unsigned char* zeros = a.head->zeros;
    // Where one tile of rows sees all weights, which are then read once, workgroups begin at different turns: rows of a power of two of
    // bytes that all workgroups read at the same column keep a few of the memory's channels busy (one row x 2048 x 131072, bf16:
    // 121 us, so 92, 5.8 TB/s).  (The tiles of rows are those that have a target: their number is the one thing beside the sizes that
    // the order of a logit's additions, and so its last bits, depend on.)
    const int begin = WHAT != kWeightGrads && a.tiles_q == 1 && once > 0 ? (int)(p0 / BP % once) : 0;
    const auto at_turn = [&](int turn) {
        const int u = (turn >= once && a.rest ? turn - once : turn) + begin;
        return u < once || begin == 0 ? u : u - once;
    };
    const int all_p = (int)(a.p.k - k_begin), all_q = (int)(a.q.k - k_begin);
    const auto left_p = [&](int turn) { return all_p - at_turn(turn) * LP::kK; };
    const auto left_q = [&](int turn) { return all_q - at_turn(turn) * LP::kK; };
    const auto offset_p = [&](int turn) { return at_turn(turn) * from_p.step; };
    const auto offset_q = [&](int turn) { return at_turn(turn) * from_q.step + (turn >= once ? a.rest : 0); };
    const auto place = [&](int u) { return lds + u * kPlace; };
    typename Wide<T>::vec fp[2][TP], fq[2][TQ];
    constexpr int kReads = TP + TQ, kProducts = TP * TQ;
    const auto read = [&](int r, int s, const char* at_p, const char* at_q) {
        if (r < TQ) fq[s & 1][r] = read_tile<T, BQ, QMAJOR>(at_q, wq + 32 * r, s);
        else fp[s & 1][r - TQ] = read_tile<T, BP, PMAJOR>(at_p, wp + 32 * (r - TQ), s);
    };
    // the products of step s, `beside(n)` behind the n-th
    const auto step = [&](int s, auto&& beside) {
#pragma unroll
        for (int n = 0; n < kProducts; ++n) {
            acc[n / TQ][n % TQ] = multiply<T>(fp[s & 1][n / TQ], fq[s & 1][n % TQ], acc[n / TQ][n % TQ]);
            beside(n);
        }
    };
    // the m-th of `of` things belongs behind product n
    const auto due = [](int n, int m, int of) { return m * kProducts / of == n; };
    // (loads of turns behind the last one bring zeros, or another part's, that nobody reads: no branch stands between the products)
#pragma unroll
    for (int u = 0; u < kPlaces - 1; ++u) {
        const int turn = u / 2;
        if (u % 2 == 0)
#pragma unroll
            for (int i = 0; i < kLoadsP; ++i) from_p.load(i, offset_p(turn), left_p(turn), zeros, place(u));
        else
#pragma unroll
            for (int i = 0; i < kLoadsQ; ++i) from_q.load(i, offset_q(turn), left_q(turn), zeros, place(u));
    }
    tile_barrier<kLoadsP + kLoadsQ>();
#pragma unroll
    for (int r = 0; r < kReads; ++r) read(r, 0, place(0), place(1));
    int unit = 0;               // the place of the turn's p
    const auto behind = [&](int n) { return lds + (unit + n >= kPlaces ? unit + n - kPlaces : unit + n) * kPlace; };
    for (int turn = 0; turn < turns; ++turn) {
        const char* at_p = behind(0);
        const char* at_q = behind(1);
        const int64_t to_p = offset_p(turn + 2), to_q = offset_q(turn + 2);
        const int some_p = left_p(turn + 2), some_q = left_q(turn + 2);
#pragma unroll
        for (int s = 0; s < kSteps - 1; ++s)
            step(s, [&](int n) {
#pragma unroll
                for (int r = 0; r < kReads; ++r)
                    if (due(n, r, kReads)) read(r, s + 1, at_p, at_q);
                if (s == 0)
#pragma unroll
                    for (int i = 0; i < kLoadsP; ++i)
                        if (due(n, i, kLoadsP)) from_p.load(i, to_p, some_p, zeros, behind(4));
            });
        tile_barrier<kLoadsP>();
        const char* next_p = behind(2);
        const char* next_q = behind(3);
        step(kSteps - 1, [&](int n) {
#pragma unroll
            for (int r = 0; r < kReads; ++r)
                if (due(n, r, kReads)) read(r, 0, next_p, next_q);
#pragma unroll
            for (int i = 0; i < kLoadsQ; ++i)
                if (due(n, i, kLoadsQ)) from_q.load(i, to_q, some_q, zeros, behind(0));
        });
        unit = unit + 2 >= kPlaces ? unit + 2 - kPlaces : unit + 2;
    }
    tile_barrier<0>();

    // What rounding the labels' gradients has left, over the rows whose label is one of the tile's classes: a product like the one
    // above, of those rows' inputs and a matrix with one element a row.  A thread looks at kEach adjacent rows at a time; the rows found
    // are gathered, 64 a turn, two turns ahead.  us a call without / with it, bf16, labels as frequent as tokens are: 4096 x 2048 x 32768
    // 1495 / 1511, 16384 x 512 x 4096 394 / 447 (half the labels in the first tile), 560 x 1568 x 3479 72 / 79.
    if constexpr (WHAT == kWeightGrads && T != HSADMM_TYPE_F32) if (a.rounded) {
        constexpr int kEach = 16, kChunk = kThreads * kEach, kW = kThreads / kWave;
        constexpr int kRowThreads = kThreads / LQ::kK;          // that make a row of the second operand
        static_assert(PMAJOR && kChunk <= 1 << 16 && kChunk * 2 <= kPlace, "the list fits its place");
        uint16_t* list = reinterpret_cast<uint16_t*>(place(2));                     // rows found, numbers in the chunk, ascending
        int* found = reinterpret_cast<int*>(place(4));                              // [2][waves]
        const auto ring = [&](int slot) { return place(slot == 2 ? 3 : slot); };    // 0, 1, 3; 4 is the second operand's
        const int class0 = a.v0 + (int)q0, classes = (int)min((int64_t)BQ, a.q.mn - q0);
        typedef int v4i __attribute__((ext_vector_type(4)));
        v4i next[kEach / 4];
        const auto look = [&](int r0) {
            const int r = r0 + (int)threadIdx.x * kEach;
#pragma unroll
            for (int u = 0; u < kEach / 4; ++u) next[u] = r + 4 * u < count ? *reinterpret_cast<const v4i*>(a.rounded + r + 4 * u) : v4i{-1, -1, -1, -1};
        };
        look(0);
        for (int r0 = 0, side = 0; r0 < count; r0 += kChunk, side ^= 1) {
            uint32_t hits = 0;
#pragma unroll
            for (int u = 0; u < kEach; ++u)
                if (r0 + (int)threadIdx.x * kEach + u < count && (uint32_t)(next[u / 4][u % 4] - class0) < (uint32_t)classes) hits |= 1u << u;
            if (r0 + kChunk < count) look(r0 + kChunk);
            int upto = __popc(hits);
            for (int o = 1; o < kWave; o <<= 1) {
                const int x = __shfl_up(upto, o, kWave);
                if (lane >= o) upto += x;
            }
            if (lane == kWave - 1) found[side * kW + wave] = upto;
            __syncthreads();
            int n = 0, at = upto - __popc(hits);
#pragma unroll
            for (int w = 0; w < kW; ++w) {
                const int x = found[side * kW + w];
                n += x;
                if (w < wave) at += x;
            }
            n = __builtin_amdgcn_readfirstlane(n);
            if (n == 0) continue;
            for (uint32_t h = hits; h != 0; h &= h - 1) list[at++] = (uint16_t)(threadIdx.x * kEach + __ffs(h) - 1);
            __syncthreads();
            const int turns = (n + LP::kK - 1) / LP::kK;
            const auto load = [&](int turn, char* to) {
#pragma unroll
                for (int i = 0; i < kLoadsP; ++i) {
                    const int slot = i * kThreads + threadIdx.x, k = slot / LP::kRow, piece = (slot % LP::kRow) ^ LP::turn(k), h = turn * LP::kK + k;
                    const int64_t mn = p0 + piece * LP::kPiece;
                    const void* from = zeros;
                    if (h < n) from = static_cast<const E*>(a.p.at) + (r0 + (int64_t)list[h]) * a.p.ld + (mn < a.p.mn ? mn : 0);
                    load_to_lds(from, to + (i * kThreads + (threadIdx.x & ~(kWave - 1))) * 16);
                }
            };
            // of the thread's row of the second operand, a turn ahead
            const int k = threadIdx.x / kRowThreads;
            int of = 0;
            float own = 0.f;
            const auto second = [&](int turn) {
                const int h = turn * LQ::kK + k;
                of = 0;
                own = 0.f;
                if (h < n) {
                    of = a.label[r0 + (int)list[h]] - class0;
                    own = a.own[r0 + (int)list[h]];
                }
            };
            second(0);
            load(0, ring(0));
            load(1, ring(1));
            for (int u = 0, slot = 0; u < turns; ++u) {
                tile_barrier<kLoadsP>();
                const char* at_p = ring(slot);
                V one;
#pragma unroll
                for (int e = 0; e < LQ::kPiece; ++e) one[e] = (of & (LQ::kPiece - 1)) == e ? (E)(own - (float)(E)own) : (E)0.f;
#pragma unroll
                for (int i = 0; i < LQ::kRow / kRowThreads; ++i) {
                    const int piece = i * kRowThreads + threadIdx.x % kRowThreads;
                    *reinterpret_cast<V*>(place(4) + (k * LQ::kRow + (piece ^ LQ::turn(k))) * 16) = piece == of / LQ::kPiece ? one : V{};
                }
                second(u + 1);
                load(u + 2, ring(slot == 0 ? 2 : slot - 1));
                slot = slot == 2 ? 0 : slot + 1;
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
#pragma unroll
                    for (int r = 0; r < kReads; ++r) read(r, s, at_p, place(4));
                    step(s, [](int) {});
                }
            }
            tile_barrier<0>();
        }
        __syncthreads();
    }

    // p of element e (0..15) of acc[i][.]: 32 i + 8 (e / 4) + 4 half + e % 4 behind wp.  Outputs of type E pass through LDS, [q][p] with
    // the pieces of a row turned by the row's number, and leave as whole rows: straight from the lanes, 16 bytes in each of 32 rows at
    // a time, a tile of logits took 35 us on top of the 70 of its products (2048 inputs, bf16).
    typedef typename ElemOf<T>::vec V4;
    constexpr int kPiece = Wide<T>::n, kRowPieces = BP / kPiece;
    static_assert(BP * BQ * (int)sizeof(E) <= kPlaces * kPlace && (kRowPieces & (kRowPieces - 1)) == 0, "the tile fits");
    const auto piece_at = [&](int q, int piece) { return lds + (q * kRowPieces + (piece ^ (q & (kRowPieces - 1)))) * 16; };
    const auto stage = [&](int i, int j, int g, v4f x) {
        const int q = wq + 32 * j + (lane & 31), p = wp + 32 * i + 8 * g + 4 * half;
        *reinterpret_cast<V4*>(piece_at(q, p / kPiece) + p % kPiece * sizeof(E)) = __builtin_convertvector(x, V4);
    };
    const auto four = [&](int i, int j, int g) { return v4f{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]}; };
    // store(q, p, piece) for every piece of the tile
    const auto leave = [&](auto&& store) {
        __syncthreads();
        for (int n = threadIdx.x; n < BQ * kRowPieces; n += kThreads)
            store(n / kRowPieces, n % kRowPieces * kPiece, *reinterpret_cast<const V*>(piece_at(n / kRowPieces, n % kRowPieces)));
    };
    if constexpr (WHAT == kLogits) {
        const int first = a.v0 + (int)p0 + wp + 4 * half;               // the class of the lane's first element
        if (a.v0 + p0 + BP > a.V) {
#pragma unroll
            for (int j = 0; j < TQ; ++j)
#pragma unroll
                for (int i = 0; i < TP; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (first + 32 * i + 8 * (e / 4) + e % 4 >= a.V) acc[i][j][e] = -__builtin_inff();
        }
        const bool keep = a.held && a.v0 + p0 + BP > a.keep0;
#pragma unroll
        for (int j = 0; j < TQ; ++j) {
            const int64_t q = q0 + wq + 32 * j + (lane & 31);
            const int own = q < count ? a.label[q] - first : -1;        // which of the wave's classes is the label
            if (__any(own >= 0 && own < BP / WP)) {
                float picked = 0.f;
                bool mine = false;
#pragma unroll
                for (int i = 0; i < TP; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const bool is = own == 32 * i + 8 * (e / 4) + e % 4;
                        picked = is ? acc[i][j][e] : picked;
                        mine |= is;
                    }
                if (mine) a.picked[q] = picked;
            }
            float top = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < TP; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) top = fmaxf(top, acc[i][j][e]);
            top = fmaxf(top, __shfl_xor(top, 32, kWave));
            // (a slab of -inf alone has the sum 0; one with a NaN the sum NaN)
            const float from = top == -__builtin_inff() ? 0.f : top;
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < TP; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float x = exp_of(acc[i][j][e] - from);
                    sum += x;
                    if constexpr (T != HSADMM_TYPE_F32) acc[i][j][e] = x * grad_unit<T>();
                }
            sum += __shfl_xor(sum, 32, kWave);
            if (half == 0 && q < count) a.slab[q * a.slabs + (a.v0 + p0 + wp) / (BP / WP)] = make_float2(top, sum);
            if (keep)
#pragma unroll
                for (int i = 0; i < TP; ++i)
#pragma unroll
                    for (int g = 0; g < 4; ++g) stage(i, j, g, four(i, j, g));
        }
        if (keep)
            leave([&](int q, int p, V x) {
                const int64_t c = a.v0 + p0 + p - a.keep0;
                if (q0 + q < count && c >= 0 && c < a.ld) *reinterpret_cast<V*>(static_cast<E*>(a.held) + (q0 + q) * a.ld + c) = x;
            });
    } else if constexpr (WHAT == kLogitGrads) {
#pragma unroll
        for (int j = 0; j < TQ; ++j) {
            const int64_t q = q0 + wq + 32 * j + (lane & 31);
            const int label = q < count ? a.label[q] : -1;
            const float2 stat = q < count ? a.stat[q] : make_float2(0.f, 0.f);
            const float own = q < count ? a.own[q] : 0.f;               // (as loss_softmax has it, to the last bit)
#pragma unroll
            for (int i = 0; i < TP; ++i)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int v = a.v0 + (int)p0 + wp + 32 * i + 8 * g + 4 * half;
                    v4f x = four(i, j, g);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float y = v + e == label ? own : exp_of(x[e] - stat.x) * stat.y * grad_unit<T>();
                        x[e] = v + e < a.V ? y : 0.f;
                    }
                    stage(i, j, g, x);
                }
        }
        leave([&](int q, int p, V x) {
            if (q0 + q < count && p0 + p < a.ld) *reinterpret_cast<V*>(static_cast<E*>(a.held) + (q0 + q) * a.ld + p0 + p) = x;
        });
    } else if constexpr (WHAT == kSums) {
#pragma unroll
        for (int j = 0; j < TQ; ++j) {
            const int64_t q = q0 + wq + 32 * j + (lane & 31);
            float* row = a.sums + part * a.sum_part + q * a.ld;
#pragma unroll
            for (int i = 0; i < TP; ++i)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int64_t c = p0 + wp + 32 * i + 8 * g + 4 * half;
                    v4f x = four(i, j, g);
                    if (q < count && c < a.ld) {
                        if (a.add) x += *reinterpret_cast<const v4f*>(row + c);
                        *reinterpret_cast<v4f*>(row + c) = x;
                    }
                }
        }
    } else {
        const float f = a.head->factor * (1.f / grad_unit<T>());
        E* out = static_cast<E*>(a.out);
#pragma unroll
        for (int j = 0; j < TQ; ++j) {
            const int64_t q = q0 + wq + 32 * j + (lane & 31);
#pragma unroll
            for (int i = 0; i < TP; ++i)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    v4f x = four(i, j, g) * f;
                    if (a.add) {
                        // (added to before it is rounded)
                        const int64_t c = p0 + wp + 32 * i + 8 * g + 4 * half;
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (q < a.q.mn && c + e < a.ld) x[e] += (float)out[q * a.ld + c + e];
                    }
                    stage(i, j, g, x);
                }
        }
        leave([&](int q, int p, V x) {
            const int64_t left = a.ld - p0 - p;
            if (q0 + q < a.q.mn && left > 0) store_piece<T>(out + (q0 + q) * a.ld + p0 + p, x, (int)min(left, (int64_t)kPiece));
        });
    }
}

// ------------------------------------------------------------------ between the products

struct SoftmaxArgs {
    LossRows r;
    const float2* slab;         // what kLogits wrote of a row ...
    int slabs;                  // (its slabs)
    int64_t pitch;
    int slab_elems;
    const float* picked;
    const float* sums;          // ... or, slab null, the logits in parts: [parts][rows][ld]
    int parts;
    int64_t sum_part;
    float2* stat;
    float* own;                 // [rows] gradients of the labels' logits ...
    int32_t* rounded;           // ... and the label where rounding them leaves something that counts, else -1
    float* held_loss;           // [rows], for the total
    float* loss;                // by original rows, may be null
    float* lse;
    const void* held;           // with slabs: of the classes from v0 on, as kLogits wrote them
    void* grads;                // [rows][ld] gradients of the logits, may be null; with slabs held itself
    int64_t rest;               // 0, or (16 bits, without slabs) bytes from grads to what their rounding leaves
    int64_t ld;
    int32_t v0, V;
};

// Four adjacent sums, over their parts in order, eight parts in flight.
__device__ __forceinline__ v4f add_parts(const float* p, int parts, int64_t part)
{
    v4f x = {0.f, 0.f, 0.f, 0.f};
    constexpr int kAtOnce = 8;
    int i = 0;
    for (; i + kAtOnce <= parts; i += kAtOnce) {
        v4f y[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) y[u] = *reinterpret_cast<const v4f*>(p + (i + u) * part);
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) x += y[u];
    }
    for (; i < parts; ++i) x += *reinterpret_cast<const v4f*>(p + i * part);
    return x;
}

__device__ __forceinline__ float2 join(float2 a, float2 b)
{
    // (a side without any value has the sum 0 and the largest value -inf; NaN in a sum stays)
    const float top = fmaxf(a.x, b.x), from = top == -__builtin_inff() ? 0.f : top;
    return make_float2(top, a.y * exp_of(a.x - from) + b.y * exp_of(b.x - from));
}

// A row per workgroup: largest logit, sum, loss, and the gradients of the logits that are held (softmax minus the label's one).  The order
// of the additions here depends on the sizes alone.  16 bits: what kLogits held is rounded already, so a gradient carries two
// roundings, but the label's own.  That one comes from its logit in fp32, as softmax - 1 of a confident row has far fewer digits than
// either, and what its rounding leaves is added by those who use it: it is most of the row's gradient, so its rounding would be as large as that of
// the outputs and the same for the whole row (1024 x 512 x 4096 in bf16, labels' softmax spread over (0, 1), error of dX against 64
// bits: 0.00215 where it was left out, 0.00166 as the rounding of dX alone).  Without slabs what the rounding of all of them leaves is written as well where the call is
// one of few terms (a.rest).
template <int T>
__global__ __launch_bounds__(kScanBlock) void loss_softmax(SoftmaxArgs a)
{
    typedef typename ElemOf<T>::type E;
    typedef typename Wide<T>::vec V;
    constexpr int n = Wide<T>::n;
    __shared__ float2 red[kScanWaves];
    const int64_t q = blockIdx.x;
    if (q >= a.r.head->count) return;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave, threads = blockDim.x;
    const int label = a.r.label[q];
    float2 s = make_float2(-__builtin_inff(), 0.f);
    float* sum_row = const_cast<float*>(a.sums) + q * a.ld;
    if (a.slab) {
        const float2* row = a.slab + q * a.pitch;
        for (int i = tid; i < a.slabs; i += threads) s = join(s, row[i]);
    } else {
        for (int c = tid * 4; c < a.V; c += threads * 4) {
            const v4f x = add_parts(sum_row + c, a.parts, a.sum_part);
            if (a.parts > 1) *reinterpret_cast<v4f*>(sum_row + c) = x;      // (read again below, behind the barrier, by other threads too)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c + e < a.V) s = join(s, make_float2(x[e], x[e] == x[e] ? 1.f : x[e]));
        }
    }
    for (int o = kWave / 2; o > 0; o >>= 1) s = join(s, make_float2(__shfl_xor(s.x, o, kWave), __shfl_xor(s.y, o, kWave)));
    if (lane == 0) red[wave] = s;
    __syncthreads();
    s = red[0];
    for (int w = 1; w < threads / kWave; ++w) s = join(s, red[w]);
    const float picked = a.slab ? a.picked[q] : sum_row[label], inv = 1.f / s.y;
    if (tid == 0) {
        // (the largest logit cancels in the loss: in the sum's logarithm a loss of 1e-3 would be rounded to the steps of a logit of 1000)
        const float log_y = logf(s.y), log_sum = s.x + log_y, x = (s.x - picked) + log_y;
        a.stat[q] = make_float2(s.x, inv);
        a.held_loss[q] = x;
        const int64_t i = a.r.row[q];
        if (a.loss) a.loss[i] = x;
        if (a.lse) a.lse[i] = log_sum;
    }
    if (!a.grads) return;
    const float own = (exp_of(picked - s.x) * inv - 1.f) * grad_unit<T>();
    if (tid == 0) {
        a.own[q] = own;
        // (a 64th of half a step of the type is lost in the rounding of what it would be added to)
        constexpr float kCounts = (T == HSADMM_TYPE_F16 ? 0x1p-11f : 0x1p-8f) / 64.f;
        a.rounded[q] = __builtin_fabsf(own - (float)(E)own) < __builtin_fabsf(own) * kCounts ? -1 : label;
    }
    E* to = static_cast<E*>(a.grads) + q * a.ld;
    E* to_rest = reinterpret_cast<E*>(reinterpret_cast<char*>(to) + a.rest);
    const E* held = static_cast<const E*>(a.held) + q * a.ld;
    for (int64_t c = (int64_t)tid * n; c < a.ld; c += threads * n) {
        const int64_t v = a.v0 + c;
        V x = {}, rest = {};
        if (v < a.V) {
            if (T != HSADMM_TYPE_F32 && a.slab) {
                const float f = exp_of(a.slab[q * a.pitch + v / a.slab_elems].x - s.x) * inv;
                x = *reinterpret_cast<const V*>(held + c);
#pragma unroll
                for (int e = 0; e < n; ++e) x[e] = (E)((float)x[e] * f);
            } else {
                const float* from = a.slab ? reinterpret_cast<const float*>(held) : sum_row;
#pragma unroll
                for (int e = 0; e < n; ++e) {
                    float y = exp_of(from[c + e] - s.x) * inv * grad_unit<T>();
                    if (v + e == label) y = own;
                    x[e] = (E)y;
                    rest[e] = (E)(v + e < a.V ? y - (float)x[e] : 0.f);
                }
            }
#pragma unroll
            for (int e = 0; e < n; ++e) {
                if (v + e == label) x[e] = (E)own;
                if (v + e >= a.V) x[e] = (E)0.f;
            }
        }
        if (a.rest) *reinterpret_cast<V*>(to_rest + c) = rest;
        *reinterpret_cast<V*>(to + c) = x;
    }
}

// The sum (mean) of the losses, in fp64 and in an order that depends on their number alone, and how many there are.  One workgroup, a
// launch of its own only where no inputs' gradients are made.
__device__ void add_losses(const LossHead* __restrict__ head, const float* __restrict__ held, int mean, float* __restrict__ total)
{
    __shared__ double red[kWaves];
    constexpr int kAtOnce = 16;
    const int count = head->count;
    double s = 0.0;
    for (int i0 = threadIdx.x; i0 < count; i0 += kAtOnce * kBlock) {
        float x[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) x[u] = held[min(i0 + u * kBlock, count - 1)];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) s += i0 + u * kBlock < count ? (double)x[u] : 0.0;
    }
    s = wave_xor_sum(s, kWave);
    if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kWaves; ++w) s += red[w];
        total[0] = (float)(mean ? s / (double)max(count, 1) : s);
        total[1] = (float)count;
    }
}
__global__ __launch_bounds__(kBlock) void loss_total(const LossHead* __restrict__ head, const float* __restrict__ held, int mean,
                                                     float* __restrict__ total)
{
    add_losses(head, held, mean, total);
}

// The gradients of the inputs: the parts' sums in order, and (`own`) what rounding the label's gradient has left times its row of W, times
// the factor, to the rows they belong to; zeros where there is no target.
// Where `total` is asked for the first workgroup makes that instead (a launch less, 3 to 5 us).
template <int T>
__global__ __launch_bounds__(kBlock) void loss_inputs(const float* __restrict__ sums, int splits, int64_t part, int64_t sum_ld, LossRows r,
                                                      typename ElemOf<T>::type* __restrict__ dX, int64_t ld, int64_t n, int cols, int lanes,
                                                      const float* __restrict__ held_loss, int mean, float* __restrict__ total,
                                                      const typename ElemOf<T>::type* __restrict__ W, const float* __restrict__ own)
{
    typedef typename ElemOf<T>::type E;
    constexpr int m = Wide<T>::n;
    if (total && blockIdx.x == 0) {
        add_losses(r.head, held_loss, mean, total);
        return;
    }
    const int64_t i = (int64_t)(blockIdx.x - (total ? 1 : 0)) * (kBlock / lanes) + threadIdx.x / lanes;
    if (i >= n) return;
    const int64_t q = r.place[i];
    const float f = r.head->factor * (1.f / grad_unit<T>());
    float left = 0.f;
    if (own && q >= 0) {
        left = own[q] - (float)(E)own[q];
        W += (int64_t)r.label[q] * cols;
    }
    for (int c = (threadIdx.x & (lanes - 1)) * m; c < cols; c += lanes * m) {
        v4f x[m / 4] = {};
        if (q >= 0) {
            typename Wide<T>::vec w = {};
            if (own) w = load_piece<T>(W + c, cols - c);
#pragma unroll
            for (int h = 0; h < m / 4; ++h) x[h] = add_parts(sums + q * sum_ld + c + 4 * h, splits, part);
            if (own)
#pragma unroll
                for (int e = 0; e < m; ++e) x[e / 4][e % 4] += left * (float)w[e];
        }
        typename Wide<T>::vec y;
#pragma unroll
        for (int e = 0; e < m; ++e) y[e] = (E)(x[e / 4][e % 4] * f);
        store_piece<T>(dX + i * ld + c, y, cols - c);
    }
}

}  // namespace
#endif
