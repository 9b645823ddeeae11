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

constexpr int kInputRows = 256;          // rows of the held copies are rounded up to this ...
constexpr int kInputCols = 64;           // ... and their columns to this (128 bytes at least)
constexpr int kZeroPage = 256;          // bytes of zeros that stand for what lies outside an operand

struct LossHead {
    int32_t count;                      // rows that have a target
    float factor;                       // what gradients are multiplied by
    int32_t pad[62];
    unsigned char zeros[kZeroPage];
};
static_assert(sizeof(LossHead) == 512, "LossHead layout");

struct LossRows {
    LossHead* head;
    int32_t* row;        // [count] the original row of a held one, ascending
    int32_t* label;      // [count]
    int32_t* place;      // [N] the held row of an original one, or -1
};

// Lists the rows whose label lies in [0, V), in order (one workgroup), and settles the rows that have none.
__global__ __launch_bounds__(kScanBlock) void loss_targets(const void* __restrict__ labels, int wide, int64_t n, int32_t V, double scale,
                                                           int mean, LossRows r, float* __restrict__ loss, float* __restrict__ lse)
{
    __shared__ int32_t sums[2][kScanWaves];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    int32_t before = 0;
    int turn = 0;
    for (int64_t i0 = 0; i0 < n; i0 += kScanBlock, turn ^= 1) {
        const int64_t i = i0 + threadIdx.x;
        const int64_t y = i < n ? index_at(labels, wide != 0, i) : -1;
        const bool has = y >= 0 && y < V;
        const unsigned long long all = __ballot(has);
        if (lane == 0) sums[turn][wave] = __popcll(all);
        __syncthreads();
        int32_t at = before;
        for (int w = 0; w < kScanWaves; ++w) {
            const int32_t s = sums[turn][w];
            before += s;
            if (w < wave) at += s;
        }
        at += __popcll(all & ((1ull << lane) - 1));
        if (i < n) {
            r.place[i] = has ? at : -1;
            if (has) {
                r.row[at] = (int32_t)i;
                r.label[at] = (int32_t)y;
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

// Copies rows of `cols` elements that lie ld apart to rows of `pitch` (a multiple of kInputCols), zeros behind the last column.  LIST:
// the rows of the list (those that have a target: what the others hold, NaN included, is not looked at again).  The products then
// load whole 16-byte pieces and know no strides.  A wave takes a row.
template <int T, bool LIST>
__global__ __launch_bounds__(kBlock) void loss_rows(const typename ElemOf<T>::type* __restrict__ src, int64_t ld, int64_t rows, int cols,
                                                    LossRows r, typename ElemOf<T>::type* __restrict__ dst, int pitch)
{
    constexpr int n = Wide<T>::n;
    const int64_t j = (int64_t)blockIdx.x * kWaves + threadIdx.x / kWave;
    if (j >= (LIST ? (int64_t)r.head->count : rows)) return;
    const typename ElemOf<T>::type* from = src + (LIST ? (int64_t)r.row[j] : j) * ld;
    for (int c = (threadIdx.x % kWave) * n; c < pitch; c += kWave * n)
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

template <int T, int B, bool KMAJOR, int THREADS>
__device__ __forceinline__ void load_tile(const Operand& o, int64_t mn0, int64_t k0, const unsigned char* zeros, char* lds)
{
    typedef TilePart<T, B, KMAJOR> L;
    typedef typename L::E E;
    constexpr int kLoads = L::kPieces / THREADS;
    static_assert(L::kPieces % THREADS == 0, "whole loads");
    const int tid = threadIdx.x;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int slot = i * THREADS + tid;
        const int row = slot / L::kRow, piece = (slot % L::kRow) ^ L::turn(row);
        const int64_t mn = KMAJOR ? mn0 + piece * L::kPiece : mn0 + row;
        const int64_t k = KMAJOR ? k0 + row : k0 + piece * L::kPiece;
        const void* from = zeros;
        if (mn < o.mn && k < o.k) from = static_cast<const E*>(o.at) + (KMAJOR ? k * o.ld + mn : mn * o.ld + k);
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                         (__attribute__((address_space(3))) void*)(lds + (i * THREADS + (tid & ~(kWave - 1))) * 16), 16, 0, 0);
    }
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

// Four adjacent elements of an output row, the first nv of them; rows may start at any element.
template <int T>
__device__ __forceinline__ void put4(typename ElemOf<T>::type* p, v4f v, int nv, bool whole, bool add)
{
    typedef typename ElemOf<T>::type E;
    typedef typename ElemOf<T>::vec V4;
    if (whole && nv == 4) {
        if (add) v += __builtin_convertvector(*reinterpret_cast<const V4*>(p), v4f);
        *reinterpret_cast<V4*>(p) = __builtin_convertvector(v, V4);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < nv) p[i] = (E)(add ? v[i] + (float)p[i] : v[i]);
}

// A tile of BP by BQ of one product per workgroup of WP by WQ waves, two tiles of k in LDS: while the matrix units work on one the
// other is loaded, one barrier a tile.  Lane l of a wave holds, of every 32 by 32 of its part, row q = l % 32 and 16 of the p.
template <int T, int BP, int BQ, int WP, int WQ, bool PMAJOR, bool QMAJOR, int WHAT>
__global__ __launch_bounds__(WP * WQ * kWave) void loss_product(ProductArgs a)
{
    typedef typename ElemOf<T>::type E;
    typedef TilePart<T, BP, PMAJOR> LP;
    typedef TilePart<T, BQ, QMAJOR> LQ;
    constexpr int kThreads = WP * WQ * kWave, TP = BP / WP / 32, TQ = BQ / WQ / 32, kSteps = 4;
    __shared__ __align__(16) char lds[2][LP::kBytes + LQ::kBytes];

    // Workgroups go round the eight dies; a die takes adjacent tiles, 8 of q by as many p, so its cache holds what they share.
    const int64_t tiles = (int64_t)a.tiles_p * a.tiles_q;
    int64_t t = blockIdx.x;
    {
        const int64_t all = tiles * a.splits, each = (all + 7) / 8, die = t % 8;
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

    const int count = a.head->count;
    if (WHAT != kWeightGrads && q0 >= count) return;
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

    const int turns = (int)((k_end - k_begin + LP::kK - 1) / LP::kK);
    const auto load = [&](int turn) {
        const int64_t k0 = k_begin + (int64_t)turn * LP::kK;
        char* to = lds[turn & 1];
        load_tile<T, BP, PMAJOR, kThreads>(a.p, p0, k0, a.head->zeros, to);
        load_tile<T, BQ, QMAJOR, kThreads>(a.q, q0, k0, a.head->zeros, to + LP::kBytes);
    };
    if (turns > 0) load(0);
    for (int turn = 0; turn < turns; ++turn) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (turn + 1 < turns) load(turn + 1);
        const char* from = lds[turn & 1];
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            typename Wide<T>::vec fp[TP], fq[TQ];
#pragma unroll
            for (int i = 0; i < TP; ++i) fp[i] = read_tile<T, BP, PMAJOR>(from, wp + 32 * i, s);
#pragma unroll
            for (int j = 0; j < TQ; ++j) fq[j] = read_tile<T, BQ, QMAJOR>(from + LP::kBytes, wq + 32 * j, s);
#pragma unroll
            for (int i = 0; i < TP; ++i)
#pragma unroll
                for (int j = 0; j < TQ; ++j) acc[i][j] = multiply<T>(fp[i], fq[j], acc[i][j]);
        }
    }

    // p of element e (0..15) of acc[i][.]: 32 i + 8 (e / 4) + 4 half + e % 4 behind wp
#pragma unroll
    for (int j = 0; j < TQ; ++j) {
        const int64_t q = q0 + wq + 32 * j + (lane & 31);
        if constexpr (WHAT == kLogits) {
            const bool live = q < count;
            const int label = live ? a.label[q] : -1;
            float top = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < TP; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int v = a.v0 + (int)p0 + wp + 32 * i + 8 * (e / 4) + 4 * half + e % 4;
                    if (v >= a.V) acc[i][j][e] = -__builtin_inff();
                    top = fmaxf(top, acc[i][j][e]);
                    if (v == label) a.picked[q] = acc[i][j][e];
                }
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
                    if constexpr (T != HSADMM_TYPE_F32) acc[i][j][e] = x;
                }
            sum += __shfl_xor(sum, 32, kWave);
            if (half == 0) a.slab[q * a.slabs + (a.v0 + p0 + wp) / (BP / WP)] = make_float2(top, sum);
            if (a.held) {
                typedef typename ElemOf<T>::vec V4;
                E* row = static_cast<E*>(a.held) + q * a.ld;
#pragma unroll
                for (int i = 0; i < TP; ++i)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const int64_t c = a.v0 + p0 + wp + 32 * i + 8 * g + 4 * half - a.keep0;
                        v4f x = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
                        if constexpr (T != HSADMM_TYPE_F32) x *= grad_unit<T>();
                        if (c >= 0 && c < a.ld) *reinterpret_cast<V4*>(row + c) = __builtin_convertvector(x, V4);
                    }
            }
        } else if constexpr (WHAT == kLogitGrads) {
            const bool live = q < count;
            const int label = live ? a.label[q] : -1;
            const float2 stat = live ? a.stat[q] : make_float2(0.f, 0.f);
            E* row = static_cast<E*>(a.held) + q * a.ld;
#pragma unroll
            for (int i = 0; i < TP; ++i)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int64_t c = p0 + wp + 32 * i + 8 * g + 4 * half;
                    v4f x;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int v = a.v0 + (int)c + e;
                        const float y = (exp_of(acc[i][j][4 * g + e] - stat.x) * stat.y - (v == label ? 1.f : 0.f)) * grad_unit<T>();
                        x[e] = live && v < a.V ? y : 0.f;
                    }
                    if (c < a.ld) *reinterpret_cast<typename ElemOf<T>::vec*>(row + c) = __builtin_convertvector(x, typename ElemOf<T>::vec);
                }
        } else if constexpr (WHAT == kSums) {
            float* row = a.sums + part * a.sum_part + q * a.ld;
#pragma unroll
            for (int i = 0; i < TP; ++i)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int64_t c = p0 + wp + 32 * i + 8 * g + 4 * half;
                    v4f x = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
                    if (c < a.ld) {
                        if (a.add) x += *reinterpret_cast<const v4f*>(row + c);
                        *reinterpret_cast<v4f*>(row + c) = x;
                    }
                }
        } else {
            if (q >= a.q.mn) continue;
            const float f = a.head->factor * (1.f / grad_unit<T>());
            E* row = static_cast<E*>(a.out) + q * a.ld;
            const bool whole = a.ld % 4 == 0;       // (an arena's layers start at multiples of four elements)
#pragma unroll
            for (int i = 0; i < TP; ++i)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int64_t c = p0 + wp + 32 * i + 8 * g + 4 * half;
                    const v4f x = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
                    const int nv = (int)min((int64_t)4, a.ld - c);
                    if (nv > 0) put4<T>(row + c, x * f, nv, whole, a.add != 0);
                }
        }
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
    float* held_loss;           // [rows], for the total
    float* loss;                // by original rows, may be null
    float* lse;
    const void* held;           // with slabs: of the classes from v0 on, as kLogits wrote them
    void* grads;                // [rows][ld] gradients of the logits, may be null; with slabs held itself
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
// of the additions depends on the sizes alone.  16 bits: what kLogits held is rounded already, so a gradient here carries two
// roundings; the label's own comes from its logit in fp32, as softmax - 1 of a confident row has far fewer digits than either.
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
            if (a.parts > 1) *reinterpret_cast<v4f*>(sum_row + c) = x;      // (read again by this thread, and for the label below)
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
        const float log_sum = s.x + logf(s.y), x = log_sum - picked;
        a.stat[q] = make_float2(s.x, inv);
        a.held_loss[q] = x;
        const int64_t i = a.r.row[q];
        if (a.loss) a.loss[i] = x;
        if (a.lse) a.lse[i] = log_sum;
    }
    if (!a.grads) return;
    const float own = (exp_of(picked - s.x) * inv - 1.f) * grad_unit<T>();
    E* to = static_cast<E*>(a.grads) + q * a.ld;
    const E* held = static_cast<const E*>(a.held) + q * a.ld;
    for (int64_t c = (int64_t)tid * n; c < a.ld; c += threads * n) {
        const int64_t v = a.v0 + c;
        V x = {};
        if (v < a.V) {
            if (T != HSADMM_TYPE_F32 && a.slab) {
                const float f = exp_of(a.slab[q * a.pitch + v / a.slab_elems].x - s.x) * inv;
                x = *reinterpret_cast<const V*>(held + c);
#pragma unroll
                for (int e = 0; e < n; ++e) x[e] = (E)((float)x[e] * f);
            } else {
                const float* from = a.slab ? reinterpret_cast<const float*>(held) : sum_row;
#pragma unroll
                for (int e = 0; e < n; ++e) x[e] = (E)(exp_of(from[c + e] - s.x) * inv * grad_unit<T>());
            }
#pragma unroll
            for (int e = 0; e < n; ++e) {
                if (v + e == label) x[e] = (E)own;
                if (v + e >= a.V) x[e] = (E)0.f;
            }
        }
        *reinterpret_cast<V*>(to + c) = x;
    }
}

// The sum (mean) of the losses, in fp64 and in an order that depends on their number alone, and how many there are.
__global__ __launch_bounds__(kBlock) void loss_total(const LossHead* __restrict__ head, const float* __restrict__ held, int mean,
                                                     float* __restrict__ total)
{
    __shared__ double red[kWaves];
    const int count = head->count;
    double s = 0.0;
    for (int i = threadIdx.x; i < count; i += kBlock) s += (double)held[i];
    s = wave_xor_sum(s, kWave);
    if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kWaves; ++w) s += red[w];
        total[0] = (float)(mean ? s / (double)max(count, 1) : s);
        total[1] = (float)count;
    }
}

// The gradients of the inputs: the parts' sums in order, times the factor, to the rows they belong to; zeros where there is no target.
template <int T>
__global__ __launch_bounds__(kBlock) void loss_inputs(const float* __restrict__ sums, int splits, int64_t part, int64_t sum_ld, LossRows r,
                                                      typename ElemOf<T>::type* __restrict__ dX, int64_t ld, int64_t n, int cols)
{
    constexpr int m = Wide<T>::n;
    const int64_t i = (int64_t)blockIdx.x * kWaves + threadIdx.x / kWave;
    if (i >= n) return;
    const int64_t q = r.place[i];
    const float f = r.head->factor * (1.f / grad_unit<T>());
    for (int c = (threadIdx.x % kWave) * m; c < cols; c += kWave * m) {
        v4f x[m / 4] = {};
        if (q >= 0)
#pragma unroll
            for (int h = 0; h < m / 4; ++h) x[h] = add_parts(sums + q * sum_ld + c + 4 * h, splits, part);
        typename Wide<T>::vec y;
#pragma unroll
        for (int e = 0; e < m; ++e) y[e] = (typename ElemOf<T>::type)(x[e / 4][e % 4] * f);
        store_piece<T>(dX + i * ld + c, y, cols - c);
    }
}

}  // namespace
#endif
