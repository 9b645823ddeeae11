// hsadmm_compact_mx / hsadmm_expand_mx: the packed buffer in blocks of 32 codes that share a power of two, quantised as it is
// packed and read back as it is scattered.
// Part of the single translation unit built from hsadmm.hip (included there, in order).
#ifndef KERNELS_MX_HPP
#define KERNELS_MX_HPP
#include "hsadmm_device.hpp"
#include "kernels_select.hpp"
#include "kernels_training.hpp"

namespace {

constexpr int kMxBlock = 32;
struct __attribute__((aligned(4))) int4_at4 { int x, y, z, w; };      // four ints at any int's address

// j / d for the unsigned numbers a layer's positions are (see DivKhw; below 2^22 the machine's own reciprocal is near enough for the
// same single step of correction).
struct DivPos {
    unsigned int d;
    float rcp;
    __device__ __forceinline__ explicit DivPos(unsigned int x) : d(x), rcp(__builtin_amdgcn_rcpf((float)x)) {}
    __device__ __forceinline__ unsigned int operator()(unsigned int j) const
    {
        if (j >= (1u << 22)) return j / d;
        unsigned int q = (unsigned int)((float)j * rcp);
        if (q * d > j) --q;
        else if ((q + 1) * d <= j) ++q;
        return q;
    }
};

// ------------------------------------------------------------------ writing

struct MxMaps {
    const int32_t* pos;
    const int32_t* cnt;
    const int32_t* kept_idx;
    const int64_t* layer_off;
    int n_layers;
};

// Four values of a block (32 values in eight adjacent lanes) -> their codes; the block's scale byte.
// The scale is the least 2^e with largest <= 2^e * top (top = 448 = 1.75 * 2^8, or 6 = 1.5 * 2^2): the largest's exponent less
// the format's, one more where its fraction is above top's.  The product with 2^-e is exact (or far below half of the smallest
// code), so a code is the nearest value, ties to even.
template <int FMT>
__device__ __forceinline__ unsigned int mx_encode4(const v4f& x, unsigned int& byte)
{
    unsigned int top = top_bits(x);
    top = max(top, row_exchange<kDppXor1>(top));
    top = max(top, row_exchange<kDppXor2>(top));
    top = max(top, row_exchange<kDppHalfMirror>(top));
    constexpr int kExp = FMT == HSADMM_MX_FP8 ? 8 : 2;
    constexpr unsigned int kFrac = FMT == HSADMM_MX_FP8 ? 0x600000u : 0x400000u;
    const int e = (int)(top >> 23) - kExp + ((top & 0x7fffffu) > kFrac ? 1 : 0);
    const bool bad = top >= 0x7f800000u;                 // an infinity or a NaN: the block reads back as NaN
    byte = bad ? 255u : (unsigned int)max(e, 0);
    const float f = __uint_as_float((254u - (unsigned int)max(e, 0)) << 23);
    v4f y;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = bad ? 0.f : x[i] * f;
    // With the largest scale the codes from the next power of two on stand for 2^128 and more: values next to the end of fp32's
    // range, which would read back as infinite, take the code below.
    constexpr int kTopByte = 254 - kExp + 1;
    constexpr float kTopCode = FMT == HSADMM_MX_FP8 ? 240.0f : 3.0f;
    if (e == kTopByte) {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = __builtin_amdgcn_fmed3f(y[i], -kTopCode, kTopCode);
    }
    if (FMT == HSADMM_MX_FP8)
        return (unsigned int)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false), true);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(__builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, y[0], y[1], 1.0f, 0), y[2], y[3],
                                                    1.0f, 1);
}

// The last layer that starts at or before packed position t (an empty layer starts where the next one does).
__device__ __forceinline__ int layer_at(const int64_t* __restrict__ layer_off, int n_layers, int64_t t)
{
    const int lane = threadIdx.x & (kWave - 1);
    int n = 0;
    for (int j = 0; j < n_layers; j += kWave) {
        const bool before = j + lane < n_layers && layer_off[j + lane] <= t;
        n += __popcll(__ballot(before));
    }
    return n - 1;
}

// The packed buffer in tiles of 4 * Q * kBlock positions, Q times four adjacent ones a thread; a tile that holds several layers
// takes them one after the other (a block of 32 is one layer's).  The grid is what the plan's own selection packs; a mask that
// keeps more has every workgroup take several tiles.  Bound by the latency of a tile's chain of loads (offsets, layer, kept row or
// column, values) and, on large networks, by the lines that hold kept elements.  Measured (values from three states in turn, us):
//   a workgroup per stretch of the layer, kept or not    ResNet-50 at 0.4, z + v: 33.3, packed tiles 27.6 (Q = 2), 24.7 (Q = 4;
//                                                        kMxWide says where which), now 23.3: 92 MB, 4.4 TB/s with a launch's 3 us
//   eight adjacent positions to a lane                   34.3: a wave's load takes every other 16 bytes and lines are fetched twice
//   Q = 4 with all the registers it would take (111)     28.0: four waves a SIMD instead of six
//   no look-up of the kept row, no division (a probe)    2.4 less: the chain of loads
//   columns, a position to a lane through LDS            ResNet-152, channels at 0.3: 113 without, 60.6, non-temporal loads 55.0, now
//                                                        52.6 (221 MB fetched for 70 MB kept: most lines hold a kept channel)
//   columns, rows read whole and kept elements put       133: a look-up of its place for every element, kept or not
//   into LDS at their places
template <int FMT, bool SUM, int Q>
__global__ __launch_bounds__(kBlock, 6) void gather_mx(const DevLayer* __restrict__ layers, const float* __restrict__ src,
                                                    const float* __restrict__ src1, MxMaps mp, uint8_t* __restrict__ codes,
                                                    uint8_t* __restrict__ scales, CopyOut co)
{
    constexpr int kTile = 4 * Q * kBlock, kPart = 8 * kBlock;       // columns of rows: kPart positions at a time
    __shared__ __align__(16) float stage[kPart];
    const int nL = mp.n_layers;
    for (int64_t t0 = (int64_t)blockIdx.x * kTile;; t0 += (int64_t)gridDim.x * kTile) {
        int l = layer_at(mp.layer_off, nL, t0);
        if (t0 >= mp.layer_off[nL]) break;
        for (; l < nL; ++l) {
            const int64_t off = mp.layer_off[l];
            if (off >= t0 + kTile) break;
            const DevLayer& L = layers[l];
            const int mode = L.mode;
            const bool channels = mode_has_channels(mode);
            const bool listed = mode == HSADMM_MODE_FILTER || mode == HSADMM_MODE_BOTH;      // kept filters in a list
            const unsigned int n0 = (unsigned int)mp.cnt[l], n1 = (unsigned int)mp.cnt[2 * nL + l];
            const int32_t* rows = mp.kept_idx + mp.cnt[nL + l];
            const int32_t* cols = rows + (mode == HSADMM_MODE_BOTH ? n0 : 0);
            const unsigned int khw = (unsigned int)L.khw, row_len = (unsigned int)L.row_len;
            const unsigned int out_len = !channels ? row_len : (mode == HSADMM_MODE_BOTH ? n1 : n0) * khw;
            const unsigned int size = (listed ? n0 : (unsigned int)L.c_out) * out_len;     // (below 2^31: part of the layer)
            if (size == 0) continue;
            const float* base = src + L.elem_off;
            const float* base1 = SUM ? src1 + L.elem_off : nullptr;
            // the tile's first position of the layer, as packed row and column
            const int lead = (int)(off > t0 ? off - t0 : 0);                                // places of the tile before the layer
            const unsigned int i0 = (unsigned int)(t0 + lead - off);
            if (i0 >= size) continue;
            const unsigned int p0 = i0 / out_len, c0 = i0 - p0 * out_len;
            const unsigned int there = size - i0;                                           // positions from there on
            const DivPos by_row(out_len);
            // codes and scale of the four positions from place `at` of the tile on
            auto put = [&](int at, const v4f& x) {
                unsigned int byte;
                const unsigned int code = mx_encode4<FMT>(x, byte);
                // (places up to the end of the layer's last block: the next layer starts behind it)
                const int64_t g = t0 + at;
                if (at >= lead && at < kTile && ((unsigned int)(at - lead) & ~(unsigned int)(kMxBlock - 1)) < there) {
                    // (non-temporal / ordinary, us: fp8, a line of codes to half a wave, 23.3 / 24.7 and 52.6 / 55.0 below; fp4, a
                    // line to a wave, the exchange of four nodes with both constraints 113.9 / 110.4)
                    if (FMT == HSADMM_MX_FP8) __builtin_nontemporal_store(code, reinterpret_cast<unsigned int*>(codes + g));
                    else *reinterpret_cast<uint16_t*>(codes + (g >> 1)) = (uint16_t)code;
                    if ((threadIdx.x & 7) == 0) scales[g / kMxBlock] = (uint8_t)byte;
                }
            };
            if (!channels && (row_len & 3) == 0) {
                v4f x[Q], y[Q];
                unsigned int o[Q];
                bool on[Q];
#pragma unroll
                for (int h = 0; h < Q; ++h) {
                    const int place = 4 * (threadIdx.x + h * kBlock) - lead;
                    on[h] = place >= 0 && (unsigned int)place < there;
                    const unsigned int j = c0 + (on[h] ? (unsigned int)place : 0u);
                    const unsigned int dp = by_row(j);
                    o[h] = (listed ? (unsigned int)rows[p0 + dp] : p0 + dp) * row_len + (j - dp * out_len);
                    x[h] = y[h] = v4f{0.f, 0.f, 0.f, 0.f};
                }
#pragma unroll
                for (int h = 0; h < Q; ++h)
                    if (on[h]) { x[h] = ld4(base + o[h]); if (SUM) y[h] = ld4(base1 + o[h]); }
#pragma unroll
                for (int h = 0; h < Q; ++h) put(4 * (threadIdx.x + h * kBlock), SUM ? x[h] + y[h] : x[h]);
            } else {
                // columns of rows, and rows that start anywhere: a position to a lane, in order through LDS.  A lane's next
                // position is kBlock further: so many rows, channels and elements of a channel.
                auto parts = [&](auto with_columns) {
                    constexpr bool kColumns = decltype(with_columns)::value;
                    constexpr int kEach = kPart / kBlock;
                    const unsigned int unit = kColumns ? khw : 1u;
                    const unsigned int width = kColumns ? out_len / khw : out_len;          // channels of a packed row
                    const DivPos by_unit(unit);
                    const unsigned int step_p = kBlock / out_len, step_c = kBlock - step_p * out_len;
                    const unsigned int step_q = kColumns ? step_c / unit : step_c, step_t = step_c - step_q * unit;
                    const unsigned int j = c0 + threadIdx.x, dp = by_row(j);
                    unsigned int p = p0 + dp, q = j - dp * out_len, t = 0;
                    if (kColumns) { t = q; q = by_unit(q); t -= q * unit; }
                    const int most = min(kTile - lead, (int)min(there + kMxBlock - 1, (unsigned int)kTile) & ~(kMxBlock - 1));
                    for (int part = 0; part < most; part += kPart) {
                        unsigned int o[kEach];
                        bool on[kEach];
                        float x[kEach], y[kEach];
#pragma unroll
                        for (int k = 0; k < kEach; ++k) {
                            on[k] = (unsigned int)(part + (int)threadIdx.x + k * kBlock) < there;
                            const unsigned int row = on[k] ? p : 0u, col = on[k] ? q : 0u;
                            o[k] = (listed ? (unsigned int)rows[row] : row) * row_len +
                                   (kColumns ? (unsigned int)cols[col] * unit + t : col);
                            p += step_p;
                            q += step_q;
                            if (kColumns) { t += step_t; if (t >= unit) { t -= unit; ++q; } }
                            if (q >= width) { q -= width; ++p; }
                        }
#pragma unroll
                        for (int k = 0; k < kEach; ++k) {
                            x[k] = on[k] ? ld1(base + o[k]) : 0.f;
                            if (SUM) y[k] = on[k] ? ld1(base1 + o[k]) : 0.f;
                        }
                        __syncthreads();                       // (the stage may still be read for the part before)
#pragma unroll
                        for (int k = 0; k < kEach; ++k) stage[threadIdx.x + k * kBlock] = SUM ? x[k] + y[k] : x[k];
                        __syncthreads();
#pragma unroll
                        for (int h = 0; h < kEach / 4; ++h) {
                            const int at = 4 * (threadIdx.x + h * kBlock);
                            put(lead + part + at, *reinterpret_cast<const v4f*>(stage + at));
                        }
                    }
                };
                if (channels) parts(std::true_type{});
                else parts(std::false_type{});
            }
        }
    }
    // the caller's copies of the kept lists and the offsets
    const int kept = mp.cnt[2 * nL - 1] + mp.cnt[nL - 1] + mp.cnt[3 * nL - 1];
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < kept; i += (int64_t)gridDim.x * kBlock)
        co.kept_idx[i] = mp.kept_idx[i];
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i <= nL; i += (int64_t)gridDim.x * kBlock)
        co.layer_off[i] = mp.layer_off[i];
}

// ------------------------------------------------------------------ reading

struct MxBuffers {
    const uint8_t* codes[HSADMM_MAX_MASKS];
    const uint8_t* scales[HSADMM_MAX_MASKS];
};

// 2^(byte - 127); 255 is NaN.
__device__ __forceinline__ float mx_scale(unsigned int byte)
{
    const unsigned int b = max(byte << 23, 0x400000u);
    return __uint_as_float(byte == 255u ? 0x7fc00000u : b);
}

// Four values from their codes (fp8: four bytes, fp4: the low two).
template <int FMT>
__device__ __forceinline__ v4f mx_decode4(unsigned int c, float scale)
{
    v2f lo, hi;
    if (FMT == HSADMM_MX_FP8) {
        lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false);
        hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    } else {
        lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0);
        hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1);
    }
    const v4f v = {lo.x, lo.y, hi.x, hi.y};
    return v * scale;
}

// The codes at positions k .. k + 3, k a multiple of 4.
template <int FMT>
__device__ __forceinline__ unsigned int mx_codes4(const uint8_t* codes, int64_t k)
{
    if (FMT == HSADMM_MX_FP8) return *reinterpret_cast<const unsigned int*>(codes + k);
    return *reinterpret_cast<const uint16_t*>(codes + (k >> 1));
}

// The mean over the buffers of the values at positions k .. k + 3, k a multiple of 4: ((d_0 + d_1) + ...) / M.  Four buffers'
// loads are in flight at once.
template <int FMT>
__device__ __forceinline__ v4f mx_mean4(const MxBuffers& b, int M, float inv_M, int64_t k)
{
    v4f z = {0.f, 0.f, 0.f, 0.f};
    int m = 0;
    for (; m + 4 <= M; m += 4) {
        unsigned int c[4], s[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) { c[j] = mx_codes4<FMT>(b.codes[m + j], k); s[j] = b.scales[m + j][k / kMxBlock]; }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const v4f d = mx_decode4<FMT>(c[j], mx_scale(s[j]));
            z = m + j == 0 ? d : z + d;                 // (0 + -0 would lose the sign)
        }
    }
    for (; m < M; ++m) {
        const v4f d = mx_decode4<FMT>(mx_codes4<FMT>(b.codes[m], k), mx_scale(b.scales[m][k / kMxBlock]));
        z = m == 0 ? d : z + d;
    }
    return z * inv_M;
}

// Smallest `lo` and largest `hi` of the workgroup, in every thread; `red`: two rows of kWaves words.
__device__ __forceinline__ void block_range(unsigned int& lo, unsigned int& hi, unsigned int (&red)[2][kWaves])
{
    lo = ~wave_umax(~lo);
    hi = wave_umax(hi);
    if ((threadIdx.x & (kWave - 1)) == 0) { red[0][threadIdx.x / kWave] = lo; red[1][threadIdx.x / kWave] = hi; }
    __syncthreads();
    lo = min(min(red[0][0], red[0][1]), min(red[0][2], red[0][3]));
    hi = max(max(red[1][0], red[1][1]), max(red[1][2], red[1][3]));
}

// dst <- the mean of M buffers on the kept elements, +0 elsewhere; DUAL: Vd <- Vd + (Zi - dst).  A workgroup takes a part
// of a flat item, a thread fours of adjacent elements.  Fours of rows that are packed whole and in whole words come straight from the
// buffers.  Other rows' elements (columns of a row, rows that start anywhere) have their places in one stretch of packed
// positions: the workgroup finds where it starts and ends, decodes it in order into LDS, a code once, and picks from there.
// An element's row, channel and column follow from the one before it; a four that lies in one row looks its row up once.
// Bound by HBM where rows are whole (ResNet-50, filters, eight nodes in fp8, with the dual update: 502 MB in 78.5 us, 6.4 TB/s), by the
// places' arithmetic and the three loads one after the other where they are not.  Measured, us:
//   an element at a time out of the buffers     ResNet-50, both constraints, four nodes in fp4: 113.0, this way 82.7, with every wave
//                                               there is 77.8; ResNet-18 of width 45, filters, two nodes in fp8: 9.7 / 8.9
//   two divisions for every element             basic 3-3-1-2 of width 120, channels, three nodes in fp4: 61.5, step by step 46.5,
//                                               whole fours 44.0; ResNet-50, channels, one node in fp8: 36.8, 30.4, 26.9
//   seven / eight waves a SIMD                  with the dual update 103.0 / 105.5 (writing and reading, as above), 78.5 / 79.2;
//                                               without 46.1 / 43.6, 41.1 / 37.8 (ResNet-18 of width 125, filters), 22.0 / 20.5
template <int FMT, bool DUAL>
__global__ __launch_bounds__(kBlock, DUAL ? 7 : 8) void scatter_mx(const FlatItem* __restrict__ items, const DevLayer* __restrict__ layers,
                                                     MxBuffers b, int M, float inv_M, MxMaps mp, float* __restrict__ dst,
                                                     const float* __restrict__ Zi, float* __restrict__ Vd)
{
    __shared__ __align__(16) float stage[kPartElems + kMxBlock];
    __shared__ unsigned int red[2][kWaves];
    FlatItem it = items[blockIdx.x / kParts];
    const int skip = (int)(blockIdx.x % kParts) * kPartElems;
    if (it.n <= skip) return;
    it.base += skip;
    it.n = min(it.n - skip, kPartElems);
    const int l = it.layer;
    const DevLayer& L = layers[l];
    const int mode = L.mode;
    const bool channels = mode_has_channels(mode);
    const unsigned int khw = (unsigned int)L.khw, row_len = (unsigned int)L.row_len;
    const unsigned int n0 = (unsigned int)mp.cnt[l], n1 = (unsigned int)mp.cnt[2 * mp.n_layers + l];
    const unsigned int in_len = !channels ? row_len : (mode == HSADMM_MODE_BOTH ? n1 : n0) * khw;
    const int32_t* row_pos = mode == HSADMM_MODE_FILTER || mode == HSADMM_MODE_BOTH ? mp.pos + L.group_base : nullptr;
    const int32_t* col_pos = mp.pos + L.group_base + (mode == HSADMM_MODE_BOTH ? L.c_out : 0);
    const int64_t seg = mp.layer_off[l];
    const unsigned int i0 = (unsigned int)(it.base - L.elem_off);
    const unsigned int r0 = i0 / row_len, c0 = i0 - r0 * row_len;
    const DivPos by_row(row_len), by_khw(khw);
    v4f z[kFlatQuads], zi[kFlatQuads], vd[kFlatQuads];
    if (DUAL) {
#pragma unroll
        for (int h = 0; h < kFlatQuads; ++h) {
            const int q = 4 * (threadIdx.x + h * kBlock), nv = min(4, it.n - q);
            zi[h] = load4<HSADMM_TYPE_F32>(Zi + it.base + q, nv);
            vd[h] = load4<HSADMM_TYPE_F32>(Vd + it.base + q, nv);
        }
    }
    if (!channels && (row_len & 3) == 0) {
#pragma unroll
        for (int h = 0; h < kFlatQuads; ++h) {
            const int q = 4 * (threadIdx.x + h * kBlock);
            z[h] = v4f{0.f, 0.f, 0.f, 0.f};
            if (q >= it.n) continue;
            const unsigned int dr = by_row(c0 + q), row = r0 + dr;
            const int p = row_pos ? row_pos[row] : (int)row;
            if (p >= 0) z[h] = mx_mean4<FMT>(b, M, inv_M, seg + (int64_t)p * row_len + (c0 + q - dr * row_len));
        }
    } else {
        constexpr unsigned int kNone = 0xffffffffu;
        unsigned int k[kFlatQuads][4], first = kNone, last = 0;
        // kColumns: channels are kept, each a run of khw columns (kRuns: of more than one); kWhole: a four lies in one row
        auto places = [&](auto with_columns, auto with_runs, auto whole) {
            constexpr bool kColumns = decltype(with_columns)::value, kRuns = decltype(with_runs)::value;
            constexpr bool kWhole = decltype(whole)::value;
            unsigned int row[kFlatQuads][4], add[kFlatQuads][4];
            int pc[kFlatQuads][4], pr[kFlatQuads][4];
#pragma unroll
            for (int h = 0; h < kFlatQuads; ++h) {
                // row, channel and column in the channel of the four's first element; the others follow step by step
                const unsigned int q = (unsigned int)min(4 * (int)(threadIdx.x + h * kBlock), kWhole ? it.n - 4 : it.n - 1);
                const unsigned int dr = by_row(c0 + q);
                unsigned int r = r0 + dr, ch = c0 + q - dr * row_len, t = 0;
                if (kRuns) { t = ch; ch = by_khw(ch); t -= ch * khw; }
                const unsigned int width = kColumns ? (unsigned int)L.c_in : row_len;
                if (kWhole && kColumns && !kRuns) {
                    const int4_at4 v = *reinterpret_cast<const int4_at4*>(col_pos + ch);
                    pc[h][0] = v.x; pc[h][1] = v.y; pc[h][2] = v.z; pc[h][3] = v.w;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool in = kWhole || (int)q + e < it.n;     // (else the four's first element's look-ups again)
                    row[h][e] = in ? r : row[h][0];
                    add[h][e] = kRuns ? t : kColumns ? 0u : ch;
                    if (!kColumns) pc[h][e] = 0;
                    else if (!kWhole || kRuns) pc[h][e] = col_pos[in ? ch : 0u];
                    if (!kRuns || ++t == khw) {
                        t = 0;
                        if (++ch == width && !kWhole) { ch = 0; ++r; }
                    }
                }
            }
#pragma unroll
            for (int h = 0; h < kFlatQuads; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    pr[h][e] = !row_pos ? (int)row[h][e] : kWhole && e > 0 ? pr[h][0] : row_pos[row[h][e]];
#pragma unroll
            for (int h = 0; h < kFlatQuads; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool on = 4 * (int)(threadIdx.x + h * kBlock) + e < it.n && pr[h][e] >= 0 && pc[h][e] >= 0;
                    const unsigned int at = (unsigned int)pr[h][e] * in_len +
                                            (kRuns ? (unsigned int)pc[h][e] * khw : (unsigned int)pc[h][e]) + add[h][e];
                    k[h][e] = on ? at : kNone;
                    first = min(first, k[h][e]);
                    last = max(last, on ? at : 0u);
                }
        };
        const std::true_type yes{};
        const std::false_type no{};
        const bool fours = (row_len & 3) == 0;
        if (!channels) places(no, no, no);
        else if (khw == 1) fours ? places(yes, no, yes) : places(yes, no, no);
        else fours ? places(yes, yes, yes) : places(yes, yes, no);
        block_range(first, last, red);
        const unsigned int from = first & ~(unsigned int)(kMxBlock - 1);
        if (first != kNone)
            for (unsigned int o = 4 * threadIdx.x; from + o <= last; o += 4 * kBlock)
                *reinterpret_cast<v4f*>(stage + o) = mx_mean4<FMT>(b, M, inv_M, seg + from + o);
        __syncthreads();
#pragma unroll
        for (int h = 0; h < kFlatQuads; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) z[h][e] = k[h][e] == kNone ? 0.f : stage[k[h][e] - from];
    }
#pragma unroll
    for (int h = 0; h < kFlatQuads; ++h) {
        const int q = 4 * (threadIdx.x + h * kBlock), nv = min(4, it.n - q);
        if (nv <= 0) continue;
        store4<HSADMM_TYPE_F32>(dst + it.base + q, z[h], nv);
        if (DUAL) store4<HSADMM_TYPE_F32>(Vd + it.base + q, vd[h] + (zi[h] - z[h]), nv);
    }
}

}  // namespace
#endif
