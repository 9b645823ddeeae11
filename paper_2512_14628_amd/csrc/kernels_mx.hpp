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

// j / d for the unsigned numbers a layer's positions are (see DivKhw).
struct DivPos {
    unsigned int d;
    float rcp;
    __device__ __forceinline__ explicit DivPos(unsigned int x) : d(x), rcp(1.0f / (float)x) {}
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

// Eight values of a block (32 values in four adjacent lanes) -> their codes; the block's scale byte.
// The scale is the least 2^e with largest <= 2^e * top (top = 448 = 1.75 * 2^8, or 6 = 1.5 * 2^2): the largest's exponent less
// the format's, one more where its fraction is above top's.  The product with 2^-e is exact (or far below half of the smallest
// code), so a code is the nearest value, ties to even.
template <int FMT>
__device__ __forceinline__ void mx_encode(const float (&x)[8], unsigned int (&codes)[2], unsigned int& byte)
{
    unsigned int top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    top = max(top, row_exchange<kDppXor1>(top));
    top = max(top, row_exchange<kDppXor2>(top));
    constexpr int kExp = FMT == HSADMM_MX_FP8 ? 8 : 2;
    constexpr unsigned int kFrac = FMT == HSADMM_MX_FP8 ? 0x600000u : 0x400000u;
    const int e = (int)(top >> 23) - kExp + ((top & 0x7fffffu) > kFrac ? 1 : 0);
    const bool bad = top >= 0x7f800000u;                 // an infinity or a NaN: the block reads back as NaN
    byte = bad ? 255u : (unsigned int)max(e, 0);
    const float f = __uint_as_float((254u - (unsigned int)max(e, 0)) << 23);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = bad ? 0.f : x[i] * f;
    // With the largest scale the codes from the next power of two on stand for 2^128 and more: values next to the end of fp32's
    // range, which would read back as infinite, take the code below.
    constexpr int kTopByte = 254 - kExp + 1;
    constexpr float kTopCode = FMT == HSADMM_MX_FP8 ? 240.0f : 3.0f;
    if (e == kTopByte) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = __builtin_amdgcn_fmed3f(y[i], -kTopCode, kTopCode);
    }
    if (FMT == HSADMM_MX_FP8) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            int c = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h], y[4 * h + 1], 0, false);
            codes[h] = (unsigned int)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h + 2], y[4 * h + 3], c, true);
        }
    } else {
        unsigned int c = 0;
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[0], y[1], 1.0f, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[2], y[3], 1.0f, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[4], y[5], 1.0f, 2);
        codes[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[6], y[7], 1.0f, 3);
        codes[1] = 0;
    }
}

// One workgroup per flat item, taken as a stretch of the layer's packed positions: a layer packs at most all of its
// elements, and the workgroups past what it does pack return.  Eight adjacent positions a thread.
template <int FMT, bool SUM>
__global__ __launch_bounds__(kBlock) void gather_mx(const FlatItem* __restrict__ items, const DevLayer* __restrict__ layers,
                                                    const float* __restrict__ src, const float* __restrict__ src1, MxMaps mp,
                                                    uint8_t* __restrict__ codes, uint8_t* __restrict__ scales, CopyOut co)
{
    const FlatItem it = items[blockIdx.x];
    const int l = it.layer;
    const DevLayer& L = layers[l];
    const unsigned int i0 = (unsigned int)(it.base - L.elem_off);
    if (i0 == 0) copy_out_layer(l, mp.cnt, mp.kept_idx, mp.n_layers, mp.layer_off, co);
    const int mode = L.mode;
    const bool channels = mode_has_channels(mode);
    const unsigned int n0 = (unsigned int)mp.cnt[l], n1 = (unsigned int)mp.cnt[2 * mp.n_layers + l];
    const int32_t* rows = mp.kept_idx + mp.cnt[mp.n_layers + l];          // kept filters, where there are any
    const int32_t* cols = rows + (mode == HSADMM_MODE_BOTH ? n0 : 0);
    const unsigned int khw = (unsigned int)L.khw, row_len = (unsigned int)L.row_len;
    const unsigned int out_len = !channels ? row_len : (mode == HSADMM_MODE_BOTH ? n1 : n0) * khw;   // of a packed row
    const unsigned int out_rows = mode == HSADMM_MODE_FILTER || mode == HSADMM_MODE_BOTH ? n0 : (unsigned int)L.c_out;
    const unsigned int size = out_rows * out_len;                          // (at most the layer's elements: below 2^31)
    if (i0 >= size) return;
    const unsigned int p0 = i0 / out_len, c0 = i0 - p0 * out_len;
    const bool listed = mode == HSADMM_MODE_FILTER || mode == HSADMM_MODE_BOTH;
    const float* base = src + L.elem_off;
    const float* base1 = SUM ? src1 + L.elem_off : nullptr;
    const DivPos by_row(out_len), by_khw(khw);
    const unsigned int i = i0 + 8 * threadIdx.x;
    float x[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const unsigned int j = c0 + 8 * threadIdx.x + 4 * h;
        const unsigned int dp = by_row(j);
        unsigned int p = p0 + dp, c = j - dp * out_len;
        const unsigned int left = i + 4 * h < size ? size - (i + 4 * h) : 0;      // positions there still are
        if (!channels && left >= 4 && c + 4 <= row_len) {
            const int64_t o = (int64_t)(listed ? rows[p] : (int)p) * row_len + c;
            v4f v = ld4(base + o);
            if (SUM) v = v + ld4(base1 + o);
            x[4 * h] = v.x; x[4 * h + 1] = v.y; x[4 * h + 2] = v.z; x[4 * h + 3] = v.w;
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float v = 0.f;
                if ((unsigned int)k < left) {
                    unsigned int col = c;
                    if (channels) {
                        const unsigned int q = khw == 1 ? c : by_khw(c);
                        col = (unsigned int)cols[q] * khw + (c - q * khw);
                    }
                    const int64_t o = (int64_t)(listed ? rows[p] : (int)p) * row_len + col;
                    v = SUM ? base[o] + base1[o] : base[o];
                    if (++c == out_len) { c = 0; ++p; }
                }
                x[4 * h + k] = v;
            }
        }
    }
    unsigned int code[2], byte;
    mx_encode<FMT>(x, code, byte);
    if ((i & ~(unsigned int)(kMxBlock - 1)) >= size) return;
    const int64_t o = mp.layer_off[l] + i;
    if (FMT == HSADMM_MX_FP8) *reinterpret_cast<uint2*>(codes + o) = uint2{code[0], code[1]};
    else *reinterpret_cast<unsigned int*>(codes + (o >> 1)) = code[0];
    if ((threadIdx.x & 3) == 0) scales[o / kMxBlock] = (uint8_t)byte;
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

// The value at packed position k of a buffer.
template <int FMT>
__device__ __forceinline__ float mx_value(const uint8_t* codes, const uint8_t* scales, int64_t k)
{
    const float s = mx_scale(scales[k / kMxBlock]);
    if (FMT == HSADMM_MX_FP8) { const v2f v = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[k], false); return v.x * s; }
    const unsigned int c = codes[k >> 1];
    const v2f v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0);
    return ((k & 1) ? v.y : v.x) * s;
}

// The values at packed positions k .. k + 3, k a multiple of 4.
template <int FMT>
__device__ __forceinline__ v4f mx_value4(const uint8_t* codes, const uint8_t* scales, int64_t k)
{
    const float s = mx_scale(scales[k / kMxBlock]);
    v2f lo, hi;
    if (FMT == HSADMM_MX_FP8) {
        const unsigned int c = *reinterpret_cast<const unsigned int*>(codes + k);
        lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false);
        hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    } else {
        const unsigned int c = *reinterpret_cast<const uint16_t*>(codes + (k >> 1));
        lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0);
        hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1);
    }
    const v4f v = {lo.x, lo.y, hi.x, hi.y};
    return v * s;
}

// dst <- the mean of M buffers on the kept elements, +0 elsewhere; DUAL: Vd <- Vd + (Zi - dst).  A workgroup takes a flat
// item, a thread fours of adjacent elements.
template <int FMT, bool DUAL>
__global__ __launch_bounds__(kBlock) void scatter_mx(const FlatItem* __restrict__ items, const DevLayer* __restrict__ layers,
                                                     MxBuffers b, int M, float inv_M, MxMaps mp, float* __restrict__ dst,
                                                     const float* __restrict__ Zi, float* __restrict__ Vd)
{
    const FlatItem it = items[blockIdx.x];
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
#pragma unroll
    for (int h = 0; h < kFlatQuads; ++h) {
        const int q = 4 * (threadIdx.x + h * kBlock);
        const int nv = min(4, it.n - q);
        if (nv <= 0) continue;
        const unsigned int dr = by_row(c0 + q);
        unsigned int row = r0 + dr, c = c0 + q - dr * row_len;
        v4f z = {0.f, 0.f, 0.f, 0.f};
        if (!channels && (row_len & 3) == 0) {
            const int p = row_pos ? row_pos[row] : (int)row;
            if (p >= 0) {
                const int64_t k = seg + (int64_t)p * row_len + c;
                z = mx_value4<FMT>(b.codes[0], b.scales[0], k);
                for (int m = 1; m < M; ++m) z = z + mx_value4<FMT>(b.codes[m], b.scales[m], k);
                z = z * inv_M;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (e >= nv) continue;
                const int p = row_pos ? row_pos[row] : (int)row;
                int64_t k = -1;
                if (p >= 0) {
                    if (!channels) k = (int64_t)p * row_len + c;
                    else {
                        const unsigned int ch = khw == 1 ? c : by_khw(c);
                        const int pc = col_pos[ch];
                        if (pc >= 0) k = (int64_t)p * in_len + (unsigned int)pc * khw + (c - ch * khw);
                    }
                }
                if (k >= 0) {
                    k += seg;
                    float v = mx_value<FMT>(b.codes[0], b.scales[0], k);
                    for (int m = 1; m < M; ++m) v = v + mx_value<FMT>(b.codes[m], b.scales[m], k);
                    z[e] = v * inv_M;
                }
                if (++c == row_len) { c = 0; ++row; }
            }
        }
        const int64_t o = it.base + q;
        store4<HSADMM_TYPE_F32>(dst + o, z, nv);
        if (DUAL) {
            const v4f d = load4<HSADMM_TYPE_F32>(Zi + o, nv) - z;
            store4<HSADMM_TYPE_F32>(Vd + o, load4<HSADMM_TYPE_F32>(Vd + o, nv) + d, nv);
        }
    }
}

}  // namespace
#endif
