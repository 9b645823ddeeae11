// hsadmm_gradient_norms / hsadmm_adamw: the replicas' own training step between two steps of the consensus (Algorithm 1,
// Phase 1; Eq. (7) with AdamW), all layers of all replicas in one launch.
// Part of the single translation unit built from hsadmm.hip (included there, in order).
#ifndef KERNELS_TRAINING_HPP
#define KERNELS_TRAINING_HPP
#include "hsadmm_device.hpp"
#include "kernels_select.hpp"

namespace {

// ------------------------------------------------------------------ flat items

// kFlatElems consecutive elements of one layer (fewer at its end): the table of the kernels that do not care about groups.  A
// workgroup takes a part of an item: kPartElems elements, kFlatQuads fours of adjacent elements a thread, kBlock fours apart, or
// (adamw_kernel) one four a thread.  A wave's access is contiguous and a wave's 64 fours are one state block.
// (An item per workgroup instead, for the largest networks, adds a tenth to the time a plan takes to make.)
constexpr int kStateBlock = 256;
constexpr int kFlatElems = 8192;
constexpr int kFlatQuads = 2;
constexpr int kPartElems = 4 * kFlatQuads * kBlock;
constexpr int kParts = kFlatElems / kPartElems;
constexpr int kAdamwElems = 4 * kBlock;                // of a workgroup of adamw_kernel
static_assert(kStateBlock == 4 * kWave, "a wave's fours are one state block");

struct FlatItem {
    int64_t base;      // arena element of the item's first element (a multiple of 4)
    int64_t block0;    // state block of the item's first element
    int32_t n;         // elements
    int32_t layer;
};
static_assert(sizeof(FlatItem) == 24, "FlatItem layout");

typedef __bf16 v4bf __attribute__((ext_vector_type(4)));
typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));

template <int T> struct ElemOf { typedef float type; typedef v4f vec; };
template <> struct ElemOf<HSADMM_TYPE_BF16> { typedef __bf16 type; typedef v4bf vec; };
template <> struct ElemOf<HSADMM_TYPE_F16> { typedef _Float16 type; typedef v4h vec; };

// Four elements of type T at p as fp32, the first nv of them (1 to 4; the others are 0).
template <int T>
__device__ __forceinline__ v4f load4(const typename ElemOf<T>::type* p, int nv)
{
    if (nv == 4)
        return __builtin_convertvector(__builtin_nontemporal_load(reinterpret_cast<const typename ElemOf<T>::vec*>(p)), v4f);
    v4f v = {0.f, 0.f, 0.f, 0.f};
    if (nv > 0) v.x = (float)p[0];
    if (nv > 1) v.y = (float)p[1];
    if (nv > 2) v.z = (float)p[2];
    return v;
}

// The first nv of four values to p, rounded to nearest.
template <int T>
__device__ __forceinline__ void store4(typename ElemOf<T>::type* p, const v4f& v, int nv)
{
    typedef typename ElemOf<T>::type E;
    if (nv == 4) {
        __builtin_nontemporal_store(__builtin_convertvector(v, typename ElemOf<T>::vec),
                                    reinterpret_cast<typename ElemOf<T>::vec*>(p));
        return;
    }
    if (nv > 0) p[0] = (E)v.x;
    if (nv > 1) p[1] = (E)v.y;
    if (nv > 2) p[2] = (E)v.z;
}

// ------------------------------------------------------------------ gradient norms

struct GradArgs { const void* G[HSADMM_MAX_REPLICAS]; };

// Sums of squares in fp64 (the square of an fp32 value is exact there): workgroup p of a replica's P takes the parts of the flat
// items p, p + P, ...; the order of the additions depends on the plan and the number of replicas only.  Bound by HBM: ResNet-152, 8
// replicas in bf16, 961 MB in 144 us (6.7 TB/s) and 4.7 in gradient_norm_finish; ResNet-18, one in fp32, 47 MB in 9.8 us and 1.9 or, in
// other runs, 3.9.  (Two to four parts in flight, both launches together: 149 to 156 us for 148, and small networks lose a microsecond
// or two.)
template <int T>
__global__ __launch_bounds__(kBlock) void gradient_sqsums(const FlatItem* __restrict__ items, int n_items, GradArgs a, int P,
                                                          double* __restrict__ part)
{
    __shared__ double red[kWaves];
    const int r = blockIdx.x / P, p = blockIdx.x - r * P;
    const typename ElemOf<T>::type* G = static_cast<const typename ElemOf<T>::type*>(a.G[r]);
    double s0 = 0.0, s1 = 0.0, s2 = 0.0, s3 = 0.0;
    for (int64_t i = p; i < (int64_t)n_items * kParts; i += P) {
        FlatItem it = items[i / kParts];
        const int skip = (int)(i % kParts) * kPartElems;
        it.base += skip;
        it.n -= skip;
        v4f g[kFlatQuads];
        // (whole parts apart: a load whose length is looked at is converted, and so waited for, where it stands: 177 us above)
        if (it.n >= kPartElems) {
#pragma unroll
            for (int k = 0; k < kFlatQuads; ++k) g[k] = load4<T>(G + it.base + 4 * (threadIdx.x + k * kBlock), 4);
        } else {
#pragma unroll
            for (int k = 0; k < kFlatQuads; ++k) {
                const int q = 4 * (threadIdx.x + k * kBlock);
                g[k] = load4<T>(G + it.base + q, min(4, it.n - q));
            }
        }
#pragma unroll
        for (int k = 0; k < kFlatQuads; ++k) {
            s0 = fma((double)g[k].x, (double)g[k].x, s0);
            s1 = fma((double)g[k].y, (double)g[k].y, s1);
            s2 = fma((double)g[k].z, (double)g[k].z, s2);
            s3 = fma((double)g[k].w, (double)g[k].w, s3);
        }
    }
    const double s = wave_xor_sum((s0 + s1) + (s2 + s3), kWave);
    if ((threadIdx.x & (kWave - 1)) == 0) red[threadIdx.x / kWave] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        double t = red[0];
        for (int w = 1; w < kWaves; ++w) t += red[w];
        part[blockIdx.x] = t;
    }
}

// One workgroup per replica: norm = sqrt(sum), scale = min(1, max_norm / norm), NaN where the norm is not finite.
__global__ __launch_bounds__(kBlock) void gradient_norm_finish(const double* __restrict__ part, int P, double max_norm,
                                                               double* __restrict__ norm, float* __restrict__ scale)
{
    __shared__ double red[kWaves];
    double s = 0.0;
    for (int i0 = 0; i0 < P; i0 += 8 * kBlock) {           // (eight loads in flight)
        double x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int i = i0 + k * kBlock + (int)threadIdx.x;
            x[k] = i < P ? part[(int64_t)blockIdx.x * P + i] : 0.0;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) s += x[k];
    }
    s = wave_xor_sum(s, kWave);
    if ((threadIdx.x & (kWave - 1)) == 0) red[threadIdx.x / kWave] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        double t = red[0];
        for (int w = 1; w < kWaves; ++w) t += red[w];
        t = sqrt(t);
        if (norm) norm[blockIdx.x] = t;
        if (scale) {
            const bool finite = t <= 1.7976931348623157e308;          // (a NaN fails the comparison)
            scale[blockIdx.x] = !finite ? __builtin_nanf("") : t > max_norm ? (float)(max_norm / t) : 1.0f;
        }
    }
}

// ------------------------------------------------------------------ AdamW

struct AdamwArgs {
    float* W[HSADMM_MAX_REPLICAS];
    const void* G[HSADMM_MAX_REPLICAS];
    void* M[HSADMM_MAX_REPLICAS];          // fp32, or e4m3 codes with the scales Ms
    void* V[HSADMM_MAX_REPLICAS];          // fp32 second moments, or codes of their roots with the scales Vs
    float* Ms[HSADMM_MAX_REPLICAS];
    float* Vs[HSADMM_MAX_REPLICAS];
    void* Wl[HSADMM_MAX_REPLICAS];         // LOW: the weights rounded to the gradients' type
    const float* Z;                        // PROX: z_i, the replica-mean dual, rho_1 per layer
    const float* U;
    const float* rho;
    const float* grad_scale;               // may be null
    const hsadmm_adamw_coef_t* coef_dev;   // may be null: coef
    hsadmm_adamw_coef_t coef;
    float beta1, one_minus_beta1, beta2, one_minus_beta2, eps;
};

// Largest of the wave's values, in every lane: four exchanges inside the rows of 16 lanes, then the four rows.
__device__ __forceinline__ unsigned int wave_umax(unsigned int x)
{
    x = max(x, row_exchange<kDppXor1>(x));
    x = max(x, row_exchange<kDppXor2>(x));
    x = max(x, row_exchange<kDppHalfMirror>(x));
    x = max(x, row_exchange<kDppMirror>(x));
    return max(max(lane_value(x, 0), lane_value(x, 16)), max(lane_value(x, 32), lane_value(x, 48)));
}

// The four values of a lane's four, from codes and the block's scale.
__device__ __forceinline__ v4f decode4(unsigned int codes, float scale)
{
    const v2f lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
    const v4f v = {lo.x, lo.y, hi.x, hi.y};
    return v * scale;
}

// Rounding numbers of a four: 32 bits each, of which the conversion uses the upper 20.  One mix per four (two
// multiplications by odd numbers, two shifts), then a multiplication by an odd number of each element's own: neighbours'
// numbers need not be independent of each other, an element's numbers of different steps do.
constexpr unsigned int kMix1 = 0x6A09E667u, kMix2 = 0xBB67AE85u, kMix3 = 0x3C6EF373u;
__device__ __forceinline__ unsigned int mix_four(unsigned int x)
{
    x *= kMix1;
    x = (x ^ (x >> 16)) * kMix2;
    return x ^ (x >> 15);
}

// Codes of four values y (already in units of the scale): rounded stochastically to e4m3, |y| <= 448.  (To nearest, a state that moves
// by less than half a code a step, as every root under beta_2 = 0.999 does, would not move at all.)
__device__ __forceinline__ unsigned int encode4(const v4f& y, unsigned int mix)
{
    int c = 0;
    c = __builtin_amdgcn_cvt_sr_fp8_f32(y.x, (int)mix, c, 0);
    c = __builtin_amdgcn_cvt_sr_fp8_f32(y.y, (int)(mix * kMix1), c, 1);
    c = __builtin_amdgcn_cvt_sr_fp8_f32(y.z, (int)(mix * kMix2), c, 2);
    c = __builtin_amdgcn_cvt_sr_fp8_f32(y.w, (int)(mix * kMix3), c, 3);
    return (unsigned int)c;
}

__device__ __forceinline__ unsigned int load_codes(const uint8_t* p, int nv)
{
    if (nv == 4) return __builtin_nontemporal_load(reinterpret_cast<const unsigned int*>(p));
    unsigned int c = 0;
    for (int i = 0; i < 3; ++i)
        if (i < nv) c |= (unsigned int)p[i] << (8 * i);
    return c;
}

__device__ __forceinline__ void store_codes(uint8_t* p, unsigned int c, int nv)
{
    if (nv == 4) { __builtin_nontemporal_store(c, reinterpret_cast<unsigned int*>(p)); return; }
    for (int i = 0; i < 3; ++i)
        if (i < nv) p[i] = (uint8_t)(c >> (8 * i));
}

// A block whose largest magnitude is below this is held as zero: its reciprocal would leave fp32's normal range.
constexpr float kStateFloor = 0x1p-100f;

// A block's scale (largest magnitude / 448) and what brings its values into units of it.  `top`: the bits of the largest
// magnitude; the bits of a NaN or an infinity are larger than any number's, so such a block's scale is not finite.
__device__ __forceinline__ float block_scale(unsigned int top, float& to_units)
{
    const float t = __uint_as_float(top);
    const bool none = t < kStateFloor;
    const float r = __builtin_amdgcn_rcpf(t);
    to_units = none ? 0.f : __builtin_fmaf(__builtin_fmaf(-t, r, 1.0f), r, r) * 448.0f;
    return none ? 0.f : t * (1.0f / 448.0f);
}

__device__ __forceinline__ unsigned int top_bits(const v4f& v)
{
    const unsigned int m = 0x7fffffffu;
    return max(max(__float_as_uint(v.x) & m, __float_as_uint(v.y) & m), max(__float_as_uint(v.z) & m, __float_as_uint(v.w) & m));
}

// The roots of four numbers >= 0 to nearest: the machine's reciprocal root and one correction of x times it (compared with the rounded
// fp64 root for every fp32 number on gfx950: no difference).  Codes are cut from the root and the moments, and a result that is one
// unit in the last place off moves a code in every millionth case.  Below 2^-64 the correction's remainder would leave fp32's
// normal range, below 2^-126 x itself: fours that hold such a number take the roots of 2^64 x there, behind a branch that most
// waves jump (without it ResNet-50, four times wider 1018 us instead of 1014).  Infinity's root is infinity.
__device__ __forceinline__ float root_of(float x)
{
    const float y = __builtin_amdgcn_rsqf(fmaxf(x, 0x1p-126f));
    const float s = x * y;
    const float r = __builtin_fmaf(__builtin_fmaf(-s, s, x), 0.5f * y, s);
    return x == __builtin_inff() ? x : r;
}

__device__ __forceinline__ v4f roots_of(const v4f& x)
{
    v4f r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = root_of(x[i]);
    if (__builtin_expect(fminf(fminf(x[0], x[1]), fminf(x[2], x[3])) < 0x1p-64f, 0)) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (x[i] < 0x1p-64f) r[i] = root_of(x[i] * 0x1p64f) * 0x1p-32f;
    }
    return r;
}

// Formulas: see hsadmm_adamw in the header.  Moments are formed in fp32, every operation rounded by itself; the weights' last
// two operations and the denominator are fused, the reciprocal is the machine's own, within one unit in the last place.
// The working copy is rounded to nearest: it is read by the forward pass only, the fp32 weights carry what the rounding loses.
// A workgroup takes 4 * kBlock elements, the `part`-th such stretch of an item, of replicas `first` to R - 1 in turn: z_i and u are read
// once for them.
// (Two fours a thread: ResNet-50, 4 replicas, 32-bit states 549 us instead of 543, 8-bit states 333 / 322, four times wider 1061 / 1014.)
template <int T, bool S8, bool PROX, bool LOW, bool FULL>
__device__ __forceinline__ void adamw_part(const FlatItem& it, int part, const AdamwArgs& a, int first, int R)
{
    typedef typename ElemOf<T>::type E;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int q = 4 * (part * kBlock + threadIdx.x);
    const int nv = FULL ? 4 : min(4, it.n - q);
    const int64_t at = it.base + q;
    // the wave's state block, and whether the layer reaches that far
    const int64_t block = it.block0 + part * kWaves + wave;
    const bool on = FULL || it.n > (part * kWaves + wave) * kStateBlock;
    const hsadmm_adamw_coef_t co = a.coef_dev ? *a.coef_dev : a.coef;
    v4f z, u;
    if (PROX) { z = load4<HSADMM_TYPE_F32>(a.Z + at, nv); u = load4<HSADMM_TYPE_F32>(a.U + at, nv); }
    const float rho = PROX ? a.rho[it.layer] : 0.f;
    for (int r = first; r < R; ++r) {
        const float s = a.grad_scale ? a.grad_scale[r] : 1.0f;
        if (!(__builtin_fabsf(s) < __builtin_inff())) continue;      // a gradient that is not finite: no step
        v4f w = load4<HSADMM_TYPE_F32>(a.W[r] + at, nv);
        const v4f g = load4<T>(static_cast<const E*>(a.G[r]) + at, nv);
        v4f m, v, rt;
        if (S8) {
            const unsigned int mc = load_codes(static_cast<const uint8_t*>(a.M[r]) + at, nv);
            const unsigned int vc = load_codes(static_cast<const uint8_t*>(a.V[r]) + at, nv);
            m = decode4(mc, on ? a.Ms[r][block] : 0.f);
            const v4f root = decode4(vc, on ? a.Vs[r][block] : 0.f);
            v = root * root;
        } else {
            m = load4<HSADMM_TYPE_F32>(static_cast<const float*>(a.M[r]) + at, nv);
            v = load4<HSADMM_TYPE_F32>(static_cast<const float*>(a.V[r]) + at, nv);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float gi = g[i] * s;
            if (PROX) gi = gi + rho * ((w[i] - z[i]) + u[i]);
            m[i] = a.beta1 * m[i] + a.one_minus_beta1 * gi;
            v[i] = a.beta2 * v[i] + a.one_minus_beta2 * (gi * gi);
        }
        rt = roots_of(v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float t = m[i] * __builtin_amdgcn_rcpf(__builtin_fmaf(rt[i], co.root, a.eps));
            w[i] = __builtin_fmaf(-co.step_size, t, w[i] * co.decay);
        }
        store4<HSADMM_TYPE_F32>(a.W[r] + at, w, nv);
        if (LOW) store4<T>(static_cast<E*>(a.Wl[r]) + at, w, nv);
        if (!S8) {
            store4<HSADMM_TYPE_F32>(static_cast<float*>(a.M[r]) + at, m, nv);
            store4<HSADMM_TYPE_F32>(static_cast<float*>(a.V[r]) + at, v, nv);
            continue;
        }
        if (!FULL) {
            // (values past the end of the layer count for nothing)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i >= nv) m[i] = rt[i] = 0.f;
        }
        float mu, vu;
        const float mscale = block_scale(wave_umax(top_bits(m)), mu), vscale = block_scale(wave_umax(top_bits(rt)), vu);
        const int64_t four = at >> 2;
        const unsigned int mix = mix_four((unsigned int)four + (unsigned int)(four >> 32) * kMix3 + co.noise + (unsigned int)r * kMix3);
        v4f ym = m * mu, yv = rt * vu;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            ym[i] = __builtin_amdgcn_fmed3f(ym[i], -448.0f, 448.0f);
            // a root that is not zero keeps a code that is not: a zero would divide by eps alone
            yv[i] = yv[i] > 0.f ? __builtin_amdgcn_fmed3f(yv[i], 0x1p-9f, 448.0f) : 0.f;
        }
        store_codes(static_cast<uint8_t*>(a.M[r]) + at, encode4(ym, mix), nv);
        store_codes(static_cast<uint8_t*>(a.V[r]) + at, encode4(yv, mix), nv);
        if (on && (threadIdx.x & (kWave - 1)) == 0) {
            a.Ms[r][block] = mscale;
            a.Vs[r][block] = vscale;
        }
    }
}

// Waves per SIMD (see pass1_waves): with every wave its registers allow in flight, a kernel of many streams crowds the memory.
// With 3, 4, 6, all 8, us: 32-bit states, ResNet-50, 4 replicas with the pull 523, 543, 560, 559 (5.85 TB/s at best), one replica in
// bf16 147, 151, 155, 157, ResNet-18 alone 55.0, 53.4, 54.4, 54.5; 8-bit states with the pull, ResNet-50, 4 replicas 353, 318, 316,
// 325 (5.83 TB/s), one 120, 110, 105, 102; without, four times wider 1517, 1275, 1065, 1001 (6.15 TB/s; more arithmetic per byte).
constexpr int adamw_waves(bool S8, bool PROX) { return !S8 ? 3 : PROX ? 6 : kAllWaves; }

template <int T, bool S8, bool PROX, bool LOW>
__global__ __launch_bounds__(kBlock) __attribute__((amdgpu_waves_per_eu(1, adamw_waves(S8, PROX)))) void adamw_kernel(const FlatItem* __restrict__ items, AdamwArgs a, int R, int each)
{
    constexpr int kEach = kFlatElems / kAdamwElems;
    unsigned int stretch = blockIdx.x;
    int first = 0, last = R;
    if (each < R) {                                               // a workgroup takes `each` of the replicas
        const unsigned int groups = (unsigned int)((R + each - 1) / each);
        stretch = blockIdx.x / groups;
        first = (int)(blockIdx.x - stretch * groups) * each;
        last = min(R, first + each);
    }
    const FlatItem it = items[stretch / kEach];
    const int part = stretch % kEach;
    if (it.n - part * kAdamwElems >= kAdamwElems) adamw_part<T, S8, PROX, LOW, true>(it, part, a, first, last);
    else if (it.n > part * kAdamwElems) adamw_part<T, S8, PROX, LOW, false>(it, part, a, first, last);
}

}  // namespace
#endif
