// AdamW over many tensors at once, with states in 32 or in 8 bits.
//
//   g = grad_scale * grad;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2
//   p = p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Every element is read and written once and nothing is shared between elements but the scale of a block of 8-bit states:
// the step is bound by memory.  Bytes an element (float32 parameters and gradients, no copy): 32-bit states 16 read + 12
// written, 8-bit states 10 + 6.  All arithmetic is float32; the constants of a step are formed on the host in double.  300,000 x 768
// elements with 8-bit states, bfloat16 gradients and copy: 3.7 GB in 0.74-0.79 ms (4.7-5.0 TB/s; a large copy makes 5.2); 61 tensors of 8M elements
// together, 32 bits: 224 MB in 53 us, one launch (4.2 TB/s).  A workgroup takes 2,048 elements of one tensor, which it finds in
// descriptors that come as an argument, so that no table has to be copied to the device first.
//
// 8-bit states: m and the root of v as e4m3 codes, with one power of two for each 128 elements.  The update of p uses the new
// m and v before they are rounded.  A root changes by 0.05 % a step, far less than the distance of two codes: rounded to
// nearest it would never move.  So a value is rounded up with a probability equal to its distance from the code below
// (16 bits of a counter generator: the same call gives the same bits), and a root above zero never becomes zero, since
// p moves by m / root.
#include <cmath>
#include <type_traits>

#include "rows.h"

#define ADAMW_ARGUMENT 4000     // bytes of descriptors that travel as an argument of a launch: 80 bytes (50 tensors) with 8-bit
                                // states, 56 bytes (71 tensors) with 32-bit states
#define ADAMW_BLOCK 128         // elements that share a scale
#define ADAMW_TILE 2048         // elements of one workgroup

struct AdamwScales { unsigned char *m, *v; u64 counter; };
struct AdamwNoScales {};
template <bool EIGHT> struct AdamwTensor : std::conditional<EIGHT, AdamwScales, AdamwNoScales>::type {
    float *param;
    const void *grad;
    void *m_data, *v_data, *copy;
    u64 n_types;                // n, and above it grad_type, copy_type (4 bits each) and wide: every array takes aligned accesses of 8
    u32 first_tile;             // in this launch
    __device__ __forceinline__ u64 n() const { return n_types & ((1ull << 48) - 1); }
    __device__ __forceinline__ int grad_type() const { return (int)(n_types >> 48) & 15; }
    __device__ __forceinline__ int copy_type() const { return (int)(n_types >> 52) & 15; }
    __device__ __forceinline__ bool wide() const { return n_types >> 56; }
};
template <bool EIGHT> struct AdamwPar {
    static constexpr int TENSORS = ADAMW_ARGUMENT / (int)sizeof(AdamwTensor<EIGHT>);
    AdamwTensor<EIGHT> t[TENSORS];
    u64 key;                    // of the step's random bits
    u32 count;
    float grad_scale, beta1, beta2, rest1, rest2, keep, rate, root_scale, eps;
};
static_assert(sizeof(AdamwPar<true>) <= 4096 && sizeof(AdamwPar<false>) <= 4096, "kernel arguments");

// The moments take a rounding for each product and sum, none fused, as a program that writes the formulas out takes them.  What a
// fused one would save is below 2^-24; but where a moment lies within that of a border, its 8-bit code would be another, and by the next
// step the parameter, now and then, by several lr.
template <bool EIGHT> __device__ __forceinline__ void adamw_update(const AdamwPar<EIGHT> &a, float g, float &p, float &m, float &v)
{
    g *= a.grad_scale;
    m = a.beta1 * m + a.rest1 * g;
    v = a.beta2 * v + a.rest2 * g * g;
    p = fmaf(p, a.keep, -a.rate * (m / fmaf(sqrtf(v), a.root_scale, a.eps)));
}

// the value of a code times a power of two (scale byte b: 2^(b - 127); 255: not a number)
__device__ __forceinline__ float scale_of(u32 byte)
{
    if (byte == 255) return __uint_as_float(0x7FC00000u);
    return byte ? __uint_as_float(byte << 23) : __uint_as_float(0x00400000u);
}
__device__ __forceinline__ void decode8(u64 codes, float scale, float (&x)[8])
{
    const u32 lo = (u32)codes, hi = (u32)(codes >> 32);
    x[0] = __builtin_amdgcn_cvt_f32_fp8((int)lo, 0);
    x[1] = __builtin_amdgcn_cvt_f32_fp8((int)lo, 1);
    x[2] = __builtin_amdgcn_cvt_f32_fp8((int)lo, 2);
    x[3] = __builtin_amdgcn_cvt_f32_fp8((int)lo, 3);
    x[4] = __builtin_amdgcn_cvt_f32_fp8((int)hi, 0);
    x[5] = __builtin_amdgcn_cvt_f32_fp8((int)hi, 1);
    x[6] = __builtin_amdgcn_cvt_f32_fp8((int)hi, 2);
    x[7] = __builtin_amdgcn_cvt_f32_fp8((int)hi, 3);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= scale;
}

// The scale byte for a block whose largest magnitude has these bits: brings it, times 1.01, into [128, 256).  (0.9 m + 0.1 g
// of values of few bits is a power of two, but for its last bit, in one block of a thousand: without the 1.01 that bit
// would choose the scale.)
__device__ __forceinline__ u32 scale_byte(float top)
{
    if (!(__float_as_uint(top) < 0x7F800000u)) return 255;      // infinite or not a number
    const u32 e = __float_as_uint(top * 1.01f) >> 23;
    return e < 7 ? 0 : e - 7 > 254 ? 254 : e - 7;
}
// code of |x| * up, up = 2^(127 - byte): three bits of fraction from 2^-6 on, steps of 2^-9 below
__device__ __forceinline__ u32 encode(float x, float up_a, float up_b, u32 random16)
{
    const float z = fabsf(x) * up_a * up_b;
    const u32 big = ((__float_as_uint(z) + (random16 << 4)) >> 20) - (120u << 3);
    const u32 small = (u32)fmaf(z, 512.0f, (float)random16 * (1.0f / 65536.0f));
    return z >= 0.015625f ? big : small;
}

// The largest of a block's magnitudes over the 16 lanes that hold it, all of which receive it.  As bits, so that an infinity
// or a NaN is the largest.
__device__ __forceinline__ float lane16_max(u32 b)
{
    u32 o = xor_lane_u32<1>(b);
    b = o > b ? o : b;
    o = xor_lane_u32<2>(b);
    b = o > b ? o : b;
    o = xor_lane_u32<7>(b);
    b = o > b ? o : b;
    o = xor_lane_u32<8>(b);
    b = o > b ? o : b;
    return __uint_as_float(b);
}

template <int DT>
__device__ __forceinline__ void load8(const void *base, u64 at, u32 have, bool wide, float (&x)[8])
{
    if (wide) {
        unpack<DT, 8>(load_pack<DT, 8>(base, at), x);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < (int)have ? (float)((const typename RowType<DT>::T *)base)[at + i] : 0.0f;
}
template <int DT>
__device__ __forceinline__ void store8(void *base, u64 at, u32 have, bool wide, const float (&x)[8])
{
    if (wide) {
        store_pack<DT, 8>(base, at, x);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < (int)have) ((typename RowType<DT>::T *)base)[at + i] = (typename RowType<DT>::T)x[i];
}
__device__ __forceinline__ u64 load_codes(const void *base, u64 at, u32 have, bool wide)
{
    if (wide) return *(const u64 *)((const char *)base + at);
    u64 c = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < (int)have) c |= (u64)((const unsigned char *)base)[at + i] << (8 * i);
    return c;
}
__device__ __forceinline__ void store_codes(void *base, u64 at, u32 have, bool wide, u64 c)
{
    if (wide) {
        *(u64 *)((char *)base + at) = c;
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < (int)have) ((unsigned char *)base)[at + i] = (unsigned char)(c >> (8 * i));
}

// A thread takes 8 neighbouring elements (16 lanes a block of 128); have = how many of them there are.
template <bool EIGHT>
__global__ __launch_bounds__(256) void k_adamw(AdamwPar<EIGHT> a)
{
    u32 lo = 0, hi = a.count - 1;       // the tensor whose tiles hold this block's
    while (lo < hi) {
        const u32 mid = (lo + hi + 1) / 2;
        if (a.t[mid].first_tile <= blockIdx.x) lo = mid;
        else hi = mid - 1;
    }
    const AdamwTensor<EIGHT> &t = a.t[lo];
    const u64 at = (u64)(blockIdx.x - t.first_tile) * ADAMW_TILE + threadIdx.x * 8;
    const u32 have = at >= t.n() ? 0 : t.n() - at < 8 ? (u32)(t.n() - at) : 8;
    const bool wide = t.wide() && have == 8;
    float p[8], g[8], m[8], v[8];
    if (have) {
        load8<DT_F32>(t.param, at, have, wide, p);
        if (t.grad_type() == DT_F32) load8<DT_F32>(t.grad, at, have, wide, g);
        else if (t.grad_type() == DT_F16) load8<DT_F16>(t.grad, at, have, wide, g);
        else load8<DT_BF16>(t.grad, at, have, wide, g);
        if constexpr (EIGHT) {
            const u64 cm = load_codes(t.m_data, at, have, wide), cv = load_codes(t.v_data, at, have, wide);
            decode8(cm, scale_of(t.AdamwScales::m[at / ADAMW_BLOCK]), m);
            decode8(cv, scale_of(t.AdamwScales::v[at / ADAMW_BLOCK]), v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= v[i];
        } else {
            load8<DT_F32>(t.m_data, at, have, wide, m);
            load8<DT_F32>(t.v_data, at, have, wide, v);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) adamw_update(a, g[i], p[i], m[i], v[i]);
        store8<DT_F32>(t.param, at, have, wide, p);
        if (t.copy) {
            if (t.copy_type() == DT_F16) store8<DT_F16>(t.copy, at, have, wide, p);
            else store8<DT_BF16>(t.copy, at, have, wide, p);
        }
        if (!EIGHT) {
            store8<DT_F32>(t.m_data, at, have, wide, m);
            store8<DT_F32>(t.v_data, at, have, wide, v);
        }
    }
    if constexpr (EIGHT) {
        u32 top_m = 0, top_v = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i >= (int)have) m[i] = v[i] = 0.0f;
            v[i] = sqrtf(v[i]);
            const u32 bm = __float_as_uint(m[i]) & 0x7FFFFFFFu, bv = __float_as_uint(v[i]) & 0x7FFFFFFFu;
            top_m = bm > top_m ? bm : top_m;
            top_v = bv > top_v ? bv : top_v;
        }
        const u32 sm = scale_byte(lane16_max(top_m)), sv = scale_byte(lane16_max(top_v));
        if (!have) return;
        // 2^(127 - byte) in two factors (byte 254: 2^-127 is below the smallest normal number)
        const int em = 127 - (sm == 255 ? 127 : (int)sm), ev = 127 - (sv == 255 ? 127 : (int)sv);
        const float um_a = __uint_as_float((em / 2 + 127) << 23), um_b = __uint_as_float((em - em / 2 + 127) << 23);
        const float uv_a = __uint_as_float((ev / 2 + 127) << 23), uv_b = __uint_as_float((ev - ev / 2 + 127) << 23);
        u64 cm = 0, cv = 0;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const u64 r = row_mix64(a.key + ROW_MIX_G * ((t.counter + at + i) / 2 + 1));
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const u32 half = (u32)(r >> (32 * h));
                const u32 code_m = encode(m[i + h], um_a, um_b, half & 0xFFFFu) | (__float_as_uint(m[i + h]) >> 31 << 7);
                u32 code_v = encode(v[i + h], uv_a, uv_b, half >> 16);
                if (v[i + h] > 0.0f && code_v == 0) code_v = 1;
                cm |= (u64)(code_m & 255u) << (8 * (i + h));
                cv |= (u64)(code_v & 255u) << (8 * (i + h));
            }
        }
        if (sm == 255) cm = 0;      // the scale says that the block's values are lost
        if (sv == 255) cv = 0;
        store_codes(t.m_data, at, have, wide, cm);
        store_codes(t.v_data, at, have, wide, cv);
        if ((threadIdx.x & 15) == 0) {
            t.AdamwScales::m[at / ADAMW_BLOCK] = (unsigned char)sm;
            t.AdamwScales::v[at / ADAMW_BLOCK] = (unsigned char)sv;
        }
    }
}

static int adamw_check(const rnnd_adamw_tensor &t)
{
    if (t.n < 0 || t.n > (int64_t)1 << 40) return RNND_ERR_BAD_SHAPE;
    if (t.state_bits != 8 && t.state_bits != 32) return RNND_ERR_UNSUPPORTED;
    if (!row_type(t.grad_dtype)) return RNND_ERR_UNSUPPORTED;
    if (t.copy && t.copy_dtype != RNND_F16 && t.copy_dtype != RNND_BF16) return RNND_ERR_UNSUPPORTED;
    if (!t.n) return RNND_OK;
    if (!t.param || !t.grad || !t.m || !t.v) return RNND_ERR_NULL;
    if (t.state_bits == 8 && (!t.m_scale || !t.v_scale)) return RNND_ERR_NULL;
    if ((uintptr_t)t.param % 4 || (uintptr_t)t.grad % dt_size(t.grad_dtype) || (t.copy && (uintptr_t)t.copy % 2)) return RNND_ERR_BAD_PARAM;
    if (t.state_bits == 32 && ((uintptr_t)t.m % 4 || (uintptr_t)t.v % 4)) return RNND_ERR_BAD_PARAM;
    if (t.state_bits == 8 && t.counter % 2) return RNND_ERR_BAD_PARAM;
    return RNND_OK;
}

struct AdamwStep {
    u64 key;
    float grad_scale, beta1, beta2, rest1, rest2, keep, rate, root_scale, eps;
};

template <bool EIGHT>
static void launch_adamw(const rnnd_adamw_tensor *tensors, int32_t count, const AdamwStep &s, hipStream_t st)
{
    AdamwPar<EIGHT> a;
    a.key = s.key;
    a.grad_scale = s.grad_scale;
    a.beta1 = s.beta1;
    a.beta2 = s.beta2;
    a.rest1 = s.rest1;
    a.rest2 = s.rest2;
    a.keep = s.keep;
    a.rate = s.rate;
    a.root_scale = s.root_scale;
    a.eps = s.eps;
    auto length = [&](int32_t i) { return tensors[i].state_bits == (EIGHT ? 8 : 32) ? (u64)tensors[i].n : 0; };
    a.count = 0;
    // a part starts at a multiple of a tile, so that its arrays are aligned as the tensor's are and its blocks of 128 are the tensor's
    auto part = [&](int32_t i, u64 first, u64 n, u64 tiles) {
        const rnnd_adamw_tensor &t = tensors[i];
        AdamwTensor<EIGHT> &d = a.t[a.count++];
        d.param = t.param + first;
        d.grad = (const char *)t.grad + first * dt_size(t.grad_dtype);
        d.m_data = (char *)t.m + first * (EIGHT ? 1 : 4);
        d.v_data = (char *)t.v + first * (EIGHT ? 1 : 4);
        d.copy = t.copy ? (char *)t.copy + first * 2 : nullptr;
        if constexpr (EIGHT) {
            d.m = t.m_scale + first / ADAMW_BLOCK;
            d.v = t.v_scale + first / ADAMW_BLOCK;
            d.counter = t.counter + first;
        }
        uintptr_t low = (uintptr_t)t.param | (uintptr_t)t.grad | (uintptr_t)t.copy;     // 16 bytes an access
        low |= EIGHT ? ((uintptr_t)t.m | (uintptr_t)t.v) << 1 : (uintptr_t)t.m | (uintptr_t)t.v;    // codes: 8
        d.n_types = n | (u64)t.grad_dtype << 48 | (u64)(t.copy ? t.copy_dtype : 0) << 52 | (u64)(low % 16 == 0) << 56;
        d.first_tile = (u32)tiles;
    };
    cut_into_launches(count, ADAMW_TILE, most_blocks(256), a.TENSORS, length, part, [&](u64 tiles) {
        hipLaunchKernelGGL(k_adamw<EIGHT>, dim3((u32)tiles), dim3(256), 0, st, a);
        a.count = 0;
    });
}

extern "C" int rnnd_adamw(const rnnd_adamw_tensor *tensors, int32_t count, int64_t step, double lr, double beta1, double beta2,
                          double eps, double weight_decay, double grad_scale, uint64_t seed, void *stream)
{
    if (count < 0) return RNND_ERR_BAD_SHAPE;
    if (count && !tensors) return RNND_ERR_NULL;
    // (written so that NaN is refused)
    if (step < 1 || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0) || !std::isfinite(eps) ||
        !std::isfinite(lr) || !std::isfinite(weight_decay) || !std::isfinite(grad_scale))
        return RNND_ERR_BAD_PARAM;
    bool any[2] = {false, false};       // tensors with 32-bit, with 8-bit states
    for (int32_t i = 0; i < count; ++i) {
        const int rc = adamw_check(tensors[i]);
        if (rc) return rc;
        if (tensors[i].n) any[tensors[i].state_bits == 8] = true;
    }
    if (!any[0] && !any[1]) return RNND_OK;
    AdamwStep s;
    s.key = row_mix64(seed + ROW_MIX_G * ((u64)step + 1));
    s.grad_scale = (float)grad_scale;
    s.beta1 = (float)beta1;
    s.beta2 = (float)beta2;
    s.rest1 = (float)(1.0 - beta1);
    s.rest2 = (float)(1.0 - beta2);
    s.keep = (float)(1.0 - lr * weight_decay);
    s.rate = (float)(lr / (1.0 - std::pow(beta1, (double)step)));
    s.root_scale = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
    s.eps = (float)eps;
    if (any[1]) launch_adamw<true>(tensors, count, s, (hipStream_t)stream);
    if (any[0]) launch_adamw<false>(tensors, count, s, (hipStream_t)stream);
    return launched("rnnd_adamw");
}
