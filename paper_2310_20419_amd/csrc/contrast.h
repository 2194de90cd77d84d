// What the calls on the softmax over squared distances share: rows prepared for the matrix cores, the products, logits by tiles with the
// sums of their exponentials, the weighted probabilities g and the gradients' products.  The mathematics is at the head of contrast.hip.
// Kernels and functions take the parameters of their call, a struct made from ContrastPar; row_counts() of that struct says which queries count.
#pragma once
#include <type_traits>
#include <utility>

#include "rows.h"

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef unsigned short us8 __attribute__((ext_vector_type(8)));
typedef unsigned short half_t;      // float16 or bfloat16, as the rows are

#define CT_PAD 256          // rows are padded to the largest tile
#define CT_K 64             // summed per step: 128 bytes of a row
#define CT_NEVER (-2)       // an id that no key has
#define CT_LOWEST (-2.0e38f)    // biases that are not above it leave a key out of the answers: in base 2 little is left of float32's range
#define CT_ROW_BLOCKS 1024  // at most, for the norms and targets of the rows of a side

__host__ __device__ constexpr int ct_up(int x, int m) { return (x + m - 1) / m * m; }

struct ContrastPar {
    const void *Q, *K;
    const int *target, *query_ids, *key_ids;
    const float *bias, *row_weight;
    float left_out;                 // the largest bias that leaves a key out
    float scale, c1;                // c1 = 2 scale log2(e)
    int B, M, d;
    int dp, Bp, Mp, dr;             // padded to CT_K; dr: d padded to the tile of the gradient products
    int tile, terms_from;           // of the logits, where a call has rules of its own (0: those of contrast_plan())
    bool keys_as_they_are;          // no copy of all of them
    int key0;                       // the first key that copies are made of and logits are formed with
    int ld_g, ld_gt;                // rows of g by rows and by columns: M and B padded to the largest tile
    size_t plane_q, plane_k, plane_qt, plane_kt, plane_g, plane_gt;     // elements
    half_t *q, *k, *qt, *kt, *g, *gt;       // copies (k: NULL where the keys are read as they are)
    u32 *tops, *top;                // float16 rows: largest weight of each block of queries, and of all, as bits
    int *first, *count;             // [M] the first query whose target the key is, and how many they are
    float *centre;                  // float32 rows: [dp] the point that they are taken from, zeros behind its d coordinates
    float *key_base;                // [M padded] (bias - scale |k|^2) log2(e), -inf where left out
    int *key_id;                    // [M padded]
    int2 *row_id;                   // [B padded] ids that a query leaves out: the target's, its own
    float2 *row_g;                  // [B padded] lse in base 2 (infinite: the query does not count), its weight (float16: scaled); lists: distill.hip
    float *row_own;                 // [B] g at the target
    float *own_logit;               // [B]
    float2 *part;                   // [B padded][parts_k] largest and sum of a row's part
    float *sum_q, *sum_k;           // [B padded][parts_k], [M padded][parts_q]: sums of the rounded g
    int parts_q, parts_k;           // one for half a tile
    float *acc_q, *acc_k;           // [splits][rows padded][dr]
    int splits_q, splits_k;
    float *loss;
    void *dQ, *dK;
};

// float16 rows: the power of two that brings weights up to `top` below 2^15
__device__ __forceinline__ int weight_exponent(u32 top) { return top >= 0x00800000u ? 14 + 127 - (int)(top >> 23) : 0; }

// ------------------------------------------------------------------------------------------------ preparation
__device__ __forceinline__ bool key_gone(const ContrastPar &c, int j)
{
    return (c.key_ids && c.key_ids[j] < 0) || (c.bias && c.bias[j] <= c.left_out);
}
__device__ __forceinline__ bool row_counts(const ContrastPar &c, int i)
{
    const int t = c.target[i];
    return (u32)t < (u32)c.M && !key_gone(c, t);
}

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int s = 32; s; s >>= 1) v += __shfl_xor(v, s);
    return v;
}

// sums over the lanes up to each
__device__ __forceinline__ int inclusive(int v, int lane)
{
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
        const int o = __shfl_up(v, k);
        if (lane >= k) v += o;
    }
    return v;
}

// Four coordinates of a row, zeros behind its end; WIDE: all rows allow it in one access.
template <int DT, bool WIDE>
__device__ __forceinline__ void load4(const void *rows, size_t row, int d, int e, float (&x)[4])
{
    if constexpr (WIDE) unpack<DT, 4>(load_pack<DT, 4>(rows, row * d + e), x);
    else
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = e + k < d ? (float)((const typename RowType<DT>::T *)rows)[row * d + e + k] : 0.0f;
}

// float32 rows: a point among the keys that count.  Of each sixteenth of the keys the first that counts is looked at, and every coordinate is the
// median of theirs: a few keys far away from all others do not move it (as they would the mean).  Coordinates that are not finite count as the
// largest; a median that is not is replaced by zero.  A launch of 4 to 6 us.
#define CT_SAMPLES 16
template <typename PAR>
__global__ __launch_bounds__(64 * CT_SAMPLES) void k_contrast_centre(PAR c)
{
    __shared__ int sample[CT_SAMPLES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int begin = (int)((long long)c.M * wave / CT_SAMPLES), end = (int)((long long)c.M * (wave + 1) / CT_SAMPLES);
    int found = -1;
    for (int j0 = begin; j0 < end && found < 0; j0 += 256) {
        bool on[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) on[k] = j0 + k * 64 + lane < end && !key_gone(c, j0 + k * 64 + lane);
#pragma unroll
        for (int k = 3; k >= 0; --k) {
            const u64 hit = __ballot(on[k]);
            if (hit) found = j0 + k * 64 + __builtin_ctzll(hit);
        }
    }
    if (lane == 0) sample[wave] = found;
    __syncthreads();
    const int e = blockIdx.x * (64 * CT_SAMPLES) + threadIdx.x;
    if (e >= c.dp) return;
    float x[CT_SAMPLES];
    int count = 0;
#pragma unroll
    for (int i = 0; i < CT_SAMPLES; ++i) {
        const int j = sample[i];
        x[i] = j >= 0 && e < c.d ? ((const float *)c.K)[(size_t)j * c.d + e] : INFINITY;
        count += j >= 0;
    }
#pragma unroll
    for (int i = 0; i < CT_SAMPLES; ++i) x[i] = x[i] < INFINITY ? x[i] : INFINITY;      // NaN too
    // neighbours exchanged, even and odd pairs in turn, until all are in order
#pragma unroll
    for (int pass = 0; pass < CT_SAMPLES; ++pass)
#pragma unroll
        for (int i = pass & 1; i + 1 < CT_SAMPLES; i += 2) {
            const float low = fminf(x[i], x[i + 1]), high = fmaxf(x[i], x[i + 1]);
            x[i] = low;
            x[i + 1] = high;
        }
    float middle = 0.0f;
#pragma unroll
    for (int i = 0; i < CT_SAMPLES; ++i) middle = count && (count - 1) / 2 == i ? x[i] : middle;
    c.centre[e] = fabsf(middle) < INFINITY ? middle : 0.0f;
}

// Four coordinates of a float32 row, taken from that point (x: as load4() left them)
__device__ __forceinline__ void from_centre(const ContrastPar &c, int e, float (&x)[4])
{
    const f32x4 m = *(const f32x4 *)&c.centre[e];
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] -= m[k];
}

// The own parts of R keys' logits, by a wavefront, and |k|^2; at < M padded, or a key is left alone.  ALL: the products read the rows of keys that are
// left out, too.  Zero times what is not a number is not zero, so those of which some are not get a base that is NaN.  ONCE: the base is rounded once, at the end.
template <int DT, bool WIDE, int R, bool ALL = false, bool ONCE = true>
__device__ __forceinline__ void key_sides(const ContrastPar &c, const int (&at)[R], int padded, int lane, float (&sum)[R])
{
    bool read[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        read[r] = at[r] < c.M && (ALL || !key_gone(c, at[r]));
        sum[r] = 0.0f;
    }
    for (int e = lane * 4; e < c.d; e += 256) {
        float x[R][4];
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (read[r]) load4<DT, WIDE>(c.K, at[r], c.d, e, x[r]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (!read[r]) continue;
            if constexpr (DT == DT_F32) from_centre(c, e, x[r]);
#pragma unroll
            for (int k = 0; k < 4; ++k) sum[r] = fmaf(x[r][k], x[r][k], sum[r]);
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) sum[r] = wave_sum(sum[r]);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (lane != r || at[r] >= padded) continue;
        const int j = at[r];
        const bool gone = j >= c.M || key_gone(c, j);
        const float bias = !gone && c.bias ? c.bias[j] : 0.0f;        // (there is none behind the last key)
        const float base = ONCE ? (float)(((double)bias - (double)c.scale * (double)sum[r]) * 1.4426950408889634) : (bias - c.scale * sum[r]) * 1.44269504f;
        c.key_base[j] = gone ? ALL && !(sum[r] < INFINITY) ? NAN : -INFINITY : base;
        c.key_id[j] = gone ? -1 : c.key_ids ? c.key_ids[j] : j;
    }
}

__device__ __forceinline__ half_t bits16(__bf16 x) { return __builtin_bit_cast(half_t, x); }
__device__ __forceinline__ half_t bits16(_Float16 x) { return __builtin_bit_cast(half_t, x); }
template <int DT> __device__ __forceinline__ float value16(half_t x)
{
    if constexpr (DT == DT_F16) return (float)__builtin_bit_cast(_Float16, x);
    else return __uint_as_float((u32)x << 16);
}

// The planes of a value: itself in 16 bits, or three bfloat16 terms.
template <int DT> constexpr int planes_of() { return DT == DT_F32 ? 3 : 1; }
template <int DT> __device__ __forceinline__ void to_planes(float x, half_t (&o)[planes_of<DT>()])
{
    if constexpr (DT == DT_F16) o[0] = bits16((_Float16)x);
    else
#pragma unroll
        for (int p = 0; p < planes_of<DT>(); ++p) {
            const __bf16 h = (__bf16)x;
            o[p] = bits16(h);
            x -= (float)h;
        }
}

// Copies of the rows that the products read: padded with zeros, in planes, by rows and by columns; rows that do not count and
// keys that are left out as zeros, whatever they hold.  One block per 64 x 64: a thread reads 16 coordinates of a row, and writes 16
// of a row and, through LDS, 16 of a column.
template <int DT, bool WIDE, typename PAR>
__device__ __forceinline__ void contrast_copy(const PAR &c, int tile_r, int c0, int q_tiles, int columns)
{
    constexpr int PLANES = planes_of<DT>();
    __shared__ u32 tile[64][33];        // [column][two rows]
    const bool keys = tile_r >= q_tiles;
    const int r0 = keys ? (tile_r - q_tiles) * 64 + c.key0 : tile_r * 64;
    const void *rows = keys ? c.K : c.Q;
    half_t *by_row = keys ? c.k : c.q, *by_col = keys ? c.kt : c.qt;
    const size_t plane_r = keys ? c.plane_k : c.plane_q, plane_c = keys ? c.plane_kt : c.plane_qt;
    const int across = keys ? c.Mp : c.Bp;
    const int x = threadIdx.x >> 2, y = (threadIdx.x & 3) * 16;
    float v[16] = {};
    if (keys ? r0 + x < c.M && !key_gone(c, r0 + x) : r0 + x < c.B && row_counts(c, r0 + x))
#pragma unroll
        for (int i = 0; i < 16; i += 4)
            if (c0 + y + i < c.d) {
                float four[4];
                load4<DT, WIDE>(rows, r0 + x, c.d, c0 + y + i, four);
                if constexpr (DT == DT_F32) from_centre(c, c0 + y + i, four);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[i + k] = four[k];
            }
    half_t o[PLANES][16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        half_t one[PLANES];
        to_planes<DT>(v[i], one);
#pragma unroll
        for (int p = 0; p < PLANES; ++p) o[p][i] = one[p];
    }
    if (c0 < c.dp)
#pragma unroll
        for (int p = 0; p < PLANES; ++p)
#pragma unroll
            for (int h = 0; h < 16; h += 8) {
                us8 l;
#pragma unroll
                for (int i = 0; i < 8; ++i) l[i] = o[p][h + i];
                *(us8 *)&by_row[p * plane_r + (size_t)(r0 + x) * c.dp + c0 + y + h] = l;
            }
    if (!columns || r0 >= across) return;       // a whole block
#pragma unroll
    for (int p = 0; p < PLANES; ++p) {
        if (p) __syncthreads();
#pragma unroll
        for (int i = 0; i < 16; ++i) ((half_t *)tile[y + i])[x] = o[p][i];
        __syncthreads();
        u32 l[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) l[i] = tile[x][y / 2 + i];
        uint4 *to = (uint4 *)&by_col[p * plane_c + (size_t)(c0 + x) * across + r0 + y];
        to[0] = make_uint4(l[0], l[1], l[2], l[3]);
        to[1] = make_uint4(l[4], l[5], l[6], l[7]);
    }
}


// ------------------------------------------------------------------------------------------------ the product
// TILE x TILE results of A B' (both with the summed index along the row) by 4 wavefronts of TILE/2 x TILE/2.  A step's 128
// bytes of a row lie in LDS as 8 pieces of 16 bytes, piece s of place p at s ^ (p % 8): the loads go straight to LDS in its
// own order (each lane fetches the piece that belongs there), and the 16 rows that a matrix instruction reads together spread over
// the banks.  LDS holds two steps.  While one half of a step is multiplied the other half's operands are read into registers, and
// the loads of the step after next are under way: one barrier a step.  There has to be a step.
//
// Which row stands at which place is chosen for what comes after the product.  A lane of a wavefront gets the results of rows
// (lane / 16) * 4 N + 4 m + r (m < N = TILE / 32, r < 4) and columns (lane % 16) * N + n (n < N): 4 N rows that lie
// together, and N columns that lie together, so that results leave in accesses of 16 bytes both by rows and by columns.
//
// LDS traffic a step: each wavefront reads TILE rows, all write 2 TILE: (4 + 2) * TILE * 128 bytes at 128 a clock, against
// TILE^2 * 128 / 4096 clocks of matrix work: 768 against 512 clocks with TILE = 128, 1,536 against 2,048 with TILE = 256.
// Rows of ld elements, ld a multiple of CT_K; rows behind the last are zeros (copies are padded to whole tiles, so they have none).
struct Operand { const half_t *p; size_t plane; int ld, rows = 0x7FFFFFFF; };

// One step.  The two that a kernel has are variables of their own: the compiler lets reads of one go past loads into the other, but would have
// reads of a variable wait for all loads into it (in the middle of every step, for those just sent off).
template <int TILE> struct ProductLds { half_t a[TILE * CT_K], b[TILE * CT_K]; };
struct NoLds {};

template <int TILE> __device__ __forceinline__ int row_at(int p)      // row of A that stands at place p
{
    constexpr int N = TILE / 32, H = TILE / 2;
    const int q = p % H, m = q >> 4, l = q & 15;
    return p - q + (l >> 2) * (4 * N) + m * 4 + (l & 3);
}
template <int TILE> __device__ __forceinline__ int col_at(int p)      // row of B that stands at place p
{
    constexpr int N = TILE / 32, H = TILE / 2;
    const int q = p % H;
    return p - q + (q & 15) * N + (q >> 4);
}

// 16 bytes of every lane from base + v + at (bytes; `bytes` of them may be read) to 1 KB of LDS, in the lanes' order
__device__ __forceinline__ void to_lds(const half_t *base, int bytes, half_t *lds, int v, int at)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc((void *)base, 0, bytes, 0x00027000),
                                             (__attribute__((address_space(3))) void *)lds, 16, v, at, 0, 0);
}

// With tiles of 256 the results take all 256 accumulation registers.  Left to itself the compiler moves some of them to and fro (180
// moves for 128 matrix instructions); as operands of the class "a" they stay.  It does not know what the instruction is, so product()
// keeps the distances it asks for: before the first, and after the last.
template <int DT> __device__ __forceinline__ void mfma_in_agprs(f32x4 &c, const us8 &a, const us8 &b)
{
    if constexpr (DT == DT_F16) asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
    else asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}
template <int DT> __device__ __forceinline__ f32x4 mfma(const us8 &a, const us8 &b, f32x4 c)
{
    if constexpr (DT == DT_F16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

template <int N> struct Half { us8 a[N], b[N]; };      // what half a step multiplies

struct Nothing { __device__ __forceinline__ void operator()(const us8 &, int) const {} };

// `meanwhile` runs while the first loads are under way; what it leaves in LDS is there behind the product.  also(b, j) is given all that is
// multiplied of B: of the lane's column j, a quarter of every step.
template <int TILE, int DT, typename F, typename G = Nothing>
__device__ __forceinline__ void product(const Operand &A, const Operand &B, int row_a, int row_b, int k_begin, int k_end,
                                        ProductLds<TILE> &even, ProductLds<TILE> &odd, f32x4 (&acc)[TILE / 32][TILE / 32], F meanwhile, G also = G())
{
    constexpr int N = TILE / 32;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int per = (k_end - k_begin) / CT_K;
    const int steps = per * (DT == DT_F32 ? 6 : 1);
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) acc[i][j] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    // each wavefront brings a quarter of the places, 8 at a time
    int va[N], vb[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int p = wave * (TILE / 4) + i * 8 + (lane >> 3), piece = (lane & 7) ^ (lane >> 3);
        va[i] = (row_at<TILE>(p) * A.ld + piece * 8) * 2;
        vb[i] = (col_at<TILE>(p) * B.ld + piece * 8) * 2;
    }
    const half_t *pa = A.p + (size_t)row_a * A.ld, *pb = B.p + (size_t)row_b * B.ld;
    const int bytes_a = (A.rows - row_a < TILE ? A.rows - row_a : TILE) * A.ld * 2, bytes_b = (B.rows - row_b < TILE ? B.rows - row_b : TILE) * B.ld * 2;
    // 1 / N of a step's loads
    auto fetch = [&](int s, ProductLds<TILE> &lds, int i) {
        int kk = s;
        const half_t *qa = pa, *qb = pb;
        if (DT == DT_F32) {         // planes (0, 0) (0, 1) (1, 0) (1, 1) (0, 2) (2, 0)
            const int pair = s / per;
            kk = s - pair * per;
            qa += (pair == 2 || pair == 3 ? 1 : pair == 5 ? 2 : 0) * A.plane;
            qb += (pair == 1 || pair == 3 ? 1 : pair == 4 ? 2 : 0) * B.plane;
        }
        const int at = (k_begin + kk * CT_K) * 2, place = (wave * (TILE / 4) + i * 8) * CT_K;
        to_lds(qa, bytes_a, &lds.a[place], va[i], at);
        to_lds(qb, bytes_b, &lds.b[place], vb[i], at);
    };
    const int ra0 = ((wave >> 1) * (TILE / 2) + (lane & 15)) * CT_K, rb0 = ((wave & 1) * (TILE / 2) + (lane & 15)) * CT_K;
    const int piece0 = ((lane >> 4) ^ (lane & 7)) * 8;
    auto read = [&](Half<N> &f, const ProductLds<TILE> &lds, int h, int i) {
        const int at = piece0 ^ (h * 32);
        f.a[i] = *(const us8 *)&lds.a[ra0 + i * 16 * CT_K + at];
        f.b[i] = *(const us8 *)&lds.b[rb0 + i * 16 * CT_K + at];
    };
    auto multiply = [&](const Half<N> &f, int i) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if constexpr (TILE == 256) mfma_in_agprs<DT>(acc[i][j], f.a[i], f.b[j]);
            else acc[i][j] = mfma<DT>(f.a[i], f.b[j], acc[i][j]);
        }
    };
    if constexpr (TILE == 256) {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) asm volatile("" : "+a"(acc[i][j]));
        asm volatile("s_nop 7" ::: "memory");
    }
    Half<N> h0, h1;
#pragma unroll
    for (int i = 0; i < N; ++i) fetch(0, even, i);
    meanwhile();
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (steps > 1)
#pragma unroll
        for (int i = 0; i < N; ++i) fetch(1, odd, i);
#pragma unroll
    for (int i = 0; i < N; ++i) read(h0, even, 0, i);
    // A wavefront issues in order: reads and loads in one lump would hold its matrix instructions back until they are accepted.  So
    // a few of them go before each N matrix instructions, the reads early enough to be there for the next half.
    auto step = [&](int s, ProductLds<TILE> &now, ProductLds<TILE> &other) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (i < N / 2) {
                read(h1, now, 1, 2 * i);
                read(h1, now, 1, 2 * i + 1);
            }
            multiply(h0, i);
            also(h0.b[i], i);
            __builtin_amdgcn_sched_barrier(0);
        }
        // the next step is there for all, and all have read this one
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        const int next = s + 2 < steps ? s + 2 : s + 1;         // (the last one is read by nobody)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (i < N / 2) {
                fetch(next, now, 2 * i);
                fetch(next, now, 2 * i + 1);
            } else {
                read(h0, other, 0, 2 * i - N);
                read(h0, other, 0, 2 * i - N + 1);
            }
            multiply(h1, i);
            also(h1.b[i], i);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    for (int s = 0; s + 1 < steps; s += 2) {
        step(s, even, odd);
        if (s + 2 < steps) step(s + 1, odd, even);
    }
    if (steps & 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) read(h1, even, 1, i);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) read(h1, odd, 1, i);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        multiply(h0, i);
        also(h0.b[i], i);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        multiply(h1, i);
        also(h1.b[i], i);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if constexpr (TILE == 256) {
        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");       // a result may be read 18 clocks behind its instruction
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) asm volatile("" : "+a"(acc[i][j]));
    }
}

// The product of float32 rows, for tiles of 128: the three terms of both operands stand in LDS together, so that six products are
// made of each step of 32 that is loaded and read once -- with product() each of the six would load and read its two again: 64 operations
// for a byte instead of 128, and both L2 and LDS were what it waited for.  LDS holds three steps, of which two are under way.
// The next step's operands are read into registers between the matrix instructions of this one.
#define CT_K3 32
struct TermsLds { half_t a[3][3][128 * CT_K3], b[3][3][128 * CT_K3]; };       // [step % 3][term]

template <typename F>
__device__ __forceinline__ void product_of_terms(const Operand &A, const Operand &B, int row_a, int row_b, int k_begin, int k_end,
                                                 TermsLds &lds, f32x4 (&acc)[4][4], F meanwhile)
{
    struct Step { us8 a[3][4], b[3][4]; };
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int steps = (k_end - k_begin) / CT_K3;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    // a row's 64 bytes are 4 pieces, piece s of place p at s ^ (p / 2 % 4); each wavefront brings a quarter of the places, 16 at a time
    int va[2], vb[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int p = (wave * 2 + i) * 16 + (lane >> 2), piece = (lane & 3) ^ (lane >> 3 & 3);
        va[i] = (row_at<128>(p) * A.ld + piece * 8) * 2;
        vb[i] = (col_at<128>(p) * B.ld + piece * 8) * 2;
    }
    const half_t *pa = A.p + (size_t)row_a * A.ld, *pb = B.p + (size_t)row_b * B.ld;
    auto fetch = [&](int s, int slot) {         // 12 loads
        const int at = (k_begin + s * CT_K3) * 2;
#pragma unroll
        for (int t = 0; t < 3; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int place = (wave * 2 + i) * 16 * CT_K3;
                to_lds(pa + t * A.plane, 128 * A.ld * 2, &lds.a[slot][t][place], va[i], at);
                to_lds(pb + t * B.plane, 128 * B.ld * 2, &lds.b[slot][t][place], vb[i], at);
            }
    };
    const int piece = (lane >> 4 ^ (lane >> 1 & 3)) * 8;
    const int ra = ((wave >> 1) * 64 + (lane & 15)) * CT_K3 + piece, rb = ((wave & 1) * 64 + (lane & 15)) * CT_K3 + piece;
    auto read = [&](Step &f, int slot, int i) {
#pragma unroll
        for (int t = 0; t < 3; ++t) {
            f.a[t][i] = *(const us8 *)&lds.a[slot][t][ra + i * 16 * CT_K3];
            f.b[t][i] = *(const us8 *)&lds.b[slot][t][rb + i * 16 * CT_K3];
        }
    };
    // all wavefronts have read what they held before, and the step that all but the last `left` loads brought is there
    auto meet = [&](int left) {
        if (left == 24) asm volatile("s_waitcnt vmcnt(24) lgkmcnt(0)" ::: "memory");
        else if (left == 12) asm volatile("s_waitcnt vmcnt(12) lgkmcnt(0)" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    int slot = 0;
    auto step = [&](const Step &now, Step &next, int s) {
        const int ahead = slot == 2 ? 0 : slot + 1;
        if (s + 1 < steps) {
            meet(s + 2 < steps ? 12 : 0);
            if (s + 3 < steps) fetch(s + 3, slot);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            read(next, ahead, i);       // (behind the last step: what nobody uses)
#pragma unroll
            for (int pair = 0; pair < 6; ++pair) {      // (0, 0) (0, 1) (1, 0) (1, 1) (0, 2) (2, 0)
                const int ta = pair == 2 || pair == 3 ? 1 : pair == 5 ? 2 : 0, tb = pair == 1 || pair == 3 ? 1 : pair == 4 ? 2 : 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = mfma<DT_BF16>(now.a[ta][i], now.b[tb][j], acc[i][j]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        slot = ahead;
    };
    fetch(0, 0);
    if (steps > 1) fetch(1, 1);
    if (steps > 2) fetch(2, 2);
    meanwhile();
    meet(steps > 2 ? 24 : steps > 1 ? 12 : 0);
    Step even, odd;
#pragma unroll
    for (int i = 0; i < 4; ++i) read(even, 0, i);
    for (int s = 0;;) {
        step(even, odd, s);
        if (++s == steps) break;
        step(odd, even, s);
        if (++s == steps) break;
    }
}

// Neighbouring tiles to the same XCD (workgroups go round the 8 of them), in blocks of 8 rows of tiles, so that what
// its L2 holds serves several of them.
__device__ __forceinline__ void tile_of(int id, int tiles_r, int tiles_c, int &r, int &c)
{
    const int total = tiles_r * tiles_c, per = total / 8;
    if (id < per * 8) id = (id & 7) * per + (id >> 3);
    if (tiles_c <= 4) {         // all columns of a row of tiles together
        r = id / tiles_c;
        c = id - r * tiles_c;
        return;
    }
    const int group = 8 * tiles_c, g = id / group, in = id - g * group;
    const int high = tiles_r - g * 8 < 8 ? tiles_r - g * 8 : 8;
    r = g * 8 + in % high;
    c = in / high;
}

// over the 16 lanes that share a row, R rows at a time
template <int S> __device__ __forceinline__ float xor_lane_f32(float v) { return __uint_as_float(xor_lane_u32<S>(__float_as_uint(v))); }
template <int R> __device__ __forceinline__ void row16_max(float (&v)[R])
{
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = fmaxf(v[r], xor_lane_f32<1>(v[r]));
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = fmaxf(v[r], xor_lane_f32<2>(v[r]));
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = fmaxf(v[r], xor_lane_f32<7>(v[r]));
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = fmaxf(v[r], xor_lane_f32<15>(v[r]));
}
template <int R> __device__ __forceinline__ void row16_sum(float (&v)[R])
{
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] += xor_lane_f32<1>(v[r]);
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] += xor_lane_f32<2>(v[r]);
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] += xor_lane_f32<7>(v[r]);
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] += xor_lane_f32<15>(v[r]);
}

// What a lane's columns and rows are after product().
template <int TILE> struct Place {
    static constexpr int N = TILE / 32;
    int row, col;       // first of 4 N rows, first of N columns
    int half_r, half_c; // number of the half tile
    int in_row, in_col; // of the tile
    __device__ __forceinline__ Place(int tile_r, int tile_c)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        half_r = tile_r * 2 + (wave >> 1);
        half_c = tile_c * 2 + (wave & 1);
        in_row = (wave >> 1) * (TILE / 2) + (lane >> 4) * (4 * N);
        in_col = (wave & 1) * (TILE / 2) + (lane & 15) * N;
        row = tile_r * TILE + in_row;
        col = tile_c * TILE + in_col;
    }
};

// What the logits of a tile need besides the product, in LDS while its first loads are under way: behind it nothing else hides the
// latency of loads from memory (one wavefront per SIMD).
// A row leaves out few keys, so most rows leave out none of a tile's.  16,384 bits say which hashes the tile's keys have, two of each; a row
// whose two ids are not among them needs no comparison (4 instructions of 14 for each logit; one hash alone is there by chance for one
// of 40 rows, and 16 rows are looked at together).
#define CT_HASH 14
template <int TILE> struct SideLds {
    int2 row_id[TILE];
    float2 row_g[TILE];
    float base[TILE];
    int id[TILE];
    u32 maybe[TILE];        // whether the row may leave out a key of the tile
    u32 seen[(1 << CT_HASH) / 32];
};
// Keys that a row lists are kept out of its sums and of g: distill.hip.
template <typename PAR> constexpr bool has_lists() { return false; }
template <int TILE, typename PAR> struct ListLds {};
__device__ __forceinline__ u32 id_hash(int id) { return (u32)id * 0x9E3779B1u >> (32 - CT_HASH); }
__device__ __forceinline__ u32 id_hash2(int id) { return (u32)id * 0x85EBCA77u >> (32 - CT_HASH); }
__device__ __forceinline__ u32 bit_at(const u32 *bits, u32 at) { return bits[at >> 5] >> (at & 31) & 1; }
// PREPARED: by key_side(); else the base is without -scale |k|^2.
template <int TILE, bool PREPARED> __device__ __forceinline__ void load_side(const ContrastPar &c, SideLds<TILE> &side, int row0, int col0)
{
    const int t = threadIdx.x;
    int id = -1;
    int2 out = make_int2(CT_NEVER, CT_NEVER);
#pragma unroll
    for (int i = 0; i < (1 << CT_HASH) / 32 / 256; ++i) side.seen[i * 256 + t] = 0;
    if (t < TILE) {
        side.row_id[t] = out = c.row_id[row0 + t];
        side.row_g[t] = c.row_g[row0 + t];
        if constexpr (!PREPARED) {
            const int j = col0 + t;
            const bool gone = j >= c.M || key_gone(c, j);
            side.base[t] = gone ? -INFINITY : c.bias ? c.bias[j] * 1.44269504f : 0.0f;
            side.id[t] = id = gone ? -1 : c.key_ids ? c.key_ids[j] : j;
        } else {
            side.base[t] = c.key_base[col0 + t];
            side.id[t] = id = c.key_id[col0 + t];
        }
    }
    __syncthreads();
    if (t < TILE && id >= 0) {
        atomicOr(&side.seen[id_hash(id) >> 5], 1u << (id_hash(id) & 31));
        atomicOr(&side.seen[id_hash2(id) >> 5], 1u << (id_hash2(id) & 31));
    }
    __syncthreads();
    if (t < TILE)
        side.maybe[t] = (bit_at(side.seen, id_hash(out.x)) & bit_at(side.seen, id_hash2(out.x))) | (bit_at(side.seen, id_hash(out.y)) & bit_at(side.seen, id_hash2(out.y)));
}

// q k' of a tile, its side tables read meanwhile
template <int TILE, int DT, bool TERMS, bool PREPARED = true, typename LDS, typename LDS2, typename F, typename G = Nothing>
__device__ __forceinline__ void logit_product(const ContrastPar &c, int tr, int tc, LDS &lds, LDS2 &lds2, SideLds<TILE> &side, f32x4 (&acc)[TILE / 32][TILE / 32], F lists,
                                              G also = G())
{
    const Operand q = {c.q, c.plane_q, c.dp}, k = !c.k ? Operand{(const half_t *)c.K, 0, c.d, c.M} : Operand{c.k, c.plane_k, c.dp};
    const auto tables = [&]() {
        load_side<TILE, PREPARED>(c, side, tr * TILE, tc * TILE);
        lists();
    };
    if constexpr (TERMS) product_of_terms(q, k, tr * TILE, tc * TILE, 0, c.dp, lds, acc, tables);
    else product<TILE, DT>(q, k, tr * TILE, tc * TILE, 0, c.dp, lds, lds2, acc, tables, also);
}

// Logits of the keys that rows leave out become -infinity, or what stands for it; nothing to do for most rows.
template <int TILE, int R, int N>
__device__ __forceinline__ void leave_out(const SideLds<TILE> &side, int row, const int (&id)[N], float (&s)[R][N], float none = -INFINITY)
{
    u32 maybe = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) maybe |= side.maybe[row + r];
    if (!__any(maybe)) return;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int2 out = side.row_id[row + r];
#pragma unroll
        for (int n = 0; n < N; ++n) s[r][n] = id[n] == out.x || id[n] == out.y ? none : s[r][n];
    }
}

// ------------------------------------------------------------------------------------------------ first product: largest and sum of every row
template <int TILE, int DT, bool TERMS, typename PAR>
__global__ __launch_bounds__(256, TILE == 256 || TERMS ? 1 : 2) void k_contrast_sums(PAR c, u32 first, int tiles_q, int tiles_k)
{
    constexpr int N = TILE / 32;
    __shared__ typename std::conditional<TERMS, TermsLds, ProductLds<TILE>>::type lds;
    __shared__ typename std::conditional<TERMS, NoLds, ProductLds<TILE>>::type lds2;
    __shared__ SideLds<TILE> side;
    __shared__ ListLds<TILE, PAR> lists;
    f32x4 acc[N][N];
    int tr, tc;
    tile_of((int)(first + blockIdx.x), tiles_q, tiles_k, tr, tc);
    logit_product<TILE, DT, TERMS>(c, tr, tc, lds, lds2, side, acc, [&]() {
        if constexpr (has_lists<PAR>()) load_lists(c, lists, tr * TILE, tc);
    });
    const Place<TILE> at(tr, tc);
    float base[N];
    int id[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        base[n] = side.base[at.in_col + n];
        id[n] = side.id[at.in_col + n];
    }
    if constexpr (has_lists<PAR>()) __syncthreads();        // all have read their operands
    // four rows at a time without a branch, so that their chains of instructions overlap; lane l of 16 keeps the rows l, l + 16
    float keep_top[N / 4], keep_sum[N / 4];
#pragma unroll
    for (int m = 0; m < N; ++m) {
        float s[4][N], top[4], sum[4];
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int n = 0; n < N; ++n) s[r][n] = fmaf(acc[m][n][r], c.c1, base[n]);
        leave_out(side, at.in_row + m * 4, id, s);
        if constexpr (has_lists<PAR>()) take_listed(std::true_type(), c, lists, (float *)&lds, tr * TILE, at.in_row + m * 4, at.in_col, s);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            top[r] = s[r][0];
#pragma unroll
            for (int n = 1; n < N; ++n) top[r] = fmaxf(top[r], s[r][n]);
        }
        row16_max(top);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float ref = top[r] == -INFINITY ? 0.0f : top[r];
            sum[r] = 0.0f;
#pragma unroll
            for (int n = 0; n < N; ++n) sum[r] += __builtin_amdgcn_exp2f(s[r][n] - ref);
        }
        row16_sum(sum);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const bool mine = (int)(threadIdx.x & 15) == m % 4 * 4 + r;
            keep_top[m / 4] = mine ? top[r] : m % 4 || r ? keep_top[m / 4] : 0.0f;
            keep_sum[m / 4] = mine ? sum[r] : m % 4 || r ? keep_sum[m / 4] : 0.0f;
        }
    }
#pragma unroll
    for (int h = 0; h < N / 4; ++h)
        c.part[(size_t)(at.row + h * 16 + (threadIdx.x & 15)) * c.parts_k + at.half_c] = make_float2(keep_top[h], keep_sum[h]);
    if constexpr (has_lists<PAR>()) write_listed(c, lists, (const float *)&lds, tr * TILE, tc);
}

// (largest, sum) of two parts; a NaN in either stays
__device__ __forceinline__ void join_parts(float &top, float &sum, float ot, float os)
{
    const float m = fmaxf(top, ot), ref = m == -INFINITY ? 0.0f : m;
    sum = sum * __builtin_amdgcn_exp2f(top - ref) + os * __builtin_amdgcn_exp2f(ot - ref);
    top = m;
}


// ------------------------------------------------------------------------------------------------ second product: g
template <int TILE, int DT, bool TERMS, typename PAR>
__global__ __launch_bounds__(256, TILE == 256 || TERMS ? 1 : 2) void k_contrast_g(PAR c, u32 first, int tiles_q, int tiles_k)
{
    constexpr int N = TILE / 32, PLANES = planes_of<DT>();
    __shared__ typename std::conditional<TERMS, TermsLds, ProductLds<TILE>>::type lds;
    __shared__ typename std::conditional<TERMS, NoLds, ProductLds<TILE>>::type lds2;
    __shared__ SideLds<TILE> side;
    __shared__ ListLds<TILE, PAR> lists;
    f32x4 acc[N][N];
    int tr, tc;
    tile_of((int)(first + blockIdx.x), tiles_q, tiles_k, tr, tc);
    logit_product<TILE, DT, TERMS>(c, tr, tc, lds, lds2, side, acc, [&]() {
        if constexpr (has_lists<PAR>()) load_lists(c, lists, tr * TILE, tc);
    });
    const Place<TILE> at(tr, tc);
    float base[N], col_sum[N] = {};
    int id[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        base[n] = side.base[at.in_col + n];
        id[n] = side.id[at.in_col + n];
    }
    constexpr int H = TILE / 2;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    constexpr int room = H * H * (PLANES == 3 ? 2 : 1), fit = sizeof(lds) / 2 / room;       // of a wavefront; how many go into the first
    half_t *turn = wave < fit ? (half_t *)&lds + wave * room : (half_t *)&lds2 + (wave - fit) * room;
    static_assert(fit >= 4 || sizeof(lds2) / 2 / room >= 4 - fit, "every wavefront has its room");
    us8 third[PLANES == 3 ? N / 2 : 1][N];
    auto turn_at = [&](int n, int pair) { return ((lane & 15) * N + n) * H + (((lane >> 4) * (N / 2) + pair) ^ (lane & 7)) * 8; };
    __syncthreads();        // all have read their operands
    float keep_sum[N / 4];
#pragma unroll
    for (int pair = 0; pair < N / 2; ++pair) {       // 8 rows at a time
        half_t o[PLANES][N][8];
        const int row0 = at.row + pair * 8;
        float row_sum[8] = {}, logit[4][N];
#pragma unroll
        for (int r8 = 0; r8 < 8; ++r8) {
            if (r8 % 4 == 0) {
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int n = 0; n < N; ++n) logit[r][n] = fmaf(acc[pair * 2 + r8 / 4][n][r], c.c1, base[n]);
                leave_out(side, at.in_row + pair * 8 + r8, id, logit);
                if constexpr (has_lists<PAR>()) take_listed(std::false_type(), c, lists, nullptr, tr * TILE, at.in_row + pair * 8 + r8, at.in_col, logit);
            }
            const float2 info = side.row_g[at.in_row + pair * 8 + r8];
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const float g = __builtin_amdgcn_exp2f(logit[r8 % 4][n] - info.x) * info.y;
                half_t x[PLANES];
                to_planes<DT>(g, x);
                float rounded = 0.0f;
#pragma unroll
                for (int p = PLANES - 1; p >= 0; --p) {
                    o[p][n][r8] = x[p];
                    rounded += value16<DT>(x[p]);
                }
                row_sum[r8] += rounded;
                col_sum[n] += rounded;
            }
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
                typedef half_t line_t __attribute__((ext_vector_type(N)));
                line_t l;
#pragma unroll
                for (int n = 0; n < N; ++n) l[n] = o[p][n][r8];
                *(line_t *)&c.g[p * c.plane_g + (size_t)(row0 + r8) * c.ld_g + at.col] = l;
            }
        }
        row16_sum(row_sum);
#pragma unroll
        for (int r8 = 0; r8 < 8; ++r8)
            keep_sum[pair / 2] = (int)(threadIdx.x & 15) == pair % 2 * 8 + r8 ? row_sum[r8] : pair % 2 || r8 ? keep_sum[pair / 2] : 0.0f;
        // by columns: 8 rows of a column are 16 bytes.  First into the wavefront's own part of LDS, in which a column's rows lie
        // together (piece k of column x at k ^ x / N % 8: both sides free of bank conflicts); a third plane waits for its turn
#pragma unroll
        for (int p = 0; p < PLANES; ++p)
#pragma unroll
            for (int n = 0; n < N; ++n) {
                us8 l;
#pragma unroll
                for (int r8 = 0; r8 < 8; ++r8) l[r8] = o[p][n][r8];
                if (p < 2) *(us8 *)&turn[p * H * H + turn_at(n, pair)] = l;
                else third[pair][n] = l;
            }
    }
    constexpr int per = H / 8;          // lanes for a column
    const int piece = lane % per;
    half_t *const to = c.gt + (size_t)(tc * TILE + (wave & 1) * H) * c.ld_gt + tr * TILE + (wave >> 1) * H + piece * 8;
    auto flush = [&](int p, const half_t *from) {
#pragma unroll 8
        for (int x = lane / per; x < H; x += 64 / per)
            *(us8 *)&to[p * c.plane_gt + (size_t)x * c.ld_gt] = *(const us8 *)&from[x * H + (piece ^ (x / N & 7)) * 8];
    };
    wave_sync();
    flush(0, turn);
    if constexpr (PLANES == 3) {
        flush(1, turn + H * H);
        wave_sync();
#pragma unroll
        for (int pair = 0; pair < N / 2; ++pair)
#pragma unroll
            for (int n = 0; n < N; ++n) *(us8 *)&turn[turn_at(n, pair)] = third[pair][n];
        wave_sync();
        flush(2, turn);
    }
#pragma unroll
    for (int h = 0; h < N / 4; ++h) c.sum_q[(size_t)(at.row + h * 16 + (threadIdx.x & 15)) * c.parts_k + at.half_c] = keep_sum[h];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        col_sum[n] += __shfl_xor(col_sum[n], 16);
        col_sum[n] += __shfl_xor(col_sum[n], 32);
        if ((threadIdx.x & 63) < 16) c.sum_k[(size_t)(at.col + n) * c.parts_q + at.half_r] = col_sum[n];
    }
}

// ------------------------------------------------------------------------------------------------ third and fourth: g k and g' q
// One launch: the parts of dq's sums, then those of dk's.
template <int TILE, int DT, typename PAR>
__global__ __launch_bounds__(256, TILE == 256 || DT == DT_F32 ? 1 : 2) void k_contrast_grad(PAR c, u32 first, int tiles_q, int tiles_k, int tiles_d)
{
    constexpr int N = TILE / 32;
    __shared__ typename std::conditional<DT == DT_F32, TermsLds, ProductLds<TILE>>::type lds;
    __shared__ typename std::conditional<DT == DT_F32, NoLds, ProductLds<TILE>>::type lds2;
    f32x4 acc[N][N];
    const int of_q = tiles_q * tiles_d * c.splits_q;
    const int block = (int)(first + blockIdx.x);
    const bool keys = block >= of_q;
    const int id = keys ? block - of_q : block, tiles = keys ? tiles_k : tiles_q, splits = keys ? c.splits_k : c.splits_q;
    const int split = id / (tiles * tiles_d);
    int tr, tc;
    tile_of(id - split * tiles * tiles_d, tiles, tiles_d, tr, tc);
    const int depth = keys ? c.Bp : c.Mp, steps = depth / CT_K;
    const int k0 = (int)((long long)steps * split / splits) * CT_K, k1 = (int)((long long)steps * (split + 1) / splits) * CT_K;
    const Operand a = keys ? Operand{c.gt, c.plane_gt, c.ld_gt} : Operand{c.g, c.plane_g, c.ld_g};
    const Operand b = keys ? Operand{c.qt, c.plane_qt, c.Bp} : Operand{c.kt, c.plane_kt, c.Mp};
    if constexpr (DT == DT_F32) product_of_terms(a, b, tr * TILE, tc * TILE, k0, k1, lds, acc, []() {});
    else product<TILE, DT>(a, b, tr * TILE, tc * TILE, k0, k1, lds, lds2, acc, []() {});
    const Place<TILE> at(tr, tc);
    const size_t rows = (size_t)((keys ? c.M : c.B) + CT_PAD - 1) / CT_PAD * CT_PAD;
    float *out = (keys ? c.acc_k : c.acc_q) + (size_t)split * rows * c.dr;
#pragma unroll
    for (int m = 0; m < N; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float *to = out + (size_t)(at.row + m * 4 + r) * c.dr + at.col;
#pragma unroll
            for (int n = 0; n < N; n += 4) *(f32x4 *)(to + n) = (f32x4){acc[m][n][r], acc[m][n + 1][r], acc[m][n + 2][r], acc[m][n + 3][r]};
        }
}

template <int DT, bool WIDE>
__device__ __forceinline__ void store4(void *rows, size_t row, int d, int e, const float (&x)[4])
{
    if constexpr (WIDE) store_pack<DT, 4>(rows, row * d + e, x);
    else
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (e + k < d) ((typename RowType<DT>::T *)rows)[row * d + e + k] = (typename RowType<DT>::T)x[k];
}

// A row of dQ or dK: the parts of its sum joined in order, less the row itself times the sum of its g.
template <int DT, bool WIDE> struct GradRow {
    const ContrastPar &c;
    bool keys;
    int row, splits, down;          // down: exponent of float16 rows' g
    const void *mine;
    const float *acc;
    size_t plane;
    float sum;
    __device__ __forceinline__ GradRow(const ContrastPar &par, int at) : c(par)
    {
        keys = at >= c.B;
        row = keys ? at - c.B : at;
        const int lane = threadIdx.x & 63, rows = keys ? c.M : c.B, parts = keys ? c.parts_q : c.parts_k;
        mine = keys ? c.K : c.Q;
        splits = keys ? c.splits_k : c.splits_q;
        const float *sums = (keys ? c.sum_k : c.sum_q) + (size_t)row * parts;
        sum = 0.0f;
        for (int t = lane; t < parts; t += 64) sum += sums[t];
        sum = wave_sum(sum);
        plane = (size_t)((rows + CT_PAD - 1) / CT_PAD * CT_PAD) * c.dr;
        acc = (keys ? c.acc_k : c.acc_q) + (size_t)row * c.dr;
        down = DT == DT_F16 ? -weight_exponent(*c.top) : 0;
    }
    // a: four coordinates of the sum; x: of the row
    __device__ __forceinline__ void load(int e, float (&a)[4], float (&x)[4]) const
    {
        for (int s = 0; s < splits; ++s) {
            const f32x4 part = *(const f32x4 *)&acc[s * plane + e];
#pragma unroll
            for (int k = 0; k < 4; ++k) a[k] += part[k];
        }
        load4<DT, WIDE>(mine, row, c.d, e, x);
        float from[4] = {x[0], x[1], x[2], x[3]};       // as the products had it
        if constexpr (DT == DT_F32) from_centre(c, e, from);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            a[k] = fmaf(-sum, from[k], a[k]);
            if (DT == DT_F16) a[k] = ldexpf(a[k], down);
        }
    }
    __device__ __forceinline__ void store(int e, float (&a)[4]) const
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) a[k] *= 2.0f * c.scale;
        store4<DT, WIDE>(keys ? c.dK : c.dQ, row, c.d, e, a);
    }
};

template <typename PAR>
__global__ void k_contrast_zero(unsigned short *p, size_t n)
{
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) p[i] = 0;
}

// ------------------------------------------------------------------------------------------------ host side

// How long `slots` workgroups take for na units of length a and nb of length b, the long ones first.
static double makespan(double a, long long na, double b, long long nb, int slots)
{
    if (a < b) {
        std::swap(a, b);
        std::swap(na, nb);
    }
    const long long r = na / slots, rem = na % slots;
    const double low = r * a, high = rem ? low + a : low;
    double t = high;
    for (int i = 0; i < 1000; ++i) {
        const long long fits = (rem ? rem * (long long)((t - high) / b + 1e-6) : 0) + (slots - rem) * (long long)((t - low) / b + 1e-6);
        if (fits >= nb) break;
        t += (double)(nb - fits) / slots < 1.0 ? b / 4 : b * (double)((nb - fits) / slots);
    }
    return t;
}

struct ContrastPlan {
    int tile, tile_g;
    bool terms;     // float32 rows: logits by product_of_terms()
};

// Tiles of 256 keep the matrix cores busier (see product()), tiles of 128 spread small problems over more CUs.
static ContrastPlan contrast_plan(ContrastPar &c, int planes)
{
    ContrastPlan p;
    auto tiles = [](int x, int t) { return (long long)(x + t - 1) / t; };
    // logits: tiles of 128 come two to a CU, one's product beside the other's logits, which is the longer part of short rows.  The whole call with
    // gradients, tiles of 128 / 256, us: 8,192 x 16,384, d = 64 418 / 464, 256 543 / 565, 384 684 / 691, 768 1,007 / 978, 1,536 1,699 / 1,601;
    // 1,000 x 11,000: d = 768 140 / 145 (172 tiles of 256 for 256 CUs), 1,536 242 / 244
    p.tile = c.tile ? c.tile : planes == 1 && c.d > 384 && tiles(c.B, 256) * tiles(c.M, 256) >= 512 ? 256 : 128;
    // float32 rows: product_of_terms() takes the LDS of a CU, so a second workgroup no longer works on its logits meanwhile.  It is ahead
    // where every workgroup has a CU of its own.  The whole call with two workgroups / with the terms together, us: 3,000 x 12,000,
    // d = 32 328 / 364, 128 368 / 416, 256 559 / 597, 384 754 / 800, 768 1,390 / 1,413, 1,536 2,680 / 2,678, 2,048 3,414 / 3,372; 2,200 x 2,200 x 128 (324 tiles)
    // 84 / 96, 700 x 4,000 x 300 (192 tiles) 109 / 104, 100 x 1,100 x 32 49.5 / 48.6.  (rnnd_contrast takes it from 321 coordinates on, where it was ahead
    // before the other product stopped waiting for its loads: its sums keep their order.)
    p.terms = planes == 3 && (c.d > (c.terms_from ? c.terms_from : 320) || tiles(c.B, 128) * tiles(c.M, 128) <= 256);
    // the gradient products: also by how much of the last tile of d would be padding.  The whole call, tiles of 128 / 256, us: 500 x 1,000 x 768
    // (18 tiles of 256) 57 / 71, 1,700 x 3,400 x 768 (63) 85 / 94, 2,048 x 4,096 x 768 (72) 88 / 98, 1,000 x 11,000 x 768 (141) 145 / 139,
    // 8,192 x 16,384 x 768 (288) 1,061 / 978; by padding, 4,096 x 8,192: d = 300 (512 for 384) 153 / 167, 600 (768 for 640) 237 / 248, 1,100 (1,280 for
    // 1,152) 393 / 409, 64 103 / 118.  (Between 64 and about 128 tiles, and at lengths like 600 and 1,100, tiles of 128 would be up to 10 % ahead.)
    const int d128 = ct_up(c.d, 128), d256 = ct_up(c.d, 256);
    p.tile_g = planes == 1 && (tiles(c.B, 256) + tiles(c.M, 256)) * (d256 / 256) >= 64 && d256 * 4 <= d128 * 5 ? 256 : 128;
    c.dp = ct_up(c.d, CT_K);
    c.Bp = ct_up(c.B, CT_K);
    c.Mp = ct_up(c.M, CT_K);
    c.dr = ct_up(c.d, p.tile_g);
    c.parts_k = 2 * (int)tiles(c.M, p.tile);
    c.parts_q = 2 * (int)tiles(c.B, p.tile);
    // parts of the gradients' sums: few tiles are split over the workgroups that run at a time; a part costs about 24 steps of the
    // product, for what it starts with and for its results, written and read again.  With 6 / 24 / 80 steps, us: 1,700 x 3,400 x 768 99 / 86 / 86,
    // 4,096 x 8,192 x 300 176 / 162 / 162, x 600 306 / 262 / 262, x 1,100 445 / 438 / 425, float32 2,000 x 10,000 x 100 234 / 233 / 242
    static const int choices[] = {1, 2, 3, 4, 6, 8, 12, 16};
    const long long tq = tiles(c.B, p.tile_g) * (c.dr / p.tile_g), tk = tiles(c.M, p.tile_g) * (c.dr / p.tile_g);
    const int steps_q = c.Mp / CT_K * (planes == 3 ? 6 : 1), steps_k = c.Bp / CT_K * (planes == 3 ? 6 : 1);
    double best = 1e300;
    for (int sq : choices)
        for (int sk : choices) {
            if ((sq > 1 && sq > c.Mp / CT_K) || (sk > 1 && sk > c.Bp / CT_K)) continue;
            const double t = makespan((double)steps_q / sq + 24, tq * sq, (double)steps_k / sk + 24, tk * sk, p.tile_g == 256 || planes == 3 ? 256 : 512);
            if (t < best * 0.999) {
                best = t;
                c.splits_q = sq;
                c.splits_k = sk;
            }
        }
    return p;
}

// more(take): arrays that a call has besides
template <typename F>
static size_t contrast_layout(ContrastPar &c, ContrastPlan &plan, int dtype, int want_grad, char *base, F more)
{
    const int planes = dtype == RNND_F32 ? 3 : 1;
    plan = contrast_plan(c, planes);
    const size_t Br = ct_up(c.B, CT_PAD), Mr = ct_up(c.M, CT_PAD);
    size_t off = 0;
    auto take = [&](auto *&p, size_t count) {
        p = (typename std::remove_reference<decltype(p)>::type)(base + off);
        off += ws_align(count * sizeof(*p));
    };
    take(c.tops, CT_ROW_BLOCKS);
    take(c.top, 1);
    more(take);
    if (planes == 3) take(c.centre, c.dp);
    take(c.key_base, Mr);
    take(c.key_id, Mr);
    take(c.row_id, Br);
    take(c.row_g, Br);
    take(c.row_own, Br);
    take(c.part, Br * c.parts_k);
    take(c.q, planes * (c.plane_q = Br * c.dp));
    c.plane_k = Mr * c.dp;
    if (!c.keys_as_they_are) take(c.k, planes * c.plane_k);
    if (want_grad) {
        take(c.qt, planes * (c.plane_qt = (size_t)c.dr * c.Bp));
        take(c.kt, planes * (c.plane_kt = (size_t)c.dr * c.Mp));
        c.ld_g = (int)Mr;
        c.ld_gt = (int)Br;
        take(c.g, planes * (c.plane_g = Br * Mr));
        take(c.gt, planes * (c.plane_gt = Mr * Br));
        take(c.sum_q, Br * c.parts_k);
        take(c.sum_k, Mr * c.parts_q);
        take(c.acc_q, (size_t)c.splits_q * Br * c.dr);
        take(c.acc_k, (size_t)c.splits_k * Mr * c.dr);
    }
    return off;
}

static int check_contrast(int64_t B, int64_t M, int32_t d, int dtype)
{
    if (!row_type(dtype)) return RNND_ERR_UNSUPPORTED;
    if (B < 0 || B > RNND_MAX_CONTRAST || M < 1 || M > RNND_MAX_CONTRAST || d < 1 || d > RNND_MAX_ROW) return RNND_ERR_BAD_SHAPE;
    return RNND_OK;
}

template <int DT, int TILE, typename PAR>
static void launch_grads(PAR &c, hipStream_t st)
{
    const int tq = ct_up(c.B, TILE) / TILE, tk = ct_up(c.M, TILE) / TILE, td = c.dr / TILE;
    in_launches((u64)td * (tq * c.splits_q + tk * c.splits_k), 256, [&](u64 first, u64 blocks) {
        hipLaunchKernelGGL((k_contrast_grad<TILE, DT, PAR>), dim3((u32)blocks), dim3(256), 0, st, c, (u32)first, tq, tk, td);
    });
}
