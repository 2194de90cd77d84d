// Softmax loss over squared distances, and its gradients: the loss that trains the rows of an index.
//
//   s_ij   = bias_j - scale |q_i - k_j|^2                       logit of key j for query i
//   loss_i = log( sum_j exp s_ij ) - s_it                       t = target[i]; the sum over the keys not left out
//   g_ij   = w_i (p_ij - [j = t]),  p_ij = exp(s_ij - lse_i)
//   dq_i   = 2 scale sum_j g_ij (k_j - q_i)                     gradients of sum_i w_i loss_i
//   dk_j   = 2 scale sum_i g_ij (q_i - k_j)
//
// |q_i|^2 is the same in a whole row and cancels, so a logit is 2 scale q.k + (bias - scale |k|^2): three products of the
// shape B x M x d (q k', g k and g' q), on the matrix cores.  The logits are never stored: the first product keeps the
// largest and the sum of each row and tile, the second forms the logits again and writes g in 16 bits, once by
// rows and once by columns, so that every product reads both operands along its sum.
//
// What is exact, what is rounded:
//   - 16-bit rows go to the matrix instructions as they are; float32 rows as three bfloat16 terms each (8 + 8 + 8 bits), of whose
//     products the six largest are summed: what is left out is below 2^-24 of |a||b|.
//   - all sums are float32.  The target is kept out of the row's sum: with x = lse over the others - s_t, loss = log(1 + e^x)
//     and p_t - 1 = -(1 - e^-loss), neither of which cancels when the loss is small.
//   - g is rounded to the type of the rows (float32 rows: three terms again).  The rounding leaves sum_j g_ij a little off
//     zero, which rows far from the origin would turn into a large error: the gradients are formed from k_j - q_i, with the sums
//     of the rounded g, as the formulas have it.  float16: g is scaled to below 2^15 first, so that it stays normal down to 2^-29
//     of the largest weight.
#include <cmath>
#include <type_traits>

#include "rows.h"

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

#define CT_TILE 128         // rows and columns of a workgroup's tile
#define CT_K 64             // summed per step: 128 bytes of a row
#define CT_NEVER (-2)       // an id that no key has

struct RowInfo { float lse, weight, own; int target, target_id, query_id; };    // lse in base 2; own = g at the target

struct ContrastPar {
    const void *Q, *K;
    const int *target, *query_ids, *key_ids;
    const float *bias, *row_weight;
    float scale, c1;                // c1 = 2 scale log2(e)
    int B, M, d;
    int dp, Bp, Mp;                 // padded to CT_K
    size_t plane_q, plane_k, plane_qt, plane_kt, plane_g, plane_gt;     // elements
    unsigned short *q, *k, *qt, *kt, *g, *gt;
    float *key_base;                // [Mp128] (bias - scale |k|^2) log2(e), -inf where left out
    int *key_id;                    // [Mp128]
    float2 *part;                   // [B][tiles of M] largest and sum of a row's tile
    float *own_logit;               // [B]
    RowInfo *row;                   // [Bp128]
    u32 *weight_top;                // largest |w| as bits
    float *sum_q, *sum_k;           // [B][tiles of M], [M][tiles of B]: sums of the rounded g
    float *acc_q, *acc_k;           // [splits][rows][d]
    int splits_q, splits_k;
    float *loss;
    void *dQ, *dK;
};

// ------------------------------------------------------------------------------------------------ preparation
__device__ __forceinline__ bool key_gone(const ContrastPar &c, int j)
{
    return (c.key_ids && c.key_ids[j] < 0) || (c.bias && c.bias[j] == -INFINITY);
}
__device__ __forceinline__ bool row_counts(const ContrastPar &c, int i)
{
    const int t = c.target[i];
    return (u32)t < (u32)c.M && !key_gone(c, t);
}

// a wavefront per key, then a thread per query
template <int DT>
__global__ __launch_bounds__(256) void k_contrast_rows(ContrastPar c, u32 key_blocks)
{
    if (blockIdx.x >= key_blocks) {
        const int i = (blockIdx.x - key_blocks) * 256 + threadIdx.x;
        const int padded = (c.B + CT_TILE - 1) / CT_TILE * CT_TILE;
        if (i >= padded) return;
        RowInfo r = {0.0f, 0.0f, 0.0f, -1, CT_NEVER, CT_NEVER};
        if (i < c.B && row_counts(c, i)) {
            r.target = c.target[i];
            r.weight = c.row_weight ? c.row_weight[i] : 1.0f;
            if (c.key_ids) {
                r.target_id = c.key_ids[r.target];
                if (c.query_ids) r.query_id = c.query_ids[i];
            }
            if (DT == DT_F16) {
                const u32 w = __float_as_uint(r.weight) & 0x7FFFFFFFu;
                if (w < 0x7F800000u) atomicMax(c.weight_top, w);
            }
        }
        c.row[i] = r;
        return;
    }
    const int j = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int padded = (c.M + CT_TILE - 1) / CT_TILE * CT_TILE;
    if (j >= padded) return;
    if (j >= c.M || key_gone(c, j)) {
        if (lane == 0) {
            c.key_base[j] = -INFINITY;
            c.key_id[j] = -1;
        }
        return;
    }
    const typename RowType<DT>::T *k = (const typename RowType<DT>::T *)c.K + (size_t)j * c.d;
    float sum = 0.0f;
    for (int e = lane; e < c.d; e += 64) {
        const float x = (float)k[e];
        sum = fmaf(x, x, sum);
    }
#pragma unroll
    for (int s = 32; s; s >>= 1) sum += __shfl_xor(sum, s);
    if (lane == 0) {
        c.key_base[j] = ((c.bias ? c.bias[j] : 0.0f) - c.scale * sum) * 1.44269504f;
        c.key_id[j] = c.key_ids ? c.key_ids[j] : -1;
    }
}

__device__ __forceinline__ unsigned short bits16(__bf16 x) { return __builtin_bit_cast(unsigned short, x); }
__device__ __forceinline__ unsigned short bits16(_Float16 x) { return __builtin_bit_cast(unsigned short, x); }

// The planes of a value: itself in 16 bits, or three bfloat16 terms.
template <int DT, int PLANES>
__device__ __forceinline__ void to_planes(float x, unsigned short (&o)[PLANES])
{
    if constexpr (PLANES == 1) {
        if constexpr (DT == DT_F16) o[0] = bits16((_Float16)x);
        else o[0] = bits16((__bf16)x);
    } else {
#pragma unroll
        for (int p = 0; p < PLANES; ++p) {
            const __bf16 h = (__bf16)x;
            o[p] = bits16(h);
            x -= (float)h;
        }
    }
}

// Copies of the rows that the products read: padded with zeros, in planes, by rows and by columns; rows that do not count and
// keys that are left out as zeros, whatever they hold.  One block per 64 x 64.
template <int DT, int PLANES>
__global__ __launch_bounds__(256) void k_contrast_copy(ContrastPar c, u32 q_tiles, int columns)
{
    __shared__ unsigned short tile[64][66];
    const bool keys = blockIdx.x >= q_tiles;
    const int r0 = (int)(keys ? blockIdx.x - q_tiles : blockIdx.x) * 64, c0 = blockIdx.y * 64;
    const int rows = keys ? c.M : c.B;
    const typename RowType<DT>::T *x = (const typename RowType<DT>::T *)(keys ? c.K : c.Q);
    unsigned short *by_row = keys ? c.k : c.q, *by_col = keys ? c.kt : c.qt;
    const size_t plane_r = keys ? c.plane_k : c.plane_q, plane_c = keys ? c.plane_kt : c.plane_qt;
    const int across = keys ? c.Mp : c.Bp;
    const int col = threadIdx.x & 63;
    unsigned short o[16][PLANES];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int r = r0 + (threadIdx.x >> 6) + 4 * i;
        float v = 0.0f;
        if (r < rows && c0 + col < c.d && (keys ? !key_gone(c, r) : row_counts(c, r))) v = (float)x[(size_t)r * c.d + c0 + col];
        to_planes<DT, PLANES>(v, o[i]);
#pragma unroll
        for (int p = 0; p < PLANES; ++p)
            if (c0 < c.dp) by_row[p * plane_r + (size_t)r * c.dp + c0 + col] = o[i][p];
    }
    if (!columns) return;
#pragma unroll
    for (int p = 0; p < PLANES; ++p) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 16; ++i) tile[(threadIdx.x >> 6) + 4 * i][col] = o[i][p];
        __syncthreads();
        if (r0 < across)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int cc = (threadIdx.x >> 6) + 4 * i;
                by_col[p * plane_c + (size_t)(c0 + cc) * across + r0 + col] = tile[col][cc];
            }
    }
}

// ------------------------------------------------------------------------------------------------ the product
// 128 x 128 results of A B' (both with the summed index along the row), 4 wavefronts of 64 x 64.  A step's 128 bytes of a
// row lie in LDS as 8 pieces of 16 bytes, piece s of row r at place s ^ (r % 8): the loads go straight to LDS in its own order
// (each lane fetches the piece that belongs at its place), and the 16 rows that a matrix instruction reads together
// spread over the banks.
template <int DT>
__device__ __forceinline__ f32x4 mfma16(const uint4 &a, const uint4 &b, f32x4 c)
{
    if constexpr (DT == DT_F16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

struct Operand { const unsigned short *p; size_t plane; int ld; };      // rows of ld elements, ld a multiple of CT_K

__device__ __forceinline__ void lds_load16(const unsigned short *from, unsigned short *to)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                     (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}

struct ProductLds { unsigned short a[2][CT_TILE * CT_K], b[2][CT_TILE * CT_K]; };

template <int PLANES> __device__ __forceinline__ void plane_pair(int i, int &a, int &b)
{
    a = b = 0;
    if constexpr (PLANES == 3) {        // (0,0) (0,1) (1,0) (1,1) (0,2) (2,0)
        a = i == 2 || i == 3 ? 1 : i == 5 ? 2 : 0;
        b = i == 1 || i == 3 ? 1 : i == 4 ? 2 : 0;
    }
}

template <int DT, int PLANES>
__device__ __forceinline__ void product(const Operand &A, const Operand &B, int row_a, int row_b, int k_begin, int k_end,
                                        ProductLds &lds, f32x4 (&acc)[4][4])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int per = (k_end - k_begin) / CT_K;
    const int steps = per * (PLANES == 3 ? 6 : 1);
    const int piece = (lane & 7) ^ (lane >> 3);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    // each wavefront brings 32 rows of A and of B, 8 at a time
    auto fetch = [&](int s, int buf) {
        int pa = 0, pb = 0, kk = s;
        if (PLANES == 3) {
            const int pair = s / per;
            kk = s - pair * per;
            plane_pair<PLANES>(pair, pa, pb);
        }
        const size_t k0 = (size_t)k_begin + (size_t)kk * CT_K + piece * 8;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = wave * 32 + i * 8;
            lds_load16(A.p + pa * A.plane + (size_t)(row_a + r + (lane >> 3)) * A.ld + k0, &lds.a[buf][r * CT_K]);
            lds_load16(B.p + pb * B.plane + (size_t)(row_b + r + (lane >> 3)) * B.ld + k0, &lds.b[buf][r * CT_K]);
        }
    };
    if (steps > 0) fetch(0, 0);
    const int ra = (wave >> 1) * 64 + (lane & 15), rb = (wave & 1) * 64 + (lane & 15);
    for (int s = 0; s < steps; ++s) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (s + 1 < steps) fetch(s + 1, (s + 1) & 1);
        const unsigned short *la = lds.a[s & 1], *lb = lds.b[s & 1];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint4 fa[4], fb[4];
            const int at = ((h * 4 + (lane >> 4)) ^ (lane & 7)) * 8;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                fa[i] = *(const uint4 *)&la[(ra + i * 16) * CT_K + at];
                fb[i] = *(const uint4 *)&lb[(rb + i * 16) * CT_K + at];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = mfma16<DT>(fa[i], fb[j], acc[i][j]);
        }
    }
    __syncthreads();
}

// the logit of acc for row info r and column j, base 2; -inf where the pair is left out
__device__ __forceinline__ float logit2(float acc, float c1, float base, int id, const RowInfo &r, int j)
{
    const float s = fmaf(acc, c1, base);
    return base == -INFINITY || ((id == r.target_id || id == r.query_id) && j != r.target) ? -INFINITY : s;
}

// ------------------------------------------------------------------------------------------------ first product: largest and sum of every row
template <int DT, int PLANES>
__global__ __launch_bounds__(256) void k_contrast_sums(ContrastPar c)
{
    __shared__ ProductLds lds;
    f32x4 acc[4][4];
    const int row0 = blockIdx.y * CT_TILE, col0 = blockIdx.x * CT_TILE;
    product<DT, PLANES>({c.q, c.plane_q, c.dp}, {c.k, c.plane_k, c.dp}, row0, col0, 0, c.dp, lds, acc);
    float2 (*half)[CT_TILE] = (float2 (*)[CT_TILE])&lds;        // [2 halves of the columns][row]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int cb = (wave & 1) * 64 + (lane & 15);
    float base[4];
    int id[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        base[j] = c.key_base[col0 + cb + j * 16];
        id[j] = c.key_id[col0 + cb + j * 16];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int local = (wave >> 1) * 64 + i * 16 + (lane >> 4) * 4 + r;
            const RowInfo info = c.row[row0 + local];
            float s[4], top = -INFINITY;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int col = col0 + cb + j * 16;
                s[j] = logit2(acc[i][j][r], c.c1, base[j], id[j], info, col);
                if (col == info.target) {
                    c.own_logit[row0 + local] = s[j];
                    s[j] = -INFINITY;
                }
                top = s[j] > top || s[j] != s[j] ? s[j] : top;
            }
            // over the 16 lanes that share the row; a NaN stays
#pragma unroll
            for (int k = 1; k < 16; k <<= 1) {
                const float o = __shfl_xor(top, k);
                top = o > top || o != o ? o : top;
            }
            float sum = 0.0f;
            if (top != -INFINITY)
#pragma unroll
                for (int j = 0; j < 4; ++j) sum += __builtin_amdgcn_exp2f(s[j] - top);
#pragma unroll
            for (int k = 1; k < 16; k <<= 1) sum += __shfl_xor(sum, k);
            if ((lane & 15) == 0) half[wave & 1][local] = make_float2(top, sum);
        }
    __syncthreads();
    if (threadIdx.x < CT_TILE && row0 + (int)threadIdx.x < c.B) {
        const float2 a = half[0][threadIdx.x], b = half[1][threadIdx.x];
        const float top = a.x > b.x || a.x != a.x ? a.x : b.x;
        const float sum = top == -INFINITY ? 0.0f : a.y * __builtin_amdgcn_exp2f(a.x - top) + b.y * __builtin_amdgcn_exp2f(b.x - top);
        c.part[(size_t)(row0 + threadIdx.x) * gridDim.x + blockIdx.x] = make_float2(top, sum);
    }
}

// A wavefront per query joins its tiles: the loss, and what the second product needs.
template <int DT>
__global__ __launch_bounds__(256) void k_contrast_loss(ContrastPar c, int tiles)
{
    const int i = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (i >= c.B) return;
    RowInfo r = c.row[i];
    float top = -INFINITY, sum = 0.0f;
    for (int t = lane; t < tiles; t += 64) {
        const float2 p = c.part[(size_t)i * tiles + t];
        if (p.x == -INFINITY) continue;
        const float m = p.x > top || p.x != p.x ? p.x : top;
        sum = (top == -INFINITY ? 0.0f : sum * __builtin_amdgcn_exp2f(top - m)) + p.y * __builtin_amdgcn_exp2f(p.x - m);
        top = m;
    }
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const float ot = __shfl_xor(top, s), os = __shfl_xor(sum, s);
        const float m = ot > top || ot != ot ? ot : top;
        sum = m == -INFINITY ? 0.0f : (top == -INFINITY ? 0.0f : sum * __builtin_amdgcn_exp2f(top - m)) +
                                          (ot == -INFINITY ? 0.0f : os * __builtin_amdgcn_exp2f(ot - m));
        top = m;
    }
    if (lane) return;
    if (r.target < 0) {
        c.loss[i] = 0.0f;
        return;
    }
    // x = lse of the others - own logit; loss = log(1 + e^x)
    const float own = c.own_logit[i], ln2 = 0.693147181f;
    float loss = 0.0f;
    if (top != -INFINITY) {
        const float x = (top - own + log2f(sum)) * ln2;
        loss = x > 0.0f ? x + log1pf(expf(-x)) : log1pf(expf(x));
    }
    c.loss[i] = loss;
    float w = r.weight;
    if (DT == DT_F16) {     // times a power of two that brings the largest weight into [2^14, 2^15)
        const u32 t = *c.weight_top;
        if (t >= 0x00800000u) w = ldexpf(w, 14 + 127 - (int)(t >> 23));
    }
    r.weight = w;
    r.own = expm1f(-loss) * w;
    r.lse = own + loss * 1.44269504f;
    c.row[i] = r;
}

// ------------------------------------------------------------------------------------------------ second product: g
template <int DT, int PLANES>
__global__ __launch_bounds__(256) void k_contrast_g(ContrastPar c)
{
    __shared__ ProductLds lds;
    f32x4 acc[4][4];
    const int row0 = blockIdx.y * CT_TILE, col0 = blockIdx.x * CT_TILE;
    product<DT, PLANES>({c.q, c.plane_q, c.dp}, {c.k, c.plane_k, c.dp}, row0, col0, 0, c.dp, lds, acc);
    float (*row_half)[CT_TILE] = (float (*)[CT_TILE])&lds, (*col_half)[CT_TILE] = row_half + 2;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int cb = (wave & 1) * 64 + (lane & 15), rb = (wave >> 1) * 64 + (lane >> 4) * 4;
    float base[4], col_sum[4] = {};
    int id[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        base[j] = c.key_base[col0 + cb + j * 16];
        id[j] = c.key_id[col0 + cb + j * 16];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        unsigned short o[4][4][PLANES];     // [row][column]
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int local = rb + i * 16 + r;
            const RowInfo info = c.row[row0 + local];
            float row_sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int col = col0 + cb + j * 16;
                const float s = logit2(acc[i][j][r], c.c1, base[j], id[j], info, col);
                float g = s == -INFINITY || info.target < 0 ? 0.0f : __builtin_amdgcn_exp2f(s - info.lse) * info.weight;
                if (col == info.target) g = info.own;
                to_planes<DT, PLANES>(g, o[r][j]);
                if constexpr (PLANES == 1) g = DT == DT_F16 ? (float)__builtin_bit_cast(_Float16, o[r][j][0]) : (float)__builtin_bit_cast(__bf16, o[r][j][0]);
                row_sum += g;
                col_sum[j] += g;
            }
#pragma unroll
            for (int k = 1; k < 16; k <<= 1) row_sum += __shfl_xor(row_sum, k);
            if ((lane & 15) == 0) row_half[wave & 1][local] = row_sum;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int col = col0 + cb + j * 16, row = row0 + rb + i * 16;
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
                if (col < c.Mp)
#pragma unroll
                    for (int r = 0; r < 4; ++r) c.g[p * c.plane_g + (size_t)(row + r) * c.Mp + col] = o[r][j][p];
                if (row < c.Bp) {
                    const uint2 four = {o[0][j][p] | (u32)o[1][j][p] << 16, o[2][j][p] | (u32)o[3][j][p] << 16};
                    *(uint2 *)&c.gt[p * c.plane_gt + (size_t)col * c.Bp + row] = four;
                }
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        col_sum[j] += __shfl_xor(col_sum[j], 16);
        col_sum[j] += __shfl_xor(col_sum[j], 32);
        if (lane < 16) col_half[wave >> 1][cb + j * 16] = col_sum[j];
    }
    __syncthreads();
    const int x = threadIdx.x & 127;
    if (threadIdx.x < 128) {
        if (row0 + x < c.B) c.sum_q[(size_t)(row0 + x) * gridDim.x + blockIdx.x] = row_half[0][x] + row_half[1][x];
    } else if (col0 + x < c.M)
        c.sum_k[(size_t)(col0 + x) * gridDim.y + blockIdx.y] = col_half[0][x] + col_half[1][x];
}

// ------------------------------------------------------------------------------------------------ third and fourth: g k and g' q
template <int DT, int PLANES>
__global__ __launch_bounds__(256) void k_contrast_grad(ContrastPar c, int keys)
{
    __shared__ ProductLds lds;
    f32x4 acc[4][4];
    const int row0 = blockIdx.y * CT_TILE, col0 = blockIdx.x * CT_TILE;
    const int rows = keys ? c.M : c.B, depth = keys ? c.Bp : c.Mp, splits = keys ? c.splits_k : c.splits_q;
    const int steps = depth / CT_K, k0 = (int)((long long)steps * blockIdx.z / splits) * CT_K,
              k1 = (int)((long long)steps * (blockIdx.z + 1) / splits) * CT_K;
    if (keys) product<DT, PLANES>({c.gt, c.plane_gt, c.Bp}, {c.qt, c.plane_qt, c.Bp}, row0, col0, k0, k1, lds, acc);
    else product<DT, PLANES>({c.g, c.plane_g, c.Mp}, {c.kt, c.plane_kt, c.Mp}, row0, col0, k0, k1, lds, acc);
    float *out = (keys ? c.acc_k : c.acc_q) + (size_t)blockIdx.z * rows * c.d;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = row0 + (wave >> 1) * 64 + i * 16 + (lane >> 4) * 4 + r, col = col0 + (wave & 1) * 64 + j * 16 + (lane & 15);
                if (row < rows && col < c.d) out[(size_t)row * c.d + col] = acc[i][j][r];
            }
}

// Joins the parts of a sum in order, takes off the row itself times the sum of its g, and rounds.  A wavefront per row.
template <int DT>
__global__ __launch_bounds__(256) void k_contrast_finish(ContrastPar c, int tiles_k, int tiles_q)
{
    const int at = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (at >= c.B + c.M) return;
    const bool keys = at >= c.B;
    const int row = keys ? at - c.B : at, rows = keys ? c.M : c.B, tiles = keys ? tiles_q : tiles_k;
    typedef typename RowType<DT>::T T;
    T *out = (T *)(keys ? c.dK : c.dQ) + (size_t)row * c.d;
    if (keys ? key_gone(c, row) : !row_counts(c, row)) {
        for (int e = lane; e < c.d; e += 64) out[e] = (T)0.0f;
        return;
    }
    const float *sums = (keys ? c.sum_k : c.sum_q) + (size_t)row * tiles;
    float sum = 0.0f;
    for (int t = lane; t < tiles; t += 64) sum += sums[t];
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) sum += __shfl_xor(sum, s);
    const T *x = (const T *)(keys ? c.K : c.Q) + (size_t)row * c.d;
    const float *acc = (keys ? c.acc_k : c.acc_q) + (size_t)row * c.d;
    const int splits = keys ? c.splits_k : c.splits_q;
    float f = 2.0f * c.scale;
    int down = 0;
    if (DT == DT_F16) {
        const u32 t = *c.weight_top;
        if (t >= 0x00800000u) down = 14 + 127 - (int)(t >> 23);
    }
    for (int e = lane; e < c.d; e += 64) {
        float a = 0.0f;
        for (int s = 0; s < splits; ++s) a += acc[(size_t)s * rows * c.d + e];
        a = fmaf(-sum, (float)x[e], a) * f;
        if (DT == DT_F16) a = ldexpf(a, -down);
        out[e] = (T)a;
    }
}

__global__ void k_contrast_clear(u32 *p) { *p = 0; }
__global__ void k_contrast_zero(unsigned short *p, size_t n)
{
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) p[i] = 0;
}

// ------------------------------------------------------------------------------------------------ host side
static int ct_up(int x, int m) { return (x + m - 1) / m * m; }

// Workgroups that a gradient product should have at least; the sum is split among them where its results are too few tiles.
static int ct_splits(int rows, int d, int depth)
{
    const long long tiles = (long long)ct_up(rows, CT_TILE) / CT_TILE * (ct_up(d, CT_TILE) / CT_TILE);
    int splits = (int)(512 / tiles);
    const int most = depth / (4 * CT_K);        // at least four steps each
    if (splits > most) splits = most;
    return splits < 1 ? 1 : splits;
}

static size_t contrast_layout(ContrastPar &c, int dtype, int want_grad, char *base)
{
    const int planes = dtype == RNND_F32 ? 3 : 1;
    const size_t Br = ct_up(c.B, CT_TILE), Mr = ct_up(c.M, CT_TILE), dr = ct_up(c.d, CT_TILE);
    const size_t tq = Br / CT_TILE, tk = Mr / CT_TILE;
    c.dp = ct_up(c.d, CT_K);
    c.Bp = ct_up(c.B, CT_K);
    c.Mp = ct_up(c.M, CT_K);
    size_t off = 0;
    auto take = [&](auto *&p, size_t count) {
        p = (typename std::remove_reference<decltype(p)>::type)(base + off);
        off += ws_align(count * sizeof(*p));
    };
    take(c.weight_top, 1);
    take(c.key_base, Mr);
    take(c.key_id, Mr);
    take(c.row, Br);
    take(c.own_logit, Br);
    take(c.part, (size_t)c.B * tk);
    take(c.q, planes * (c.plane_q = Br * c.dp));
    take(c.k, planes * (c.plane_k = Mr * c.dp));
    if (want_grad) {
        c.splits_q = ct_splits(c.B, c.d, c.Mp);
        c.splits_k = ct_splits(c.M, c.d, c.Bp);
        take(c.qt, planes * (c.plane_qt = dr * c.Bp));
        take(c.kt, planes * (c.plane_kt = dr * c.Mp));
        take(c.g, planes * (c.plane_g = Br * c.Mp));
        take(c.gt, planes * (c.plane_gt = Mr * c.Bp));
        take(c.sum_q, (size_t)c.B * tk);
        take(c.sum_k, (size_t)c.M * tq);
        take(c.acc_q, (size_t)c.splits_q * c.B * c.d);
        take(c.acc_k, (size_t)c.splits_k * c.M * c.d);
    }
    return off;
}

static int check_contrast(int64_t B, int64_t M, int32_t d, int dtype)
{
    if (!row_type(dtype)) return RNND_ERR_UNSUPPORTED;
    if (B < 0 || B > RNND_MAX_CONTRAST || M < 1 || M > RNND_MAX_CONTRAST || d < 1 || d > RNND_MAX_ROW) return RNND_ERR_BAD_SHAPE;
    return RNND_OK;
}

extern "C" int rnnd_contrast_workspace(int64_t B, int64_t M, int32_t d, int dtype, int want_grad, size_t *bytes)
{
    const int rc = check_contrast(B, M, d, dtype);
    if (rc) return rc;
    if (!bytes) return RNND_ERR_NULL;
    if (!B) {
        *bytes = 0;
        return RNND_OK;
    }
    ContrastPar c = {};
    c.B = (int)B;
    c.M = (int)M;
    c.d = d;
    *bytes = contrast_layout(c, dtype, want_grad, nullptr);
    return RNND_OK;
}

template <int DT>
static void launch_contrast(ContrastPar &c, int want_grad, hipStream_t st)
{
    constexpr int PLANES = DT == DT_F32 ? 3 : 1;
    const u32 tq = ct_up(c.B, CT_TILE) / CT_TILE, tk = ct_up(c.M, CT_TILE) / CT_TILE, td = ct_up(c.d, CT_TILE) / CT_TILE;
    if (DT == DT_F16) hipLaunchKernelGGL(k_contrast_clear, dim3(1), dim3(1), 0, st, c.weight_top);
    const u32 key_blocks = tk * CT_TILE / 4;
    hipLaunchKernelGGL(k_contrast_rows<DT>, dim3(key_blocks + (tq * CT_TILE + 255) / 256), dim3(256), 0, st, c, key_blocks);
    // (by columns the padding of d up to a whole tile is written too: the products read it)
    hipLaunchKernelGGL((k_contrast_copy<DT, PLANES>), dim3(tq * 2 + tk * 2, want_grad ? td * 2 : c.dp / 64), dim3(256), 0, st, c, tq * 2, want_grad);
    hipLaunchKernelGGL((k_contrast_sums<DT, PLANES>), dim3(tk, tq), dim3(256), 0, st, c);
    hipLaunchKernelGGL(k_contrast_loss<DT>, dim3((c.B + 3) / 4), dim3(256), 0, st, c, (int)tk);
    if (!want_grad) return;
    hipLaunchKernelGGL((k_contrast_g<DT, PLANES>), dim3(tk, tq), dim3(256), 0, st, c);
    hipLaunchKernelGGL((k_contrast_grad<DT, PLANES>), dim3(td, tq, c.splits_q), dim3(256), 0, st, c, 0);
    hipLaunchKernelGGL((k_contrast_grad<DT, PLANES>), dim3(td, tk, c.splits_k), dim3(256), 0, st, c, 1);
    hipLaunchKernelGGL(k_contrast_finish<DT>, dim3((c.B + c.M + 3) / 4), dim3(256), 0, st, c, (int)tk, (int)tq);
}

extern "C" int rnnd_contrast(const void *Q, int64_t B, const void *K, int64_t M, int32_t d, int dtype, int metric, const int32_t *target,
                             const int32_t *query_ids, const int32_t *key_ids, const float *key_bias, const float *row_weight, float scale,
                             float *loss, void *dQ, void *dK, void *workspace, size_t workspace_bytes, void *stream)
{
    const int rc = check_contrast(B, M, d, dtype);
    if (rc) return rc;
    if (metric != RNND_L2SQ) return RNND_ERR_UNSUPPORTED;
    if (!K || (B && (!Q || !target || !loss)) || (query_ids && !key_ids)) return RNND_ERR_NULL;
    if (B && (dQ == nullptr) != (dK == nullptr)) return RNND_ERR_NULL;
    const size_t size = dt_size(dtype);
    if (((uintptr_t)Q | (uintptr_t)K | (uintptr_t)dQ | (uintptr_t)dK) % size) return RNND_ERR_BAD_PARAM;
    if (((uintptr_t)target | (uintptr_t)query_ids | (uintptr_t)key_ids | (uintptr_t)key_bias | (uintptr_t)row_weight | (uintptr_t)loss) % 4)
        return RNND_ERR_BAD_PARAM;
    if (!std::isfinite(scale)) return RNND_ERR_BAD_PARAM;
    const int want_grad = dK != nullptr;
    if (!B) {       // no query: no gradient reaches a key
        if (!want_grad) return RNND_OK;
        const size_t n = (size_t)M * d * size / 2, blocks = (n + 1023) / 1024;
        hipLaunchKernelGGL(k_contrast_zero, dim3((u32)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, (hipStream_t)stream,
                           (unsigned short *)dK, n);
        return launched("rnnd_contrast");
    }
    ContrastPar c = {};
    c.Q = Q;
    c.K = K;
    c.target = target;
    c.query_ids = query_ids;
    c.key_ids = key_ids;
    c.bias = key_bias;
    c.row_weight = row_weight;
    c.scale = scale;
    c.c1 = (float)(2.0 * scale * 1.4426950408889634);
    c.B = (int)B;
    c.M = (int)M;
    c.d = d;
    c.loss = loss;
    c.dQ = dQ;
    c.dK = dK;
    if (!workspace) return RNND_ERR_NULL;
    if ((uintptr_t)workspace % 16) return RNND_ERR_BAD_PARAM;
    if (workspace_bytes < contrast_layout(c, dtype, want_grad, (char *)workspace)) return RNND_ERR_SCRATCH;
    if (dtype == RNND_F32) launch_contrast<DT_F32>(c, want_grad, (hipStream_t)stream);
    else if (dtype == RNND_F16) launch_contrast<DT_F16>(c, want_grad, (hipStream_t)stream);
    else launch_contrast<DT_BF16>(c, want_grad, (hipStream_t)stream);
    return launched("rnnd_contrast");
}
