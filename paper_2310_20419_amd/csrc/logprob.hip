// Log probabilities under the softmax over squared distances, its entropy, and the most probable keys in their exact order.
//
//   s_ij = bias_j - scale |q_i - k_j|^2,  lse_i = log sum_j exp s_ij,  log P_ij = s_ij - lse_i,  H_i = -sum_j P_ij log P_ij
//
// In one pass over the logits: of every row and part of the keys the largest logit m, sum exp(s - m) and sum exp(s - m) (s - m), which join
// like the first two do (all terms of the third have one sign: H = log sum - third / sum loses nothing), all in float32 and base 2.
//
// Alternatives.  The same pass keeps of each group of keys (8, or 4 with small tiles) the largest and the second largest logit; the number of the
// largest one's key stands in the lowest bits of its significand.  k keys are at least as large as the k-th largest of any values that are
// logits of different keys, so a bound on the k-th logit follows from the parts' largest, a better one from the groups of those parts, and
// what lies above the better one is little more than k keys.  Their distances are summed again in double precision from the rows as
// they are, and these decide the order.  The first pass is off by some error E: keys down to 2 E below the bound are taken along, so E costs
// time but changes no answer.  E is a bound from the rows' norms and the biases, of the keys that can be that probable: with scale > 0
// a logit of at least t has scale |q - k|^2 <= (largest bias) - t, so a key a long way off, or with a bias far below zero, does not count for it.  Where more keys than there is room for lie that close
// together (thousands of copies of a row), all groups above the bound are gone through in double precision instead.
#include <cmath>

#include "contrast.h"

#define LP_ROOM 256             // groups above the bound, and keys among them, that a wavefront has room for
#define LP_NONE (-3.0e38f)      // stands for -infinity where bits are put into the significand
#define LP_LIMIT (LP_NONE * 0.99f)      // logits that are not above it count as -infinity
#define LP_FAR (-1024.0f)        // 2^LP_FAR is 0 in float32, and times a sum it is still a number
#define LP_LOG2E 1.4426950408889634
#define LP_FEW 8                // queries at a time that are summed from differences
#define LP_ALONE 512            // queries, for each of which there is room for a block of eight wavefronts

struct LogprobPar : ContrastPar {
    int alternatives;
    float *logprob, *entropy, *top_logprob;
    int *top_ids;
    float *part_w;              // [B padded][parts_k] sum of 2^(s - top) (s - top), s in base 2
    float2 *groups;             // [B padded][parts_k][groups of a part] largest and second largest
    int group_shift, part_shift;    // keys of a group, groups of a part: powers of two
    float *most;                // [2][CT_ROW_BLOCKS] largest |k|^2 and bias_size() of a block of keys
    int most_blocks;
    bool squares;               // |k|^2 comes from the product's pass over the keys
    int few;                    // logits are from differences: the whole of s
};

__device__ __forceinline__ bool row_counts(const LogprobPar &, int) { return true; }

__device__ __forceinline__ bool leaves_out(const LogprobPar &c, int i, int j)
{
    return key_gone(c, j) || (c.query_ids && c.key_ids[j] == c.query_ids[i]);
}

// ------------------------------------------------------------------------------------------------ preparation
// What of a bias counts for the error of the largest logits; what is not a number counts as infinite.  Biases below zero: logits that reach t have
// biases of at least t, which counts for itself -- unless a negative scale makes them large again.
__device__ __forceinline__ float bias_size(const LogprobPar &c, float b)
{
    const float x = c.scale < 0.0f ? fabsf(b) : b <= 0.0f ? 0.0f : b;       // (without a sign: their bits are compared)
    return x < INFINITY ? x : INFINITY;
}
// The largest of a block's keys.
struct MostLds { u32 norm, bias; };
__device__ __forceinline__ void most_of(MostLds &most, const LogprobPar &c, int j, float norm)
{
    if (j >= c.M || key_gone(c, j)) return;
    atomicMax(&most.norm, __float_as_uint(norm < INFINITY ? norm : INFINITY));
    atomicMax(&most.bias, __float_as_uint(c.bias ? bias_size(c, c.bias[j]) : 0.0f));
}

// A wavefront per row, keys first; then the copies of the rows (contrast_copy()).  key_blocks: 0 where the keys have been prepared.
template <int DT, bool WIDE>
__global__ __launch_bounds__(256) void k_logprob_prepare(LogprobPar c, u32 first, int key_blocks, int row_blocks, int q_tiles, int across)
{
    __shared__ MostLds most;
    const int block = (int)(first + blockIdx.x), id = block - key_blocks - row_blocks;
    if (id >= 0) {
        contrast_copy<DT, WIDE>(c, id / across, id % across * 64, q_tiles, 0);
        return;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (block < key_blocks) {
        if (threadIdx.x == 0) most = {0, 0};
        __syncthreads();
        const int padded = ct_up(c.M, CT_PAD);
        for (int at = (block * 4 + wave) * 4; at < padded; at += key_blocks * 16) {
            const int four[4] = {at, at + 1, at + 2, at + 3};
            float norm[4];
            if (c.keys_as_they_are) key_sides<DT, WIDE, 4, true>(c, four, padded, lane, norm);
            else key_sides<DT, WIDE, 4>(c, four, padded, lane, norm);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (lane == r) most_of(most, c, at + r, norm[r]);
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            c.most[block] = __uint_as_float(most.norm);
            c.most[CT_ROW_BLOCKS + block] = __uint_as_float(most.bias);
        }
        return;
    }
    for (int at = (block - key_blocks) * 256 + threadIdx.x; at < ct_up(c.B, CT_PAD); at += row_blocks * 256) {
        c.row_id[at] = make_int2(CT_NEVER, at < c.B && c.query_ids ? c.query_ids[at] : CT_NEVER);
        c.row_g[at] = make_float2(0.0f, 0.0f);
    }
    if (c.squares && block == key_blocks && threadIdx.x < 8) c.most[(threadIdx.x >> 2) * CT_ROW_BLOCKS + (threadIdx.x & 3)] = 0.0f;
}

// ------------------------------------------------------------------------------------------------ the logits by tiles
// Larger of two, NaN if one is: one instruction (fmaxf() first makes sure that both are no signalling NaN, two more where they come from bits)
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }
// over the 16 lanes that share a row
template <int R> __device__ __forceinline__ void row16_larger(float (&v)[R])
{
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = larger(v[r], xor_lane_f32<1>(v[r]));
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = larger(v[r], xor_lane_f32<2>(v[r]));
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = larger(v[r], xor_lane_f32<7>(v[r]));
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = larger(v[r], xor_lane_f32<15>(v[r]));
}

// Puts a logit into the largest two of its group.
__device__ __forceinline__ void into_group(float &most, float &second, float s, int n, int group)
{
    const float x = __uint_as_float((__float_as_uint(s) & ~(u32)(group - 1)) | (u32)n);
    second = __builtin_amdgcn_fmed3f(most, second, x);      // most >= second
    most = larger(most, x);
}

// Sums of squares of what the product multiplies: |k|^2 without another pass over the keys.  (The dot product instruction of bfloat16 pairs rounds
// in between: |k|^2 = 1 of 768 coordinates was off by 2 %.)
template <int DT, int N> struct SquaresOf {
    float (&sum)[N];
    __device__ __forceinline__ void operator()(const us8 &b, int j) const
    {
#pragma unroll
        for (int h = 0; h < 8; ++h) sum[j] = fmaf(value16<DT>(b[h]), value16<DT>(b[h]), sum[j]);
    }
};

// Keys as they are: rows of those that are left out are multiplied too; what is not a number stays in its own column.
// Left-out keys have LP_NONE for a logit, and logits below it count as it; NaN stays NaN, and makes the sum NaN.
template <int TILE, int DT, bool TERMS, bool TOPS, bool SQUARES>
__global__ __launch_bounds__(256, TILE == 256 || TERMS ? 1 : 2) void k_logprob_sums(LogprobPar c, u32 first, int tiles_q, int tiles_k)
{
    constexpr int N = TILE / 32;
    __shared__ typename std::conditional<TERMS, TermsLds, ProductLds<TILE>>::type lds;
    __shared__ typename std::conditional<TERMS, NoLds, ProductLds<TILE>>::type lds2;
    __shared__ SideLds<TILE> side;
    f32x4 acc[N][N];
    int tr, tc;
    tile_of((int)(first + blockIdx.x), tiles_q, tiles_k, tr, tc);
    tc += c.key0 / TILE;
    float base[N], norm[N] = {};
    if constexpr (SQUARES) logit_product<TILE, DT, TERMS, false>(c, tr, tc, lds, lds2, side, acc, []() {}, SquaresOf<DT, N>{norm});
    else logit_product<TILE, DT, TERMS>(c, tr, tc, lds, lds2, side, acc, []() {});
    const Place<TILE> at(tr, tc);
    int id[N];
    bool odd[N], any_odd = false;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        base[n] = side.base[at.in_col + n];
        id[n] = side.id[at.in_col + n];
        const bool gone = id[n] < 0;
        if constexpr (SQUARES) {
            norm[n] += __shfl_xor(norm[n], 16);
            norm[n] += __shfl_xor(norm[n], 32);
            odd[n] = gone && !(norm[n] < INFINITY);
            if (!gone) base[n] = fmaf(-c.scale * norm[n], 1.44269504f, base[n]);
        } else {
            odd[n] = gone && base[n] != base[n];
            if (odd[n]) base[n] = LP_NONE;
        }
        any_odd |= odd[n];
        base[n] = base[n] < LP_NONE ? LP_NONE : base[n];        // (NaN stays)
    }
    any_odd = __any(any_odd);
    if constexpr (SQUARES && TOPS) {
        if (tr == 0 && threadIdx.x < 128) {         // the two wavefronts that have all columns
            float most = 0.0f, bias = 0.0f;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (id[n] < 0 || odd[n]) continue;
                most = fmaxf(most, norm[n] < INFINITY ? norm[n] : INFINITY);
                if (c.bias) bias = fmaxf(bias, bias_size(c, side.base[at.in_col + n] * 0.7f));
            }
#pragma unroll
            for (int x = 8; x; x >>= 1) {
                most = fmaxf(most, __shfl_xor(most, x));
                bias = fmaxf(bias, __shfl_xor(bias, x));
            }
            if ((threadIdx.x & 63) == 0) {
                atomicMax((u32 *)&c.most[0], __float_as_uint(most));
                atomicMax((u32 *)&c.most[CT_ROW_BLOCKS], __float_as_uint(bias));
            }
        }
    }
    // as in k_contrast_sums; and a lane's N columns of a row are a group
    float keep_top[N / 4], keep_sum[N / 4], keep_w[N / 4];
#pragma unroll
    for (int m = 0; m < N; ++m) {
        float s[4][N], top[4], sum[4], w[4];
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int n = 0; n < N; ++n) s[r][n] = larger(fmaf(acc[m][n][r], c.c1, base[n]), LP_NONE);
        leave_out(side, at.in_row + m * 4, id, s, LP_NONE);
        if constexpr (DT != DT_F32)
            if (any_odd)
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int n = 0; n < N; ++n) s[r][n] = odd[n] ? LP_NONE : s[r][n];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            top[r] = s[r][0];       // (a number in the lowest bits would be more than the range of the exponential where a step is: from 2^28 on)
#pragma unroll
            for (int n = 1; n < N; ++n) top[r] = larger(top[r], s[r][n]);
            if constexpr (TOPS) {
                float most = LP_NONE, second = LP_NONE;
#pragma unroll
                for (int n = 0; n < N; ++n) into_group(most, second, s[r][n], n, N);
                c.groups[((size_t)(at.row + m * 4 + r) * c.parts_k + at.half_c) * 16 + (threadIdx.x & 15)] = make_float2(most, second);
            }
        }
        row16_larger(top);
        const float largest = larger(larger(top[0], top[1]), larger(top[2], top[3]));
        if (__any(largest > 1.0e37f))       // LP_NONE less that may be -infinity; what is below zero is nothing beside it
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int n = 0; n < N; ++n) s[r][n] = top[r] > 1.0e37f ? larger(s[r][n], 0.0f) : s[r][n];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float ref = top[r] > LP_LIMIT ? top[r] : 0.0f;
            top[r] = top[r] > LP_LIMIT ? top[r] : -INFINITY;
            sum[r] = w[r] = 0.0f;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const float x = s[r][n] - ref, e = __builtin_amdgcn_exp2f(x);
                sum[r] += e;
                w[r] = fmaf(e, x, w[r]);
            }
        }
        row16_sum(sum);
        row16_sum(w);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const bool mine = (int)(threadIdx.x & 15) == m % 4 * 4 + r;
            keep_top[m / 4] = mine ? top[r] : m % 4 || r ? keep_top[m / 4] : 0.0f;
            keep_sum[m / 4] = mine ? sum[r] : m % 4 || r ? keep_sum[m / 4] : 0.0f;
            keep_w[m / 4] = mine ? w[r] : m % 4 || r ? keep_w[m / 4] : 0.0f;
        }
    }
#pragma unroll
    for (int h = 0; h < N / 4; ++h) {
        const size_t to = (size_t)(at.row + h * 16 + (threadIdx.x & 15)) * c.parts_k + at.half_c;
        c.part[to] = make_float2(keep_top[h], keep_sum[h]);
        c.part_w[to] = keep_w[h];
    }
}

// (largest, sum, weighted sum) of two parts; a NaN in either sum stays
__device__ __forceinline__ void join_three(float &top, float &sum, float &w, float ot, float os, float ow)
{
    const float m = fmaxf(top, ot), ref = m == -INFINITY ? 0.0f : m;
    const float da = fmaxf(top - ref, LP_FAR), db = fmaxf(ot - ref, LP_FAR), fa = __builtin_amdgcn_exp2f(da), fb = __builtin_amdgcn_exp2f(db);
    w = fa * fmaf(sum, da, w) + fb * fmaf(os, db, ow);
    sum = sum * fa + os * fb;
    top = m;
}

// V coordinates of a row from e on, of which those behind `end` are zeros.  WIDE: all rows allow it in one aligned access.  Others are loaded in one access
// all the same where they are whole (the hardware takes any address of a global load), and one by one at the end of the row.
template <int DT, int V, bool WIDE>
__device__ __forceinline__ Pack<DT, V> load_piece(const void *rows, size_t row, int e, int end)
{
    typedef typename RowType<DT>::T T;
    if constexpr (WIDE) return load_pack<DT, V>(rows, row + e);
    else {
        const T *from = (const T *)rows + row + e;
        Pack<DT, V> p;
        if (e + V <= end) __builtin_memcpy(&p, from, sizeof(p));
        else
#pragma unroll
            for (int k = 0; k < V; ++k) p.v[k] = e + k < end ? from[k] : (T)0.0f;
        return p;
    }
}

// ------------------------------------------------------------------------------------------------ the logits of a few queries
// Up to 8 queries: no matrix tile would be filled, and the call is bound by reading the keys once.  8 lanes take a row, 16 bytes each; distances
// are summed from differences.  Query coordinates come from LDS, as many of all queries as fit at a time.  A wavefront takes 16, 32 or 64 keys
// at a time by itself, and then a lane each of them for the sums; a block of four takes a part of the keys.
#define LP_CHUNK 8192           // coordinates in LDS, at most
template <int NB> constexpr int few_rows() { return NB <= 2 ? 4 : 2; }      // of a lane at a time

template <int DT, int NB, bool WIDE>
__global__ __launch_bounds__(256) void k_logprob_few(LogprobPar c, int wave_keys, int passes)
{
    constexpr int V = DT == DT_F32 ? 4 : 8, R = few_rows<NB>(), AHEAD = 8 / R;
    extern __shared__ __align__(16) float query[];         // [NB][chunk], then [4][NB][64] distances
    __shared__ float sums[4][NB][3];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane & 7;
    const int chunk = c.d <= LP_CHUNK / NB ? (c.d + 7) & ~7 : LP_CHUNK / NB;
    float *const far_of = query + NB * chunk + wave * NB * 64;
    auto stage = [&](int e0) {
        for (int b = 0; b < NB; ++b)
            for (int t = threadIdx.x; t < chunk; t += 256)
                query[b * chunk + t] = e0 + t < c.d ? (float)((const typename RowType<DT>::T *)c.Q)[(size_t)(b < c.B ? b : c.B - 1) * c.d + e0 + t] : 0.0f;
    };
    if (chunk >= c.d) stage(0);
    __syncthreads();
    float top[NB], sum[NB], w[NB], biases = 0.0f;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        top[b] = -INFINITY;
        sum[b] = w[b] = 0.0f;
    }
    const int part_keys = wave_keys * 4 * passes;
    for (int pass = 0; pass < passes; ++pass) {
        const int in_part = (pass * 4 + wave) * wave_keys, key0 = blockIdx.x * part_keys + in_part;
        // what the lane's key needs besides its distances, while these are formed
        const int mine = key0 + lane;
        const bool on = lane < wave_keys && mine < c.M && !key_gone(c, mine);
        const float bias = on && c.bias ? c.bias[mine] : 0.0f;
        const int name = on && c.query_ids ? c.key_ids[mine] : 0;
        for (int r0 = 0; r0 < wave_keys; r0 += 8 * R) {
            float acc[NB][R] = {};
            size_t row[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int j = key0 + r0 + r * 8 + (lane >> 3);
                row[r] = (size_t)(j < c.M ? j : c.M - 1) * c.d;
            }
            for (int e0 = 0; e0 < c.d; e0 += chunk) {
                if (chunk < c.d) {
                    __syncthreads();
                    stage(e0);
                    __syncthreads();
                }
                const int end = c.d - e0 < chunk ? c.d - e0 : chunk;
                for (int e1 = 0; e1 < end; e1 += AHEAD * 8 * V) {
                    Pack<DT, V> packs[AHEAD][R];
#pragma unroll
                    for (int a = 0; a < AHEAD; ++a) {
                        const int e = e1 + a * 8 * V + sub * V, from = e < end ? e : 0;
#pragma unroll
                        for (int r = 0; r < R; ++r) packs[a][r] = load_piece<DT, V, WIDE>(c.K, row[r] + e0, from, end);
                    }
#pragma unroll
                    for (int a = 0; a < AHEAD; ++a) {
                        const int e = e1 + a * 8 * V + sub * V;
                        __builtin_amdgcn_sched_barrier(0);      // (packs stay packed until their turn: half the registers)
                        if (e >= end) continue;
                        float x[R][V];
#pragma unroll
                        for (int r = 0; r < R; ++r) unpack<DT, V>(packs[a][r], x[r]);
#pragma unroll
                        for (int b = 0; b < NB; ++b)
#pragma unroll
                            for (int k = 0; k < V; k += 4) {
                                const f32x4 q = *(const f32x4 *)&query[b * chunk + e + k];
#pragma unroll
                                for (int r = 0; r < R; ++r)
#pragma unroll
                                    for (int h = 0; h < 4; ++h) {
                                        const float diff = x[r][k + h] - q[h];
                                        acc[b][r] = fmaf(diff, diff, acc[b][r]);
                                    }
                            }
                    }
                }
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    acc[b][r] += xor_lane_f32<1>(acc[b][r]);
                    acc[b][r] += xor_lane_f32<2>(acc[b][r]);
                    acc[b][r] += xor_lane_f32<7>(acc[b][r]);
                }
                // lane b of the 8 writes query b
                float far = acc[0][r];
#pragma unroll
                for (int b = 1; b < NB; ++b) far = sub == b ? acc[b][r] : far;
                if (sub < NB) far_of[sub * 64 + r0 + r * 8 + (lane >> 3)] = far;
            }
        }
        wave_sync();
        if (on) biases = fmaxf(biases, bias_size(c, bias));
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            if (b >= c.B) break;
            float s = !on || (c.query_ids && name == c.query_ids[b]) ? -INFINITY : (bias - c.scale * far_of[b * 64 + lane]) * 1.44269504f;
            s = s <= LP_LIMIT ? -INFINITY : s;      // (NaN stays)
            if (c.alternatives) {       // 8 lanes are a group
                float x = __uint_as_float((__float_as_uint(fmaxf(s, LP_NONE)) & ~7u) | (u32)sub), y = LP_NONE;
                auto with = [&](float ox, float oy) {
                    y = fmaxf(fminf(x, ox), fmaxf(y, oy));
                    x = fmaxf(x, ox);
                };
                with(xor_lane_f32<1>(x), xor_lane_f32<1>(y));
                with(xor_lane_f32<2>(x), xor_lane_f32<2>(y));
                with(xor_lane_f32<7>(x), xor_lane_f32<7>(y));
                if (sub == 0 && lane < wave_keys)
                    c.groups[((size_t)b * gridDim.x + blockIdx.x) * (part_keys / 8) + (in_part + lane) / 8] = make_float2(x, y);
            }
            const float m = fmaxf(top[b], s), ref = m == -INFINITY ? 0.0f : m;      // a lane's own
            const float da = fmaxf(top[b] - ref, LP_FAR), x = s - ref, fa = __builtin_amdgcn_exp2f(da), e = __builtin_amdgcn_exp2f(x);
            w[b] = fmaf(e, fmaxf(x, LP_FAR), fa * fmaf(sum[b], da, w[b]));
            sum[b] = fmaf(sum[b], fa, e);
            top[b] = m;
        }
        wave_sync();
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        if (b >= c.B) break;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) join_three(top[b], sum[b], w[b], __shfl_xor(top[b], s), __shfl_xor(sum[b], s), __shfl_xor(w[b], s));
        if (lane == 0) {
            sums[wave][b][0] = top[b];
            sums[wave][b][1] = sum[b];
            sums[wave][b][2] = w[b];
        }
    }
#pragma unroll
    for (int s = 32; s; s >>= 1) biases = fmaxf(biases, __shfl_xor(biases, s));
    if (lane == 0) far_of[0] = biases;
    __syncthreads();
    const int b = threadIdx.x;
    if (b < NB && b < c.B) {
        float t = sums[0][b][0], u = sums[0][b][1], v = sums[0][b][2];
        for (int h = 1; h < 4; ++h) {
            join_three(t, u, v, sums[h][b][0], sums[h][b][1], sums[h][b][2]);
            biases = fmaxf(biases, far_of[h * NB * 64]);        // (of the first wavefront; it reads the others')
        }
        c.part[(size_t)b * gridDim.x + blockIdx.x] = make_float2(t, u);
        c.part_w[(size_t)b * gridDim.x + blockIdx.x] = v;
        if (b == 0) c.most[blockIdx.x] = biases;
    }
}

// ------------------------------------------------------------------------------------------------ the answers
// |q_i - k_j|^2 in double precision, by 8 lanes
template <int DT, bool WIDE>
__device__ __forceinline__ double exact_distance(const LogprobPar &c, int i, int j, int sub)
{
    constexpr int V = DT == DT_F32 ? 4 : 8, AHEAD = WIDE ? 4 : 2;
    double sum = 0.0;
    const size_t q = (size_t)i * c.d, k = (size_t)j * c.d;
    for (int e1 = sub * V; e1 < c.d; e1 += AHEAD * 8 * V) {
        Pack<DT, V> px[AHEAD], py[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int e = e1 + a * 8 * V, from = e < c.d ? e : e1;
            py[a] = load_piece<DT, V, WIDE>(c.K, k, from, c.d);
            px[a] = load_piece<DT, V, WIDE>(c.Q, q, from, c.d);
        }
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            __builtin_amdgcn_sched_barrier(0);
            if (e1 + a * 8 * V >= c.d) continue;
            float x[V], y[V];
            unpack<DT, V>(px[a], x);
            unpack<DT, V>(py[a], y);
#pragma unroll
            for (int h = 0; h < V; ++h) {
                const double diff = (double)x[h] - (double)y[h];
                sum = fma(diff, diff, sum);
            }
        }
    }
    sum += __shfl_xor(sum, 1);
    sum += __shfl_xor(sum, 2);
    sum += __shfl_xor(sum, 4);
    return sum;
}

// What the product's logits leave out: |q - centre|^2, by a wavefront
template <int DT, bool WIDE>
__device__ __forceinline__ double query_norm(const LogprobPar &c, int i, int lane)
{
    double sum = 0.0;
    for (int e = lane * 4; e < c.d; e += 256) {
        float x[4];
        load4<DT, WIDE>(c.Q, i, c.d, e, x);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const double v = (double)x[k] - (DT == DT_F32 && e + k < c.d ? (double)c.centre[e + k] : 0.0);
            sum = fma(v, v, sum);
        }
    }
#pragma unroll
    for (int s = 32; s; s >>= 1) sum += __shfl_xor(sum, s);
    return sum;
}

__device__ __forceinline__ u32 in_order(float x)        // unsigned integers in the order of the numbers
{
    const u32 b = __float_as_uint(x);
    return b ^ (b >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float from_order(u32 o) { return __uint_as_float(o ^ (o >> 31 ? 0x80000000u : 0xFFFFFFFFu)); }

// A bound from below on the k-th largest of a wavefront's values (-infinity where there are fewer): the highest 24 bits of it.
__device__ __forceinline__ float kth_largest(const float (&v)[LP_ROOM / 64], int k)
{
    u32 o[LP_ROOM / 64], at = 0;
#pragma unroll
    for (int h = 0; h < LP_ROOM / 64; ++h) o[h] = in_order(v[h]);
    for (int bit = 31; bit >= 8; --bit) {
        const u32 t = at | 1u << bit;
        int count = 0;
#pragma unroll
        for (int h = 0; h < LP_ROOM / 64; ++h) count += (int)__popcll(__ballot(o[h] >= t));
        if (count >= k) at = t;
    }
    return at >= in_order(-INFINITY) ? from_order(at) : -INFINITY;
}

// A query's selection.  The keys' values overlay the groups' logits, which are no longer needed then; one place more for the target.
template <int PARTS> struct FinishLds {
    union {
        struct { float most[LP_ROOM], second[LP_ROOM]; };
        double value[LP_ROOM];
    };
    int group[LP_ROOM];
    union {
        int part[2 * PARTS];        // until the groups are known
        struct { int key[LP_ROOM + 1]; float bias[LP_ROOM + 1]; };
    };
    double target, lse, norm;
    int found;                      // keys; -1: no room
    bool bad;
};

// What the wavefronts of a query exchange: each one's sums, and the largest two parts of each lane; then the bound (NaN: there is nothing to look for), and how
// many parts and groups above it all have found.
template <int WAVES> struct TeamLds {
    float top[WAVES], sum[WAVES], w[WAVES], biases[WAVES], first[WAVES][64], second[WAVES][64];
    float cut;
    int parts, groups;
};
template <> struct TeamLds<1> {};

// A query by WAVES wavefronts (1: two queries a block).  A query by itself waits for dependent loads most of the time, so with few queries eight wavefronts
// take one: they join the parts and look for the groups above the bound together (the order in which they find them does not matter), the
// first selects among these, and all form the distances of the keys that are left.  (1 x 1,000,000 x 96 float32 13 us; 19 where one does all but the distances.)
template <int DT, bool WIDE, int WAVES>
__global__ __launch_bounds__(WAVES == 1 ? 128 : 64 * WAVES, WAVES == 1 ? 5 : 1) void k_logprob_finish(LogprobPar c)
{
    constexpr int QUERIES = WAVES == 1 ? 2 : 1, PARTS = WAVES == 1 ? 256 : 512, DEEP = WAVES == 1 ? 4 : 8;
    __shared__ FinishLds<PARTS> of_queries[QUERIES];
    __shared__ TeamLds<WAVES> team;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), sub = lane & 7;
    const int i = WAVES == 1 ? blockIdx.x * 2 + wave : blockIdx.x, worker = WAVES == 1 ? 0 : wave;
    if (i >= c.B) return;       // (blocks of one query: never)
    FinishLds<PARTS> &lds = of_queries[WAVES == 1 ? wave : 0];
    const int k = c.alternatives, size = 1 << c.group_shift;
    const float2 *part = c.part + (size_t)i * c.parts_k;
    const float2 *groups = c.groups + ((size_t)i * c.parts_k << c.part_shift);
    int *ids = c.top_ids + (size_t)i * k;
    float *tops = c.top_logprob + (size_t)i * k;
    float cut = -INFINITY;
    bool asked = false;         // for a target that can be
    int target = 0;
    float top = -INFINITY, sum = 0.0f, w = 0.0f, first = -INFINITY, second = -INFINITY, norms = 0.0f, biases = 0.0f;
    for (int t0 = worker * 64 + lane; t0 < c.parts_k; t0 += WAVES * 64 * 4) {
        float2 p[4];
        float pw[4], most[4];
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const int t = t0 + h * WAVES * 64;
            p[h] = t < c.parts_k ? part[t] : make_float2(-INFINITY, 0.0f);
            pw[h] = t < c.parts_k ? c.part_w[(size_t)i * c.parts_k + t] : 0.0f;
            most[h] = c.few && t < c.parts_k ? c.most[t] : 0.0f;
        }
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            join_three(top, sum, w, p[h].x, p[h].y, pw[h]);
            second = fmaxf(second, fminf(first, p[h].x));
            first = fmaxf(first, p[h].x);
            biases = fmaxf(biases, most[h]);
        }
    }
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        join_three(top, sum, w, __shfl_xor(top, s), __shfl_xor(sum, s), __shfl_xor(w, s));
        biases = fmaxf(biases, __shfl_xor(biases, s));
    }
    if constexpr (WAVES > 1) {
        team.first[worker][lane] = first;
        team.second[worker][lane] = second;
        if (lane == 0) {
            team.top[worker] = top;
            team.sum[worker] = sum;
            team.w[worker] = w;
            team.biases[worker] = biases;
        }
        if (threadIdx.x == 0) team.parts = team.groups = 0;
        __syncthreads();
        if (worker == 0)
#pragma unroll
            for (int v = 1; v < WAVES; ++v) {
                join_three(top, sum, w, team.top[v], team.sum[v], team.w[v]);
                biases = fmaxf(biases, team.biases[v]);
                const float a = team.first[v][lane], b = team.second[v][lane];
                second = fmaxf(fmaxf(second, b), fminf(first, a));
                first = fmaxf(first, a);
            }
    }
    int n = 0, found = 0;
    bool full = false, look = false, bad = false;
    double norm = 0.0;
    // A bound on the logits to look at, from a bound t on the k-th one as the first pass has it (with the key's number in it).  k keys have t or more
    // there, so with logits off by E the k-th is not below t - E, and what is not below that is not below t - 2 E in the first pass.  In base 2, u a step:
    //   a few queries: a sum of d squares, which are bias - logit: E = u (d + 16) (largest bias + |t|)
    //   tiles: a sum of d products of one rounding each (float32 rows: six times as many), its scaling, the key's own sum and bias:
    //   E = u (2 a scale |q||k| + b scale |k|^2 + 2 |bias|), a and b from d.  For the largest |k| and |bias|; or, with scale > 0, for what keys with logits
    //   down to t - E can have: scale (|k| - |q|)^2 <= R + E with R = largest bias + scale |q|^2 - t.  E takes (0.1 |q||k| + 0.01 |k|^2) scale at most
    //   beside the biases (d = 65,536), so 0.9 |k| <= |q| + sqrt(R / scale) + sqrt(0.1 |q||k|), the last not above 0.32 |q| + 0.08 |k|.
    float q = 0.0f;
    auto below = [&](float t) {
        if (t <= LP_NONE) return -INFINITY;
        const float u = 1.19209290e-7f;
        float error;
        if (c.few) error = u * (float)(c.d + 16) * (1.45f * biases + fabsf(t));
        else {
            float size = biases, k = sqrtf(norms);
            if (c.scale >= 0.0f) {
                const float own = c.scale * q * q;
                size = fmaxf(size, 0.7f * fabsf(t) + own);
                const float room = fmaxf(biases + own - 0.693147181f * t, 0.0f) + 1.0e-5f * size;       // (and the roundings of its own)
                k = c.scale > 0.0f ? fminf(k, 1.61f * q + 1.23f * sqrtf(room / c.scale)) : 0.0f;
            }
            error = 1.46f * u * (fabsf(c.scale) * (2.0f * ((DT == DT_F32 ? 6.0f : 1.0f) * c.d + 16.0f) * q * k + (float)(c.d + 16) * k * k) + 2.0f * size);
        }
        const float b = t - 2.0f * error - fabsf(t) * 4.0e-6f;
        return b > LP_NONE ? b : -INFINITY;
    };
    if (worker == 0) {
        if (c.logprob) target = c.target[i];
        if (!c.few && k)
#pragma unroll
            for (int h = 0; h < CT_ROW_BLOCKS / 256; ++h) {     // (a multiple of 64 blocks)
                const int b = h * 256 + lane * 4;
                if (b >= c.most_blocks) continue;
                const f32x4 x = *(const f32x4 *)&c.most[b], y = *(const f32x4 *)&c.most[CT_ROW_BLOCKS + b];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    norms = fmaxf(norms, x[e]);
                    biases = fmaxf(biases, y[e]);
                }
            }
        if (c.logprob) asked = (u32)target < (u32)c.M && !leaves_out(c, i, target);
        norm = c.few ? 0.0 : query_norm<DT, WIDE>(c, i, lane);
        q = sqrtf((float)norm);
        if (!c.few)
#pragma unroll
            for (int s = 1; s < 64; s <<= 1) {
                norms = fmaxf(norms, __shfl_xor(norms, s));
                biases = fmaxf(biases, __shfl_xor(biases, s));
            }
        const bool none = sum == 0.0f;
        bad = !(sum >= 0.0f && sum < INFINITY);
        if (c.entropy && lane == 0) {
            const float h = (log2f(sum) - w / sum) * 0.693147181f;
            c.entropy[i] = none ? 0.0f : bad ? NAN : h < 0.0f ? 0.0f : h;
        }
        look = k && !none && !bad;
        if (none || bad) {
            for (int e = lane; e < k; e += 64) {
                ids[e] = -1;
                tops[e] = bad ? NAN : -INFINITY;
            }
        } else if (k) {
            float v[LP_ROOM / 64];
#pragma unroll
            for (int h = 0; h < LP_ROOM / 64; ++h) v[h] = h == 0 ? first : h == 1 ? second : -INFINITY;
            cut = below(kth_largest(v, k));
        }
    }
    bool gathered = false;
    if constexpr (WAVES > 1) {
        if (threadIdx.x == 0) team.cut = look ? cut : NAN;
        __syncthreads();
        const float bound = team.cut;
        if (bound == bound) {
            // places for a wavefront's finds behind those of the others
            auto place = [&](int *count, u64 on) {
                int at = 0;
                if (lane == 0) at = atomicAdd(count, (int)__popcll(on));
                return __builtin_amdgcn_readfirstlane(at) + (int)__popcll(on & lanes_below(lane));
            };
            for (int p0 = worker * 64; p0 < c.parts_k; p0 += WAVES * 64 * 4) {
                float largest[4];
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    const int p = p0 + h * WAVES * 64 + lane;
                    largest[h] = p < c.parts_k ? part[p].x : -INFINITY;
                }
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    const u64 on = __ballot(largest[h] > -INFINITY && largest[h] >= bound);
                    if (!on) continue;
                    const int to = place(&team.parts, on);
                    if ((on >> lane & 1) && to < 2 * PARTS) lds.part[to] = p0 + h * WAVES * 64 + lane;
                }
            }
            __syncthreads();
            const int parts = team.parts, items = parts <= 2 * PARTS ? parts << c.part_shift : 0;
            for (int t0 = worker * 64; t0 < items; t0 += WAVES * 64 * 4) {
                float2 v[4];
                int g[4];
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    const int t = t0 + h * WAVES * 64 + lane;
                    g[h] = t < items ? (lds.part[t >> c.part_shift] << c.part_shift) + (t & ((1 << c.part_shift) - 1)) : -1;
                    v[h] = g[h] >= 0 ? groups[g[h]] : make_float2(-INFINITY, -INFINITY);
                }
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    const u64 on = __ballot(v[h].x > LP_LIMIT && v[h].x >= bound);
                    if (!on) continue;
                    const int to = place(&team.groups, on);
                    if ((on >> lane & 1) && to < LP_ROOM) {
                        lds.most[to] = v[h].x;
                        lds.second[to] = v[h].y;
                        lds.group[to] = g[h];
                    }
                }
            }
            __syncthreads();
            gathered = parts <= 2 * PARTS && team.groups <= LP_ROOM;     // else one by one, which makes room
            if (gathered) n = team.groups;
        }
    }
    if (worker == 0) {
        if (look) {
            // of the groups above the bound, those above a better one
            auto tighten = [&]() {
                if (n < k) return;
                wave_sync();
                float a[LP_ROOM / 64], b[LP_ROOM / 64];
                int g[LP_ROOM / 64];
#pragma unroll
                for (int h = 0; h < LP_ROOM / 64; ++h) {
                    const int e = h * 64 + lane;
                    a[h] = e < n ? lds.most[e] : -INFINITY;
                    b[h] = e < n ? lds.second[e] : -INFINITY;
                    g[h] = e < n ? lds.group[e] : 0;
                }
                cut = fmaxf(cut, below(kth_largest(a, k)));
                wave_sync();
                n = 0;
#pragma unroll
                for (int h = 0; h < LP_ROOM / 64; ++h) {
                    const u64 on = __ballot(a[h] > -INFINITY && a[h] >= cut);
                    if (on >> lane & 1) {
                        const int to = n + (int)__popcll(on & lanes_below(lane));
                        lds.most[to] = a[h];
                        lds.second[to] = b[h];
                        lds.group[to] = g[h];
                    }
                    n += (int)__popcll(on);
                }
                wave_sync();
            };
            int parts = 0;
            for (int p0 = 0; p0 < c.parts_k && !full && !gathered; p0 += PARTS) {
                float largest[PARTS / 64];
#pragma unroll
                for (int h = 0; h < PARTS / 64; ++h) largest[h] = p0 + h * 64 + lane < c.parts_k ? part[p0 + h * 64 + lane].x : -INFINITY;
#pragma unroll
                for (int h = 0; h < PARTS / 64; ++h) {
                    const u64 on = __ballot(largest[h] > -INFINITY && largest[h] >= cut);
                    if (on >> lane & 1) lds.part[parts + (int)__popcll(on & lanes_below(lane))] = p0 + h * 64 + lane;
                    parts += (int)__popcll(on);
                }
                if (parts <= PARTS && p0 + PARTS < c.parts_k) continue;        // there is room for the next ones
                wave_sync();
                const int items = parts << c.part_shift;
                for (int t0 = 0; t0 < items && !full; t0 += 64 * DEEP) {
                    float2 v[DEEP];
                    int g[DEEP];
#pragma unroll
                    for (int h = 0; h < DEEP; ++h) {
                        const int t = t0 + h * 64 + lane;
                        g[h] = t < items ? (lds.part[t >> c.part_shift] << c.part_shift) + (t & ((1 << c.part_shift) - 1)) : -1;
                        v[h] = g[h] >= 0 ? groups[g[h]] : make_float2(-INFINITY, -INFINITY);
                    }
#pragma unroll
                    for (int h = 0; h < DEEP; ++h) {
                        u64 on = __ballot(v[h].x > LP_LIMIT && v[h].x >= cut);
                        if (!on) continue;
                        if (n + (int)__popcll(on) > LP_ROOM && !full) {
                            tighten();
                            on = __ballot(v[h].x > LP_LIMIT && v[h].x >= cut);
                            full = n + (int)__popcll(on) > LP_ROOM;
                        }
                        if (full) continue;
                        if (on >> lane & 1) {
                            const int to = n + (int)__popcll(on & lanes_below(lane));
                            lds.most[to] = v[h].x;
                            lds.second[to] = v[h].y;
                            lds.group[to] = g[h];
                        }
                        n += (int)__popcll(on);
                    }
                }
                wave_sync();
                parts = 0;
            }
            if (!full) tighten();
            wave_sync();
            // the keys: the largest of a group, or all where the second is above the bound too
            for (int e = 0; e < n && !full; e += 64) {
                const bool in = e + lane < n && lds.most[e + lane] >= cut;
                const int g = in ? lds.group[e + lane] : 0;
                const int mine = !in ? 0 : lds.second[e + lane] >= cut && lds.second[e + lane] > LP_LIMIT ? size : 1;
                int upto = inclusive(mine, lane);
                const int all = __builtin_amdgcn_readlane(upto, 63);
                if (found + all > LP_ROOM) {
                    full = true;
                    break;
                }
                upto += found - mine;
                if (mine == 1) lds.key[upto] = (g << c.group_shift) + (int)(__float_as_uint(lds.most[e + lane]) & (u32)(size - 1));
                else
                    for (int h = 0; h < mine; ++h) lds.key[upto + h] = (g << c.group_shift) + h;
                found += all;
            }
            wave_sync();
            for (int e = lane; e < found && !full; e += 64) {
                const int j = lds.key[e];
                const bool on = j < c.M && !leaves_out(c, i, j);
                if (!on) lds.key[e] = -1;
                lds.bias[e] = on && c.bias ? c.bias[j] : 0.0f;
            }
        }
        if (lane == 0) {
            lds.key[LP_ROOM] = asked ? target : -1;
            lds.bias[LP_ROOM] = asked && c.bias ? c.bias[target] : 0.0f;
            lds.lse = (double)top + log2((double)sum);
            lds.norm = norm;
            lds.found = full ? -1 : found;
            lds.bad = bad;
        }
    }
    if constexpr (WAVES > 1) __syncthreads();
    else wave_sync();
    norm = lds.norm;
    bad = lds.bad;
    found = lds.found;
    full = found < 0;
    const double lse = lds.lse;
    auto logit = [&](float bias, int j) {       // in base 2 and the frame of the sums; by 8 lanes
        return ((double)bias - (double)c.scale * (exact_distance<DT, WIDE>(c, i, j, sub) - norm)) * LP_LOG2E;
    };
    auto log_of = [&](double s) {   // (a probability is not above 1)
        const double l = (s - lse) * 0.69314718055994531;
        return bad ? NAN : s <= LP_LIMIT && lse > -INFINITY ? -INFINITY : (float)(l < 0.0 ? l : 0.0);
    };
    // the target behind the keys
    for (int e = worker * 8; e < (full ? 0 : found) + 1; e += WAVES * 8) {
        const int n = full ? 0 : found, at = e + (lane >> 3) < n ? e + (lane >> 3) : LP_ROOM, j = lds.key[at];
        const double s = logit(lds.bias[at], j < 0 ? 0 : j);
        if (sub == 0 && e + (lane >> 3) <= n) {
            if (at < LP_ROOM) lds.value[at] = s;
            else lds.target = s;
        }
    }
    if constexpr (WAVES > 1) __syncthreads();
    else wave_sync();
    if (worker) return;
    if (c.logprob && lane == 0) c.logprob[i] = lds.key[LP_ROOM] >= 0 ? log_of(lds.target) : 0.0f;
    if (!k || bad || lse == -INFINITY) return;
    if (!full) {
        int valid = 0;
        for (int e = 0; e < found; e += 64) {
            const int j = e + lane < found ? lds.key[e + lane] : -1;
            const double s = j >= 0 ? lds.value[e + lane] : 0.0;
            const bool on = j >= 0 && s > LP_LIMIT;
            int rank = 0;
#pragma unroll 4
            for (int o = 0; o < found; ++o) {
                const double os = lds.value[o];
                const int oj = lds.key[o];
                rank += oj >= 0 && (os > s || (os == s && oj < j));
            }
            if (on && rank < k) {
                ids[rank] = j;
                tops[rank] = log_of(s);
            }
            valid += (int)__popcll(__ballot(on));
        }
        for (int e = valid + lane; e < k; e += 64) {
            ids[e] = -1;
            tops[e] = -INFINITY;
        }
        return;
    }
    // No room: every key of a group above the bound, in the order of their positions, into a list of the k best so far.  The bound stays valid:
    // keys that are not looked at are below k others.
    found = 0;
    for (int g0 = 0; g0 < c.parts_k << c.part_shift; g0 += 64) {
        const int g = g0 + lane;
        const float largest = g < c.parts_k << c.part_shift ? groups[g].x : -INFINITY;
        for (u64 on = __ballot(largest > LP_LIMIT && largest >= cut); on; on &= on - 1) {
            const int key0 = (g0 + __builtin_ctzll(on)) << c.group_shift, j = key0 + (lane >> 3);
            bool in = lane >> 3 < size && j < c.M && !leaves_out(c, i, j);
            const double s = logit(in && c.bias ? c.bias[j] : 0.0f, in ? j : 0);
            in &= s > LP_LIMIT;
            for (int h = 0; h < size; ++h) {
                if (!__builtin_amdgcn_readlane((int)in, h * 8)) continue;
                const double x = __shfl(s, h * 8);
                // its place: behind those that are at least as large
                const double a = lane < found ? lds.value[lane] : 0.0, b = 64 + lane < found ? lds.value[64 + lane] : 0.0;
                const int ka = lane < found ? lds.key[lane] : 0, kb = 64 + lane < found ? lds.key[64 + lane] : 0;
                const int at = (int)__popcll(__ballot(lane < found && a >= x)) + (int)__popcll(__ballot(64 + lane < found && b >= x));
                if (at >= k) continue;
                wave_sync();
                if (lane >= at && lane < found && lane + 1 < k) {
                    lds.value[lane + 1] = a;
                    lds.key[lane + 1] = ka;
                }
                if (64 + lane >= at && 64 + lane < found && 65 + lane < k) {
                    lds.value[65 + lane] = b;
                    lds.key[65 + lane] = kb;
                }
                if (lane == 0) {
                    lds.value[at] = x;
                    lds.key[at] = key0 + h;
                }
                found = found < k ? found + 1 : k;
                wave_sync();
            }
        }
    }
    for (int e = lane; e < k; e += 64) {
        ids[e] = e < found ? lds.key[e] : -1;
        tops[e] = e < found ? log_of(lds.value[e]) : -INFINITY;
    }
}

// ------------------------------------------------------------------------------------------------ host side
struct LogprobPlan {
    ContrastPlan tiles;
    int slab;           // queries of a run through the keys
    half_t *spare;      // room for copies of key_rows keys, where the keys could be read as they are but for where they lie
    int key_rows;
    bool copied;
    int wave_keys, passes;      // a few queries: keys of a wavefront at a time, and how many times
};

#define LP_BYTES ((size_t)1 << 30)      // of a run's parts and groups

// Up to 8 queries at a time by differences, or all by tiles.  Float32 keys have to be copied in three terms for the tiles, which costs as much as many
// runs of 8 through a large table.  8 queries / 64 by tiles, us: 10,000 x 96 24 / 40, 100,000 x 100 34 / 98, 1,000,000 x 32 80 / 543, 1,000,000 x 96 121 / 759,
// 300,000 x 768 201 / 1,319; below, both in us, by coordinates and by keys.  (16-bit keys: 300,000 x 768, 8 queries 144 us, 9 to 128 by tiles 186, 256 225.)
static bool few_queries(int B, int M, int d, int dtype)
{
    const double size = 1e-6 * M * d, keys = 1e-3 * M;
    return B <= LP_FEW || (dtype == RNND_F32 && (B + LP_FEW - 1) / LP_FEW * (22.0 + 0.75 * size + 0.03 * keys) < 35.0 + 4.5 * size + 0.33 * keys);
}

// Keys of 16 bits whose rows are whole steps of the product are read where they are.  Where they do not lie at a multiple of 16 bytes they are copied after
// all, as many at a time as there is room for: neither the workspace nor the order of sums goes by addresses.
#define LP_SPARE 16384
static size_t layout(LogprobPar &c, LogprobPlan &plan, int dtype, char *base)
{
    size_t off = 0;
    auto take = [&](auto *&p, size_t count) {
        p = (typename std::remove_reference<decltype(p)>::type)(base + off);
        off += ws_align(count * sizeof(*p));
    };
    const int queries = c.B;
    c.few = few_queries(c.B, c.M, c.d, dtype);
    if (c.few) {
        if (c.B > LP_FEW) c.B = LP_FEW;
        // parts: they are gone through twice in the end, so not more than some 2,000 (1,024 / 2,048 / 4,096: 1 x 1,000,000 x 96 float32 84 / 80 / 78 us,
        // 8 queries 127 / 119 / 128)
        plan.wave_keys = c.B <= 2 ? 32 : 16;
        plan.passes = 1;
        auto parts = [&]() { return (c.M + plan.wave_keys * 4 * plan.passes - 1) / (plan.wave_keys * 4 * plan.passes); };
        while (plan.wave_keys < 64 && parts() > 512) plan.wave_keys *= 2;
        while (parts() > 2048) plan.passes *= 2;
        plan.slab = c.B;
        c.parts_k = c.most_blocks = parts();
        c.group_shift = 3;
        c.part_shift = __builtin_ctz(plan.wave_keys * plan.passes / 2);
        take(c.most, c.parts_k);
        take(c.part, (size_t)c.B * c.parts_k);
        take(c.part_w, (size_t)c.B * c.parts_k);
        if (c.alternatives) take(c.groups, (size_t)c.B * c.parts_k << c.part_shift);
        c.B = queries;
        return off;
    }
    // Tiles: as contrast_plan(), but that there is one product.  16-bit rows, tiles of 128 / 256, us: up to 128 queries, where half of one of 256 would be padding,
    // 100 x 300,000, d = 128 90 / 110, 256 97 / 124, 768 188 / 222; more of them read the keys once instead of twice, 200 x 300,000, d = 64 92 / 100, 128 102 / 111,
    // 192 131 / 120, 256 148 / 131, 768 256 / 226, 400 x 300,000 x 256 250 / 241; 8,192 x 16,384, d = 128 160 / 171, 256 199 / 198, 384 232 / 231, 768 338 / 321.
    // Float32 rows, two workgroups / terms together: 3,000 x 12,000, d = 100 102 / 128, 768 368 / 399, 1,536 693 / 717; 700 x 4,000 x 300 59 / 56.
    const bool large = (c.B + 255LL) / 256 * ((c.M + 255LL) / 256) >= 512 && c.B > 128 && c.d > (c.B <= 1024 ? 160 : 320);
    c.tile = dtype != RNND_F32 && large ? 256 : 128;
    c.terms_from = 1536;
    plan.tiles = contrast_plan(c, dtype == RNND_F32 ? 3 : 1);
    c.keys_as_they_are = dtype != RNND_F32 && c.d % CT_K == 0;
    // Their norms come from the product's pass over them where few tiles do that for every key.  Norms by themselves / along with the product, us:
    // bfloat16, 200 x 300,000 x 768 (one row of tiles) 373 / 226, 2,048 x 10,000 x 768 (8) 81 / 79, 8,192 x 16,384 x 768 (32) 303 / 328; float16,
    // 1,000 x 11,000 x 768 63 / 56
    c.squares = c.keys_as_they_are && c.B <= 1024;
    c.part_shift = 4;
    const size_t row = (size_t)c.parts_k * (12 + (c.alternatives ? 16 * 8 : 0));
    const size_t rows = LP_BYTES / row / CT_PAD * CT_PAD;
    plan.slab = rows < CT_PAD ? CT_PAD : rows < (size_t)queries ? (int)rows : queries;
    c.B = plan.slab < queries ? plan.slab : queries;
    off = contrast_layout(c, plan.tiles, dtype, 0, base, [](auto &) {});     // (tiles for the queries of a run)
    c.group_shift = plan.tiles.tile == 256 ? 3 : 2;
    const size_t Br = ct_up(c.B, CT_PAD);
    take(c.most, 2 * CT_ROW_BLOCKS);
    take(c.part_w, Br * c.parts_k);
    plan.key_rows = ct_up(c.M, CT_PAD) < LP_SPARE ? ct_up(c.M, CT_PAD) : LP_SPARE;
    if (c.keys_as_they_are) take(plan.spare, (size_t)plan.key_rows * c.dp);
    if (c.alternatives) take(c.groups, (Br * c.parts_k) << c.part_shift);
    c.B = queries;
    return off;
}

static int check_logprob(int64_t B, int64_t M, int32_t d, int dtype, int32_t alternatives)
{
    const int rc = check_contrast(B, M, d, dtype);
    if (rc) return rc;
    return alternatives < 0 || alternatives > RNND_MAX_LISTED ? RNND_ERR_BAD_PARAM : RNND_OK;
}

extern "C" int rnnd_logprob_workspace(int64_t B, int64_t M, int32_t d, int dtype, int32_t alternatives, size_t *bytes)
{
    const int rc = check_logprob(B, M, d, dtype, alternatives);
    if (rc) return rc;
    if (!bytes) return RNND_ERR_NULL;
    if (!B) {
        *bytes = 0;
        return RNND_OK;
    }
    LogprobPar c = {};
    LogprobPlan plan = {};
    c.B = (int)B;
    c.M = (int)M;
    c.d = d;
    c.alternatives = alternatives;
    *bytes = layout(c, plan, dtype, nullptr);
    return RNND_OK;
}

template <int DT, int TILE, bool TERMS>
static void launch_sums(const LogprobPar &c, int keys, hipStream_t st)
{
    const int tq = ct_up(c.B, TILE) / TILE, tk = ct_up(keys, TILE) / TILE;
    in_launches((u64)tq * tk, 256, [&](u64 first, u64 blocks) {
        const dim3 grid((u32)blocks), block(256);
        if constexpr (DT != DT_F32)
            if (c.squares) {
                if (c.alternatives) hipLaunchKernelGGL((k_logprob_sums<TILE, DT, TERMS, true, true>), grid, block, 0, st, c, (u32)first, tq, tk);
                else hipLaunchKernelGGL((k_logprob_sums<TILE, DT, TERMS, false, true>), grid, block, 0, st, c, (u32)first, tq, tk);
                return;
            }
        if (c.alternatives) hipLaunchKernelGGL((k_logprob_sums<TILE, DT, TERMS, true, false>), grid, block, 0, st, c, (u32)first, tq, tk);
        else hipLaunchKernelGGL((k_logprob_sums<TILE, DT, TERMS, false, false>), grid, block, 0, st, c, (u32)first, tq, tk);
    });
}

template <int DT, bool WIDE>
static void launch_logprob(LogprobPar &c, const LogprobPlan &plan, bool wide_few, hipStream_t st)
{
    if (c.few) {
        const dim3 grid(c.parts_k), block(256);
#define LP_LAUNCH(NB) \
        const int chunk = c.d <= LP_CHUNK / NB ? (c.d + 7) & ~7 : LP_CHUNK / NB; \
        const size_t bytes = (size_t)(NB * chunk + 4 * NB * 64) * 4; \
        if (wide_few) hipLaunchKernelGGL((k_logprob_few<DT, NB, true>), grid, block, bytes, st, c, plan.wave_keys, plan.passes); \
        else hipLaunchKernelGGL((k_logprob_few<DT, NB, false>), grid, block, bytes, st, c, plan.wave_keys, plan.passes)
        if (c.B == 1) { LP_LAUNCH(1); }
        else if (c.B == 2) { LP_LAUNCH(2); }
        else if (c.B <= 4) { LP_LAUNCH(4); }
        else { LP_LAUNCH(8); }
#undef LP_LAUNCH
    } else {
        const int Br = ct_up(c.B, CT_PAD), Mr = ct_up(c.M, CT_PAD), across = c.dp / 64;
        const bool keys = c.most_blocks == 0;       // not yet prepared
        const int key_blocks = !keys || c.squares ? 0 : Mr / 4 < CT_ROW_BLOCKS ? Mr / 4 : CT_ROW_BLOCKS, row_blocks = Br / CT_PAD < CT_ROW_BLOCKS ? Br / CT_PAD : CT_ROW_BLOCKS;
        if (keys) c.most_blocks = c.squares ? 4 : key_blocks;      // (with squares: one, which all tiles go into)
        if constexpr (DT == DT_F32)
            if (keys)
                hipLaunchKernelGGL(k_contrast_centre<LogprobPar>, dim3((c.dp + 64 * CT_SAMPLES - 1) / (64 * CT_SAMPLES)), dim3(64 * CT_SAMPLES), 0, st, c);
        // keys' sides, queries' ids and copies of rows, by blocks
        auto prepare = [&](const LogprobPar &p, int sides, int ids, int query_rows, int key_rows) {
            in_launches((u64)(sides + ids) + (u64)((query_rows + key_rows) / 64) * across, 256, [&](u64 first, u64 blocks) {
                hipLaunchKernelGGL((k_logprob_prepare<DT, WIDE>), dim3((u32)blocks), dim3(256), 0, st, p, (u32)first, sides, ids, query_rows / 64, across);
            });
        };
        auto sums = [&](const LogprobPar &p, int keys_of_it) {
            if constexpr (DT != DT_F32) {
                if (plan.tiles.tile == 256) launch_sums<DT, 256, false>(p, keys_of_it, st);
                else launch_sums<DT, 128, false>(p, keys_of_it, st);
            } else if (plan.tiles.terms) launch_sums<DT, 128, true>(p, keys_of_it, st);
            else launch_sums<DT, 128, false>(p, keys_of_it, st);
        };
        prepare(c, key_blocks, row_blocks, Br, keys && !c.keys_as_they_are ? Mr : 0);
        if (!plan.copied) sums(c, c.M);
        else
            for (int key0 = 0; key0 < c.M; key0 += plan.key_rows) {
                LogprobPar p = c;
                p.key0 = key0;
                p.k = plan.spare - (size_t)key0 * c.dp;     // rows go by the keys' numbers
                const int rows = Mr - key0 < plan.key_rows ? Mr - key0 : plan.key_rows;
                prepare(p, 0, 0, 0, rows);
                sums(p, c.M - key0 < rows ? c.M - key0 : rows);     // (tiles behind the last key have no place)
            }
    }
#define LP_LAUNCH(WAVES, BLOCKS, THREADS) \
    if (wide_few) hipLaunchKernelGGL((k_logprob_finish<DT, true, WAVES>), dim3(BLOCKS), dim3(THREADS), 0, st, c); \
    else hipLaunchKernelGGL((k_logprob_finish<DT, false, WAVES>), dim3(BLOCKS), dim3(THREADS), 0, st, c)
    if (c.B <= LP_ALONE) { LP_LAUNCH(8, c.B, 512); }
    else { LP_LAUNCH(1, (c.B + 1) / 2, 128); }
#undef LP_LAUNCH
}

extern "C" int rnnd_logprob(const void *Q, int64_t B, const void *K, int64_t M, int32_t d, int dtype, int metric, const int32_t *target,
                            const int32_t *query_ids, const int32_t *key_ids, const float *key_bias, float scale, int32_t alternatives,
                            float *logprob, float *entropy, int32_t *top_ids, float *top_logprob, void *workspace, size_t workspace_bytes,
                            void *stream)
{
    const int rc = check_logprob(B, M, d, dtype, alternatives);
    if (rc) return rc;
    if (metric != RNND_L2SQ) return RNND_ERR_UNSUPPORTED;
    if (!K || (B && !Q) || (query_ids && !key_ids)) return RNND_ERR_NULL;
    if (B && ((target == nullptr) != (logprob == nullptr) || (alternatives && (!top_ids || !top_logprob)))) return RNND_ERR_NULL;
    const size_t size = dt_size(dtype);
    if (((uintptr_t)Q | (uintptr_t)K) % size) return RNND_ERR_BAD_PARAM;
    if (((uintptr_t)target | (uintptr_t)query_ids | (uintptr_t)key_ids | (uintptr_t)key_bias | (uintptr_t)logprob | (uintptr_t)entropy |
         (uintptr_t)top_ids | (uintptr_t)top_logprob) % 4)
        return RNND_ERR_BAD_PARAM;
    if (!std::isfinite(scale)) return RNND_ERR_BAD_PARAM;
    if (!B) return RNND_OK;
    LogprobPar c = {};
    LogprobPlan plan = {};
    c.Q = Q;
    c.K = K;
    c.target = target;
    c.query_ids = query_ids;
    c.key_ids = key_ids;
    c.bias = key_bias;
    c.left_out = CT_LOWEST;
    c.scale = scale;
    c.c1 = (float)(2.0 * scale * LP_LOG2E);
    c.B = (int)B;
    c.M = (int)M;
    c.d = d;
    c.alternatives = alternatives;
    c.logprob = logprob;
    c.entropy = entropy;
    c.top_ids = top_ids;
    c.top_logprob = top_logprob;
    if (!workspace) return RNND_ERR_NULL;
    if ((uintptr_t)workspace % 16) return RNND_ERR_BAD_PARAM;
    if (workspace_bytes < layout(c, plan, dtype, (char *)workspace)) return RNND_ERR_SCRATCH;
    plan.copied = c.keys_as_they_are && (uintptr_t)K % 16;
    hipStream_t st = (hipStream_t)stream;
    const int vec = row_vec(d, Q, (int)size, K, (int)size);
    const bool wide_few = vec >= (dtype == RNND_F32 ? 4 : 8);
    const int queries = c.B;
    for (int q0 = 0; q0 < queries; q0 += plan.slab) {
        c.B = queries - q0 < plan.slab ? queries - q0 : plan.slab;
        c.Q = (const char *)Q + (size_t)q0 * d * size;
        c.target = target ? target + q0 : nullptr;
        c.query_ids = query_ids ? query_ids + q0 : nullptr;
        c.logprob = logprob ? logprob + q0 : nullptr;
        c.entropy = entropy ? entropy + q0 : nullptr;
        c.top_ids = top_ids ? top_ids + (size_t)q0 * alternatives : nullptr;
        c.top_logprob = top_logprob ? top_logprob + (size_t)q0 * alternatives : nullptr;
#define RNND_LOGPROB(DT) \
        if (vec >= 4) launch_logprob<DT, true>(c, plan, wide_few, st); \
        else launch_logprob<DT, false>(c, plan, wide_few, st)
        if (dtype == RNND_F32) { RNND_LOGPROB(DT_F32); }
        else if (dtype == RNND_F16) { RNND_LOGPROB(DT_F16); }
        else { RNND_LOGPROB(DT_BF16); }
#undef RNND_LOGPROB
    }
    return launched("rnnd_logprob");
}
