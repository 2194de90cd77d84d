// Softmax loss over squared distances, and its gradients: the loss that trains the rows of an index.
//
//   s_ij   = bias_j - scale |q_i - k_j|^2                       logit of key j for query i
//   loss_i = log( sum_j exp s_ij ) - s_it                       t = target[i]; the sum over the keys not left out
//   g_ij   = w_i p_ij (j != t), g_it = -w_i (1 - p_it),  p_ij = exp(s_ij - lse_i)
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
//   - a logit formed so is off by some 2^-24 scale |q||k| and 2^-24 scale |k|^2, in which distances between rows far from the origin
//     drown (768 coordinates around 10, scale 5: losses off by 0.06; around 100: by 33).  Distances do not change when all rows are moved, so
//     float32 rows are first taken from a point among the keys (k_contrast_centre), and the error goes with the rows' distances from it.
//     16-bit rows stay as they are: their coordinates would no longer fit 16 bits.
//   - all sums are float32.  The target is kept out of the row's sum: with x = lse over the others - s_t, loss = log(1 + e^x)
//     and 1 - p_t = 1 - e^-loss, neither of which cancels when the loss is small.
//   - g of the other keys is rounded to the type of the rows (float32 rows: three terms again; float16: scaled to below 2^15 by
//     a power of two for all weights, so that it is normal down to 2^-29 of the largest).  The term of the target, as a rule the
//     largest, is added in float32 at the end.  Rounding leaves the sums of g a little off what they should be, which rows far from
//     the origin would turn into a large error: the gradients are formed from k_j - q_i, with the sums of the rounded g, as
//     the formulas have it.
//
// What bounds it.  The work that the loss cannot do without is three products; forming the logits again is a fourth, which costs less
// than writing them in 32 bits and reading them back.  8,192 x 16,384 x 768 bfloat16, 0.98-1.00 ms (three library products of that shape: 0.64):
// preparation 35 us; largest and sums 250 (825 TFLOP/s); g 330 (625, and 537 MB written: one wavefront per SIMD, so that what
// follows a tile's product is not hidden behind another's); g k and g' q 434 (950; the library's products 971 to 1,003); joining the parts 48.  Float32 rows of
// 100 coordinates, 2,000 x 10,000, 228 us: six products for each, and g in three terms twice, 250 MB written by the second product (65 us)
// and read by the third (93).  Small calls are seven launches that wait for each other (16-bit rows six): 100 x 1,100 x 32 50 to 54 us.
#include <cmath>

#include "contrast.h"

// A wavefront per row: keys first, then queries.  A key's own part of its logits, a query's logit of its target.
template <int DT, bool WIDE>
__device__ __forceinline__ void contrast_rows(const ContrastPar &c, int block, int key_blocks, int row_blocks)
{
    __shared__ u32 most;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const bool keys = block < key_blocks;
    if (DT == DT_F16 && !keys) {        // (a whole block)
        if (threadIdx.x == 0) most = 0;
        __syncthreads();
    }
    const int blocks = keys ? key_blocks : row_blocks;
    const int padded = ((keys ? c.M : c.B) + CT_PAD - 1) / CT_PAD * CT_PAD;
    for (int at = (block - (keys ? 0 : key_blocks)) * 4 + wave; at < padded; at += blocks * 4) {
        if (keys) {
            const int one[1] = {at};
            float norm[1];
            key_sides<DT, WIDE, 1, false, false>(c, one, padded, lane, norm);
            if (lane == 0 && at < c.M) {
                c.first[at] = 0x7FFFFFFF;
                c.count[at] = 0;
            }
        } else {
            const bool on = at < c.B && row_counts(c, at);
            float dot = 0.0f, norm = 0.0f;
            int t = -1;
            if (on) {
                t = c.target[at];
                for (int e = lane * 4; e < c.d; e += 256) {
                    float x[4], y[4];
                    load4<DT, WIDE>(c.Q, at, c.d, e, x);
                    load4<DT, WIDE>(c.K, t, c.d, e, y);
                    if constexpr (DT == DT_F32) {
                        from_centre(c, e, x);
                        from_centre(c, e, y);
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        dot = fmaf(x[k], y[k], dot);
                        norm = fmaf(y[k], y[k], norm);
                    }
                }
            }
            dot = wave_sum(dot);
            norm = wave_sum(norm);
            if (lane == 0) {
                c.row_id[at] = make_int2(on ? c.key_ids ? c.key_ids[t] : t : CT_NEVER, on && c.query_ids ? c.query_ids[at] : CT_NEVER);
                const float w = on ? c.row_weight ? c.row_weight[at] : 1.0f : 0.0f;
                c.row_g[at] = make_float2(INFINITY, w);
                if (at < c.B) {
                    c.row_own[at] = w;
                    c.own_logit[at] = fmaf(dot, c.c1, ((on && c.bias ? c.bias[t] : 0.0f) - c.scale * norm) * 1.44269504f);
                }
                const u32 bits = __float_as_uint(w) & 0x7FFFFFFFu;
                if (DT == DT_F16 && bits < 0x7F800000u) atomicMax(&most, bits);
            }
        }
    }
    if (DT == DT_F16 && !keys) {
        __syncthreads();
        if (threadIdx.x == 0) c.tops[block - key_blocks] = most;
    }
}

// Both in one launch (neither reads what the other writes): small calls are bound by the number of dependent launches.  first: here and
// below, how many blocks earlier launches took (in_launches()).
template <int DT, bool WIDE>
__global__ __launch_bounds__(256) void k_contrast_prepare(ContrastPar c, u32 first, int key_blocks, int row_blocks, int q_tiles, int across, int columns)
{
    const int block = (int)(first + blockIdx.x), id = block - key_blocks - row_blocks;
    if (id < 0) contrast_rows<DT, WIDE>(c, block, key_blocks, row_blocks);
    else contrast_copy<DT, WIDE>(c, id / across, id % across * 64, q_tiles, columns);
}

// A wavefront per query joins its parts: the loss, and what the second product needs.
template <int DT>
__global__ __launch_bounds__(256) void k_contrast_loss(ContrastPar c, int row_blocks)
{
    const int i = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    int up = 0;
    if constexpr (DT == DT_F16) {
        __shared__ u32 most;
        if (threadIdx.x == 0) most = 0;
        __syncthreads();
        u32 top = 0;
        for (int b = threadIdx.x; b < row_blocks; b += 256) top = c.tops[b] > top ? c.tops[b] : top;
        atomicMax(&most, top);
        __syncthreads();
        up = weight_exponent(most);
        if (blockIdx.x == 0 && threadIdx.x == 0) *c.top = most;
    }
    if (i >= c.B) return;
    float top = -INFINITY, sum = 0.0f;
    for (int t = lane; t < c.parts_k; t += 64) {
        const float2 p = c.part[(size_t)i * c.parts_k + t];
        join_parts(top, sum, p.x, p.y);
    }
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) join_parts(top, sum, __shfl_xor(top, s), __shfl_xor(sum, s));
    if (lane) return;
    if (!row_counts(c, i)) {
        c.loss[i] = 0.0f;
        c.row_own[i] = 0.0f;
        return;
    }
    // x = lse of the others - own logit; loss = log(1 + e^x)
    const float own = c.own_logit[i];
    float loss = 0.0f;
    if (!(top == -INFINITY && sum == 0.0f)) {
        const float x = (top - own + log2f(sum)) * 0.693147181f;
        loss = x > 0.0f ? x + log1pf(expf(-x)) : log1pf(expf(x));
    }
    c.loss[i] = loss;
    const float w = c.row_own[i];
    c.row_own[i] = w * expm1f(-loss);
    c.row_g[i] = make_float2(own + loss * 1.44269504f, ldexpf(w, up));
    const int t = c.target[i];
    atomicMin(&c.first[t], i);
    atomicAdd(&c.count[t], 1);
}

// A key that is the target of more than CT_SHARED queries takes their terms by a whole block: it looks for them in CT_LOOK targets at a time, each
// wavefront sums a part of those found, in order, and the parts are added in the end.  8,192 x 16,384 x 768 bfloat16 with one target for all
// queries, a tenth of them, each its own, us: 2,085, 1,175, 1,059 (a wavefront that looked for each and waited for it: 15,931, 2,557, 1,063);
// 8,192 x 16 x 768 280 (1,366), 100,000 x 64 x 768 1,850 (5,633).
#define CT_SHARED 8
#define CT_LOOK 4096
#define CT_FINISH 4         // wavefronts of a block; 8 or 16 are faster here (1,641 and 1,434) and slower elsewhere (1,078 -> 1,087 and 1,104)
struct SharedLds {
    unsigned short list[CT_LOOK];
    int found[CT_LOOK / 64];
    f32x4 part[CT_FINISH - 1][64];
};
template <int DT, bool WIDE>
__device__ __forceinline__ void contrast_shared(const ContrastPar &c, int at, SharedLds &lds)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = at - c.B;
    for (int e0 = 0; e0 < c.d; e0 += 256) {
        const int e = e0 + lane * 4;
        const bool in = e < c.d;
        float term[4] = {}, x[4] = {};
        if (in) load4<DT, WIDE>(c.K, row, c.d, e, x);
        int left = c.count[row];
        for (int b = c.first[row]; left > 0 && b < c.B; b += CT_LOOK) {
            constexpr int WORDS = CT_LOOK / 64 / CT_FINISH;     // ballots of a wavefront
            u32 mine = 0;
#pragma unroll 4
            for (int w = 0; w < WORDS; ++w) {
                const int i = b + (wave * WORDS + w) * 64 + lane;
                mine |= (u32)(i < c.B && c.target[i] == row) << w;
            }
            for (int w = 0; w < WORDS; ++w) {
                const u64 hit = __ballot(mine >> w & 1);
                if (lane == 0) lds.found[wave * WORDS + w] = __popcll(hit);
            }
            __syncthreads();
            const int here = lds.found[lane], upto = inclusive(here, lane), n = __builtin_amdgcn_readlane(upto, 63);
            for (int w = 0; w < WORDS; ++w) {
                const int word = wave * WORDS + w;
                const u64 hit = __ballot(mine >> w & 1);
                if (mine >> w & 1)
                    lds.list[__builtin_amdgcn_readlane(upto - here, word) + __popcll(hit & lanes_below(lane))] = (unsigned short)(word * 64 + lane);
            }
            __syncthreads();
            const int end = n * (wave + 1) / CT_FINISH;
            // rows that a wavefront has on the way; eight of float32 spill so much that every call pays for it (2,000 x 10,000 x 100: 241 us, four 239)
            constexpr int ROWS = DT == DT_F32 ? 4 : 8;
            for (int j = n * wave / CT_FINISH; in && j < end; j += ROWS) {
                float y[ROWS][4], own[ROWS];
#pragma unroll
                for (int k = 0; k < ROWS; ++k) {
                    const int i = b + lds.list[j + k < end ? j + k : end - 1];
                    own[k] = c.row_own[i];
                    load4<DT, WIDE>(c.Q, i, c.d, e, y[k]);
                }
#pragma unroll
                for (int k = 0; k < ROWS; ++k)
                    if (j + k < end)
#pragma unroll
                        for (int h = 0; h < 4; ++h) term[h] = fmaf(own[k], y[k][h] - x[h], term[h]);
            }
            left -= n;
            __syncthreads();        // the lists are used again
        }
        if (wave) lds.part[wave - 1][lane] = (f32x4){term[0], term[1], term[2], term[3]};
        __syncthreads();
        if (wave == 0) {
            const GradRow<DT, WIDE> mine(c, at);
            if (in) {
                float a[4] = {};
                mine.load(e, a, x);
                for (int w = 0; w < CT_FINISH - 1; ++w)
#pragma unroll
                    for (int k = 0; k < 4; ++k) term[k] += lds.part[w][lane][k];
#pragma unroll
                for (int k = 0; k < 4; ++k) a[k] += term[k];
                mine.store(e, a);
            }
        }
        __syncthreads();
    }
}

// Joins the parts of a sum, takes off the row itself times the sum of its g, adds the target's term, and rounds.  A wavefront per row,
// four coordinates a lane; then the block's keys that many queries share.  The rows of a block lie gridDim.x apart, so that neighbouring keys of this kind
// are those of different blocks.  Every wavefront sees for itself whether there are any: a barrier for all would hold the fast ones back (8,192 x
// 16,384 x 768, random targets: 1,091 -> 1,107 us).  Eight wavefronts per SIMD, though contrast_shared() spills then: five cost every call more (1,078 -> 1,087).
template <int DT, bool WIDE>
__global__ __launch_bounds__(64 * CT_FINISH, 8) void k_contrast_finish(ContrastPar c)
{
    __shared__ SharedLds lds;
    const int lane = threadIdx.x & 63, total = c.B + c.M, mine_at = (int)(blockIdx.x + lane * gridDim.x);
    const u64 shared = __ballot(lane < CT_FINISH && mine_at >= c.B && mine_at < total && c.count[mine_at - c.B] > CT_SHARED);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), at = (int)(blockIdx.x + wave * gridDim.x);
    const bool keys = at >= c.B;
    const int row = keys ? at - c.B : at;
    if (at >= total || shared >> wave & 1) {
    } else if (keys ? key_gone(c, row) : !row_counts(c, row)) {
        const float zero[4] = {};
        for (int e = lane * 4; e < c.d; e += 256) store4<DT, WIDE>(keys ? c.dK : c.dQ, row, c.d, e, zero);
    } else {
        const int found = keys ? c.count[row] : 1, first = keys ? found ? c.first[row] : 0 : c.target[row];
        const GradRow<DT, WIDE> mine(c, at);
        const void *theirs = keys ? c.Q : c.K;
        for (int e0 = 0; e0 < c.d; e0 += 256) {        // all lanes stay: the search below needs them
            const int e = e0 + lane * 4;
            const bool in = e < c.d;
            float a[4] = {}, x[4] = {};
            if (in) mine.load(e, a, x);
            // the target's term; a key that is the target of several queries takes them in their order
            int i = first;
            for (int left = found; left > 0; --left) {
                if (in) {
                    const float own = c.row_own[keys ? i : row];
                    float y[4];
                    load4<DT, WIDE>(theirs, i, c.d, e, y);
#pragma unroll
                    for (int k = 0; k < 4; ++k) a[k] = fmaf(own, y[k] - x[k], a[k]);
                }
                if (left == 1) break;
                int next = -1;
                for (int b = i + 1; b < c.B && next < 0; b += 256) {
                    int t[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) t[k] = b + k * 64 + lane < c.B ? c.target[b + k * 64 + lane] : -1;
#pragma unroll
                    for (int k = 3; k >= 0; --k) {
                        const u64 hit = __ballot(t[k] == row);
                        if (hit) next = b + k * 64 + __builtin_ctzll(hit);
                    }
                }
                if (next < 0) break;
                i = next;
            }
            if (in) mine.store(e, a);
        }
    }
    for (u64 left = shared; left; left &= left - 1) contrast_shared<DT, WIDE>(c, (int)(blockIdx.x + __builtin_ctzll(left) * gridDim.x), lds);
}

// ------------------------------------------------------------------------------------------------ host side
static size_t layout(ContrastPar &c, ContrastPlan &plan, int dtype, int want_grad, char *base)
{
    return contrast_layout(c, plan, dtype, want_grad, base, [&](auto &take) {
        take(c.first, c.M);
        take(c.count, c.M);
        take(c.own_logit, ct_up(c.B, CT_PAD));
    });
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
    ContrastPlan plan;
    c.B = (int)B;
    c.M = (int)M;
    c.d = d;
    *bytes = layout(c, plan, dtype, want_grad, nullptr);
    return RNND_OK;
}

template <int DT, int TILE, bool TERMS>
static void launch_products(ContrastPar &c, int want_grad, int row_blocks, hipStream_t st)
{
    static_assert(DT != DT_F32 || TILE == 128, "g of three planes takes more registers than tiles of 256 leave");
    const int tq = ct_up(c.B, TILE) / TILE, tk = ct_up(c.M, TILE) / TILE;
    in_launches((u64)tq * tk, 256, [&](u64 first, u64 blocks) {
        hipLaunchKernelGGL((k_contrast_sums<TILE, DT, TERMS, ContrastPar>), dim3((u32)blocks), dim3(256), 0, st, c, (u32)first, tq, tk);
    });
    hipLaunchKernelGGL(k_contrast_loss<DT>, dim3((c.B + 3) / 4), dim3(256), 0, st, c, row_blocks);
    if (!want_grad) return;
    in_launches((u64)tq * tk, 256, [&](u64 first, u64 blocks) {
        hipLaunchKernelGGL((k_contrast_g<TILE, DT, TERMS, ContrastPar>), dim3((u32)blocks), dim3(256), 0, st, c, (u32)first, tq, tk);
    });
}
template <int DT, bool WIDE>
static void launch_contrast(ContrastPar &c, const ContrastPlan &plan, int want_grad, hipStream_t st)
{
    const int Br = ct_up(c.B, CT_PAD), Mr = ct_up(c.M, CT_PAD);
    const int key_blocks = Mr / 4 < CT_ROW_BLOCKS ? Mr / 4 : CT_ROW_BLOCKS, row_blocks = Br / 4 < CT_ROW_BLOCKS ? Br / 4 : CT_ROW_BLOCKS;
    // (by columns the padding of d up to a whole tile is written too: the products read it)
    const int across = (want_grad ? c.dr : c.dp) / 64;
    if constexpr (DT == DT_F32)
        hipLaunchKernelGGL(k_contrast_centre<ContrastPar>, dim3((c.dp + 64 * CT_SAMPLES - 1) / (64 * CT_SAMPLES)), dim3(64 * CT_SAMPLES), 0, st, c);
    in_launches((u64)(key_blocks + row_blocks) + (u64)((Br + Mr) / 64) * across, 256, [&](u64 first, u64 blocks) {
        hipLaunchKernelGGL((k_contrast_prepare<DT, WIDE>), dim3((u32)blocks), dim3(256), 0, st, c, (u32)first, key_blocks, row_blocks, Br / 64, across,
                           want_grad);
    });
    if constexpr (DT != DT_F32) {
        if (plan.tile == 256) launch_products<DT, 256, false>(c, want_grad, row_blocks, st);
        else launch_products<DT, 128, false>(c, want_grad, row_blocks, st);
    } else if (plan.terms) launch_products<DT, 128, true>(c, want_grad, row_blocks, st);
    else launch_products<DT, 128, false>(c, want_grad, row_blocks, st);
    if (!want_grad) return;
    if constexpr (DT != DT_F32) {
        if (plan.tile_g == 256) launch_grads<DT, 256>(c, st);
        else launch_grads<DT, 128>(c, st);
    } else
        launch_grads<DT, 128>(c, st);
    hipLaunchKernelGGL((k_contrast_finish<DT, WIDE>), dim3((c.B + c.M + CT_FINISH - 1) / CT_FINISH), dim3(64 * CT_FINISH), 0, st, c);
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
        hipLaunchKernelGGL(k_contrast_zero<ContrastPar>, dim3((u32)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, (hipStream_t)stream,
                           (unsigned short *)dK, n);
        return launched("rnnd_contrast");
    }
    ContrastPar c = {};
    ContrastPlan plan;
    c.Q = Q;
    c.K = K;
    c.target = target;
    c.query_ids = query_ids;
    c.key_ids = key_ids;
    c.bias = key_bias;
    c.left_out = -INFINITY;
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
    if (workspace_bytes < layout(c, plan, dtype, want_grad, (char *)workspace)) return RNND_ERR_SCRATCH;
    hipStream_t st = (hipStream_t)stream;
    int vec = row_vec(d, Q, (int)size, K, (int)size);
    if (want_grad) {
        const int vg = row_vec(d, dQ, (int)size, dK, (int)size);
        vec = vg < vec ? vg : vec;
    }
#define RNND_CONTRAST(DT) \
    if (vec >= 4) launch_contrast<DT, true>(c, plan, want_grad, st); \
    else launch_contrast<DT, false>(c, plan, want_grad, st)
    if (dtype == RNND_F32) { RNND_CONTRAST(DT_F32); }
    else if (dtype == RNND_F16) { RNND_CONTRAST(DT_F16); }
    else { RNND_CONTRAST(DT_BF16); }
#undef RNND_CONTRAST
    return launched("rnnd_contrast");
}
