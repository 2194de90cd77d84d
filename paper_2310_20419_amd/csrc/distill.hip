// Distillation: the divergence of the softmax over squared distances from what another model said, and its gradients.
//
//   s_ij   = bias_j - scale |q_i - k_j|^2,  P_ij = exp(s_ij - lse_i)          the student, over all keys that are not left out
//   p_it   = the teacher's probability of entry t of the list of query i; r_i what it leaves to the keys off the list
//   loss_i = sum_t p_it (log p_it - log P_it) + r_i (log r_i - log R_i),  R_i the student's mass off the list
//   g_ij   = w_i (P_ij - p_ij) on the list, w_i P_ij (1 - r_i / R_i) off it   (without a rest: w_i P_ij)
//   dq_i   = 2 scale sum_j g_ij (k_j - q_i),  dk_j = 2 scale sum_i g_ij (q_i - k_j)
//
// The products are those of rnnd_contrast (contrast.h), with lists in the place of targets: the sums of a row are of the keys off its
// list, so that neither R nor what follows from it is a small difference of large numbers, and the logits of listed keys are written
// out by the tile that they lie in.  The lists are sorted by key, with the place where every tile begins, so a tile marks its listed
// keys in a bitmap in LDS while its first loads are under way; a key's place in the list is the number of marks before it in its row.
// Off the list g is a factor of the row times 2^(s - the largest logit there), w (R - r) over the sum there: again no difference
// of large numbers where a key has little of both.  It is rounded to the type of the rows for the products (float32 rows: three terms).
// Listed keys have the largest g, of both signs, and often rows that lie close together, so that rounded ones would leave an error of the
// size of the gradient (float16, 300 queries, lists of 7: 3.5e-4 of its norm, where rounding the result costs 2.1e-4): theirs is float32, kept
// out of the products, and added row by row at the end.  For the gradient of a key a bitmap says which queries list it.
// The teacher's probabilities are summed in double precision: 1 - sum p of a teacher that is sure is a small difference, and there are few of them.
#include <cmath>

#include "contrast.h"

struct DistillPar : ContrastPar {
    const int *ids;             // [B][entries]
    const float *logits;
    int entries, tail;
    int tiles_k;                // tiles of the logits across the keys
    int *list_key;              // [B padded][entries] keys that count, ascending; from here on a row's lists are in this order
    float *list_p, *list_s, *list_g;    // the teacher's probability; the logit in base 2; g
    float2 *list_sum;           // [B] sum of the list's p, r
    unsigned char *list_at;     // [B padded][tiles_k + 1] place of a tile's first key; of the end
    u32 *marks;                 // [M][words] the queries that list a key
    int words;
};

__device__ __forceinline__ bool entry_counts(const DistillPar &c, int i, int e)
{
    const int j = c.ids[(size_t)i * c.entries + e];
    return (u32)j < (u32)c.M && !(c.logits[(size_t)i * c.entries + e] == -INFINITY) && !key_gone(c, j) &&
           !(c.query_ids && c.key_ids[j] == c.query_ids[i]);
}
__device__ __forceinline__ bool row_counts(const DistillPar &c, int i)
{
    for (int e = 0; e < c.entries; ++e)
        if (entry_counts(c, i, e)) return true;
    return false;
}

// ------------------------------------------------------------------------------------------------ a row's marks in a tile
template <> constexpr bool has_lists<DistillPar>() { return true; }

template <int TILE> struct ListLds<TILE, DistillPar> {
    u32 bits[TILE * TILE / 32];
    u32 cols[TILE];                             // of the row's first four keys of this tile, a byte each
    unsigned char first[TILE], count[TILE];     // place of the row's first key of this tile in its list, and how many they are
};

template <int TILE>
__device__ __forceinline__ void load_lists(const DistillPar &c, ListLds<TILE, DistillPar> &lists, int row0, int tile_c)
{
    const int t = threadIdx.x;
#pragma unroll
    for (int i = 0; i < TILE * TILE / 32 / 256; ++i) lists.bits[i * 256 + t] = 0;
    __syncthreads();
    if (t >= TILE) return;
    const unsigned char *ends = &c.list_at[(size_t)(row0 + t) * (c.tiles_k + 1) + tile_c];
    const int first = ends[0], n = ends[1] - first;
    lists.first[t] = (unsigned char)first;
    lists.count[t] = (unsigned char)n;
    const int *keys = &c.list_key[(size_t)(row0 + t) * c.entries + first];
    u32 cols = 0;
    for (int e = 0; e < n; ++e) {
        const int col = keys[e] - tile_c * TILE;
        atomicOr(&lists.bits[(t * TILE + col) >> 5], 1u << (col & 31));
        if (e < 4) cols |= (u32)col << (8 * e);
    }
    lists.cols[t] = cols;
}

template <int TILE>
__device__ __forceinline__ u32 marks_at(const ListLds<TILE, DistillPar> &lists, int row, int col)
{
    return lists.bits[(row * TILE + col) >> 5] >> (col & 31) & ((1u << (TILE / 32)) - 1);
}
// marks of the row before the column
template <int TILE>
__device__ __forceinline__ int marks_before(const ListLds<TILE, DistillPar> &lists, int row, int col)
{
    if (lists.count[row] < 2) return 0;
    const u32 *words = &lists.bits[row * TILE >> 5];
    int n = __popc(words[col >> 5] & ((1u << (col & 31)) - 1));
    for (int w = 0; w < col >> 5; ++w) n += __popc(words[w]);
    return n;
}

// Four rows' logits: those of listed keys become -infinity.  WRITE: the first of a lane's N columns goes to `room` (LDS, a place for each row and lane of
// the 32 that share it), from where write_listed() takes it; others, which are rare, go to their place at once.  (Finding that place for
// every listed key here held the wavefront up: 8,192 x 16,384 x 768, lists of 32, 366 us for the logits and their sums.)
template <bool WRITE, int TILE, int N>
__device__ __forceinline__ void take_listed(std::integral_constant<bool, WRITE>, const DistillPar &c, const ListLds<TILE, DistillPar> &lists, float *room,
                                            int row0, int row, int col, float (&s)[4][N])
{
    u32 marks[4], any = 0;
#pragma unroll
    for (int r = 0; r < 4; ++r) any |= marks[r] = marks_at(lists, row + r, col);
    if (!__any(any)) return;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if constexpr (WRITE) {
            const u32 more = marks[r] & (marks[r] - 1);
            if (__any(more)) {
                if (more) {
                    float *to = &c.list_s[(size_t)(row0 + row + r) * c.entries + lists.first[row + r] + marks_before(lists, row + r, col)];
#pragma unroll
                    for (int n = 0; n < N; ++n)
                        if (marks[r] >> n & 1) *to++ = s[r][n];
                }
            }
            float first = s[r][N - 1];
#pragma unroll
            for (int n = N - 2; n >= 0; --n) first = marks[r] >> n & 1 ? s[r][n] : first;
            if (marks[r]) room[(row + r) * 32 + col / N] = first;
        }
#pragma unroll
        for (int n = 0; n < N; ++n) s[r][n] = marks[r] >> n & 1 ? -INFINITY : s[r][n];
    }
}

template <int TILE>
__device__ __forceinline__ void write_listed(const DistillPar &c, const ListLds<TILE, DistillPar> &lists, const float *room, int row0, int tile_c)
{
    constexpr int N = TILE / 32;
    __syncthreads();
    const int t = threadIdx.x;
    if (t >= TILE) return;
    const size_t from = (size_t)(row0 + t) * c.entries + lists.first[t];
    const int n = lists.count[t];
    const u32 cols = lists.cols[t];
    for (int e = 0; e < n; ++e) {
        const int col = e < 4 ? (int)(cols >> (8 * e) & 0xFF) : c.list_key[from + e] - tile_c * TILE;
        if (!(marks_at(lists, t, col & ~(N - 1)) & ((1u << (col & (N - 1))) - 1))) c.list_s[from + e] = room[t * 32 + col / N];
    }
}

// ------------------------------------------------------------------------------------------------ preparation
__device__ __forceinline__ double wave_sum_f64(double v)
{
#pragma unroll
    for (int s = 32; s; s >>= 1) v += __shfl_xor(v, s);
    return v;
}
__device__ __forceinline__ float wave_max_f32(float v)
{
#pragma unroll
    for (int s = 32; s; s >>= 1) v = fmaxf(v, __shfl_xor(v, s));
    return v;
}

// A query's list, by a wavefront: entries that count in the order of their keys, each key once (the first entry that names it), and
// the teacher's probabilities.  keys: the wavefront's own place in LDS.
#define DS_MAX RNND_MAX_LISTED
__device__ __forceinline__ void distill_row(const DistillPar &c, int i, int lane, int *keys, int logit_tile)
{
    const size_t from = (size_t)i * c.entries;
    u64 k[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int e = r * 64 + lane;
        k[r] = i < c.B && e < c.entries && entry_counts(c, i, e) ? (u64)(u32)c.ids[from + e] << 8 | (u32)e : ~0ull;
    }
    wave_sort<2>(k);
    const u64 before[2] = {shfl_up1_u64(k[0]), shfl_up1_u64(k[1])}, last = shfl_u64(k[0], 63);
    bool on[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const u64 b = lane ? before[r] : r ? last : ~0ull;
        on[r] = k[r] != ~0ull && (b == ~0ull || b >> 8 != k[r] >> 8);
    }
    const u64 m0 = __ballot(on[0]), m1 = __ballot(on[1]);
    const int n0 = (int)__popcll(m0), n = n0 + (int)__popcll(m1);
    const int at[2] = {(int)__popcll(m0 & lanes_below(lane)), n0 + (int)__popcll(m1 & lanes_below(lane))};
    float l[2];
    double p[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) l[r] = on[r] ? c.logits[from + (k[r] & 0xFF)] : -INFINITY;
    const float most = n ? wave_max_f32(fmaxf(l[0], l[1])) : 0.0f, top = c.tail ? fmaxf(most, 0.0f) : most;      // (above 0 the sum is above 1)
#pragma unroll
    for (int r = 0; r < 2; ++r) p[r] = on[r] ? exp((double)l[r] - (double)top) : 0.0;
    const double sum = wave_sum_f64(p[0] + p[1]);
    const double rest = c.tail && top == 0.0f && sum < 1.0 ? 1.0 - sum : 0.0, mass = n ? sum + rest : 1.0;
#pragma unroll
    for (int r = 0; r < 2; ++r)
        if (on[r]) {
            keys[at[r]] = (int)(k[r] >> 8);
            c.list_key[from + at[r]] = (int)(k[r] >> 8);
            c.list_p[from + at[r]] = (float)(p[r] / mass);
        }
    wave_sync();
    unsigned char *ends = &c.list_at[(size_t)i * (c.tiles_k + 1)];
    for (int t = lane; t <= c.tiles_k; t += 64) {
        int lo = 0, hi = n;         // keys below the tile's first
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (keys[mid] < t * logit_tile) lo = mid + 1;
            else hi = mid;
        }
        ends[t] = (unsigned char)lo;
    }
    wave_sync();
    if (lane == 0) {
        if (i < c.B) c.list_sum[i] = make_float2((float)(sum / mass), (float)(rest / mass));
        c.row_id[i] = make_int2(CT_NEVER, n && c.query_ids ? c.query_ids[i] : CT_NEVER);
        const float w = n ? c.row_weight ? c.row_weight[i] : 1.0f : 0.0f;
        c.row_g[i] = make_float2(INFINITY, w);
        c.row_own[i] = w;
    }
}

// A wavefront per row, keys first; then the copies of the rows (contrast_copy()), in the same launch.
template <int DT, bool WIDE>
__global__ __launch_bounds__(256) void k_distill_prepare(DistillPar c, u32 first, int key_blocks, int row_blocks, int q_tiles, int across, int columns, int logit_tile)
{
    __shared__ int keys_of[4][DS_MAX];
    __shared__ u32 most;
    const int block = (int)(first + blockIdx.x), id = block - key_blocks - row_blocks;
    if (id >= 0) {
        contrast_copy<DT, WIDE>(c, id / across, id % across * 64, q_tiles, columns);
        return;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (block < key_blocks) {
        const int padded = ct_up(c.M, CT_PAD);
        for (int at = (block * 4 + wave) * 4; at < padded; at += key_blocks * 16) {
            const int four[4] = {at, at + 1, at + 2, at + 3};
            float norm[4];
            key_sides<DT, WIDE, 4>(c, four, padded, lane, norm);
            if (!c.dK) continue;
            for (int t = lane; t < (c.M - at < 4 ? c.M - at : 4) * c.words; t += 64) c.marks[(size_t)at * c.words + t] = 0;
        }
        return;
    }
    if (threadIdx.x == 0) most = 0;
    __syncthreads();
    for (int at = (block - key_blocks) * 4 + wave; at < ct_up(c.B, CT_PAD); at += row_blocks * 4) {
        distill_row(c, at, lane, keys_of[wave], logit_tile);
        if (DT == DT_F16 && lane == 0) {
            const u32 bits = __float_as_uint(c.row_own[at]) & 0x7FFFFFFFu;
            if (bits < 0x7F800000u) atomicMax(&most, bits);
        }
    }
    __syncthreads();
    if (DT == DT_F16 && threadIdx.x == 0) c.tops[block - key_blocks] = most;
}

// ------------------------------------------------------------------------------------------------ the loss
// A wavefront per query joins the parts of its sum and its list: the loss, and what the second product needs.
template <int DT>
__global__ __launch_bounds__(256) void k_distill_loss(DistillPar c, int row_blocks)
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
    const int n = c.list_at[(size_t)i * (c.tiles_k + 1) + c.tiles_k];
    if (!n) {
        if (lane == 0) c.loss[i] = 0.0f;
        return;
    }
    float top = -INFINITY, sum = 0.0f;
    for (int t = lane; t < c.parts_k; t += 64) {
        const float2 part = c.part[(size_t)i * c.parts_k + t];
        join_parts(top, sum, part.x, part.y);
    }
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) join_parts(top, sum, __shfl_xor(top, s), __shfl_xor(sum, s));
    float s[2], p[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int e = r * 64 + lane;
        s[r] = e < n ? c.list_s[(size_t)i * c.entries + e] : -INFINITY;
        p[r] = e < n ? c.list_p[(size_t)i * c.entries + e] : 0.0f;
    }
    const float2 mass = c.list_sum[i];
    const bool others = top > -INFINITY || !(sum == 0.0f);      // keys off the list
    float rest = mass.y;
    if (!others && rest > 0.0f) {       // nothing can have what the teacher left: the list alone
        rest = 0.0f;
#pragma unroll
        for (int r = 0; r < 2; ++r) p[r] /= mass.x;
    }
    // The loss is a difference of sums that are larger than it where teacher and student agree, so it is formed in double precision: its error is that
    // of the logits and their sums.
    const float m = fmaxf(top, wave_max_f32(fmaxf(s[0], s[1]))), ref = m == -INFINITY ? 0.0f : m;
    const double x[2] = {(double)s[0] - (double)ref, (double)s[1] - (double)ref}, e[2] = {exp2(x[0]), exp2(x[1])};
    const double off = others ? (double)sum * exp2((double)top - (double)ref) : 0.0, total = off + wave_sum_f64(e[0] + e[1]), log_total = log2(total);
    const float w = c.row_own[i], up_w = ldexpf(w, up);
    double loss = 0.0;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int at = r * 64 + lane;
        if (at >= n) continue;
        // (an entry whose probability is below the smallest float has none)
        if (!(p[r] == 0.0f)) loss = fma((double)p[r], log2((double)p[r]) - (x[r] - log_total), loss);
        if (!c.dK) continue;
        c.list_g[(size_t)i * c.entries + at] = w * (float)(e[r] / total - (double)p[r]);
        const int j = c.list_key[(size_t)i * c.entries + at];
        atomicOr(&c.marks[(size_t)j * c.words + (i >> 5)], 1u << (i & 31));
    }
    loss = wave_sum_f64(loss);
    if (lane) return;
    if (rest > 0.0f) {
        const double log_off = (double)top - (double)ref + log2((double)sum);
        loss = fma((double)rest, log2((double)rest) - (log_off - log_total), loss);
    }
    // (the sum off the list as a factor: its logarithm would be lost in the steps of logits of many millions)
    if (others) c.row_g[i] = make_float2(top, (float)((double)up_w * (off / total - (double)rest) / (double)sum));
    c.loss[i] = (float)(loss * 0.69314718055994531);
}

// ------------------------------------------------------------------------------------------------ joining the gradients' parts
// A wavefront per row, queries first: the listed terms, four coordinates a lane and H of these at a time.  A key that more than DS_SHARED queries
// list is summed by the whole block, a part of the queries to each wavefront, and their sums are added in order.  The keys of a block lie
// apart, so that neighbouring keys of this kind are those of different blocks.
#define DS_FINISH 8             // wavefronts of a block
#define DS_SHARED 128
#define DS_RUN 64               // words of marks looked at together, one for each lane; by a whole block fewer, so that all its wavefronts have some
#define DS_RUN_SHARED 4         // (no more than DS_SHARED queries)
#define DS_ROWS 4               // rows on the way
struct KeyLds {
    unsigned short list[DS_FINISH][DS_SHARED];
    f32x4 part[DS_FINISH][64];
    u32 shared;                 // wavefronts whose keys these are
};

// Adds g (row - x) of n entries; lane e holds entry e: its row's number and its g.  e0: the first coordinate; x: the row of the sum.
template <int DT, bool WIDE, int H>
__device__ __forceinline__ void add_terms(const DistillPar &c, const void *rows, int e0, const float (&x)[H][4], int number, float g, int n, int lane,
                                          float (&sum)[H][4])
{
    typedef typename RowType<DT>::T T;
    for (int j = 0; j < n; j += DS_ROWS) {
        Pack<DT, 4> packs[DS_ROWS][H];
#pragma unroll
        for (int r = 0; r < DS_ROWS; ++r) {
            const T *row = (const T *)rows + (size_t)__builtin_amdgcn_readlane(number, j + r < n ? j + r : n - 1) * c.d;
#pragma unroll
            for (int h = 0; h < H; ++h) {
                const int e = e0 + h * 256 + lane * 4, from = e < c.d ? e : 0;      // (what lies behind the row is not stored)
                if constexpr (WIDE) packs[r][h] = load_pack<DT, 4>(row, from);
                else
#pragma unroll
                    for (int k = 0; k < 4; ++k) packs[r][h].v[k] = from + k < c.d ? row[from + k] : (T)0.0f;
            }
        }
#pragma unroll
        for (int r = 0; r < DS_ROWS; ++r) {
            const float own = j + r < n ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(g), j + r < n ? j + r : n - 1)) : 0.0f;
#pragma unroll
            for (int h = 0; h < H; ++h) {
                float y[4];
                unpack<DT, 4>(packs[r][h], y);
#pragma unroll
                for (int k = 0; k < 4; ++k) sum[h][k] = fmaf(own, y[k] - x[h][k], sum[h][k]);
            }
        }
    }
}

// Terms of the queries that list key j, of the runs of `words` words of marks first, first + step, ..; list: the wavefront's own.
template <int DT, bool WIDE, int H>
__device__ __forceinline__ void add_queries(const DistillPar &c, int j, int e0, const float (&x)[H][4], int words, int first, int step, unsigned short *list,
                                            int lane, float (&sum)[H][4])
{
    for (int run = first; run * words < c.words; run += step) {
        const int at = run * words + lane;
        u32 marks = lane < words && at < c.words ? c.marks[(size_t)j * c.words + at] : 0;
        const int here = (int)__popc(marks), upto = inclusive(here, lane), n = __builtin_amdgcn_readlane(upto, 63);
        if (!n) continue;
        for (int to = upto - here; marks; marks &= marks - 1) list[to++] = (unsigned short)(lane * 32 + __builtin_ctz(marks));
        wave_sync();
        for (int t = 0; t < n; t += 64) {
            const int i = t + lane < n ? run * words * 32 + list[t + lane] : -1;
            float g = 0.0f;
            if (i >= 0) {
                const int *keys = &c.list_key[(size_t)i * c.entries];
                int lo = 0, hi = c.list_at[(size_t)i * (c.tiles_k + 1) + c.tiles_k] - 1;        // it is there
                while (lo < hi) {
                    const int mid = (lo + hi) >> 1;
                    if (keys[mid] < j) lo = mid + 1;
                    else hi = mid;
                }
                g = c.list_g[(size_t)i * c.entries + lo];
            }
            add_terms<DT, WIDE, H>(c, c.Q, e0, x, i, g, n - t < 64 ? n - t : 64, lane, sum);
        }
        wave_sync();
    }
}

template <int DT, bool WIDE, int H>
__device__ __forceinline__ void load_row(const DistillPar &c, const void *rows, int row, int e0, int lane, float (&x)[H][4])
{
#pragma unroll
    for (int h = 0; h < H; ++h) {
        const int e = e0 + h * 256 + lane * 4;
        load4<DT, WIDE>(rows, row, c.d, e < c.d ? e : 0, x[h]);
    }
}
// The parts of the products and the listed terms, rounded
template <int DT, bool WIDE, int H>
__device__ __forceinline__ void finish_row(const DistillPar &c, const GradRow<DT, WIDE> &mine, int e0, int lane, const float (&sum)[H][4])
{
#pragma unroll
    for (int h = 0; h < H; ++h) {
        const int e = e0 + h * 256 + lane * 4;
        if (e >= c.d) continue;
        float a[4] = {}, own[4];
        mine.load(e, a, own);
#pragma unroll
        for (int k = 0; k < 4; ++k) a[k] += sum[h][k];
        mine.store(e, a);
    }
}

template <int DT, bool WIDE>
__device__ __forceinline__ void no_gradient(const DistillPar &c, void *to, int row, int lane)
{
    const float zero[4] = {};
    for (int e = lane * 4; e < c.d; e += 256) store4<DT, WIDE>(to, row, c.d, e, zero);
}

// how many queries list a key
__device__ __forceinline__ int queries_of(const DistillPar &c, int j, int lane)
{
    const u32 *marks = &c.marks[(size_t)j * c.words];
    int n = 0;
    for (int t = lane; t < c.words; t += 256) {
        u32 m[4];
#pragma unroll
        for (int h = 0; h < 4; ++h) m[h] = t + h * 64 < c.words ? marks[t + h * 64] : 0;
#pragma unroll
        for (int h = 0; h < 4; ++h) n += (int)__popc(m[h]);
    }
#pragma unroll
    for (int s = 32; s; s >>= 1) n += __shfl_xor(n, s);
    return __builtin_amdgcn_readfirstlane(n);
}

template <int DT, bool WIDE, int H>
__global__ __launch_bounds__(64 * DS_FINISH) void k_distill_finish(DistillPar c, int query_blocks)
{
    __shared__ KeyLds lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if ((int)blockIdx.x < query_blocks) {
        const int i = blockIdx.x * DS_FINISH + wave;
        if (i >= c.B) return;
        const int n = c.list_at[(size_t)i * (c.tiles_k + 1) + c.tiles_k];
        if (!n) return no_gradient<DT, WIDE>(c, c.dQ, i, lane);
        const GradRow<DT, WIDE> mine(c, i);
        for (int e0 = 0; e0 < c.d; e0 += 256 * H) {
            float x[H][4], sum[H][4] = {};
            load_row<DT, WIDE, H>(c, c.Q, i, e0, lane, x);
            for (int t = 0; t < n; t += 64) {
                const size_t e = (size_t)i * c.entries + t + lane;
                const bool on = t + lane < n;
                add_terms<DT, WIDE, H>(c, c.K, e0, x, on ? c.list_key[e] : 0, on ? c.list_g[e] : 0.0f, n - t < 64 ? n - t : 64, lane, sum);
            }
            finish_row<DT, WIDE, H>(c, mine, e0, lane, sum);
        }
        return;
    }
    const int first = blockIdx.x - query_blocks, apart = gridDim.x - query_blocks;
    if (threadIdx.x == 0) lds.shared = 0;
    __syncthreads();
    // a key of the wavefront's own, then those of the block that are summed together
    int j = first + wave * apart;
    bool alone = false;
    if (j < c.M) {
        if (key_gone(c, j)) no_gradient<DT, WIDE>(c, c.dK, j, lane);
        else if (queries_of(c, j, lane) <= DS_SHARED) alone = true;
        else if (lane == 0) atomicOr(&lds.shared, 1u << wave);
    }
    u32 left = 0;
    for (bool own = true;; own = false) {
        if (!own) {
            if (!left) break;
            j = first + __builtin_ctz(left) * apart;
            left &= left - 1;
        }
        if (!own || alone) {
            const GradRow<DT, WIDE> mine(c, c.B + j);
            for (int e0 = 0; e0 < c.d; e0 += 256 * H) {
                float x[H][4], sum[H][4] = {};
                load_row<DT, WIDE, H>(c, c.K, j, e0, lane, x);
                add_queries<DT, WIDE, H>(c, j, e0, x, own ? DS_RUN : DS_RUN_SHARED, own ? 0 : wave, own ? 1 : DS_FINISH, lds.list[wave], lane, sum);
                if (!own) {
#pragma unroll
                    for (int h = 0; h < H; ++h) {
                        __syncthreads();
                        lds.part[wave][lane] = (f32x4){sum[h][0], sum[h][1], sum[h][2], sum[h][3]};
                        __syncthreads();
                        for (int w = 1; wave == 0 && w < DS_FINISH; ++w)
#pragma unroll
                            for (int k = 0; k < 4; ++k) sum[h][k] += lds.part[w][lane][k];
                    }
                    if (wave) continue;
                }
                finish_row<DT, WIDE, H>(c, mine, e0, lane, sum);
            }
        }
        if (own) {
            __syncthreads();
            left = lds.shared;
        }
    }
}

// ------------------------------------------------------------------------------------------------ host side
static size_t layout(DistillPar &c, ContrastPlan &plan, int dtype, int want_grad, char *base)
{
    c.terms_from = 1536;
    return contrast_layout(c, plan, dtype, want_grad, base, [&](auto &take) {
        const size_t Br = ct_up(c.B, CT_PAD);
        c.tiles_k = c.parts_k / 2;
        take(c.list_key, Br * c.entries);
        take(c.list_p, Br * c.entries);
        take(c.list_s, Br * c.entries);
        take(c.list_g, Br * c.entries);
        take(c.list_sum, Br);
        take(c.list_at, Br * (c.tiles_k + 1));
        if (want_grad) {
            c.words = (c.B + 31) / 32;
            take(c.marks, (size_t)c.M * c.words);
        }
    });
}

static int check_distill(int64_t B, int64_t M, int32_t d, int dtype, int32_t entries)
{
    const int rc = check_contrast(B, M, d, dtype);
    if (rc) return rc;
    return entries < 1 || entries > DS_MAX ? RNND_ERR_BAD_PARAM : RNND_OK;
}

extern "C" int rnnd_distill_workspace(int64_t B, int64_t M, int32_t d, int dtype, int32_t entries, int want_grad, size_t *bytes)
{
    const int rc = check_distill(B, M, d, dtype, entries);
    if (rc) return rc;
    if (!bytes) return RNND_ERR_NULL;
    if (!B) {
        *bytes = 0;
        return RNND_OK;
    }
    DistillPar c = {};
    ContrastPlan plan;
    c.B = (int)B;
    c.M = (int)M;
    c.d = d;
    c.entries = entries;
    *bytes = layout(c, plan, dtype, want_grad, nullptr);
    return RNND_OK;
}

template <int DT, int TILE, bool TERMS>
static void launch_products(DistillPar &c, int want_grad, int row_blocks, hipStream_t st)
{
    const int tq = ct_up(c.B, TILE) / TILE, tk = ct_up(c.M, TILE) / TILE;
    in_launches((u64)tq * tk, 256, [&](u64 first, u64 blocks) {
        hipLaunchKernelGGL((k_contrast_sums<TILE, DT, TERMS, DistillPar>), dim3((u32)blocks), dim3(256), 0, st, c, (u32)first, tq, tk);
    });
    hipLaunchKernelGGL(k_distill_loss<DT>, dim3((c.B + 3) / 4), dim3(256), 0, st, c, row_blocks);
    if (!want_grad) return;
    in_launches((u64)tq * tk, 256, [&](u64 first, u64 blocks) {
        hipLaunchKernelGGL((k_contrast_g<TILE, DT, TERMS, DistillPar>), dim3((u32)blocks), dim3(256), 0, st, c, (u32)first, tq, tk);
    });
}

template <int DT, bool WIDE>
static void launch_distill(DistillPar &c, const ContrastPlan &plan, int want_grad, hipStream_t st)
{
    const int Br = ct_up(c.B, CT_PAD), Mr = ct_up(c.M, CT_PAD);
    const int key_blocks = Mr / 4 < CT_ROW_BLOCKS ? Mr / 4 : CT_ROW_BLOCKS, row_blocks = Br / 4 < CT_ROW_BLOCKS ? Br / 4 : CT_ROW_BLOCKS;
    const int across = (want_grad ? c.dr : c.dp) / 64;
    if constexpr (DT == DT_F32)
        hipLaunchKernelGGL(k_contrast_centre<DistillPar>, dim3((c.dp + 64 * CT_SAMPLES - 1) / (64 * CT_SAMPLES)), dim3(64 * CT_SAMPLES), 0, st, c);
    in_launches((u64)(key_blocks + row_blocks) + (u64)((Br + Mr) / 64) * across, 256, [&](u64 first, u64 blocks) {
        hipLaunchKernelGGL((k_distill_prepare<DT, WIDE>), dim3((u32)blocks), dim3(256), 0, st, c, (u32)first, key_blocks, row_blocks, Br / 64, across,
                           want_grad, plan.tile);
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
    const int query_blocks = (c.B + DS_FINISH - 1) / DS_FINISH;
    const dim3 grid(query_blocks + (c.M + DS_FINISH - 1) / DS_FINISH), block(64 * DS_FINISH);
    if (c.d <= 256) hipLaunchKernelGGL((k_distill_finish<DT, WIDE, 1>), grid, block, 0, st, c, query_blocks);
    else if (c.d <= 512) hipLaunchKernelGGL((k_distill_finish<DT, WIDE, 2>), grid, block, 0, st, c, query_blocks);
    else hipLaunchKernelGGL((k_distill_finish<DT, WIDE, 3>), grid, block, 0, st, c, query_blocks);
}

extern "C" int rnnd_distill(const void *Q, int64_t B, const void *K, int64_t M, int32_t d, int dtype, int metric, const int32_t *teacher_ids,
                            const float *teacher_logits, int32_t entries, int tail, const int32_t *query_ids, const int32_t *key_ids,
                            const float *key_bias, const float *row_weight, float scale, float *loss, void *dQ, void *dK, void *workspace,
                            size_t workspace_bytes, void *stream)
{
    const int rc = check_distill(B, M, d, dtype, entries);
    if (rc) return rc;
    if (metric != RNND_L2SQ) return RNND_ERR_UNSUPPORTED;
    if (!K || (B && (!Q || !teacher_ids || !teacher_logits || !loss)) || (query_ids && !key_ids)) return RNND_ERR_NULL;
    if (B && (dQ == nullptr) != (dK == nullptr)) return RNND_ERR_NULL;
    const size_t size = dt_size(dtype);
    if (((uintptr_t)Q | (uintptr_t)K | (uintptr_t)dQ | (uintptr_t)dK) % size) return RNND_ERR_BAD_PARAM;
    if (((uintptr_t)teacher_ids | (uintptr_t)teacher_logits | (uintptr_t)query_ids | (uintptr_t)key_ids | (uintptr_t)key_bias | (uintptr_t)row_weight |
         (uintptr_t)loss) % 4)
        return RNND_ERR_BAD_PARAM;
    if (!std::isfinite(scale) || (tail != 0 && tail != 1)) return RNND_ERR_BAD_PARAM;
    const int want_grad = dK != nullptr;
    if (!B) {       // no query: no gradient reaches a key
        if (!want_grad) return RNND_OK;
        const size_t n = (size_t)M * d * size / 2, blocks = (n + 1023) / 1024;
        hipLaunchKernelGGL(k_contrast_zero<DistillPar>, dim3((u32)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, (hipStream_t)stream,
                           (unsigned short *)dK, n);
        return launched("rnnd_distill");
    }
    DistillPar c = {};
    ContrastPlan plan;
    c.Q = Q;
    c.K = K;
    c.ids = teacher_ids;
    c.logits = teacher_logits;
    c.entries = entries;
    c.tail = tail;
    c.query_ids = query_ids;
    c.key_ids = key_ids;
    c.bias = key_bias;
    c.left_out = CT_LOWEST;
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
#define RNND_DISTILL(DT) \
    if (vec >= 4) launch_distill<DT, true>(c, plan, want_grad, st); \
    else launch_distill<DT, false>(c, plan, want_grad, st)
    if (dtype == RNND_F32) { RNND_DISTILL(DT_F32); }
    else if (dtype == RNND_F16) { RNND_DISTILL(DT_F16); }
    else { RNND_DISTILL(DT_BF16); }
#undef RNND_DISTILL
    return launched("rnnd_distill");
}
