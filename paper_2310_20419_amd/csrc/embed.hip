// Rows looked up by id, and the gradient of the table they come from.
//
//   out[t] = scale * table[ids[t]]                               (zero where ids[t] is no row of the table)
//   grad[v] (+)= scale * sum of dout[t] over the t with ids[t] = v, in ascending t
//
// Both only move rows: a lookup reads and writes n of them, a gradient reads n and writes V (added to what is there:
// reads and writes the rows that are named).  The gradient's sums are in float32 and in a fixed order, whatever
// the launch: the tokens are sorted by id (stable), and every sum runs over neighbours in that order.
#include "rows.h"

// ------------------------------------------------------------------------------------------------ lookup
#define EMBED_ITEMS 4

// A block takes rows_per_block rows; a thread one piece of VEC coordinates of EMBED_ITEMS rows at a time: their ids,
// then their pieces, are on the way together.
template <int DT, int OT, int VEC>
__global__ __launch_bounds__(256) void k_embed(const void *__restrict__ table, u32 V, u32 pieces, const int *__restrict__ ids,
                                               u64 n, float scale, void *__restrict__ out, u32 rows_per_block)
{
    const u64 row0 = (u64)blockIdx.x * rows_per_block;
    const u32 rows = (u32)(n - row0 < rows_per_block ? n - row0 : rows_per_block);
    const u32 total = rows * pieces;
    for (u32 base = threadIdx.x; base < total; base += 256 * EMBED_ITEMS) {
        int id[EMBED_ITEMS];
        u32 row[EMBED_ITEMS], piece[EMBED_ITEMS];
        Pack<DT, VEC> p[EMBED_ITEMS];
#pragma unroll
        for (int i = 0; i < EMBED_ITEMS; ++i) {
            const u32 at = base + 256 * i;
            row[i] = at / pieces;
            piece[i] = at - row[i] * pieces;
            id[i] = at < total ? ids[row0 + row[i]] : -1;
        }
#pragma unroll
        for (int i = 0; i < EMBED_ITEMS; ++i)
            if ((u32)id[i] < V) p[i] = load_pack<DT, VEC>(table, ((u64)(u32)id[i] * pieces + piece[i]) * VEC);
#pragma unroll
        for (int i = 0; i < EMBED_ITEMS; ++i) {
            if (base + 256 * i >= total) break;
            float x[VEC];
            unpack<DT, VEC>(p[i], x);
#pragma unroll
            for (int k = 0; k < VEC; ++k) x[k] = (u32)id[i] < V ? x[k] * scale : 0.0f;
            store_pack<OT, VEC>(out, ((row0 + row[i]) * pieces + piece[i]) * VEC, x);
        }
    }
}

template <int DT, int OT>
static void launch_embed(const void *table, int64_t V, int d, const int32_t *ids, int64_t n, float scale, void *out, hipStream_t st)
{
    const int vec = row_vec(d, table, dt_size(DT), out, dt_size(OT));
    const u32 pieces = d / vec;
    u64 rows = (256 * EMBED_ITEMS + pieces - 1) / pieces;      // one trip per block; small calls: one row per block at least
    const u64 blocks_min = (n + rows - 1) / rows;
    if (blocks_min > 0x7FFFFFFFull) rows = (n + 0x7FFFFFFEll) / 0x7FFFFFFFll;
    const dim3 grid((u32)((n + rows - 1) / rows));
#define RNND_EMBED(VEC) hipLaunchKernelGGL((k_embed<DT, OT, VEC>), grid, dim3(256), 0, st, table, (u32)V, pieces, ids, (u64)n, scale, out, (u32)rows)
    switch (vec) {
    case 8: RNND_EMBED(8); break;
    case 4: RNND_EMBED(4); break;
    case 2: RNND_EMBED(2); break;
    default: RNND_EMBED(1);
    }
#undef RNND_EMBED
}

#define RNND_FOR_TYPES(A, B, F)                                   \
    switch ((A) * 4 + (B)) {                                      \
    case RNND_F32 * 4 + RNND_F32: F(DT_F32, DT_F32); break;       \
    case RNND_F32 * 4 + RNND_F16: F(DT_F32, DT_F16); break;       \
    case RNND_F32 * 4 + RNND_BF16: F(DT_F32, DT_BF16); break;     \
    case RNND_F16 * 4 + RNND_F32: F(DT_F16, DT_F32); break;       \
    case RNND_F16 * 4 + RNND_F16: F(DT_F16, DT_F16); break;       \
    case RNND_F16 * 4 + RNND_BF16: F(DT_F16, DT_BF16); break;     \
    case RNND_BF16 * 4 + RNND_F32: F(DT_BF16, DT_F32); break;     \
    case RNND_BF16 * 4 + RNND_F16: F(DT_BF16, DT_F16); break;     \
    default: F(DT_BF16, DT_BF16);                                 \
    }

static int check_rows(int64_t V, int32_t d, int64_t n, int type_a, int type_b)
{
    if (!row_type(type_a) || !row_type(type_b)) return RNND_ERR_UNSUPPORTED;
    if (V < 1 || V > 2147483646LL || d < 1 || d > RNND_MAX_ROW || n < 0 || n > 2147483646LL) return RNND_ERR_BAD_SHAPE;
    return RNND_OK;
}

extern "C" int rnnd_embed(const void *table, int64_t V, int32_t d, int dtype, const int32_t *ids, int64_t n, float scale,
                          void *out, int out_dtype, void *stream)
{
    const int rc = check_rows(V, d, n, dtype, out_dtype);
    if (rc) return rc;
    if (!table || (n && (!ids || !out))) return RNND_ERR_NULL;
    if ((uintptr_t)table % dt_size(dtype) || (uintptr_t)ids % 4 || (uintptr_t)out % dt_size(out_dtype)) return RNND_ERR_BAD_PARAM;
    if (!n) return RNND_OK;
#define RNND_F(A, B) launch_embed<A, B>(table, V, d, ids, n, scale, out, (hipStream_t)stream)
    RNND_FOR_TYPES(dtype, out_dtype, RNND_F)
#undef RNND_F
    return launched("rnnd_embed");
}

// ------------------------------------------------------------------------------------------------ tokens sorted by id
// Pairs (id, token), least significant digit first, up to SORT_BITS bits a pass, three launches each: every block counts its
// digits, a wavefront per digit makes the counts of the blocks offsets, every block places its tokens.  A block's order
// is kept (stable) because its wavefronts number equal digits lane by lane, with a ballot per bit.  An id that is no row
// sorts as V, behind all rows.
#define SORT_BITS 10
#define SORT_DIGITS (1 << SORT_BITS)
#define SORT_THREADS 512
#define SORT_WAVES (SORT_THREADS / 64)
#define SORT_ITEMS 4
#define SORT_TILE (SORT_THREADS * SORT_ITEMS)
#define SORT_SMALL 4096     // up to here every token counts the tokens before it: one launch

struct SortPass {
    const int *ids;             // first pass: the caller's ids; else null
    const uint2 *in;            // (key, token)
    uint2 *out;
    u32 *hist;                  // [digits][blocks]
    u32 *totals;                // [digits]
    unsigned char *named;       // first pass: set to 1 for every row that an id names (may be null)
    u32 n, V, blocks;
    int shift, bits;
};

__device__ __forceinline__ u32 id_key(int id, u32 V) { return (u32)id < V ? (u32)id : V; }

__global__ __launch_bounds__(SORT_THREADS) void k_sort_count(SortPass s)
{
    __shared__ u32 count[SORT_DIGITS];
    const u32 digits = 1u << s.bits;
    for (u32 i = threadIdx.x; i < digits; i += SORT_THREADS) count[i] = 0;
    __syncthreads();
    const u32 base = blockIdx.x * SORT_TILE;
#pragma unroll
    for (int i = 0; i < SORT_ITEMS; ++i) {
        const u32 t = base + i * SORT_THREADS + threadIdx.x;
        if (t >= s.n) continue;
        const u32 key = s.ids ? id_key(s.ids[t], s.V) : s.in[t].x;
        if (s.named && key < s.V) s.named[key] = 1;
        atomicAdd(&count[(key >> s.shift) & (digits - 1)], 1u);
    }
    __syncthreads();
    for (u32 i = threadIdx.x; i < digits; i += SORT_THREADS) s.hist[(size_t)i * s.blocks + blockIdx.x] = count[i];
}

__device__ __forceinline__ u32 wave_inclusive(u32 v, int lane)
{
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
        const u32 o = __shfl_up(v, k);
        if (lane >= k) v += o;
    }
    return v;
}

// one wavefront per digit: exclusive sums of its counts over the blocks
__global__ __launch_bounds__(64) void k_sort_offsets(SortPass s)
{
    const int lane = threadIdx.x;
    u32 *h = s.hist + (size_t)blockIdx.x * s.blocks;
    u32 sum = 0;
    for (u32 b = 0; b < s.blocks; b += 64) {
        const u32 v = b + lane < s.blocks ? h[b + lane] : 0;
        const u32 inc = wave_inclusive(v, lane);
        if (b + lane < s.blocks) h[b + lane] = sum + inc - v;
        sum += __shfl(inc, 63);
    }
    if (lane == 0) s.totals[blockIdx.x] = sum;
}

__global__ __launch_bounds__(SORT_THREADS) void k_sort_place(SortPass s)
{
    constexpr int PER = SORT_DIGITS / SORT_THREADS;     // digits of a thread
    __shared__ u32 count[SORT_WAVES][SORT_DIGITS];
    __shared__ u32 wave_total[SORT_WAVES];
    const u32 digits = 1u << s.bits;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (u32 i = threadIdx.x; i < SORT_WAVES * SORT_DIGITS; i += SORT_THREADS) (&count[0][0])[i] = 0;
    // a wavefront owns SORT_ITEMS * 64 neighbouring tokens, so that its order is the order of the input
    const u32 base = blockIdx.x * SORT_TILE + wave * (64 * SORT_ITEMS);
    uint2 item[SORT_ITEMS];
    u32 rank[SORT_ITEMS];
#pragma unroll
    for (int i = 0; i < SORT_ITEMS; ++i) {
        const u32 t = base + i * 64 + lane;
        item[i] = make_uint2(0, 0);
        if (t < s.n) item[i] = s.ids ? make_uint2(id_key(s.ids[t], s.V), t) : s.in[t];
    }
    // where each digit starts: exclusive sums of the totals, and of this block's counts
    u32 first[PER], mine = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const u32 digit = threadIdx.x * PER + k;
        first[k] = mine;
        mine += digit < digits ? s.totals[digit] : 0;
    }
    const u32 inc = wave_inclusive(mine, lane);
    if (lane == 63) wave_total[wave] = inc;
    __syncthreads();
    u32 before_waves = inc - mine;
    for (int w = 0; w < wave; ++w) before_waves += wave_total[w];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const u32 digit = threadIdx.x * PER + k;
        first[k] += before_waves + (digit < digits ? s.hist[(size_t)digit * s.blocks + blockIdx.x] : 0);
    }
#pragma unroll
    for (int i = 0; i < SORT_ITEMS; ++i) {
        const bool on = base + i * 64 + lane < s.n;
        const u32 digit = (item[i].x >> s.shift) & (digits - 1);
        u64 same = __ballot(on);
        for (int b = 0; b < s.bits; ++b) {
            const bool bit = digit >> b & 1;
            const u64 set = __ballot(bit);
            same &= bit ? set : ~set;
        }
        const u32 ahead = __popcll(same & lanes_below(lane));
        u32 before = 0;
        if (on) before = count[wave][digit];
        wave_sync();
        if (on && ahead == 0) count[wave][digit] = before + __popcll(same);
        wave_sync();
        rank[i] = before + ahead;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        u32 at = first[k];
        for (int w = 0; w < SORT_WAVES; ++w) {
            const u32 n = count[w][threadIdx.x * PER + k];
            count[w][threadIdx.x * PER + k] = at;
            at += n;
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < SORT_ITEMS; ++i)
        if (base + i * 64 + lane < s.n) s.out[count[wave][(item[i].x >> s.shift) & (digits - 1)] + rank[i]] = item[i];
}

// Few tokens, one launch: 32 lanes per token count the tokens that sort before it -- those of a smaller key, and those before it
// of the same.  Blocks behind the first token_blocks clear the whole gradient meanwhile: its 16-byte words, and what lies before
// and behind them.
__global__ __launch_bounds__(256) void k_sort_small(const int *__restrict__ ids, u32 n, u32 V, uint2 *__restrict__ out, u32 *hot,
                                                    u32 token_blocks, uint4 *words, size_t n_words, unsigned char *head, u32 head_bytes,
                                                    unsigned char *tail, u32 tail_bytes)
{
    __shared__ u32 keys[SORT_SMALL];
    if (blockIdx.x >= token_blocks) {
        const u32 b = blockIdx.x - token_blocks, blocks = gridDim.x - token_blocks;
        for (size_t i = (size_t)b * 256 + threadIdx.x; i < n_words; i += (size_t)blocks * 256) words[i] = make_uint4(0, 0, 0, 0);
        if (b == 0 && threadIdx.x < head_bytes) head[threadIdx.x] = 0;
        if (b == 0 && threadIdx.x < tail_bytes) tail[threadIdx.x] = 0;
        return;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) *hot = 0;
    for (u32 t = threadIdx.x; t < n; t += 256) keys[t] = id_key(ids[t], V);
    __syncthreads();
    const u32 t = blockIdx.x * 8 + (threadIdx.x >> 5), sub = threadIdx.x & 31;
    const u32 key = t < n ? keys[t] : 0;
    u32 before = 0;
    for (u32 j = sub; j < n; j += 32) before += keys[j] < key + (j < t);
#pragma unroll
    for (int k = 16; k; k >>= 1) before += __shfl_xor(before, k);
    if (t < n && sub == 0) out[before] = make_uint2(key, t);
}

// ------------------------------------------------------------------------------------------------ gradient
// The sorted tokens are cut into chunks.  A lane takes VEC coordinates of a chunk (no lane needs another, so they are counted
// through, whatever the length of a row), and sums the rows of one id after the other.  An id whose tokens end at most one chunk behind the chunk they start in is summed by
// that chunk's lanes alone (they read on, and the next chunk's leave them out).  A longer one -- words as frequent as "the" --
// leaves one partial sum per chunk, which k_grad_join adds in order, a whole block for each such id and slab.
#define GRAD_UNROLL 8       // divides every chunk
#define GRAD_SLOTS 2        // partial sums of a chunk: 0 = of an id that started before it, 1 = of the id that goes on after it
#define JOIN_THREADS 512

struct GradPar {
    const void *dout;
    const uint2 *item;          // sorted (key, token)
    void *grad;
    float *partial;             // [chunks][GRAD_SLOTS][d]
    u32 *hot;                   // [0] how many, [1 ..] chunks in which a long id starts
    const unsigned char *named; // [V] whether a row is named (the others are cleared here)
    u32 n, V, chunk, chunks, pieces, slabs, reduce_blocks, clear_rows;
    int accumulate;
    float scale;
};

template <int GT, int VEC>
__device__ __forceinline__ void grad_write(const GradPar &g, u32 id, u32 piece, float (&acc)[VEC])
{
    const u64 at = ((u64)id * g.pieces + piece) * VEC;
#pragma unroll
    for (int k = 0; k < VEC; ++k) acc[k] *= g.scale;
    if (g.accumulate) {
        float old[VEC];
        unpack<GT, VEC>(load_pack<GT, VEC>(g.grad, at), old);
#pragma unroll
        for (int k = 0; k < VEC; ++k) acc[k] += old[k];
    }
    store_pack<GT, VEC>(g.grad, at, acc);
}

template <int DT, int GT, int VEC>
__global__ __launch_bounds__(256) void k_grad_reduce(GradPar g)
{
    if (blockIdx.x >= g.reduce_blocks) {        // the other blocks clear the rows that no token names, clear_rows each
        const float zero[VEC] = {};
        const u64 v0 = (u64)(blockIdx.x - g.reduce_blocks) * g.clear_rows;
        const u32 rows = (u32)(g.V - v0 < g.clear_rows ? g.V - v0 : g.clear_rows);
        for (u32 i = threadIdx.x; i < rows * g.pieces; i += 256) {
            const u32 r = i / g.pieces;
            if (!g.named[v0 + r]) store_pack<GT, VEC>(g.grad, (v0 * g.pieces + i) * VEC, zero);
        }
        return;
    }
    const u64 flat = (u64)blockIdx.x * 256 + threadIdx.x;
    const u32 c = (u32)(flat / g.pieces), piece = (u32)(flat - (u64)c * g.pieces);
    if (c >= g.chunks) return;
    const u64 begin64 = (u64)c * g.chunk;
    const u32 begin = (u32)begin64, end = g.n - begin < g.chunk ? g.n : begin + g.chunk, C = g.chunk;
    u32 id = g.item[begin].x;
    if (id >= g.V) return;
    const bool incoming = begin > 0 && g.item[begin - 1].x == id;
    // (sorted: the tokens of `id` end at or before position x if x is the end or holds another key)
    const bool skip = incoming && (begin - C == 0 || g.item[begin - C - 1].x != id) && ((u64)begin + C >= g.n || g.item[begin + C].x != id);
    bool first = incoming;          // still in the id that started before the chunk
    const u32 last = g.item[end - 1].x;
    const bool goes_on = end < g.n && g.item[end].x == last && last < g.V && !(incoming && last == id);
    const bool hot = goes_on && (u64)end + C < g.n && g.item[end + C].x == last;
    const u32 stop = goes_on && !hot ? (g.n - end < C ? g.n : end + C) : end;      // and no further than the key `last`

    float acc[VEC] = {};
    bool some = false;
    for (u32 t = begin; t < stop; t += GRAD_UNROLL) {
        uint2 it[GRAD_UNROLL];
        Pack<DT, VEC> row[GRAD_UNROLL];
#pragma unroll
        for (int i = 0; i < GRAD_UNROLL; ++i) it[i] = g.item[t + i < stop ? t + i : stop - 1];
#pragma unroll
        for (int i = 0; i < GRAD_UNROLL; ++i) {
            const u32 at = t + i;
            if (at >= stop || (at >= end && it[i].x != last)) it[i].x = 0xFFFFFFFFu;      // nothing there for this chunk
            if (it[i].x < g.V && !(skip && first && it[i].x == id)) row[i] = load_pack<DT, VEC>(g.dout, ((u64)it[i].y * g.pieces + piece) * VEC);
        }
        bool done = false;
#pragma unroll
        for (int i = 0; i < GRAD_UNROLL; ++i) {
            if (done) break;
            if (it[i].x != id) {
                if (some) {
                    if (first) store_pack<DT_F32, VEC>(g.partial, ((u64)c * GRAD_SLOTS * g.pieces + piece) * VEC, acc);
                    else grad_write<GT, VEC>(g, id, piece, acc);
                }
#pragma unroll
                for (int k = 0; k < VEC; ++k) acc[k] = 0.0f;
                some = false;
                first = false;
                id = it[i].x;
                if (id >= g.V) { done = true; break; }
            }
            if (skip && first) continue;
            float x[VEC];
            unpack<DT, VEC>(row[i], x);
#pragma unroll
            for (int k = 0; k < VEC; ++k) acc[k] += x[k];
            some = true;
        }
        if (done) break;
    }
    if (!some) return;
    if (first || hot) {
        store_pack<DT_F32, VEC>(g.partial, (((u64)c * GRAD_SLOTS + (first ? 0 : 1)) * g.pieces + piece) * VEC, acc);
        if (!first && piece == 0) g.hot[1 + atomicAdd(&g.hot[0], 1u)] = c;
    } else
        grad_write<GT, VEC>(g, id, piece, acc);
}

// One block per long id and slab: its groups take every (JOIN_THREADS / G)-th partial sum, four at a time, and their sums are added
// in the groups' order.
template <int GT, int VEC, int G>
__global__ __launch_bounds__(JOIN_THREADS) void k_grad_join(GradPar g)
{
    constexpr u32 groups = JOIN_THREADS / G;
    __shared__ float part[groups][G * VEC];
    const u32 lane = threadIdx.x % G, group = threadIdx.x / G;
    const u32 work = g.hot[0] * g.slabs;
    for (u32 at = blockIdx.x; at < work; at += gridDim.x) {
        const u32 c = g.hot[1 + at / g.slabs], piece = at % g.slabs * G + lane;
        const u32 id = g.item[(u64)(c + 1) * g.chunk - 1].x;
        u32 lo = c + 1, hi = (g.n - 1) / g.chunk;      // the last chunk whose first token is of `id`: a long id fills c + 1
        while (lo < hi) {
            const u32 mid = lo + (hi - lo + 1) / 2;
            if (g.item[(u64)mid * g.chunk].x == id) lo = mid;
            else hi = mid - 1;
        }
        const u32 chunks = lo - c + 1;
        float acc[VEC] = {};
        if (piece < g.pieces)
            for (u32 j0 = group; j0 < chunks; j0 += 4 * groups) {
                Pack<DT_F32, VEC> p[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const u32 j = j0 + u * groups;
                    if (j < chunks) p[u] = load_pack<DT_F32, VEC>(g.partial, (((u64)(c + j) * GRAD_SLOTS + (j == 0 ? 1 : 0)) * g.pieces + piece) * VEC);
                }
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (j0 + u * groups < chunks)
#pragma unroll
                        for (int k = 0; k < VEC; ++k) acc[k] += p[u].v[k];
            }
#pragma unroll
        for (int k = 0; k < VEC; ++k) part[group][lane * VEC + k] = acc[k];
        __syncthreads();
        if (group == 0 && piece < g.pieces) {
            const u32 most = groups < chunks ? groups : chunks;
            for (u32 j = 1; j < most; ++j)
#pragma unroll
                for (int k = 0; k < VEC; ++k) acc[k] += part[j][lane * VEC + k];
            grad_write<GT, VEC>(g, id, piece, acc);
        }
        __syncthreads();
    }
}

__global__ void k_grad_clear(u32 *p, size_t words)
{
    for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < words; i += (size_t)gridDim.x * blockDim.x) p[i] = 0;
}

struct GradPlan {
    u32 chunk, chunks, blocks;
    int passes, bits;
    size_t o_item[2], o_hist, o_totals, o_partial, o_hot, o_named, bytes;
};

static GradPlan grad_plan(int64_t n, int d, int64_t V)
{
    GradPlan p = {};
    // Long chunks leave fewer partial sums; short calls need chunks short enough to occupy the GPU: two wavefronts per SIMD, of about
    // 256 coordinates each.
    p.chunk = 128;
    while (p.chunk > 8 && n / p.chunk * ((d + 255) / 256) < 4096) p.chunk >>= 1;
    p.chunks = (u32)((n + p.chunk - 1) / p.chunk);
    p.blocks = (u32)((n + SORT_TILE - 1) / SORT_TILE);
    int bits = 1;
    while ((V >> bits) != 0) ++bits;          // keys 0 .. V
    p.passes = n <= SORT_SMALL ? 0 : (bits + SORT_BITS - 1) / SORT_BITS;
    p.bits = p.passes ? (bits + p.passes - 1) / p.passes : 0;
    size_t off = 0;
    auto take = [&](size_t b) { const size_t o = off; off += ws_align(b); return o; };
    for (int i = 0; i < 2; ++i) p.o_item[i] = take(i && !p.passes ? 0 : (size_t)n * 8);
    p.o_hist = take(p.passes ? (size_t)SORT_DIGITS * p.blocks * 4 : 0);
    p.o_totals = take(p.passes ? SORT_DIGITS * 4 : 0);
    p.o_partial = take((size_t)p.chunks * GRAD_SLOTS * d * 4);
    p.o_named = take(p.passes ? (size_t)V : 0);
    p.o_hot = take((size_t)(p.chunks + 1) * 4);       // (right behind `named`: its first word is cleared with it)
    p.bytes = off;
    return p;
}

extern "C" int rnnd_embed_grad_workspace(int64_t n, int32_t d, int64_t V, size_t *bytes)
{
    const int rc = check_rows(V, d, n, RNND_F32, RNND_F32);
    if (rc) return rc;
    if (!bytes) return RNND_ERR_NULL;
    *bytes = grad_plan(n, d, V).bytes;
    return RNND_OK;
}

template <int GT, int VEC, int G>
static void launch_join(GradPar &g, hipStream_t st)
{
    g.slabs = (g.pieces + G - 1) / G;
    const u64 units = (u64)g.chunks * g.slabs;
    hipLaunchKernelGGL((k_grad_join<GT, VEC, G>), dim3((u32)(units < 1024 ? units : 1024)), dim3(JOIN_THREADS), 0, st, g);
}
template <int DT, int GT, int VEC>
static void launch_grad_vec(GradPar &g, int d, bool clear, hipStream_t st)
{
    g.pieces = d / VEC;
    g.reduce_blocks = (u32)(((u64)g.chunks * g.pieces + 255) / 256);
    g.clear_rows = 2048 / g.pieces > 1 ? 2048 / g.pieces : 1;
    while (clear && (u64)g.V > (u64)g.clear_rows << 30) g.clear_rows <<= 1;
    const u32 clear_blocks = clear ? (g.V + g.clear_rows - 1) / g.clear_rows : 0;
    hipLaunchKernelGGL((k_grad_reduce<DT, GT, VEC>), dim3(g.reduce_blocks + clear_blocks), dim3(256), 0, st, g);
    if (g.chunks <= 2) return;      // no id of more than two chunks' tokens
    if (g.pieces <= 8) launch_join<GT, VEC, 8>(g, st);
    else if (g.pieces <= 16) launch_join<GT, VEC, 16>(g, st);
    else if (g.pieces <= 32) launch_join<GT, VEC, 32>(g, st);
    else launch_join<GT, VEC, 64>(g, st);
}
template <int DT, int GT>
static void launch_grad(GradPar &g, int d, bool clear, hipStream_t st)
{
    const int vec = row_vec(d, g.dout, dt_size(DT), g.grad, dt_size(GT));
    if constexpr (DT != DT_F32)
        if (vec == 8) return launch_grad_vec<DT, GT, 8>(g, d, clear, st);
    if (vec >= 4) launch_grad_vec<DT, GT, 4>(g, d, clear, st);
    else if (vec == 2) launch_grad_vec<DT, GT, 2>(g, d, clear, st);
    else launch_grad_vec<DT, GT, 1>(g, d, clear, st);
}

extern "C" int rnnd_embed_grad(const void *dout, int dtype, const int32_t *ids, int64_t n, int32_t d, float scale, int64_t V,
                               void *grad, int grad_dtype, int accumulate, void *workspace, size_t workspace_bytes, void *stream)
{
    const int rc = check_rows(V, d, n, dtype, grad_dtype);
    if (rc) return rc;
    if (!grad || (n && (!dout || !ids))) return RNND_ERR_NULL;
    if (accumulate != 0 && accumulate != 1) return RNND_ERR_BAD_PARAM;
    if ((uintptr_t)dout % dt_size(dtype) || (uintptr_t)ids % 4 || (uintptr_t)grad % dt_size(grad_dtype)) return RNND_ERR_BAD_PARAM;
    if (!n && accumulate) return RNND_OK;
    const GradPlan p = grad_plan(n, d, V);
    if (!workspace) return RNND_ERR_NULL;
    if ((uintptr_t)workspace % 16) return RNND_ERR_BAD_PARAM;
    if (workspace_bytes < p.bytes) return RNND_ERR_SCRATCH;
    hipStream_t st = (hipStream_t)stream;
    char *w = (char *)workspace;
    uint2 *item[2] = {(uint2 *)(w + p.o_item[0]), (uint2 *)(w + p.o_item[1])};
    u32 *hot = (u32 *)(w + p.o_hot);
    unsigned char *named = (unsigned char *)(w + p.o_named);
    int at = 0;
    if (!p.passes) {
        const size_t bytes = accumulate ? 0 : (size_t)V * d * dt_size(grad_dtype);
        size_t head = (16 - (uintptr_t)grad % 16) % 16;
        if (head > bytes) head = bytes;
        const size_t words = (bytes - head) / 16;
        const u32 tail = (u32)(bytes - head - words * 16);
        const u32 token_blocks = (u32)((n + 7) / 8) + (n ? 0 : 1), clear_blocks = accumulate ? 0 : (u32)(words / 1024 < 2048 ? words / 1024 + 1 : 2048);
        hipLaunchKernelGGL(k_sort_small, dim3(token_blocks + clear_blocks), dim3(256), 0, st, ids, (u32)n, (u32)V, item[0], hot, token_blocks,
                           (uint4 *)((char *)grad + head), words, (unsigned char *)grad, (u32)head, (unsigned char *)grad + head + words * 16, tail);
    } else {
        // the number of long ids, and (all rows written) which rows are named
        const size_t from = accumulate ? p.o_hot : p.o_named, words = (p.o_hot + 4 - from) / 4;
        const size_t blocks = (words + 1023) / 1024;
        hipLaunchKernelGGL(k_grad_clear, dim3((u32)(blocks < 2048 ? blocks : 2048)), dim3(256), 0, st, (u32 *)(w + from), words);
        at = 1;
        for (int i = 0; i < p.passes; ++i) {
            SortPass s;
            s.ids = i ? nullptr : ids;
            s.in = item[at];
            at ^= 1;
            s.out = item[at];
            s.hist = (u32 *)(w + p.o_hist);
            s.totals = (u32 *)(w + p.o_totals);
            s.named = i || accumulate ? nullptr : named;
            s.n = (u32)n;
            s.V = (u32)V;
            s.blocks = p.blocks;
            s.shift = i * p.bits;
            s.bits = p.bits;
            hipLaunchKernelGGL(k_sort_count, dim3(p.blocks), dim3(SORT_THREADS), 0, st, s);
            hipLaunchKernelGGL(k_sort_offsets, dim3(1u << p.bits), dim3(64), 0, st, s);
            hipLaunchKernelGGL(k_sort_place, dim3(p.blocks), dim3(SORT_THREADS), 0, st, s);
        }
    }
    if (!n) return launched("rnnd_embed_grad");
    GradPar g = {};
    g.dout = dout;
    g.item = item[at];
    g.grad = grad;
    g.partial = (float *)(w + p.o_partial);
    g.hot = hot;
    g.named = named;
    g.n = (u32)n;
    g.V = (u32)V;
    g.chunk = p.chunk;
    g.chunks = p.chunks;
    g.accumulate = accumulate;
    g.scale = scale;
#define RNND_F(A, B) launch_grad<A, B>(g, d, !accumulate && p.passes, st)
    RNND_FOR_TYPES(dtype, grad_dtype, RNND_F)
#undef RNND_F
    return launched("rnnd_embed_grad");
}
