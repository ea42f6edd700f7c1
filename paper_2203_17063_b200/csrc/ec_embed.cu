// Embedding lookup with scaling, and its gradient by sorted tokens.
//
// Lookup: out[t] = scale * table[token[t]].  A gather of whole rows: bound by memory (distinct rows read once, T rows
// written), nothing to reuse but L2.
//
// Gradient: grad[v] = scale * sum of dout[t] over token[t] = v.  The tokens are sorted (stable, so a row's positions stay in
// ascending order), then the sorted tokens and the table's rows are walked together as one path of T + V steps: a token
// step adds a row of dout to the running sum, a row step writes the sum out and starts the next.  Token p of the sorted order
// is step p + key[p] of the path, so the path is cut into equal shares by a search for the share's first step; every row of
// dout is read once, every row of grad written once, and a token that makes up a tenth of the text is spread over as many
// shares as it takes.  A row that crosses the border of a share leaves partial sums in fp32, joined in share order by a second
// small kernel: no atomics on values, the same bits every run.

#include "ec_vec.cuh"

namespace ec {
namespace {

// ---- lookup ------------------------------------------------------------------------------------------------------

constexpr int LK_THREADS = 256;
constexpr int LK_INFLIGHT = 4;          // vectors a lane has in flight

template <class IDX, class TI, class TO, int W>
__global__ void __launch_bounds__(LK_THREADS)
lookup_kernel(const TI* __restrict__ table, size_t table_stride, size_t V, size_t D, const IDX* __restrict__ tokens, size_t T,
              float scale, TO* __restrict__ out, size_t out_stride) {
    const int lane = threadIdx.x & 31;
    const size_t t = (size_t)blockIdx.x * (LK_THREADS / 32) + (threadIdx.x >> 5);
    if (t >= T) return;
    const long long tok = (long long)tokens[t];
    const bool there = tok >= 0 && (unsigned long long)tok < V;
    const TI* row = table + (there ? (size_t)tok : 0) * table_stride;
    TO* dst = out + t * out_stride;
    for (size_t c0 = (size_t)blockIdx.y * (32 * W * LK_INFLIGHT); c0 < D; c0 += (size_t)gridDim.y * (32 * W * LK_INFLIGHT)) {
        raw_vec<TI, W> v[LK_INFLIGHT];
#pragma unroll
        for (int q = 0; q < LK_INFLIGHT; ++q) {
            const size_t c = c0 + (size_t)(q * 32 + lane) * W;
            if (there && c < D) v[q] = load_raw<TI, W>(row + c);
        }
#pragma unroll
        for (int q = 0; q < LK_INFLIGHT; ++q) {
            const size_t c = c0 + (size_t)(q * 32 + lane) * W;
            if (c >= D) continue;
            float x[W];
            if (there) {
                unpack<TI, W>(v[q], x);
#pragma unroll
                for (int e = 0; e < W; ++e) x[e] *= scale;
            } else {
#pragma unroll
                for (int e = 0; e < W; ++e) x[e] = 0.0f;
            }
            store_vec<TO, W>(dst + c, x);
        }
    }
}

template <class IDX, class TI, class TO>
int launch_lookup(const void* table, size_t V, size_t D, size_t ts, const void* tokens, size_t T, float scale, void* out,
                  size_t os, cudaStream_t st) {
    constexpr int W = sizeof(TI) == 2 ? 8 : 4;
    const bool vec = D % W == 0 && rows_aligned(table, ts, sizeof(TI), W) && rows_aligned(out, os, sizeof(TO), W);
    const unsigned gx = (unsigned)((T + LK_THREADS / 32 - 1) / (LK_THREADS / 32));
    const size_t per = 32 * (size_t)(vec ? W : 1) * LK_INFLIGHT, pieces = (D + per - 1) / per;
    const dim3 grid(gx, (unsigned)(pieces < 64 ? pieces : 64));
    if (vec)
        lookup_kernel<IDX, TI, TO, W><<<grid, LK_THREADS, 0, st>>>((const TI*)table, ts, V, D, (const IDX*)tokens, T, scale, (TO*)out, os);
    else
        lookup_kernel<IDX, TI, TO, 1><<<grid, LK_THREADS, 0, st>>>((const TI*)table, ts, V, D, (const IDX*)tokens, T, scale, (TO*)out, os);
    EC_CUDA(cudaGetLastError());
    return EC_OK;
}

// ---- sorting the tokens ------------------------------------------------------------------------------------------
// Least-significant-digit radix sort of (key, position), 9 bits a pass at most: count per tile, scan over the tiles of every
// digit, scatter.  key = token, or V for a token that gives nothing (it sorts behind every row).

constexpr int SORT_THREADS = 256, SORT_WARPS = SORT_THREADS / 32, SORT_ITEMS = 8, SORT_TILE = SORT_THREADS * SORT_ITEMS;
constexpr int SORT_BITS = 9, SORT_BINS = 1 << SORT_BITS;

template <class IDX>
__device__ __forceinline__ uint32_t token_key(const IDX* tokens, size_t t, uint32_t V, long long skip) {
    const long long tok = (long long)tokens[t];
    return tok < 0 || tok >= (long long)V || tok == skip ? V : (uint32_t)tok;
}

struct SortArgs {
    const void* tokens;             // first pass
    const uint32_t* keys_in; const uint32_t* pos_in;
    uint32_t* keys_out; uint32_t* pos_out;
    uint32_t* hist;                 // [bins][tiles]
    uint32_t* totals;               // [bins]
    uint32_t* joins;                // number of joins: cleared here for the kernels that follow
    uint32_t T, V, tiles;
    long long skip;
    int shift, bins;
};

template <class IDX, bool FIRST>
__device__ __forceinline__ uint32_t sort_load_key(const SortArgs& a, uint32_t i) {
    if (FIRST) return token_key(static_cast<const IDX*>(a.tokens), i, a.V, a.skip);
    return a.keys_in[i];
}

template <class IDX, bool FIRST>
__global__ void __launch_bounds__(SORT_THREADS) sort_count_kernel(const SortArgs a) {
    grid_dependency_wait();
    __shared__ uint32_t s_n[SORT_BINS];
    for (int d = threadIdx.x; d < a.bins; d += SORT_THREADS) s_n[d] = 0;
    __syncthreads();
    const uint32_t base = blockIdx.x * SORT_TILE;
#pragma unroll
    for (int q = 0; q < SORT_ITEMS; ++q) {
        const uint32_t i = base + q * SORT_THREADS + threadIdx.x;
        if (i < a.T) atomicAdd(&s_n[(sort_load_key<IDX, FIRST>(a, i) >> a.shift) & (a.bins - 1)], 1u);   // (integers: order is free)
    }
    __syncthreads();
    for (int d = threadIdx.x; d < a.bins; d += SORT_THREADS) a.hist[(size_t)d * a.tiles + blockIdx.x] = s_n[d];
    if (FIRST && blockIdx.x == 0 && threadIdx.x == 0) *a.joins = 0;
}

__device__ __forceinline__ uint32_t warp_inclusive(uint32_t x, int lane) {
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
    }
    return x;
}

// one warp per digit: exclusive scan of its counts over the tiles, and their total
__global__ void __launch_bounds__(SORT_THREADS) sort_scan_kernel(const SortArgs a) {
    grid_dependency_wait();
    const int lane = threadIdx.x & 31, d = blockIdx.x * SORT_WARPS + (threadIdx.x >> 5);
    if (d >= a.bins) return;
    uint32_t* h = a.hist + (size_t)d * a.tiles;
    uint32_t sum = 0;
    for (uint32_t b = 0; b < a.tiles; b += 32) {
        const uint32_t x = b + lane < a.tiles ? h[b + lane] : 0u, in = warp_inclusive(x, lane);
        if (b + lane < a.tiles) h[b + lane] = sum + in - x;
        sum += __shfl_sync(0xffffffffu, in, 31);
    }
    if (lane == 0) a.totals[d] = sum;
}

// s_out[d] = exclusive scan of in[d] over the bins (at most 512, two per thread of 256)
__device__ __forceinline__ void block_scan_bins(const uint32_t* in, uint32_t* s_out, uint32_t* s_warp, int bins) {
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const uint32_t x0 = 2 * tid < bins ? in[2 * tid] : 0u, x1 = 2 * tid + 1 < bins ? in[2 * tid + 1] : 0u;
    const uint32_t inc = warp_inclusive(x0 + x1, lane);
    if (lane == 31) s_warp[w] = inc;
    __syncthreads();
    uint32_t before = 0;
    for (int q = 0; q < w; ++q) before += s_warp[q];
    if (2 * tid < bins) s_out[2 * tid] = before + inc - x0 - x1;
    if (2 * tid + 1 < bins) s_out[2 * tid + 1] = before + inc - x1;
    __syncthreads();
}

template <class IDX, bool FIRST>
__global__ void __launch_bounds__(SORT_THREADS) sort_scatter_kernel(const SortArgs a) {
    grid_dependency_wait();
    __shared__ uint32_t s_base[SORT_BINS], s_scan[SORT_WARPS];
    __shared__ uint32_t s_n[SORT_WARPS][SORT_BINS];
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    for (int d = tid; d < SORT_WARPS * SORT_BINS; d += SORT_THREADS) (&s_n[0][0])[d] = 0;
    block_scan_bins(a.totals, s_base, s_scan, a.bins);
    // A warp owns 32 * SORT_ITEMS consecutive items; lane l of step q has item q * 32 + l, so (warp, step, lane) is their order.
    const uint32_t base = blockIdx.x * SORT_TILE + w * (32 * SORT_ITEMS) + lane;
    uint32_t key[SORT_ITEMS], pos[SORT_ITEMS], rank[SORT_ITEMS];
#pragma unroll
    for (int q = 0; q < SORT_ITEMS; ++q) {
        const uint32_t i = base + q * 32;
        key[q] = i < a.T ? sort_load_key<IDX, FIRST>(a, i) : 0xffffffffu;
        pos[q] = FIRST ? i : i < a.T ? a.pos_in[i] : 0u;
    }
#pragma unroll
    for (int q = 0; q < SORT_ITEMS; ++q) {
        const bool in = base + q * 32 < a.T;
        const uint32_t d = in ? (key[q] >> a.shift) & (a.bins - 1) : (uint32_t)a.bins;     // items past the end: a digit of their own
        const uint32_t same = __match_any_sync(0xffffffffu, d);
        const uint32_t below = __popc(same & ((1u << lane) - 1u));
        const uint32_t old = in ? s_n[w][d] : 0u;
        __syncwarp();
        if (in && below == 0) s_n[w][d] = old + __popc(same);
        __syncwarp();
        rank[q] = old + below;
    }
    __syncthreads();
    for (int d = tid; d < a.bins; d += SORT_THREADS) {
        uint32_t sum = s_base[d] + a.hist[(size_t)d * a.tiles + blockIdx.x];
        for (int q = 0; q < SORT_WARPS; ++q) {
            const uint32_t n = s_n[q][d];
            s_n[q][d] = sum;
            sum += n;
        }
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < SORT_ITEMS; ++q) {
        if (base + q * 32 >= a.T) continue;
        const uint32_t p = s_n[w][(key[q] >> a.shift) & (a.bins - 1)] + rank[q];
        a.keys_out[p] = key[q];
        a.pos_out[p] = pos[q];
    }
}

// ---- the walk ----------------------------------------------------------------------------------------------------

constexpr int GR_THREADS = 256;
constexpr int GR_INFLIGHT = 8;          // rows of dout a thread has in flight
constexpr int GR_MAX_SHARE = 64;
constexpr int GR_TOKENS = 1024;         // most path steps of a block

// How a call is cut: groups of G threads take shares of C path steps; a block holds GR_THREADS / G groups.
struct GradPlan {
    int W, G, C;                        // elements per thread, threads per group, steps per share
    unsigned shares, blocks, slices;    // shares = groups in all (a multiple of the groups of a block)
};

GradPlan grad_plan(size_t T, size_t V, size_t D, int W) {
    GradPlan p;
    p.W = W;
    const size_t lanes = (D + W - 1) / W;
    p.G = 8;
    while (p.G < GR_THREADS && (size_t)p.G < lanes) p.G *= 2;
    p.slices = (unsigned)((lanes + p.G - 1) / p.G);
    const unsigned groups = GR_THREADS / p.G;
    const size_t steps = T + V;
    p.C = GR_TOKENS / (int)groups < GR_MAX_SHARE ? GR_TOKENS / (int)groups : GR_MAX_SHARE;
    while (p.C > 8 && (steps / ((size_t)p.C * groups)) * p.slices < 148 * 8) p.C /= 2;
    p.blocks = (unsigned)((steps + (size_t)p.C * groups - 1) / ((size_t)p.C * groups));
    p.shares = p.blocks * groups;
    return p;
}

constexpr uint32_t NO_ROW = 0xffffffffu;

struct GradArgs {
    const uint32_t* keys; const uint32_t* pos;      // sorted tokens, their positions
    uint32_t* begins;                               // [shares] the row a share begins in the middle of, or NO_ROW
    float* head;                                    // [shares][D] sum of the share's part of the row it begins in, if it ends there
    float* tail;                                    // [shares][D] sum of the share's part of the row it ends in
    uint32_t* joins;                                // [0] number of rows to join, then (share of the row's end, row) pairs
    uint32_t T, V;
    size_t D, in_stride, out_stride;
    float scale;
    int G, C, accumulate;
};

// Number of sorted tokens p with p + key[p] < d: the tokens among the first d steps of the path.  One warp, 33 sections at a time.
__device__ __forceinline__ uint32_t path_search(const uint32_t* __restrict__ keys, uint32_t T, uint32_t V, uint32_t d, int lane) {
    uint32_t lo = d > V ? d - V : 0u, hi = d < T ? d : T;
    while (lo < hi) {
        const uint32_t step = (hi - lo + 31) / 32, p = lo + lane * step;
        const bool less = p < hi && p + keys[p] < d;
        const uint32_t n = __popc(__ballot_sync(0xffffffffu, less));
        if (n == 0) break;
        const uint32_t top = lo + n * step;
        lo = lo + (n - 1) * step + 1;
        hi = top < hi ? top : hi;
    }
    return lo;
}

template <class TO, int W>
__device__ __forceinline__ void write_row(TO* p, float (&acc)[W], float scale, bool add) {
    float x[W];
#pragma unroll
    for (int e = 0; e < W; ++e) x[e] = scale * acc[e] + 0.0f;      // (+0 for a row without tokens, whatever the scale's sign)
    if (add) {
        float old[W];
        if constexpr (sizeof(TO) * W > 16) {
            constexpr int H = W / 2;
            float a[H], b[H];
            load_vec<TO, H>(p, a);
            load_vec<TO, H>(p + H, b);
#pragma unroll
            for (int e = 0; e < H; ++e) { old[e] = a[e]; old[H + e] = b[e]; }
        } else {
            load_vec<TO, W>(p, old);
        }
#pragma unroll
        for (int e = 0; e < W; ++e) x[e] += old[e];
    }
    store_vec<TO, W>(p, x);
}

template <class TI, class TO, int W>
__global__ void __launch_bounds__(GR_THREADS) grad_walk_kernel(const GradArgs a, const TI* __restrict__ dout, TO* __restrict__ grad) {
    grid_dependency_wait();
    __shared__ uint32_t s_key[GR_TOKENS + 1], s_pos[GR_TOKENS];      // s_key[0]: the token before the block's first
    __shared__ uint32_t s_cut[2];
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const uint32_t groups = GR_THREADS / a.G, total = a.T + a.V;
    const uint32_t d0 = blockIdx.x * groups * a.C, d1 = d0 + groups * a.C < total ? d0 + groups * a.C : total;
    if (w < 2) {
        const uint32_t i = path_search(a.keys, a.T, a.V, w == 0 ? d0 : d1, lane);
        if (lane == 0) s_cut[w] = i;
    }
    __syncthreads();
    const uint32_t i0 = s_cut[0], n = s_cut[1] - i0;
    if (tid == 0) s_key[0] = i0 > 0 ? a.keys[i0 - 1] : 0xffffffffu;
    for (uint32_t q = tid; q < n; q += GR_THREADS) {
        s_key[q + 1] = a.keys[i0 + q];
        s_pos[q] = a.pos[i0 + q];
    }
    __syncthreads();

    const uint32_t g = tid / a.G;
    const uint32_t b = d0 + g * a.C < total ? d0 + g * a.C : total, e = b + a.C < total ? b + a.C : total;   // the share's steps
    uint32_t lo = 0, hi = n;
    while (lo < hi) {                                                // tokens of the block before the share
        const uint32_t m = (lo + hi) / 2;
        if (i0 + m + s_key[m + 1] < b) lo = m + 1; else hi = m;
    }
    uint32_t i = lo;
    hi = n;
    while (lo < hi) {
        const uint32_t m = (lo + hi) / 2;
        if (i0 + m + s_key[m + 1] < e) lo = m + 1; else hi = m;
    }
    const uint32_t i_end = lo;
    uint32_t j = b - (i0 + i);
    const uint32_t j_end = e - (i0 + i_end);
    const uint32_t share = blockIdx.x * groups + g;
    const bool inside = j < a.V && s_key[i] == j;                    // the row goes on from the share before
    const size_t c = ((size_t)blockIdx.y * a.G + (tid & (a.G - 1))) * W;
    const bool mine = c < a.D;
    const bool note = blockIdx.y == 0 && (tid & (a.G - 1)) == 0;
    if (note) a.begins[share] = inside ? j : NO_ROW;

    float acc[W];
#pragma unroll
    for (int x = 0; x < W; ++x) acc[x] = 0.0f;
    bool open = inside, first = inside;                              // the row has tokens; it began in an earlier share
    auto row_end = [&]() {
        if (first) {
            if (mine) store_vec<float, W>(a.head + (size_t)share * a.D + c, acc);
            if (note) {
                const uint32_t k = atomicAdd(a.joins, 1u);           // (the list's order does not matter: every row joins for itself)
                a.joins[1 + 2 * k] = share;
                a.joins[2 + 2 * k] = j;
            }
        } else if (mine && (open || !a.accumulate)) {
            write_row<TO, W>(grad + (size_t)j * a.out_stride + c, acc, a.scale, a.accumulate != 0);
        }
        ++j;
        open = first = false;
#pragma unroll
        for (int x = 0; x < W; ++x) acc[x] = 0.0f;
    };
    while (i < i_end) {
        raw_vec<TI, W> v[GR_INFLIGHT];
        const int cnt = i_end - i < GR_INFLIGHT ? (int)(i_end - i) : GR_INFLIGHT;
#pragma unroll
        for (int q = 0; q < GR_INFLIGHT; ++q)
            if (q < cnt && mine && s_key[i + q + 1] < a.V) v[q] = load_raw<TI, W>(dout + (size_t)s_pos[i + q] * a.in_stride + c);
#pragma unroll
        for (int q = 0; q < GR_INFLIGHT; ++q) {
            if (q < cnt) {
                const uint32_t k = s_key[i + q + 1];
                while (j < k) row_end();
                if (k < a.V) {
                    open = true;
                    if (mine) {
                        float x[W];
                        unpack<TI, W>(v[q], x);
#pragma unroll
                        for (int z = 0; z < W; ++z) acc[z] += x[z];
                    }
                }
            }
        }
        i += cnt;
    }
    while (j < j_end) row_end();
    if (open && mine) store_vec<float, W>(a.tail + (size_t)share * a.D + c, acc);
}

// ---- joining the rows that cross shares --------------------------------------------------------------------------
// Row j ends in share s and began in share f < s: its sum is tail[f] + ... + tail[s-1] + head[s].  A block takes 128 columns;
// its eight warps add up contiguous parts of the range, then the parts in order.

constexpr int JN_THREADS = 256, JN_WARPS = JN_THREADS / 32;

template <class TO>
__global__ void __launch_bounds__(JN_THREADS) grad_join_kernel(const GradArgs a, TO* __restrict__ grad) {
    grid_dependency_wait();
    __shared__ float s_part[JN_WARPS][128];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const uint32_t count = a.joins[0];
    for (uint32_t k = blockIdx.x; k < count; k += gridDim.x) {
        const uint32_t s = a.joins[1 + 2 * k], j = a.joins[2 + 2 * k];
        uint32_t f = s;                                              // first share: go back while a share begins inside this row
        for (;;) {
            const bool in = f >= (uint32_t)lane + 1 && a.begins[f - lane] == j;    // (share 0 begins in no row)
            const uint32_t run = __ballot_sync(0xffffffffu, in);
            const int ones = run == 0xffffffffu ? 32 : __ffs(~run) - 1;
            f -= ones;
            if (ones < 32) break;
        }
        const uint32_t n = s - f;                                    // tails f .. s-1
        const uint32_t p0 = f + (uint32_t)((unsigned long long)n * w / JN_WARPS), p1 = f + (uint32_t)((unsigned long long)n * (w + 1) / JN_WARPS);
        for (size_t c0 = (size_t)blockIdx.y * 128; c0 < a.D; c0 += (size_t)gridDim.y * 128) {
            float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
            for (uint32_t p = p0; p < p1; ++p) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const size_t c = c0 + q * 32 + lane;
                    if (c < a.D) x[q] += a.tail[(size_t)p * a.D + c];
                }
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) s_part[w][q * 32 + lane] = x[q];
            __syncthreads();
            const size_t c = c0 + threadIdx.x;
            if (threadIdx.x < 128 && c < a.D) {
                float sum[1] = {0.0f};
                for (int q = 0; q < JN_WARPS; ++q) sum[0] += s_part[q][threadIdx.x];
                sum[0] += a.head[(size_t)s * a.D + c];
                write_row<TO, 1>(grad + (size_t)j * a.out_stride + c, sum, a.scale, a.accumulate != 0);
            }
            __syncthreads();
        }
    }
}

// ---- host --------------------------------------------------------------------------------------------------------

struct GradLayout {
    size_t keys[2], pos[2], hist, totals, joins, begins, head, tail, total;
    uint32_t tiles;
    int passes, bits;
};
// The widest plan of the two (vector or element-wise rows) sizes the workspace.
void grad_layout(size_t T, size_t V, size_t D, GradLayout* L) {
    size_t off = 0;
    L->tiles = (uint32_t)((T + SORT_TILE - 1) / SORT_TILE);
    int nb = 1;
    while ((V >> nb) != 0) ++nb;                       // keys are 0 .. V
    L->passes = (nb + SORT_BITS - 1) / SORT_BITS;
    L->bits = (nb + L->passes - 1) / L->passes;
    for (int q = 0; q < 2; ++q) {
        L->keys[q] = off; off = align_up(off + T * 4, 256);
        L->pos[q] = off; off = align_up(off + T * 4, 256);
    }
    L->hist = off; off = align_up(off + (size_t)SORT_BINS * L->tiles * 4, 256);
    L->totals = off; off = align_up(off + SORT_BINS * 4, 256);
    size_t shares = 0;
    const int widths[3] = {1, 4, 8};
    for (int q = 0; q < 3; ++q) {
        const size_t s = grad_plan(T, V, D, widths[q]).shares;
        shares = s > shares ? s : shares;
    }
    L->joins = off; off = align_up(off + (1 + 2 * shares) * 4, 256);
    L->begins = off; off = align_up(off + shares * 4, 256);
    L->head = off; off = align_up(off + shares * D * 4, 256);
    L->tail = off; off = align_up(off + shares * D * 4, 256);
    L->total = off;
}

template <class IDX>
int sort_tokens(SortArgs a, const GradLayout& L, char* ws, cudaStream_t st) {
    a.bins = 1 << L.bits;
    for (int pass = 0; pass < L.passes; ++pass) {
        a.shift = pass * L.bits;
        const int src = (pass + 1) & 1, dst = pass & 1;
        a.keys_in = reinterpret_cast<const uint32_t*>(ws + L.keys[src]);
        a.pos_in = reinterpret_cast<const uint32_t*>(ws + L.pos[src]);
        a.keys_out = reinterpret_cast<uint32_t*>(ws + L.keys[dst]);
        a.pos_out = reinterpret_cast<uint32_t*>(ws + L.pos[dst]);
        if (pass == 0) EC_CUDA(launch_dependent(sort_count_kernel<IDX, true>, a.tiles, SORT_THREADS, 0, st, a));
        else EC_CUDA(launch_dependent(sort_count_kernel<IDX, false>, a.tiles, SORT_THREADS, 0, st, a));
        EC_CUDA(launch_dependent(sort_scan_kernel, (unsigned)((a.bins + SORT_WARPS - 1) / SORT_WARPS), SORT_THREADS, 0, st, a));
        if (pass == 0) EC_CUDA(launch_dependent(sort_scatter_kernel<IDX, true>, a.tiles, SORT_THREADS, 0, st, a));
        else EC_CUDA(launch_dependent(sort_scatter_kernel<IDX, false>, a.tiles, SORT_THREADS, 0, st, a));
    }
    return EC_OK;
}

template <class TI, class TO, int W>
int launch_walk(GradArgs a, const GradPlan& p, const void* dout, void* grad, cudaStream_t st) {
    a.G = p.G;
    a.C = p.C;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 1; cfg.stream = st;
    cfg.gridDim = dim3(p.blocks, p.slices); cfg.blockDim = dim3(GR_THREADS);
    EC_CUDA(cudaLaunchKernelEx(&cfg, grad_walk_kernel<TI, TO, W>, a, static_cast<const TI*>(dout), static_cast<TO*>(grad)));
    const size_t cols = (a.D + 127) / 128;
    cfg.gridDim = dim3(p.shares < 148 ? p.shares : 148, (unsigned)(cols < 16 ? cols : 16)); cfg.blockDim = dim3(JN_THREADS);
    EC_CUDA(cudaLaunchKernelEx(&cfg, grad_join_kernel<TO>, a, static_cast<TO*>(grad)));
    return EC_OK;
}

constexpr size_t EMBED_MAX = 0x7ffffffeull, EMBED_MAX_D = (size_t)1 << 24;

bool embed_sizes_ok(size_t T, size_t V, size_t D) { return V >= 1 && V <= EMBED_MAX && T <= EMBED_MAX && D >= 1 && D <= EMBED_MAX_D; }

}  // namespace
}  // namespace ec

using namespace ec;

extern "C" {

int ec_embed_lookup(const void* table, size_t V, size_t D, size_t table_stride, ec_dtype_t table_dtype, const void* tokens,
                    ec_index_t index, size_t T, float scale, void* out, size_t out_stride, ec_dtype_t out_dtype,
                    ec_stream_t stream) {
    if (!table || (T > 0 && (!tokens || !out)) || !embed_sizes_ok(T, V, D)) return EC_ERR_INVALID;
    if (table_stride < D || out_stride < D || (index != EC_INDEX_32 && index != EC_INDEX_64)) return EC_ERR_INVALID;
    if (!is_real_dtype(table_dtype) || !is_real_dtype(out_dtype)) return EC_ERR_UNSUPPORTED;
    if (T == 0) return EC_OK;
    return with_types(table_dtype, out_dtype, [&](auto ti, auto to) {
        using TI = decltype(ti); using TO = decltype(to);
        if (index == EC_INDEX_32) return launch_lookup<int32_t, TI, TO>(table, V, D, table_stride, tokens, T, scale, out, out_stride, stream);
        return launch_lookup<int64_t, TI, TO>(table, V, D, table_stride, tokens, T, scale, out, out_stride, stream);
    });
}

size_t ec_embed_grad_workspace_bytes(size_t T, size_t V, size_t D) {
    if (!embed_sizes_ok(T, V, D) || T + V > EMBED_MAX) return 0;
    GradLayout L;
    grad_layout(T, V, D, &L);
    return L.total;
}

int ec_embed_grad(const void* dout, size_t dout_stride, ec_dtype_t dout_dtype, const void* tokens, ec_index_t index, size_t T,
                  size_t V, size_t D, float scale, int64_t skip_token, int accumulate, void* grad, size_t grad_stride,
                  ec_dtype_t grad_dtype, void* workspace, size_t workspace_bytes, ec_stream_t stream) {
    if (!grad || (T > 0 && (!dout || !tokens)) || !embed_sizes_ok(T, V, D) || T + V > EMBED_MAX) return EC_ERR_INVALID;
    if (dout_stride < D || grad_stride < D || (index != EC_INDEX_32 && index != EC_INDEX_64)) return EC_ERR_INVALID;
    if (!is_real_dtype(dout_dtype) || !is_real_dtype(grad_dtype)) return EC_ERR_UNSUPPORTED;
    GradLayout L;
    grad_layout(T, V, D, &L);
    if (!workspace || workspace_bytes < L.total || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return EC_ERR_CAPACITY;
    if (T == 0 && accumulate) return EC_OK;
    char* ws = static_cast<char*>(workspace);
    const int last = (L.passes - 1) & 1;
    GradArgs a = {};
    a.keys = reinterpret_cast<const uint32_t*>(ws + L.keys[last]);
    a.pos = reinterpret_cast<const uint32_t*>(ws + L.pos[last]);
    a.joins = reinterpret_cast<uint32_t*>(ws + L.joins);
    a.begins = reinterpret_cast<uint32_t*>(ws + L.begins);
    a.head = reinterpret_cast<float*>(ws + L.head);
    a.tail = reinterpret_cast<float*>(ws + L.tail);
    a.T = (uint32_t)T; a.V = (uint32_t)V; a.D = D;
    a.in_stride = dout_stride; a.out_stride = grad_stride;
    a.scale = scale; a.accumulate = accumulate != 0;
    if (T > 0) {
        SortArgs s = {};
        s.tokens = tokens;
        s.hist = reinterpret_cast<uint32_t*>(ws + L.hist);
        s.totals = reinterpret_cast<uint32_t*>(ws + L.totals);
        s.joins = a.joins;
        s.T = a.T; s.V = a.V; s.tiles = L.tiles;
        s.skip = skip_token;
        const int rc = index == EC_INDEX_32 ? sort_tokens<int32_t>(s, L, ws, stream) : sort_tokens<int64_t>(s, L, ws, stream);
        if (rc != EC_OK) return rc;
    } else {
        EC_CUDA(cudaMemsetAsync(a.joins, 0, 4, stream));
    }
    return with_types(dout_dtype, grad_dtype, [&](auto ti, auto to) {
        using TI = decltype(ti); using TO = decltype(to);
        constexpr int W = sizeof(TI) == 2 ? 8 : 4;
        const bool vec = D % W == 0 && rows_aligned(dout, dout_stride, sizeof(TI), W) && rows_aligned(grad, grad_stride, sizeof(TO), W);
        if (vec) return launch_walk<TI, TO, W>(a, grad_plan(T, V, D, W), dout, grad, stream);
        return launch_walk<TI, TO, 1>(a, grad_plan(T, V, D, 1), dout, grad, stream);
    });
}

}  // extern "C"
