// Embedding lookup with scaling, and its gradient by sorted tokens.
//
// Lookup: out[t] = scale * table[token[t]].  A gather of whole rows: bound by memory (distinct rows read once, T rows
// written), nothing to reuse but L2.
//
// Gradient: grad[v] = scale * sum of dout[t] over token[t] = v.  The tokens are sorted (stable, so a row's positions stay in
// ascending order), then the sorted tokens and the table's rows are laid out as one path of T + V steps: a token step reads a
// row of dout, a row step writes a row of grad.  Token p of the sorted order is step p + key[p] of the path, so the path is
// cut into equal stretches, a block each, by a search for a stretch's first step; every row of dout is read once, every row of
// grad written once, and a token that makes up a tenth of the text is spread over as many blocks as it takes.  A row that
// crosses the border between two shares leaves partial sums in fp32, joined in share order by a second small kernel: no
// atomics on values, the same bits every run.

#include <atomic>

#include "ec_vec.cuh"

namespace ec {
namespace {

// The kernels here start while their predecessor in the stream still drains; what they read may be its results, so no pointer is
// declared unaliased: the compiler would read it through the non-coherent path, whose lines the wait does not promise to renew.

// ---- lookup ------------------------------------------------------------------------------------------------------

constexpr int LK_THREADS = 256;
constexpr int LK_INFLIGHT = 4;          // vectors a lane has in flight

template <class IDX, class TI, class TO, int W>
__global__ void __launch_bounds__(LK_THREADS)
lookup_kernel(const TI* table, size_t table_stride, size_t V, size_t D, const IDX* tokens, size_t T,
              float scale, TO* out, size_t out_stride) {
    grid_dependency_wait();
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

// The widest unit (1, 2, 4 or, for bf16 input, 8 elements) that the row length and both sides' alignment allow.
template <class TI, class TO>
int unit_of(size_t D, const void* in, size_t in_stride, const void* out, size_t out_stride) {
    for (int u = sizeof(TI) == 2 ? 8 : 4; u > 1; u /= 2)
        if (D % u == 0 && rows_aligned(in, in_stride, sizeof(TI), u) && rows_aligned(out, out_stride, sizeof(TO), u)) return u;
    return 1;
}

template <class IDX, class TI, class TO>
int launch_lookup(const void* table, size_t V, size_t D, size_t ts, const void* tokens, size_t T, float scale, void* out,
                  size_t os, cudaStream_t st) {
    const int u = unit_of<TI, TO>(D, table, ts, out, os);
    const unsigned gx = (unsigned)((T + LK_THREADS / 32 - 1) / (LK_THREADS / 32));
    const size_t per = 32 * (size_t)u * LK_INFLIGHT, pieces = (D + per - 1) / per;
    const dim3 grid(gx, (unsigned)(pieces < 64 ? pieces : 64));
    auto launch = [&](auto kernel) {
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr; cfg.numAttrs = 1; cfg.stream = st;
        cfg.gridDim = grid; cfg.blockDim = dim3(LK_THREADS);
        EC_CUDA(cudaLaunchKernelEx(&cfg, kernel, (const TI*)table, ts, V, D, (const IDX*)tokens, T, scale, (TO*)out, os));
        return (int)EC_OK;
    };
    if constexpr (sizeof(TI) == 2) {
        if (u == 8) return launch(lookup_kernel<IDX, TI, TO, 8>);
    }
    if (u == 4) return launch(lookup_kernel<IDX, TI, TO, 4>);
    if (u == 2) return launch(lookup_kernel<IDX, TI, TO, 2>);
    return launch(lookup_kernel<IDX, TI, TO, 1>);
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

// Up to 65536 tokens: the whole sort in one launch, by one cluster of 1 to 8 blocks.  A thread keeps its items in registers; a
// pass ranks them inside the block, the blocks exchange their digit counts, and every item is sent to its place in some
// block's shared memory (the last pass: in global memory).
constexpr int CS_THREADS = 512, CS_WARPS = CS_THREADS / 32, CS_MAX_ITEMS = 16;

struct ClusterSortArgs {
    const void* tokens;
    uint32_t* keys; uint32_t* pos;
    uint32_t* joins;
    uint32_t T, V;
    long long skip;
    int bits, passes;
};

__device__ __forceinline__ void sort_cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t peer_address(const void* p, uint32_t rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return a;
}
__device__ __forceinline__ uint32_t peer_load(uint32_t address) {
    uint32_t x;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(x) : "r"(address));
    return x;
}
__device__ __forceinline__ void peer_store(uint32_t address, uint32_t x, uint32_t y) {
    asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(address), "r"(x), "r"(y) : "memory");
}

template <class IDX, int ITEMS>
__global__ void __launch_bounds__(CS_THREADS) sort_cluster_kernel(const ClusterSortArgs a) {
    grid_dependency_wait();
    extern __shared__ uint2 s_items[];                             // [ITEMS * CS_THREADS]: items of the next pass
    __shared__ uint32_t s_n[CS_WARPS][SORT_BINS];
    __shared__ uint32_t s_total[SORT_BINS], s_base[SORT_BINS], s_warp[CS_WARPS];
    constexpr uint32_t HOLD = ITEMS * CS_THREADS;                  // items of a block (a power of two)
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const uint32_t rank = blockIdx.x, blocks = gridDim.x;          // (one cluster: a block's number is its rank)
    const uint32_t base = rank * HOLD + w * (32 * ITEMS) + lane;   // (warp, step, lane) is the items' order
    if (rank == 0 && tid == 0) *a.joins = 0;
    uint32_t key[ITEMS], pos[ITEMS], at[ITEMS];
#pragma unroll
    for (int q = 0; q < ITEMS; ++q) {
        const uint32_t i = base + q * 32;
        key[q] = i < a.T ? token_key(static_cast<const IDX*>(a.tokens), i, a.V, a.skip) : 0u;
        pos[q] = i;
    }
    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = pass * a.bits;
        const uint32_t bins = 1u << a.bits;
        for (uint32_t d = lane; d < bins; d += 32) s_n[w][d] = 0;  // (a warp counts in its own row)
        __syncwarp();
        uint32_t same[ITEMS];
#pragma unroll
        for (int q = 0; q < ITEMS; ++q)                            // items past the end: a digit of their own
            same[q] = __match_any_sync(0xffffffffu, base + q * 32 < a.T ? (key[q] >> shift) & (bins - 1) : bins);
#pragma unroll
        for (int q = 0; q < ITEMS; ++q) {
            const bool in = base + q * 32 < a.T;
            const uint32_t d = (key[q] >> shift) & (bins - 1), below = __popc(same[q] & ((1u << lane) - 1u));
            const uint32_t old = in ? s_n[w][d] : 0u;
            __syncwarp();
            if (in && below == 0) s_n[w][d] = old + __popc(same[q]);
            __syncwarp();
            at[q] = old + below;
        }
        __syncthreads();
        if (tid < (int)bins) {                                     // a thread per digit: the warps' counts become their offsets
            uint32_t n[CS_WARPS], sum = 0;
#pragma unroll
            for (int q = 0; q < CS_WARPS; ++q) n[q] = s_n[q][tid];
#pragma unroll
            for (int q = 0; q < CS_WARPS; ++q) {
                s_n[q][tid] = sum;
                sum += n[q];
            }
            s_total[tid] = sum;
        }
        uint32_t before = 0, all = 0;
        if (blocks == 1) {
            if (tid < (int)bins) all = s_total[tid];
        } else {
            sort_cluster_sync();
            if (tid < (int)bins) {
                uint32_t n[8];
#pragma unroll
                for (uint32_t r = 0; r < 8; ++r) n[r] = r < blocks ? peer_load(peer_address(&s_total[tid], r)) : 0u;
#pragma unroll
                for (uint32_t r = 0; r < 8; ++r) {
                    before += r < rank ? n[r] : 0u;
                    all += n[r];
                }
            }
        }
        const uint32_t inc = warp_inclusive(all, lane);
        if (lane == 31) s_warp[w] = inc;
        __syncthreads();
        for (int q = 0; q < w; ++q) before += s_warp[q];
        if (tid < (int)bins) s_base[tid] = before + inc - all;
        __syncthreads();
        const bool last = pass + 1 == a.passes;
#pragma unroll
        for (int q = 0; q < ITEMS; ++q) {
            if (base + q * 32 >= a.T) continue;
            const uint32_t d = (key[q] >> shift) & (bins - 1), p = s_base[d] + s_n[w][d] + at[q];
            if (last) {
                a.keys[p] = key[q];
                a.pos[p] = pos[q];
            } else {
                peer_store(peer_address(&s_items[p % HOLD], p / HOLD), key[q], pos[q]);
            }
        }
        if (blocks > 1) sort_cluster_sync();                       // (the last one: no block goes while another may read its counts)
        else __syncthreads();
        if (!last) {
#pragma unroll
            for (int q = 0; q < ITEMS; ++q) {
                const uint2 x = s_items[w * (32 * ITEMS) + q * 32 + lane];
                key[q] = x.x;
                pos[q] = x.y;
            }
        }
    }
}

template <class IDX, int ITEMS>
int launch_cluster_sort(const ClusterSortArgs& a, unsigned blocks, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = blocks; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 2; cfg.stream = st;
    cfg.gridDim = dim3(blocks); cfg.blockDim = dim3(CS_THREADS);
    cfg.dynamicSmemBytes = (size_t)ITEMS * CS_THREADS * 8;
    if (cfg.dynamicSmemBytes > 8 * 1024) {                         // (beside 37 KB of static shared memory)
        static std::atomic<uint64_t> ready{0};                     // devices on which the limit is raised
        int dev = 0;
        EC_CUDA(cudaGetDevice(&dev));
        if (dev >= 64 || !(ready.load(std::memory_order_relaxed) >> dev & 1u)) {
            EC_CUDA(cudaFuncSetAttribute(sort_cluster_kernel<IDX, ITEMS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)cfg.dynamicSmemBytes));
            if (dev < 64) ready.fetch_or(1ull << dev, std::memory_order_relaxed);
        }
    }
    EC_CUDA(cudaLaunchKernelEx(&cfg, sort_cluster_kernel<IDX, ITEMS>, a));
    return EC_OK;
}

// ---- the walk ----------------------------------------------------------------------------------------------------

constexpr int GR_THREADS = 256;
constexpr int GR_INFLIGHT = 8;          // rows of dout a thread has in flight (131072 x 2048: 303 us; four: 313; eight in 64 registers: 312)
constexpr int GR_MAX_SHARE = 64;
constexpr int GR_STEPS = 1024;          // most path steps of a block
constexpr int GR_LONG = 32;             // a row with this many tokens before a share's border is cut there; a shorter one goes to the next share
constexpr uint32_t NO_ROW = 0xffffffffu;

// How a call is cut: a block takes C path steps for each of its GR_THREADS / G groups; a group's share of its tokens is even.
struct GradPlan {
    int U, G, C;                        // elements a unit, threads a group, path steps a group
    unsigned shares, blocks, slices;    // shares = groups in all (a multiple of the groups of a block)
};

// W: elements a thread takes of a row, as W / U units G units apart
GradPlan grad_plan(size_t steps, size_t D, int U, int W) {
    GradPlan p;
    p.U = U;
    const size_t lanes = (D + W - 1) / W;
    p.G = 8;
    while (p.G < GR_THREADS && (size_t)p.G < lanes) p.G *= 2;
    p.slices = (unsigned)((lanes + p.G - 1) / p.G);
    const unsigned groups = GR_THREADS / p.G;
    p.C = GR_STEPS / (int)groups < GR_MAX_SHARE ? GR_STEPS / (int)groups : GR_MAX_SHARE;
    // (12289 tokens on 50021 x 1001: 76 us; with half or twice as many blocks asked for 81 / 80)
    while (p.C > 8 && (steps / ((size_t)p.C * groups)) * p.slices < 148 * 8) p.C /= 2;
    p.blocks = (unsigned)((steps + (size_t)p.C * groups - 1) / ((size_t)p.C * groups));
    p.shares = p.blocks * groups;
    return p;
}

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

// Where the border of a block at path step d lies: number of sorted tokens before it and row.  That is the tokens p with
// p + key[p] < d, found by one warp, 33 sections at a time - moved back to a row's first token if the border falls between
// two tokens of the row and fewer than GR_LONG of them lie before it, so that only long rows are cut and joined later.
// A gradient that is added to what is there has no rows to fill with zeros: its path is the tokens alone, the border at token d
// (4096 tokens on 65536 x 1024 fp32: 31 -> 23.5 us; 12289 on 50021 x 1001: 81 -> 75).
__device__ __forceinline__ void border(const uint32_t* keys, uint32_t T, uint32_t V, bool rows, uint32_t d, int lane, uint32_t* tokens, uint32_t* row) {
    uint32_t lo = !rows ? d : d > V ? d - V : 0u, hi = d < T ? d : T;
    while (lo < hi) {
        const uint32_t step = (hi - lo + 31) / 32, p = lo + lane * step;
        const bool less = p < hi && p + keys[p] < d;
        const uint32_t n = __popc(__ballot_sync(0xffffffffu, less));
        if (n == 0) break;
        const uint32_t top = lo + n * step;
        lo = lo + (n - 1) * step + 1;
        hi = top < hi ? top : hi;
    }
    const uint32_t j = rows ? d - lo : lo < T ? keys[lo] : V;
    const uint32_t same = __ballot_sync(0xffffffffu, lo < T && lo > (uint32_t)lane && keys[lo] == j && keys[lo - 1 - lane] == j);
    static_assert(GR_LONG == 32, "one look back of a warp");
    *tokens = same == 0xffffffffu ? lo : lo - (uint32_t)(__ffs(~same) - 1);
    *row = j;
}

// n zeros from p on by one warp, in 16-byte pieces wherever p lies
template <class TO>
__device__ __forceinline__ void zero_span(TO* p, size_t n, uint32_t lane) {
    constexpr uint32_t W = 16 / sizeof(TO);
    const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15u) / (uint32_t)sizeof(TO);
    const size_t head = off == 0 ? 0 : W - off < n ? W - off : n, vecs = (n - head) / W;
    const uint32_t rest = (uint32_t)(n - head - vecs * W);
    const float zero[1] = {0.0f};
    uint4* q = reinterpret_cast<uint4*>(p + head) + lane;
    if (lane < head) store_vec<TO, 1>(p + lane, zero);
    if (lane < rest) store_vec<TO, 1>(p + head + vecs * W + lane, zero);
#pragma unroll 4
    for (size_t i = lane; i < vecs; i += 32, q += 32) __stcs(q, make_uint4(0u, 0u, 0u, 0u));
}

template <class TO, int U>
__device__ __forceinline__ void write_unit(TO* p, const float* acc, float scale, bool add) {
    float x[U];
#pragma unroll
    for (int e = 0; e < U; ++e) x[e] = scale * acc[e];
    if (add) {
        float old[U];
        if constexpr (sizeof(TO) * U > 16) {
            constexpr int H = U / 2;
            float a[H], b[H];
            load_vec<TO, H>(p, a);
            load_vec<TO, H>(p + H, b);
#pragma unroll
            for (int e = 0; e < H; ++e) { old[e] = a[e]; old[H + e] = b[e]; }
        } else {
            load_vec<TO, U>(p, old);
        }
#pragma unroll
        for (int e = 0; e < U; ++e) x[e] += old[e];
    }
    store_vec<TO, U>(p, x);
}

// A block takes a stretch of the path: its rows without tokens are written with zeros by the warps in turn, its tokens are shared
// out evenly to the groups.
template <class TI, class TO, int U, int NU>
__global__ void __launch_bounds__(GR_THREADS, 3) grad_walk_kernel(const GradArgs a, const TI* dout, TO* grad) {
    grid_dependency_wait();
    __shared__ uint32_t s_key[GR_STEPS + GR_LONG + 2], s_pos[GR_STEPS + GR_LONG];      // s_key[0], s_key[n + 1]: the tokens before and behind the block's
    __shared__ uint32_t s_has[(GR_STEPS + GR_LONG) / 32 + 1];                          // bit r: row rows0 + r has tokens
    __shared__ uint32_t s_tok[2], s_rowat[2];
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const uint32_t groups = GR_THREADS / a.G, total = a.T + (a.accumulate ? 0u : a.V);
    const uint32_t d0 = blockIdx.x * groups * a.C, d1 = d0 + groups * a.C < total ? d0 + groups * a.C : total;
    if (w < 2) {
        uint32_t i, j;
        border(a.keys, a.T, a.V, !a.accumulate, w == 0 ? d0 : d1, lane, &i, &j);
        if (lane == 0) { s_tok[w] = i; s_rowat[w] = j; }
    } else {
        for (uint32_t q = tid - 64; q < sizeof(s_has) / 4; q += GR_THREADS - 64) s_has[q] = 0;
    }
    __syncthreads();
    const uint32_t i0 = s_tok[0], n = s_tok[1] - i0, row0 = s_rowat[0], row1 = s_rowat[1];
    for (uint32_t q = tid; q < n + 2; q += GR_THREADS) {
        const uint32_t k = i0 + q > 0 && i0 + q <= a.T ? a.keys[i0 + q - 1] : NO_ROW;
        s_key[q] = k;
        if (q > 0 && q <= n) s_pos[q - 1] = a.pos[i0 + q - 1];
        if (!a.accumulate && k >= row0 && k < row1) atomicOr(&s_has[(k - row0) >> 5], 1u << ((k - row0) & 31));      // (bits: order is free)
    }
    __syncthreads();

    // the group's share of the tokens; borders inside a row move as the block's do
    const uint32_t g = tid / a.G, member = tid & (a.G - 1);
    auto inner = [&](uint32_t i) {
        if (i == 0 || i >= n || s_key[i] != s_key[i + 1]) return i;
        uint32_t f = i > GR_LONG ? i - GR_LONG : 0, hi = i;
        const uint32_t k = s_key[i];
        while (f < hi) {                                             // the row's first token in the block, looking back GR_LONG tokens
            const uint32_t m = (f + hi) / 2;
            if (s_key[m + 1] < k) f = m + 1; else hi = m;
        }
        return i - f < GR_LONG && s_key[f] != k ? f : i;             // (s_key[f] == k: it began before the block, behind a border that cuts it)
    };
    const uint32_t each = (n + groups - 1) / groups;
    uint32_t i = inner(g * each < n ? g * each : n);
    const uint32_t i_end = inner((g + 1) * each < n ? (g + 1) * each : n);
    const uint32_t share = blockIdx.x * groups + g;
    uint32_t row = s_key[i];                                         // the current row: it goes on from the share before, or there is none yet
    const bool inside = row < a.V && row == s_key[i + 1];
    const bool note = blockIdx.y == 0 && member == 0;
    if (note) a.begins[share] = inside ? row : NO_ROW;

    const size_t c0 = ((size_t)blockIdx.y * a.G * NU + member) * U;  // unit u: columns c0 + u G U ...
    const size_t cstep = (size_t)a.G * U;
    bool mine[NU];
#pragma unroll
    for (int u = 0; u < NU; ++u) mine[u] = c0 + u * cstep < a.D;
    constexpr int FLY = GR_INFLIGHT / (NU > 2 ? 2 : 1);
    raw_vec<TI, U> v[FLY][NU];
    uint32_t key[FLY];
    auto fetch = [&] {                                               // (no branch around a load: it would be waited for in it)
        const TI* src[FLY];
#pragma unroll
        for (int q = 0; q < FLY; ++q) {
            const uint32_t at = i + q < i_end ? i + q : i;
            key[q] = s_key[at + 1];
            src[q] = dout + (size_t)s_pos[at] * a.in_stride + c0;    // (a token that gives nothing has a position as well)
        }
#pragma unroll
        for (int q = 0; q < FLY; ++q)
#pragma unroll
            for (int u = 0; u < NU; ++u)
                if (i + q < i_end && mine[u]) v[q][u] = load_raw<TI, U>(src[q] + u * cstep);
    };
    if (i < i_end) fetch();
    if (!a.accumulate) {                                             // zeros, while the first rows are on their way
        const size_t first = (size_t)blockIdx.y * a.G * NU * U, width = (size_t)a.G * NU * U;
        const uint32_t cols = (uint32_t)(a.D - first < width ? a.D - first : width), rows = row1 - row0;
        const bool dense = cols == a.D && a.out_stride == a.D;       // rows follow each other without gaps
        const uint32_t hi = rows * (w + 1) / (GR_THREADS / 32);
        for (uint32_t r = rows * w / (GR_THREADS / 32); r < hi;) {   // the warp's rows: runs [r, e) without tokens
            const uint32_t none = ~s_has[r >> 5] >> (r & 31);
            if (none == 0) { r = (r | 31) + 1; continue; }
            r += __ffs(none) - 1;
            uint32_t e = r;
            while (e < hi) {
                const uint32_t some = s_has[e >> 5] >> (e & 31);
                if (some != 0) { e += __ffs(some) - 1; break; }
                e = (e | 31) + 1;
            }
            if (e > hi) e = hi;
            TO* p = grad + (size_t)(row0 + r) * a.out_stride + first;
            if (dense) {
                if (r < e) zero_span(p, (size_t)(e - r) * cols, lane);
            } else {
                for (uint32_t q = r; q < e; ++q, p += a.out_stride) zero_span(p, cols, lane);
            }
            r = e;
        }
    }
    float acc[NU][U];
    auto clear = [&] {
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int x = 0; x < U; ++x) acc[u][x] = 0.0f;
    };
    clear();
    bool open = inside, first = inside;                              // there is a current row; it began in an earlier share
    auto close = [&] {
        if (first) {
#pragma unroll
            for (int u = 0; u < NU; ++u)
                if (mine[u]) store_vec<float, U>(a.head + (size_t)share * a.D + c0 + u * cstep, acc[u]);
            if (note) {
                const uint32_t q = atomicAdd(a.joins, 1u);           // (the list's order does not matter: every row joins for itself)
                a.joins[1 + 2 * q] = share;
                a.joins[2 + 2 * q] = row;
            }
        } else {
            TO* out = grad + (size_t)row * a.out_stride + c0;
#pragma unroll
            for (int u = 0; u < NU; ++u)
                if (mine[u]) write_unit<TO, U>(out + u * cstep, acc[u], a.scale, a.accumulate != 0);
        }
        first = false;
        clear();
    };
    while (i < i_end) {
#pragma unroll
        for (int q = 0; q < FLY; ++q) {
            if (i + q < i_end) {
                const uint32_t k = key[q];
                if (k != row || !open) {
                    if (open) close();
                    row = k;
                    open = k < a.V;
                }
                if (open) {
#pragma unroll
                    for (int u = 0; u < NU; ++u)
                        if (mine[u]) {
                            float x[U];
                            unpack<TI, U>(v[q][u], x);
#pragma unroll
                            for (int z = 0; z < U; ++z) acc[u][z] += x[z];
                        }
                }
            }
        }
        i += FLY;
        if (i < i_end) fetch();
    }
    if (open) {
        if (s_key[i_end + 1] != row) {
            close();
        } else {
#pragma unroll
            for (int u = 0; u < NU; ++u)
                if (mine[u]) store_vec<float, U>(a.tail + (size_t)share * a.D + c0 + u * cstep, acc[u]);
        }
    }
}

// ---- joining the rows that cross shares --------------------------------------------------------------------------
// Row j ends in share s and began in share f < s: its sum is tail[f] + ... + tail[s-1] + head[s].  A block takes 128 columns;
// its eight warps add up contiguous parts of the range, then the parts in order.

constexpr int JN_THREADS = 256, JN_WARPS = JN_THREADS / 32;

template <class TO>
__global__ void __launch_bounds__(JN_THREADS) grad_join_kernel(const GradArgs a, TO* grad) {
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
                write_unit<TO, 1>(grad + (size_t)j * a.out_stride + c, sum, a.scale, a.accumulate != 0);
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
// Sized for either input type (4 or 8 elements of a row a thread).
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
    for (int W = 4; W <= 8; W += 4) {
        for (size_t steps : {T, T + V}) {
            const size_t n = steps == 0 ? 0 : grad_plan(steps, D, 1, W).shares;
            shares = n > shares ? n : shares;
        }
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
    if (a.T <= 8u * CS_THREADS * CS_MAX_ITEMS) {
        ClusterSortArgs c = {};
        c.tokens = a.tokens; c.joins = a.joins;
        c.keys = reinterpret_cast<uint32_t*>(ws + L.keys[(L.passes - 1) & 1]);
        c.pos = reinterpret_cast<uint32_t*>(ws + L.pos[(L.passes - 1) & 1]);
        c.T = a.T; c.V = a.V; c.skip = a.skip; c.bits = L.bits; c.passes = L.passes;
        unsigned blocks = 1;                                       // few items a thread first, then more blocks
        while (blocks < 8 && a.T > blocks * CS_THREADS) blocks *= 2;
        const unsigned per = (a.T + blocks * CS_THREADS - 1) / (blocks * CS_THREADS);
        if (per <= 1) return launch_cluster_sort<IDX, 1>(c, blocks, st);
        if (per <= 2) return launch_cluster_sort<IDX, 2>(c, blocks, st);
        if (per <= 4) return launch_cluster_sort<IDX, 4>(c, blocks, st);
        if (per <= 8) return launch_cluster_sort<IDX, 8>(c, blocks, st);
        return launch_cluster_sort<IDX, 16>(c, blocks, st);
    }
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

template <class TI, class TO, int U>
int launch_walk(GradArgs a, const void* dout, void* grad, cudaStream_t st) {
    constexpr int W = sizeof(TI) == 2 ? 8 : 4;
    const GradPlan p = grad_plan((size_t)a.T + (a.accumulate ? 0 : a.V), a.D, U, W);
    a.G = p.G;
    a.C = p.C;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 1; cfg.stream = st;
    cfg.gridDim = dim3(p.blocks, p.slices); cfg.blockDim = dim3(GR_THREADS);
    EC_CUDA(cudaLaunchKernelEx(&cfg, grad_walk_kernel<TI, TO, U, W / U>, a, static_cast<const TI*>(dout), static_cast<TO*>(grad)));
    if (a.T <= GR_LONG) return EC_OK;                  // no row is long enough to be cut
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
    if (!on_grid(table, in_bytes(table_dtype)) || !on_grid(out, in_bytes(out_dtype)) || !on_grid(tokens, index == EC_INDEX_32 ? 4 : 8)) return EC_ERR_INVALID;
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
    if (!on_grid(dout, in_bytes(dout_dtype)) || !on_grid(grad, in_bytes(grad_dtype)) || !on_grid(tokens, index == EC_INDEX_32 ? 4 : 8)) return EC_ERR_INVALID;
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
        const int u = unit_of<TI, TO>(D, dout, dout_stride, grad, grad_stride);
        if constexpr (sizeof(TI) == 2) {
            if (u == 8) return launch_walk<TI, TO, 8>(a, dout, grad, stream);
        }
        if (u == 4) return launch_walk<TI, TO, 4>(a, dout, grad, stream);
        if (u == 2) return launch_walk<TI, TO, 2>(a, dout, grad, stream);
        return launch_walk<TI, TO, 1>(a, dout, grad, stream);
    });
}

}  // extern "C"
