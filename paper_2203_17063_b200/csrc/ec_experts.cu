// Matrix products grouped by expert, ragged sizes.
//
//   forward       y[r] = W_e x[r]                      for the rows r of expert e
//   input grad    dx[r] = W_e^T dy[r]
//   weight grad   dW_e = sum over the rows r of e of dy[r] x[r]^T
//
// Rows are sorted by expert: expert e owns rows displs[e] .. displs[e+1]-1 (displs as ec_allgatherv leaves it, on the
// device: the host never learns the sizes).  Every block derives the list of tiles from displs itself.

#include "ec_vec.cuh"

namespace ec {
namespace {

constexpr int MAX_EXPERTS = EC_MAX_EXPERTS;
constexpr size_t MAX_ROWS = 0x7fffffffull - 1024;       // a tile past the last row still has a row number

enum { EX_FORWARD = 0, EX_INPUT = 1, EX_WEIGHT = 2 };

struct ExpertArgs {
    const void* x; size_t x_stride;        // rows of K (forward, weight grad)
    const void* dy; size_t dy_stride;      // rows of N (input grad, weight grad)
    const void* w;                         // [E][N][K]
    void* out; size_t out_stride;          // y [T][N], dx [T][K], or dW [E][N][K]
    const int64_t* displs; uint32_t* status;
    size_t T;
    int E, N, K, accumulate;
};

// The row ranges of the experts in shared memory, and the number of row tiles of `tile` rows before each expert.  All threads
// of the block; returns false (and block 0 says so in *status) if displs does not ascend within [0, T].
template <int THREADS>
__device__ bool expert_ranges(const ExpertArgs& a, int tile, int* s_row, int* s_tile, int* s_warp) {
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    bool ok = true;
    int carry = 0;
    for (int e0 = 0; e0 < a.E; e0 += THREADS) {
        const int e = e0 + tid;
        int n = 0;
        if (e < a.E) {
            const long long b = a.displs[e], d = a.displs[e + 1];
            if (b < 0 || d < b || d > (long long)a.T) {
                ok = false;
            } else {
                s_row[e] = (int)b;
                if (e == a.E - 1) s_row[a.E] = (int)d;
                n = (int)((d - b + tile - 1) / tile);
            }
        }
        int inc = n;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, inc, d);
            if (lane >= d) inc += y;
        }
        if (lane == 31) s_warp[w] = inc;
        __syncthreads();
        int before = carry, all = carry;
        for (int q = 0; q < THREADS / 32; ++q) {
            if (q < w) before += s_warp[q];
            all += s_warp[q];
        }
        if (e < a.E) s_tile[e] = before + inc - n;
        carry = all;
        __syncthreads();
    }
    if (tid == 0) s_tile[a.E] = carry;
    ok = __syncthreads_and(ok ? 1 : 0) != 0;
    if (blockIdx.x == 0 && tid == 0 && a.status != nullptr) *a.status = ok ? 0u : 1u;
    return ok;
}
// the expert whose row tiles contain tile t
__device__ __forceinline__ int expert_of(const int* s_tile, int E, int t) {
    int lo = 0, hi = E - 1;
    while (lo < hi) {
        const int m = (lo + hi + 1) / 2;
        if (s_tile[m] <= t) lo = m; else hi = m - 1;
    }
    return lo;
}

// ---- products on the fp32 units: any type, any alignment ---------------------------------------------------------
// C[i][j] = sum_l A(i, l) B(l, j) for tiles of 64 x 64, 4 x 4 values a thread, 16 steps of l at a time.

constexpr int SC_TILE = 64, SC_STEP = 16, SC_THREADS = 256;

template <class TI, class TO, int MODE>
__global__ void __launch_bounds__(SC_THREADS) expert_scalar_kernel(const ExpertArgs a) {
    __shared__ int s_row[MAX_EXPERTS + 1], s_tile[MAX_EXPERTS + 1], s_warp[SC_THREADS / 32];
    __shared__ float s_a[SC_STEP][SC_TILE + 4], s_b[SC_STEP][SC_TILE + 4];
    if (!expert_ranges<SC_THREADS>(a, SC_TILE, s_row, s_tile, s_warp)) return;
    const int rows_out = MODE == EX_WEIGHT ? a.N : 0, cols_out = MODE == EX_FORWARD ? a.N : a.K;
    const int jt = (cols_out + SC_TILE - 1) / SC_TILE, it = (rows_out + SC_TILE - 1) / SC_TILE;
    const long long tiles = MODE == EX_WEIGHT ? (long long)a.E * it * jt : (long long)s_tile[a.E] * jt;
    const int tid = threadIdx.x, ti = tid / 16, tj = tid % 16;
    const TI* x = static_cast<const TI*>(a.x);
    const TI* dy = static_cast<const TI*>(a.dy);
    for (long long t = blockIdx.x; t < tiles; t += gridDim.x) {
        int e, i0, i1, len;
        const int j0 = (int)(t % jt) * SC_TILE;
        const int q = (int)(t / jt);
        if (MODE == EX_WEIGHT) {
            e = q / it;
            i0 = (q - e * it) * SC_TILE;
            i1 = a.N;
            len = s_row[e + 1] - s_row[e];
        } else {
            e = expert_of(s_tile, a.E, q);
            i0 = s_row[e] + (q - s_tile[e]) * SC_TILE;
            i1 = s_row[e + 1];
            len = MODE == EX_FORWARD ? a.K : a.N;
        }
        if (MODE == EX_WEIGHT && a.accumulate && len == 0) continue;
        const TI* w = static_cast<const TI*>(a.w) + (size_t)e * a.N * a.K;
        float acc[4][4] = {};
        for (int l0 = 0; l0 < len; l0 += SC_STEP) {
            for (int p = tid; p < SC_STEP * SC_TILE; p += SC_THREADS) {
                // forward: A = x (adjacent in l), B = W (adjacent in l); input: A = dy (l), B = W (j); weight: A = dy (i), B = x (j)
                int l = MODE == EX_WEIGHT ? p / SC_TILE : p % SC_STEP, i = MODE == EX_WEIGHT ? p % SC_TILE : p / SC_STEP;
                float v = 0.0f;
                if (l0 + l < len && i0 + i < i1) {
                    if (MODE == EX_FORWARD) v = unpack_one<TI>(x[(size_t)(i0 + i) * a.x_stride + l0 + l]);
                    if (MODE == EX_INPUT) v = unpack_one<TI>(dy[(size_t)(i0 + i) * a.dy_stride + l0 + l]);
                    if (MODE == EX_WEIGHT) v = unpack_one<TI>(dy[(size_t)(s_row[e] + l0 + l) * a.dy_stride + i0 + i]);
                }
                s_a[l][i] = v;
                l = MODE == EX_FORWARD ? p % SC_STEP : p / SC_TILE;
                const int j = MODE == EX_FORWARD ? p / SC_STEP : p % SC_TILE;
                v = 0.0f;
                if (l0 + l < len && j0 + j < cols_out) {
                    if (MODE == EX_FORWARD) v = unpack_one<TI>(w[(size_t)(j0 + j) * a.K + l0 + l]);
                    if (MODE == EX_INPUT) v = unpack_one<TI>(w[(size_t)(l0 + l) * a.K + j0 + j]);
                    if (MODE == EX_WEIGHT) v = unpack_one<TI>(x[(size_t)(s_row[e] + l0 + l) * a.x_stride + j0 + j]);
                }
                s_b[l][j] = v;
            }
            __syncthreads();
#pragma unroll
            for (int l = 0; l < SC_STEP; ++l) {
                float u[4], v[4];
#pragma unroll
                for (int p = 0; p < 4; ++p) { u[p] = s_a[l][ti * 4 + p]; v[p] = s_b[l][tj * 4 + p]; }
#pragma unroll
                for (int p = 0; p < 4; ++p)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[p][r] = fmaf(u[p], v[r], acc[p][r]);
            }
            __syncthreads();
        }
        TO* out = static_cast<TO*>(a.out) + (MODE == EX_WEIGHT ? (size_t)e * a.N * a.K : 0);
        const size_t os = MODE == EX_WEIGHT ? (size_t)a.K : a.out_stride;
        for (int p = 0; p < 4; ++p)
            for (int r = 0; r < 4; ++r) {
                const int i = i0 + ti * 4 + p, j = j0 + tj * 4 + r;
                if (i >= i1 || j >= cols_out) continue;
                TO* d = out + (size_t)i * os + j;
                const float one[1] = {acc[p][r] + (MODE == EX_WEIGHT && a.accumulate ? unpack_one<TO>(*d) : 0.0f)};
                store_vec<TO, 1>(d, one);
            }
    }
}

template <int MODE>
int launch_experts(const ExpertArgs& a, ec_dtype_t dtype, ec_dtype_t out_dtype, cudaStream_t st) {
    return with_types(dtype, out_dtype, [&](auto ti, auto to) {
        using TI = decltype(ti); using TO = decltype(to);
        expert_scalar_kernel<TI, TO, MODE><<<148 * 4, SC_THREADS, 0, st>>>(a);
        EC_CUDA(cudaGetLastError());
        return (int)EC_OK;
    });
}

int check(const ExpertArgs& a, ec_dtype_t dtype, ec_dtype_t out_dtype, int mode) {
    if (a.T > MAX_ROWS || a.E < 1 || a.N < 1 || a.K < 1 || !a.displs || (!a.out && (a.T > 0 || mode == EX_WEIGHT))) return EC_ERR_INVALID;
    if (mode != EX_WEIGHT && !a.w) return EC_ERR_INVALID;
    if (mode != EX_INPUT && ((a.T > 0 && !a.x) || a.x_stride < (size_t)a.K)) return EC_ERR_INVALID;
    if (mode != EX_FORWARD && ((a.T > 0 && !a.dy) || a.dy_stride < (size_t)a.N)) return EC_ERR_INVALID;
    if (mode != EX_WEIGHT && a.out_stride < (size_t)(mode == EX_FORWARD ? a.N : a.K)) return EC_ERR_INVALID;
    if (a.E > EC_MAX_EXPERTS || a.N > (1 << 20) || a.K > (1 << 20)) return EC_ERR_CAPACITY;
    if (!is_real_dtype(dtype) || !is_real_dtype(out_dtype)) return EC_ERR_UNSUPPORTED;
    return EC_OK;
}

}  // namespace
}  // namespace ec

using namespace ec;

extern "C" {

int ec_expert_forward(const void* x, size_t x_stride, const int64_t* displs, int E, const void* w, ec_dtype_t dtype, size_t T, int N,
                      int K, void* y, size_t y_stride, ec_dtype_t y_dtype, uint32_t* status, ec_stream_t stream) {
    ExpertArgs a = {};
    a.x = x; a.x_stride = x_stride; a.w = w; a.out = y; a.out_stride = y_stride;
    a.displs = displs; a.status = status; a.T = T; a.E = E; a.N = N; a.K = K;
    const int rc = check(a, dtype, y_dtype, EX_FORWARD);
    return rc != EC_OK ? rc : launch_experts<EX_FORWARD>(a, dtype, y_dtype, stream);
}

int ec_expert_input_grad(const void* dy, size_t dy_stride, const int64_t* displs, int E, const void* w, ec_dtype_t dtype, size_t T,
                         int N, int K, void* dx, size_t dx_stride, ec_dtype_t dx_dtype, uint32_t* status, ec_stream_t stream) {
    ExpertArgs a = {};
    a.dy = dy; a.dy_stride = dy_stride; a.w = w; a.out = dx; a.out_stride = dx_stride;
    a.displs = displs; a.status = status; a.T = T; a.E = E; a.N = N; a.K = K;
    const int rc = check(a, dtype, dx_dtype, EX_INPUT);
    return rc != EC_OK ? rc : launch_experts<EX_INPUT>(a, dtype, dx_dtype, stream);
}

int ec_expert_weight_grad(const void* dy, size_t dy_stride, const void* x, size_t x_stride, const int64_t* displs, int E,
                          ec_dtype_t dtype, size_t T, int N, int K, void* dw, ec_dtype_t dw_dtype, int accumulate, uint32_t* status,
                          ec_stream_t stream) {
    ExpertArgs a = {};
    a.dy = dy; a.dy_stride = dy_stride; a.x = x; a.x_stride = x_stride; a.out = dw;
    a.displs = displs; a.status = status; a.T = T; a.E = E; a.N = N; a.K = K; a.accumulate = accumulate != 0;
    const int rc = check(a, dtype, dw_dtype, EX_WEIGHT);
    return rc != EC_OK ? rc : launch_experts<EX_WEIGHT>(a, dtype, dw_dtype, stream);
}

}  // extern "C"
