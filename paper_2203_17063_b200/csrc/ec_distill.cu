// Distillation from a teacher's top logits: loss, gradient, or both in one pass.
//
//   u = z / tau,  lse = log sum_v exp(u_v),  a_k = teacher logit / tau
//   p_k = exp(a_k - A),  A = log sum over the row's entries of exp(a_k), or the teacher's own log-sum if it is given
//   loss = w sum_k p_k (log p_k - u_{i_k} + lse)
//   dz_v = g (m exp(u_v - lse) - sum over k with i_k = v of p_k),   m = sum_k p_k,  g = w / tau [* dloss]
//
// A row of logits is read once, its gradient written once: bound by memory.  Exponentials are taken to base 2 (one fused
// multiply-add and one ex2 an element); maxima, sums and the gradient are fp32, rounded once when the gradient is bf16.
// Every thread keeps the maximum of what it has seen and the sum of exponentials below it; a block joins its threads in a
// fixed order.  The gradient is first written as if no entry were in the teacher's list; the list's entries follow behind a
// barrier, each written by the block that owns its column.

#include <cooperative_groups.h>

#include "ec_vec.cuh"

namespace ec {
namespace {

namespace cg = cooperative_groups;

constexpr int MAX_TOP = EC_DISTILL_MAX_TOP;
constexpr float LOG2E = 1.44269504088896340736f, LOG2E_REST = 1.92596299112661746887e-8f;   // log2 e = LOG2E + LOG2E_REST

enum { MODE_LOSS = 0, MODE_GRAD = 1, MODE_STEP = 2 };

struct DistillArgs {
    const void* logits; size_t stride;
    const void* top_index; const void* top_logit;
    const float* teacher_lse; const float* weight; const float* dloss;
    float* loss; float* lse;               // lse: written by the loss, read by the gradient alone
    void* grad; size_t grad_stride;
    size_t V;
    float inv_tau;
    int K, index64, top_bf16;
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
    return x;
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    return x;
}
// exp2(c (x - m)) for logits x, m: one fused multiply-add where c m is far inside fp32's range, else (rows masked with the
// type's lowest value throughout) by the difference, which cannot overflow to a NaN.
struct Below {
    float c, m, cm;
    bool fused;
    __device__ Below(float c_, float m_) : c(c_), m(m_ == -INFINITY ? 0.0f : m_), cm(c_ * m), fused(fabsf(cm) < 1e38f) {}
    __device__ float operator()(float x) const { return ex2(fused ? fmaf(x, c, -cm) : (x - m) * c); }
};
// (maximum, sum below it) of two parts; a part without anything has maximum -inf and sum 0
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2, float c) {
    const float top = fmaxf(m, m2), ref = top == -INFINITY ? 0.0f : top;
    s = s * ex2((m - ref) * c) + s2 * ex2((m2 - ref) * c);
    m = top;
}

// Rows may start anywhere on the element grid.  A row is seen as vectors of 16 bytes on the 16-byte grid; its first and last
// vector may stick out of it and are then accessed element by element.
template <class T>
struct Row {
    static constexpr int W = 16 / (int)sizeof(T);
    const T* p;              // first element
    size_t V;
    int h;                   // elements between the 16-byte boundary at or before p and p
    __device__ Row(const T* p_, size_t V_) : p(p_), V(V_), h((int)((reinterpret_cast<uintptr_t>(p_) & 15u) / sizeof(T))) {}
    __device__ size_t vectors() const { return (V + h + W - 1) / W; }
    __device__ bool whole(size_t i) const { return i * W >= (size_t)h && (i + 1) * W <= V + h; }
    __device__ raw_vec<T, W> load(size_t i) const {
        if (whole(i)) return load_raw<T, W>(p - h + i * W);
        raw_vec<T, W> r;
#pragma unroll
        for (int e = 0; e < W; ++e) {
            const size_t x = i * W + e;
            uint32_t b = sizeof(T) == 4 ? 0xff800000u : 0xff80u;          // -inf: nothing there
            if (x >= (size_t)h && x < V + h) b = load_raw<T, 1>(p + (x - h)).u[0];
            if (sizeof(T) == 4) r.u[e] = b;
            else if (e & 1) r.u[e / 2] |= b << 16;
            else r.u[e / 2] = b;
        }
        return r;
    }
};
// the same positions of the gradient's row; `aligned`: its rows lie on the 16-byte grid as the logits' rows do
template <class T>
__device__ __forceinline__ void store_row(const Row<T>& row, T* dst, bool aligned, size_t i, const float (&x)[16 / sizeof(T)]) {
    constexpr int W = Row<T>::W;
    if (aligned && row.whole(i)) {
        store_vec<T, W>(dst + (i * W - row.h), x);
        return;
    }
#pragma unroll
    for (int e = 0; e < W; ++e) {
        const size_t c = i * W + e;
        if (c >= (size_t)row.h && c < row.V + row.h) {
            const float one[1] = {x[e]};
            store_vec<T, 1>(dst + (c - row.h), one);
        }
    }
}

// What the block knows of the row's teacher (shared memory).
struct Teacher {
    float mass, part;        // sum of p_k; sum over the block's own columns of p_k (log p_k - u_k)
    int any;                 // the row has an entry
};

// One warp: the teacher's entries of row t.  [c0, c1): the block's columns, whose logits are fetched.
template <class T>
__device__ void teacher_row(const DistillArgs& a, size_t t, const T* z, size_t c0, size_t c1, int lane, int* s_idx, float* s_p, float* s_z,
                            Teacher* out) {
    const size_t base = t * (size_t)a.K;
    float top = -INFINITY;
    int any = 0;
    for (int k = lane; k < a.K; k += 32) {
        const long long i = a.index64 ? static_cast<const int64_t*>(a.top_index)[base + k] : static_cast<const int32_t*>(a.top_index)[base + k];
        const bool there = i >= 0 && (unsigned long long)i < a.V;
        float l = -INFINITY;
        if (there)
            l = (a.top_bf16 ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(a.top_logit)[base + k] << 16)
                            : static_cast<const float*>(a.top_logit)[base + k]) * a.inv_tau;
        s_idx[k] = there ? (int)i : -1;
        s_p[k] = l;
        s_z[k] = there && (size_t)i >= c0 && (size_t)i < c1 ? unpack_one<T>(z[i]) : 0.0f;
        any |= there ? 1 : 0;
        top = l > top || l != l ? l : top;              // (a NaN stays)
    }
    any = __any_sync(0xffffffffu, any);
    float A;
    if (a.teacher_lse != nullptr) {
        A = a.teacher_lse[t];
    } else {
        const bool bad = __any_sync(0xffffffffu, top != top);
        top = bad ? NAN : warp_max(top);
        if (top == -INFINITY) any = 0;                  // entries, but none with any weight
        const float ref = top == -INFINITY ? 0.0f : top;
        float s = 0.0f;
        for (int k = lane; k < a.K; k += 32) s += expf(s_p[k] - ref);
        A = ref + logf(warp_sum(s));
    }
    float mass = 0.0f, part = 0.0f;
    for (int k = lane; k < a.K; k += 32) {
        const float logp = s_p[k] - A, p = s_idx[k] >= 0 ? expf(logp) : 0.0f;
        s_p[k] = p;
        mass += p;
        if (p != 0.0f && (size_t)s_idx[k] >= c0 && (size_t)s_idx[k] < c1) part += p * (logp - s_z[k] * a.inv_tau);
    }
    mass = warp_sum(mass);
    part = warp_sum(part);
    if (lane == 0) {
        out->mass = mass;
        out->part = part;
        out->any = any;
    }
    __syncwarp();
}

template <class T, int THREADS, int MODE>
__global__ void __launch_bounds__(THREADS) distill_kernel(const DistillArgs a) {
    constexpr int W = Row<T>::W, WARPS = THREADS / 32;
    __shared__ int s_idx[MAX_TOP];
    __shared__ float s_p[MAX_TOP], s_z[MAX_TOP];
    __shared__ float s_max[WARPS], s_sum[WARPS];
    __shared__ Teacher s_teacher;
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const size_t t = blockIdx.x;
    const T* z = static_cast<const T*>(a.logits) + t * a.stride;
    T* dz = MODE == MODE_LOSS ? nullptr : static_cast<T*>(a.grad) + t * a.grad_stride;
    const Row<T> row(z, a.V);
    const bool aligned = MODE != MODE_LOSS && ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(dz)) & 15u) == 0;
    const size_t n = row.vectors();
    const float c = a.inv_tau * LOG2E;
    float weight = a.weight != nullptr ? a.weight[t] : 1.0f;
    if (MODE == MODE_GRAD && a.dloss != nullptr) weight *= a.dloss[t];

    if (w == 0) teacher_row<T>(a, t, z, 0, a.V, lane, s_idx, s_p, s_z, &s_teacher);
    float M, S;                          // largest logit, sum of exponentials below it
    if (MODE == MODE_GRAD) {
        __syncthreads();
    } else {
        float m = -INFINITY, s = 0.0f;
        if (weight != 0.0f)
            for (size_t i = tid; i < n; i += THREADS) {
                float x[W];
                unpack<T, W>(row.load(i), x);
                float top = x[0];
#pragma unroll
                for (int e = 1; e < W; ++e) top = fmaxf(top, x[e]);
                const float m2 = fmaxf(m, top);
                const Below below(c, m2);
                float add = 0.0f;
#pragma unroll
                for (int e = 0; e < W; ++e) add += below(x[e]);
                s = s * ex2((m - below.m) * c) + add;
                m = m2;
            }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) join(m, s, __shfl_xor_sync(0xffffffffu, m, d), __shfl_xor_sync(0xffffffffu, s, d), c);
        if (lane == 0) { s_max[w] = m; s_sum[w] = s; }
        __syncthreads();
        M = s_max[0];
        S = s_sum[0];
        for (int q = 1; q < WARPS; ++q) join(M, S, s_max[q], s_sum[q], c);
    }
    const float mass = s_teacher.mass, lse = MODE == MODE_GRAD ? a.lse[t] : fmaf(M, a.inv_tau, logf(S));
    const bool skip = weight == 0.0f || s_teacher.any == 0 || (MODE == MODE_GRAD ? lse : M) == -INFINITY;   // nothing to learn from this row
    if (MODE != MODE_GRAD && tid == 0) {
        a.loss[t] = skip ? 0.0f : weight * (s_teacher.part + mass * lse);
        a.lse[t] = skip ? -INFINITY : lse;
    }
    if (MODE == MODE_LOSS) return;
    // m exp(u - lse) g = G exp2(c z - off)
    const float g = weight * a.inv_tau;
    float G, off;
    bool fused;
    if (MODE == MODE_GRAD) {                                       // off = lse log2 e, its rounding error moved into G
        off = lse * LOG2E;
        fused = fabsf(off) < 1e38f;
        G = g * mass * (fused ? ex2(-(fmaf(lse, LOG2E, -off) + lse * LOG2E_REST)) : 1.0f);
    } else {
        off = c * M;
        fused = fabsf(off) < 1e38f;
        G = g * mass / S;
    }
    auto scaled = [&](float x) {
        if (fused) return G * ex2(fmaf(x, c, -off));
        return G * ex2(MODE == MODE_GRAD ? fmaf(x, a.inv_tau, -lse) * LOG2E : (x - M) * c);
    };
    for (size_t i = tid; i < n; i += THREADS) {
        float x[W];
        if (skip) {
#pragma unroll
            for (int e = 0; e < W; ++e) x[e] = 0.0f;
        } else {
            unpack<T, W>(row.load(i), x);
#pragma unroll
            for (int e = 0; e < W; ++e) x[e] = scaled(x[e]);
        }
        store_row<T>(row, dz, aligned, i, x);
    }
    if (skip) return;
    __syncthreads();
    for (int k = tid; k < a.K; k += THREADS) {
        const int i = s_idx[k];
        if (i < 0) continue;
        float p = 0.0f;                                    // an index that is listed twice: both count
        for (int q = 0; q < a.K; ++q) p += s_idx[q] == i ? s_p[q] : 0.0f;
        const float d[1] = {scaled(s_z[k]) - g * p};
        store_vec<T, 1>(dz + i, d);
    }
}

template <int MODE>
int launch_distill(const DistillArgs& a, size_t T, ec_dtype_t dtype, cudaStream_t st) {
    if (dtype == EC_F32) distill_kernel<float, 512, MODE><<<(unsigned)T, 512, 0, st>>>(a);
    else distill_kernel<bf16_t, 512, MODE><<<(unsigned)T, 512, 0, st>>>(a);
    EC_CUDA(cudaGetLastError());
    return EC_OK;
}

int check(const DistillArgs& a, size_t T, ec_dtype_t dtype, ec_index_t index, ec_dtype_t top_dtype, float temperature, int mode) {
    if (T > 0x7ffffffeull || a.V < 1 || a.V > 0x7ffffffeull || a.K < 1 || !(temperature > 0.0f) || !(temperature < INFINITY)) return EC_ERR_INVALID;
    if (a.stride < a.V || (mode != MODE_LOSS && a.grad_stride < a.V) || (index != EC_INDEX_32 && index != EC_INDEX_64)) return EC_ERR_INVALID;
    if (T > 0 && (!a.logits || !a.top_index || !a.top_logit || !a.lse || (mode != MODE_GRAD && !a.loss) || (mode != MODE_LOSS && !a.grad)))
        return EC_ERR_INVALID;
    if (mode != MODE_LOSS && a.grad == a.logits && a.grad_stride != a.stride) return EC_ERR_INVALID;
    if (a.K > EC_DISTILL_MAX_TOP) return EC_ERR_CAPACITY;
    if (!is_real_dtype(dtype) || !is_real_dtype(top_dtype)) return EC_ERR_UNSUPPORTED;
    return EC_OK;
}

DistillArgs pack(const void* logits, size_t stride, size_t V, const void* top_index, ec_index_t index, const void* top_logit,
                 ec_dtype_t top_dtype, int K, float temperature, const float* weight, const float* teacher_lse) {
    DistillArgs a = {};
    a.logits = logits; a.stride = stride; a.V = V;
    a.top_index = top_index; a.index64 = index == EC_INDEX_64;
    a.top_logit = top_logit; a.top_bf16 = top_dtype == EC_BF16;
    a.K = K; a.inv_tau = 1.0f / temperature;
    a.weight = weight; a.teacher_lse = teacher_lse;
    return a;
}

}  // namespace
}  // namespace ec

using namespace ec;

extern "C" {

int ec_distill_loss(const void* logits, size_t logits_stride, ec_dtype_t dtype, size_t T, size_t V, const void* top_index,
                    ec_index_t index, const void* top_logit, ec_dtype_t top_dtype, int K, float temperature, const float* weight,
                    const float* teacher_lse, float* loss, float* lse, ec_stream_t stream) {
    DistillArgs a = pack(logits, logits_stride, V, top_index, index, top_logit, top_dtype, K, temperature, weight, teacher_lse);
    a.loss = loss; a.lse = lse;
    const int rc = check(a, T, dtype, index, top_dtype, temperature, MODE_LOSS);
    return rc != EC_OK || T == 0 ? rc : launch_distill<MODE_LOSS>(a, T, dtype, stream);
}

int ec_distill_grad(const void* logits, size_t logits_stride, ec_dtype_t dtype, size_t T, size_t V, const void* top_index,
                    ec_index_t index, const void* top_logit, ec_dtype_t top_dtype, int K, float temperature, const float* weight,
                    const float* teacher_lse, const float* lse, const float* dloss, void* grad, size_t grad_stride,
                    ec_stream_t stream) {
    DistillArgs a = pack(logits, logits_stride, V, top_index, index, top_logit, top_dtype, K, temperature, weight, teacher_lse);
    a.lse = const_cast<float*>(lse); a.dloss = dloss; a.grad = grad; a.grad_stride = grad_stride;
    const int rc = check(a, T, dtype, index, top_dtype, temperature, MODE_GRAD);
    return rc != EC_OK || T == 0 ? rc : launch_distill<MODE_GRAD>(a, T, dtype, stream);
}

int ec_distill_step(const void* logits, size_t logits_stride, ec_dtype_t dtype, size_t T, size_t V, const void* top_index,
                    ec_index_t index, const void* top_logit, ec_dtype_t top_dtype, int K, float temperature, const float* weight,
                    const float* teacher_lse, float* loss, float* lse, void* grad, size_t grad_stride, ec_stream_t stream) {
    DistillArgs a = pack(logits, logits_stride, V, top_index, index, top_logit, top_dtype, K, temperature, weight, teacher_lse);
    a.loss = loss; a.lse = lse; a.grad = grad; a.grad_stride = grad_stride;
    const int rc = check(a, T, dtype, index, top_dtype, temperature, MODE_STEP);
    return rc != EC_OK || T == 0 ? rc : launch_distill<MODE_STEP>(a, T, dtype, stream);
}

}  // extern "C"
