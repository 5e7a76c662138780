// Rows of logits: log probabilities of given tokens with the entropy and the top alternatives, and
// distillation from a teacher's top logits, with their gradients.
//
// With y = scale * z over a row of V logits, m = max y, s = sum exp(y - m), lse = m + log s and
// p = exp(y - lse):
//   logp     = y_t - lse,   entropy = log s - sum p (y - m),   alternatives: the K largest z
//   d/dz_v   = scale [ g (1[v = t] - p_v) - h p_v (log p_v + entropy) ]
//   distill  = sum_k q_k (log q_k - log p_k) (+ q_T (log q_T - log p_T) for the mass outside the ids)
//   d/dz_v   = weight scale [ p_v (Q + q_T - (q_T / p_T outside the ids)) - q_v ]
// A column at -inf has p = 0 and adds nothing; a row without any other column has lse = -inf.
#include "qs_lm.cuh"

namespace {

using namespace qs;

constexpr int NT = 256;

struct RowArgs {
    long long N, V;
    const void* logits;
    long long stride;
    float scale;
    Ids tok;                       // given tokens (N) or the teacher's ids (N x K)
    int K;                         // alternatives, or ids per row
    float* logp; float* lse; float* entropy;
    void* top_ids; float* top_logp;
    const void* teacher; int teacher_type;
    float teacher_scale;
    int tail;
    float* loss; float* log_tail;
    // gradients
    const float* in_lse; const float* in_entropy; const float* in_log_tail;
    const float* g1; const float* g2;      // of logp and of the entropy; g1: of the loss
    float g_all;                           // where g1 is null
    void* grad; long long grad_stride;
    int* status;
};

struct Stat { float m, s, u; };            // max, sum of e = exp(y - m), sum of e (y - m) in units of log 2

__device__ __forceinline__ Stat join(Stat a, Stat b, float c2) {
    const float m = fmaxf(a.m, b.m);
    if (m == neg_inf()) return Stat{m, a.s + b.s, a.u + b.u};
    const float da = a.m == neg_inf() ? -2000.0f : (a.m - m) * c2, db = b.m == neg_inf() ? -2000.0f : (b.m - m) * c2;
    const float wa = ex2(da), wb = ex2(db);
    return Stat{m, fmaf(a.s, wa, b.s * wb), fmaf(wa, fmaf(a.s, fmaxf(da, -2000.0f), a.u), wb * fmaf(b.s, fmaxf(db, -2000.0f), b.u))};
}

__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

__device__ Stat block_join(Stat v, float c2) {
    __shared__ Stat part[NT / 32];
    for (int o = 16; o; o >>= 1) {
        Stat w{__shfl_xor_sync(~0u, v.m, o), __shfl_xor_sync(~0u, v.s, o), __shfl_xor_sync(~0u, v.u, o)};
        v = join(v, w, c2);
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = part[0];
    for (int w = 1; w < NT / 32; ++w) v = join(v, part[w], c2);
    return v;
}

__device__ float block_sum(float v) {
    __shared__ float part[NT / 32];
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0f;
    for (int w = 0; w < NT / 32; ++w) v += part[w];
    return v;
}

__device__ unsigned long long block_max(unsigned long long v) {
    __shared__ unsigned long long part[NT / 32];
    for (int o = 16; o; o >>= 1) {
        const unsigned long long w = __shfl_xor_sync(~0u, v, o);
        v = w > v ? w : v;
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = part[0];
    for (int w = 1; w < NT / 32; ++w) v = part[w] > v ? part[w] : v;
    return v;
}

// whole number that orders alternatives: larger logit first, then lower index (-0 equals +0)
__device__ __forceinline__ unsigned long long order_key(float z, uint32_t i) {
    const uint32_t b = __float_as_uint(z + 0.0f);
    return ((unsigned long long)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32) | (uint32_t)~i;
}

template <class T, bool SKIP>
__device__ Stat row_stat(const RowArgs& a, const T* z, const uint32_t* ids) {
    const float c2 = a.scale * LOG2E;
    auto skip = [&](long long i) {
        bool found = false;
        for (int k = 0; SKIP && k < a.K; ++k) found |= ids[k] == (uint32_t)i;
        return found;
    };
    float m = neg_inf();
    for (long long i = threadIdx.x; i < a.V; i += NT)
        if (!skip(i)) m = fmaxf(m, to_float(z[i]));
    Stat v{m, 0.0f, 0.0f};
    for (long long i = threadIdx.x; i < a.V; i += NT) {
        if (skip(i)) continue;
        const float f = to_float(z[i]);
        const float y = m == neg_inf() ? f + (f == f ? neg_inf() : f) : (f - m) * c2;
        const float yc = max_nan(y, -2000.0f), e = ex2(yc);
        v.s += e;
        v.u = fmaf(e, yc, v.u);
    }
    return block_join(v, c2);
}

template <class T>
__global__ void __launch_bounds__(NT) token_logp_kernel(const RowArgs a) {
    for (long long n = blockIdx.x; n < a.N; n += gridDim.x) {
        const T* z = static_cast<const T*>(a.logits) + n * a.stride;
        const Stat v = row_stat<T, false>(a, z, nullptr);
        const bool empty = v.m == neg_inf() && v.s == v.s && v.s == 0.0f;
        const float ls = logf(v.s);
        const float lse = empty ? neg_inf() : fmaf(v.m, a.scale, ls);
        if (threadIdx.x == 0) {
            if (a.lse) a.lse[n] = lse;
            if (a.entropy) a.entropy[n] = empty ? 0.0f : ls - LN2 * (v.u / v.s);
            if (a.logp) {
                const long long t = a.tok.at(n);
                float lp = 0.0f;
                if (t >= a.V) {
                    flag_status(a.status, QS_INVALID_ARG);
                    lp = quiet_nan();
                } else if (t >= 0) {
                    lp = empty ? neg_inf() : (to_float(z[t]) - v.m) * a.scale - ls;
                }
                a.logp[n] = lp;
            }
        }
        unsigned long long last = ~0ull;
        for (int k = 0; k < a.K; ++k) {
            unsigned long long best = 0;
            for (long long i = threadIdx.x; i < a.V; i += NT) {
                const float f = to_float(z[i]);
                if (!(f > neg_inf())) continue;
                const unsigned long long key = order_key(f, (uint32_t)i);
                if (key < last && key > best) best = key;
            }
            best = block_max(best);
            last = best;
            if (threadIdx.x == 0) {
                const bool none = best == 0 || !(lse == lse);
                const uint32_t i = ~(uint32_t)best;
                const long long id = none ? -1 : (long long)i;
                if (a.tok.wide) static_cast<long long*>(a.top_ids)[n * a.K + k] = id;
                else static_cast<int*>(a.top_ids)[n * a.K + k] = (int)id;
                a.top_logp[n * a.K + k] = !(lse == lse) ? lse : none ? neg_inf() : (to_float(z[i]) - v.m) * a.scale - ls;
            }
        }
        __syncthreads();
    }
}

template <class T>
__global__ void __launch_bounds__(NT) token_logp_grad_kernel(const RowArgs a) {
    for (long long n = blockIdx.x; n < a.N; n += gridDim.x) {
        const T* z = static_cast<const T*>(a.logits) + n * a.stride;
        T* out = static_cast<T*>(a.grad) + n * a.grad_stride;
        const long long t = a.tok.p ? a.tok.at(n) : -1;
        const float g = t < 0 ? 0.0f : t >= a.V ? quiet_nan() : a.g1 ? a.g1[n] : a.g_all;
        const float h = a.g2 ? a.g2[n] : 0.0f, ent = a.g2 ? a.in_entropy[n] : 0.0f, lse = a.in_lse[n];
        if (t >= a.V && threadIdx.x == 0) flag_status(a.status, QS_INVALID_ARG);
        for (long long i = threadIdx.x; i < a.V; i += NT) {
            const float lc = max_nan(fmaf(to_float(z[i]), a.scale, -lse), -1400.0f), p = ex2(lc * LOG2E);
            float d = -p * fmaf(h, lc + ent, g);
            if (i == t) d += g;
            out[i] = from_float<T>(lse == neg_inf() ? (t < a.V ? 0.0f : g) : d * a.scale);
        }
    }
}

__device__ __forceinline__ float teacher_at(const RowArgs& a, long long i) {
    return a.teacher_type == QS_F32 ? static_cast<const float*>(a.teacher)[i]
         : a.teacher_type == QS_BF16 ? to_float(static_cast<const __nv_bfloat16*>(a.teacher)[i])
                                     : to_float(static_cast<const __half*>(a.teacher)[i]);
}

struct Teacher { float Q, rest; bool bad; };

// q[k], log q[k] and the ids of a row into shared memory; ids that name no column become NO_ID
constexpr uint32_t NO_ID = 0xffffffffu;
__device__ Teacher load_teacher(const RowArgs& a, long long n, float* q, float* logq, uint32_t* ids) {
    __syncthreads();
    __shared__ int bad;
    if (threadIdx.x == 0) bad = 0;
    __syncthreads();
    for (int k = threadIdx.x; k < a.K; k += NT) {
        const long long id = a.tok.at(n * a.K + k);
        if (id >= a.V) { bad = 1; flag_status(a.status, QS_INVALID_ARG); }
        ids[k] = id < 0 || id >= a.V ? NO_ID : (uint32_t)id;
        logq[k] = ids[k] == NO_ID ? neg_inf() : teacher_at(a, n * a.K + k) * a.teacher_scale;
    }
    __syncthreads();
    float m = neg_inf(), total = 0.0f;
    if (a.tail) m = 0.0f;
    else for (int k = 0; k < a.K; ++k) m = fmaxf(m, logq[k]);
    for (int k = 0; k < a.K; ++k) total += logq[k] == neg_inf() ? 0.0f : ex2((logq[k] - m) * LOG2E);
    const float lt = logf(total);
    __syncthreads();
    for (int k = threadIdx.x; k < a.K; k += NT) {
        const float l = logq[k];
        const float v = l == neg_inf() ? l : a.tail ? l : l - m - lt;
        logq[k] = v;
        q[k] = v == neg_inf() ? 0.0f : ex2(v * LOG2E);
    }
    __syncthreads();
    Teacher t{0.0f, 0.0f, bad != 0};
    for (int k = 0; k < a.K; ++k) t.Q += q[k];
    if (a.tail) t.rest = t.Q == t.Q ? fmaxf(0.0f, 1.0f - t.Q) : t.Q;
    return t;
}

// the gradient row: p = exp(scale * z - m_scaled) / s with the two parts of lse apart
template <class T>
__device__ void distill_row_grad(const RowArgs& a, long long n, const T* z, const Teacher& t, const float* q, const uint32_t* ids,
                                 float m, float ls, float lse, float log_tail, bool split) {
    T* out = static_cast<T*>(a.grad) + n * a.grad_stride;
    const float w = (a.g1 ? a.g1[n] : a.g_all) * a.scale;
    const float in = t.bad ? quiet_nan() : t.Q + t.rest;
    // p q_T / p_T: from the ratio q_T / p_T, or exponent by exponent where p_T is too small for it
    const bool thin = a.tail && t.rest > 0.0f && log_tail < -60.0f;
    const float ratio = t.rest > 0.0f && !thin ? t.rest * ex2(-log_tail * LOG2E) : t.rest;
    for (long long i = threadIdx.x; i < a.V; i += NT) {
        const float f = to_float(z[i]);
        const float lp = split ? (f - m) * a.scale - ls : fmaf(f, a.scale, -lse);
        const float p = ex2(lp * LOG2E);
        float qv = 0.0f;
        bool member = false;
        for (int k = 0; k < a.K; ++k)
            if (ids[k] == (uint32_t)i) { qv += q[k]; member = true; }
        float d = p * (member ? in : thin ? in : in - ratio) - qv;
        if (thin && !member && log_tail > neg_inf()) d -= ratio * ex2((lp - log_tail) * LOG2E);
        if (lse == neg_inf()) d = t.bad ? in : 0.0f;
        out[i] = from_float<T>(w * d);
    }
}

template <class T>
__global__ void __launch_bounds__(NT) distill_kernel(const RowArgs a) {
    __shared__ float q[QS_MAX_TOP], logq[QS_MAX_TOP];
    __shared__ uint32_t ids[QS_MAX_TOP];
    for (long long n = blockIdx.x; n < a.N; n += gridDim.x) {
        const T* z = static_cast<const T*>(a.logits) + n * a.stride;
        const Teacher t = load_teacher(a, n, q, logq, ids);
        const Stat v = row_stat<T, false>(a, z, nullptr);
        const bool empty = v.m == neg_inf() && v.s == 0.0f;
        const float ls = logf(v.s), lse = empty ? neg_inf() : fmaf(v.m, a.scale, ls);
        float log_tail = 0.0f;
        if (a.tail) {
            const Stat o = row_stat<T, true>(a, z, ids);
            float in = 0.0f;                     // the named columns' share, each once
            for (int k = threadIdx.x; k < a.K; k += NT) {
                bool first = ids[k] != NO_ID;
                for (int j = 0; j < k; ++j) first &= ids[j] != ids[k];
                if (first) in += ex2((to_float(z[ids[k]]) - v.m) * a.scale * LOG2E);
            }
            in = block_sum(in);
            const bool none = empty || (o.m == neg_inf() && o.s == 0.0f);
            log_tail = none ? neg_inf() : (o.m - v.m) * a.scale + logf(o.s) - ls;
            // near 1 the difference of the two logs would cancel
            if (log_tail > -0.5f) log_tail = -log1pf(in / (o.s * ex2((o.m - v.m) * a.scale * LOG2E)));
        }
        float part = 0.0f;
        for (int k = threadIdx.x; k < a.K; k += NT) {
            if (ids[k] == NO_ID || q[k] == 0.0f) continue;
            const float lp = empty ? neg_inf() : (to_float(z[ids[k]]) - v.m) * a.scale - ls;
            part += q[k] * (logq[k] - lp);
        }
        float loss = block_sum(part);
        if (a.tail && t.rest != 0.0f) loss += t.rest * (logf(t.rest) - log_tail);
        if (t.bad) loss = quiet_nan();
        if (threadIdx.x == 0) {
            if (a.loss) a.loss[n] = loss;
            if (a.lse) a.lse[n] = lse;
            if (a.tail && a.log_tail) a.log_tail[n] = log_tail;
        }
        __syncthreads();
        if (a.grad) distill_row_grad<T>(a, n, z, t, q, ids, v.m, ls, lse, log_tail, true);
    }
}

template <class T>
__global__ void __launch_bounds__(NT) distill_grad_kernel(const RowArgs a) {
    __shared__ float q[QS_MAX_TOP], logq[QS_MAX_TOP];
    __shared__ uint32_t ids[QS_MAX_TOP];
    for (long long n = blockIdx.x; n < a.N; n += gridDim.x) {
        const T* z = static_cast<const T*>(a.logits) + n * a.stride;
        const Teacher t = load_teacher(a, n, q, logq, ids);
        distill_row_grad<T>(a, n, z, t, q, ids, 0.0f, 0.0f, a.in_lse[n], a.tail ? a.in_log_tail[n] : 0.0f, false);
    }
}

#define QS_LAUNCH_BY_TYPE(kernel, type, grid, st, args)                                   \
    do {                                                                                  \
        if ((type) == QS_F32) kernel<float><<<grid, NT, 0, st>>>(args);                   \
        else if ((type) == QS_BF16) kernel<__nv_bfloat16><<<grid, NT, 0, st>>>(args);     \
        else kernel<__half><<<grid, NT, 0, st>>>(args);                                   \
    } while (0)

bool bad_rows(int64_t N, int64_t V, int type, int64_t stride, float scale) {
    return N < 0 || V < 1 || !size_of_type(type) || stride < V || !(scale > 0.0f) || !std::isfinite(scale);
}
bool rows_too_large(int64_t N, int64_t V) { return N > (1ll << 30) || V > (1ll << 30); }
bool ok_floats(const void* p) { return aligned_to(p, 4); }

// the gradient may take the logits' own place, row for row; any other overlap is refused
bool overlap(const void* z, int64_t stride, const void* g, int64_t g_stride, int64_t N, int64_t V, int size) {
    const uintptr_t z0 = reinterpret_cast<uintptr_t>(z), g0 = reinterpret_cast<uintptr_t>(g);
    if (z0 == g0 && stride == g_stride) return false;
    const uintptr_t z1 = z0 + ((N - 1) * stride + V) * size, g1 = g0 + ((N - 1) * g_stride + V) * size;
    return z0 < g1 && g0 < z1;
}

}  // namespace

extern "C" {

int qs_token_logp(int64_t N, int64_t V, const void* logits, int type, int64_t row_stride, const void* tokens, int token_type,
                  float scale, int top, float* logp, float* lse, float* entropy, void* top_ids, float* top_logp, int* status,
                  void* cuda_stream) {
    if (bad_rows(N, V, type, row_stride, scale) || !is_id_type(token_type) || top < 0 || top > QS_MAX_TOP || top > V) return QS_INVALID_ARG;
    if (rows_too_large(N, V)) return QS_TOO_LARGE;
    if (N == 0) return QS_OK;
    const int id_bytes = token_type == QS_I64 ? 8 : 4;
    if (!logits || !aligned_to(logits, size_of_type(type)) || (logp && !tokens) || !aligned_to(tokens, id_bytes) || !ok_floats(logp) ||
        !ok_floats(lse) || !ok_floats(entropy) || !ok_floats(status) ||
        (top && (!top_ids || !top_logp || !aligned_to(top_ids, id_bytes) || !ok_floats(top_logp)))) return QS_INVALID_ARG;
    RowArgs a{};
    a.N = N; a.V = V; a.logits = logits; a.stride = row_stride; a.scale = scale;
    a.tok = Ids{tokens, token_type == QS_I64}; a.K = top;
    a.logp = logp; a.lse = lse; a.entropy = entropy; a.top_ids = top_ids; a.top_logp = top_logp; a.status = status;
    const int grid = (int)(N < 65536 ? N : 65536);
    QS_LAUNCH_BY_TYPE(token_logp_kernel, type, grid, static_cast<cudaStream_t>(cuda_stream), a);
    return launch_status();
}

int qs_token_logp_grad(int64_t N, int64_t V, const void* logits, int type, int64_t row_stride, const void* tokens, int token_type,
                       float scale, const float* lse, const float* entropy, const float* grad_logp, float grad_logp_all,
                       const float* grad_entropy, void* grad, int64_t grad_stride, int* status, void* cuda_stream) {
    if (bad_rows(N, V, type, row_stride, scale) || !is_id_type(token_type) || grad_stride < V) return QS_INVALID_ARG;
    if (rows_too_large(N, V)) return QS_TOO_LARGE;
    if (N == 0) return QS_OK;
    const int size = size_of_type(type);
    if (!logits || !grad || !lse || (grad_entropy && !entropy) || !aligned_to(logits, size) || !aligned_to(grad, size) ||
        !aligned_to(tokens, token_type == QS_I64 ? 8 : 4) || !ok_floats(lse) || !ok_floats(entropy) || !ok_floats(grad_logp) ||
        !ok_floats(grad_entropy) || !ok_floats(status) || overlap(logits, row_stride, grad, grad_stride, N, V, size)) return QS_INVALID_ARG;
    RowArgs a{};
    a.N = N; a.V = V; a.logits = logits; a.stride = row_stride; a.scale = scale;
    a.tok = Ids{tokens, token_type == QS_I64};
    a.in_lse = lse; a.in_entropy = entropy; a.g1 = grad_logp; a.g_all = grad_logp_all; a.g2 = grad_entropy;
    a.grad = grad; a.grad_stride = grad_stride; a.status = status;
    const int grid = (int)(N < 65536 ? N : 65536);
    QS_LAUNCH_BY_TYPE(token_logp_grad_kernel, type, grid, static_cast<cudaStream_t>(cuda_stream), a);
    return launch_status();
}

int qs_distill(int64_t N, int64_t V, int K, const void* logits, int type, int64_t row_stride, const void* ids, int id_type,
               const void* teacher, int teacher_type, float scale, float teacher_scale, int tail, float* loss, float* lse,
               float* log_tail, const float* weight, float weight_all, void* grad, int64_t grad_stride, int* status, void* cuda_stream) {
    if (bad_rows(N, V, type, row_stride, scale) || !is_id_type(id_type) || !size_of_type(teacher_type) || K < 1 || K > QS_MAX_TOP ||
        !std::isfinite(teacher_scale) || (grad && grad_stride < V)) return QS_INVALID_ARG;
    if (rows_too_large(N, V)) return QS_TOO_LARGE;
    if (N == 0) return QS_OK;
    const int size = size_of_type(type);
    if (!logits || !ids || !teacher || !aligned_to(logits, size) || !aligned_to(ids, id_type == QS_I64 ? 8 : 4) ||
        !aligned_to(teacher, size_of_type(teacher_type)) || !ok_floats(loss) || !ok_floats(lse) || !ok_floats(log_tail) || !ok_floats(weight) ||
        !ok_floats(status) || (grad && (!aligned_to(grad, size) || overlap(logits, row_stride, grad, grad_stride, N, V, size)))) return QS_INVALID_ARG;
    RowArgs a{};
    a.N = N; a.V = V; a.logits = logits; a.stride = row_stride; a.scale = scale;
    a.tok = Ids{ids, id_type == QS_I64}; a.K = K; a.teacher = teacher; a.teacher_type = teacher_type; a.teacher_scale = teacher_scale;
    a.tail = tail != 0; a.loss = loss; a.lse = lse; a.log_tail = log_tail; a.g1 = weight; a.g_all = weight_all;
    a.grad = grad; a.grad_stride = grad_stride; a.status = status;
    const int grid = (int)(N < 65536 ? N : 65536);
    QS_LAUNCH_BY_TYPE(distill_kernel, type, grid, static_cast<cudaStream_t>(cuda_stream), a);
    return launch_status();
}

int qs_distill_grad(int64_t N, int64_t V, int K, const void* logits, int type, int64_t row_stride, const void* ids, int id_type,
                    const void* teacher, int teacher_type, float scale, float teacher_scale, int tail, const float* lse,
                    const float* log_tail, const float* weight, float weight_all, void* grad, int64_t grad_stride, int* status,
                    void* cuda_stream) {
    if (bad_rows(N, V, type, row_stride, scale) || !is_id_type(id_type) || !size_of_type(teacher_type) || K < 1 || K > QS_MAX_TOP ||
        !std::isfinite(teacher_scale) || grad_stride < V) return QS_INVALID_ARG;
    if (rows_too_large(N, V)) return QS_TOO_LARGE;
    if (N == 0) return QS_OK;
    const int size = size_of_type(type);
    if (!logits || !ids || !teacher || !lse || (tail && !log_tail) || !grad || !aligned_to(logits, size) ||
        !aligned_to(ids, id_type == QS_I64 ? 8 : 4) || !aligned_to(teacher, size_of_type(teacher_type)) || !ok_floats(lse) ||
        !ok_floats(log_tail) || !ok_floats(weight) || !ok_floats(status) || !aligned_to(grad, size) ||
        overlap(logits, row_stride, grad, grad_stride, N, V, size)) return QS_INVALID_ARG;
    RowArgs a{};
    a.N = N; a.V = V; a.logits = logits; a.stride = row_stride; a.scale = scale;
    a.tok = Ids{ids, id_type == QS_I64}; a.K = K; a.teacher = teacher; a.teacher_type = teacher_type; a.teacher_scale = teacher_scale;
    a.tail = tail != 0; a.in_lse = lse; a.in_log_tail = log_tail; a.g1 = weight; a.g_all = weight_all;
    a.grad = grad; a.grad_stride = grad_stride; a.status = status;
    const int grid = (int)(N < 65536 ? N : 65536);
    QS_LAUNCH_BY_TYPE(distill_grad_kernel, type, grid, static_cast<cudaStream_t>(cuda_stream), a);
    return launch_status();
}

}  // extern "C"
