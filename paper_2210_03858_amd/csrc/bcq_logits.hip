// Operators on logits: log probabilities of given tokens with entropy and the best alternatives, distillation from a
// teacher's top logits, and their gradients.  Formulas and conventions: include/bcq.h.
//
// One workgroup takes one row and walks it once per quantity (maximum, sums, gradient; one walk per alternative).
#include "../../include/bcq.h"

#include "bcq_internal.h"

#include <math.h>

namespace bcq {

constexpr int LG_THREADS = 256;
constexpr float LG_LOG2E = 1.4426950408889634f;
constexpr float LG_LN2 = 0.6931471805599453f;
constexpr int LG_SEGMENT = 65536;  // columns whose list membership one bitmap holds

__device__ __forceinline__ float lg_exp2(float v) { return __builtin_amdgcn_exp2f(v); }

// A float as an unsigned number of the same order (-0 as +0); 0 is below every number.  NaN is not passed in.
__device__ __forceinline__ uint32_t lg_key(float v) {
    const uint32_t u = __float_as_uint(v + 0.0f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

template <typename V, typename F>
__device__ __forceinline__ V lg_block_reduce(V v, F op, V* lds) {
    const int tid = threadIdx.x;
    __syncthreads();
    lds[tid] = v;
    __syncthreads();
    for (int s = LG_THREADS / 2; s > 0; s >>= 1) {
        if (tid < s) lds[tid] = op(lds[tid], lds[tid + s]);
        __syncthreads();
    }
    return lds[0];
}
__device__ __forceinline__ float lg_add(float a, float b) { return a + b; }
__device__ __forceinline__ float lg_max(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ uint64_t lg_max64(uint64_t a, uint64_t b) { return a > b ? a : b; }

struct LogprobsOut {
    float *logp, *entropy, *lse, *stats, *top_logit, *top_logp;
    int32_t* top_index;
};

template <typename XT>
__global__ __launch_bounds__(LG_THREADS) void logprobs_kernel(const XT* __restrict__ x, int64_t stride, int V,
                                                              const int64_t* __restrict__ tokens, float c, int k, LogprobsOut out) {
    __shared__ float lds[LG_THREADS];
    __shared__ uint64_t lds64[LG_THREADS];
    const int64_t t = blockIdx.x;
    const int tid = threadIdx.x;
    const XT* row = x + t * stride;
    const float c2 = c * LG_LOG2E;
    const int64_t token = tokens ? tokens[t] : -1;
    if (token < 0 && !out.entropy && !out.lse && k == 0) {
        if (tid == 0) {
            if (out.logp) out.logp[t] = 0.f;
            if (out.stats) out.stats[2 * t] = out.stats[2 * t + 1] = 0.f;
        }
        return;
    }
    float m = -INFINITY;
    for (int i = tid; i < V; i += LG_THREADS) m = fmaxf(m, Elem<XT>::load(row + i));
    m = lg_block_reduce(m, lg_max, lds);
    if (m == -INFINITY) m = 0.f;
    float S = 0.f, E = 0.f;
    for (int i = tid; i < V; i += LG_THREADS) {
        const float d = (Elem<XT>::load(row + i) - m) * c2, e = lg_exp2(d);
        S += e;
        E += e * fmaxf(d, -1e4f);
    }
    S = lg_block_reduce(S, lg_add, lds);
    E = lg_block_reduce(E, lg_add, lds);
    const float l2 = log2f(S);  // -inf: nothing left
    if (tid == 0) {
        if (out.logp) {
            float v = 0.f;
            if (token >= V) v = NAN;
            else if (token >= 0) v = S == 0.f ? -INFINITY : (Elem<XT>::load(row + token) - m) * c - l2 * LG_LN2;
            out.logp[t] = v;
        }
        if (out.entropy) out.entropy[t] = S == 0.f ? 0.f : (l2 - E / S) * LG_LN2;
        if (out.lse) out.lse[t] = S == 0.f ? -INFINITY : m * c + l2 * LG_LN2;
        if (out.stats) {
            out.stats[2 * t] = m;
            out.stats[2 * t + 1] = l2;
        }
    }
    uint64_t below = ~(uint64_t)0;
    for (int r = 0; r < k; ++r) {
        uint64_t best = 0;
        for (int i = tid; i < V; i += LG_THREADS) {
            const float v = Elem<XT>::load(row + i);
            if (v == v) {
                const uint64_t key = ((uint64_t)lg_key(v) << 32) | (uint32_t)~i;
                if (key < below) best = lg_max64(best, key);
            }
        }
        best = lg_block_reduce(best, lg_max64, lds64);
        below = best;
        if (tid == 0) {
            const int i = best ? (int)~(uint32_t)best : -1;
            const float v = best ? Elem<XT>::load(row + i) : -INFINITY;
            if (out.top_index) out.top_index[t * k + r] = i;
            if (out.top_logit) out.top_logit[t * k + r] = v;
            if (out.top_logp) out.top_logp[t * k + r] = S == 0.f ? -INFINITY : (v - m) * c - l2 * LG_LN2;
        }
    }
}

template <typename XT>
__global__ __launch_bounds__(LG_THREADS) void logprobs_bwd_kernel(const XT* x, int64_t stride, int V,
                                                                  const int64_t* __restrict__ tokens, float c,
                                                                  const float* __restrict__ stats, const float* __restrict__ dlogp,
                                                                  const float* __restrict__ entropy,
                                                                  const float* __restrict__ dentropy, XT* dx, int64_t dstride) {
    const int64_t t = blockIdx.x;
    const int tid = threadIdx.x;
    const XT* row = x + t * stride;
    XT* drow = dx + t * dstride;
    const int64_t token = tokens ? tokens[t] : -1;
    float g = token >= 0 ? dlogp[t] : 0.f;
    const float h = dentropy ? dentropy[t] : 0.f;
    const float m = stats[2 * t], l2 = stats[2 * t + 1];
    if ((g == 0.f && h == 0.f) || l2 == -INFINITY) {
        for (int i = tid; i < V; i += LG_THREADS) Elem<XT>::store(drow + i, 0.f);
        return;
    }
    if (token >= V) g = NAN;
    const float c2 = c * LG_LOG2E;
    // dx = q (A + B ln2 log2 q) with log2 q = (x - m) c2 - l2
    const float A = -c * (g + (h != 0.f ? h * entropy[t] : 0.f)), B = -c * h * LG_LN2;
    for (int i = tid; i < V; i += LG_THREADS) {
        const float d = (Elem<XT>::load(row + i) - m) * c2 - l2, q = lg_exp2(d);
        float v = q * (A + B * fmaxf(d, -1e4f));
        if (i == token) v += c * g;
        Elem<XT>::store(drow + i, v);
    }
}

// ---- distillation -----------------------------------------------------------------------------------------------
// The teacher's side of a row and the student's logits at the list, one entry per thread (k <= LG_THREADS / 2).
struct ListLds {
    int index[BCQ_LOGITS_MAX_K];
    double p[BCQ_LOGITS_MAX_K], lp[BCQ_LOGITS_MAX_K];
    float s[BCQ_LOGITS_MAX_K];
    double sum[4];  // sum of p; sum of p ln p; entries; invalid entries
};

template <typename XT>
__device__ void lg_load_list(ListLds& L, const XT* row, int V, const float* __restrict__ z, const int32_t* __restrict__ index,
                             int k, const float* __restrict__ teacher_lse, double c) {
    const int tid = threadIdx.x;
    __syncthreads();
    if (tid < k) {
        L.index[tid] = index[tid];
        L.lp[tid] = (double)z[tid] * c;
        L.s[tid] = L.index[tid] >= 0 && L.index[tid] < V ? Elem<XT>::load(row + L.index[tid]) : -INFINITY;
    }
    __syncthreads();
    if (tid == 0) {
        double top = -INFINITY, sum = 0.0;
        for (int i = 0; i < k; ++i)
            if (L.index[i] >= 0) top = L.lp[i] > top || L.lp[i] != L.lp[i] ? L.lp[i] : top;
        if (top == -INFINITY) top = 0.0;
        double norm = teacher_lse ? (double)*teacher_lse : 0.0;
        if (!teacher_lse) {
            for (int i = 0; i < k; ++i) sum += L.index[i] >= 0 ? exp(L.lp[i] - top) : 0.0;
            norm = sum > 0.0 || sum != sum ? top + log(sum) : 0.0;
        }
        double P = 0.0, H = 0.0, count = 0.0, bad = 0.0;
        for (int i = 0; i < k; ++i) {
            const double lp = L.lp[i] - norm, p = L.index[i] >= 0 ? exp(lp) : 0.0;
            L.lp[i] = lp;
            L.p[i] = p;
            P += p;
            if (p != 0.0) H += p * lp;
            count += L.index[i] >= 0;
            bad += L.index[i] >= V;
        }
        L.sum[0] = P;
        L.sum[1] = H;
        L.sum[2] = count;
        L.sum[3] = bad;
    }
    __syncthreads();
}

// Sets the bits of the listed columns of [first, first + LG_SEGMENT) in bits
__device__ void lg_mark(uint32_t* bits, const ListLds& L, int k, int first) {
    __syncthreads();
    for (int w = threadIdx.x; w < LG_SEGMENT / 32; w += LG_THREADS) bits[w] = 0;
    __syncthreads();
    if ((int)threadIdx.x < k) {
        const int i = L.index[threadIdx.x] - first;
        if (L.index[threadIdx.x] >= 0 && i >= 0 && i < LG_SEGMENT) atomicOr(bits + i / 32, 1u << (i % 32));
    }
    __syncthreads();
}

// stats of a row: shift m and factor f of the unlisted entries' gradient f 2^((x - m) c2); shift and log2 of the sum of all
// entries.  Without a rest every entry counts as unlisted for m, and f = P / (S c).
template <typename XT>
__global__ __launch_bounds__(LG_THREADS) void distill_kernel(const XT* __restrict__ x, int64_t stride, int V,
                                                             const float* __restrict__ top_logit, const int32_t* __restrict__ top_index,
                                                             int k, const float* __restrict__ teacher_lse, float c,
                                                             const float* __restrict__ weight, float* __restrict__ loss,
                                                             float* __restrict__ stats) {
    __shared__ float lds[LG_THREADS];
    __shared__ ListLds L;
    __shared__ uint32_t bits[LG_SEGMENT / 32];
    const int64_t t = blockIdx.x;
    const int tid = threadIdx.x;
    const XT* row = x + t * stride;
    const float c2 = c * LG_LOG2E;
    const bool rest = teacher_lse != nullptr;
    if (weight && weight[t] == 0.f) {
        if (tid == 0) loss[t] = 0.f;
        return;
    }
    lg_load_list(L, row, V, top_logit + t * k, top_index + t * k, k, rest ? teacher_lse + t : nullptr, (double)c);
    float m = -INFINITY;
    for (int first = 0; first < V; first += LG_SEGMENT) {
        if (rest) lg_mark(bits, L, k, first);
        const int last = V - first < LG_SEGMENT ? V : first + LG_SEGMENT;
        for (int i = first + tid; i < last; i += LG_THREADS)
            if (!rest || !((bits[(i - first) / 32] >> ((i - first) % 32)) & 1u)) m = fmaxf(m, Elem<XT>::load(row + i));
    }
    m = lg_block_reduce(m, lg_max, lds);
    float m_all = m;
    if (m == -INFINITY) m = 0.f;
    float S = 0.f;
    for (int first = 0; first < V; first += LG_SEGMENT) {
        if (rest) lg_mark(bits, L, k, first);
        const int last = V - first < LG_SEGMENT ? V : first + LG_SEGMENT;
        for (int i = first + tid; i < last; i += LG_THREADS)
            if (!rest || !((bits[(i - first) / 32] >> ((i - first) % 32)) & 1u)) S += lg_exp2((Elem<XT>::load(row + i) - m) * c2);
    }
    S = lg_block_reduce(S, lg_add, lds);
    if (tid != 0) return;
    double S_all = S;
    int distinct = 0;
    if (rest)
        for (int i = 0; i < k; ++i) m_all = fmaxf(m_all, L.s[i]);
    if (m_all == -INFINITY) m_all = 0.f;
    if (rest) {
        S_all = S == 0.f ? 0.0 : (double)S * exp2((double)((m - m_all) * c2));
        for (int i = 0; i < k; ++i) {
            bool twice = L.index[i] < 0;
            for (int j = 0; j < i; ++j) twice |= L.index[j] == L.index[i];
            if (twice) continue;
            ++distinct;
            S_all += exp2((double)((L.s[i] - m_all) * c2));
        }
    }
    const double l_all = S_all == 0.0 ? 0.0 : log(S_all);
    double r = rest && distinct < V ? 1.0 - L.sum[0] : 0.0;
    if (r < 0.0) r = 0.0;
    double value = L.sum[1], factor = L.sum[0] / S_all;
    for (int i = 0; i < k; ++i)
        if (L.p[i] != 0.0) value -= L.p[i] * ((double)(L.s[i] - m_all) * c - l_all);
    if (rest) {
        const double lrest = log((double)S) + (double)((m - m_all) * c2) * M_LN2 - l_all;
        if (r != 0.0) value += r * (log(r) - lrest);
        factor = S == 0.f ? 0.0 : (exp(lrest) - r) / S;
    }
    factor /= c;
    value /= (double)c * c;
    double l2 = l_all * M_LOG2E;
    if (S_all == 0.0) {  // nothing left
        factor = 0.0;
        l2 = -INFINITY;
    }
    if (L.sum[2] == 0.0) {
        value = factor = 0.0;
    } else if (L.sum[3] != 0.0) {
        value = factor = l2 = NAN;
    }
    loss[t] = (float)value;
    if (stats) {
        stats[4 * t] = m;
        stats[4 * t + 1] = (float)factor;
        stats[4 * t + 2] = m_all;
        stats[4 * t + 3] = (float)l2;
    }
}

template <typename XT>
__global__ __launch_bounds__(LG_THREADS) void distill_bwd_kernel(const XT* x, int64_t stride, int V, const float* __restrict__ top_logit,
                                                                 const int32_t* __restrict__ top_index, int k,
                                                                 const float* __restrict__ teacher_lse, float c,
                                                                 const float* __restrict__ stats, const float* __restrict__ weight,
                                                                 XT* dx, int64_t dstride) {
    __shared__ ListLds L;
    const int64_t t = blockIdx.x;
    const int tid = threadIdx.x;
    const XT* row = x + t * stride;
    XT* drow = dx + t * dstride;
    const float c2 = c * LG_LOG2E;
    const float w = weight ? weight[t] : 1.f;
    if (w == 0.f) {
        for (int i = tid; i < V; i += LG_THREADS) Elem<XT>::store(drow + i, 0.f);
        return;
    }
    lg_load_list(L, row, V, top_logit + t * k, top_index + t * k, k, teacher_lse ? teacher_lse + t : nullptr, (double)c);
    const float m = stats[4 * t], f = w * stats[4 * t + 1], m_all = stats[4 * t + 2], l2 = stats[4 * t + 3];
    for (int i = tid; i < V; i += LG_THREADS) {
        const float e = lg_exp2((Elem<XT>::load(row + i) - m) * c2);
        Elem<XT>::store(drow + i, f == 0.f ? 0.f : f * e);
    }
    __syncthreads();
    if (tid < k && L.index[tid] >= 0 && L.index[tid] < V) {
        double p = 0.0;
        for (int j = 0; j < k; ++j)
            if (L.index[j] == L.index[tid]) p += L.p[j];
        const double q = exp2((double)((L.s[tid] - m_all) * c2) - (double)l2);
        const double P = teacher_lse ? 1.0 : L.sum[0];
        Elem<XT>::store(drow + L.index[tid], l2 == -INFINITY ? 0.f : (float)((P * q - p) * w / c));
    }
}

}  // namespace bcq

// ---- C entry points -----------------------------------------------------------------------------------------------
namespace {

bcq_status check_logits(int64_t T, int64_t V, int64_t stride, int k, float temperature) {
    if (T < 0 || T > bcq::host::kMaxTokens || V < 1 || V > BCQ_LOGITS_MAX_V || stride < V) return BCQ_ERR_SHAPE;
    if (stride > bcq::host::kMaxElems || (T > 0 && stride > bcq::host::kMaxElems / T)) return BCQ_ERR_SHAPE;
    if (k < 0 || k > BCQ_LOGITS_MAX_K) return BCQ_ERR_SHAPE;
    if (!(temperature > 0.f) || !isfinite(temperature) || !isfinite(1.0f / temperature)) return BCQ_ERR_SHAPE;
    return BCQ_OK;
}
bool dtype_ok(int dtype) { return dtype == BCQ_F32 || dtype == BCQ_BF16; }
template <size_t N>
bool off(const void* p) { return (reinterpret_cast<uintptr_t>(p) & (N - 1)) != 0; }
bool off_element(const void* p, int dtype) { return dtype == BCQ_BF16 ? off<2>(p) : off<4>(p); }
bcq_status done(hipError_t e) { return e == hipSuccess ? BCQ_OK : BCQ_ERR_DEVICE; }

size_t workspace_need(int op, int64_t T) { return op == BCQ_OP_DISTILL_FWD_BWD ? (size_t)T * 16 : 0; }

}  // namespace

extern "C" {

bcq_status bcq_logits_workspace_bytes(int op, int64_t T, int64_t V, int k, int dtype, size_t* out) {
    if (!out) return BCQ_ERR_NULL;
    if (op < BCQ_OP_LOGPROBS_FWD || op > BCQ_OP_DISTILL_FWD_BWD) return BCQ_ERR_DTYPE;
    const bcq_status s = check_logits(T, V, V, k, 1.f);
    if (s != BCQ_OK) return s;
    if (op != BCQ_OP_LOGPROBS_FWD && k < 1) return BCQ_ERR_SHAPE;
    if (!dtype_ok(dtype)) return BCQ_ERR_DTYPE;
    *out = workspace_need(op, T);
    return BCQ_OK;
}

bcq_status bcq_logprobs_fwd(const void* logits, int dtype, int64_t T, int64_t V, int64_t row_stride, const int64_t* tokens,
                            float temperature, int k, float* logp, float* entropy, float* lse, float* stats,
                            int32_t* top_index, float* top_logit, float* top_logp, void* workspace,
                            size_t workspace_bytes, void* stream) {
    if (!logits || (tokens == nullptr) != (logp == nullptr)) return BCQ_ERR_NULL;
    if (!logp && !entropy && !lse && !stats && !(k > 0 && (top_index || top_logit || top_logp))) return BCQ_ERR_NULL;
    bcq_status s = check_logits(T, V, row_stride, k, temperature);
    if (s != BCQ_OK) return s;
    if (!dtype_ok(dtype)) return BCQ_ERR_DTYPE;
    if (off_element(logits, dtype) || off<8>(tokens) || off<4>(logp) || off<4>(entropy) || off<4>(lse) || off<4>(stats) ||
        off<4>(top_index) || off<4>(top_logit) || off<4>(top_logp))
        return BCQ_ERR_ALIGN;
    (void)workspace;
    (void)workspace_bytes;
    if (!bcq::host::device_ok()) return BCQ_ERR_DEVICE;
    if (T == 0) return BCQ_OK;
    const float c = 1.0f / temperature;
    if (!top_index && !top_logit && !top_logp) k = 0;
    const bcq::LogprobsOut out{logp, entropy, lse, stats, top_logit, top_logp, top_index};
    hipStream_t st = (hipStream_t)stream;
    const dim3 grid((unsigned)T), block(bcq::LG_THREADS);
    if (dtype == BCQ_BF16)
        BCQ_LAUNCH(bcq::logprobs_kernel<bcq::bf16_t>, grid, block, 0, st, (const bcq::bf16_t*)logits, row_stride, (int)V, tokens, c, k, out);
    else
        BCQ_LAUNCH(bcq::logprobs_kernel<float>, grid, block, 0, st, (const float*)logits, row_stride, (int)V, tokens, c, k, out);
    return done(hipGetLastError());
}

bcq_status bcq_logprobs_bwd(const void* logits, int dtype, int64_t T, int64_t V, int64_t row_stride, const int64_t* tokens,
                            float temperature, const float* stats, const float* dlogp, const float* entropy,
                            const float* dentropy, void* dlogits, int64_t grad_stride, void* stream) {
    if (!logits || !stats || !dlogits || (tokens == nullptr) != (dlogp == nullptr) || (entropy == nullptr) != (dentropy == nullptr) ||
        (!dlogp && !dentropy))
        return BCQ_ERR_NULL;
    bcq_status s = check_logits(T, V, row_stride, 0, temperature);
    if (s == BCQ_OK) s = check_logits(T, V, grad_stride, 0, temperature);
    if (s != BCQ_OK) return s;
    if (logits == dlogits && row_stride != grad_stride) return BCQ_ERR_SHAPE;
    if (!dtype_ok(dtype)) return BCQ_ERR_DTYPE;
    if (off_element(logits, dtype) || off_element(dlogits, dtype) || off<8>(tokens) || off<4>(stats) || off<4>(dlogp) ||
        off<4>(entropy) || off<4>(dentropy))
        return BCQ_ERR_ALIGN;
    if (!bcq::host::device_ok()) return BCQ_ERR_DEVICE;
    if (T == 0) return BCQ_OK;
    const float c = 1.0f / temperature;
    hipStream_t st = (hipStream_t)stream;
    const dim3 grid((unsigned)T), block(bcq::LG_THREADS);
    if (dtype == BCQ_BF16)
        BCQ_LAUNCH(bcq::logprobs_bwd_kernel<bcq::bf16_t>, grid, block, 0, st, (const bcq::bf16_t*)logits, row_stride, (int)V, tokens, c,
                   stats, dlogp, entropy, dentropy, (bcq::bf16_t*)dlogits, grad_stride);
    else
        BCQ_LAUNCH(bcq::logprobs_bwd_kernel<float>, grid, block, 0, st, (const float*)logits, row_stride, (int)V, tokens, c, stats,
                   dlogp, entropy, dentropy, (float*)dlogits, grad_stride);
    return done(hipGetLastError());
}

}  // extern "C"

namespace {

struct DistillCall {
    const void* logits;
    int dtype;
    int64_t T, V, row_stride;
    const float* top_logit;
    const int32_t* top_index;
    int k;
    const float* teacher_lse;
    float temperature;
};

bcq_status check_distill(const DistillCall& a) {
    const bcq_status s = check_logits(a.T, a.V, a.row_stride, a.k, a.temperature);
    if (s != BCQ_OK) return s;
    if (a.k < 1) return BCQ_ERR_SHAPE;
    return BCQ_OK;
}
bool distill_misaligned(const DistillCall& a) {
    return off_element(a.logits, a.dtype) || off<4>(a.top_logit) || off<4>(a.top_index) || off<4>(a.teacher_lse);
}

hipError_t run_distill_fwd(const DistillCall& a, const float* weight, float* loss, float* stats, hipStream_t st) {
    const dim3 grid((unsigned)a.T), block(bcq::LG_THREADS);
    const float c = 1.0f / a.temperature;
    if (a.dtype == BCQ_BF16)
        BCQ_LAUNCH(bcq::distill_kernel<bcq::bf16_t>, grid, block, 0, st, (const bcq::bf16_t*)a.logits, a.row_stride, (int)a.V, a.top_logit,
                   a.top_index, a.k, a.teacher_lse, c, weight, loss, stats);
    else
        BCQ_LAUNCH(bcq::distill_kernel<float>, grid, block, 0, st, (const float*)a.logits, a.row_stride, (int)a.V, a.top_logit,
                   a.top_index, a.k, a.teacher_lse, c, weight, loss, stats);
    return hipGetLastError();
}
hipError_t run_distill_bwd(const DistillCall& a, const float* stats, const float* weight, void* dlogits, int64_t grad_stride,
                           hipStream_t st) {
    const dim3 grid((unsigned)a.T), block(bcq::LG_THREADS);
    const float c = 1.0f / a.temperature;
    if (a.dtype == BCQ_BF16)
        BCQ_LAUNCH(bcq::distill_bwd_kernel<bcq::bf16_t>, grid, block, 0, st, (const bcq::bf16_t*)a.logits, a.row_stride, (int)a.V,
                   a.top_logit, a.top_index, a.k, a.teacher_lse, c, stats, weight, (bcq::bf16_t*)dlogits, grad_stride);
    else
        BCQ_LAUNCH(bcq::distill_bwd_kernel<float>, grid, block, 0, st, (const float*)a.logits, a.row_stride, (int)a.V, a.top_logit,
                   a.top_index, a.k, a.teacher_lse, c, stats, weight, (float*)dlogits, grad_stride);
    return hipGetLastError();
}

}  // namespace

extern "C" {

bcq_status bcq_distill_fwd(const void* logits, int dtype, int64_t T, int64_t V, int64_t row_stride, const float* top_logit,
                           const int32_t* top_index, int k, const float* teacher_lse, float temperature, float* loss,
                           float* stats, void* workspace, size_t workspace_bytes, void* stream) {
    if (!logits || !top_logit || !top_index || !loss) return BCQ_ERR_NULL;
    const DistillCall a{logits, dtype, T, V, row_stride, top_logit, top_index, k, teacher_lse, temperature};
    const bcq_status s = check_distill(a);
    if (s != BCQ_OK) return s;
    if (!dtype_ok(dtype)) return BCQ_ERR_DTYPE;
    if (distill_misaligned(a) || off<4>(loss) || off<4>(stats)) return BCQ_ERR_ALIGN;
    (void)workspace;
    (void)workspace_bytes;
    if (!bcq::host::device_ok()) return BCQ_ERR_DEVICE;
    if (T == 0) return BCQ_OK;
    return done(run_distill_fwd(a, nullptr, loss, stats, (hipStream_t)stream));
}

bcq_status bcq_distill_bwd(const void* logits, int dtype, int64_t T, int64_t V, int64_t row_stride, const float* top_logit,
                           const int32_t* top_index, int k, const float* teacher_lse, float temperature,
                           const float* stats, const float* dloss, void* dlogits, int64_t grad_stride, void* stream) {
    if (!logits || !top_logit || !top_index || !stats || !dloss || !dlogits) return BCQ_ERR_NULL;
    const DistillCall a{logits, dtype, T, V, row_stride, top_logit, top_index, k, teacher_lse, temperature};
    bcq_status s = check_distill(a);
    if (s == BCQ_OK) s = check_logits(T, V, grad_stride, k, temperature);
    if (s != BCQ_OK) return s;
    if (logits == dlogits && row_stride != grad_stride) return BCQ_ERR_SHAPE;
    if (!dtype_ok(dtype)) return BCQ_ERR_DTYPE;
    if (distill_misaligned(a) || off_element(dlogits, dtype) || off<4>(stats) || off<4>(dloss)) return BCQ_ERR_ALIGN;
    if (!bcq::host::device_ok()) return BCQ_ERR_DEVICE;
    if (T == 0) return BCQ_OK;
    return done(run_distill_bwd(a, stats, dloss, dlogits, grad_stride, (hipStream_t)stream));
}

bcq_status bcq_distill_fwd_bwd(const void* logits, int dtype, int64_t T, int64_t V, int64_t row_stride,
                               const float* top_logit, const int32_t* top_index, int k, const float* teacher_lse,
                               float temperature, const float* weight, float* loss, void* dlogits, int64_t grad_stride,
                               void* workspace, size_t workspace_bytes, void* stream) {
    if (!logits || !top_logit || !top_index || !loss || !dlogits) return BCQ_ERR_NULL;
    const DistillCall a{logits, dtype, T, V, row_stride, top_logit, top_index, k, teacher_lse, temperature};
    bcq_status s = check_distill(a);
    if (s == BCQ_OK) s = check_logits(T, V, grad_stride, k, temperature);
    if (s != BCQ_OK) return s;
    if (logits == dlogits && row_stride != grad_stride) return BCQ_ERR_SHAPE;
    if (!dtype_ok(dtype)) return BCQ_ERR_DTYPE;
    if (distill_misaligned(a) || off_element(dlogits, dtype) || off<4>(weight) || off<4>(loss)) return BCQ_ERR_ALIGN;
    const size_t need = workspace_need(BCQ_OP_DISTILL_FWD_BWD, T);
    if (need && !workspace) return BCQ_ERR_NULL;
    if (need && bcq::host::misaligned(workspace)) return BCQ_ERR_ALIGN;
    if (workspace_bytes < need) return BCQ_ERR_WORKSPACE;
    if (!bcq::host::device_ok()) return BCQ_ERR_DEVICE;
    if (T == 0) return BCQ_OK;
    float* stats = static_cast<float*>(workspace);
    const hipError_t e = run_distill_fwd(a, weight, loss, stats, (hipStream_t)stream);
    if (e != hipSuccess) return BCQ_ERR_DEVICE;
    return done(run_distill_bwd(a, stats, weight, dlogits, grad_stride, (hipStream_t)stream));
}

}  // extern "C"
