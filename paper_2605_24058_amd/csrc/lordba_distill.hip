// Learning from a teacher's top logits: a token's loss and its gradient with respect to the logits.
//
// A workgroup has a token.  The loss is one pass over the row with the running maximum m and the running sum of exp((z - m) / u); with both terms and
// a temperature other than 1 a second sum runs beside it.  The gradient is another pass, q = exp((z - m) / u) / sum, and what the teacher and the label
// take off is put in behind it at the few entries concerned, each computed anew and rounded once.  What bounds it is memory: a row is read for the loss, read
// again (from the caches) and written for the gradient.
#include <algorithm>
#include <cmath>

#include "lordba_dev_util.h"
#include "lordba_results.h"

namespace {

constexpr float kLog2e = 1.44269504088896f, kLowest = -3.402823466e38f;

struct DistillArgs {
    const void* z;
    const int32_t* index;
    const void* top;
    const int32_t* labels;
    const float* d_loss;
    float *loss, *kept;       // the pass for the loss: outputs; the gradient alone: kept is an input, loss null
    void* grad;               // or null
    int64_t V, first;
    int32_t k;
    float u, soft, hard;
};

template <class E>
struct Pack;   // 16 bytes of a row
template <>
struct Pack<_Float16> {
    static constexpr int N = 8;
    __device__ static __forceinline__ void get(const _Float16* p, float (&v)[N]) {
        const h8 h = as_h8(load16_any(p));
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = static_cast<float>(h[e]);
    }
    __device__ static __forceinline__ void put(_Float16* p, const float (&v)[N]) {
        h8 h;
#pragma unroll
        for (int e = 0; e < N; ++e) h[e] = static_cast<_Float16>(v[e]);
        *reinterpret_cast<u4_any*>(p) = __builtin_bit_cast(u4, h);
    }
};
template <>
struct Pack<float> {
    static constexpr int N = 4;
    typedef float f4_any __attribute__((ext_vector_type(4), aligned(4)));
    __device__ static __forceinline__ void get(const float* p, float (&v)[N]) {
        const f4_any h = *reinterpret_cast<const f4_any*>(p);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = h[e];
    }
    __device__ static __forceinline__ void put(float* p, const float (&v)[N]) { *reinterpret_cast<f4_any*>(p) = f4_any{v[0], v[1], v[2], v[3]}; }
};

// Running maximum and sums.  The maximum starts at the lowest number, so that entries of -infinity add 0 and a row of nothing else has the sum 0.
template <bool TWO>
struct Running {
    float m = kLowest, s = 0.f, s1 = 0.f;   // s: exp((z - m) / u); s1: exp(z - m)
    template <int N>
    __device__ __forceinline__ void add(const float (&v)[N], float c) {
        float most = v[0];
#pragma unroll
        for (int e = 1; e < N; ++e) most = fmaxf(most, v[e]);
        most = fmaxf(most, m);
        s *= __builtin_amdgcn_exp2f((m - most) * c);
        if constexpr (TWO) s1 *= __builtin_amdgcn_exp2f((m - most) * kLog2e);
        m = most;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            s += __builtin_amdgcn_exp2f((v[e] - m) * c);
            if constexpr (TWO) s1 += __builtin_amdgcn_exp2f((v[e] - m) * kLog2e);
        }
    }
    __device__ __forceinline__ void join(float om, float os, float os1, float c) {
        const float most = fmaxf(m, om);
        s = s * __builtin_amdgcn_exp2f((m - most) * c) + os * __builtin_amdgcn_exp2f((om - most) * c);
        if constexpr (TWO) s1 = s1 * __builtin_amdgcn_exp2f((m - most) * kLog2e) + os1 * __builtin_amdgcn_exp2f((om - most) * kLog2e);
        m = most;
    }
};

template <int THREADS>
__device__ __forceinline__ float block_max(float v, float* scratch) {
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) v = fmaxf(v, __shfl_xor(v, s));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
    __syncthreads();
    v = scratch[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) v = fmaxf(v, scratch[w]);
    return v;
}
template <int THREADS>
__device__ __forceinline__ float block_sum(float v, float* scratch) {
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) v += __shfl_xor(v, s);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
    __syncthreads();
    v = scratch[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) v += scratch[w];
    return v;
}

template <class E, int THREADS, bool TWO>
__global__ __launch_bounds__(THREADS) void lordba_distill_kernel(DistillArgs a) {
    constexpr int N = Pack<E>::N;
    __shared__ float scratch[3 * THREADS / 64];
    __shared__ int32_t index[LORDBA_MAX_TOP + 1];           // (the label last)
    __shared__ float p[LORDBA_MAX_TOP + 1], at[LORDBA_MAX_TOP + 1];   // the teacher's probability, the student's logit
    const int64_t t = a.first + blockIdx.x, V = a.V;
    const E* const z = static_cast<const E*>(a.z) + t * V;
    E* const grad = a.grad ? static_cast<E*>(a.grad) + t * V : nullptr;
    const int tid = threadIdx.x;

    // The teacher's entries that are there, and their probabilities.
    float most = kLowest;
    bool mine = false;
    for (int i = tid; i < a.k; i += THREADS) {
        const int32_t v = a.index[t * a.k + i];
        const float l = static_cast<float>(static_cast<const E*>(a.top)[t * a.k + i]);
        const bool there = v >= 0 && v < V && l != -__builtin_inff();
        index[i] = there ? v : -1;
        p[i] = l;
        mine = mine || there;
        if (there) most = fmaxf(most, l);
    }
    const int32_t label = a.labels && a.hard != 0.f ? a.labels[t] : -1;
    const bool has_hard = label >= 0 && label < V, has_soft = a.soft != 0.f && __syncthreads_or(mine);
    if (!has_soft && !has_hard) {
        if (tid == 0) {
            if (a.loss) a.loss[t] = 0.f;
            if (a.loss && a.kept) a.kept[3 * t] = a.kept[3 * t + 1] = a.kept[3 * t + 2] = 0.f;
        }
        if (grad)
            for (int64_t i = tid; i < V; i += THREADS) grad[i] = static_cast<E>(0.f);
        return;
    }
    const float cu = kLog2e / a.u;
    most = block_max<THREADS>(most, scratch);
    float total = 0.f;
    for (int i = tid; i < a.k; i += THREADS)
        if (index[i] >= 0) total += __builtin_amdgcn_exp2f((p[i] - most) * cu);
    total = block_sum<THREADS>(total, scratch);
    const float log_total = logf(total);

    // The row, in 16-byte pieces that start on 16 bytes; what is in front of and behind them one by one.
    const int64_t head = min(V, static_cast<int64_t>((16 - (reinterpret_cast<uintptr_t>(z) & 15)) % 16 / sizeof(E))), pieces = (V - head) / N;
    const int64_t tail = head + pieces * N;
    const bool one_by_one = tid < head + (V - tail);
    const int64_t single = tid < head ? tid : tail + (tid - head);   // (fewer than 2 N of them)

    const float c = TWO || a.soft != 0.f ? cu : kLog2e;   // (with one sum: u is 1 where both terms are wanted)
    float m, inverse, inverse1;
    if (a.loss) {
        Running<TWO> run;
        if (one_by_one) {
            const float v[1] = {static_cast<float>(z[single])};
            run.add(v, c);
        }
        for (int64_t i = tid; i < pieces; i += THREADS) {
            float v[N];
            Pack<E>::get(z + head + i * N, v);
            run.add(v, c);
        }
#pragma unroll
        for (int s = 32; s > 0; s >>= 1) run.join(__shfl_xor(run.m, s), __shfl_xor(run.s, s), TWO ? __shfl_xor(run.s1, s) : 0.f, c);
        __syncthreads();
        if ((tid & 63) == 0) scratch[tid >> 6] = run.m, scratch[THREADS / 64 + (tid >> 6)] = run.s, scratch[2 * THREADS / 64 + (tid >> 6)] = run.s1;
        __syncthreads();
        run.m = scratch[0], run.s = scratch[THREADS / 64], run.s1 = scratch[2 * THREADS / 64];
#pragma unroll
        for (int w = 1; w < THREADS / 64; ++w) run.join(scratch[w], scratch[THREADS / 64 + w], scratch[2 * THREADS / 64 + w], c);
        const float s1 = TWO ? run.s1 : run.s;
        m = run.m, inverse = 1.f / run.s, inverse1 = 1.f / s1;
        // (-infinity wherever no entry is a number)
        const float log_s = logf(run.s), log_s1 = logf(s1);
        float part = 0.f;
        for (int i = tid; i < a.k; i += THREADS)
            if (index[i] >= 0) {
                at[i] = static_cast<float>(z[index[i]]);
                const float lp = (p[i] - most) / a.u - log_total, pr = __builtin_amdgcn_exp2f((p[i] - most) * cu) / total;
                p[i] = pr;
                if (pr != 0.f) part += pr * (lp - ((at[i] - m) / a.u - log_s));
            }
        part = block_sum<THREADS>(part, scratch);
        if (tid == 0) {
            float loss = has_soft ? a.soft * a.u * a.u * part : 0.f;
            if (has_hard) loss -= a.hard * ((static_cast<float>(z[label]) - m) - log_s1);
            a.loss[t] = loss;
            if (a.kept) a.kept[3 * t] = m, a.kept[3 * t + 1] = run.s, a.kept[3 * t + 2] = s1;
        }
    } else {
        m = a.kept[3 * t], inverse = 1.f / a.kept[3 * t + 1], inverse1 = 1.f / a.kept[3 * t + 2];
        for (int i = tid; i < a.k; i += THREADS)
            if (index[i] >= 0) at[i] = static_cast<float>(z[index[i]]), p[i] = __builtin_amdgcn_exp2f((p[i] - most) * cu) / total;
    }
    if (!grad) return;
    const float dl = a.d_loss[t], ws = has_soft ? a.soft * a.u * dl : 0.f, wh = has_hard ? a.hard * dl : 0.f;
    auto soft_of = [&](float v) { return __builtin_amdgcn_exp2f((v - m) * cu) * inverse; };
    auto hard_of = [&](float v) { return __builtin_amdgcn_exp2f((v - m) * kLog2e) * inverse1; };
    auto slope = [&](float v) { return (has_soft ? ws * soft_of(v) : 0.f) + (has_hard ? wh * hard_of(v) : 0.f); };
    if (tid == 0 && has_hard) {
        index[a.k] = label;
        at[a.k] = static_cast<float>(z[label]);
    }
    __syncthreads();   // (everybody has the logits at the entries before the first is overwritten)
    if (one_by_one) grad[single] = static_cast<E>(slope(static_cast<float>(z[single])));
    for (int64_t i = tid; i < pieces; i += THREADS) {
        float v[N];
        Pack<E>::get(z + head + i * N, v);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = slope(v[e]);
        Pack<E>::put(grad + head + i * N, v);
    }
    __syncthreads();
    // The entries that the teacher or the label names: the first of those that name the same one adds up what they take off.
    for (int i = tid; i < a.k + (has_hard ? 1 : 0); i += THREADS) {
        const int32_t v = index[i];
        if (v < 0 || (i < a.k && !has_soft)) continue;
        bool named = false;
        for (int j = 0; has_soft && j < i; ++j) named = named || index[j] == v;
        if (named) continue;
        float off = 0.f;
        for (int j = i; has_soft && j < a.k; ++j) off += index[j] == v ? p[j] : 0.f;
        float d = 0.f;
        if (has_soft) d += ws * (soft_of(at[i]) - off);
        if (has_hard) d += wh * (hard_of(at[i]) - (v == label ? 1.f : 0.f));
        grad[v] = static_cast<E>(d);
    }
}

template <class E, int THREADS, bool TWO>
lordba_status distill_launch(DistillArgs a, int64_t T, hipStream_t stream) {
    constexpr int64_t kMost = (static_cast<int64_t>(1) << 31) / THREADS / 2;   // (a launch counts threads in 32 bits)
    for (a.first = 0; a.first < T; a.first += kMost) {
        hipLaunchKernelGGL((lordba_distill_kernel<E, THREADS, TWO>), dim3(static_cast<unsigned>(std::min(kMost, T - a.first))), dim3(THREADS), 0, stream, a);
        const lordba_status st = i8_launched();
        if (st != LORDBA_OK) return st;
    }
    return LORDBA_OK;
}

template <class E>
lordba_status distill(const DistillArgs& a, int64_t T, hipStream_t stream) {
    const bool two = a.soft != 0.f && a.hard != 0.f && a.u != 1.f;
    return two ? distill_launch<E, 512, true>(a, T, stream) : distill_launch<E, 512, false>(a, T, stream);
}

lordba_status run(const void* logits, int type, const lordba_teacher* w, const float* d_loss, float* loss, float* kept, const float* kept_in,
                  void* d_logits, int64_t T, int64_t V, void* stream) {
    if (T < 0 || T > INT32_MAX || V < 1 || V > (1 << 24)) return LORDBA_ERR_DIM;
    if (!w) return LORDBA_ERR_NULL;
    if (w->k < 0 || w->k > LORDBA_MAX_TOP) return LORDBA_ERR_DIM;
    if ((type != LORDBA_F16 && type != LORDBA_F32) || !(w->temperature > 0.f) || !std::isfinite(w->temperature) || !std::isfinite(w->soft) ||
        !std::isfinite(w->hard))
        return LORDBA_ERR_VALUE;
    if (T == 0) return LORDBA_OK;
    if (!logits || (!loss && !kept_in) || (d_loss == nullptr) != (d_logits == nullptr) || (kept_in && !d_loss) ||
        (w->k > 0 && (!w->top_index || !w->top_logits)))
        return LORDBA_ERR_NULL;
    const size_t item = type == LORDBA_F16 ? 2 : 4, nz = static_cast<size_t>(T) * V * item, n = static_cast<size_t>(T);
    if (i8_misaligned(logits, item) || i8_misaligned(w->top_logits, item) || i8_misaligned(d_logits, item) || i8_misaligned(w->top_index, 4) ||
        i8_misaligned(w->labels, 4) || i8_misaligned(d_loss, 4) || i8_misaligned(loss, 4) || i8_misaligned(kept, 4) || i8_misaligned(kept_in, 4))
        return LORDBA_ERR_ALIGN;
    const Span out[] = {{loss, 4 * n}, {kept, 12 * n}, {d_logits, nz}};
    const Span in[] = {{d_logits == logits ? nullptr : logits, nz}, {w->top_index, 4 * n * w->k}, {w->top_logits, item * n * w->k},
                       {w->labels, 4 * n}, {d_loss, 4 * n}, {kept_in, 12 * n}};
    if (aliased(out, in) || i8_overlap(loss, 4 * n, logits, nz) || i8_overlap(kept, 12 * n, logits, nz)) return LORDBA_ERR_ALIAS;
    const lordba_status dev = check_device();
    if (dev != LORDBA_OK) return dev;
    const DistillArgs a = {logits, w->top_index, w->top_logits, w->labels, d_loss, loss, kept_in ? const_cast<float*>(kept_in) : kept, d_logits, V, 0,
                           static_cast<int32_t>(w->k), w->temperature, w->soft, w->hard};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return type == LORDBA_F16 ? distill<_Float16>(a, T, st) : distill<float>(a, T, st);
}

}  // namespace

extern "C" lordba_status lordba_distill(const void* logits, int type, const lordba_teacher* teacher, const float* d_loss, float* loss, float* kept,
                                        void* d_logits, int64_t T, int64_t V, void* stream) {
    if (T > 0 && !loss) return LORDBA_ERR_NULL;
    return run(logits, type, teacher, d_loss, loss, kept, nullptr, d_logits, T, V, stream);
}

extern "C" lordba_status lordba_distill_backward(const float* d_loss, const void* logits, int type, const float* kept, const lordba_teacher* teacher,
                                                 void* d_logits, int64_t T, int64_t V, void* stream) {
    if (T > 0 && (!kept || !d_loss)) return LORDBA_ERR_NULL;
    return run(logits, type, teacher, d_loss, nullptr, nullptr, kept, d_logits, T, V, stream);
}
