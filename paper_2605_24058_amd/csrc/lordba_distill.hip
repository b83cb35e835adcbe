// Learning from a teacher's top logits: a token's loss and its gradient with respect to the logits.
//
// A workgroup has a token.  The loss is one pass over the row with the running maximum m and the running sum of exp((z - m) / u); with both terms and
// a temperature other than 1 a second sum runs beside it.  The gradient is another pass, q = exp((z - m) / u) / sum, and what the teacher and the label
// take off is put in behind it at the few entries concerned, each computed anew and rounded once.  What bounds it is memory: a row is read for the loss
// and written for the gradient (2048 x 32000 in fp16, both at once: 262 MB in 57.8 us, 4.5 TB/s, of 5.1 that a large copy reaches); a single row waits for
// its chain of latencies (11 us at 32000).
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
    __device__ static __forceinline__ void take(u4 p, float (&v)[N]) {
        const h8 h = as_h8(p);
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
    __device__ static __forceinline__ void take(u4 p, float (&v)[N]) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = __uint_as_float(p[e]);
    }
    __device__ static __forceinline__ void put(float* p, const float (&v)[N]) { *reinterpret_cast<f4_any*>(p) = f4_any{v[0], v[1], v[2], v[3]}; }
};

// Running maximum and sums.  The maximum starts at the lowest number, so that entries of -infinity add 0 and a row of nothing else has the sum 0.
template <bool TWO>
struct Running {
    float m = kLowest, s = 0.f, s1 = 0.f;   // s: exp((z - m) / u); s1: exp(z - m)
    template <int N>
    __device__ __forceinline__ void raise(const float (&v)[N], float c) {   // the maximum to that of v too
        float most = v[0];
#pragma unroll
        for (int e = 1; e < N; ++e) most = fmaxf(most, v[e]);
        most = fmaxf(most, m);
        s *= __builtin_amdgcn_exp2f((m - most) * c);
        if constexpr (TWO) s1 *= __builtin_amdgcn_exp2f((m - most) * kLog2e);
        m = most;
    }
    template <int N>
    __device__ __forceinline__ void sum(const float (&v)[N], float c) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            s += __builtin_amdgcn_exp2f((v[e] - m) * c);
            if constexpr (TWO) s1 += __builtin_amdgcn_exp2f((v[e] - m) * kLog2e);
        }
    }
};

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) v = fmaxf(v, __shfl_xor(v, s));
    return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) v += __shfl_xor(v, s);
    return v;
}
// What this wave has written to LDS is what it reads from here on (the hardware keeps a wave's order; the compiler has to as well).
__device__ __forceinline__ void in_wave_order() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
}

constexpr int kInWave = 64;   // entries up to which the first wave compares them with each other

// One wave deals with the teacher and the label while the others wait for the row; the workgroup meets twice, when the sums of its waves are there and when
// the gradient is written but for the entries that the teacher or the label names.
// NV > 0: the row lies in registers, NV pieces a thread, requested all at once and read once; 0: rows longer than that, read in turn for either pass.
template <class E, int THREADS, int NV, bool TWO>
__global__ __launch_bounds__(THREADS) void lordba_distill_kernel(DistillArgs a) {
    constexpr int N = Pack<E>::N, W = THREADS / 64;
    __shared__ float partial[3][W], teacher[2];   // largest, sums of the waves; the teacher's largest logit and its sum
    __shared__ int32_t some;                      // whether the teacher has an entry
    extern __shared__ int32_t index[];            // [k]; then, as many each:
    float* const p = reinterpret_cast<float*>(index + a.k);   // the teacher's logit,
    float* const off = p + a.k;                               // what the entry takes off, of all that name the same one; below 0 where another one stands for it;
    float* const at = off + a.k;                              // the student's logit, and behind the last the label's
    const int64_t t = a.first + blockIdx.x, V = a.V;
    const E* const z = static_cast<const E*>(a.z) + t * V;
    E* const grad = a.grad ? static_cast<E*>(a.grad) + t * V : nullptr;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    // The row, in 16-byte pieces that start on 16 bytes; what is in front of and behind them one by one.
    const int64_t head = min(V, static_cast<int64_t>((16 - (reinterpret_cast<uintptr_t>(z) & 15)) % 16 / sizeof(E))), pieces = (V - head) / N;
    const int64_t tail = head + pieces * N;
    const bool one_by_one = tid < head + (V - tail);
    const int64_t single = tid < head ? tid : tail + (tid - head);   // (fewer than 2 N of them)
    u4 held[NV > 0 ? NV : 1];
    if (NV > 0 && pieces > 0) {
#pragma unroll
        for (int j = 0; j < NV; ++j) held[j] = load16(z + head + min<int64_t>(tid + j * THREADS, pieces - 1) * N);
    }
    auto each_piece = [&](auto f) __attribute__((always_inline)) {   // four requested together
        for (int64_t i = tid; i < pieces; i += 4 * THREADS) {
            u4 v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = load16(z + head + min(i + j * THREADS, pieces - 1) * N);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (i + j * THREADS < pieces) f(i + j * THREADS, v[j]);
        }
    };
    const float alone = one_by_one ? static_cast<float>(z[single]) : 0.f;

    const int32_t label = a.labels && a.hard != 0.f ? a.labels[t] : -1;
    const bool has_hard = label >= 0 && label < V;
    const float cu = kLog2e / a.u;
    if (wave == 0) {
        float most = kLowest;
        bool mine = false;
        for (int i = lane; i < a.k; i += 64) {
            const int32_t v = a.index[t * a.k + i];
            const float l = static_cast<float>(static_cast<const E*>(a.top)[t * a.k + i]);
            const bool there = v >= 0 && v < V && l != -__builtin_inff() && a.soft != 0.f;
            index[i] = there ? v : -1;
            p[i] = l;
            at[i] = there ? static_cast<float>(z[v]) : 0.f;
            mine = mine || there;
            if (there) most = fmaxf(most, l);
        }
        most = wave_max(most);
        in_wave_order();
        float total = 0.f;
        for (int i = lane; i < a.k; i += 64)
            if (index[i] >= 0) total += __builtin_amdgcn_exp2f((p[i] - most) * cu);
        total = wave_sum(total);
        if (a.k <= kInWave) {   // (entries that another one stands for: the first that names it adds up)
            const int32_t v = lane < a.k ? index[lane] : -1;
            const float pr = v >= 0 ? __builtin_amdgcn_exp2f((p[lane] - most) * cu) / total : 0.f;
            float sum = 0.f;
            bool named = false;
            for (int j = 0; j < a.k; ++j) {
                const bool same = __shfl(v, j) == v;
                sum += same ? __shfl(pr, j) : 0.f;
                named = named || (same && j < lane);
            }
            if (lane < a.k) off[lane] = v < 0 || named ? -1.f : sum;
        }
        if (lane == 0) {
            teacher[0] = most, teacher[1] = total;
            at[a.k] = has_hard ? static_cast<float>(z[label]) : 0.f;
        }
        const bool any = __any(mine);
        if (lane == 0) some = any;
    }

    const float c = TWO || a.soft != 0.f ? cu : kLog2e;   // (with one sum: u is 1 where both terms are wanted)
    float m, s, s1;
    if (a.loss) {
        Running<TWO> run;
        if constexpr (NV > 0) {   // this thread's largest first
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (tid + j * THREADS < pieces) {
                    float v[N];
                    Pack<E>::take(held[j], v);
#pragma unroll
                    for (int e = 0; e < N; ++e) run.m = fmaxf(run.m, v[e]);
                }
            if (one_by_one) run.m = fmaxf(run.m, alone);
            run.m = wave_max(run.m);
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (tid + j * THREADS < pieces) {
                    float v[N];
                    Pack<E>::take(held[j], v);
                    run.sum(v, c);
                }
        } else {
            each_piece([&](int64_t, u4 piece) __attribute__((always_inline)) {
                float v[N];
                Pack<E>::take(piece, v);
                run.raise(v, c);
                run.sum(v, c);
            });
        }
        if (one_by_one) {
            const float v[1] = {alone};
            if constexpr (NV == 0) run.raise(v, c);
            run.sum(v, c);
        }
        if constexpr (NV == 0) {
            const float most = wave_max(run.m);
            run.s *= __builtin_amdgcn_exp2f((run.m - most) * c);
            if constexpr (TWO) run.s1 *= __builtin_amdgcn_exp2f((run.m - most) * kLog2e);
            run.m = most;
        }
        run.s = wave_sum(run.s);
        if constexpr (TWO) run.s1 = wave_sum(run.s1);
        if (lane == 0) partial[0][wave] = run.m, partial[1][wave] = run.s, partial[2][wave] = run.s1;
    }
    __syncthreads();
    const bool has_soft = some != 0;
    if (a.loss) {
        m = partial[0][0];
#pragma unroll
        for (int w = 1; w < W; ++w) m = fmaxf(m, partial[0][w]);
        s = 0.f, s1 = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            s += partial[1][w] * __builtin_amdgcn_exp2f((partial[0][w] - m) * c);
            if constexpr (TWO) s1 += partial[2][w] * __builtin_amdgcn_exp2f((partial[0][w] - m) * kLog2e);
        }
        if constexpr (!TWO) s1 = s;
    } else {
        m = a.kept[3 * t], s = a.kept[3 * t + 1], s1 = a.kept[3 * t + 2];
    }
    if (a.loss && wave == 0) {   // (log 0 = -infinity wherever no logit is a number)
        const float log_s = logf(s), log_total = logf(teacher[1]);
        float part = 0.f;
        for (int i = lane; i < a.k; i += 64)
            if (index[i] >= 0) {
                const float arg = p[i] - teacher[0], pr = __builtin_amdgcn_exp2f(arg * cu) / teacher[1];
                // u times the difference of the logarithms, without a quotient that small temperatures would take past the range
                if (pr != 0.f) part += pr * ((arg - (at[i] - m)) + a.u * (log_s - log_total));
            }
        part = wave_sum(part);
        if (lane == 0) {
            float loss = has_soft ? a.soft * a.u * part : 0.f;
            if (has_hard) loss -= a.hard * ((at[a.k] - m) - logf(s1));
            a.loss[t] = loss;
            const bool none = !has_soft && !has_hard;
            if (a.kept) a.kept[3 * t] = none ? 0.f : m, a.kept[3 * t + 1] = none ? 0.f : s, a.kept[3 * t + 2] = none ? 0.f : s1;
        }
    }
    if (!grad) return;
    if (a.k > kInWave) {
        for (int i = tid; i < a.k; i += THREADS) {
            const int32_t v = index[i];
            bool named = v < 0;
            float sum = 0.f;
            for (int j = 0; j < a.k; ++j) {
                const bool same = index[j] == v;
                named = named || (same && j < i);
                if (same && !named) sum += __builtin_amdgcn_exp2f((p[j] - teacher[0]) * cu);
            }
            off[i] = named ? -1.f : sum / teacher[1];
        }
    }
    const float dl = a.d_loss[t], inverse = 1.f / s, inverse1 = 1.f / s1, ws = has_soft ? a.soft * a.u * dl : 0.f, wh = has_hard ? a.hard * dl : 0.f;
    // A logit's slope: ws q + wh r, with sum_i p_i and 1 taken off where asked.
    auto slope = [&](float v, float off_q, float off_r) __attribute__((always_inline)) {
        float d = 0.f;
        if (has_soft) d += ws * (__builtin_amdgcn_exp2f((v - m) * cu) * inverse - off_q);
        if (has_hard) d += wh * (__builtin_amdgcn_exp2f((v - m) * kLog2e) * inverse1 - off_r);
        return d;
    };
    if (one_by_one) grad[single] = static_cast<E>(slope(alone, 0.f, 0.f));
    auto write = [&](int64_t i, u4 piece) __attribute__((always_inline)) {
        float v[N];
        Pack<E>::take(piece, v);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = slope(v[e], 0.f, 0.f);
        Pack<E>::put(grad + head + i * N, v);
    };
    if constexpr (NV > 0) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (tid + j * THREADS < pieces) write(tid + j * THREADS, held[j]);
    } else {
        each_piece(write);
    }
    __syncthreads();
    for (int i = tid; i < a.k; i += THREADS)
        if (off[i] >= 0.f || off[i] != off[i]) grad[index[i]] = static_cast<E>(slope(at[i], off[i], index[i] == label ? 1.f : 0.f));
    if (tid == 0 && has_hard) {   // the label, where the teacher does not name it
        bool named = false;
        for (int j = 0; j < a.k; ++j) named = named || index[j] == label;
        if (!named) grad[label] = static_cast<E>(slope(at[a.k], 0.f, 1.f));
    }
}

template <class E, int THREADS, int NV, bool TWO>
lordba_status distill_launch(DistillArgs a, int64_t T, hipStream_t stream) {
    constexpr int64_t kMost = (static_cast<int64_t>(1) << 31) / THREADS / 2;   // (a launch counts threads in 32 bits)
    for (a.first = 0; a.first < T; a.first += kMost) {
        hipLaunchKernelGGL((lordba_distill_kernel<E, THREADS, NV, TWO>), dim3(static_cast<unsigned>(std::min(kMost, T - a.first))), dim3(THREADS), static_cast<size_t>(a.k) * 16 + 4, stream, a);
        const lordba_status st = i8_launched();
        if (st != LORDBA_OK) return st;
    }
    return LORDBA_OK;
}

// Short rows lie in the registers of as many threads as they fill; long ones too where loss and gradient are asked for at once and a workgroup's registers hold
// them: 2048 x 32000 57.8 us in fp16 and 119 in fp32, read twice 59.6 and 128.  One pass alone over rows of that length is quicker in a loop, of
// which more workgroups run side by side: the loss in fp16 26.2 us (held 27.0), in fp32 41 (61), the gradient 44.9 (49.2) and 107 (107).  Rows beyond that:
// 500 x 131072 in fp16 62.7 us with 1024 threads, 66.5 with 512, 73.6 held.
template <class E, bool TWO>
lordba_status distill(const DistillArgs& a, int64_t T, hipStream_t stream) {
    const int64_t pieces = a.V / Pack<E>::N;
    const bool step = a.loss && a.grad;
    if (pieces <= 64 * 4) return distill_launch<E, 64, 4, TWO>(a, T, stream);
    if (pieces <= 256 * 4) return distill_launch<E, 256, 4, TWO>(a, T, stream);
    if (pieces <= 512 * 8) return step ? distill_launch<E, 512, 8, TWO>(a, T, stream) : distill_launch<E, 256, 0, TWO>(a, T, stream);
    if (pieces <= 1024 * 8) return step ? distill_launch<E, 1024, 8, TWO>(a, T, stream) : distill_launch<E, 512, 0, TWO>(a, T, stream);
    return distill_launch<E, 1024, 0, TWO>(a, T, stream);
}
template <class E>
lordba_status distill(const DistillArgs& a, int64_t T, hipStream_t stream) {
    return a.soft != 0.f && a.hard != 0.f && a.u != 1.f ? distill<E, true>(a, T, stream) : distill<E, false>(a, T, stream);
}

lordba_status run(const void* logits, int type, const lordba_teacher* w, const float* d_loss, float* loss, float* kept, const float* kept_in,
                  void* d_logits, int64_t T, int64_t V, void* stream) {
    if (T < 0 || T > INT32_MAX || V < 1 || V > (1 << 24)) return LORDBA_ERR_DIM;
    if (!w) return LORDBA_ERR_NULL;
    if (w->k < 0 || w->k > LORDBA_MAX_TOP) return LORDBA_ERR_DIM;
    if ((type != LORDBA_F16 && type != LORDBA_F32) || !(w->temperature > 0.f) || !std::isnormal(w->temperature) || !std::isfinite(w->soft) ||
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
