// echo_distill.hip -- distillation from a teacher's top logits over a vocabulary or a shard of one, on gfx950.
//
// Per row, at temperature T: q = softmax of the teacher's logits / T over its entries in the vocabulary, p = softmax of the
// logits / T over the vocabulary, loss = T^2 sum over entries of q (log q - log p), and the logits' gradient T (p - q) grad_loss,
// in which the q of one id add up.
#include "echo_teacher.h"

namespace echo {
namespace {

__device__ __forceinline__ TeacherIn teacher_in(const DistillArgs &a) {
    return TeacherIn{a.ids, a.teacher, a.index_type, a.teacher_type, a.top, a.vocab_start, a.vocab_size, a.inv_t};
}
// The entries with the logits of their columns.
template <class T>
__device__ __forceinline__ Teacher entries_of(const DistillArgs &a, int64_t row, int first, int cols, Entry *entries) {
    const TeacherIn in = teacher_in(a);
    const Teacher t = teacher_of(in, row, first, cols, a.cols, entries);
    const T *l = static_cast<const T *>(a.logits) + row * a.logits_stride;
    take_logits(entries, a.top, [&](int at) ECHO_INLINE { return (float)l[at]; });
    return t;
}
// Exponentials of logits / T relative to that of a logit `base`.  Logits' distances are taken before they are divided by T: at logits / T of
// 10^10, whose last place is 1024, the maximum's own exponential is 1 and the others follow from their distances alone.
// 1 / T and log2(e) / T are arguments: made by every lane they cost a row of 51201 of bf16 two registers more than there are, 126 us and not 111.
struct Relative {
    float base, k;      // k: log2(e) / T
    __device__ __forceinline__ float operator()(float l) const { return __builtin_amdgcn_exp2f((l - base) * k); }
};
// Probabilities from a given lse.
struct Given {
    float lse, inv_t;
    __device__ __forceinline__ float operator()(float l) const { return exp_of(scaled(l, inv_t) - lse); }
};
// The gradient where the teacher has a mass, over what its row has there.
template <class T, class X>
__device__ __forceinline__ void put_entries(T *grad, const Entry *entries, int top, X exp_at, float scale, float g) {
    for (int k = threadIdx.x % kWave; k < top; k += kWave) {
        const Entry e = entries[k];
        if (e.at >= 0) grad[e.at] = (T)(exp_at(e.x) * scale - e.mass * g);
    }
}
__device__ __forceinline__ float finish_row(const DistillArgs &a, int64_t row, const Teacher &t, const Entry *entries, float top, float sum) {
    const float inv_t = a.inv_t, more = logf(sum), lse = top == -kInf ? -kInf : top * inv_t + more;
    // the loss takes logits from their maximum on, the target as they are
    const float cross = a.loss ? cross_of(entries, a.top, top != -kInf ? top : 0.0f) * inv_t : 0.0f;
    const float target = a.target ? cross_of(entries, a.top, 0.0f) * inv_t : 0.0f;
    if (threadIdx.x % kWave == 0) {
        if (a.lse) a.lse[row] = lse;
        if (a.target) a.target[row] = target;
        if (a.entropy) a.entropy[row] = -t.prior;
        if (a.loss)
            a.loss[row] = !t.trained ? 0.0f : lse == -kInf ? kInf : a.temperature * a.temperature * (t.prior - cross + more);
    }
    return lse;
}
// Stores that are already on their way are behind this: what the whole team wrote is where later stores find it.
template <int WAVES>
__device__ __forceinline__ void settled() {
    __threadfence_block();
    if constexpr (WAVES > 1) __syncthreads();
    else __builtin_amdgcn_s_waitcnt(0);
}

// A team a row, as in cross entropy: the row is read once and its gradient written from registers.  The gradient is then
// written over at the teacher's ids.  Memory bounds it: 2048 x 51200 of bf16 with 64 ids a row takes 85 us with its gradient, 4.9 TB/s, on new
// logits (cross entropy 79); while one wavefront prepares the teacher's entries, the others take their maxima and sums.
template <class T, int THREADS, int E>
constexpr int kDistillWaves = THREADS == 1024 && E * sizeof(T) <= 128 ? 8 : 1;
template <class T, int THREADS, int E, bool CUT>
__global__ __launch_bounds__((Team<T, THREADS, E, CUT>::BLOCK), (kDistillWaves<T, THREADS, E>)) void k_distill(DistillArgs a) {
    using Q = Team<T, THREADS, E, CUT>;
    constexpr int N = Q::N, P = Q::P;
    const Q q(a.cols);
    extern __shared__ __attribute__((aligned(16))) char space[];
    Entry *entries = reinterpret_cast<Entry *>(space) + q.team * a.top;
    __shared__ float4 lds[2][Q::WAVES];
    const float k2 = a.k2;
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * Q::TEAMS + q.team; row < a.rows; row += (int64_t)gridDim.x * Q::TEAMS) {
        const T *l = static_cast<const T *>(a.logits) + row * a.logits_stride;
        V<T, N> x[P];
        q.load(l, x, T(-kInf));
        Teacher t{};
        if (q.wave == 0) t = entries_of<T>(a, row, 0, a.cols, entries);
        float top = -kInf, sum = 0.0f;
#pragma unroll
        for (int k = 0; k < P; ++k) {
            const F<N> f = widen<T, N>(x[k]);
#pragma unroll
            for (int j = 0; j < N; ++j) top = fmaxf(top, f[j]);
            if constexpr (kDistillWaves<T, THREADS, E> > 1) asm volatile("" : "+v"(top));
        }
        forget<T, N, P>(x);
        top = wave_max(top);
        const Relative from{top == -kInf ? 0.0f : top, k2};
#pragma unroll
        for (int k = 0; k < P; ++k) {
            const F<N> f = widen<T, N>(x[k]);
#pragma unroll
            for (int j = 0; j < N; ++j) sum += from(f[j]);
            if constexpr (kDistillWaves<T, THREADS, E> > 1) asm volatile("" : "+v"(sum));
        }
        forget<T, N, P>(x);
        sum = wave_sum(sum);
        bool trained = t.trained;
        if constexpr (Q::WAVES > 1) {
            if (q.lane % kWave == 0) lds[turn][q.wave] = make_float4(top, sum, t.trained ? 1.0f : 0.0f, 0.0f);
            __syncthreads();      // also: the teacher's logits have been read, and grad may be logits
            const float4 p = lds[turn][q.lane % Q::WAVES];
            top = ring_max<Q::WAVES>(p.x);
            sum = ring_sum<Q::WAVES>(p.x == -kInf ? p.y : p.y * Relative{top, k2}(p.x));
            trained = ring_sum<Q::WAVES>(p.z) > 0.0f;      // the first wavefront's
            turn ^= 1;
        }
        if (sum != sum) top = sum;      // a row of NaN alone has no maximum but a sum
        if (q.wave == 0) finish_row(a, row, t, entries, top, sum);
        if (!a.grad) continue;
        const bool live = trained && top != -kInf;
        const Relative share{top, k2};
        const float g = a.grad_loss[row] * a.temperature, scale = g / sum;
#pragma unroll
        for (int k = 0; k < P; ++k) {
            F<N> f = 0.0f;
            if (live) {
                f = widen<T, N>(x[k]);
#pragma unroll
                for (int j = 0; j < N; ++j) f[j] = share(f[j]) * scale;
            }
            x[k] = round_to<T, N>(f);
            if constexpr (kDistillWaves<T, THREADS, E> > 1) forget<T, N, 1>(reinterpret_cast<V<T, N>(&)[1]>(x[k]));
        }
        T *d = static_cast<T *>(a.grad) + row * a.grad_stride;
        q.drop(d, x);
        settled<Q::WAVES>();
        if (q.wave == 0 && live) put_entries(d, entries, a.top, share, scale, g);
    }
}

// Rows too wide for registers, or of less than a piece: read once for the statistics and once more for the gradient.
template <class T>
__global__ __launch_bounds__(kWideBlock) void k_distill_wide(DistillArgs a) {
    constexpr int N = kN<T>, STEP = kWideBlock * N;
    extern __shared__ __attribute__((aligned(16))) char space[];
    Entry *entries = reinterpret_cast<Entry *>(space);
    __shared__ float4 lds[kWideWaves];
    const float k2 = a.k2;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *l = static_cast<const T *>(a.logits) + row * a.logits_stride;
        Teacher t{};
        if (threadIdx.x < kWave) t = entries_of<T>(a, row, 0, a.cols, entries);
        float top = -kInf, sum = 0.0f;
#pragma unroll 4
        for (int c = threadIdx.x * N; c < a.cols; c += STEP) {
            const F<N> f = widen<T, N>(load<N>(l, c, a.cols, T(-kInf)));
            float m = top;
#pragma unroll
            for (int j = 0; j < N; ++j) m = fmaxf(m, f[j]);
            const Relative from{m == -kInf ? 0.0f : m, k2};
            sum *= top == -kInf ? 1.0f : from(top);
#pragma unroll
            for (int j = 0; j < N; ++j) sum += from(f[j]);
            top = m;
        }
        const float mine = top;
        top = wave_max(top);
        sum = wave_sum(mine == -kInf ? sum : sum * Relative{top, k2}(mine));
        __syncthreads();      // the last row's readers are done
        if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = make_float4(top, sum, t.trained ? 1.0f : 0.0f, 0.0f);
        __syncthreads();
#pragma unroll
        for (int v = 0; v < kWideWaves; ++v) top = fmaxf(top, lds[v].x);
        sum = 0.0f;
#pragma unroll
        for (int v = 0; v < kWideWaves; ++v) {
            const float4 p = lds[v];
            sum += p.x == -kInf ? p.y : p.y * Relative{top, k2}(p.x);
        }
        const bool live = lds[0].z > 0.0f && (top != -kInf || sum != sum);
        if (sum != sum) top = sum;
        if (threadIdx.x < kWave) finish_row(a, row, t, entries, top, sum);
        if (!a.grad) continue;
        T *d = static_cast<T *>(a.grad) + row * a.grad_stride;
        const Relative share{top, k2};
        const float g = a.grad_loss[row] * a.temperature, scale = g / sum;
        for (int c = threadIdx.x * N; c < a.cols; c += STEP) {
            F<N> f = 0.0f;
            if (live) {
                f = widen<T, N>(load<N>(l, c, a.cols));
#pragma unroll
                for (int j = 0; j < N; ++j) f[j] = share(f[j]) * scale;
            }
            store<N>(d, c, a.cols, round_to<T, N>(f));
        }
        settled<kWideWaves>();
        if (threadIdx.x < kWave && live) put_entries(d, entries, a.top, share, scale, g);
    }
}

// The gradient alone, from the whole vocabulary's lse: a workgroup takes a stretch of one row, and the teacher's entries in it.
// 1000 x 12801 of half precision with 33 ids a row: 15.3 us, 3.3 TB/s, since each of a row's two workgroups prepares its entries.
constexpr int kGradPieces = 4;
template <class T>
__global__ __launch_bounds__(256) void k_distill_grad(DistillArgs a) {
    constexpr int N = kN<T>, K = kGradPieces, SPAN = K * 256 * N;
    extern __shared__ __attribute__((aligned(16))) char space[];
    Entry *entries = reinterpret_cast<Entry *>(space);
    __shared__ int lds;
    const float inv_t = a.inv_t;
    const int spans = (a.cols + SPAN - 1) / SPAN;
    const int64_t n = a.rows * spans;
    for (int64_t id = blockIdx.x; id < n; id += gridDim.x) {
        const int64_t row = id / spans;
        const int first = (int)(id - row * spans) * SPAN, from = first + threadIdx.x * N;
        const T *l = static_cast<const T *>(a.logits) + row * a.logits_stride;
        T *d = static_cast<T *>(a.grad) + row * a.grad_stride;
        V<T, N> raw[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            raw[k] = T(0);
            if (from + k * 256 * N < a.cols) raw[k] = load<N>(l, from + k * 256 * N, a.cols);
        }
        if (threadIdx.x < kWave) {
            const Teacher t = entries_of<T>(a, row, first, SPAN, entries);
            if (threadIdx.x == 0) lds = t.trained;
        }
        __syncthreads();      // also: the teacher's logits have been read
        const float lse = a.lse_in[row], g = a.grad_loss[row] * a.temperature;
        const bool live = lds && lse != -kInf;
        const Given share{lse, inv_t};
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = from + k * 256 * N;
            if (c >= a.cols) continue;
            F<N> f = 0.0f;
            if (live) {
                f = widen<T, N>(raw[k]);
#pragma unroll
                for (int j = 0; j < N; ++j) f[j] = share(f[j]) * g;
            }
            drop<N>(d, c, a.cols, round_to<T, N>(f));
        }
        settled<4>();
        if (threadIdx.x < kWave && live) put_entries(d, entries, a.top, share, g, g);
    }
}

template <class A>
hipError_t launch_with(void (*kernel)(A), unsigned grid, int block, size_t lds, hipStream_t s, A a) {
    void *args[] = {&a};
    return hipLaunchKernel(reinterpret_cast<const void *>(kernel), dim3(grid), dim3(block), args, lds, s);
}
template <class T, bool CUT>
hipError_t rows(const DistillArgs &a, hipStream_t s) {
    const size_t each = sizeof(Entry) * a.top;
    const auto run = [&](auto kernel, int threads) {
        const int teams = threads < 256 ? 256 / threads : 1;
        return launch_with(kernel, grid_of((a.rows + teams - 1) / teams), threads * teams, each * teams, s, a);
    };
    if (a.cols < kN<T> || a.cols > 1024 * 64)
        return launch_with(k_distill_wide<T>, grid_of(a.rows), kWideBlock, each, s, a);
    if (a.cols <= 64 * 8) return run(k_distill<T, 64, 8, CUT>, 64);
    if (a.cols <= 64 * 32) return run(k_distill<T, 64, 32, CUT>, 64);
    if (a.cols <= 256 * 32) return run(k_distill<T, 256, 32, CUT>, 256);
    if (a.cols <= 512 * 32) return run(k_distill<T, 512, 32, CUT>, 512);
    if (a.cols <= 1024 * 32) return run(k_distill<T, 1024, 32, CUT>, 1024);
    if (a.cols <= 1024 * 48) return run(k_distill<T, 1024, 48, CUT>, 1024);
    return run(k_distill<T, 1024, 64, CUT>, 1024);
}
template <class T>
hipError_t distill(const DistillArgs &a, hipStream_t s) {
    if (a.lse_in) {
        constexpr int SPAN = kGradPieces * 256 * kN<T>;
        return launch_with(k_distill_grad<T>, grid_of(a.rows * ((a.cols + SPAN - 1) / SPAN)), 256, sizeof(Entry) * a.top, s, a);
    }
    return a.cols % kN<T> ? rows<T, true>(a, s) : rows<T, false>(a, s);
}
}  // namespace

hipError_t launch_distill(const DistillArgs &a, int type, hipStream_t s) {
    switch (type) {
        case ECHO_F32: return distill<float>(a, s);
        case ECHO_F16: return distill<f16>(a, s);
        default: return distill<bf16>(a, s);
    }
}

}  // namespace echo
