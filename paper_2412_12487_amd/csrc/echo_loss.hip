// echo_loss.hip -- cross entropy over a vocabulary or a shard of one, and its gradient, on gfx950.
#include "echo_ops_device.h"

namespace echo {
namespace {

// What a row's loss and gradient are computed with.
struct LossRow {
    bool trained;      // the target is an id of the vocabulary
    int at;            // its column here, or -1
};
template <class I>
__device__ __forceinline__ LossRow loss_row(const LossArgs &a, int64_t row) {
    const int64_t t = id_at<I>(a.targets, row);
    const bool trained = t >= 0 && t < a.vocab_size;
    return LossRow{trained, trained ? shard_row(t, a.vocab_start, a.cols) : -1};
}
// exp(x), x <= 0 but for a row's rounding: one multiplication and the hardware's 2^x.  The product's rounding
// makes the result |x| 2^-24 of itself wrong, as does that of x itself.
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }

// exp(l - base) * scale - [column = target] * g for the columns col .. col + N - 1.  The target is looked for once a piece:
// with a comparison an element a pass of 2048 x 51200 took 107.2 us instead of 103.6 (79.4 now, for the reason at k_loss).
template <int N>
__device__ __forceinline__ F<N> loss_grad(F<N> l, float base, float scale, int col, int at, float g) {
    F<N> d;
#pragma unroll
    for (int j = 0; j < N; ++j) d[j] = exp_of(l[j] - base) * scale;
    if ((unsigned)(at - col) < (unsigned)N) {      // at is -1 or a column
#pragma unroll
        for (int j = 0; j < N; ++j) d[j] -= col + j == at ? g : 0.0f;
    }
    return d;
}
// Log of the sum of exponentials from a maximum and a sum relative to it, written with the row's loss.  The loss
// and a gradient in the same pass are taken from the maximum and the sum, not from their rounded total: in a row of
// large logits (one masked throughout with the type's lowest value, say) the logarithm is below the maximum's last place.
__device__ __forceinline__ float finish_row(const LossArgs &a, int64_t row, const LossRow &r, float hit, float top, float sum,
                                            bool writes) {
    const float more = logf(sum), lse = top == -kInf ? -kInf : top + more;
    if (writes) {
        if (a.lse) a.lse[row] = lse;
        if (a.target) a.target[row] = hit;
        if (a.loss) a.loss[row] = !r.trained ? 0.0f : lse == -kInf ? kInf : (top - hit) + more;
    }
    return lse;
}

// A team a row, which is read once and stays in registers as it came; with a gradient it is written
// from there.  Each wavefront takes its maximum and its sum of exponentials relative to it; the team joins
// them with one exchange.  Memory bounds it: 2048 x 51200 of bf16 with its gradient takes 65.5 us, 6.4 TB/s, on logits that
// the 256 MB cache still has, and 79.4 a pass on new ones, 5.3 TB/s.  Without a gradient the workgroups of a launch read
// together and reduce together: 512 x 25600 in 9.6 us, 2.7 TB/s.
// Wavefronts a SIMD that a variant's registers have to leave room for: two workgroups of 16 wavefronts on a compute unit, one
// reading while the other computes or writes, where the row takes at most half of the 64 registers that each lane then
// has.  A pass of 2048 x 51200 of bf16 took 103.6 us with 95 to 128 registers and one workgroup, and 77.9 with two.  The
// compiler stays within 64 because each piece's sums are closed before the next piece is converted (the empty asm in the loops).
template <class T, int THREADS, int E>
constexpr int kLossWaves = THREADS == 1024 && E * sizeof(T) <= 128 ? 8 : 1;
template <class T, class I, int THREADS, int E, bool CUT>
__global__ __launch_bounds__((Team<T, THREADS, E, CUT>::BLOCK), (kLossWaves<T, THREADS, E>)) void k_loss(LossArgs a) {
    using Q = Team<T, THREADS, E, CUT>;
    constexpr int N = Q::N, P = Q::P;
    const Q q(a.cols);
    __shared__ float2 lds[2][Q::WAVES];
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * Q::TEAMS + q.team; row < a.rows; row += (int64_t)gridDim.x * Q::TEAMS) {
        const T *l = static_cast<const T *>(a.logits) + row * a.logits_stride;
        V<T, N> x[P];
        q.load(l, x, T(-kInf));
        const LossRow r = loss_row<I>(a, row);
        const float hit = r.at >= 0 ? (float)l[r.at] : 0.0f, g = a.grad ? a.grad_loss[row] : 0.0f;
        float top = -kInf, sum = 0.0f;
#pragma unroll
        for (int k = 0; k < P; ++k) {
            const F<N> f = widen<T, N>(x[k]);
#pragma unroll
            for (int j = 0; j < N; ++j) top = fmaxf(top, f[j]);
            if constexpr (kLossWaves<T, THREADS, E> > 1) asm volatile("" : "+v"(top));
        }
        forget<T, N, P>(x);
        top = wave_max(top);
        const float base = top == -kInf ? 0.0f : top;      // nothing here: the sum is 0
#pragma unroll
        for (int k = 0; k < P; ++k) {
            const F<N> f = widen<T, N>(x[k]);
#pragma unroll
            for (int j = 0; j < N; ++j) sum += exp_of(f[j] - base);
            if constexpr (kLossWaves<T, THREADS, E> > 1) asm volatile("" : "+v"(sum));
        }
        forget<T, N, P>(x);
        sum = wave_sum(sum);
        if constexpr (Q::WAVES > 1) {
            if (q.lane % kWave == 0) lds[turn][q.wave] = make_float2(top, sum);
            __syncthreads();      // also: every lane has read the target's logit, and grad may be logits
            const float2 p = lds[turn][q.lane % Q::WAVES];      // a wavefront's in a lane
            top = ring_max<Q::WAVES>(p.x);
            sum = ring_sum<Q::WAVES>(p.x == -kInf ? p.y : p.y * exp_of(p.x - top));      // p.y is 0 there, or NaN
            turn ^= 1;
        }
        // a row of NaN alone has no maximum but a sum
        if (sum != sum) top = sum;
        const float lse = finish_row(a, row, r, hit, top, sum, q.lane == 0), scale = g / sum;
        if (!a.grad) continue;
        const bool live = r.trained && lse != -kInf;
#pragma unroll
        for (int k = 0; k < P; ++k) {
            F<N> f = 0.0f;
            if (live) f = loss_grad<N>(widen<T, N>(x[k]), top, scale, q.col(k), r.at, g);
            x[k] = round_to<T, N>(f);
            if constexpr (kLossWaves<T, THREADS, E> > 1) forget<T, N, 1>(reinterpret_cast<V<T, N>(&)[1]>(x[k]));
        }
        q.drop(static_cast<T *>(a.grad) + row * a.grad_stride, x);
    }
}

// Rows too wide for registers, or of less than a piece: one workgroup a row, read once for a running maximum and sum a lane, and
// with a gradient once more.  2048 x 65544 of bf16: 55.4 us without a gradient, 4.8 TB/s, and 133.6 with one.
template <class T, class I>
__global__ __launch_bounds__(kWideBlock) void k_loss_wide(LossArgs a) {
    constexpr int N = kN<T>, STEP = kWideBlock * N;
    __shared__ float2 lds[kWideWaves];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *l = static_cast<const T *>(a.logits) + row * a.logits_stride;
        const LossRow r = loss_row<I>(a, row);
        const float hit = r.at >= 0 ? (float)l[r.at] : 0.0f;
        float top = -kInf, sum = 0.0f;
#pragma unroll 4
        for (int c = threadIdx.x * N; c < a.cols; c += STEP) {
            const F<N> f = widen<T, N>(load<N>(l, c, a.cols, T(-kInf)));
            float m = top;
#pragma unroll
            for (int j = 0; j < N; ++j) m = fmaxf(m, f[j]);
            const float base = m == -kInf ? 0.0f : m;
            sum *= top == -kInf ? 1.0f : exp_of(top - base);      // before a first finite logit the sum is 0, or NaN
#pragma unroll
            for (int j = 0; j < N; ++j) sum += exp_of(f[j] - base);
            top = m;
        }
        const float mine = top;
        top = wave_max(top);
        sum = wave_sum(mine == -kInf ? sum : sum * exp_of(mine - top));
        __syncthreads();      // the last row's readers are done
        if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = make_float2(top, sum);
        __syncthreads();
#pragma unroll
        for (int v = 0; v < kWideWaves; ++v) top = fmaxf(top, lds[v].x);
        sum = 0.0f;
#pragma unroll
        for (int v = 0; v < kWideWaves; ++v) {
            const float2 p = lds[v];
            sum += p.x == -kInf ? p.y : p.y * exp_of(p.x - top);
        }
        if (sum != sum) top = sum;
        const float lse = finish_row(a, row, r, hit, top, sum, threadIdx.x == 0);
        if (!a.grad) continue;
        T *d = static_cast<T *>(a.grad) + row * a.grad_stride;
        const bool live = r.trained && lse != -kInf;
        const float g = a.grad_loss[row], scale = g / sum;
        for (int c = threadIdx.x * N; c < a.cols; c += STEP) {
            F<N> f = 0.0f;
            if (live) f = loss_grad<N>(widen<T, N>(load<N>(l, c, a.cols)), top, scale, c, r.at, g);
            store<N>(d, c, a.cols, round_to<T, N>(f));
        }
    }
}

// The gradient alone, K pieces a lane of one row's stretch of 256 * K pieces: 512 x 25600 of bf16 in 10.7 us, 4.9 TB/s.
constexpr int kGradPieces = 2;
template <class T, class I>
__global__ __launch_bounds__(256) void k_loss_grad(LossArgs a) {
    constexpr int N = kN<T>, K = kGradPieces, SPAN = K * 256 * N;
    const int spans = (a.cols + SPAN - 1) / SPAN;
    const int64_t n = a.rows * spans;
    for (int64_t id = blockIdx.x; id < n; id += gridDim.x) {
        const int64_t row = id / spans;
        const int from = (int)(id - row * spans) * SPAN + threadIdx.x * N;
        const T *l = static_cast<const T *>(a.logits) + row * a.logits_stride;
        T *d = static_cast<T *>(a.grad) + row * a.grad_stride;
        V<T, N> raw[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            raw[k] = T(0);
            if (from + k * 256 * N < a.cols) raw[k] = load<N>(l, from + k * 256 * N, a.cols);
        }
        const LossRow r = loss_row<I>(a, row);
        const float lse = a.lse_in[row], g = a.grad_loss[row];
        const bool live = r.trained && lse != -kInf;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = from + k * 256 * N;
            if (c >= a.cols) continue;
            F<N> f = 0.0f;
            if (live) f = loss_grad<N>(widen<T, N>(raw[k]), lse, g, c, r.at, g);
            drop<N>(d, c, a.cols, round_to<T, N>(f));
        }
    }
}

template <class T, class I, bool CUT>
hipError_t loss(const LossArgs &a, hipStream_t s) {
    const auto run = [&](auto kernel, int threads) {
        const int teams = threads < 256 ? 256 / threads : 1;
        return launch(kernel, dim3(grid_of((a.rows + teams - 1) / teams)), dim3(threads * teams), s, a);
    };
    if (a.cols < kN<T> || a.cols > 1024 * 64)
        return launch(k_loss_wide<T, I>, dim3(grid_of(a.rows)), dim3(kWideBlock), s, a);
    if (a.cols <= 64 * 8) return run(k_loss<T, I, 64, 8, CUT>, 64);
    if (a.cols <= 64 * 32) return run(k_loss<T, I, 64, 32, CUT>, 64);
    if (a.cols <= 256 * 32) return run(k_loss<T, I, 256, 32, CUT>, 256);
    if (a.cols <= 512 * 32) return run(k_loss<T, I, 512, 32, CUT>, 512);
    if (a.cols <= 1024 * 32) return run(k_loss<T, I, 1024, 32, CUT>, 1024);
    // A lane computes on every piece that the variant has, also past the row's end: 2048 rows of 33000 columns of bf16 take
    // 64.0 us with 64 elements a lane and 46.0 with 40, 48000 columns 65.3 us with 64 and 61.2 with 48; 56 elements
    // gained nothing over 64 (51200 columns: 65.1 us with either).
    if (a.cols <= 1024 * 40) return run(k_loss<T, I, 1024, 40, CUT>, 1024);
    if (a.cols <= 1024 * 48) return run(k_loss<T, I, 1024, 48, CUT>, 1024);
    return run(k_loss<T, I, 1024, 64, CUT>, 1024);
}
template <class T, class I>
hipError_t loss_grad_alone(const LossArgs &a, hipStream_t s) {
    constexpr int SPAN = kGradPieces * 256 * kN<T>;
    return launch(k_loss_grad<T, I>, dim3(grid_of(a.rows * ((a.cols + SPAN - 1) / SPAN))), dim3(256), s, a);
}

}  // namespace

template <class T, class I>
static hipError_t loss_rows(const LossArgs &a, hipStream_t s) {
    return a.cols % kN<T> ? loss<T, I, true>(a, s) : loss<T, I, false>(a, s);
}
template <class I>
static hipError_t loss_of(const LossArgs &a, int type, bool grad_alone, hipStream_t s) {
    switch (type) {
        case ECHO_F32: return grad_alone ? loss_grad_alone<float, I>(a, s) : loss_rows<float, I>(a, s);
        case ECHO_F16: return grad_alone ? loss_grad_alone<f16, I>(a, s) : loss_rows<f16, I>(a, s);
        default: return grad_alone ? loss_grad_alone<bf16, I>(a, s) : loss_rows<bf16, I>(a, s);
    }
}
hipError_t launch_loss(const LossArgs &a, int type, int index_type, hipStream_t s) {
    return index_type == ECHO_I64 ? loss_of<int64_t>(a, type, false, s) : loss_of<int32_t>(a, type, false, s);
}
hipError_t launch_loss_grad(const LossArgs &a, int type, int index_type, hipStream_t s) {
    return index_type == ECHO_I64 ? loss_of<int64_t>(a, type, true, s) : loss_of<int32_t>(a, type, true, s);
}

}  // namespace echo
