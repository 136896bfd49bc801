// echo_ops.hip -- gfx950 kernels of the training-step operators (echo_ops.h).
//
// All of them move bytes: nothing multiplies matrices, and every operator's floor is the time
// to read its inputs and write its outputs once.  A lane moves 16 bytes of activations at a time with the
// alignment of one element (the hardware takes 16 bytes from any address), rows that fit stay in registers between
// their statistics and their result, sums and statistics are held in 32 bits, and no result depends
// on the order in which workgroups run.
#include "echo_ops_internal.h"

namespace echo {
namespace {

using bf16 = __bf16;
using f16 = _Float16;

constexpr int kWave = 64;
constexpr unsigned kMaxGrid = 1u << 20;  // workgroups of a launch, at most; kernels stride over the rest
constexpr float kInf = __builtin_huge_valf();

// Elements of 16 bytes: what a lane moves at a time of activations of type T.
template <class T>
constexpr int kN = 16 / sizeof(T);
template <class T, int N>
struct VecOf {
    typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};
template <class T, int N>
using V = typename VecOf<T, N>::type;
template <int N>
using F = V<float, N>;

// Elements col .. col + N - 1 of a row of `cols`; `fill` stands where the row has ended.
template <int N, class T>
__device__ __forceinline__ V<T, N> load(const T *row, int col, int cols, T fill = T(0)) {
    if (col + N <= cols) return *reinterpret_cast<const V<T, N> *>(row + col);
    V<T, N> v;
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = col + j < cols ? row[col + j] : fill;
    return v;
}
// load of data that nothing reads again soon.
template <int N, class T>
__device__ __forceinline__ V<T, N> stream(const T *row, int col, int cols) {
    if (col + N <= cols) return __builtin_nontemporal_load(reinterpret_cast<const V<T, N> *>(row + col));
    return load<N>(row, col, cols);
}
template <int N, class T>
__device__ __forceinline__ void store(T *row, int col, int cols, V<T, N> v) {
    if (col + N <= cols) {
        *reinterpret_cast<V<T, N> *>(row + col) = v;
        return;
    }
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (col + j < cols) row[col + j] = v[j];
}
// store of results that stream out: whole 16-byte pieces of a lane, side by side over the lanes.
// Measured on layer norm of 2048 x 8192: 29.0 us with plain stores, 26.7 with these.
template <int N, class T>
__device__ __forceinline__ void drop(T *row, int col, int cols, V<T, N> v) {
    static_assert(N == kN<T>, "");
    if (col + N <= cols)
        __builtin_nontemporal_store(v, reinterpret_cast<V<T, N> *>(row + col));
    else
        store<N>(row, col, cols, v);
}
template <class T, int N>
__device__ __forceinline__ F<N> widen(V<T, N> v) {
    return __builtin_convertvector(v, F<N>);
}
template <class T, int N>
__device__ __forceinline__ V<T, N> round_to(F<N> v) {
    return __builtin_convertvector(v, V<T, N>);
}

// Sum and maximum over a wavefront, the same in every lane: rotations within 16 lanes (each lane then has
// its 16 lanes' value, in one order), then the four groups in order.  A maximum passes over NaN: a row
// with a NaN has it in its sum.
template <int BY>
__device__ __forceinline__ float rotated(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + BY, 0xf, 0xf, false));
}
__device__ __forceinline__ float lane_of(float v, int lane) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}
__device__ __forceinline__ float wave_sum(float v) {
    v += rotated<8>(v);
    v += rotated<4>(v);
    v += rotated<2>(v);
    v += rotated<1>(v);
    return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}
__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, rotated<8>(v));
    v = fmaxf(v, rotated<4>(v));
    v = fmaxf(v, rotated<2>(v));
    v = fmaxf(v, rotated<1>(v));
    return fmaxf(fmaxf(lane_of(v, 0), lane_of(v, 16)), fmaxf(lane_of(v, 32), lane_of(v, 48)));
}

// Sum over a workgroup of WAVES wavefronts, added in the order of the wavefronts.
template <int WAVES>
__device__ __forceinline__ float block_sum(float v, float *lds) {
    v = wave_sum(v);
    __syncthreads();
    if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = v;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s += lds[w];
    return s;
}

template <class A, class... B>
hipError_t launch(void (*kernel)(A, B...), dim3 grid, dim3 block, hipStream_t s, A a, B... rest) {
    void *args[] = {&a, &rest...};
    return hipLaunchKernel(reinterpret_cast<const void *>(kernel), grid, block, args, 0, s);
}
unsigned grid_of(int64_t n) { return (unsigned)(n < 1 ? 1 : n < (int64_t)kMaxGrid ? n : (int64_t)kMaxGrid); }

// A piece as 32-bit words.
template <class T, int N>
struct WordsOf {
    typedef int type __attribute__((ext_vector_type(N * sizeof(T) / 4)));
};
template <class T, int N>
using Words = typename WordsOf<T, N>::type;
template <class T, int N>
__device__ __forceinline__ Words<T, N> words_of(V<T, N> v) {
    return __builtin_bit_cast(Words<T, N>, v);
}
// Keeps the compiler from holding what it made of v: from here on v is converted anew.
template <class T, int N>
__device__ __forceinline__ void forget(V<T, N> &v) {
    Words<T, N> w = words_of<T, N>(v);
    asm volatile("" : "+v"(w));
    v = __builtin_bit_cast(V<T, N>, w);
}

// A team of THREADS lanes holds a row of up to THREADS * E elements in registers, E a lane, as K pieces of 16
// bytes of T: lane i has the pieces k * THREADS + i.  Narrow teams share a workgroup of four wavefronts.
// Only one piece of a row can be cut off by its end: it is moved element by element, apart from the
// others, so that they need no code for it.
template <class T, int THREADS, int E>
struct Team {
    static constexpr int N = kN<T>, K = E / N, BLOCK = THREADS < 256 ? 256 : THREADS, TEAMS = BLOCK / THREADS,
                         WAVES = THREADS / kWave;
    static_assert(K * N == E, "");
    const int lane = threadIdx.x % THREADS, wave = __builtin_amdgcn_readfirstlane(lane / kWave),
              team = __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS), cols, left = cols % N;
    __device__ __forceinline__ explicit Team(int c) : cols(c) {}
    __device__ __forceinline__ unsigned col(int k) const { return (unsigned)(k * THREADS + lane) * N; }
    __device__ __forceinline__ bool whole(int k) const { return (int)col(k) + N <= cols; }
    // elements that wavefront w has of the row
    __device__ __forceinline__ int count(int w) const {
        int n = 0;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int rest = cols - (k * THREADS + w * kWave) * N;
            n += rest < 0 ? 0 : rest < kWave * N ? rest : kWave * N;
        }
        return n;
    }
    template <class U>
    __device__ __forceinline__ void load(const U *row, V<U, N> (&v)[K], U fill = U(0)) const {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = fill;
            if (whole(k)) v[k] = *reinterpret_cast<const V<U, N> *>(row + col(k));
        }
        if (left == 0) return;
        const int piece = cols / N;
        if (lane != piece % THREADS) return;
        V<U, N> t = fill;
#pragma unroll
        for (int j = 0; j < N - 1; ++j) t[j] = j < left ? row[piece * N + j] : fill;
#pragma unroll
        for (int k = 0; k < K; ++k) {      // by masks: an index would put v into memory
            const int m = -(int)(k == piece / THREADS);
            v[k] = __builtin_bit_cast(V<U, N>, (words_of<U, N>(t) & m) | (words_of<U, N>(v[k]) & ~m));
        }
    }
    template <bool DROP, class U>
    __device__ __forceinline__ void put(U *row, const V<U, N> (&v)[K]) const {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (!whole(k)) continue;
            V<U, N> *p = reinterpret_cast<V<U, N> *>(row + col(k));
            if constexpr (DROP)
                __builtin_nontemporal_store(v[k], p);
            else
                *p = v[k];
        }
        if (left == 0) return;
        const int piece = cols / N;
        if (lane != piece % THREADS) return;
        Words<U, N> w = 0;
#pragma unroll
        for (int k = 0; k < K; ++k) w |= words_of<U, N>(v[k]) & -(int)(k == piece / THREADS);
        const V<U, N> t = __builtin_bit_cast(V<U, N>, w);
#pragma unroll
        for (int j = 0; j < N - 1; ++j)
            if (j < left) row[piece * N + j] = t[j];
    }
    // Results that stream out: past the caches, in whole 16-byte pieces side by side over the lanes.
    // Measured on layer norm of 2048 x 8192 with a residual: 29.0 us with plain stores, 26.7 with these.
    __device__ __forceinline__ void drop(T *row, const V<T, N> (&v)[K]) const { put<true>(row, v); }
    template <class U>
    __device__ __forceinline__ void store(U *row, const V<U, N> (&v)[K]) const {
        put<false>(row, v);
    }
};

// ---------------------------------------------------------------- layer norm

// A team a row, which is read once.  The mean and the sum of squares about it are taken per wavefront, both
// from the registers, and joined over the team's wavefronts (n, mean, squares) in their order, so the team
// waits for itself once a row.
template <class T, class W, int THREADS, int E>
__global__ __launch_bounds__((Team<T, THREADS, E>::BLOCK)) void k_norm(NormArgs a) {
    using Q = Team<T, THREADS, E>;
    constexpr int N = Q::N, K = Q::K;
    constexpr bool kEarly = E <= 16;      // the weights wait in registers while the team joins its sums
    const Q q(a.cols);
    __shared__ float2 lds[2][Q::WAVES];
    const W *w = static_cast<const W *>(a.weight), *b = static_cast<const W *>(a.bias);
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * Q::TEAMS + q.team; row < a.rows; row += (int64_t)gridDim.x * Q::TEAMS) {
        V<T, N> x[K];
        V<W, N> wv[K], bv[K];
        q.load(static_cast<const T *>(a.x) + row * a.x_stride, x);
        if (a.residual) {
            V<T, N> r[K];
            q.load(static_cast<const T *>(a.residual) + row * a.residual_stride, r);
#pragma unroll
            for (int k = 0; k < K; ++k) x[k] = round_to<T, N>(widen<T, N>(x[k]) + widen<T, N>(r[k]));
            q.drop(static_cast<T *>(a.sum) + row * a.cols, x);
        }
        if constexpr (kEarly) {
            q.load(w, wv);
            if (b) q.load(b, bv);
        }
        float s = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const F<N> f = widen<T, N>(x[k]);
#pragma unroll
            for (int j = 0; j < N; ++j) s += f[j];
            forget<T, N>(x[k]);
        }
        const int n = q.count(q.wave);
        float mean = n ? wave_sum(s) / (float)n : 0.0f, squares = 0.0f;
        if (n == kWave * E) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const F<N> d = widen<T, N>(x[k]) - mean;
#pragma unroll
                for (int j = 0; j < N; ++j) squares += d[j] * d[j];
                forget<T, N>(x[k]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const F<N> d = widen<T, N>(x[k]) - mean;
#pragma unroll
                for (int j = 0; j < N; ++j) squares += (int)q.col(k) + j < a.cols ? d[j] * d[j] : 0.0f;
                forget<T, N>(x[k]);
            }
        }
        squares = wave_sum(squares);
        if constexpr (Q::WAVES > 1) {
            if (q.lane % kWave == 0) lds[turn][q.wave] = make_float2(mean, squares);
            __syncthreads();
            float all = 0.0f;
#pragma unroll
            for (int v = 0; v < Q::WAVES; ++v) all += (float)q.count(v) * lds[turn][v].x;
            mean = all / (float)a.cols;
            squares = 0.0f;
#pragma unroll
            for (int v = 0; v < Q::WAVES; ++v) {
                const float2 p = lds[turn][v];
                const float m = (float)q.count(v), d = p.x - mean;
                squares += m ? p.y + m * d * d : 0.0f;
            }
            turn ^= 1;      // the next row's exchange does not meet this one's readers
        }
        const float rstd = 1.0f / sqrtf(squares / (float)a.cols + a.eps);
        if constexpr (!kEarly) {
            q.load(w, wv);
            if (b) q.load(b, bv);
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            F<N> f = (widen<T, N>(x[k]) - mean) * rstd * widen<W, N>(wv[k]);
            if (b) f += widen<W, N>(bv[k]);
            x[k] = round_to<T, N>(f);
        }
        q.drop(static_cast<T *>(a.y) + row * a.cols, x);
        if (q.lane == 0) {
            a.mean[row] = mean;
            a.rstd[row] = rstd;
        }
    }
}

constexpr int kWideBlock = 1024, kWideWaves = kWideBlock / kWave;

// Rows too wide for registers: one workgroup a row, which is read three times (sum, squares about the
// mean, result), from the cache after the first.
template <class T, class W>
__global__ __launch_bounds__(kWideBlock) void k_norm_wide(NormArgs a) {
    constexpr int N = kN<T>, STEP = kWideBlock * N;
    __shared__ float lds[kWideWaves];
    const int from = threadIdx.x * N;
    const W *w = static_cast<const W *>(a.weight), *b = static_cast<const W *>(a.bias);
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
        const T *h = x;
        float s = 0.0f;
        if (a.residual) {
            const T *r = static_cast<const T *>(a.residual) + row * a.residual_stride;
            T *sum = static_cast<T *>(a.sum) + row * a.cols;
            for (int c = from; c < a.cols; c += STEP) {
                const V<T, N> v = round_to<T, N>(widen<T, N>(load<N>(x, c, a.cols)) + widen<T, N>(load<N>(r, c, a.cols)));
                store<N>(sum, c, a.cols, v);
                const F<N> f = widen<T, N>(v);
                for (int j = 0; j < N; ++j) s += f[j];
            }
            h = sum;      // each lane reads back what it wrote
        } else {
            for (int c = from; c < a.cols; c += STEP) {
                const F<N> f = widen<T, N>(load<N>(x, c, a.cols));
                for (int j = 0; j < N; ++j) s += f[j];
            }
        }
        const float mean = block_sum<kWideWaves>(s, lds) / (float)a.cols;
        s = 0.0f;
        for (int c = from; c < a.cols; c += STEP) {
            const F<N> f = widen<T, N>(load<N>(h, c, a.cols));
            for (int j = 0; j < N; ++j) {
                const float d = c + j < a.cols ? f[j] - mean : 0.0f;
                s += d * d;
            }
        }
        const float rstd = 1.0f / sqrtf(block_sum<kWideWaves>(s, lds) / (float)a.cols + a.eps);
        T *y = static_cast<T *>(a.y) + row * a.cols;
        for (int c = from; c < a.cols; c += STEP) {
            F<N> f = (widen<T, N>(load<N>(h, c, a.cols)) - mean) * rstd * widen<W, N>(load<N>(w, c, a.cols));
            if (b) f += widen<W, N>(load<N>(b, c, a.cols));
            store<N>(y, c, a.cols, round_to<T, N>(f));
        }
        if (threadIdx.x == 0) {
            a.mean[row] = mean;
            a.rstd[row] = rstd;
        }
    }
}

template <class T, class W>
hipError_t norm(const NormArgs &a, hipStream_t s) {
    // The narrowest team that holds the row: few lanes idle, few wavefronts wait for each other.
    const auto run = [&](auto kernel, int threads) {
        const int teams = threads < 256 ? 256 / threads : 1;
        return launch(kernel, dim3(grid_of((a.rows + teams - 1) / teams)), dim3(threads * teams), s, a);
    };
    if (a.cols <= 64 * 8) return run(k_norm<T, W, 64, 8>, 64);
    if (a.cols <= 64 * 16) return run(k_norm<T, W, 64, 16>, 64);
    if (a.cols <= 256 * 8) return run(k_norm<T, W, 256, 8>, 256);
    if (a.cols <= 256 * 16) return run(k_norm<T, W, 256, 16>, 256);
    if (a.cols <= 512 * 16) return run(k_norm<T, W, 512, 16>, 512);
    if (a.cols <= 512 * 24) return run(k_norm<T, W, 512, 24>, 512);
    if (a.cols <= 512 * 32) return run(k_norm<T, W, 512, 32>, 512);
    return launch(k_norm_wide<T, W>, dim3(grid_of(a.rows)), dim3(kWideBlock), s, a);
}

// Gradients, x and dy read once.  A team takes every (teams of the launch)-th row and keeps its lanes' columns
// of dweight and dbias in registers, which leaves the chip few wavefronts; so the next two rows are on
// their way while one is worked on (fewer where wide rows fill the registers by themselves).  A
// workgroup leaves one row of each weight sum in `part`.
template <class T, class W, int THREADS, int E>
__global__ __launch_bounds__((Team<T, THREADS, E>::BLOCK)) void k_norm_grad(NormGradArgs a) {
    using Q = Team<T, THREADS, E>;
    constexpr int N = Q::N, K = Q::K;
    constexpr int kRows = E * sizeof(T) <= 48 ? 3 : E * sizeof(T) <= 64 ? 2 : 1;      // in registers
    struct Row {
        V<T, N> x[K], dy[K], past[K];
        float mean, rstd;
    };
    const Q q(a.cols);
    __shared__ float2 lds[2][Q::WAVES];
    const int64_t step = (int64_t)gridDim.x * Q::TEAMS;
    V<W, N> wv[K];
    F<N> dw[K], db[K];
    int turn = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) dw[k] = db[k] = 0.0f;
    const auto fetch = [&](Row &r, int64_t row) {
        if (row >= a.rows) return;
        q.load(static_cast<const T *>(a.x) + row * a.x_stride, r.x);
        q.load(static_cast<const T *>(a.dy) + row * a.dy_stride, r.dy);
        if (a.grad_residual) q.load(static_cast<const T *>(a.grad_residual) + row * a.grad_residual_stride, r.past);
        r.mean = a.mean[row];
        r.rstd = a.rstd[row];
    };
    const auto work = [&](Row &r, int64_t row) {
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            // past the row's end dy and weight are 0, and so are g and its products, unless the row has
            // no finite statistics: then all of it has none
            const F<N> d = widen<T, N>(r.dy[k]), n = (widen<T, N>(r.x[k]) - r.mean) * r.rstd, g = d * widen<W, N>(wv[k]);
            dw[k] += d * n;
            db[k] += d;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                s1 += g[j];
                s2 += g[j] * n[j];
            }
            forget<T, N>(r.x[k]);
            forget<T, N>(r.dy[k]);
        }
        s1 = wave_sum(s1);
        s2 = wave_sum(s2);
        if constexpr (Q::WAVES > 1) {
            if (q.lane % kWave == 0) lds[turn][q.wave] = make_float2(s1, s2);
            __syncthreads();
            s1 = s2 = 0.0f;
#pragma unroll
            for (int v = 0; v < Q::WAVES; ++v) {
                s1 += lds[turn][v].x;
                s2 += lds[turn][v].y;
            }
            turn ^= 1;
        }
        s1 /= (float)a.cols;
        s2 /= (float)a.cols;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const F<N> n = (widen<T, N>(r.x[k]) - r.mean) * r.rstd, g = widen<T, N>(r.dy[k]) * widen<W, N>(wv[k]);
            F<N> d = r.rstd * (g - s1 - n * s2);
            if (a.grad_residual) d += widen<T, N>(r.past[k]);
            r.x[k] = round_to<T, N>(d);
        }
        q.drop(static_cast<T *>(a.dx) + row * a.cols, r.x);
    };
    // every wavefront of a team makes the same turns; narrow teams meet at no barrier here
    Row r0, r1, r2;
    int64_t row = (int64_t)blockIdx.x * Q::TEAMS + q.team;
    fetch(r0, row);
    if constexpr (kRows > 1) fetch(r1, row + step);
    if constexpr (kRows > 2) fetch(r2, row + 2 * step);
    q.load(static_cast<const W *>(a.weight), wv);
    while (row < a.rows) {
        work(r0, row);
        fetch(r0, row + kRows * step);
        row += step;
        if constexpr (kRows > 1) {
            if (row >= a.rows) break;
            work(r1, row);
            fetch(r1, row + kRows * step);
            row += step;
        }
        if constexpr (kRows > 2) {
            if (row >= a.rows) break;
            work(r2, row);
            fetch(r2, row + kRows * step);
            row += step;
        }
    }
    float *p = a.part + (int64_t)blockIdx.x * 2 * a.cols;
    if constexpr (Q::TEAMS > 1) {      // the workgroup's teams, in order
        __shared__ F<N> sums[Q::TEAMS - 1][2 * K][THREADS];
        if (q.team) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                sums[q.team - 1][k][q.lane] = dw[k];
                sums[q.team - 1][K + k][q.lane] = db[k];
            }
        }
        __syncthreads();
        if (q.team) return;
#pragma unroll
        for (int t = 0; t < Q::TEAMS - 1; ++t)
#pragma unroll
            for (int k = 0; k < K; ++k) {
                dw[k] += sums[t][k][q.lane];
                db[k] += sums[t][K + k][q.lane];
            }
    }
    q.store(p, dw);
    q.store(p + a.cols, db);
}

// Rows too wide for that: dx, one workgroup a row, read twice.
template <class T, class W>
__global__ __launch_bounds__(kWideBlock) void k_norm_dx_wide(NormGradArgs a) {
    constexpr int N = kN<T>, STEP = kWideBlock * N;
    __shared__ float lds[kWideWaves];
    const int from = threadIdx.x * N;
    const W *w = static_cast<const W *>(a.weight);
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *dy = static_cast<const T *>(a.dy) + row * a.dy_stride;
        const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float s1 = 0.0f, s2 = 0.0f;
        for (int c = from; c < a.cols; c += STEP) {
            const F<N> n = (widen<T, N>(load<N>(x, c, a.cols)) - mean) * rstd;
            const F<N> g = widen<T, N>(load<N>(dy, c, a.cols)) * widen<W, N>(load<N>(w, c, a.cols));
            for (int j = 0; j < N; ++j) {
                s1 += g[j];
                s2 += c + j < a.cols ? g[j] * n[j] : 0.0f;
            }
        }
        s1 = block_sum<kWideWaves>(s1, lds) / (float)a.cols;
        s2 = block_sum<kWideWaves>(s2, lds) / (float)a.cols;
        T *dx = static_cast<T *>(a.dx) + row * a.cols;
        for (int c = from; c < a.cols; c += STEP) {
            const F<N> n = (widen<T, N>(load<N>(x, c, a.cols)) - mean) * rstd;
            const F<N> g = widen<T, N>(load<N>(dy, c, a.cols)) * widen<W, N>(load<N>(w, c, a.cols));
            F<N> d = rstd * (g - s1 - n * s2);
            if (a.grad_residual)
                d += widen<T, N>(load<N>(static_cast<const T *>(a.grad_residual) + row * a.grad_residual_stride, c, a.cols));
            store<N>(dx, c, a.cols, round_to<T, N>(d));
        }
    }
}

// ... and the weights' gradients over part blockIdx.y of the rows (a contiguous run), a tile of columns a
// wavefront.
template <class T>
__global__ __launch_bounds__(64) void k_norm_dw_wide(NormGradArgs a) {
    constexpr int N = kN<T>;
    const int c = (blockIdx.x * kWave + threadIdx.x) * N;
    if (c >= a.cols) return;
    const int64_t lo = a.rows * blockIdx.y / a.parts, hi = a.rows * (blockIdx.y + 1) / a.parts;
    F<N> dw = 0.0f, db = 0.0f;
    for (int64_t row = lo; row < hi; ++row) {
        const F<N> n = (widen<T, N>(load<N>(static_cast<const T *>(a.x) + row * a.x_stride, c, a.cols)) - a.mean[row]) * a.rstd[row];
        const F<N> dy = widen<T, N>(load<N>(static_cast<const T *>(a.dy) + row * a.dy_stride, c, a.cols));
        dw += dy * n;
        db += dy;
    }
    float *p = a.part + (int64_t)blockIdx.y * 2 * a.cols;
    store<N>(p, c, a.cols, dw);
    store<N>(p + a.cols, c, a.cols, db);
}

// Sums the parts: 64 columns a workgroup, its wavefronts take turns at the parts and are added in order.
constexpr int kJoinWaves = 16;
template <class G>
__global__ __launch_bounds__(kJoinWaves * kWave) void k_norm_join(NormGradArgs a) {
    __shared__ float lds[kJoinWaves][kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, c = blockIdx.x * kWave + lane;
    G *out = static_cast<G *>(blockIdx.y ? a.dbias : a.dweight);
    if (!out) return;
    float s = 0.0f;
    if (c < a.cols) {
        const float *p = a.part + (int64_t)blockIdx.y * a.cols + c;
#pragma unroll 16
        for (int k = wave; k < a.parts; k += kJoinWaves) s += p[(int64_t)k * 2 * a.cols];
    }
    lds[wave][lane] = s;
    __syncthreads();
    if (wave || c >= a.cols) return;
#pragma unroll
    for (int v = 1; v < kJoinWaves; ++v) s += lds[v][lane];
    if (a.accumulate) s += (float)out[c];
    out[c] = (G)s;
}

// Widest row whose gradient's team holds it in registers.
constexpr int64_t kGradCols = 512 * 32;
constexpr int grad_threads(int64_t cols) {
    return cols <= 64 * 16 ? 64 : cols <= 256 * 16 ? 256 : 512;
}

template <class T, class W, class G>
hipError_t norm_grad(const NormGradArgs &a, hipStream_t s) {
    hipError_t e = hipSuccess;
    const auto run = [&](auto kernel) {
        const int threads = grad_threads(a.cols);
        return launch(kernel, dim3((unsigned)a.parts), dim3(threads < 256 ? 256 : threads), s, a);
    };
    if (!a.rows) {
    } else if (a.cols > kGradCols) {
        const unsigned tiles = (unsigned)((a.cols + kWave * kN<T> - 1) / (kWave * kN<T>));
        if ((e = launch(k_norm_dw_wide<T>, dim3(tiles, (unsigned)a.parts), dim3(64), s, a))) return e;
        // dx comes second: it may lie where dy is
        e = launch(k_norm_dx_wide<T, W>, dim3(grid_of(a.rows)), dim3(kWideBlock), s, a);
    } else if (a.cols <= 64 * 8) {
        e = run(k_norm_grad<T, W, 64, 8>);
    } else if (a.cols <= 64 * 16) {
        e = run(k_norm_grad<T, W, 64, 16>);
    } else if (a.cols <= 256 * 8) {
        e = run(k_norm_grad<T, W, 256, 8>);
    } else if (a.cols <= 256 * 16) {
        e = run(k_norm_grad<T, W, 256, 16>);
    } else if (a.cols <= 512 * 16) {
        e = run(k_norm_grad<T, W, 512, 16>);
    } else if (a.cols <= 512 * 24) {
        e = run(k_norm_grad<T, W, 512, 24>);
    } else {
        e = run(k_norm_grad<T, W, 512, 32>);
    }
    if (e) return e;
    return launch(k_norm_join<G>, dim3((unsigned)((a.cols + kWave - 1) / kWave), 2), dim3(kJoinWaves * kWave), s, a);
}

// ---------------------------------------------------------------- embedding

template <class I>
__device__ __forceinline__ int64_t id_at(const void *ids, int64_t t) {
    return (int64_t)static_cast<const I *>(ids)[t];
}
// Row of the shard that an id names, or -1.  Subtracted without sign: any id is allowed.
__device__ __forceinline__ int shard_row(int64_t id, int64_t start, int vocab) {
    const uint64_t v = (uint64_t)id - (uint64_t)start;
    return v < (uint64_t)vocab ? (int)v : -1;
}

// A wavefront copies K pieces of every lane of one token's row, all on their way at once.
template <class T, class I, int K>
__global__ __launch_bounds__(256) void k_embed(EmbedArgs a) {
    constexpr int N = kN<T>, SPAN = K * kWave * N;
    const int lane = threadIdx.x % kWave, spans = (a.cols + SPAN - 1) / SPAN;
    const int64_t n = a.rows * spans;
    for (int64_t id = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave; id < n; id += (int64_t)gridDim.x * 4) {
        const int64_t t = id / spans;
        const int v = shard_row(id_at<I>(a.ids, t), a.vocab_start, a.vocab), from = (int)(id - t * spans) * SPAN + lane * N;
        T *out = static_cast<T *>(a.out) + t * a.cols;
        const T *w = static_cast<const T *>(a.weight) + (int64_t)(v < 0 ? 0 : v) * a.weight_stride;
        V<T, N> r[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = from + k * kWave * N;
            r[k] = T(0);
            if (v >= 0 && c < a.cols) r[k] = load<N>(w, c, a.cols);
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = from + k * kWave * N;
            if (c >= a.cols) continue;
            if (v >= 0) r[k] = round_to<T, N>(widen<T, N>(r[k]) * a.scale);
            drop<N>(out, c, a.cols, r[k]);
        }
    }
}

// A wavefront writes zeros to a row.
template <class T>
__device__ __forceinline__ void zero_row(T *row, int cols) {
    for (int c = threadIdx.x % kWave * kN<T>; c < cols; c += kWave * kN<T>) store<kN<T>>(row, c, cols, V<T, kN<T>>(T(0)));
}

// Tokens are sorted by their row's slot: 2^bits sorting workgroups take 64 slots each, and a row's
// workgroup is its low bits, so that the frequent ids, which vocabularies number first, do not meet in one.
__host__ __device__ __forceinline__ int slot_of(int row, int bits) { return ((row & ((1 << bits) - 1)) << 6) + (row >> bits); }
int sort_bits(int64_t vocab) {
    int b = 0;
    while ((int64_t(kWave) << b) < vocab) ++b;
    return b;
}

// Workspace of the gradient: where each slot's tokens begin, the tokens sorted by slot, the row of
// each sorted place, and two rows of 32-bit sums for every chunk of sorted places, for the runs of tokens of one
// row that are longer than a chunk: of the run that reaches in from the chunk before, and of the one that goes
// on into the next.  runs[0].x counts those runs, runs[1 ..] are they: row, first and last chunk, in any
// order.
struct EmbedSpace {
    int *begin, *token, *row;
    int4 *runs;
    float *part;
};
int64_t round16(int64_t n) { return (n + 15) & ~int64_t(15); }
EmbedSpace embed_space(void *p, int64_t rows, int64_t vocab, int64_t chunks) {
    char *c = static_cast<char *>(p);
    EmbedSpace w;
    w.begin = reinterpret_cast<int *>(c);
    w.token = reinterpret_cast<int *>(c += round16(((int64_t(kWave) << sort_bits(vocab)) + 1) * 4));
    w.row = reinterpret_cast<int *>(c += round16(rows * 4));
    w.runs = reinterpret_cast<int4 *>(c += round16(rows * 4));
    w.part = reinterpret_cast<float *>(c + (chunks + 1) * 16);
    return w;
}
// Columns that a wavefront takes at a time.
template <class T>
constexpr int kTile = kWave * kN<T>;
int64_t tiles_of(int64_t cols, int tile) { return (cols + tile - 1) / tile; }

// Sorted places of a chunk: few enough to give the chip wavefronts, and no fewer.  A wavefront looks at two
// chunks, one place a lane.
int embed_chunk(int64_t rows, int64_t cols) {
    int c = 4;
    while (c < kWave / 2 && (rows + c - 1) / c * tiles_of(cols, kTile<bf16>) > 16384) c *= 2;
    return c;
}

// Tokens sorted by slot, ascending within one.  A workgroup owns 64 slots and reads every
// id, each wavefront its share of the tokens: they count their rows' tokens (in LDS) and those of the slots
// before them, which says where each row and each wavefront's part of it begins, and then
// place the tokens in order.  A lane's place among those of its 64 tokens with the same row follows from six
// ballots, one for each bit of the row's number in the workgroup.  No scan over workgroups and no atomics whose
// order matters: one launch sorts.  A lane reads LOADS ids at a time, and a share of as many only once.
constexpr int kSortWaves = 16;
template <class I, int LOADS>
__global__ __launch_bounds__(kSortWaves * kWave) void k_embed_sort(EmbedGradArgs a, EmbedSpace ws, int bits) {
    __shared__ int counts[kSortWaves][kWave], befores[kSortWaves];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, waves = blockDim.x / kWave;
    const int block = blockIdx.x, mask = (1 << bits) - 1;
    const uint64_t below = (uint64_t(1) << lane) - 1;
    const int64_t share = (a.rows + waves * kWave - 1) / (waves * kWave) * kWave;
    const int64_t lo = share * wave, hi = lo + share < a.rows ? lo + share : a.rows;
    const bool once = share <= LOADS * kWave;
    // A token's row with the workgroup's number taken out of its low bits and those bits turned to the
    // top: its slot here if that is below 64.  No row (~0) is of the last group and of no slot.
    int before = 0;
    unsigned v[LOADS];
    const auto slots_at = [&](int64_t t, bool count) {
        I id[LOADS];
        const bool all = t + LOADS * kWave <= hi;
#pragma unroll
        for (int k = 0; k < LOADS; ++k) {
            const int64_t u = t + k * kWave + lane;
            id[k] = static_cast<const I *>(a.ids)[all || u < hi ? u : hi - 1];
        }
#pragma unroll
        for (int k = 0; k < LOADS; ++k) {
            unsigned row = (unsigned)shard_row((int64_t)id[k], a.vocab_start, a.vocab);
            if (!all && t + k * kWave + lane >= hi) row = ~0u;
            const unsigned x = row ^ (unsigned)block;
            v[k] = __builtin_amdgcn_alignbit(x, x, bits);
            if (!count) continue;
            before += __popcll(__ballot((int)(row & mask) < block));
            if (v[k] < kWave) atomicAdd(&counts[wave][v[k]], 1);
        }
    };
    counts[wave][lane] = 0;
    for (int64_t t = lo; t < hi; t += LOADS * kWave) slots_at(t, true);
    if (lane == 0) befores[wave] = before;
    __syncthreads();
    int total = 0, at = 0;      // at: tokens of row `lane` in the wavefronts before this one
    before = 0;
    for (int w = 0; w < waves; ++w) {
        if (w == wave) at = total;
        total += counts[w][lane];
        before += befores[w];
    }
    int start = total;          // inclusive prefix sum over the lanes, made exclusive
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const int up = __shfl_up(start, d);
        if (lane >= d) start += up;
    }
    start += before - total;
    if (wave == 0) {
        ws.begin[block * kWave + lane] = start;
        if (block == 0 && lane == 0) ws.runs[0].x = 0;
        if (block == mask && lane == kWave - 1) ws.begin[block * kWave + kWave] = start + total;
    }
    __syncthreads();            // every wavefront has read the counts: they become the next free places
    volatile int *next = counts[wave];
    next[lane] = start + at;
    for (int64_t t = lo; t < hi; t += LOADS * kWave) {
        if (!once) slots_at(t, false);
#pragma unroll
        for (int k = 0; k < LOADS; ++k) {
            const bool mine = v[k] < kWave;
            uint64_t same = __ballot(mine);
            if (!same) continue;
            if (same & (same - 1)) {      // more than one: who else has this lane's slot
#pragma unroll
                for (int b = 0; b < 6; ++b) {
                    const bool bit = v[k] >> b & 1;
                    const uint64_t set = __ballot(bit);
                    same &= bit ? set : ~set;
                }
            }
            if (!mine) continue;
            const int place = next[v[k]] + __popcll(same & below);
            ws.token[place] = (int)(t + k * kWave + lane);
            ws.row[place] = block + (int)(v[k] << bits);
            if (!(same & below)) next[v[k]] = place + __popcll(same);
        }
    }
}

template <class G>
__device__ __forceinline__ G *row_of(const EmbedGradArgs &a, int row) {
    return static_cast<G *>(a.dweight) + (int64_t)row * a.cols;
}

// A wavefront sums the runs that begin in one chunk of sorted places over one tile of columns.  Runs
// of up to a chunk are finished, past the chunk's end where they go on; of a longer run every chunk's
// wavefront leaves the sum of its places in ws.part.  Work is split by tokens, so an id that many tokens
// share costs no more than many ids.  The wavefronts after those write zeros to the rows that no token names
// (accumulate: there are none).
template <class T, class G>
__global__ __launch_bounds__(256) void k_embed_sum(EmbedGradArgs a, EmbedSpace ws, int bits, int chunk, int64_t sums) {
    constexpr int N = kN<T>, kAhead = 4;
    const int lane = threadIdx.x % kWave;
    const int64_t id = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave, tiles = (a.cols + kTile<T> - 1) / kTile<T>;
    if (id >= sums) {
        for (int64_t v = id - sums; v < a.vocab; v += (int64_t)gridDim.x * 4 - sums) {
            const int slot = slot_of((int)v, bits);
            if (a.rows && ws.begin[slot] != ws.begin[slot + 1]) continue;
            zero_row(row_of<G>(a, (int)v), a.cols);
        }
        return;
    }
    const int64_t j = id / tiles, base = j * chunk;
    const int c = (int)(id % tiles) * kTile<T> + lane * N;
    const int64_t n = ws.begin[kWave << bits];
    if (base >= n) return;
    const int m = (int)(n - base < chunk ? n - base : chunk);      // places of this chunk
    const int64_t at = base + lane;
    const bool seen = lane < 2 * chunk && at < n;                  // places of this one and the next
    const int row = seen ? ws.row[at] : -1, token = seen ? ws.token[at] : 0;
    const int past = j > 0 && lane < chunk ? ws.row[at - chunk] : -1;
    const int first = __builtin_amdgcn_readlane(row, 0), last = __builtin_amdgcn_readlane(row, m - 1);
    // the run that reaches in: places before the chunk, and in it (as far as is seen)
    const int before = __popcll(__ballot(past == first)), head = __popcll(__ballot(row == first));
    const bool in = before > 0, in_long = in && before + head > chunk;
    // the run at the chunk's end, if it begins here
    const uint64_t same = __ballot(row == last);
    const int tail = __ffsll((unsigned long long)same) - 1, length = __popcll(same);
    const bool out_long = !(in && tail == 0) && length > chunk;
    const int begin = in && !in_long ? head : 0;
    const int end = out_long || (in && tail == 0) ? m : tail + length;
    const int after = __shfl_down(row, 1);
    const uint64_t ends = __ballot(lane < end && (lane == end - 1 || after != row));
    bool inner = !in_long;
    F<N> s = 0.0f;
    for (int i = begin; i < end; i += kAhead) {
        V<T, N> r[kAhead];
        V<G, N> old[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (i + k >= end || c >= a.cols) continue;
            r[k] = stream<N>(static_cast<const T *>(a.dy) + (int64_t)__builtin_amdgcn_readlane(token, i + k) * a.dy_stride,
                           c, a.cols);
            if (a.accumulate && ends >> (i + k) & 1)
                old[k] = load<N>(row_of<G>(a, __builtin_amdgcn_readlane(row, i + k)), c, a.cols);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (i + k >= end || c >= a.cols) continue;
            s += widen<T, N>(r[k]);
            if (!(ends >> (i + k) & 1)) continue;
            if (!inner || (out_long && i + k >= tail)) {
                store<N>(ws.part + (j * 2 + inner) * a.cols, c, a.cols, s);
            } else {
                s *= a.scale;
                if (a.accumulate) s += widen<G, N>(old[k]);
                store<N>(row_of<G>(a, __builtin_amdgcn_readlane(row, i + k)), c, a.cols, round_to<G, N>(s));
            }
            inner = true;
            s = 0.0f;
        }
    }
    if (out_long && c == 0)
        ws.runs[1 + atomicAdd(&ws.runs[0].x, 1)] =
            make_int4(last, (int)j, (ws.begin[slot_of(last, bits) + 1] - 1) / chunk, 0);
}

// Finishes the runs longer than a chunk: the sums of a run's chunks, four wavefronts taking turns, joined in
// order.
template <class G, int N>
__global__ __launch_bounds__(256) void k_embed_join(EmbedGradArgs a, EmbedSpace ws) {
    constexpr int TILE = kWave * N;
    __shared__ F<N> lds[3][kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int64_t tiles = (a.cols + TILE - 1) / TILE, n = ws.runs[0].x * tiles;
    for (int64_t id = blockIdx.x; id < n; id += gridDim.x) {
        const int4 run = ws.runs[1 + id / tiles];
        const int64_t j = run.y;
        const int c = (int)(id % tiles) * TILE + lane * N;
        G *out = row_of<G>(a, run.x);
        F<N> s = 0.0f;
        V<G, N> old = G(0);
        if (c < a.cols) {
            if (wave == 0) {
                s = load<N>(ws.part + (j * 2 + 1) * a.cols, c, a.cols);
                if (a.accumulate) old = load<N>(out, c, a.cols);
            }
#pragma unroll 8
            for (int64_t k = j + 1 + wave; k <= run.z; k += 4) s += load<N>(ws.part + k * 2 * a.cols, c, a.cols);
        }
        if (wave) lds[wave - 1][lane] = s;
        __syncthreads();
        if (!wave && c < a.cols) {
            for (int w = 0; w < 3; ++w) s += lds[w][lane];
            s *= a.scale;
            if (a.accumulate) s += widen<G, N>(old);
            store<N>(out, c, a.cols, round_to<G, N>(s));
        }
        __syncthreads();
    }
}

template <class I>
hipError_t embed_sort(const EmbedGradArgs &a, const EmbedSpace &ws, int bits, hipStream_t s) {
    const int64_t rounds = (a.rows + kWave - 1) / kWave;
    const int waves = rounds < kSortWaves ? (int)rounds : kSortWaves;
    const dim3 grid(1u << bits), block(waves * kWave);
    return launch(rounds <= kSortWaves       ? k_embed_sort<I, 1>
                  : rounds <= 4 * kSortWaves ? k_embed_sort<I, 4>
                                             : k_embed_sort<I, 16>,
                  grid, block, s, a, ws, bits);
}

template <class T, class G>
hipError_t embed_grad(const EmbedGradArgs &a, int index_type, hipStream_t s) {
    const int bits = sort_bits(a.vocab), chunk = embed_chunk(a.rows, a.cols);
    const int64_t chunks = (a.rows + chunk - 1) / chunk, tiles = tiles_of(a.cols, kTile<T>);
    const int64_t sums = (chunks * tiles + 3) / 4 * 4;
    const EmbedSpace ws = embed_space(a.workspace, a.rows, a.vocab, chunks);
    hipError_t e = hipSuccess;
    if (a.rows) {
        e = index_type == ECHO_I64 ? embed_sort<int64_t>(a, ws, bits, s) : embed_sort<int32_t>(a, ws, bits, s);
        if (e) return e;
    }
    const int64_t fills = a.accumulate ? 0 : grid_of((a.vocab + 3) / 4);
    if ((e = launch(k_embed_sum<T, G>, dim3((unsigned)(sums / 4 + fills)), dim3(256), s, a, ws, bits, chunk, sums))) return e;
    // as many workgroups as the chip holds: how many runs there are to join is not known here
    const int64_t joins = (chunks - 1) * tiles;
    if (joins > 0) e = launch(k_embed_join<G, kN<T>>, dim3((unsigned)(joins < 2048 ? joins : 2048)), dim3(256), s, a, ws);
    return e;
}

// ---------------------------------------------------------------- cross entropy

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

// (exp(l - lse) - [column = target]) * g for the columns col .. col + N - 1.
template <int N>
__device__ __forceinline__ F<N> loss_grad(F<N> l, float lse, int col, int at, float g) {
    F<N> d;
#pragma unroll
    for (int j = 0; j < N; ++j) d[j] = (exp_of(l[j] - lse) - (col + j == at ? 1.0f : 0.0f)) * g;
    return d;
}
// Log of the sum of exponentials from a maximum and a sum relative to it, written with the row's loss.
__device__ __forceinline__ float finish_row(const LossArgs &a, int64_t row, const LossRow &r, float hit, float top, float sum,
                                            bool writes) {
    const float lse = top == -kInf ? -kInf : top + logf(sum);
    if (writes) {
        if (a.lse) a.lse[row] = lse;
        if (a.target) a.target[row] = hit;
        if (a.loss) a.loss[row] = !r.trained ? 0.0f : lse == -kInf ? kInf : lse - hit;
    }
    return lse;
}

// A team a row, which is read once and stays in registers as it came; with a gradient it is written
// from there.  Each wavefront takes its maximum and its sum of exponentials relative to it; the team joins
// them with one exchange.
template <class T, class I, int THREADS, int E>
__global__ __launch_bounds__((Team<T, THREADS, E>::BLOCK)) void k_loss(LossArgs a) {
    using Q = Team<T, THREADS, E>;
    constexpr int N = Q::N, K = Q::K;
    const Q q(a.cols);
    __shared__ float2 lds[2][Q::WAVES];
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * Q::TEAMS + q.team; row < a.rows; row += (int64_t)gridDim.x * Q::TEAMS) {
        const T *l = static_cast<const T *>(a.logits) + row * a.logits_stride;
        V<T, N> x[K];
        q.load(l, x, T(-kInf));
        const LossRow r = loss_row<I>(a, row);
        const float hit = r.at >= 0 ? (float)l[r.at] : 0.0f, g = a.grad ? a.grad_loss[row] : 0.0f;
        float top = -kInf, sum = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const F<N> f = widen<T, N>(x[k]);
#pragma unroll
            for (int j = 0; j < N; ++j) top = fmaxf(top, f[j]);
            forget<T, N>(x[k]);
        }
        top = wave_max(top);
        const float base = top == -kInf ? 0.0f : top;      // nothing here: the sum is 0
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (k * THREADS * N >= a.cols) continue;
            const F<N> f = widen<T, N>(x[k]);
#pragma unroll
            for (int j = 0; j < N; ++j) sum += exp_of(f[j] - base);
            forget<T, N>(x[k]);
        }
        sum = wave_sum(sum);
        if constexpr (Q::WAVES > 1) {
            if (q.lane % kWave == 0) lds[turn][q.wave] = make_float2(top, sum);
            __syncthreads();      // also: every lane has read the target's logit, and grad may be logits
#pragma unroll
            for (int v = 0; v < Q::WAVES; ++v) top = fmaxf(top, lds[turn][v].x);
            sum = 0.0f;
#pragma unroll
            for (int v = 0; v < Q::WAVES; ++v) {
                const float2 p = lds[turn][v];
                sum += p.x == -kInf ? p.y : p.y * exp_of(p.x - top);      // p.y is 0, or NaN
            }
            turn ^= 1;
        }
        // a row of NaN alone has no maximum but a sum
        const float lse = finish_row(a, row, r, hit, sum != sum ? sum : top, sum, q.lane == 0);
        if (!a.grad) continue;
        const bool live = r.trained && lse != -kInf;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            F<N> f = 0.0f;
            if (live) f = loss_grad<N>(widen<T, N>(x[k]), lse, q.col(k), r.at, g);
            x[k] = round_to<T, N>(f);
        }
        q.drop(static_cast<T *>(a.grad) + row * a.grad_stride, x);
    }
}

// Rows too wide for registers: one workgroup a row, read once for a running maximum and sum a lane, and
// with a gradient once more.
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
        const float lse = finish_row(a, row, r, hit, sum != sum ? sum : top, sum, threadIdx.x == 0);
        if (!a.grad) continue;
        T *d = static_cast<T *>(a.grad) + row * a.grad_stride;
        const bool live = r.trained && lse != -kInf;
        const float g = a.grad_loss[row];
        for (int c = threadIdx.x * N; c < a.cols; c += STEP) {
            F<N> f = 0.0f;
            if (live) f = loss_grad<N>(widen<T, N>(load<N>(l, c, a.cols)), lse, c, r.at, g);
            store<N>(d, c, a.cols, round_to<T, N>(f));
        }
    }
}

// The gradient alone, K pieces a lane of one row's stretch of 256 * K pieces.
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
            if (live) f = loss_grad<N>(widen<T, N>(raw[k]), lse, c, r.at, g);
            drop<N>(d, c, a.cols, round_to<T, N>(f));
        }
    }
}

template <class T, class I>
hipError_t loss(const LossArgs &a, hipStream_t s) {
    const auto run = [&](auto kernel, int threads) {
        const int teams = threads < 256 ? 256 / threads : 1;
        return launch(kernel, dim3(grid_of((a.rows + teams - 1) / teams)), dim3(threads * teams), s, a);
    };
    if (a.cols <= 64 * 8) return run(k_loss<T, I, 64, 8>, 64);
    if (a.cols <= 64 * 32) return run(k_loss<T, I, 64, 32>, 64);
    if (a.cols <= 256 * 32) return run(k_loss<T, I, 256, 32>, 256);
    if (a.cols <= 512 * 32) return run(k_loss<T, I, 512, 32>, 512);
    if (a.cols <= 1024 * 32) return run(k_loss<T, I, 1024, 32>, 1024);
    if (a.cols <= 1024 * 64) return run(k_loss<T, I, 1024, 64>, 1024);
    return launch(k_loss_wide<T, I>, dim3(grid_of(a.rows)), dim3(kWideBlock), s, a);
}
template <class T, class I>
hipError_t loss_grad_alone(const LossArgs &a, hipStream_t s) {
    constexpr int SPAN = kGradPieces * 256 * kN<T>;
    return launch(k_loss_grad<T, I>, dim3(grid_of(a.rows * ((a.cols + SPAN - 1) / SPAN))), dim3(256), s, a);
}

}  // namespace

// A part is a workgroup of the gradient's kernel.  More of them fill the chip, but every one leaves 8 bytes a
// column to write and read again: at most one wave of workgroups over the 256 compute units (two of narrow teams).
int norm_grad_parts(int64_t rows, int64_t cols) {
    const int threads = grad_threads(cols), teams = cols > kGradCols || threads >= 256 ? 1 : 256 / threads;
    const int64_t n = (rows + teams - 1) / teams, most = cols > kGradCols ? 64 : threads <= 256 ? 512 : 256;
    return (int)(n < most ? n : most);
}
int64_t embed_grad_bytes(int64_t rows, int64_t cols, int64_t vocab) {
    if (!rows) return 0;
    const int chunk = embed_chunk(rows, cols);
    return round16(((int64_t(kWave) << sort_bits(vocab)) + 1) * 4) + 2 * round16(rows * 4) +
           ((rows + chunk - 1) / chunk + 1) * 16 + (rows + chunk - 1) / chunk * 2 * cols * 4;
}

hipError_t launch_norm(const NormArgs &a, int type, int weight_type, hipStream_t s) {
    const bool same = type == weight_type;
    switch (type) {
        case ECHO_F32: return norm<float, float>(a, s);
        case ECHO_F16: return same ? norm<f16, f16>(a, s) : norm<f16, float>(a, s);
        default: return same ? norm<bf16, bf16>(a, s) : norm<bf16, float>(a, s);
    }
}

template <class T>
static hipError_t norm_grad_of(const NormGradArgs &a, bool wide_weight, bool wide_grad, hipStream_t s) {
    if (wide_weight) return norm_grad<T, float, float>(a, s);
    return wide_grad ? norm_grad<T, T, float>(a, s) : norm_grad<T, T, T>(a, s);
}
hipError_t launch_norm_grad(const NormGradArgs &a, int type, int weight_type, int grad_type, hipStream_t s) {
    const bool ww = weight_type == ECHO_F32, wg = grad_type == ECHO_F32;
    switch (type) {
        case ECHO_F32: return norm_grad<float, float, float>(a, s);
        case ECHO_F16: return norm_grad_of<f16>(a, ww, wg, s);
        default: return norm_grad_of<bf16>(a, ww, wg, s);
    }
}

template <class T, class I>
static hipError_t embed(const EmbedArgs &a, hipStream_t s) {
    // as many pieces a lane as the row has, up to four
    const auto run = [&](auto kernel, int pieces) {
        const int64_t span = (int64_t)pieces * kTile<T>;
        return launch(kernel, dim3(grid_of((a.rows * ((a.cols + span - 1) / span) + 3) / 4)), dim3(256), s, a);
    };
    if (a.cols <= kTile<T>) return run(k_embed<T, I, 1>, 1);
    if (a.cols <= 2 * kTile<T>) return run(k_embed<T, I, 2>, 2);
    return run(k_embed<T, I, 4>, 4);
}
template <class I>
static hipError_t embed_of(const EmbedArgs &a, int type, hipStream_t s) {
    switch (type) {
        case ECHO_F32: return embed<float, I>(a, s);
        case ECHO_F16: return embed<f16, I>(a, s);
        default: return embed<bf16, I>(a, s);
    }
}
hipError_t launch_embed(const EmbedArgs &a, int type, int index_type, hipStream_t s) {
    return index_type == ECHO_I64 ? embed_of<int64_t>(a, type, s) : embed_of<int32_t>(a, type, s);
}

hipError_t launch_embed_grad(const EmbedGradArgs &a, int type, int index_type, int grad_type, hipStream_t s) {
    const bool wide = grad_type == ECHO_F32;
    switch (type) {
        case ECHO_F32: return embed_grad<float, float>(a, index_type, s);
        case ECHO_F16: return wide ? embed_grad<f16, float>(a, index_type, s) : embed_grad<f16, f16>(a, index_type, s);
        default: return wide ? embed_grad<bf16, float>(a, index_type, s) : embed_grad<bf16, bf16>(a, index_type, s);
    }
}

template <class I>
static hipError_t loss_of(const LossArgs &a, int type, bool grad_alone, hipStream_t s) {
    switch (type) {
        case ECHO_F32: return grad_alone ? loss_grad_alone<float, I>(a, s) : loss<float, I>(a, s);
        case ECHO_F16: return grad_alone ? loss_grad_alone<f16, I>(a, s) : loss<f16, I>(a, s);
        default: return grad_alone ? loss_grad_alone<bf16, I>(a, s) : loss<bf16, I>(a, s);
    }
}
hipError_t launch_loss(const LossArgs &a, int type, int index_type, hipStream_t s) {
    return index_type == ECHO_I64 ? loss_of<int64_t>(a, type, false, s) : loss_of<int32_t>(a, type, false, s);
}
hipError_t launch_loss_grad(const LossArgs &a, int type, int index_type, hipStream_t s) {
    return index_type == ECHO_I64 ? loss_of<int64_t>(a, type, true, s) : loss_of<int32_t>(a, type, true, s);
}

}  // namespace echo
