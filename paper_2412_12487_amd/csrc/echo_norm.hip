// echo_norm.hip -- layer norm and its gradient on gfx950.
#include "echo_ops_device.h"

namespace echo {
namespace {

// A team a row, which is read once.  The mean and the sum of squares about it are taken per wavefront, both
// from the registers, and joined over the team's wavefronts (n, mean, squares) in their order, so the team
// waits for itself once a row.  Memory bounds it: 2048 x 8192 of bf16 with a residual in 22.0 us a pass, 6.1 TB/s; one row
// takes 2.3 us.
template <class T, class W, int THREADS, int E, bool CUT>
__global__ __launch_bounds__((Team<T, THREADS, E, CUT>::BLOCK)) void k_norm(NormArgs a) {
    using Q = Team<T, THREADS, E, CUT>;
    constexpr int N = Q::N, K = Q::K, P = Q::P;
    constexpr bool kEarly = E <= 16;      // the weights wait in registers while the team joins its sums
    const Q q(a.cols);
    __shared__ float2 lds[2][Q::WAVES];
    const W *w = static_cast<const W *>(a.weight), *b = static_cast<const W *>(a.bias);
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * Q::TEAMS + q.team; row < a.rows; row += (int64_t)gridDim.x * Q::TEAMS) {
        V<T, N> x[P];
        V<W, N> wv[P], bv[P];
        q.load(static_cast<const T *>(a.x) + row * a.x_stride, x);
        if (a.residual) {
            V<T, N> r[P];
            q.load(static_cast<const T *>(a.residual) + row * a.residual_stride, r);
#pragma unroll
            for (int k = 0; k < P; ++k) x[k] = round_to<T, N>(widen<T, N>(x[k]) + widen<T, N>(r[k]));
            q.drop(static_cast<T *>(a.sum) + row * a.cols, x);
        }
        if constexpr (kEarly) {
            q.load(w, wv);
            if (b) q.load(b, bv);
        }
        float s = 0.0f;
#pragma unroll
        for (int k = 0; k < P; ++k) {
            const F<N> f = widen<T, N>(x[k]);
#pragma unroll
            for (int j = 0; j < N; ++j) s += f[j];
        }
        forget<T, N, P>(x);
        const int n = q.count(q.wave);
        float mean = n ? wave_sum(s) / (float)n : 0.0f, squares = 0.0f;
#pragma unroll
        for (int k = 0; k < P; ++k) {
            const F<N> d = widen<T, N>(x[k]) - mean;
            if (q.has(k)) {
#pragma unroll
                for (int j = 0; j < N; ++j) squares += k < K || j < q.left ? d[j] * d[j] : 0.0f;
            }
        }
        forget<T, N, P>(x);
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
        for (int k = 0; k < P; ++k) {
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

// Rows too wide for registers (or of less than a piece): one workgroup a row, which is read three times (sum, squares about the
// mean, result), from the cache after the first.  2048 x 20480 of bf16 in 34.3 us, 4.9 TB/s.
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

template <class T, class W, bool CUT>
hipError_t norm(const NormArgs &a, hipStream_t s) {
    // The narrowest team that holds the row: few lanes idle, few wavefronts wait for each other.
    const auto run = [&](auto kernel, int threads) {
        const int teams = threads < 256 ? 256 / threads : 1;
        return launch(kernel, dim3(grid_of((a.rows + teams - 1) / teams)), dim3(threads * teams), s, a);
    };
    if (a.cols < kN<T> || a.cols > 512 * 32)
        return launch(k_norm_wide<T, W>, dim3(grid_of(a.rows)), dim3(kWideBlock), s, a);
    if (a.cols <= 64 * 8) return run(k_norm<T, W, 64, 8, CUT>, 64);
    if (a.cols <= 64 * 16) return run(k_norm<T, W, 64, 16, CUT>, 64);
    if (a.cols <= 256 * 8) return run(k_norm<T, W, 256, 8, CUT>, 256);
    if (a.cols <= 256 * 16) return run(k_norm<T, W, 256, 16, CUT>, 256);
    if (a.cols <= 256 * 24) return run(k_norm<T, W, 256, 24, CUT>, 256);
    if (a.cols <= 512 * 16) return run(k_norm<T, W, 512, 16, CUT>, 512);
    if (a.cols <= 512 * 24) return run(k_norm<T, W, 512, 24, CUT>, 512);
    return run(k_norm<T, W, 512, 32, CUT>, 512);
}

// Gradients, x and dy read once.  A team takes every (teams of the launch)-th row and keeps its lanes' columns
// of dweight and dbias in registers, which leaves the chip few wavefronts; so the next row is on its way
// while one is worked on, where its lanes hold only 8 elements of a row (with 16 the registers of the second
// row cost more wavefronts than it hides).  A workgroup leaves one row of each weight sum in `part`.
// 2048 x 12288 of bf16 with a residual's gradient: 39.1 us, 5.1 TB/s, and 5.3 us for the join.  Narrower rows are
// further from memory's rate (2048 x 4096: 16.0 us, 3.1 TB/s, and 3.9): few wavefronts a SIMD, each waiting for its row.
template <class T, class W, int THREADS, int E, bool CUT>
__global__ __launch_bounds__((Team<T, THREADS, E, CUT>::BLOCK)) void k_norm_grad(NormGradArgs a) {
    using Q = Team<T, THREADS, E, CUT>;
    constexpr int N = Q::N, K = Q::K, P = Q::P;
    constexpr int kRows = E <= 8 ? 2 : 1;      // in registers
    struct Row {
        V<T, N> x[P], dy[P], past[P];
        float mean, rstd;
    };
    const Q q(a.cols);
    __shared__ float2 lds[2][Q::WAVES];
    const int64_t step = (int64_t)gridDim.x * Q::TEAMS;
    V<W, N> wv[P];
    F<N> dw[P], db[P];
    int turn = 0;
#pragma unroll
    for (int k = 0; k < P; ++k) dw[k] = db[k] = 0.0f;
    const auto fetch = [&](Row &r, int64_t row) {
        if (row >= a.rows) return;
        q.fetch(static_cast<const T *>(a.x) + row * a.x_stride, r.x);
        q.fetch(static_cast<const T *>(a.dy) + row * a.dy_stride, r.dy);
        if (a.grad_residual) q.fetch(static_cast<const T *>(a.grad_residual) + row * a.grad_residual_stride, r.past);
        r.mean = a.mean[row];
        r.rstd = a.rstd[row];
    };
    const auto work = [&](Row &r, int64_t row) {
        float s1 = 0.0f, s2 = 0.0f;
        q.settle(r.x, T(0));
        q.settle(r.dy, T(0));
        if (a.grad_residual) q.settle(r.past, T(0));
#pragma unroll
        for (int k = 0; k < P; ++k) {
            // past the row's end dy and weight are 0, and so is g.  n is made 0 there too: the product of a finite mean
            // and a finite rstd can pass 32 bits, and infinity times 0 would be the whole row's
            F<N> n = (widen<T, N>(r.x[k]) - (q.has(k) ? r.mean : 0.0f)) * r.rstd;
            if (k == K) {
#pragma unroll
                for (int j = 0; j < N; ++j) n[j] = j < q.left ? n[j] : 0.0f;
            }
            const F<N> d = widen<T, N>(r.dy[k]), g = d * widen<W, N>(wv[k]);
            dw[k] += d * n;
            db[k] += d;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                s1 += g[j];
                s2 += g[j] * n[j];
            }
        }
        forget<T, N, P>(r.x);
        forget<T, N, P>(r.dy);
        s1 = wave_sum(s1);
        s2 = wave_sum(s2);
        if constexpr (Q::WAVES > 1) {
            if (q.lane % kWave == 0) lds[turn][q.wave] = make_float2(s1, s2);
            __syncthreads();
            constexpr int R = Q::WAVES <= 8 ? Q::WAVES : 16;
            const int v = q.lane % R;      // a wavefront's sums in a lane
            const float2 p = v < Q::WAVES ? lds[turn][v] : make_float2(0.0f, 0.0f);
            s1 = ring_sum<R>(p.x);
            s2 = ring_sum<R>(p.y);
            turn ^= 1;
        }
        s1 /= (float)a.cols;
        s2 /= (float)a.cols;
#pragma unroll
        for (int k = 0; k < P; ++k) {
            const F<N> n = (widen<T, N>(r.x[k]) - r.mean) * r.rstd, g = widen<T, N>(r.dy[k]) * widen<W, N>(wv[k]);
            F<N> d = r.rstd * (g - s1 - n * s2);
            if (a.grad_residual) d += widen<T, N>(r.past[k]);
            r.x[k] = round_to<T, N>(d);
        }
        q.drop(static_cast<T *>(a.dx) + row * a.cols, r.x);
    };
    // every wavefront of a team makes the same turns; narrow teams meet at no barrier here
    Row r0, r1;
    int64_t row = (int64_t)blockIdx.x * Q::TEAMS + q.team;
    fetch(r0, row);
    if constexpr (kRows > 1) fetch(r1, row + step);
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
    }
    float *p = a.part + (int64_t)blockIdx.x * 2 * a.cols;
    if constexpr (Q::TEAMS > 1) {      // the workgroup's teams, in order
        __shared__ F<N> sums[Q::TEAMS - 1][2 * P][THREADS];
        if (q.team) {
#pragma unroll
            for (int k = 0; k < P; ++k) {
                sums[q.team - 1][k][q.lane] = dw[k];
                sums[q.team - 1][P + k][q.lane] = db[k];
            }
        }
        __syncthreads();
        if (q.team) return;
#pragma unroll
        for (int t = 0; t < Q::TEAMS - 1; ++t)
#pragma unroll
            for (int k = 0; k < P; ++k) {
                dw[k] += sums[t][k][q.lane];
                db[k] += sums[t][P + k][q.lane];
            }
    }
    q.store(p, dw);
    q.store(p + a.cols, db);
}

// Rows too wide for that, or of less than a piece: dx, one workgroup a row, read twice.  2048 x 16392 of bf16: 44.9 us,
// after 23.4 for the weights' gradients below, which read x and dy again, and 4.7 for their join.
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
constexpr int64_t kGradCols = 512 * 32, kCutGradCols = 512 * 24;

template <class T, class W, bool CUT>
hipError_t norm_grad_rows(const NormGradArgs &a, hipStream_t s) {
    const int whole = a.cols - a.cols % kN<T>;      // what is left of a cut row has a place of its own
    const auto run = [&](auto kernel, int threads) {
        return launch(kernel, dim3((unsigned)a.parts), dim3(threads < 256 ? 256 : threads), s, a);
    };
    if (!whole || whole > (CUT ? kCutGradCols : kGradCols)) {
        const unsigned tiles = (unsigned)((a.cols + kWave * kN<T> - 1) / (kWave * kN<T>));
        const hipError_t e = launch(k_norm_dw_wide<T>, dim3(tiles, (unsigned)a.parts), dim3(64), s, a);
        // dx comes second: it may lie where dy is
        return e ? e : launch(k_norm_dx_wide<T, W>, dim3(grid_of(a.rows)), dim3(kWideBlock), s, a);
    }
    if (whole <= 64 * 8) return run(k_norm_grad<T, W, 64, 8, CUT>, 64);
    if (whole <= 64 * 16) return run(k_norm_grad<T, W, 64, 16, CUT>, 64);
    if (whole <= 256 * 8) return run(k_norm_grad<T, W, 256, 8, CUT>, 256);
    if (whole <= 512 * 8) return run(k_norm_grad<T, W, 512, 8, CUT>, 512);
    if (whole <= 768 * 8) return run(k_norm_grad<T, W, 768, 8, CUT>, 768);
    if constexpr (CUT) {      // the rest of a cut row takes 50 registers, which larger workgroups do not have
        if (whole <= 512 * 16) return run(k_norm_grad<T, W, 512, 16, CUT>, 512);
        return run(k_norm_grad<T, W, 512, 24, CUT>, 512);
    } else {
        if (whole <= 1024 * 8) return run(k_norm_grad<T, W, 1024, 8, CUT>, 1024);
        if (whole <= 768 * 16) return run(k_norm_grad<T, W, 768, 16, CUT>, 768);
        // 2048 x 16384: 45.5 us of bf16 with 16 wavefronts and 49.1 with 8; of f32 110.3 and 95.5.  An f32 row fits the
        // registers of neither: with 8 wavefronts a lane has 256 and spills 115 (80 bytes of scratch), with 16 it has 128
        if constexpr (sizeof(T) == 2)
            return run(k_norm_grad<T, W, 1024, 16, CUT>, 1024);
        else
            return run(k_norm_grad<T, W, 512, 32, CUT>, 512);
    }
}

template <class T, class W, class G>
hipError_t norm_grad(const NormGradArgs &a, hipStream_t s) {
    hipError_t e = hipSuccess;
    if (a.rows) e = a.cols % kN<T> ? norm_grad_rows<T, W, true>(a, s) : norm_grad_rows<T, W, false>(a, s);
    if (e) return e;
    return launch(k_norm_join<G>, dim3((unsigned)((a.cols + kWave - 1) / kWave), 2), dim3(kJoinWaves * kWave), s, a);
}

}  // namespace

// A part is a workgroup of the gradient's kernel.  More of them fill the chip, but every one leaves 8 bytes a
// column to write and read again: one wave of workgroups over the 256 compute units, two of those of four
// wavefronts.
int norm_grad_parts(int64_t rows, int64_t cols) {
    const int teams = cols <= 64 * 16 ? 4 : 1;
    const int64_t n = (rows + teams - 1) / teams, most = cols > kGradCols ? 64 : cols <= 256 * 8 ? 512 : 256;
    return (int)(n < most ? n : most);
}

template <class T, class W>
static hipError_t norm_of(const NormArgs &a, hipStream_t s) {
    return a.cols % kN<T> ? norm<T, W, true>(a, s) : norm<T, W, false>(a, s);
}
hipError_t launch_norm(const NormArgs &a, int type, int weight_type, hipStream_t s) {
    const bool same = type == weight_type;
    switch (type) {
        case ECHO_F32: return norm_of<float, float>(a, s);
        case ECHO_F16: return same ? norm_of<f16, f16>(a, s) : norm_of<f16, float>(a, s);
        default: return same ? norm_of<bf16, bf16>(a, s) : norm_of<bf16, float>(a, s);
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

}  // namespace echo
