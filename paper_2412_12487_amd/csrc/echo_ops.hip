// echo_ops.hip -- gfx950 kernels of the training-step operators (echo_ops.h).
//
// All of them move bytes: nothing multiplies matrices, and every operator's floor is the time
// to read its inputs and write its outputs once.  Activations are read eight elements at a time with the
// alignment of one element (the hardware loads 16 bytes from any address), sums and statistics are
// held in 32 bits, and no result depends on the order in which workgroups run.
#include "echo_ops_internal.h"

namespace echo {
namespace {

using bf16 = __bf16;
using f16 = _Float16;

constexpr int kWave = 64;
constexpr int kVec = 8;                  // elements that a lane loads at a time
constexpr unsigned kMaxGrid = 1u << 20;  // workgroups of a launch, at most; kernels stride over the rest

template <class T>
struct Vec {
    typedef T type __attribute__((ext_vector_type(kVec), aligned(sizeof(T))));
};
template <class T>
using V8 = typename Vec<T>::type;
using F8 = V8<float>;

// Elements col .. col + 7 of a row of `cols`; `fill` stands where the row has ended.
template <class T>
__device__ __forceinline__ V8<T> load8(const T *row, int col, int cols, T fill = T(0)) {
    if (col + kVec <= cols) return *reinterpret_cast<const V8<T> *>(row + col);
    V8<T> v;
#pragma unroll
    for (int j = 0; j < kVec; ++j) v[j] = col + j < cols ? row[col + j] : fill;
    return v;
}
template <class T>
__device__ __forceinline__ void store8(T *row, int col, int cols, V8<T> v) {
    if (col + kVec <= cols) {
        *reinterpret_cast<V8<T> *>(row + col) = v;
        return;
    }
#pragma unroll
    for (int j = 0; j < kVec; ++j)
        if (col + j < cols) row[col + j] = v[j];
}
template <class T>
__device__ __forceinline__ F8 widen(V8<T> v) {
    return __builtin_convertvector(v, F8);
}
template <class T>
__device__ __forceinline__ V8<T> round_to(F8 v) {
    return __builtin_convertvector(v, V8<T>);
}

// Sum and maximum over a wavefront, the same in every lane.  A maximum passes over NaN: a row with a
// NaN has it in its sum.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = kWave / 2; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int d = kWave / 2; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
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
template <int WAVES>
__device__ __forceinline__ float block_max(float v, float *lds) {
    v = wave_max(v);
    __syncthreads();
    if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = v;
    __syncthreads();
    float s = lds[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) s = fmaxf(s, lds[w]);
    return s;
}

template <class F, class... A>
hipError_t launch(void (*kernel)(F, A...), dim3 grid, dim3 block, hipStream_t s, F f, A... rest) {
    void *args[] = {&f, &rest...};
    return hipLaunchKernel(reinterpret_cast<const void *>(kernel), grid, block, args, 0, s);
}
unsigned grid_of(int64_t n) { return (unsigned)(n < 1 ? 1 : n < (int64_t)kMaxGrid ? n : (int64_t)kMaxGrid); }

// ---------------------------------------------------------------- layer norm

// One workgroup a row, which is read three times (sum, squares about the mean, result).
template <class T, class W>
__global__ __launch_bounds__(256) void k_norm(NormArgs a) {
    __shared__ float lds[4];
    const W *w = static_cast<const W *>(a.weight), *b = static_cast<const W *>(a.bias);
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
        const T *h = x;
        float s = 0.0f;
        if (a.residual) {
            const T *r = static_cast<const T *>(a.residual) + row * a.residual_stride;
            T *sum = static_cast<T *>(a.sum) + row * a.cols;
            for (int c = threadIdx.x * kVec; c < a.cols; c += 256 * kVec) {
                const V8<T> v = round_to<T>(widen<T>(load8(x, c, a.cols)) + widen<T>(load8(r, c, a.cols)));
                store8(sum, c, a.cols, v);
                const F8 f = widen<T>(v);
                for (int j = 0; j < kVec; ++j) s += f[j];
            }
            h = sum;      // each lane reads back what it wrote
        } else {
            for (int c = threadIdx.x * kVec; c < a.cols; c += 256 * kVec) {
                const F8 f = widen<T>(load8(x, c, a.cols));
                for (int j = 0; j < kVec; ++j) s += f[j];
            }
        }
        const float mean = block_sum<4>(s, lds) / (float)a.cols;
        s = 0.0f;
        for (int c = threadIdx.x * kVec; c < a.cols; c += 256 * kVec) {
            const F8 f = widen<T>(load8(h, c, a.cols));
            for (int j = 0; j < kVec; ++j) {
                const float d = c + j < a.cols ? f[j] - mean : 0.0f;
                s += d * d;
            }
        }
        const float rstd = 1.0f / sqrtf(block_sum<4>(s, lds) / (float)a.cols + a.eps);
        T *y = static_cast<T *>(a.y) + row * a.cols;
        for (int c = threadIdx.x * kVec; c < a.cols; c += 256 * kVec) {
            F8 f = (widen<T>(load8(h, c, a.cols)) - mean) * rstd * widen<W>(load8(w, c, a.cols));
            if (b) f += widen<W>(load8(b, c, a.cols));
            store8(y, c, a.cols, round_to<T>(f));
        }
        if (threadIdx.x == 0) {
            a.mean[row] = mean;
            a.rstd[row] = rstd;
        }
    }
}

// dx, one workgroup a row, read twice.
template <class T, class W>
__global__ __launch_bounds__(256) void k_norm_dx(NormGradArgs a) {
    __shared__ float lds[4];
    const W *w = static_cast<const W *>(a.weight);
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *dy = static_cast<const T *>(a.dy) + row * a.dy_stride;
        const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float s1 = 0.0f, s2 = 0.0f;
        for (int c = threadIdx.x * kVec; c < a.cols; c += 256 * kVec) {
            const F8 n = (widen<T>(load8(x, c, a.cols)) - mean) * rstd;
            const F8 g = widen<T>(load8(dy, c, a.cols)) * widen<W>(load8(w, c, a.cols));
            for (int j = 0; j < kVec; ++j) {
                s1 += g[j];
                s2 += c + j < a.cols ? g[j] * n[j] : 0.0f;
            }
        }
        s1 = block_sum<4>(s1, lds) / (float)a.cols;
        s2 = block_sum<4>(s2, lds) / (float)a.cols;
        T *dx = static_cast<T *>(a.dx) + row * a.cols;
        for (int c = threadIdx.x * kVec; c < a.cols; c += 256 * kVec) {
            const F8 n = (widen<T>(load8(x, c, a.cols)) - mean) * rstd;
            const F8 g = widen<T>(load8(dy, c, a.cols)) * widen<W>(load8(w, c, a.cols));
            F8 d = rstd * (g - s1 - n * s2);
            if (a.grad_residual)
                d += widen<T>(load8(static_cast<const T *>(a.grad_residual) + row * a.grad_residual_stride, c, a.cols));
            store8(dx, c, a.cols, round_to<T>(d));
        }
    }
}

// The weights' gradients over part blockIdx.y of the rows (a contiguous run), 64 x 8 columns a wavefront.
template <class T>
__global__ __launch_bounds__(64) void k_norm_dw(NormGradArgs a) {
    const int c = (blockIdx.x * kWave + threadIdx.x) * kVec;
    if (c >= a.cols) return;
    const int64_t lo = a.rows * blockIdx.y / a.parts, hi = a.rows * (blockIdx.y + 1) / a.parts;
    F8 dw = 0.0f, db = 0.0f;
    for (int64_t row = lo; row < hi; ++row) {
        const F8 n = (widen<T>(load8(static_cast<const T *>(a.x) + row * a.x_stride, c, a.cols)) - a.mean[row]) * a.rstd[row];
        const F8 dy = widen<T>(load8(static_cast<const T *>(a.dy) + row * a.dy_stride, c, a.cols));
        dw += dy * n;
        db += dy;
    }
    float *p = a.part + (int64_t)blockIdx.y * 2 * a.cols;
    store8(p, c, a.cols, dw);
    store8(p + a.cols, c, a.cols, db);
}

// Sums the parts in order.
template <class G>
__global__ __launch_bounds__(64) void k_norm_join(NormGradArgs a) {
    const int c = blockIdx.x * kWave + threadIdx.x;
    G *out = static_cast<G *>(blockIdx.y ? a.dbias : a.dweight);
    if (c >= a.cols || !out) return;
    const float *p = a.part + (int64_t)blockIdx.y * a.cols + c;
    float s = 0.0f;
    for (int k = 0; k < a.parts; ++k) s += p[(int64_t)k * 2 * a.cols];
    if (a.accumulate) s += (float)out[c];
    out[c] = (G)s;
}

template <class T, class W>
hipError_t norm(const NormArgs &a, hipStream_t s) {
    return launch(k_norm<T, W>, dim3(grid_of(a.rows)), dim3(256), s, a);
}
template <class T, class W, class G>
hipError_t norm_grad(const NormGradArgs &a, hipStream_t s) {
    hipError_t e = hipSuccess;
    const unsigned tiles = (unsigned)((a.cols + kWave * kVec - 1) / (kWave * kVec));
    // dx comes second: it may lie where dy is
    if (a.rows && (e = launch(k_norm_dw<T>, dim3(tiles, (unsigned)a.parts), dim3(64), s, a))) return e;
    if (a.rows && (e = launch(k_norm_dx<T, W>, dim3(grid_of(a.rows)), dim3(256), s, a))) return e;
    return launch(k_norm_join<G>, dim3((unsigned)((a.cols + kWave - 1) / kWave), 2), dim3(64), s, a);
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

template <class T, class I>
__global__ __launch_bounds__(256) void k_embed(EmbedArgs a) {
    for (int64_t t = blockIdx.x; t < a.rows; t += gridDim.x) {
        const int v = shard_row(id_at<I>(a.ids, t), a.vocab_start, a.vocab);
        T *out = static_cast<T *>(a.out) + t * a.cols;
        const T *w = static_cast<const T *>(a.weight) + (int64_t)(v < 0 ? 0 : v) * a.weight_stride;
        for (int c = threadIdx.x * kVec; c < a.cols; c += 256 * kVec) {
            V8<T> r = T(0);
            if (v >= 0) r = round_to<T>(widen<T>(load8(w, c, a.cols)) * a.scale);
            store8(out, c, a.cols, r);
        }
    }
}

// Workspace of the gradient: where each row's tokens begin, and the tokens sorted by row.
struct EmbedSpace {
    int *begin, *token;
};
int64_t round16(int64_t n) { return (n + 15) & ~int64_t(15); }
EmbedSpace embed_space(void *p, int64_t vocab) {
    char *c = static_cast<char *>(p);
    return EmbedSpace{reinterpret_cast<int *>(c), reinterpret_cast<int *>(c + round16((vocab + 1) * 4))};
}

// Tokens sorted by row of the shard, ascending within a row.  Each wavefront owns 64 rows (one a lane)
// and reads every id twice: it counts its rows' tokens and those of the rows before them, which
// says where its rows begin, and then places its tokens in order.  Lanes whose ids name the same row
// are placed together, in the order of the lanes.
template <class I>
__global__ __launch_bounds__(64) void k_embed_sort(EmbedGradArgs a, EmbedSpace ws) {
    const int lane = threadIdx.x, first = blockIdx.x * kWave;
    const uint64_t below = (uint64_t(1) << lane) - 1;
    int count = 0, before = 0;
    for (int64_t t = 0; t < a.rows; t += kWave) {
        const int v = t + lane < a.rows ? shard_row(id_at<I>(a.ids, t + lane), a.vocab_start, a.vocab) : -1;
        before += __popcll(__ballot(v >= 0 && v < first));
        uint64_t mine = __ballot(v >= first && v - first < kWave);
        while (mine) {
            const int row = __shfl(v, __ffsll((unsigned long long)mine) - 1);
            const uint64_t same = __ballot(v == row);
            if (lane == row - first) count += __popcll(same);
            mine &= ~same;
        }
    }
    int at = count;      // exclusive prefix sum over the lanes
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const int up = __shfl_up(at, d);
        if (lane >= d) at += up;
    }
    at += before - count;
    if (first + lane < a.vocab) ws.begin[first + lane] = at;
    if (first + lane == a.vocab - 1) ws.begin[a.vocab] = at + count;
    for (int64_t t = 0; t < a.rows; t += kWave) {
        const int v = t + lane < a.rows ? shard_row(id_at<I>(a.ids, t + lane), a.vocab_start, a.vocab) : -1;
        uint64_t mine = __ballot(v >= first && v - first < kWave);
        while (mine) {
            const int row = __shfl(v, __ffsll((unsigned long long)mine) - 1);
            const uint64_t same = __ballot(v == row);
            const int base = __shfl(at, row - first);
            if (v == row) ws.token[base + __popcll(same & below)] = (int)(t + lane);
            if (lane == row - first) at += __popcll(same);
            mine &= ~same;
        }
    }
}

// One workgroup a row of the table.
template <class T, class G>
__global__ __launch_bounds__(256) void k_embed_dw(EmbedGradArgs a, EmbedSpace ws) {
    for (int v = blockIdx.x; v < a.vocab; v += gridDim.x) {
        const int lo = a.rows ? ws.begin[v] : 0, hi = a.rows ? ws.begin[v + 1] : 0;
        if (a.accumulate && lo == hi) continue;
        G *out = static_cast<G *>(a.dweight) + (int64_t)v * a.cols;
        for (int c = threadIdx.x * kVec; c < a.cols; c += 256 * kVec) {
            F8 s = 0.0f;
            for (int k = lo; k < hi; ++k)
                s += widen<T>(load8(static_cast<const T *>(a.dy) + (int64_t)ws.token[k] * a.dy_stride, c, a.cols));
            s *= a.scale;
            if (a.accumulate) s += widen<G>(load8(out, c, a.cols));
            store8(out, c, a.cols, round_to<G>(s));
        }
    }
}

template <class T, class G>
hipError_t embed_grad(const EmbedGradArgs &a, int index_type, hipStream_t s) {
    const EmbedSpace ws = embed_space(a.workspace, a.vocab);
    const dim3 sorters((unsigned)((a.vocab + kWave - 1) / kWave));
    hipError_t e = hipSuccess;
    if (a.rows)
        e = index_type == ECHO_I64 ? launch(k_embed_sort<int64_t>, sorters, dim3(kWave), s, a, ws)
                                   : launch(k_embed_sort<int32_t>, sorters, dim3(kWave), s, a, ws);
    if (e) return e;
    return launch(k_embed_dw<T, G>, dim3(grid_of(a.vocab)), dim3(256), s, a, ws);
}

// ---------------------------------------------------------------- cross entropy

constexpr float kInf = __builtin_huge_valf();

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
// (exp(l - lse) - [column = target]) * g for the columns col .. col + 7.
__device__ __forceinline__ F8 loss_grad8(F8 l, float lse, int col, int at, float g) {
    F8 d;
#pragma unroll
    for (int j = 0; j < kVec; ++j) d[j] = (expf(l[j] - lse) - (col + j == at ? 1.0f : 0.0f)) * g;
    return d;
}

template <class T, class I>
__global__ __launch_bounds__(256) void k_loss(LossArgs a) {
    __shared__ float lds[4];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *l = static_cast<const T *>(a.logits) + row * a.logits_stride;
        const LossRow r = loss_row<I>(a, row);
        const float hit = r.at >= 0 ? (float)l[r.at] : 0.0f;
        float top = -kInf;
        for (int c = threadIdx.x * kVec; c < a.cols; c += 256 * kVec) {
            const F8 f = widen<T>(load8(l, c, a.cols, T(-kInf)));
            for (int j = 0; j < kVec; ++j) top = fmaxf(top, f[j]);
        }
        top = block_max<4>(top, lds);
        if (top == -kInf) top = 0.0f;      // nothing left of the row: the sum is 0 and its log -inf
        float s = 0.0f;
        for (int c = threadIdx.x * kVec; c < a.cols; c += 256 * kVec) {
            const F8 f = widen<T>(load8(l, c, a.cols, T(-kInf)));
            for (int j = 0; j < kVec; ++j) s += expf(f[j] - top);
        }
        const float lse = top + logf(block_sum<4>(s, lds));
        if (threadIdx.x == 0) {
            if (a.lse) a.lse[row] = lse;
            if (a.target) a.target[row] = hit;
            if (a.loss) a.loss[row] = !r.trained ? 0.0f : lse == -kInf ? kInf : lse - hit;
        }
        if (!a.grad) continue;
        T *d = static_cast<T *>(a.grad) + row * a.grad_stride;
        const bool live = r.trained && lse != -kInf;
        const float g = a.grad_loss[row];
        __syncthreads();      // the target's logit has been read: grad may be logits
        for (int c = threadIdx.x * kVec; c < a.cols; c += 256 * kVec) {
            F8 f = 0.0f;
            if (live) f = loss_grad8(widen<T>(load8(l, c, a.cols)), lse, c, r.at, g);
            store8(d, c, a.cols, round_to<T>(f));
        }
    }
}

template <class T, class I>
__global__ __launch_bounds__(256) void k_loss_grad(LossArgs a) {
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *l = static_cast<const T *>(a.logits) + row * a.logits_stride;
        T *d = static_cast<T *>(a.grad) + row * a.grad_stride;
        const LossRow r = loss_row<I>(a, row);
        const float lse = a.lse_in[row], g = a.grad_loss[row];
        const bool live = r.trained && lse != -kInf;
        for (int c = threadIdx.x * kVec; c < a.cols; c += 256 * kVec) {
            F8 f = 0.0f;
            if (live) f = loss_grad8(widen<T>(load8(l, c, a.cols)), lse, c, r.at, g);
            store8(d, c, a.cols, round_to<T>(f));
        }
    }
}

}  // namespace

int norm_grad_parts(int64_t rows, int64_t) { return (int)(rows < 64 ? rows : 64); }
int64_t embed_grad_bytes(int64_t rows, int64_t, int64_t vocab) {
    return rows ? round16((vocab + 1) * 4) + round16(rows * 4) : 0;
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

template <class I>
static hipError_t embed_of(const EmbedArgs &a, int type, hipStream_t s) {
    const dim3 grid(grid_of(a.rows)), block(256);
    switch (type) {
        case ECHO_F32: return launch(k_embed<float, I>, grid, block, s, a);
        case ECHO_F16: return launch(k_embed<f16, I>, grid, block, s, a);
        default: return launch(k_embed<bf16, I>, grid, block, s, a);
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
    const dim3 grid(grid_of(a.rows)), block(256);
    switch (type) {
        case ECHO_F32: return launch(grad_alone ? k_loss_grad<float, I> : k_loss<float, I>, grid, block, s, a);
        case ECHO_F16: return launch(grad_alone ? k_loss_grad<f16, I> : k_loss<f16, I>, grid, block, s, a);
        default: return launch(grad_alone ? k_loss_grad<bf16, I> : k_loss<bf16, I>, grid, block, s, a);
    }
}
hipError_t launch_loss(const LossArgs &a, int type, int index_type, hipStream_t s) {
    return index_type == ECHO_I64 ? loss_of<int64_t>(a, type, false, s) : loss_of<int32_t>(a, type, false, s);
}
hipError_t launch_loss_grad(const LossArgs &a, int type, int index_type, hipStream_t s) {
    return index_type == ECHO_I64 ? loss_of<int64_t>(a, type, true, s) : loss_of<int32_t>(a, type, true, s);
}

}  // namespace echo
