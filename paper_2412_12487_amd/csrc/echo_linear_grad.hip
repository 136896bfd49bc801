// echo_linear_grad.hip -- gradients of hidden states and of the output table from the logits' gradient, on gfx950.
#include "echo_linear.h"

namespace echo {
namespace {

template <class U>
__device__ __forceinline__ void put4(U *out, int left, F4 d, bool add) {
    typedef V<U, 4> U4;
    if (left >= 4) {
        if (add) d += __builtin_convertvector(*reinterpret_cast<const U4 *>(out), F4);
        *reinterpret_cast<U4 *>(out) = __builtin_convertvector(d, U4);
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < left) out[e] = (U)(d[e] + (add ? (float)out[e] : 0.0f));
}

// i over the hidden size, across the rows of operand a; j over rows (deep) or over the vocabulary.  Results of 16 bits leave in whole
// rows: the table's gradient of 512 x 1024 over 51200 ids took 87 us with 8 bytes a lane of 16 rows at a time and takes 75.
template <class T, class U, class S, bool DEEP>
__device__ __forceinline__ void out_tile(const OutArgs &a, int id, [[maybe_unused]] char *t0, [[maybe_unused]] char *t1) {
    const Place at = place_of(a.m, id);
    F4 acc[S::BI][S::BJ];
#ifdef __HIP_DEVICE_COMPILE__      // reads shared memory transposed, which the host's pass does not know
    multiply<T, false, DEEP, S>(a.m, at, t0, t1, acc);
#endif
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wi = wave / S::WJ, wj = wave % S::WJ;
    const int i0 = at.ti * S::TI + wi * S::BI * 16 + (lane / 16) * 4, j0 = at.tj * S::TJ + wj * S::BJ * 16 + lane % 16;
    const float scale = a.parts ? 1.0f : *a.scale * (a.factor / kUnit<T>);
    if constexpr (sizeof(U) == 2) {
        if (!a.parts && !a.accumulate) {
            const Outgoing<S, U> outgoing(t0, t1, wave, lane);
            __syncthreads();      // the last step has been read
#pragma unroll
            for (int b = 0; b < S::BJ; ++b)
#pragma unroll
                for (int k = 0; k < S::BI; ++k) outgoing.put(k, b, acc[k][b] * scale);
            const int i = at.ti * S::TI + wi * S::BI * 16, j = at.tj * S::TJ + wj * S::BJ * 16;
            return outgoing.flush(static_cast<U *>(a.out) + (int64_t)j * a.m.ni + i, a.m.ni, a.m.nj - j, a.m.ni - i);
        }
    }
#pragma unroll
    for (int b = 0; b < S::BJ; ++b) {
        const int j = j0 + b * 16;
        if (j >= a.m.nj) continue;
#pragma unroll
        for (int k = 0; k < S::BI; ++k) {
            const int i = i0 + k * 16;
            if (i >= a.m.ni) continue;
            const F4 d = acc[k][b] * scale;
            if (a.parts)
                put4(a.parts + at.split * a.part + (int64_t)j * a.m.ni + i, a.m.ni - i, d, a.add_parts);
            else
                put4(static_cast<U *>(a.out) + (int64_t)j * a.m.ni + i, a.m.ni - i, d, a.accumulate);
        }
    }
}
template <class T, class U, class S, bool DEEP>
__global__ __launch_bounds__(S::THREADS, S::THREADS / 256) void k_out(OutArgs a) {
    __shared__ __attribute__((aligned(16))) char t0[S::BYTES];
    __shared__ __attribute__((aligned(16))) char t1[S::BYTES];
    out_tile<T, U, S, DEEP>(a, blockIdx.x, t0, t1);
}
// Both gradients in one launch, where neither fills the GPU (8 rows of 6592, 256 ids: 6 us in place of 12), the longer
// sums first: the hidden states' of type U, the table's of type W.
template <class T, class U, class W, class S>
__global__ __launch_bounds__(S::THREADS, S::THREADS / 256) void k_both(OutArgs hidden, OutArgs table, int table_first) {
    __shared__ __attribute__((aligned(16))) char t0[S::BYTES];
    __shared__ __attribute__((aligned(16))) char t1[S::BYTES];
    const int of_hidden = hidden.m.tiles_i * hidden.m.tiles_j * hidden.m.splits, of_table = table.m.tiles_i * table.m.tiles_j * table.m.splits;
    const int id = table_first ? (int)blockIdx.x - of_table : (int)blockIdx.x;
    if (table_first ? id >= 0 : id < of_hidden)
        out_tile<T, U, S, true>(hidden, id, t0, t1);
    else
        out_tile<T, W, S, false>(table, table_first ? (int)blockIdx.x : id - of_hidden, t0, t1);
}

// Sums the parts: four wavefronts take a quarter of them each, in their order, of 256 elements side by side.
template <class U>
__global__ __launch_bounds__(256) void k_gather(GatherArgs a, float unit) {
    __shared__ F4 lds[4][kWave];
    const float scale = *a.scale * (a.factor / unit);
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, begin = a.splits * wave / 4, end = a.splits * (wave + 1) / 4;
    for (int64_t first = (int64_t)blockIdx.x * 256; first < a.n; first += (int64_t)gridDim.x * 256) {
        const int64_t at = first + lane * 4;
        const int left = a.n - at < 4 ? (int)(a.n - at) : 4;
        F4 d = 0.0f;
#pragma unroll 4
        for (int p = begin; p < end; ++p) {
            const float *from = a.parts + p * a.n + at;
            if (left == 4) {
                d += *reinterpret_cast<const V<float, 4> *>(from);
            } else {
                for (int e = 0; e < left; ++e) d[e] += from[e];
            }
        }
        __syncthreads();
        lds[wave][lane] = d;
        __syncthreads();
        if (wave || left <= 0) continue;
        put4(static_cast<U *>(a.out) + at, left, (((lds[0][lane] + lds[1][lane]) + lds[2][lane]) + lds[3][lane]) * scale, a.accumulate);
    }
}

// No rows: the table's gradient is zeros.
__global__ __launch_bounds__(256) void k_zero(unsigned short *out, int64_t n) {
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < n; at += (int64_t)gridDim.x * 256) out[at] = 0;
}

template <class T, class U, bool DEEP>
hipError_t out(const OutArgs &a, int shape, hipStream_t s) {
    const dim3 grid((unsigned)(a.m.tiles_i * a.m.tiles_j * a.m.splits));
    switch (shape) {
        case 0: return launch(k_out<T, U, Wide, DEEP>, grid, dim3(Wide::THREADS), s, a);
        default: return launch(k_out<T, U, Middle, DEEP>, grid, dim3(Middle::THREADS), s, a);
    }
}
template <class T, class U>
hipError_t out(const OutArgs &a, bool deep, int shape, hipStream_t s) {
    return deep ? out<T, U, true>(a, shape, s) : out<T, U, false>(a, shape, s);
}

}  // namespace

hipError_t launch_out(const OutArgs &a, int type, int out_type, bool deep, int shape, hipStream_t s) {
    if (type == ECHO_F16) return out_type == ECHO_F32 ? out<f16, float>(a, deep, shape, s) : out<f16, f16>(a, deep, shape, s);
    return out_type == ECHO_F32 ? out<bf16, float>(a, deep, shape, s) : out<bf16, bf16>(a, deep, shape, s);
}
hipError_t launch_both(const OutArgs &a, const OutArgs &b, int type, int grad_type, hipStream_t s) {
    const dim3 grid((unsigned)(a.m.tiles_i * a.m.tiles_j * a.m.splits + b.m.tiles_i * b.m.tiles_j * b.m.splits)), block(Middle::THREADS);
    const bool wide = grad_type == ECHO_F32;
    const int t = (int64_t)b.m.steps * a.m.splits > (int64_t)a.m.steps * b.m.splits;
    switch (type) {
        case ECHO_F32: return launch(k_both<bf16, float, float, Middle>, grid, block, s, a, b, t);
        case ECHO_F16:
            return wide ? launch(k_both<f16, f16, float, Middle>, grid, block, s, a, b, t) : launch(k_both<f16, f16, f16, Middle>, grid, block, s, a, b, t);
        default:
            return wide ? launch(k_both<bf16, bf16, float, Middle>, grid, block, s, a, b, t)
                        : launch(k_both<bf16, bf16, bf16, Middle>, grid, block, s, a, b, t);
    }
}
hipError_t launch_zero(void *out, int64_t bytes, hipStream_t s) {
    return launch(k_zero, dim3(grid_of((bytes / 2 + 255) / 256)), dim3(256), s, static_cast<unsigned short *>(out), bytes / 2);
}
hipError_t launch_gather(const GatherArgs &a, int type, int out_type, hipStream_t s) {
    const dim3 grid(grid_of((a.n + 255) / 256));
    const float unit = type == ECHO_F16 ? kUnit<f16> : 1.0f;
    switch (out_type) {
        case ECHO_F32: return launch(k_gather<float>, grid, dim3(256), s, a, unit);
        case ECHO_F16: return launch(k_gather<f16>, grid, dim3(256), s, a, unit);
        default: return launch(k_gather<bf16>, grid, dim3(256), s, a, unit);
    }
}

}  // namespace echo
