// echo_ops_device.h -- what the kernels of the training-step operators (echo_ops.h) share.
//
// All but the output head's (echo_product.h) move bytes: every operator's floor is the time
// to read its inputs and write its outputs once.  A lane moves 16 bytes of activations at a time with the
// alignment of one element (the hardware takes 16 bytes from any address), rows that fit stay in registers between
// their statistics and their result, sums and statistics are held in 32 bits, and no result depends
// on the order in which workgroups run.
#pragma once

#include "echo_ops_internal.h"

// Kernels' lambdas that are called more than once: left as functions, what they capture goes through memory.
#define ECHO_INLINE __attribute__((always_inline))

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
// store of results that stream out: whole 16-byte pieces of a lane, side by side over the lanes (Team::drop has the figure).
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
// Sum and maximum over every N lanes side by side that hold N values in turn (N a power of two, at most 16).
template <int N>
__device__ __forceinline__ float ring_sum(float v) {
    if constexpr (N > 1) return ring_sum<N / 2>(v + rotated<N / 2>(v));
    return v;
}
template <int N>
__device__ __forceinline__ float ring_max(float v) {
    if constexpr (N > 1) return ring_max<N / 2>(fmaxf(v, rotated<N / 2>(v)));
    return v;
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

// Workgroup of the kernels for rows that registers do not hold.
constexpr int kWideBlock = 1024, kWideWaves = kWideBlock / kWave;

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
[[maybe_unused]] unsigned grid_of(int64_t n) { return (unsigned)(n < 1 ? 1 : n < (int64_t)kMaxGrid ? n : (int64_t)kMaxGrid); }

// A row's address, the same in every lane, in scalar registers.  Left to itself the compiler keeps
// a running address a lane for every piece of every row that a loop visits, 30 registers a piece.
template <class U>
__device__ __forceinline__ U *row_base(U *p) {
    asm volatile("" : "+s"(p));
    return p;
}
// A piece as 32-bit words.
template <class T, int N>
struct WordsOf {
    typedef int type __attribute__((ext_vector_type(N * sizeof(T) / 4)));
};
template <class T, int N>
using Words = typename WordsOf<T, N>::type;
// Keeps the compiler from holding what it made of v: from here on v is converted anew.
template <class T, int N, int M>
__device__ __forceinline__ void forget(V<T, N> (&v)[M]) {
#pragma unroll
    for (int k = 0; k < M; ++k) {
        Words<T, N> w = __builtin_bit_cast(Words<T, N>, v[k]);
        asm volatile("" : "+v"(w));
        v[k] = __builtin_bit_cast(V<T, N>, w);
    }
}

// A team of THREADS lanes holds a row of up to THREADS * E elements in registers, E a lane, as K pieces of 16
// bytes of T: lane i has the pieces k * THREADS + i.  Narrow teams share a workgroup of four wavefronts.
// CUT rows are not whole pieces (cols % N != 0): what their end leaves is piece K, of the team's last lane
// alone.  It comes as the row's last N elements, and settle() moves them to their places, apart, so that a row can
// be on its way while another is worked on.  A row has one whole piece at least.
template <class T, int THREADS, int E, bool CUT>
struct Team {
    static constexpr int N = kN<T>, K = E / N, P = K + CUT, BLOCK = THREADS < 256 ? 256 : THREADS, TEAMS = BLOCK / THREADS,
                         WAVES = THREADS / kWave;
    static_assert(K * N == E, "");
    const int lane = threadIdx.x % THREADS, wave = __builtin_amdgcn_readfirstlane(lane / kWave),
              team = __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS), cols, left = CUT ? cols % N : 0;
    __device__ __forceinline__ explicit Team(int c) : cols(c) {}
    __device__ __forceinline__ bool ends() const { return lane == THREADS - 1; }
    // whether this lane has piece k
    __device__ __forceinline__ bool has(int k) const {
        return k < K ? lane * N + N <= cols - k * THREADS * N : ends();
    }
    __device__ __forceinline__ int col(int k) const { return k < K ? (k * THREADS + lane) * N : cols - left; }
    // elements that wavefront w has of the row
    __device__ __forceinline__ int count(int w) const {
        int n = w == WAVES - 1 ? left : 0;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int rest = cols / N - k * THREADS - w * kWave;      // whole pieces from its first lane on
            n += (rest < 0 ? 0 : rest < kWave ? rest : kWave) * N;
        }
        return n;
    }
    // 32-bit offsets of the lanes from a piece's address, which is the same in all of them
    template <class U>
    __device__ __forceinline__ const V<U, N> *at(const U *row, int k) const {
        return reinterpret_cast<const V<U, N> *>(reinterpret_cast<const char *>(row + k * THREADS * N) +
                                                 (unsigned)(lane * N * sizeof(U)));
    }
    template <class U>
    __device__ __forceinline__ void fetch(const U *row, V<U, N> (&v)[P], U fill = U(0)) const {
        row = row_base(row);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = fill;
            if (has(k)) v[k] = *at(row, k);
        }
        if constexpr (CUT) {
            v[K] = fill;
            if (ends()) v[K] = *reinterpret_cast<const V<U, N> *>(row + (cols - N));
        }
    }
    template <class U>
    __device__ __forceinline__ void settle(V<U, N> (&v)[P], U fill) const {
        if constexpr (CUT) {
            if (!ends()) return;
            V<U, N> t = v[K];
#pragma unroll
            for (int b = N / 2; b; b /= 2) {
                V<U, N> moved;
#pragma unroll
                for (int j = 0; j < N; ++j) moved[j] = j + b < N ? t[(j + b) % N] : fill;
                t = (N - left) & b ? moved : t;
            }
            v[K] = t;
        }
    }
    template <class U>
    __device__ __forceinline__ void load(const U *row, V<U, N> (&v)[P], U fill = U(0)) const {
        fetch(row, v, fill);
        settle(v, fill);
    }
    template <bool DROP, class U>
    __device__ __forceinline__ void put(U *row, const V<U, N> (&v)[P]) const {
        row = row_base(row);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (!has(k)) continue;
            V<U, N> *p = const_cast<V<U, N> *>(at(row, k));
            if constexpr (DROP)
                __builtin_nontemporal_store(v[k], p);
            else
                *p = v[k];
        }
        if constexpr (CUT) {
            if (!ends()) return;
#pragma unroll
            for (int j = 0; j < N - 1; ++j)
                if (j < left) row[cols - left + j] = v[K][j];
        }
    }
    // Results that stream out: past the caches, in whole 16-byte pieces side by side over the lanes.
    // When they came in, a pass of layer norm of 2048 x 8192 of bf16 with a residual went from 29.0 to 26.7 us with them
    // (22.0 now).
    __device__ __forceinline__ void drop(T *row, const V<T, N> (&v)[P]) const { put<true>(row, v); }
    template <class U>
    __device__ __forceinline__ void store(U *row, const V<U, N> (&v)[P]) const {
        put<false>(row, v);
    }
};

template <class I>
__device__ __forceinline__ int64_t id_at(const void *ids, int64_t t) {
    return (int64_t)static_cast<const I *>(ids)[t];
}
// Row of the shard that an id names, or -1.  Subtracted without sign: any id is allowed.
__device__ __forceinline__ int shard_row(int64_t id, int64_t start, int vocab) {
    const uint64_t v = (uint64_t)id - (uint64_t)start;
    return v < (uint64_t)vocab ? (int)v : -1;
}

}  // namespace
}  // namespace echo
