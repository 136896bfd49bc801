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
// load8 of data that nothing reads again soon.
template <class T>
__device__ __forceinline__ V8<T> stream8(const T *row, int col, int cols, T fill = T(0)) {
    if (col + kVec <= cols) return __builtin_nontemporal_load(reinterpret_cast<const V8<T> *>(row + col));
    return load8(row, col, cols, fill);
}
// A wavefront writes zeros to a row, 16 bytes a lane.
template <class T>
__device__ __forceinline__ void zero_row(T *row, int cols) {
    constexpr int n = 16 / sizeof(T);
    typedef T Z __attribute__((ext_vector_type(n), aligned(sizeof(T))));
    for (int c = threadIdx.x % kWave * n; c < cols; c += kWave * n) {
        if (c + n <= cols) {
            *reinterpret_cast<Z *>(row + c) = Z(T(0));
        } else {
            for (int j = c; j < cols; ++j) row[j] = T(0);
        }
    }
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
constexpr int kTile = kWave * kVec;      // columns that a wavefront takes at a time
int64_t tiles_of(int64_t cols) { return (cols + kTile - 1) / kTile; }

// Sorted places of a chunk: few enough to give the chip wavefronts, and no fewer.  A wavefront looks at two
// chunks, one place a lane.
int embed_chunk(int64_t rows, int64_t cols) {
    int c = 4;
    while (c < kWave / 2 && (rows + c - 1) / c * tiles_of(cols) > 16384) c *= 2;
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
    constexpr int kAhead = 4;
    const int lane = threadIdx.x % kWave;
    const int64_t id = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave, tiles = (a.cols + kTile - 1) / kTile;
    if (id >= sums) {
        for (int64_t v = id - sums; v < a.vocab; v += (int64_t)gridDim.x * 4 - sums) {
            const int slot = slot_of((int)v, bits);
            if (a.rows && ws.begin[slot] != ws.begin[slot + 1]) continue;
            zero_row(row_of<G>(a, (int)v), a.cols);
        }
        return;
    }
    const int64_t j = id / tiles, base = j * chunk;
    const int c = (int)(id % tiles) * kTile + lane * kVec;
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
    F8 s = 0.0f;
    for (int i = begin; i < end; i += kAhead) {
        V8<T> r[kAhead];
        V8<G> old[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (i + k >= end || c >= a.cols) continue;
            r[k] = stream8(static_cast<const T *>(a.dy) + (int64_t)__builtin_amdgcn_readlane(token, i + k) * a.dy_stride,
                           c, a.cols);
            if (a.accumulate && ends >> (i + k) & 1)
                old[k] = load8(row_of<G>(a, __builtin_amdgcn_readlane(row, i + k)), c, a.cols);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (i + k >= end || c >= a.cols) continue;
            s += widen<T>(r[k]);
            if (!(ends >> (i + k) & 1)) continue;
            if (!inner || (out_long && i + k >= tail)) {
                store8(ws.part + (j * 2 + inner) * a.cols, c, a.cols, s);
            } else {
                s *= a.scale;
                if (a.accumulate) s += widen<G>(old[k]);
                store8(row_of<G>(a, __builtin_amdgcn_readlane(row, i + k)), c, a.cols, round_to<G>(s));
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
template <class G>
__global__ __launch_bounds__(256) void k_embed_join(EmbedGradArgs a, EmbedSpace ws) {
    __shared__ F8 lds[3][kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int64_t tiles = (a.cols + kTile - 1) / kTile, n = ws.runs[0].x * tiles;
    for (int64_t id = blockIdx.x; id < n; id += gridDim.x) {
        const int4 run = ws.runs[1 + id / tiles];
        const int64_t j = run.y;
        const int c = (int)(id % tiles) * kTile + lane * kVec;
        G *out = row_of<G>(a, run.x);
        F8 s = 0.0f;
        V8<G> old = G(0);
        if (c < a.cols) {
            if (wave == 0) {
                s = load8(ws.part + (j * 2 + 1) * a.cols, c, a.cols);
                if (a.accumulate) old = load8(out, c, a.cols);
            }
#pragma unroll 8
            for (int64_t k = j + 1 + wave; k <= run.z; k += 4) s += load8(ws.part + k * 2 * a.cols, c, a.cols);
        }
        if (wave) lds[wave - 1][lane] = s;
        __syncthreads();
        if (!wave && c < a.cols) {
            for (int w = 0; w < 3; ++w) s += lds[w][lane];
            s *= a.scale;
            if (a.accumulate) s += widen<G>(old);
            store8(out, c, a.cols, round_to<G>(s));
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
    const int64_t chunks = (a.rows + chunk - 1) / chunk, tiles = tiles_of(a.cols);
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
    if (joins > 0) e = launch(k_embed_join<G>, dim3((unsigned)(joins < 2048 ? joins : 2048)), dim3(256), s, a, ws);
    return e;
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
