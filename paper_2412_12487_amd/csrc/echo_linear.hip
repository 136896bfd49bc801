// echo_linear.hip -- losses taken straight from hidden states and the output table, on gfx950: the logits' tiles with
// their statistics or their gradient, and what prepares and joins them.
#include "echo_linear.h"

namespace echo {
namespace {

// A row's place in the loss: whether it is trained on, and with one target a row its column here or -1.
struct Row {
    bool trained;
    int at;
};
__device__ __forceinline__ Row row_of(const HeadArgs &a, int64_t target) {
    const bool trained = target >= 0 && target < a.vocab_size;
    return Row{trained, trained ? shard_row(target, a.vocab_start, a.vocab) : -1};
}

// The teacher's entries of a tile: a cell of 16 bits for each of its logits, 0 or the entry's number and one more.  Cells of
// 4 columns side by side are exchanged within a row, so that a wavefront's 16 rows meet different banks.
template <class S>
struct Cells {
    static constexpr int PITCH = S::TI * 2, ROWS = S::BYTES / PITCH < S::TJ ? S::BYTES / PITCH : S::TJ, MASK = S::TI / 16 - 1;
    static_assert(2 * ROWS >= S::TJ, "two buffers hold the cells");
    char *t0, *t1;
    __device__ __forceinline__ char *cell(int j, int i) const {
        char *t = j < ROWS ? t0 : t1;
        return t + (j < ROWS ? j : j - ROWS) * PITCH + (((i / 4) ^ ((j & MASK) << 2)) * 8);
    }
    // every entry of the rows j0 .. j0 + TJ - 1 whose column is in i0 .. i0 + TI - 1
    __device__ __forceinline__ void fill(const HeadArgs &a, int i0, int j0) const {
        __syncthreads();      // the last step has been read
        typedef __attribute__((ext_vector_type(4))) int I4;
        for (int c = threadIdx.x * 16; c < ROWS * PITCH; c += S::THREADS * 16) {
            *reinterpret_cast<I4 *>(t0 + c) = 0;
            if (ROWS < S::TJ) *reinterpret_cast<I4 *>(t1 + c) = 0;
        }
        __syncthreads();
        const int rows = a.rows - j0 < S::TJ ? a.rows - j0 : S::TJ, n = rows * a.top;
        const int *local = a.local + (int64_t)j0 * a.top;
        // eight loads on their way: one at a time, the logits of 512 x 1024 with 32 entries a row took 91 us and not 86
        constexpr int AT_ONCE = 8;
        for (int e0 = threadIdx.x; e0 < n; e0 += AT_ONCE * S::THREADS) {
            int column[AT_ONCE];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) column[k] = local[e0 + k * S::THREADS < n ? e0 + k * S::THREADS : n - 1];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const int e = e0 + k * S::THREADS;
                const unsigned i = (unsigned)(column[k] - i0);       // -1 where there is none
                if (e < n && i < (unsigned)S::TI && column[k] >= 0) {
                    const int j = e / a.top;
                    *reinterpret_cast<unsigned short *>(cell(j, i) + (i % 4) * 2) = (unsigned short)(e - j * a.top + 1);
                }
            }
        }
        __syncthreads();
    }
};

// The largest finite |grad_loss| of the rows that are trained on, or 1 where there is none above 0: what the gradient's shares are
// relative to, so that rows of one weight have it exactly.  What stands in other rows, infinities among it, is not their concern.
template <int THREADS, class Trained>
__device__ __forceinline__ float largest_of(const float *grad_loss, int rows, Trained trained) {
    float top = 0.0f;
#pragma unroll 4
    for (int n = threadIdx.x; n < rows; n += THREADS) {      // without branches, so that four rows are on their way
        const float g = fabsf(grad_loss[n]);
        top = fmaxf(top, (trained(n) & (g < kInf)) ? g : 0.0f);
    }
    return top;
}
template <int THREADS>
__device__ __forceinline__ void write_scale(float top, float *scale, float *lds) {
    top = wave_max(top);
    if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = top;
    __syncthreads();
    if (threadIdx.x) return;
    for (int w = 1; w < THREADS / kWave; ++w) top = fmaxf(top, lds[w]);
    *scale = top > 0.0f ? top : 1.0f;
}
template <int THREADS, class I>
__device__ __forceinline__ float largest_of(const float *grad_loss, int rows, const void *targets, int64_t vocab_size) {
    return largest_of<THREADS>(grad_loss, rows, [=](int n) ECHO_INLINE { return (uint64_t)id_at<I>(targets, n) < (uint64_t)vocab_size; });
}
// Once the teacher's entries are prepared.
template <int THREADS>
__device__ __forceinline__ void write_scale(const HeadArgs &a, float *lds) {
    const float2 *prior = a.prior;
    const float top = a.top          ? largest_of<THREADS>(a.grad_loss, a.rows, [=](int n) ECHO_INLINE { return prior[n].y > 0.0f; })
                      : a.wide_index ? largest_of<THREADS, int64_t>(a.grad_loss, a.rows, a.targets, a.vocab_size)
                                     : largest_of<THREADS, int32_t>(a.grad_loss, a.rows, a.targets, a.vocab_size);
    write_scale<THREADS>(top, a.scale_out, lds);
}

// Tiles of logits, i over the vocabulary and j over the rows.  2048 x 8192 over 49152 ids in wide tiles: 1.21 to 1.34 ms, 1230 to 1360
// TFLOP/s (a library product alone: 1340); the last rounding, maxima and exponentials of a tile take 13 us of a round's 205.
//   kLoss: each row's maximum and sum of exponentials over a wavefront's columns, and the logits of its target or entries.
//   kKeep: the same, and the exponentials, relative to that maximum.
//   kGrad: the gradient's share of each logit, (p - q) * grad_loss / scale, rounded to the elements' type.
enum { kLoss, kKeep, kGrad };
template <class T, class S, int MODE, int PLANES>
__global__ __launch_bounds__(S::THREADS, S::THREADS / 256) void k_logits(HeadArgs a) {
    __shared__ __attribute__((aligned(16))) char t0[S::BYTES];
    __shared__ __attribute__((aligned(16))) char t1[S::BYTES];
    if constexpr (MODE == kKeep)
        if ((int)blockIdx.x == a.m.tiles_i * a.m.tiles_j)
            return write_scale<S::THREADS>(a, reinterpret_cast<float *>(t0));
    const Place at = place_of(a.m, blockIdx.x);
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wi = wave / S::WJ, wj = wave % S::WJ;
    const int i0 = at.ti * S::TI, j0 = at.tj * S::TJ, il = wi * S::BI * 16 + (lane / 16) * 4, jl = wj * S::BJ * 16 + lane % 16;
    F4 acc[S::BI][S::BJ];
    multiply<T, true, true, S>(a.m, at, t0, t1, acc);
    // What a lane's rows need, all loads together; of rows past the end, the last one's.
    int64_t target[S::BJ];
    float2 whole_of[S::BJ];
    float grad_of[S::BJ], mass_of[S::BJ];
#pragma unroll
    for (int b = 0; b < S::BJ; ++b) {
        const int n = j0 + jl + b * 16 < a.rows ? j0 + jl + b * 16 : a.rows - 1;
        if (!a.top) target[b] = a.wide_index ? id_at<int64_t>(a.targets, n) : id_at<int32_t>(a.targets, n);
        if constexpr (MODE == kGrad) {
            whole_of[b] = a.whole ? a.whole[n] : make_float2(a.lse[n], 1.0f);
            grad_of[b] = a.grad_loss[n];
            if (a.top) mass_of[b] = a.prior[n].y;
        }
    }
    const Cells<S> cells{t0, t1};
    if (a.top) cells.fill(a, a.first + i0, j0);      // entries' columns count from the shard's first id
    using Quad = __attribute__((ext_vector_type(4))) unsigned short;
    // Everything per element counts here, 128 of them a lane.  Maxima are of the products, and exponentials 2^((D - top) k) with
    // k = log2(e) / T: distances between numbers of one size are exact, so that the maximum's own is 1 whatever the logits' size.
    // (2^(D k - top k) in one fused operation has the rounding of top k in its exponent: 0.06 at logits of 2^20, 4 at 2^27.)
    const float k2 = a.inv_t * kLog2e;
    if (i0 + S::TI > a.m.ni) {
#pragma unroll
        for (int k = 0; k < S::BI; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i0 + il + k * 16 + e >= a.m.ni)
#pragma unroll
                    for (int b = 0; b < S::BJ; ++b) acc[k][b][e] = -kInf;
    }
    if constexpr (MODE != kGrad) {
#pragma unroll
        for (int b = 0; b < S::BJ; ++b) {
            const int n = j0 + jl + b * 16;
            const bool live = n < a.rows;
            float top = -kInf;
#pragma unroll
            for (int k = 0; k < S::BI; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) top = fmaxf(top, acc[k][b][e]);
            if (!a.top) {
                const int hit = live ? row_of(a, target[b]).at - a.first - (i0 + il) : -1;      // below 0 where it is not here
                if (hit >= 0 && hit < S::BI * 16) {
#pragma unroll
                    for (int k = 0; k < S::BI; ++k)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (k * 16 + e == hit) a.hits[n] = acc[k][b][e];
                }
            } else {
#pragma unroll
                for (int k = 0; k < S::BI; ++k) {
                    const Quad entry = *reinterpret_cast<const Quad *>(cells.cell(jl + b * 16, il + k * 16));
                    if (!__builtin_bit_cast(int64_t, entry) || !live) continue;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (entry[e]) a.hits[(int64_t)n * a.top + entry[e] - 1] = acc[k][b][e];
                }
            }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float base = top == -kInf ? 0.0f : top;
            float sum = 0.0f;
#pragma unroll
            for (int k = 0; k < S::BI; ++k) {
                F4 d;
#pragma unroll
                for (int e = 0; e < 4; ++e) sum += d[e] = __builtin_amdgcn_exp2f((acc[k][b][e] - base) * k2);
                if constexpr (MODE == kKeep && sizeof(Kept<T, PLANES>) == 2) {
                    acc[k][b] = d;
                } else if constexpr (MODE == kKeep) {
                    using K = Kept<T, PLANES>;
                    const int v = i0 + il + k * 16;
                    if (live && v < a.prob_cols) {
                        typedef __attribute__((ext_vector_type(4))) K K4;
                        *reinterpret_cast<K4 *>(static_cast<K *>(a.kept) + n * a.kept_stride + v) =
                            __builtin_convertvector(d * kKeptUnit<T, PLANES>, K4);
                    }
                }
            }
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (live && lane < 16) a.stats[((int64_t)at.ti * S::WI + wi) * a.rows + n] = make_float2(top, sum);
        }
        if constexpr (MODE == kKeep && sizeof(Kept<T, PLANES>) == 2) {
            using K = Kept<T, PLANES>;
            const Outgoing<S, K> outgoing(t0, t1, wave, lane);
            __syncthreads();      // the last step and the cells have been read
#pragma unroll
            for (int b = 0; b < S::BJ; ++b)
#pragma unroll
                for (int k = 0; k < S::BI; ++k) outgoing.put(k, b, acc[k][b] * kKeptUnit<T, PLANES>);
            const int v = i0 + wi * S::BI * 16, n = j0 + wj * S::BJ * 16;
            outgoing.flush(static_cast<K *>(a.kept) + n * a.kept_stride + v, a.kept_stride, a.rows - n, a.prob_cols - v);
        }
    } else {
        // In a loss's own call probabilities are 2^((D - top) k) / sum, from a given lse exp(D / T - lse).
        const float scale = *a.scale, times = a.whole ? 1.0f : a.inv_t, k2_of = a.whole ? k2 : kLog2e;
#pragma unroll
        for (int b = 0; b < S::BJ; ++b) {
            const int n = j0 + jl + b * 16;
            bool live = n < a.rows;
            int hit = -1;
            float base = 0.0f, g = 0.0f, each = 0.0f;
            if (live) {
                const Row r = a.top ? Row{mass_of[b] > 0.0f, -1} : row_of(a, target[b]);
                hit = r.at - a.first;      // below 0 where it is not here
                base = whole_of[b].x;
                live = r.trained && (a.whole ? whole_of[b].y != 0.0f : base != -kInf);
                g = grad_of[b] / scale * kUnit<T>;
                each = g / whole_of[b].y;
            }
            if (PLANES > 1 && n >= a.prob_rows) continue;
            char *row = a.prob + n * a.prob_stride;
#pragma unroll
            for (int k = 0; k < S::BI; ++k) {
                const int i = il + k * 16, v = i0 + i;
                if (PLANES > 1 && v >= a.prob_cols) continue;
                F4 d = 0.0f;
                if (live) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) d[e] = __builtin_amdgcn_exp2f((scaled(acc[k][b][e], times) - base) * k2_of) * each;
                    if (!a.top) {
                        if ((unsigned)(hit - v) < 4u) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) d[e] -= v + e == hit ? g : 0.0f;
                        }
                    } else {
                        const Quad entry = *reinterpret_cast<const Quad *>(cells.cell(jl + b * 16, i));
                        if (__builtin_bit_cast(int64_t, entry)) {
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (entry[e]) d[e] -= a.q[(int64_t)n * a.top + entry[e] - 1] * g;
                        }
                    }
                    if (i0 + S::TI > a.m.ni) {      // past the vocabulary's end, where a logit of NaN would be one
#pragma unroll
                        for (int e = 0; e < 4; ++e) d[e] = v + e < a.m.ni ? d[e] : 0.0f;
                    }
                }
                if constexpr (PLANES == 1) {
                    acc[k][b] = d;
                    continue;
                }
                typedef __attribute__((ext_vector_type(4))) T T4;
#pragma unroll
                for (int plane = 0; plane < PLANES; ++plane) {
                    const T4 h = __builtin_convertvector(d, T4);
                    *reinterpret_cast<T4 *>(row + v * 2 + plane * a.prob_plane) = h;
                    if (plane + 1 < PLANES) d -= __builtin_convertvector(h, F4);
                }
            }
        }
        if constexpr (PLANES == 1) {
            const Outgoing<S, T> outgoing(t0, t1, wave, lane);
            __syncthreads();      // the last step and the cells have been read
#pragma unroll
            for (int b = 0; b < S::BJ; ++b)
#pragma unroll
                for (int k = 0; k < S::BI; ++k) outgoing.put(k, b, acc[k][b]);
            const int v = i0 + wi * S::BI * 16, n = j0 + wj * S::BJ * 16;
            outgoing.flush(reinterpret_cast<T *>(a.prob + n * a.prob_stride) + v, a.prob_stride / 2, a.prob_rows - n, a.prob_cols - v);
        }
    }
}

template <int N>
struct Count {
    static constexpr int value = N;
};

// A part of the sum of each logit, for products of few tiles: workgroups take parts of the hidden size.
template <class T, class S>
__global__ __launch_bounds__(S::THREADS, S::THREADS < 256 ? 1 : S::THREADS / 256) void k_parts(PartsArgs a) {
    __shared__ __attribute__((aligned(16))) char t0[S::BYTES];
    __shared__ __attribute__((aligned(16))) char t1[S::BYTES];
    if ((int)blockIdx.x == a.m.tiles_i * a.m.tiles_j * a.m.splits) {
        const TeacherIn &in = a.in;
        const float top = in.top ? largest_of<S::THREADS>(a.grad_loss, a.m.nj, [&](int n) ECHO_INLINE { return has_mass(in, n); })
                          : in.index_type == ECHO_I64 ? largest_of<S::THREADS, int64_t>(a.grad_loss, a.m.nj, in.ids, in.vocab_size)
                                                      : largest_of<S::THREADS, int32_t>(a.grad_loss, a.m.nj, in.ids, in.vocab_size);
        return write_scale<S::THREADS>(top, a.scale_out, reinterpret_cast<float *>(t0));
    }
    const Place at = place_of(a.m, blockIdx.x);
    F4 acc[S::BI][S::BJ];
    multiply<T, true, true, S>(a.m, at, t0, t1, acc);
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int i0 = at.ti * S::TI + wave / S::WJ * S::BI * 16 + (lane / 16) * 4, j0 = at.tj * S::TJ + wave % S::WJ * S::BJ * 16 + lane % 16;
#pragma unroll
    for (int b = 0; b < S::BJ; ++b)
#pragma unroll
        for (int k = 0; k < S::BI; ++k)
            if (j0 + b * 16 < a.m.nj && i0 + k * 16 < a.ld)
                *reinterpret_cast<F4 *>(a.parts + at.split * a.part + (int64_t)(j0 + b * 16) * a.ld + i0 + k * 16) = acc[k][b];
}

// A workgroup a row of logits in parts: they are summed and give the row's statistics and its loss.  With a gradient the sums
// take the first part's place, and a second pass gives its shares.
template <class T, int PLANES, int BLOCK>
__global__ __launch_bounds__(BLOCK) void k_rows(RowsArgs a) {
    constexpr int WAVES = BLOCK / kWave, STEP = BLOCK * 4;
    extern __shared__ __attribute__((aligned(16))) char space[];
    Entry *entries = reinterpret_cast<Entry *>(space);
    __shared__ float4 lds[WAVES];
    // what the lambdas use stands by itself: with the arguments captured whole they went to scratch memory, 30 us of
    // 500 x 4099 in place of 13
    const int n = blockIdx.x, splits = a.splits, ld = a.ld, vocab = a.vocab;
    const bool keeps = a.prob != nullptr;
    const int64_t part = a.part, plane_bytes = a.prob_plane;
    const float inv_t = a.in.inv_t, k2 = inv_t * kLog2e;
    char *prob = a.prob + n * a.prob_stride;
    const auto put = [&](int c, auto d) ECHO_INLINE {
        constexpr int N = sizeof(d) / 4;
#pragma unroll
        for (int plane = 0; plane < PLANES; ++plane) {
            const V<T, N> h = round_to<T, N>(d);
            *reinterpret_cast<V<T, N> *>(prob + c * 2 + plane * plane_bytes) = h;
            if (plane + 1 < PLANES) d -= widen<T, N>(h);
        }
    };
    if (n >= a.rows) {      // fills the last step of the table's gradient
        for (int c = threadIdx.x * 4; c < a.cols; c += STEP) put(c, F<4>(0.0f));
        return;
    }
    float *x = a.parts + (int64_t)n * a.ld;
    Teacher t{};
    int at = -1;
    if (!a.in.top) {
        const int64_t id = index_at(a.in.ids, a.in.index_type, n);
        t.trained = id >= 0 && id < a.in.vocab_size;
        at = t.trained ? shard_row(id, a.in.vocab_start, a.vocab) : -1;
    } else if (threadIdx.x < kWave) {
        t = teacher_of(a.in, n, 0, a.vocab, a.vocab, entries);
    }
    // G pieces of 4 columns together, P of their parts at a time: 16 loads are on their way
    const auto sum_parts = [&](int c, auto &d) ECHO_INLINE {
        constexpr int G = sizeof(d) / sizeof(F4), P = 16 / G;
#pragma unroll
        for (int g = 0; g < G; ++g) d[g] = 0.0f;
        for (int p0 = 0; p0 < splits; p0 += P) {
            F4 v[P][G];
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int g = 0; g < G; ++g) {      // no branch between them: past the end the last is read again
                    const int which = p0 + p < splits ? p0 + p : splits - 1, at = c + g * STEP < ld ? c + g * STEP : ld - 4;
                    v[p][g] = *reinterpret_cast<const F4 *>(x + (int64_t)which * part + at);
                }
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int g = 0; g < G; ++g)
                    if (p0 + p < splits) d[g] += v[p][g];
        }
#pragma unroll
        for (int g = 0; g < G; ++g)
            if (keeps && c + g * STEP < ld) *reinterpret_cast<F4 *>(x + c + g * STEP) = d[g];
    };
    // a logit's product after the pass
    const auto product = [&](int c) ECHO_INLINE {
        float d = x[c];
        if (keeps) return d;
#pragma unroll 8
        for (int p = 1; p < splits; ++p) d += x[p * part + c];
        return d;
    };
    // relative to products, as in the tiles
    const auto exp_from = [&](float d, float base) ECHO_INLINE { return __builtin_amdgcn_exp2f((d - base) * k2); };
    float top = -kInf, sum = 0.0f;
    const auto pass = [&](auto groups) ECHO_INLINE {
        constexpr int G = decltype(groups)::value;
        for (int c = threadIdx.x * 4; c < ld; c += G * STEP) {
            F4 d[G];
            sum_parts(c, d);
            float m = top;
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (c + g * STEP + e >= vocab) d[g][e] = -kInf;
                    m = fmaxf(m, d[g][e]);
                }
            const float base = m == -kInf ? 0.0f : m;
            sum *= top == -kInf ? 1.0f : exp_from(top, base);      // before a first finite logit the sum is 0, or NaN
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum += exp_from(d[g][e], base);
            top = m;
        }
    };
    if (a.ld <= STEP)
        pass(Count<1>{});
    else
        pass(Count<2>{});
    const float mine = top;
    top = wave_max(top);
    sum = wave_sum(mine == -kInf ? sum : sum * exp_from(mine, top));
    if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = make_float4(top, sum, t.trained ? 1.0f : 0.0f, 0.0f);
    __threadfence_block();
    __syncthreads();      // also: the row's logits are where its first part was
    const bool trained = lds[0].z > 0.0f;
    if (a.in.top && threadIdx.x < kWave) take_logits(entries, a.in.top, product);
    float lse;
    if (a.lse_in) {
        lse = a.lse_in[n];
    } else {
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, lds[w].x);
        sum = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float4 p = lds[w];
            sum += p.x == -kInf ? p.y : p.y * exp_from(p.x, top);
        }
        if (sum != sum) top = sum;      // a row of NaN alone has no maximum but a sum
        const float more = logf(sum);
        lse = top == -kInf ? -kInf : top * inv_t + more;
        if (threadIdx.x < kWave) {
            // the loss takes logits from their maximum on, the target as they are
            const auto sum_from = [&](float from) ECHO_INLINE {
                return (a.in.top ? cross_of(entries, a.in.top, from) : at >= 0 ? product(at) - from : 0.0f) * inv_t;
            };
            const float cross = a.loss ? sum_from(lse != -kInf ? top : 0.0f) : 0.0f, target = a.target ? sum_from(0.0f) : 0.0f;
            if (threadIdx.x == 0) {
                if (a.lse) a.lse[n] = lse;
                if (a.target) a.target[n] = target;
                if (a.entropy) a.entropy[n] = -t.prior;
                if (a.loss) a.loss[n] = !trained ? 0.0f : lse == -kInf ? kInf : a.square * (t.prior - cross + more);
            }
        }
    }
    if (!a.prob) return;
    // Probabilities of a loss's own call are 2^((D - top) k) / sum, of a given lse exp(x - lse): the lse of 32 bits would make them off by
    // its own rounding, 0.03 at logits of 2^20.
    const bool given = a.lse_in, live = trained && (given ? lse != -kInf : sum != 0.0f);
    const float g = live ? a.grad_loss[n] / *a.scale * kUnit<T> : 0.0f;
    const float times = given ? inv_t : 1.0f, base = given ? lse : top, k = given ? kLog2e : k2, part_of_sum = given ? 1.0f : 1.0f / sum;
    const auto share = [&](float d) ECHO_INLINE { return __builtin_amdgcn_exp2f((scaled(d, times) - base) * k) * part_of_sum; };
#pragma unroll 4
    for (int c = threadIdx.x * 4; c < a.cols; c += STEP) {
        F<4> d = 0.0f;
        if (live) {
            const F4 f = *reinterpret_cast<const F4 *>(x + c);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float p = share(f[e]) - (c + e == at ? 1.0f : 0.0f);
                d[e] = c + e < a.vocab ? p * g : 0.0f;
            }
        }
        put(c, d);
    }
    if (!a.in.top || !live) return;
    __threadfence_block();
    __syncthreads();      // what the entries are written over has arrived
    if (threadIdx.x >= kWave) return;
    for (int k = threadIdx.x; k < a.in.top; k += kWave) {
        const Entry e = entries[k];
        if (e.at >= 0) put(e.at, F<1>((share(e.x) - e.mass) * g));
    }
}

// The gradient's shares from the exponentials that the loss's pass kept, in place where they are of 16 bits; where the target
// is or the teacher has a mass, from the logit itself.  A workgroup takes a stretch of one row.
// Memory bounds it: 2048 x 51200 of bfloat16 in 70 us, 6.0 TB/s, where the logits' second product would take 1.4 ms at hidden
// size 8192 (19 us and 80 us for 512 rows at 1024).
constexpr int kSpan = 256 * 8 * 2;
template <class T, int PLANES>
__global__ __launch_bounds__(256) void k_shares(ShareArgs a) {
    using K = Kept<T, PLANES>;
    const int spans = (a.cols + kSpan - 1) / kSpan;
    const float most = *a.scale, k2 = a.inv_t * kLog2e;
    for (int64_t id = blockIdx.x; id < (int64_t)a.prob_rows * spans; id += gridDim.x) {
        const int n = (int)(id / spans), from = (int)(id - (int64_t)n * spans) * kSpan;
        bool live = n < a.rows;
        float2 row = make_float2(0.0f, 1.0f);      // largest product and sum of exponentials
        float g = 0.0f;
        int hit = -1;
        if (live) {
            row = a.whole[n];
            g = a.grad_loss[n] / most * kUnit<T>;
            bool trained;
            if (a.top) {
                trained = a.prior[n].y > 0.0f;
            } else {
                const int64_t t = a.wide_index ? id_at<int64_t>(a.targets, n) : id_at<int32_t>(a.targets, n);
                trained = t >= 0 && t < a.vocab_size;
                hit = trained ? shard_row(t, a.vocab_start, a.vocab) : -1;
            }
            live = trained && row.y != 0.0f;      // a row of NaN has a sum of NaN
        }
        const auto share = [&](float product) ECHO_INLINE { return __builtin_amdgcn_exp2f((product - row.x) * k2) / row.y; };
        const auto put = [&](int c, auto d) ECHO_INLINE {
            constexpr int N = sizeof(d) / 4;
            char *out = a.prob + n * a.prob_stride + c * 2;
#pragma unroll
            for (int plane = 0; plane < PLANES; ++plane) {
                const V<T, N> h = round_to<T, N>(d);
                *reinterpret_cast<V<T, N> *>(out + plane * a.prob_plane) = h;
                if (plane + 1 < PLANES) d -= widen<T, N>(h);
            }
        };
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int c = from + (k * 256 + threadIdx.x) * 8;
            if (c >= a.cols) continue;
            F<8> d = 0.0f;
            if (live) {
                const int part = c < a.split ? c / a.part0 : a.split / a.part0 + (c - a.split) / a.part1;
                const float top = a.stats[(int64_t)part * a.rows + n].x;
                d = widen<K, 8>(*reinterpret_cast<const V<K, 8> *>(static_cast<const K *>(a.kept) + (int64_t)n * a.cols + c)) *
                    (share(top) * g / kKeptUnit<T, PLANES>);
                if ((unsigned)(hit - c) < 8u) {
                    const float p = (share(a.hits[n]) - 1.0f) * g;
#pragma unroll
                    for (int j = 0; j < 8; ++j) d[j] = c + j == hit ? p : d[j];
                }
            }
            put(c, d);
        }
        if (!a.top) continue;
        __threadfence_block();
        __syncthreads();      // what the entries are written over has arrived
        if (!live) continue;
        for (int k = threadIdx.x; k < a.top; k += 256) {
            const int64_t e = (int64_t)n * a.top + k;
            const int c = a.local[e];
            if ((unsigned)(c - from) < (unsigned)kSpan && c >= 0) put(c, F<1>((share(a.hits[e]) - a.q[e]) * g));
        }
    }
}

// Joins the parts' statistics of 16 rows: lanes of 16 over the rows, 64 over the parts.
__global__ __launch_bounds__(1024) void k_join(JoinArgs a) {
    __shared__ float2 part[64][17];
    const int r = threadIdx.x % 16, w = threadIdx.x / 16;
    const int n = blockIdx.x * 16 + r;
    // maxima and hits are of the products
    const float inv_t = a.inv_t, k2 = inv_t * kLog2e;
    const auto moved = [&](float2 p, float to) ECHO_INLINE { return p.x == -kInf ? p.y : p.y * __builtin_amdgcn_exp2f((p.x - to) * k2); };      // p.y is 0 there, or NaN
    float top = -kInf, sum = 0.0f;
    if (n < a.rows) {
#pragma unroll 4
        for (int t = w; t < a.parts; t += 64) {
            const float2 p = a.stats[(int64_t)t * a.rows + n];
            const float m = fmaxf(top, p.x);
            sum = moved(make_float2(top, sum), m) + moved(p, m);
            top = m;
        }
    }
    part[w][r] = make_float2(top, sum);
    for (int by = 32; by; by /= 2) {
        __syncthreads();
        if (w < by) {
            const float2 p = part[w][r], o = part[w + by][r];
            const float m = fmaxf(p.x, o.x);
            part[w][r] = make_float2(m, moved(p, m) + moved(o, m));
        }
    }
    __syncthreads();
    top = part[0][r].x;
    sum = part[0][r].y;
    float cross = 0.0f, target = 0.0f;
    if (a.top) {
        // the loss takes logits from their maximum on, the target as they are
        const float from = top != -kInf && sum == sum ? top : 0.0f;
        if (n < a.rows) {
            for (int k = w; k < a.top; k += 64) {
                const int64_t e = (int64_t)n * a.top + k;
                if (a.local[e] < 0) continue;
                const float q = a.q[e], x = a.hits[e];
                cross += q * ((x - from) * inv_t);
                target += q * (x * inv_t);
            }
        }
        for (int by = 32; by; by /= 2) {
            __syncthreads();
            part[w][r] = make_float2(cross, target);
            __syncthreads();
            if (w < by) {
                const float2 o = part[w + by][r];
                cross += o.x;
                target += o.y;
            }
        }
    }
    if (w || n >= a.rows) return;
    if (sum != sum) top = sum;      // a row of NaN alone has no maximum but a sum
    const float more = logf(sum), lse = top == -kInf ? -kInf : top * inv_t + more;
    if (a.lse) a.lse[n] = lse;
    if (a.whole) a.whole[n] = make_float2(top, sum);
    if (!a.top) {
        const int64_t t = a.wide_index ? id_at<int64_t>(a.targets, n) : id_at<int32_t>(a.targets, n);
        const bool trained = t >= 0 && t < a.vocab_size;
        const float hit = trained && shard_row(t, a.vocab_start, a.vocab) >= 0 ? a.hits[n] : 0.0f;
        if (a.target) a.target[n] = hit * inv_t;
        if (a.loss) a.loss[n] = !trained ? 0.0f : lse == -kInf ? kInf : (top - hit) * inv_t + more;
        return;
    }
    const float2 prior = a.prior[n];
    const bool trained = prior.y > 0.0f;
    if (a.target) a.target[n] = target;
    if (a.entropy) a.entropy[n] = -prior.x;
    if (a.loss) a.loss[n] = !trained ? 0.0f : lse == -kInf ? kInf : a.square * (prior.x - cross + more);
}

// The teacher's entries of every row, a wavefront a row.
__global__ __launch_bounds__(256) void k_teacher(TeacherArgs a) {
    extern __shared__ __attribute__((aligned(16))) char space[];
    const int lane = threadIdx.x % kWave;
    Entry *entries = reinterpret_cast<Entry *>(space) + threadIdx.x / kWave * a.in.top;
    for (int64_t n = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave; n < a.rows; n += (int64_t)gridDim.x * 4) {
        const Teacher t = teacher_of(a.in, n, 0, a.vocab, a.vocab, entries);
        for (int k = lane; k < a.in.top; k += kWave) {
            a.local[n * a.in.top + k] = entries[k].at;
            a.q[n * a.in.top + k] = entries[k].mass;
        }
        if (lane == 0) a.prior[n] = make_float2(t.prior, t.trained ? 1.0f : 0.0f);
    }
}

// For a gradient whose loss was another call's; else the loss's launch has a workgroup for it.
__global__ __launch_bounds__(1024) void k_scale(HeadArgs a) {
    __shared__ float lds[16];
    write_scale<1024>(a, lds);
}

// Rows laid out for the products: PLANES planes of 16 bits, rows filled up with zeros to whole steps.  One launch for both
// matrices; the second may have no rows.
template <class U, class T, int PLANES>
__global__ __launch_bounds__(256) void k_layout(LayoutArgs one, LayoutArgs two) {
    const int pieces = one.width / 8;
    const int64_t all = (one.rows + two.rows) * pieces;
    for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < all; id += (int64_t)gridDim.x * 256) {
        int64_t row = id / pieces;
        const int c = (int)(id - row * pieces) * 8;
        const bool second = row >= one.rows;
        const LayoutArgs &a = second ? two : one;
        if (second) row -= one.rows;
        F<8> f = widen<U, 8>(load<8>(static_cast<const U *>(a.from) + row * a.stride, c, a.cols));
#pragma unroll
        for (int plane = 0; plane < PLANES; ++plane) {
            const V<T, 8> h = round_to<T, 8>(f);
            *reinterpret_cast<H8<T> *>(a.to + plane * a.plane + (row * a.width + c) * 2) = __builtin_bit_cast(H8<T>, h);
            if (plane + 1 < PLANES) f -= widen<T, 8>(h);
        }
    }
}

template <class T, int MODE, int PLANES>
hipError_t logits(const HeadArgs &a, int shape, hipStream_t s) {
    const dim3 grid(a.m.tiles_i * a.m.tiles_j + (a.scale_out ? 1 : 0));
    switch (shape) {
        case 0: return launch(k_logits<T, Wide, MODE, PLANES>, grid, dim3(Wide::THREADS), s, a);
        case 1: return launch(k_logits<T, Middle, MODE, PLANES>, grid, dim3(Middle::THREADS), s, a);
        default: return launch(k_logits<T, Thin, MODE, PLANES>, grid, dim3(Thin::THREADS), s, a);
    }
}
template <class T, int PLANES>
hipError_t logits(const HeadArgs &a, int mode, int shape, hipStream_t s) {
    return mode == kGrad ? logits<T, kGrad, PLANES>(a, shape, s)
                         : mode == kKeep ? logits<T, kKeep, PLANES>(a, shape, s) : logits<T, kLoss, 1>(a, shape, s);
}
template <class T>
hipError_t parts(const PartsArgs &a, int shape, hipStream_t s) {
    const dim3 grid(a.m.tiles_i * a.m.tiles_j * a.m.splits + (a.scale_out ? 1 : 0));
    if (shape == 1) return launch(k_parts<T, Middle>, grid, dim3(Middle::THREADS), s, a);
    return launch(k_parts<T, Thin>, grid, dim3(Thin::THREADS), s, a);
}
hipError_t launch_parts(const PartsArgs &a, int type, int shape, hipStream_t s) {
    return type == ECHO_F16 ? parts<f16>(a, shape, s) : parts<bf16>(a, shape, s);
}
template <class T, int PLANES>
hipError_t rows(const RowsArgs &a, hipStream_t s) {
    void *args[] = {const_cast<RowsArgs *>(&a)};
    // 3 rows of 9024 in 14 parts take 19 us with 512 lanes a row and 13 with 1024; 4 rows of 4352 7.5 and 8.5
    const int block = a.ld <= 1024 ? 256 : a.ld <= (a.rows <= 128 ? 8192 : 16384) ? 512 : 1024;
    const void *kernel = block == 256   ? reinterpret_cast<const void *>(k_rows<T, PLANES, 256>)
                         : block == 512 ? reinterpret_cast<const void *>(k_rows<T, PLANES, 512>)
                                        : reinterpret_cast<const void *>(k_rows<T, PLANES, 1024>);
    return hipLaunchKernel(kernel, dim3(a.prob ? a.prob_rows : a.rows), dim3(block), args, sizeof(Entry) * a.in.top, s);
}
hipError_t launch_rows(const RowsArgs &a, int type, int planes, hipStream_t s) {
    if (type == ECHO_F16) return planes == 2 ? rows<f16, 2>(a, s) : rows<f16, 1>(a, s);
    return planes == 3 ? rows<bf16, 3>(a, s) : planes == 2 ? rows<bf16, 2>(a, s) : rows<bf16, 1>(a, s);
}
hipError_t launch_join(const JoinArgs &a, hipStream_t s) { return launch(k_join, dim3((a.rows + 15) / 16), dim3(1024), s, a); }
hipError_t launch_teacher(const TeacherArgs &a, hipStream_t s) {
    void *args[] = {const_cast<TeacherArgs *>(&a)};
    return hipLaunchKernel(reinterpret_cast<const void *>(k_teacher), dim3(grid_of((a.rows + 3) / 4)), dim3(256), args,
                           4 * sizeof(Entry) * a.in.top, s);
}
hipError_t launch_scale(const HeadArgs &a, hipStream_t s) {
    return launch(k_scale, dim3(1), dim3(1024), s, a);
}
hipError_t launch_layout(const LayoutArgs &a, const LayoutArgs &b, int type, hipStream_t s) {
    const dim3 grid(grid_of(((a.rows + b.rows) * (a.width / 8) + 255) / 256));
    switch (type) {
        case ECHO_F32: return launch(k_layout<float, bf16, 3>, grid, dim3(256), s, a, b);
        case ECHO_F16: return launch(k_layout<f16, f16, 1>, grid, dim3(256), s, a, b);
        default: return launch(k_layout<bf16, bf16, 1>, grid, dim3(256), s, a, b);
    }
}

hipError_t launch_shares(const ShareArgs &a, int type, hipStream_t s) {
    const dim3 grid(grid_of((int64_t)a.prob_rows * ((a.cols + kSpan - 1) / kSpan)));
    switch (type) {
        case ECHO_F32: return launch(k_shares<bf16, 3>, grid, dim3(256), s, a);
        case ECHO_F16: return launch(k_shares<f16, 1>, grid, dim3(256), s, a);
        default: return launch(k_shares<bf16, 1>, grid, dim3(256), s, a);
    }
}

constexpr int64_t kProbBytes = int64_t(1) << 30;      // of the logits' gradient at a time
constexpr int64_t kProbCols = int64_t(1) << 21;
int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
int tiles(int64_t n, int t) { return (int)((n + t - 1) / t); }

// Shapes of a product's tiles along one of its sides: `shape0` up to `split`, `shape1` from there on.
//
// Wide tiles do the most work for what they read, one on a compute unit at a time; where they leave the launch's last round
// mostly empty, what is left of the side after the full rounds takes middle ones, two on a compute unit.  A round of 256
// wide tiles of logits takes 19, 36 and 205 us for sums of 256, 1024 and 8192; one of 512 middle tiles, half the work, 12, 23 and 123 us, and up
// to 256 of them 11, 18 and 84 us: hence the costs, in units of a wide round.  Thin tiles (logits alone) are for up to 64 rows.
struct Ranges {
    int split, shape0, shape1;
};
int side(int shape) { return shape == 1 ? 128 : 256; }
double middle_cost(int64_t n, int64_t other) {
    const int64_t t = (int64_t)tiles(n, 128) * tiles(other, 128), rest = t % 512;
    return (double)(t / 512) * 0.62 + (rest > 256 ? 0.62 : rest ? 0.42 : 0.0);
}
Ranges ranges_of(int64_t n, int64_t other) {
    const int64_t across = tiles(other, 256), along = tiles(n, 256);
    const double wide = (double)((along * across + 255) / 256), middle = middle_cost(n, other);
    const int64_t whole = along * across / 256 * 256 / across;      // tiles along the side in full rounds
    const double mixed = whole > 0 && whole < along
                             ? (double)((whole * across + 255) / 256) + middle_cost(n - whole * 256, other) + 0.05
                             : wide + middle;
    if (middle < wide && middle <= mixed) return Ranges{(int)n, 1, 1};
    return mixed < wide ? Ranges{(int)whole * 256, 0, 1} : Ranges{(int)n, 0, 0};
}
// Parts of the sum that middle tiles take where they leave compute units idle: behind full rounds of wide ones (256 x 8192 of the
// table's gradient, 128 tiles, over 16384 rows: 217 us whole and 103 in parts), or by themselves (224 x 1346 of it over 7320 rows of
// 32 bits, 22 tiles of 690 steps, took 550 us whole).
int tail_splits(int64_t n, int64_t other, int64_t steps) {
    const int64_t t = (int64_t)tiles(n, 128) * tiles(other, 128);
    int64_t splits = 512 / t;
    if (splits > steps / 16) splits = steps / 16;
    return splits > 32 ? 32 : splits < 1 ? 1 : (int)splits;
}
int64_t tail_bytes(const Ranges &r, int64_t n, int64_t other, int64_t steps) {
    const int64_t middle = n - (r.shape0 == 1 ? 0 : r.split);
    const int splits = middle > 0 ? tail_splits(middle, other, steps) : 1;
    return splits > 1 ? splits * middle * other * 4 : 0;
}
Ranges logits_ranges(int64_t n, int64_t rows) { return rows <= 64 ? Ranges{(int)n, 2, 2} : ranges_of(n, rows); }
// Columns of a part of the logits' statistics: what one wavefront of a tile has.
int part_of(int shape) { return shape == 0 ? Wide::TI / Wide::WI : shape == 1 ? Middle::TI / Middle::WI : Thin::TI / Thin::WI; }
int parts_of(int n, int shape) { return shape == 1 ? tiles(n, 128) * Middle::WI : tiles(n, 256) * (shape ? Thin::WI : Wide::WI); }
void tile(Product &m, int ni, int nj, int shape) {
    m.tiles_i = tiles(ni, side(shape));
    m.tiles_j = tiles(nj, shape == 2 ? 64 : side(shape));
}

// Sizes of a call's products, and where its workspace has what.
struct Plan {
    int planes, pairs;             // of the logits' products
    int share_planes, share_pairs; // of the gradients'
    int width;                     // hidden size in whole steps
    bool copy_hidden, copy_weight;
    Ranges logits;                 // the loss's
    int stats_parts;
    bool few;                      // few tiles of logits: their sum is split, and rows are worked on by themselves
    int few_shape, few_splits;
    bool keep;                     // the loss's pass keeps its exponentials for the gradient
    int64_t prob_rows, prob_cols, pieces;
    Ranges out;                    // the hidden states' gradient
    int splits;
    bool parts;
    int64_t hidden, weight, stats, whole, hits, local, q, prior, scale, prob, kept, part, sums, tail, bytes;
};
bool direct(const void *p, int64_t stride, int type, int cols) {
    return type != ECHO_F32 && cols % kDepth == 0 && stride % 8 == 0 && stride <= int64_t(1) << 22 && (uintptr_t)p % 16 == 0;
}
Plan plan_of(const LinearArgs &a) {
    Plan p{};
    p.planes = a.type == ECHO_F32 ? 3 : 1;
    p.pairs = a.type == ECHO_F32 ? 6 : 1;
    p.width = (int)up(a.cols, kDepth);
    p.copy_hidden = !direct(a.hidden, a.hidden_stride, a.type, a.cols);
    p.copy_weight = !direct(a.weight, a.weight_stride, a.type, a.cols);
    const auto take = [&](int64_t n) {
        const int64_t at = p.bytes;
        p.bytes += up(n, 256);
        return at;
    };
    if (p.copy_hidden) p.hidden = take(a.rows * p.width * 2 * p.planes);
    if (p.copy_weight) p.weight = take((int64_t)a.vocab * p.width * 2 * p.planes);
    p.few = false;
    if (a.rows * up(a.vocab, kDepth) * 2 * p.planes <= kProbBytes) {
        // Up to a workgroup a compute unit: a step takes such a launch 0.6 us whatever its tiles; parts of at least 8 steps, two
        // workgroups a compute unit at most.  Long rows want long sums, since one workgroup reads a row again: one row of
        // 1024 over 51200 ids takes 29 us with tiles alone and 32 so.
        const int shape = a.rows <= 64 ? 2 : 1;
        Product m{};
        tile(m, a.vocab, (int)a.rows, shape);
        const int64_t wg = (int64_t)m.tiles_i * m.tiles_j, steps = (int64_t)(p.width / kDepth) * p.pairs;
        if (wg <= 256 && (a.vocab <= 16384 || steps >= 32)) {
            int64_t splits = 512 / wg;
            if (splits > steps / 8) splits = steps / 8;
            if (splits > 32) splits = 32;
            p.few = true;
            p.few_shape = shape;
            p.few_splits = splits < 1 ? 1 : (int)splits;
            p.sums = take(p.few_splits * a.rows * up(a.vocab, kDepth) * 4);
        }
    }
    if (a.top && !p.few) {
        p.local = take(a.rows * a.top * 4);
        p.q = take(a.rows * a.top * 4);
        p.prior = take(a.rows * 8);
    }
    if (a.forward && !p.few) {
        p.logits = logits_ranges(a.vocab, a.rows);
        p.stats_parts = parts_of(p.logits.split, p.logits.shape0);
        if (p.logits.split < a.vocab) p.stats_parts += parts_of(a.vocab - p.logits.split, p.logits.shape1);
        p.stats = take(p.stats_parts * a.rows * 8);
        p.hits = take(a.rows * (a.top ? a.top : 1) * 4);
    }
    if (a.grads) {
        p.scale = take(4);
        // Of few rows a single rounding of a share to 16 bits may be most of an output's error (two rows of half precision: 1.75
        // times the plain form's): they are held in two planes, at no cost that counts there.
        p.share_planes = a.type == ECHO_F32 ? 3 : p.few && a.rows <= 64 ? 2 : 1;
        p.share_pairs = a.type == ECHO_F32 ? 6 : p.share_planes;
        p.prob_rows = up(a.rows, kDepth);
        const int64_t whole = up(a.vocab, kDepth);
        int64_t most = kProbBytes / (p.prob_rows * 2 * p.share_planes) / 256 * 256;
        most = most < 256 ? 256 : most > kProbCols ? kProbCols : most;
        p.pieces = (whole + most - 1) / most;
        p.prob_cols = p.pieces == 1 ? whole : up((whole + p.pieces - 1) / p.pieces, 256);
        p.prob = take(p.prob_rows * p.prob_cols * 2 * p.share_planes);
        p.keep = a.forward && p.pieces == 1 && !p.few;
        if (a.forward && !p.few) p.whole = take(a.rows * 8);
        if (p.keep) p.kept = a.type == ECHO_BF16 ? p.prob : take(a.rows * p.prob_cols * 4);
        const int64_t middle = (int64_t)tiles(a.cols, 128) * tiles(a.rows, 128), steps = p.prob_cols / kDepth * p.share_pairs;
        p.out = ranges_of(a.rows, a.cols);
        // too few tiles to fill the GPU: workgroups take parts of the sum
        int64_t splits = middle < 512 ? 512 / middle : 1;
        if (splits > steps / 4) splits = steps / 4;
        if (splits > 64) splits = 64;
        p.splits = splits < 1 ? 1 : (int)splits;
        if (p.splits > 1) p.out = Ranges{(int)a.rows, 1, 1};
        p.parts = p.splits > 1 || p.pieces > 1;
        if (p.parts) p.part = take(p.splits * a.rows * a.cols * 4);
        // the last piece may be narrower than the others, and have another tail
        const int64_t last = a.vocab - (p.pieces - 1) * p.prob_cols, each = p.pieces > 1 ? p.prob_cols : last, sum = p.prob_rows / kDepth * p.share_pairs;
        int64_t tail = p.parts ? 0 : tail_bytes(p.out, a.rows, a.cols, steps);
        for (const int64_t n : {each, last}) {
            const int64_t b = tail_bytes(ranges_of(n, a.cols), n, a.cols, sum);
            tail = tail < b ? b : tail;
        }
        p.tail = take(tail);
    }
    return p;
}

}  // namespace

int64_t linear_bytes(const LinearArgs &a) { return plan_of(a).bytes; }

#define ECHO_HIP(call)                        \
    do {                                      \
        const hipError_t e_ = (call);         \
        if (e_ != hipSuccess) return e_;      \
    } while (0)

namespace {

// Logits of the columns from h.first on (h.m.a begins there): h.m.ni of them, and zeros of the gradient up to `cover`.
hipError_t run_logits(const HeadArgs &head, int type, int mode, int cover, const Ranges &r, hipStream_t s) {
    for (int from = 0, to; from < cover; from = to) {
        to = from || r.split >= head.m.ni ? cover : r.split;
        const int shape = from ? r.shape1 : r.shape0;
        HeadArgs h = head;
        h.m.a.p += from * h.m.a.stride;
        h.m.a.rows -= from;
        h.m.ni = (to < head.m.ni ? to : head.m.ni) - from;
        h.first += from;
        h.prob_cols = to - from;
        if (h.prob) h.prob += (int64_t)from * 2;
        if (h.kept) h.kept = static_cast<char *>(h.kept) + (int64_t)from * (type == ECHO_BF16 ? 2 : 4);
        if (from) h.scale_out = nullptr;
        if (from) h.stats += (int64_t)parts_of(from, r.shape0) * h.rows;
        tile(h.m, to - from, h.m.nj, shape);
        hipError_t e;
        switch (type) {
            case ECHO_F32: e = logits<bf16, 3>(h, mode, shape, s); break;
            case ECHO_F16: e = logits<f16, 1>(h, mode, shape, s); break;
            default: e = logits<bf16, 1>(h, mode, shape, s); break;
        }
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
// D of a product along j.
// Middle tiles take parts of a long sum, in `tail`, where they would leave compute units idle.
hipError_t run_out(const OutArgs &all, int type, int out_type, bool deep, const Ranges &r, float *tail, hipStream_t s) {
    const int64_t elem = out_type == ECHO_F32 ? 4 : 2;
    for (int from = 0, to; from < all.m.nj; from = to) {
        to = from ? all.m.nj : r.split;
        const int shape = from ? r.shape1 : r.shape0;
        OutArgs o = all;
        o.m.nj = to - from;
        o.m.b.p += deep ? from * o.m.b.stride : (int64_t)from * 2;
        if (deep)
            o.m.b.rows -= from;
        else
            o.m.b.width -= from;
        o.out = static_cast<char *>(o.out) + (int64_t)from * o.m.ni * elem;
        if (o.parts) o.parts += (int64_t)from * o.m.ni;
        const int splits = shape == 1 && !o.parts ? tail_splits(o.m.nj, o.m.ni, (int64_t)o.m.steps * o.m.pairs) : 1;
        if (splits > 1) {
            o.m.splits = splits;
            o.parts = tail;
            o.part = (int64_t)o.m.nj * o.m.ni;
            o.add_parts = false;
        }
        tile(o.m, o.m.ni, o.m.nj, shape);
        hipError_t e = launch_out(o, type, out_type, deep, shape, s);
        if (e == hipSuccess && splits > 1)
            e = launch_gather(GatherArgs{tail, o.part, splits, o.scale, o.factor, o.out, o.accumulate}, type, out_type, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_linear(const LinearArgs &a, hipStream_t s) {
    if (!a.rows) return launch_zero(a.dweight, (int64_t)a.vocab * a.cols * (a.grad_type == ECHO_F32 ? 4 : 2), s);
    const Plan p = plan_of(a);
    char *w = static_cast<char *>(a.workspace);
    const int64_t row_bytes = (int64_t)p.width * 2;
    Operand hidden{static_cast<const char *>(a.hidden), a.hidden_stride * 2, 0, a.rows, p.width},
        weight{static_cast<const char *>(a.weight), a.weight_stride * 2, 0, a.vocab, p.width};
    LayoutArgs laid[2] = {};
    int copies = 0;
    if (p.copy_weight) {
        weight = Operand{w + p.weight, row_bytes, a.vocab * row_bytes, a.vocab, p.width};
        laid[copies++] = LayoutArgs{a.weight, a.weight_stride, a.vocab, a.cols, p.width, w + p.weight, weight.plane};
    }
    if (p.copy_hidden) {
        hidden = Operand{w + p.hidden, row_bytes, a.rows * row_bytes, a.rows, p.width};
        laid[copies++] = LayoutArgs{a.hidden, a.hidden_stride, a.rows, a.cols, p.width, w + p.hidden, hidden.plane};
    }
    if (copies) ECHO_HIP(launch_layout(laid[0], laid[1], a.type, s));
    HeadArgs h{};
    h.rows = (int)a.rows;
    h.vocab = a.vocab;
    h.inv_t = 1.0f / a.temperature;
    h.targets = a.targets;
    h.wide_index = a.index_type == ECHO_I64;
    h.top = a.top;
    h.vocab_start = a.vocab_start;
    h.vocab_size = a.vocab_size;
    const TeacherIn in{a.targets, a.teacher, a.index_type, a.teacher_type, a.top, a.vocab_start, a.vocab_size, h.inv_t};
    if (a.top && !p.few) {
        const TeacherArgs t{in, a.rows, a.vocab, reinterpret_cast<int *>(w + p.local), reinterpret_cast<float *>(w + p.q),
                            reinterpret_cast<float2 *>(w + p.prior)};
        ECHO_HIP(launch_teacher(t, s));
        h.local = t.local;
        h.q = t.q;
        h.prior = t.prior;
    }
    h.m = Product{weight, hidden, a.vocab, (int)a.rows, 0, 0, p.width / kDepth, p.pairs, 1};
    if (a.grads) {
        h.scale = reinterpret_cast<float *>(w + p.scale);
        h.prob = w + p.prob;
        h.prob_stride = p.prob_cols * 2;
        h.prob_plane = p.prob_rows * h.prob_stride;
        h.prob_rows = (int)p.prob_rows;
        h.prob_cols = (int)p.prob_cols;
        h.grad_loss = a.grad_loss;
    }
    if (p.few) {
        PartsArgs c{};
        c.m = h.m;
        c.m.splits = p.few_splits;
        c.ld = (int)up(a.vocab, kDepth);
        c.parts = reinterpret_cast<float *>(w + p.sums);
        c.part = a.rows * c.ld;
        c.in = in;
        c.grad_loss = a.grad_loss;
        c.scale_out = a.grads ? reinterpret_cast<float *>(w + p.scale) : nullptr;
        tile(c.m, a.vocab, h.rows, p.few_shape);
        ECHO_HIP(launch_parts(c, a.type, p.few_shape, s));
        ECHO_HIP(launch_rows(RowsArgs{c.parts, c.part, p.few_splits, c.ld, h.rows, a.vocab, (int)p.prob_cols, in,
                                      a.temperature * a.temperature, a.lse, a.target, a.entropy, a.loss, a.forward ? nullptr : a.lse_in,
                                      a.grad_loss, h.scale, a.grads ? h.prob : nullptr, h.prob_stride, h.prob_plane, h.prob_rows},
                             a.type, p.share_planes, s));
    } else if (a.forward) {
        h.stats = reinterpret_cast<float2 *>(w + p.stats);
        h.hits = reinterpret_cast<float *>(w + p.hits);
        h.kept = p.keep ? w + p.kept : nullptr;
        h.kept_stride = p.prob_cols;
        h.scale_out = p.keep ? reinterpret_cast<float *>(w + p.scale) : nullptr;
        ECHO_HIP(run_logits(h, a.type, p.keep ? kKeep : kLoss, p.keep ? (int)p.prob_cols : a.vocab, p.logits, s));
        ECHO_HIP(launch_join(JoinArgs{h.stats, h.prior, h.hits, h.q, h.local, h.targets, h.wide_index, h.top, h.rows, h.vocab,
                                      p.stats_parts, h.vocab_start, h.vocab_size, h.inv_t, a.temperature * a.temperature, a.lse, a.target,
                                      a.entropy, a.loss, a.grads ? reinterpret_cast<float2 *>(w + p.whole) : nullptr}, s));
    }
    if (!a.grads) return hipSuccess;
    h.whole = a.forward && !p.few ? reinterpret_cast<float2 *>(w + p.whole) : nullptr;
    h.lse = a.lse_in;
    h.scale_out = reinterpret_cast<float *>(w + p.scale);
    if (!p.keep && !p.few) ECHO_HIP(launch_scale(h, s));
    h.scale_out = nullptr;
    const Operand prob{h.prob, h.prob_stride, h.prob_plane, p.prob_rows, (int)p.prob_cols};
    const int64_t grad_elem = a.grad_type == ECHO_F32 ? 4 : 2;
    float *parts = p.parts ? reinterpret_cast<float *>(w + p.part) : nullptr, *tail = reinterpret_cast<float *>(w + p.tail);
    for (int64_t piece = 0; piece < p.pieces; ++piece) {
        const int64_t first = piece * p.prob_cols, left = a.vocab - first;
        const int n = (int)(left < p.prob_cols ? left : p.prob_cols);
        Operand table = weight;
        table.p += first * weight.stride;
        table.rows = n;
        h.first = (int)first;
        h.m.a = table;
        h.m.ni = n;
        if (p.keep) {
            const ShareArgs c{h.stats, h.whole, h.prior, h.hits, h.q, h.grad_loss, h.scale, h.local, h.targets, w + p.kept, h.wide_index,
                              h.top, h.rows, h.vocab, (int)p.prob_cols, h.vocab_start, h.vocab_size, h.inv_t, p.logits.split,
                              part_of(p.logits.shape0), part_of(p.logits.shape1), h.prob, h.prob_stride, h.prob_plane, h.prob_rows};
            ECHO_HIP(launch_shares(c, a.type, s));
        } else if (!p.few) {
            ECHO_HIP(run_logits(h, a.type, kGrad, (int)p.prob_cols, logits_ranges(p.prob_cols, a.rows), s));
        }
        OutArgs o{};
        o.scale = h.scale;
        o.factor = a.temperature;
        o.m = Product{table, prob, a.cols, (int)a.rows, 0, 0, (int)(p.prob_cols / kDepth), p.share_pairs, p.splits};
        o.parts = parts;
        o.part = a.rows * a.cols;
        o.add_parts = piece > 0;
        o.out = a.dhidden;
        const Ranges table_out = ranges_of(n, a.cols);
        const bool both = p.out.split == a.rows && p.out.shape0 == 1 && table_out.split == n && table_out.shape0 == 1;
        OutArgs first_out = o;
        tile(first_out.m, a.cols, h.rows, 1);
        if (!both) ECHO_HIP(run_out(o, a.type, a.type, true, p.out, tail, s));
        o.m = Product{hidden, prob, a.cols, n, 0, 0, (int)(p.prob_rows / kDepth), p.share_pairs, 1};
        o.parts = nullptr;
        o.out = static_cast<char *>(a.dweight) + first * a.cols * grad_elem;
        o.accumulate = a.accumulate;
        if (both) {
            const int splits = tail_splits(n, a.cols, (int64_t)o.m.steps * o.m.pairs);
            tile(o.m, a.cols, n, 1);
            if (splits > 1) {
                o.m.splits = splits;
                o.parts = tail;
                o.part = (int64_t)n * a.cols;
                o.add_parts = false;
            }
            ECHO_HIP(launch_both(first_out, o, a.type, a.grad_type, s));
            if (splits > 1)
                ECHO_HIP(launch_gather(GatherArgs{tail, o.part, splits, o.scale, o.factor, o.out, o.accumulate}, a.type, a.grad_type, s));
        } else {
            ECHO_HIP(run_out(o, a.type, a.grad_type, false, table_out, tail, s));
        }
    }
    if (parts)
        ECHO_HIP(launch_gather(GatherArgs{parts, a.rows * a.cols, p.splits, h.scale, a.temperature, a.dhidden, false}, a.type, a.type, s));
    return hipSuccess;
}

}  // namespace echo
