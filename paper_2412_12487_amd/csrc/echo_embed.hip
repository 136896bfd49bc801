// echo_embed.hip -- embedding lookup and the table's gradient by sorted tokens on gfx950.
#include "echo_ops_device.h"

namespace echo {
namespace {

// A wavefront copies K pieces of every lane of one token's row, all on their way at once.  Memory bounds it: 16384 x
// 8192 of bf16 from an eighth of the table in 53.5 us, 5.9 TB/s.
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
// Latency bounds it: 512 tokens over 512 workgroups take 4.1 us, 16384 over 128 workgroups 14.9 us.  Many tokens and a large
// table together are bound by the workgroups all reading every id: 2^20 tokens over 4096 workgroups some 5 ms.
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
// share costs no more than many ids.  Memory
// bounds it: 16384 x 12288 of bf16 into 6400 rows in 86.1 us, 5.6 TB/s.  The wavefronts after those write zeros to the rows that no token names
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

}  // namespace

int64_t embed_grad_bytes(int64_t rows, int64_t cols, int64_t vocab) {
    if (!rows) return 0;
    const int chunk = embed_chunk(rows, cols);
    return round16(((int64_t(kWave) << sort_bits(vocab)) + 1) * 4) + 2 * round16(rows * 4) +
           ((rows + chunk - 1) / chunk + 1) * 16 + (rows + chunk - 1) / chunk * 2 * cols * 4;
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

}  // namespace echo
