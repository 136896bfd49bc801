// echo_product.h -- tiles of matrix products on the matrix cores of gfx950, for the output head's kernels.
//
//   D[j][i] = sum over k of A(i, k) B(j, k)
//
// in 32 bits, of operands of 16 bits.  A workgroup has TI x TJ of D in registers and takes k in steps of 64: both operands'
// pieces of a step go from memory straight into one of two buffers of shared memory, while the matrix
// instructions work on the other one.  An operand lies with k along its rows (DEEP) or across them; the latter is
// transposed on its way out of shared memory (ds_read_b64_tr_b16).  Reads past an operand's end give zeros.
//
// What bounds a long sum (2048 x 8192 over 49152 to 51200, wide tiles): matrix instructions are busy two thirds of the time at
// 1.9 to 2.0 GHz, 1260 to 1360 TFLOP/s with k along both operands' rows, 1320 with k across one and 1170 across both.  With every step
// read from the same place, and so from the nearest cache, they reach 1470, 1420 and 1270; with no loads at all, on constant data,
// 2270, 2230 and 1830: what is left is power and the loads' way into shared memory, not its reads (a quarter of the time) or bank
// conflicts: steps have none, a tile that leaves through shared memory 1024 cycles at its end.
#pragma once

#include "echo_ops_device.h"

namespace echo {
namespace {

// An operand: `rows` rows of `width` elements of 16 bits, `stride` bytes apart, in planes `plane` bytes apart.
// Rows begin at multiples of 16 bytes and hold whole pieces of 64 elements; 255 strides stay below 2^31.
struct Operand {
    const char *p;
    int64_t stride, plane, rows;
    int width;
};
struct Product {
    Operand a, b;
    int ni, nj;               // size of D
    int tiles_i, tiles_j;
    int steps;                // of 64 along k, in a plane
    int pairs;                // products of planes that are summed: 1, 2 of two planes of b, or 6 of 3 planes each
    int splits;               // parts of the steps, each in a workgroup of its own
};
// 3 planes of 8 significant bits each make 24: the products that matter, of planes (a, b).
__device__ __forceinline__ int plane_a(int pair) { return (0x120100 >> (4 * pair)) & 3; }   // 0 0 1 0 2 1
__device__ __forceinline__ int plane_b(int pair) { return (0x102010 >> (4 * pair)) & 3; }   // 0 1 0 2 0 1

using F4 = __attribute__((ext_vector_type(4))) float;
template <class T>
using H8 = __attribute__((ext_vector_type(8))) T;
using S4 = __attribute__((ext_vector_type(4))) short;
using LdsPtr = __attribute__((address_space(3))) void *;

constexpr int kDepth = 64;

__device__ __forceinline__ F4 mfma(H8<bf16> a, H8<bf16> b, F4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ F4 mfma(H8<f16> a, H8<f16> b, F4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// Where the 16-byte piece c of row r lies in shared memory: pieces are exchanged within a row so that the lanes which
// read together meet different banks.
__device__ __forceinline__ int turned(int k) { return (k & 3) | ((k >> 3) & 1) << 2; }

// One operand's share of a step: R rows of D's side, from memory to shared memory and from there to registers.
template <class T, int R, bool DEEP, int WAVES>
struct Feed {
    static constexpr int BYTES = R * kDepth * 2, LOADS = BYTES / (WAVES * 1024), UNITS = R / 16;
    static_assert(LOADS * WAVES * 1024 == BYTES, "");
    const char *origin, *p;
    int64_t left0, left, advance, plane;
    unsigned off[LOADS];
    __device__ __forceinline__ Feed(const Operand &o, int64_t row, int wave, int lane) {
        origin = o.p + (DEEP ? row * o.stride : row * 2);
        left0 = (o.rows - 1 - (DEEP ? row : 0)) * o.stride + ((int64_t)o.width - (DEEP ? 0 : row)) * 2;
        advance = DEEP ? kDepth * 2 : kDepth * o.stride;
        plane = o.plane;
#pragma unroll
        for (int n = 0; n < LOADS; ++n) {
            const int q = (n * WAVES + wave) * kWave + lane, PIECES = DEEP ? 8 : R / 8, r = q / PIECES, c = q % PIECES;
            const int from = DEEP ? c ^ (r & 7) : c ^ ((turned(r) & (UNITS - 1)) << 1);
            off[n] = (unsigned)(r * o.stride) + from * 16;
        }
    }
    __device__ __forceinline__ void seek(int in_plane, int step) {
        const int64_t by = step * advance;
        p = origin + in_plane * plane + by;
        left = left0 - by;
    }
    // starts the loads of a step and goes on to the next
    __device__ __forceinline__ void fetch(char *lds, int wave) {
        // a step may begin past the operand's end, where the other one is padded further
        const unsigned records = left > 0xffffffffll ? 0xffffffffu : left < 0 ? 0u : (unsigned)left;
        const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(p), 0, records, 0x00020000);
#pragma unroll
        for (int n = 0; n < LOADS; ++n)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (LdsPtr)(lds + (n * WAVES + wave) * 1024), 16, off[n], 0, 0, 0);
        p += advance;
        left -= advance;
    }
    // A lane's place in a fragment of 16 rows and 32 of k: it has row lane % 16 and k 8 * (lane / 16) .. + 7.  `first` is the
    // wavefront's first unit of 16 rows.  Across k, fragments' addresses are xor-ed together where they are read: kept in
    // registers for both buffers they did not fit (2048 x 51200 x 8192: 2.72 ms with the spills, 1.56 without).
    struct Reader {
        unsigned at, mix;
        __device__ __forceinline__ Reader(int first, int lane) {
            if constexpr (DEEP) {
                at = (first * 16 + lane % 16) * 128;
                mix = ((lane / 16) ^ (lane & 7)) * 16;      // the second half's piece is 4 further: the other one of a pair
            } else {
                const int k = (lane / 16) * 8 + (lane % 16) / 4;
                at = k * (R * 2) + (lane % 4) * 8;
                mix = ((turned(k) & (UNITS - 1)) ^ first) << 5;
            }
        }
        __device__ __forceinline__ H8<T> frag(const char *lds, int unit, int half) const {
            if constexpr (DEEP) {
                return *reinterpret_cast<const H8<T> *>(lds + (at + (mix ^ (half * 64))) + unit * 2048);
            } else {
#ifdef __HIP_DEVICE_COMPILE__      // the builtin is the GPU's
                unsigned m = mix;
                asm volatile("" : "+v"(m));      // not to be kept for every unit
                const char *from = lds + (((unit << 5) ^ m) + at);
                typedef __attribute__((address_space(3))) S4 *Lds4;
                const S4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4)(from + half * (32 * R * 2)));
                const S4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4)(from + half * (32 * R * 2) + 4 * R * 2));
                return __builtin_bit_cast(H8<T>, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#else
                return H8<T>{};
#endif
            }
        }
    };
};

template <int TI_, int TJ_, int WI_, int WJ_>
struct Shape {
    static constexpr int TI = TI_, TJ = TJ_, WI = WI_, WJ = WJ_, WAVES = WI * WJ, THREADS = WAVES * kWave;
    static constexpr int BI = TI / WI / 16, BJ = TJ / WJ / 16;       // blocks of 16 x 16 that a wavefront has
    static constexpr int BYTES = (TI + TJ) * kDepth * 2;             // of a step in shared memory
};
// A workgroup's place in D.  Workgroups go to the eight dies in turn; those of one die take neighbouring tiles, and
// eight tiles along j before the next along i, so that their operands meet in that die's cache.
struct Place {
    int ti, tj, split;
};
__device__ __forceinline__ Place place_of(const Product &m, int id) {
    const int tiles = m.tiles_i * m.tiles_j, all = tiles * m.splits;
    const int die = id % 8, each = all / 8, more = all % 8;
    int t = die * each + (die < more ? die : more) + id / 8;
    const int split = t / tiles;
    t -= split * tiles;
    const int group = t / (8 * m.tiles_i), first = group * 8, wide = m.tiles_j - first < 8 ? m.tiles_j - first : 8;
    t -= group * 8 * m.tiles_i;
    return Place{t / wide, first + t % wide, split};
}

// A wavefront's part of D on its way out in 16 bits: four elements of a lane lie side by side, and 16 lanes with
// them, 32 bytes; through shared memory a row of 128 or 256 bytes is written at once.  Pieces are exchanged within a row so that lanes meet
// different banks.  The buffers have been read by everybody before put.
template <class S, class K>
struct Outgoing {
    static constexpr int PITCH = S::BI * 32, PIECES = PITCH / 16, ROWS = S::BJ * 16, BYTES = ROWS * PITCH, AT_ONCE = kWave / PIECES;
    static_assert(sizeof(K) == 2 && S::WAVES * BYTES <= 2 * S::BYTES && S::BYTES % BYTES == 0, "");
    char *area;
    int lane;
    __device__ __forceinline__ Outgoing(char *t0, char *t1, int wave, int l) : lane(l) {
        constexpr int EACH = S::BYTES / BYTES;
        area = (wave < EACH ? t0 + wave * BYTES : t1 + (wave - EACH) * BYTES);
    }
    __device__ __forceinline__ void put(int k, int b, F4 d) const {
        typedef __attribute__((ext_vector_type(4))) K K4;
        const int row = b * 16 + lane % 16, piece = k * 2 + lane / 32;
        *reinterpret_cast<K4 *>(area + row * PITCH + ((piece ^ (row & (PIECES - 1))) * 16) + (lane / 16 % 2) * 8) = __builtin_convertvector(d, K4);
    }
    // rows `stride` elements apart, of which `rows` and `cols` of this part exist
    __device__ __forceinline__ void flush(K *out, int64_t stride, int rows, int cols) const {
        const int piece = lane % PIECES, left = cols - piece * 8;
#pragma unroll
        for (int r0 = 0; r0 < ROWS; r0 += AT_ONCE) {
            const int row = r0 + lane / PIECES;
            const V<K, 8> v = *reinterpret_cast<const V<K, 8> *>(area + row * PITCH + ((piece ^ (row & (PIECES - 1))) * 16));
            if (row >= rows) continue;
            K *at = out + row * stride + piece * 8;
            if (left >= 8) {
                *reinterpret_cast<V<K, 8> *>(at) = v;
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < left) at[j] = v[j];
            }
        }
    }
};

// D's tile in registers: acc[a][b][e] belongs to i = a * 16 + 4 * (lane / 16) + e and j = b * 16 + lane % 16 of the wavefront's part.
template <class T, bool ADEEP, bool BDEEP, class S, class Acc>
__device__ __forceinline__ void multiply(const Product &m, const Place &at, char *t0, char *t1, Acc &acc) {
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wi = wave / S::WJ, wj = wave % S::WJ;
    using FA = Feed<T, S::TI, ADEEP, S::WAVES>;
    using FB = Feed<T, S::TJ, BDEEP, S::WAVES>;
    FA fa(m.a, (int64_t)at.ti * S::TI, wave, lane);
    FB fb(m.b, (int64_t)at.tj * S::TJ, wave, lane);
    const int all = m.steps * m.pairs, begin = (int)((unsigned)all * (unsigned)at.split / (unsigned)m.splits),
              end = (int)((unsigned)all * (unsigned)(at.split + 1) / (unsigned)m.splits);
    int pair = begin / m.steps, step = begin - pair * m.steps;
    fa.seek(plane_a(pair), step);
    fb.seek(plane_b(pair), step);
    const auto fetch = [&](char *t) ECHO_INLINE {
        fa.fetch(t, wave);
        fb.fetch(t + FA::BYTES, wave);
        if (++step == m.steps) {
            step = 0;
            ++pair;
            fa.seek(plane_a(pair), 0);
            fb.seek(plane_b(pair), 0);
        }
    };
#pragma unroll
    for (int a = 0; a < S::BI; ++a)
#pragma unroll
        for (int b = 0; b < S::BJ; ++b) acc[a][b] = 0.0f;
    const typename FA::Reader ra(wi * S::BI, lane);
    const typename FB::Reader rb(wj * S::BJ, lane);
    // A step is 2 * BI items, each a fragment of a with the BJ fragments of b of its half.  Fragments of a are read AHEAD items before
    // their turn, those of b a half before; so the last items of a step read what follows.  In front of them stands
    // the barrier, which says two things: the next step is in shared memory for everybody (each wavefront has waited for
    // its own loads), and everybody has read all of this one, whose buffer takes the step after the next.
    constexpr int ITEMS = 2 * S::BI, AHEAD = 4, HELD = 8;
    static_assert(S::BJ == AHEAD && S::BI >= AHEAD && ITEMS % HELD == 0, "one fragment of b an item");
    H8<T> x[HELD], y[2][S::BJ];
    const auto turn = [&](char *mine, char *next, bool goes_on, bool more) ECHO_INLINE {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            if (i == ITEMS - AHEAD && goes_on) {
                __builtin_amdgcn_s_waitcnt(0x0070);      // vmcnt(0), lgkmcnt(0)
                __syncthreads();
            }
            if (i < S::BJ) y[1][i] = rb.frag(mine + FA::BYTES, i, 1);
            if (i < ITEMS - AHEAD) {
                x[(i + AHEAD) % HELD] = ra.frag(mine, (i + AHEAD) % S::BI, (i + AHEAD) / S::BI);
            } else if (goes_on) {
                y[0][i - (ITEMS - AHEAD)] = rb.frag(next + FA::BYTES, i - (ITEMS - AHEAD), 0);
                x[(i + AHEAD) % HELD] = ra.frag(next, i - (ITEMS - AHEAD), 0);
            }
#pragma unroll
            for (int b = 0; b < S::BJ; ++b)
                acc[i % S::BI][b] = mfma(x[i % HELD], y[i / S::BI][b], acc[i % S::BI][b]);
            if (i == ITEMS - AHEAD && more) fetch(mine);
            __builtin_amdgcn_sched_barrier(0);      // the order is meant
        }
    };
    int s = begin;
    if (s < end) {
        fetch(t0);
        __builtin_amdgcn_s_waitcnt(0x0070);
        __syncthreads();
        if (s + 1 < end) fetch(t1);
#pragma unroll
        for (int b = 0; b < S::BJ; ++b) y[0][b] = rb.frag(t0 + FA::BYTES, b, 0);
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) x[a] = ra.frag(t0, a, 0);
    }
    for (; s + 3 < end; s += 2) {
        turn(t0, t1, true, true);
        turn(t1, t0, true, true);
    }
    for (; s < end; s += 2) {
        turn(t0, t1, s + 1 < end, s + 2 < end);
        if (s + 1 < end) turn(t1, t0, s + 2 < end, false);
    }
}

}  // namespace
}  // namespace echo
