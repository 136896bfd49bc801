// echo_teacher.h -- a teacher's distribution over its top ids, for the kernels of distillation.
#pragma once

#include "echo_ops_device.h"

namespace echo {

// What a teacher says: `top` ids a row and their logits.
struct TeacherIn {
    const void *ids, *logits;
    int index_type, type, top;
    int64_t vocab_start, vocab_size;
    float inv_t;
};

namespace {

constexpr float kLog2e = 1.44269504088896341f;

// exp(x), x <= 0 but for a row's rounding: one multiplication and the hardware's 2^x.  The product's rounding
// makes the result |x| 2^-24 of itself wrong, as does that of x itself.
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// A logit / T as a number of 32 bits, by itself: an lse that is given is such a number, and above each of them.  Fused with the
// subtraction of the lse, the product would not be rounded, and the largest logit's probability be up to exp of half its last place.
__device__ __forceinline__ float scaled(float l, float inv_t) {
#pragma clang fp contract(off)
    return l * inv_t;
}
__device__ __forceinline__ int64_t index_at(const void *ids, int index_type, int64_t at) {
    return index_type == ECHO_I64 ? id_at<int64_t>(ids, at) : id_at<int32_t>(ids, at);
}
__device__ __forceinline__ float value_at(const void *p, int type, int64_t at) {
    if (type == ECHO_F32) return static_cast<const float *>(p)[at];
    return type == ECHO_F16 ? (float)static_cast<const f16 *>(p)[at] : (float)static_cast<const bf16 *>(p)[at];
}
// Whether an id of a row has a mass, where its entries are not prepared: its first entry tells that of most rows.
__device__ __forceinline__ bool has_mass(const TeacherIn &t, int64_t row) {
    for (int k = 0; k < t.top; ++k) {
        const int64_t id = index_at(t.ids, t.index_type, row * t.top + k);
        if (id >= 0 && id < t.vocab_size && value_at(t.logits, t.type, row * t.top + k) != -kInf) return true;
    }
    return false;
}

// An entry: its column here (or -1), and the mass of its id, which the first entry of an id that has one holds.  `x` is for
// the logit of that column.  One wavefront prepares a row's entries in shared memory, and each lane reads again only
// what it wrote itself: entries lane, lane + 64, ...
struct Entry {
    int at;
    float mass, x;
};
struct Teacher {
    bool trained;      // an id of the vocabulary has a mass
    float prior;       // sum of q log q over the entries, also of those that name an id together
};
// The row's entries whose columns are in [first, first + cols).
//
// Latency bounds it: the ids are compared with each other as 64 lanes against each lane's in turn, and only where one comes
// twice are masses added up.  With loads from memory in that loop a row of 64 entries took 13 us and one of 128 51 us, with
// loads from shared memory 7 and 22 us.
__device__ __forceinline__ Teacher teacher_of(const TeacherIn &t, int64_t row, int first, int cols, int vocab, Entry *entries) {
    const int lane = threadIdx.x % kWave;
    const int64_t from = row * t.top;
    const auto logit = [&](int k) ECHO_INLINE {
        const int64_t id = index_at(t.ids, t.index_type, from + k);
        const float z = value_at(t.logits, t.type, from + k);      // beside the id, not behind it
        return id >= 0 && id < t.vocab_size ? z : -kInf;
    };
    float top = -kInf, sum = 0.0f, prior = 0.0f;
    for (int k = lane; k < t.top; k += kWave) {
        const float z = logit(k);
        entries[k].x = z;
        top = fmaxf(top, z);
    }
    top = wave_max(top);
    // distances from the largest logit, before they are divided by T: of logits far from 0 they are exact
    const float base = top == -kInf ? 0.0f : top;
    const auto distance = [&](int k) ECHO_INLINE { return (entries[k].x - base) * t.inv_t; };
    for (int k = lane; k < t.top; k += kWave) sum += expf(distance(k));
    sum = wave_sum(sum);
    const bool live = sum != 0.0f;      // NaN too
    const float log_sum = logf(sum);
    for (int k = lane; k < t.top; k += kWave) {
        const float d = distance(k), q = live ? expf(d) / sum : 0.0f;
        if (q != 0.0f) prior += q * (d - log_sum);
        int at = q != 0.0f ? shard_row(index_at(t.ids, t.index_type, from + k), t.vocab_start, vocab) : -1;
        if ((unsigned)(at - first) >= (unsigned)cols) at = -1;
        entries[k].at = at;
        entries[k].mass = at >= 0 ? q : 0.0f;
    }
    prior = wave_sum(prior);
    // every lane sees the wavefront's entries from here on
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    for (int k0 = 0; k0 < t.top; k0 += kWave) {
        const int k = k0 + lane, mine = k < t.top ? entries[k].at : -1;
        bool twice = false;
        for (int o0 = 0; o0 < t.top; o0 += kWave) {
            const int theirs = o0 + lane < t.top ? entries[o0 + lane].at : -1, n = t.top - o0 < kWave ? t.top - o0 : kWave;
            for (int j = 0; j < n; j += 8) {      // -1 past the end
#pragma unroll
                for (int i = 0; i < 8; ++i) twice |= __builtin_amdgcn_readlane(theirs, j + i) == mine && o0 + j + i != k;
            }
        }
        if (!__builtin_amdgcn_ballot_w64(twice && mine >= 0)) continue;
        float mass = 0.0f;
        bool later = false;
        if (mine >= 0) {
            for (int o = 0; o < t.top; ++o) {
                if (entries[o].at != mine) continue;
                mass += expf(distance(o)) / sum;
                later |= o < k;
            }
        }
        // x is read above by every lane, and at stays: the mass of a later entry of an id is dropped where it is used
        if (k < t.top && mine >= 0) entries[k].mass = later ? -1.0f : mass;
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    for (int k = lane; k < t.top; k += kWave)
        if (entries[k].mass < 0.0f) entries[k] = Entry{-1, 0.0f, 0.0f};
    return Teacher{live, prior};
}
// The logits of the entries' columns; before this, x is the teacher's.
template <class X>
__device__ __forceinline__ void take_logits(Entry *entries, int top, X logit_at) {
    for (int k = threadIdx.x % kWave; k < top; k += kWave) {
        const int at = entries[k].at;
        entries[k].x = at >= 0 ? logit_at(at) : 0.0f;
    }
}
// The entries' share of the loss's cross term, of logits taken from `from` on.
__device__ __forceinline__ float cross_of(const Entry *entries, int top, float from) {
    float cross = 0.0f;
    for (int k = threadIdx.x % kWave; k < top; k += kWave) {
        const Entry e = entries[k];
        if (e.at >= 0) cross += e.mass * (e.x - from);
    }
    return wave_sum(cross);
}

}  // namespace
}  // namespace echo
