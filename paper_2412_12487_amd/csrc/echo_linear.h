// echo_linear.h -- arguments of the output head's kernels and the tiles that they come in.
#pragma once

#include "echo_product.h"
#include "echo_teacher.h"

namespace echo {

struct HeadArgs {
    Product m;                    // a: the table's rows, b: the hidden states
    int rows, vocab;              // rows, and ids held here
    int first;                    // column that the product's first one is
    float inv_t;
    const void *targets;          // one target a row, where top is 0
    int wide_index, top;
    int64_t vocab_start, vocab_size;
    const int *local;             // [rows][top]: an entry's column here, or -1
    const float *q;               // [rows][top]
    const float2 *prior;          // [rows]: sum of q log q, and 1 where the row is trained on
    float2 *stats;                // [parts][rows]: largest product, and sum of exponentials relative to it, of a wavefront's columns
    float *hits;                  // products of the target or of the entries
    const float2 *whole;          // [rows]: largest product and sum of exponentials relative to it, or null: lse is given
    const float *lse, *grad_loss, *scale;
    float *scale_out;             // one workgroup more writes it, or null
    char *prob;                   // [planes][prob_rows][.]: the gradient's shares
    int64_t prob_stride, prob_plane;
    int prob_rows, prob_cols;     // columns that are written, from the product's first on
    void *kept;                   // [rows][kept_stride]: exponentials
    int64_t kept_stride;
};
struct ShareArgs {
    const float2 *stats, *whole, *prior;      // whole [rows]: largest product and sum of exponentials relative to it
    const float *hits, *q, *grad_loss, *scale;
    const int *local;
    const void *targets, *kept;
    int wide_index, top, rows, vocab, cols;
    int64_t vocab_start, vocab_size;
    float inv_t;
    int split, part0, part1;      // columns that a part of the statistics has, before `split` and from it on
    char *prob;                   // [planes][prob_rows][cols]
    int64_t prob_stride, prob_plane;
    int prob_rows;
};
struct JoinArgs {
    const float2 *stats, *prior;
    const float *hits, *q;
    const int *local;
    const void *targets;
    int wide_index, top, rows, vocab, parts;
    int64_t vocab_start, vocab_size;
    float inv_t, square;          // 1 / T, T^2
    float *lse, *target, *entropy, *loss;
    float2 *whole;                // or null
};
struct TeacherArgs {
    TeacherIn in;
    int64_t rows;
    int vocab;
    int *local;
    float *q;
    float2 *prior;
};
struct PartsArgs {
    Product m;
    float *parts;                 // [splits][rows][ld]
    int64_t part;
    int ld;
    TeacherIn in;                 // top is 0 with one target a row: its ids are the targets
    const float *grad_loss;
    float *scale_out;             // one workgroup more writes it, or null
};
// Rows whose logits are in parts of the sum.
struct RowsArgs {
    float *parts;                 // [splits][rows][ld]
    int64_t part;                 // elements from a part to the next
    int splits, ld, rows, vocab, cols;      // cols: of the gradient's shares
    TeacherIn in;                 // top is 0 with one target a row: its ids are the targets
    float square;
    float *lse, *target, *entropy, *loss;
    const float *lse_in, *grad_loss, *scale;
    char *prob;                   // or null
    int64_t prob_stride, prob_plane;
    int prob_rows;
};
struct LayoutArgs {
    const void *from;
    int64_t stride, rows;         // stride in elements
    int cols, width;
    char *to;
    int64_t plane;
};
// D of a product, or a part's share of it, times what the head's gradient is relative to.
struct OutArgs {
    Product m;
    const float *scale;
    float factor;
    float *parts;                 // [splits][nj][ni] of 32 bits, or null: D is whole
    int64_t part;                 // elements from a part to the next
    bool add_parts;               // parts are added to
    void *out;                    // [nj][ni]
    bool accumulate;
};
struct GatherArgs {
    const float *parts;
    int64_t n;                    // elements of a part
    int splits;
    const float *scale;
    float factor;
    void *out;
    bool accumulate;
};

namespace {
// Shapes of the tiles.  Wide: 256 x 256 by 8 wavefronts.  Middle: 128 x 128 by 4.  Thin: 256 x 64 by 4, for few rows.
using Wide = Shape<256, 256, 2, 4>;
using Middle = Shape<128, 128, 2, 2>;
using Thin = Shape<256, 64, 4, 1>;
// Shares of the gradient lie in [-1, 1]; those of half precision are taken 2^14 times as large, since
// most of a softmax is below its smallest number.
template <class T>
constexpr float kUnit = 1.0f;
template <>
constexpr float kUnit<f16> = 16384.0f;
// What the exponentials of a row are kept as between the loss's pass and the gradient's: of bfloat16 as half
// precision, 2^15 times as large, whose rounding of 2^-11 is small beside that to bfloat16 (2^-8) and
// whose smallest step is 2^-39; of the others in 32 bits, since a second rounding of half precision would
// be as large as the first.
template <class T, int PLANES>
struct KeptOf {
    using type = float;
};
template <>
struct KeptOf<bf16, 1> {
    using type = f16;
};
template <class T, int PLANES>
using Kept = typename KeptOf<T, PLANES>::type;
template <class T, int PLANES>
constexpr float kKeptUnit = sizeof(Kept<T, PLANES>) == 2 ? 32768.0f : 1.0f;
}  // namespace

// deep: b's sum runs along its rows (the hidden states' gradient), or across them (the table's)
hipError_t launch_out(const OutArgs &a, int type, int out_type, bool deep, int shape, hipStream_t s);
// both of them by middle tiles in one launch
hipError_t launch_both(const OutArgs &dhidden, const OutArgs &dweight, int type, int grad_type, hipStream_t s);
hipError_t launch_zero(void *out, int64_t bytes, hipStream_t s);
hipError_t launch_gather(const GatherArgs &a, int type, int out_type, hipStream_t s);

}  // namespace echo
