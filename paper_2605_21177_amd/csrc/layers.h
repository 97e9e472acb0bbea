// Internal interface between the C ABI of the layer and update operators (layers_api.cpp) and their kernels.
#ifndef CHUNKFT_LAYERS_H
#define CHUNKFT_LAYERS_H

#include <cstddef>
#include <cstdint>

namespace chunkft {

// ------------------------------------------------------------------ norm layer (norm.hip)
struct NormProblem {
  const void* X;
  const void* w;       // scale, or nullptr (ones)
  const void* b;       // shift, or nullptr (zeros)
  int64_t ldx, T, n;
  float eps;
  bool subtract_mean;
};

struct NormGrads {
  const float* stats;  // [T][2]
  const void* dY;
  void* dX;            // or nullptr
  int64_t lddy, lddx;
  float* dw;           // columns [w0, w1) at dw[0 ..], or nullptr
  float* db;
  int64_t w0, w1, b0, b1;
  int accumulate;
};

// Lanes that hold a row and 16-byte pieces each of them has; 0 lanes: a row that a workgroup cannot hold.
struct RowShape {
  int32_t lanes, pieces;
};
RowShape norm_forward_shape(int64_t n, int dtype);
RowShape norm_backward_shape(int64_t n, int dtype);
constexpr int kNormBackThreads = 512;    // of a workgroup of the backward pass, if a row takes no more

// Workgroups that a backward pass leaves partial sums of the vectors' gradients from; each leaves two rows of norm_pitch floats.
int64_t norm_parts(int64_t T, int64_t n, int dtype, int compute_units);
inline int64_t norm_pitch(int64_t n) { return (n + 31) / 32 * 32; }

int launch_norm_forward(const NormProblem& p, int dtype, void* Y, int64_t ldy, float* stats, void* stream);
int launch_norm_backward(const NormProblem& p, int dtype, const NormGrads& g, float* ws, void* stream);

// out[i] (+)= sum over the parts, in a fixed order, of ws[part * stride + first + i], i < count (0: not wanted; one of them is).
struct SumTarget {
  float* out;
  int64_t first, count;
};
int launch_sum_parts(const float* ws, int64_t parts, int64_t stride, const SumTarget& t0, const SumTarget& t1, int accumulate,
                     void* stream);

// ---------------------------------------------------------------- linear layer (linear.hip)
enum Act : int { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_SILU = 3 };

struct LinearProblem {
  const void* X;
  const void* W;
  const void* bias;      // or nullptr
  const void* residual;  // or nullptr
  int64_t ldx, ldw, ldr, out, in, T;
  int32_t dtype, act;
};

struct LinearGrads {
  const void* dY;
  const void* Z;         // nullptr without an activation
  void* dZ;              // nullptr without an activation
  void* dX;              // or nullptr
  int64_t lddy, ldz, lddz, lddx;
  float* db;             // columns [b0, b1), or nullptr
  int64_t b0, b1;
  int accumulate;
};

constexpr int kGateLanes = 32, kGateRows = 8;       // of the pass over dy and z: lanes along the columns, rows at a time

// Rows of partial sums (of norm_pitch(out) floats) that a backward pass leaves for the bias.
int64_t linear_parts(int64_t T, int64_t out, int dtype, int compute_units);

// How a product [M, K] x [K, N] is cut: square tiles of `tile` (bf16: 64 is 64 x 128), `slabs` runs of kslab values of k.
struct LinearPlan {
  int32_t tile, slabs;
  int64_t kslab;
  bool pack;            // operands are copied to rows of whole 128-byte lines, first, where they are not so already
};
// How its operands come: in rows of 16-byte pieces, which the direct loads take (bf16), through registers, or copied to such rows.
enum LinearRows : int { ROWS_IN_PIECES = 0, ROWS_AS_THEY_LIE = 1, ROWS_COPIED = 2 };
LinearPlan linear_plan(int64_t M, int64_t N, int64_t K, int dtype, int compute_units, LinearRows rows = ROWS_IN_PIECES);
// What a call runs by.  pieces: both operands' rows, with their addresses and strides, are such as the direct loads take; across: B
// is [K, N] (otherwise [N, K]).
LinearPlan linear_choice(int64_t M, int64_t N, int64_t K, int dtype, int compute_units, bool across, bool pieces);
// Rows and elements of a row of a packed operand (whole stages of k, whole lines), and bytes of the workspace's parts, in this order: the
// slabs' sums, A [M, K], B ([N, K], or [K, N] across).  From the shape alone: they are enough for either choice.
inline int64_t packed_pitch(int64_t n) { return (n + 63) / 64 * 64; }
struct LinearSpace {
  size_t slabs, a, b;
};
LinearSpace linear_space(int64_t M, int64_t N, int64_t K, int dtype, int compute_units, bool across);
bool linear_takes_few(int64_t T, int64_t out, int64_t in, int dtype);   // the forward pass is one pass over the weights, whatever the plan

int launch_linear_forward(const LinearProblem& p, void* Y, int64_t ldy, void* Z, int64_t ldz, float* ws, void* stream);
int launch_linear_backward(const LinearProblem& p, const LinearGrads& g, float* ws, void* stream);

// ------------------------------------------------------- orthogonalised update (orthogonalize.hip)
struct OrthoProblem {
  int64_t rows, cols;
  int32_t parts;         // of the products' operands: 1: 11 digits, 2: 22
  int32_t steps;
  float eps;
  // what is orthogonalised: G (bf16 or fp32), or the momentum step on g and m
  const void* G;
  int64_t ldg;
  int32_t g_dtype;
  float* m;              // nullptr: G itself
  float momentum;
  bool nesterov;
  // where it goes: O, or the update
  void* O;
  int64_t ldo;
  int32_t o_dtype;
  float* master;         // nullptr: O
  void* W;
  int32_t w_kind;        // WKind
  float lr, scale, weight_decay;
};

// How the product of an r x r result over K is cut: tiles of its lower half, slabs of kslab values of k.
struct NsCut {
  int32_t tile, slabs;
  int64_t kslab;
};
NsCut ns_cut(int64_t r, int64_t K, int parts, int compute_units);
int ns_apply_tile(int64_t rows, int64_t cols, int64_t K, int parts, int compute_units);
inline int64_t ns_half_tiles(int64_t r, int tile) {
  const int64_t n = (r + tile - 1) / tile;
  return n * (n + 1) / 2;
}

constexpr int kNsNormBlocks = 1024;      // most partial sums of the norm
struct NsLayout {
  int64_t rows_p, cols_p, r;             // padded to whole stages of k; the padded small side
  size_t x, a, diag, sums, total;        // bytes of a buffer of X, of A, of a diagonal, of the slabs' sums, of all
};
NsLayout ns_layout(int64_t rows, int64_t cols, int parts, int compute_units);

int launch_orthogonalize(const OrthoProblem& p, void* ws, void* stream);

}  // namespace chunkft
#endif
