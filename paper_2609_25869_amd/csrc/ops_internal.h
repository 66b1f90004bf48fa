// Internal declarations of libbsa_ops.so: arguments and launchers of the rotary
// position and window attention kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace bsa_ops {

enum DType { kBf16 = 0, kF16 = 1, kF32 = 2 };

struct Strides {
  int64_t b, h, n;  // batch, head, token; elements
};

struct RopeArgs {
  const void* x[3];  // q, k, v (null: none)
  void* y[3];
  Strides xs[3], ys[3];
  int32_t heads[3];
  int32_t batch, seq, d, P;
  int32_t end0, end1;  // first pair of axis 1 and of axis 2
  int32_t inverse;
  int32_t g1, g2;      // grid, height and width
  int64_t volume;      // tokens of the grid
  int32_t origin[3];
  int32_t kv_rows;
  const double* freq;
  const int32_t* positions;  // null: grid
  int64_t ps0, ps1;
  const int32_t* lengths;
  const int32_t* rows;
};

// A launch counts its threads in 32 bits.
inline bool fits_launch(int64_t blocks, int threads) { return blocks <= (int64_t)0xffffffff / threads; }

hipError_t launch_rope(int dtype, bool interleaved, const RopeArgs& a, hipStream_t s);

// Window attention.  A row is one query of one head; the rows of the heads that
// share a key head are numbered token by token (row = token * group + head
// within the group), so a workgroup's rows look at neighbouring positions.
struct WindowArgs {
  const void* q;
  const void* k;
  const void* v;
  void* o;
  float* lse;  // may be null
  Strides qs, ks, vs, os;
  int32_t B, H, Hkv, group, Nq, Nkv;
  int32_t left, right, sinks;  // left, right: at most kFar, which reaches every key
  float scale;                 // of the scores
  float scale_log2;            // scale * log2(e)
  const int32_t* q_len;
  const int32_t* kv_len;
  int32_t deal;          // see item_of_slot
  int32_t later_longer;  // rows see the more keys the later they are
  int32_t ntiles;  // row tiles per key head
  int32_t nsplit;  // slices of a row tile's keys (forward)
  float* part;     // partial states of the slices
  // backward
  const void* dout;
  void* dq;
  void* dk;
  void* dv;
  Strides dos, dqs, dks, dvs;
  float* stats;        // [B, H, 2, stat_rows]: base-2 LSE, and row sums of dO * O
  int64_t stat_rows;   // at least Nq + 63: whole tiles of rows may be read
  // dK/dV: key tiles per key head, those that hold sinks (the first ones), and the
  // slices that the queries of a tile with and without sinks are cut into
  int32_t nktiles, nsink, sink_slices, slices;
  int32_t deep;  // which dK/dV kernel
};

// Key tiles of one key head as work items of the dK/dV kernel: the slices of the
// tiles without sinks, then those of the others.  A tile cut into several slices has
// partial sums in the workspace, in the order of the items.
inline __host__ __device__ int64_t dkv_items(const WindowArgs& a) {
  return (int64_t)a.nsink * a.sink_slices + (int64_t)(a.nktiles - a.nsink) * a.slices;
}
inline __host__ __device__ int64_t dkv_parts(const WindowArgs& a) {
  return (a.sink_slices > 1 ? (int64_t)a.nsink * a.sink_slices : 0) +
         (a.slices > 1 ? (int64_t)(a.nktiles - a.nsink) * a.slices : 0);
}

constexpr int32_t kFar = 1 << 30;

hipError_t launch_window_forward(int dtype, int d, const WindowArgs& a, hipStream_t s);
hipError_t launch_window_backward(int dtype, int d, const WindowArgs& a, hipStream_t s);

// Shape of the launches, from the host's sizes alone.
struct ForwardPlan {
  int32_t tile_rows, ntiles, nsplit;
  int64_t part_floats;  // of the workspace
};
ForwardPlan plan_forward(const WindowArgs& a, int d);
// Sets the backward pass's tile counts, slices and stat_rows; returns the floats of
// its workspace (stats, then partial sums).
int64_t plan_backward(WindowArgs* a, int d);

}  // namespace bsa_ops
