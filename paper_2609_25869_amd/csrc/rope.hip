// Rotary positions on up to three axes.
//
// One thread owns one item of a token's head rows - four interleaved pairs, or
// eight pairs (i, i + P), or one pair where P is no multiple of eight - forms
// the sines and cosines of its pairs once and turns that item in every
// `lanes`-th head of Q and K (and copies it in V).  Consecutive threads hold
// consecutive items, then consecutive heads.
//
// Angles are counted in turns: position * (freq / 2 pi) in 64 bits, less the
// nearest integer, so a position of any size keeps the 2^-25 turns of the
// 32-bit remainder (formed in 32 bits, position 100000 would be off by 0.008
// radians).
//
// The work is the memory traffic: every element is read and written once (115200 tokens,
// Q and K of 24 heads of 128 in bfloat16: 492 us, 5.8 TB/s read and written; a prompt of
// 32768 tokens, 32 and 8 heads of 128, by positions: 137 us in the half layout, 4.9 TB/s,
// 140 interleaved).  One pair a thread, where P is no multiple of eight, moves single
// elements: 171 us with 60 pairs.  One token takes 5.3 us, of which 3.8 are left without
// pairs: the kernel's start, and a row's way through memory and back; the rest is a
// thread's eight sines, formed from 64-bit products.
#include "ops_internal.h"

namespace bsa_ops {

namespace {

constexpr int kThreads = 256;
constexpr double kInv2Pi = 0.15915494309189533576888376337251436;

enum Mode { kInterleaved, kHalf8, kHalf1 };

template <typename T>
struct alignas(16) Vec8 {
  T e[8];
};

template <Mode M>
__host__ __device__ inline int items_of(int d, int P) {
  return M == kInterleaved ? d / 8 : M == kHalf8 ? P / 8 + (d - 2 * P) / 8 : P + (d - 2 * P);
}

// One item of a head row: loaded, turned, stored.
template <typename T, Mode M>
struct Item {
  Vec8<T> v, z;  // kHalf1: element 0 alone; z: the pairs' second elements

  __device__ void load(const T* x, int item, int P) {
    if constexpr (M == kInterleaved) {
      v = *reinterpret_cast<const Vec8<T>*>(x + 8 * item);
    } else if constexpr (M == kHalf8) {
      if (8 * item < P) {
        v = *reinterpret_cast<const Vec8<T>*>(x + 8 * item);
        z = *reinterpret_cast<const Vec8<T>*>(x + P + 8 * item);
      } else {
        v = *reinterpret_cast<const Vec8<T>*>(x + P + 8 * item);  // 2 P + 8 (item - P / 8)
      }
    } else {
      v.e[0] = item < P ? x[item] : x[P + item];
      if (item < P) z.e[0] = x[P + item];
    }
  }
  __device__ void store(T* y, int item, int P) const {
    if constexpr (M == kInterleaved) {
      *reinterpret_cast<Vec8<T>*>(y + 8 * item) = v;
    } else if constexpr (M == kHalf8) {
      if (8 * item < P) {
        *reinterpret_cast<Vec8<T>*>(y + 8 * item) = v;
        *reinterpret_cast<Vec8<T>*>(y + P + 8 * item) = z;
      } else {
        *reinterpret_cast<Vec8<T>*>(y + P + 8 * item) = v;
      }
    } else {
      y[item < P ? item : P + item] = v.e[0];
      if (item < P) y[P + item] = z.e[0];
    }
  }
  // the first n pairs of the item (elements past the pairs keep their bits)
  __device__ void turn(const float* co, const float* si, int n) {
    constexpr int kPairs = M == kInterleaved ? 4 : M == kHalf8 ? 8 : 1;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      T& a = M == kInterleaved ? v.e[2 * i] : v.e[i];
      T& b = M == kInterleaved ? v.e[2 * i + 1] : z.e[i];
      if (i < n) {
        const float u = (float)a, w = (float)b;
        a = (T)(u * co[i] - w * si[i]);
        b = (T)(u * si[i] + w * co[i]);
      }
    }
  }
};

// A block holds tokens_per_block tokens: thread = (token, lane, item), item fastest.
template <typename T, Mode M>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a, int items, int lanes, int tokens_per_block) {
  const int per_token = items * lanes;
  const int in_block = threadIdx.x / per_token, rest = threadIdx.x % per_token;
  const int item = rest % items, lane = rest / items;
  const int64_t token = (int64_t)blockIdx.x * tokens_per_block + in_block;
  const int64_t tokens = (int64_t)a.batch * a.seq;
  if (in_block >= tokens_per_block || token >= tokens) return;
  // (a 64-bit division is a hundred instructions)
  const int b = tokens <= 0x7fffffff ? (int)token / a.seq : (int)(token / a.seq);
  const int n = (int)(token - (int64_t)b * a.seq);
  if (a.lengths && n >= a.lengths[b]) return;

  constexpr int kPairs = M == kInterleaved ? 4 : M == kHalf8 ? 8 : 1;
  const int pair0 = item * kPairs;
  int32_t pos[3];
  bool turned = true;
  if (a.positions) {
    const int32_t* p = a.positions + b * a.ps1 + n;
    // axes without pairs are not read
    pos[0] = a.end0 > 0 ? p[0] : 0;
    pos[1] = a.end1 > a.end0 ? p[a.ps0] : 0;
    pos[2] = a.P > a.end1 ? p[2 * a.ps0] : 0;
  } else {
    const int w = n % a.g2, r = n / a.g2;
    pos[0] = r / a.g1 + a.origin[0];
    pos[1] = r % a.g1 + a.origin[1];
    pos[2] = w + a.origin[2];
    turned = n < a.volume;
  }
  const int n_pairs = turned ? a.P - pair0 : 0;  // of the item: all of them where it is kPairs or more
  float co[kPairs], si[kPairs];
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    co[i] = 1.f;
    si[i] = 0.f;
    if (i < n_pairs) {
      const int pr = pair0 + i;
      const int p = pr < a.end0 ? pos[0] : pr < a.end1 ? pos[1] : pos[2];
      double t = (double)p * (a.freq[pr] * kInv2Pi);
      t -= rint(t);
      sincospif((float)(2.0 * t), &si[i], &co[i]);
      if (a.inverse) si[i] = -si[i];
    }
  }

  // the token's rows in one tensor: kBatch heads are loaded before the first is stored
  auto rows_of = [&](int t, int64_t row, int pairs) {
    const T* x = static_cast<const T*>(a.x[t]) + b * a.xs[t].b + n * a.xs[t].n;
    T* y = static_cast<T*>(a.y[t]) + b * a.ys[t].b + row * a.ys[t].n;
    constexpr int kBatch = sizeof(T) == 2 && M == kInterleaved ? 6 : 3;
    for (int h0 = lane; h0 < a.heads[t]; h0 += kBatch * lanes) {
      Item<T, M> r[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const int h = h0 + i * lanes;
        if (h < a.heads[t]) r[i].load(x + h * a.xs[t].h, item, a.P);
      }
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const int h = h0 + i * lanes;
        if (h >= a.heads[t]) continue;
        r[i].turn(co, si, pairs);
        r[i].store(y + h * a.ys[t].h, item, a.P);
      }
    }
  };
  rows_of(0, n, n_pairs);
  const int64_t row = n + (a.rows ? (int64_t)a.rows[b] : 0);
  if (row < 0 || row >= a.kv_rows) return;
  rows_of(1, row, n_pairs);
  rows_of(2, row, 0);
}

template <typename T, Mode M>
hipError_t launch(const RopeArgs& a, hipStream_t s) {
  const int items = items_of<M>(a.d, a.P);
  const int most = a.heads[0] > a.heads[1] ? a.heads[0] : a.heads[1];
  const int64_t tokens = (int64_t)a.batch * a.seq;
  if (tokens == 0) return hipSuccess;
  // Threads per token: with enough tokens to fill the card four heads side by side,
  // so that the sines and cosines are formed for a quarter of the heads each; else as
  // many as a block holds.
  constexpr int64_t kFill = int64_t(256) * 2048;  // threads the card holds
  int lanes = kThreads / items < 1 ? 1 : kThreads / items;
  if (lanes > most) lanes = most;
  if (lanes > 4 && tokens * items * 4 >= kFill) lanes = 4;
  const int per_block = kThreads / (items * lanes);
  const int64_t blocks = (tokens + per_block - 1) / per_block;
  if (!fits_launch(blocks, kThreads)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((rope_kernel<T, M>), dim3((unsigned)blocks), dim3(kThreads), 0, s, a, items, lanes, per_block);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_type(bool interleaved, const RopeArgs& a, hipStream_t s) {
  if (interleaved) return launch<T, kInterleaved>(a, s);
  if (a.P % 8 == 0) return launch<T, kHalf8>(a, s);
  return launch<T, kHalf1>(a, s);
}

}  // namespace

hipError_t launch_rope(int dtype, bool interleaved, const RopeArgs& a, hipStream_t s) {
  if (dtype == kBf16) return launch_type<__bf16>(interleaved, a, s);
  if (dtype == kF16) return launch_type<_Float16>(interleaved, a, s);
  return launch_type<float>(interleaved, a, s);
}

}  // namespace bsa_ops
