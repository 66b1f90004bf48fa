// Rotary positions on up to three axes.
//
// One thread owns one item of a token's head row - four interleaved pairs, or
// eight pairs (i, i + P), or one pair where P is no multiple of eight - forms
// the sines and cosines of its pairs once and turns that item in every
// `lanes`-th head of Q and K (and copies it in V).  Consecutive threads hold
// consecutive 16-byte items, then consecutive heads.
//
// Angles are counted in turns: position * (freq / 2 pi) in 64 bits, less the
// nearest integer, so a position of any size keeps the 2^-25 turns of the
// 32-bit remainder (formed in 32 bits, position 100000 would be off by 0.008
// radians).
//
// The work is the memory traffic: every element is read and written once.
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

template <typename T, Mode M>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a, int items, int lanes, int64_t total) {
  const int64_t idx = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (idx >= total) return;
  const int item = (int)(idx % items);
  const int64_t rest = idx / items;
  const int lane = (int)(rest % lanes);
  const int64_t token = rest / lanes;
  const int b = (int)(token / a.seq), n = (int)(token % a.seq);
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
  float co[kPairs], si[kPairs];
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    const int pr = pair0 + i;
    co[i] = 1.f;
    si[i] = 0.f;
    if (turned && pr < a.P) {
      const int p = pr < a.end0 ? pos[0] : pr < a.end1 ? pos[1] : pos[2];
      double t = (double)p * (a.freq[pr] * kInv2Pi);
      t -= rint(t);
      sincospif((float)(2.0 * t), &si[i], &co[i]);
      if (a.inverse) si[i] = -si[i];
    }
  }

  const int64_t row_in_kv = n + (a.rows ? (int64_t)a.rows[b] : 0);
  const bool kv_fits = row_in_kv >= 0 && row_in_kv < a.kv_rows;
  const int hq = a.heads[0], hk = hq + a.heads[1], all = hk + a.heads[2];
  for (int c = lane; c < all; c += lanes) {
    const int t = c < hq ? 0 : c < hk ? 1 : 2;
    if (t > 0 && !kv_fits) break;
    const int h = c - (t == 0 ? 0 : t == 1 ? hq : hk);
    const T* x = static_cast<const T*>(a.x[t]) + b * a.xs[t].b + h * a.xs[t].h + n * a.xs[t].n;
    T* y = static_cast<T*>(a.y[t]) + b * a.ys[t].b + h * a.ys[t].h + (t == 0 ? n : row_in_kv) * a.ys[t].n;
    if constexpr (M == kInterleaved) {
      Vec8<T> v = *reinterpret_cast<const Vec8<T>*>(x + 8 * item);
      if (t < 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float u = (float)v.e[2 * i], w = (float)v.e[2 * i + 1];
          // elements past the pairs (and unturned tokens) keep their bits: 1 and 0
          // multiply exactly, but for infinities
          if (pair0 + i < a.P && turned) {
            v.e[2 * i] = (T)(u * co[i] - w * si[i]);
            v.e[2 * i + 1] = (T)(u * si[i] + w * co[i]);
          }
        }
      }
      *reinterpret_cast<Vec8<T>*>(y + 8 * item) = v;
    } else if constexpr (M == kHalf8) {
      if (pair0 < a.P) {
        Vec8<T> v = *reinterpret_cast<const Vec8<T>*>(x + pair0);
        Vec8<T> z = *reinterpret_cast<const Vec8<T>*>(x + a.P + pair0);
        if (t < 2 && turned) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float u = (float)v.e[i], w = (float)z.e[i];
            v.e[i] = (T)(u * co[i] - w * si[i]);
            z.e[i] = (T)(u * si[i] + w * co[i]);
          }
        }
        *reinterpret_cast<Vec8<T>*>(y + pair0) = v;
        *reinterpret_cast<Vec8<T>*>(y + a.P + pair0) = z;
      } else {
        const int at = 2 * a.P + 8 * (item - a.P / 8);
        *reinterpret_cast<Vec8<T>*>(y + at) = *reinterpret_cast<const Vec8<T>*>(x + at);
      }
    } else {
      if (item < a.P) {
        T v = x[item], z = x[a.P + item];
        if (t < 2 && turned) {
          const float u = (float)v, w = (float)z;
          v = (T)(u * co[0] - w * si[0]);
          z = (T)(u * si[0] + w * co[0]);
        }
        y[item] = v;
        y[a.P + item] = z;
      } else {
        y[a.P + item] = x[a.P + item];
      }
    }
  }
}

template <typename T, Mode M>
hipError_t launch(const RopeArgs& a, hipStream_t s) {
  const int items = items_of<M>(a.d, a.P);
  const int all = a.heads[0] + a.heads[1] + a.heads[2];
  const int64_t tokens = (int64_t)a.batch * a.seq;
  // Threads per token: a head each where tokens are few; with enough of them
  // four heads side by side, so that the sines and cosines of a token are
  // formed for a quarter of its heads each.
  int lanes = all;
  constexpr int64_t kFill = int64_t(256) * 2048;  // threads the card holds
  if (tokens * items * 4 >= kFill && all > 4) lanes = 4;
  const int64_t total = tokens * items * lanes;
  if (total == 0) return hipSuccess;
  const int64_t blocks = (total + kThreads - 1) / kThreads;
  if (blocks > 0x7fffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL((rope_kernel<T, M>), dim3((unsigned)blocks), dim3(kThreads), 0, s, a, items, lanes, total);
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
