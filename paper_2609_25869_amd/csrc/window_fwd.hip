// Window attention forward for gfx950: a workgroup of NW waves owns 32 * NW rows
// (query tokens x the heads that share a key head), each wave 32 of them, and
// walks the keys that any of them sees - the first `sinks` and one contiguous
// range - in tiles of 8 KB of K and 8 KB of V that come straight from memory to a
// ring in LDS.
//
// Scores are computed transposed, S^T = K Q^T (v_mfma 32x32x16): a lane then owns
// one row and 16 keys of each 32, so the softmax state is one number per lane and
// O^T += V^T P^T takes the lane's own probabilities as its operand.
#include "window_common.h"

// (Kernel bodies are kept from the host's pass, which drops the launch stub of a
// template whose device builtins it cannot check.)

namespace bsa_ops {

namespace {

constexpr int kMaxSplit = 64;

template <typename T, int D, int NW>
__global__ __launch_bounds__(64 * NW) void window_fwd_kernel(WindowArgs a) {
#ifdef __HIP_DEVICE_COMPILE__
  using E = Elem<T>;
  using R = Rows<D>;
  typedef typename E::x8 x8;
  constexpr int TK = kTileKeys<D>, TQ = 32 * NW, kStages = 4;
  constexpr int kNKB = TK / 32, kTile = TK * R::kBytes;
  static_assert(kTile == 8192, "K and V tiles are 8 KB");
  using Load = TileLoad<D, TK, NW>;
  constexpr int kGroup = 2 * Load::kLoads;  // loads of one tile pair per wave
  // each slot is an array of its own: the compiler then sees that reads of one
  // never alias the loads that fill another, and leaves those in flight
  __shared__ __attribute__((aligned(1024))) uint8_t ring0[2 * kTile];
  __shared__ __attribute__((aligned(1024))) uint8_t ring1[2 * kTile];
  __shared__ __attribute__((aligned(1024))) uint8_t ring2[2 * kTile];
  __shared__ __attribute__((aligned(1024))) uint8_t ring3[2 * kTile];
  auto slot = [&](int i) -> uint8_t* { return i == 0 ? ring0 : i == 1 ? ring1 : i == 2 ? ring2 : ring3; };

  const int64_t item = item_of_slot(blockIdx.x, (int64_t)a.ntiles * a.nsplit * a.B * a.Hkv);
  const int split = (int)(item % a.nsplit);
  const int64_t rest = item / a.nsplit;
  const int tile = (int)(rest % a.ntiles), bh = (int)(rest / a.ntiles);
  const int b = bh / a.Hkv, kvh = bh % a.Hkv;
  const Seq sq(a, b);
  const int nrows = sq.q_len * a.group, r0 = tile * TQ;
  if (r0 >= nrows) return;
  KeyTiles kt;
  kt.init<TK>(a, sq, r0 / a.group, (min(r0 + TQ, nrows) - 1) / a.group);
  const int t_begin = (int)((int64_t)kt.nt * split / a.nsplit), t_end = (int)((int64_t)kt.nt * (split + 1) / a.nsplit);

  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, hh = lane >> 5;
  const int row = r0 + 32 * w + n;
  const bool live = row < nrows;
  const int qi = live ? row / a.group : 0, qh = kvh * a.group + (live ? row % a.group : 0);
  const int lo = sq.lo(a, qi), hi = live ? sq.hi(a, qi) : -1;

  x8 qf[R::kSteps];
  {
    const T* qp = static_cast<const T*>(a.q) + b * a.qs.b + qh * a.qs.h + qi * a.qs.n;
#pragma unroll
    for (int c = 0; c < R::kSteps; ++c) qf[c] = *reinterpret_cast<const x8*>(qp + 16 * c + 8 * hh);
  }

  Load lk, lv;
  lk.init(a.ks.n, w, lane);
  lv.init(a.vs.n, w, lane);
  const char* kb = reinterpret_cast<const char*>(static_cast<const T*>(a.k) + b * a.ks.b + kvh * a.ks.h);
  const char* vb = reinterpret_cast<const char*>(static_cast<const T*>(a.v) + b * a.vs.b + kvh * a.vs.h);
  // tiles past the slice load no row (they clear their slot)
  auto issue = [&](int t, uint8_t* s) {
    const int j = kt.key<TK>(t), rows = t < t_end ? kt.limit(t) - j : 0;
    lk.issue(kb + (int64_t)j * a.ks.n * 2, rows, s, w);
    lv.issue(vb + (int64_t)j * a.vs.n * 2, rows, s + kTile, w);
  };

  int koff[R::kSteps], voff[2][R::kBlocks];
#pragma unroll
  for (int c = 0; c < R::kSteps; ++c) koff[c] = R::row_read(lane, c);
#pragma unroll
  for (int r = 0; r < 2; ++r) {
#pragma unroll
    for (int d = 0; d < R::kBlocks; ++d) voff[r][d] = R::tr_read(lane, r, d);
  }

  f32x16 o[R::kBlocks];
#pragma unroll
  for (int d = 0; d < R::kBlocks; ++d) o[d] = f32x16{};
  float m = kNegInf, l = 0.f;
  // tiles between the highest first key and the lowest last key of the wave's
  // rows need no mask
  const int wave_last = min(r0 + 32 * w + 31, nrows - 1);
  const int full_lo = wave_last >= r0 + 32 * w ? sq.lo(a, wave_last / a.group) : kFar;
  const int full_hi = wave_last >= r0 + 32 * w ? sq.hi(a, (r0 + 32 * w) / a.group) : -1;

  if (t_begin < t_end) {
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) issue(t_begin + s, slot(s));
  }
  for (int t0 = t_begin; t0 < t_end; t0 += kStages) {
#pragma unroll
    for (int u = 0; u < kStages; ++u) {
      const int t = t0 + u;
      if (t >= t_end) break;
      wait_vm_lgkm<(kStages - 2) * kGroup>();
      block_sync();
      issue(t + kStages - 1, slot((u + kStages - 1) % kStages));
      const uint8_t* ks = slot(u);
      const uint8_t* vs = ks + kTile;
      const int j0 = kt.key<TK>(t);
      f32x16 s[kNKB];
#pragma unroll
      for (int kb2 = 0; kb2 < kNKB; ++kb2) {
        s[kb2] = f32x16{};
#pragma unroll
        for (int c = 0; c < R::kSteps; ++c)
          s[kb2] = E::mfma(*reinterpret_cast<const x8*>(ks + kb2 * 32 * R::kBytes + koff[c]), qf[c], s[kb2]);
      }
      const bool full = (j0 >= full_lo || j0 + TK <= a.sinks) && j0 + TK - 1 <= full_hi;
      if (!full) {
#pragma unroll
        for (int kb2 = 0; kb2 < kNKB; ++kb2) {
          const uint32_t bits = visible_bits(j0 + 32 * kb2, lo, hi, a.sinks) >> (4 * hh);
#pragma unroll
          for (int i = 0; i < 16; ++i) s[kb2][i] = (bits >> ((i >> 2) * 8 + (i & 3))) & 1u ? s[kb2][i] : kNegInf;
        }
      }
      float mx = kNegInf;
#pragma unroll
      for (int kb2 = 0; kb2 < kNKB; ++kb2) {
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[kb2][i]);
      }
      mx = fmaxf(mx, other_half(mx, lane)) * a.scale_log2;
      const float m_new = fmaxf(m, mx);
      const float ref = m_new == kNegInf ? 0.f : m_new;
      const float alpha = fast_exp2(m - ref);
      m = m_new;
      u32x4 p[2 * kNKB];
      float sum = 0.f;
#pragma unroll
      for (int kb2 = 0; kb2 < kNKB; ++kb2) {
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
          const float p0 = fast_exp2(__builtin_fmaf(s[kb2][i], a.scale_log2, -ref));
          const float p1 = fast_exp2(__builtin_fmaf(s[kb2][i + 1], a.scale_log2, -ref));
          sum += p0 + p1;
          p[2 * kb2 + i / 8][(i % 8) / 2] = pack2<T>(p0, p1);
        }
      }
      l = l * alpha + sum;
#pragma unroll
      for (int d = 0; d < R::kBlocks; ++d) o[d] *= alpha;
#pragma unroll
      for (int c = 0; c < 2 * kNKB; ++c) {
#pragma unroll
        for (int d = 0; d < R::kBlocks; ++d)
          o[d] = E::mfma(read_tr_pair<T>(vs + c * 16 * R::kBytes + voff[0][d], vs + c * 16 * R::kBytes + voff[1][d]),
                         __builtin_bit_cast(x8, p[c]), o[d]);
      }
    }
  }
  wait_vm_lgkm<0>();  // no load may still write LDS when the workgroup ends

  l += other_half(l, lane);
  if (!live) return;
  if (a.nsplit == 1) {
    const float inv = l > 0.f ? 1.f / l : 0.f;
    T* op = static_cast<T*>(a.o) + b * a.os.b + qh * a.os.h + qi * a.os.n;
#pragma unroll
    for (int d = 0; d < R::kBlocks; ++d) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        u32x2 v;
        v[0] = pack2<T>(o[d][4 * g] * inv, o[d][4 * g + 1] * inv);
        v[1] = pack2<T>(o[d][4 * g + 2] * inv, o[d][4 * g + 3] * inv);
        *reinterpret_cast<u32x2*>(op + d * 32 + 8 * g + 4 * hh) = v;
      }
    }
    if (a.lse && hh == 0) a.lse[((int64_t)b * a.H + qh) * a.Nq + qi] = l > 0.f ? (m + __log2f(l)) * kLn2 : kNegInf;
  } else {
    // state of the slice: [row][slice] of O, then of (m, l)
    const int64_t rows = (int64_t)a.B * a.Hkv * a.Nq * a.group;
    const int64_t at = ((int64_t)bh * a.Nq * a.group + row) * a.nsplit + split;
    float* po = a.part + at * D;
#pragma unroll
    for (int d = 0; d < R::kBlocks; ++d) {
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4*>(po + d * 32 + 8 * g + 4 * hh) =
            f32x4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
    }
    if (hh == 0) *reinterpret_cast<f32x2*>(a.part + rows * a.nsplit * D + 2 * at) = f32x2{m, l};
  }
#endif
}

// Joins the slices of a row: one wave per row, lane s holding the maximum and the
// sum of slice s, then D / 4 lanes per slice adding up O.
template <typename T, int D>
__global__ __launch_bounds__(256) void window_join_kernel(WindowArgs a) {
  const int lane = threadIdx.x & 63;
  const int per = a.Nq * a.group;
  const int64_t rows = (int64_t)a.B * a.Hkv * per;
  const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= rows) return;
  const int bh = (int)(r / per), row = (int)(r % per);
  const int b = bh / a.Hkv, kvh = bh % a.Hkv;
  const Seq sq(a, b);
  if (row >= sq.q_len * a.group) return;
  const float* ml = a.part + rows * a.nsplit * D + 2 * (r * a.nsplit);
  float m = kNegInf, l = 0.f;
  if (lane < a.nsplit) {
    m = ml[2 * lane];
    l = ml[2 * lane + 1];
  }
  float top = m;
#pragma unroll
  for (int x = 32; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
  const float wgt = m == kNegInf ? 0.f : fast_exp2(m - top);
  float sum = wgt * l;
#pragma unroll
  for (int x = 32; x; x >>= 1) sum += __shfl_xor(sum, x);
  constexpr int kCols = D / 4, kPar = 64 / kCols;
  const int col = (lane % kCols) * 4;
  const float* po = a.part + r * a.nsplit * D + col;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < a.nsplit; s0 += kPar) {
    const int s = s0 + lane / kCols;
    const float f = __shfl(wgt, s & 63);
    if (s < a.nsplit && f != 0.f) acc += f * *reinterpret_cast<const f32x4*>(po + (int64_t)s * D);
  }
#pragma unroll
  for (int x = kCols; x < 64; x <<= 1) {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], x);
  }
  const float inv = sum > 0.f ? 1.f / sum : 0.f;
  const int qi = row / a.group, qh = kvh * a.group + row % a.group;
  if (lane < kCols) {
    u32x2 v;
    v[0] = pack2<T>(acc[0] * inv, acc[1] * inv);
    v[1] = pack2<T>(acc[2] * inv, acc[3] * inv);
    *reinterpret_cast<u32x2*>(static_cast<T*>(a.o) + b * a.os.b + qh * a.os.h + qi * a.os.n + col) = v;
  }
  if (a.lse && lane == 0)
    a.lse[((int64_t)b * a.H + qh) * a.Nq + qi] = sum > 0.f ? (top + __log2f(sum)) * kLn2 : kNegInf;
}

template <typename T, int D>
hipError_t launch(const WindowArgs& a, const ForwardPlan& p, hipStream_t s) {
  const int64_t n = (int64_t)p.ntiles * p.nsplit * a.B * a.Hkv;
  if (n == 0) return hipSuccess;
  if (n > 0x7fffffff) return hipErrorInvalidValue;
  if (p.tile_rows == 32)
    hipLaunchKernelGGL((window_fwd_kernel<T, D, 1>), dim3((unsigned)n), dim3(64), 0, s, a);
  else
    hipLaunchKernelGGL((window_fwd_kernel<T, D, 4>), dim3((unsigned)n), dim3(256), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.nsplit == 1) return e;
  const int64_t rows = (int64_t)a.B * a.Hkv * a.Nq * a.group;
  hipLaunchKernelGGL((window_join_kernel<T, D>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

// A row tile of 32 rows (one wave) where no key head has more, else of 128 (four
// waves that share every K and V tile).  Where that gives too few workgroups for
// the card, each row tile's keys are cut into slices of at least four tiles.
ForwardPlan plan_forward(const WindowArgs& a, int d) {
  ForwardPlan p{};
  const int64_t rows = (int64_t)a.Nq * a.group;
  const int tk = 4096 / d;
  p.tile_rows = rows <= 32 ? 32 : 128;
  p.ntiles = (int32_t)((rows + p.tile_rows - 1) / p.tile_rows);
  const int64_t wgs = (int64_t)p.ntiles * a.B * a.Hkv;
  const int64_t want = p.tile_rows == 32 ? 1024 : 512;
  int64_t keys = (int64_t)a.left + a.right + 1 + (p.tile_rows + a.group - 1) / a.group;
  keys = keys < a.Nkv ? keys + (a.sinks < a.Nkv - keys ? a.sinks : a.Nkv - keys) : a.Nkv;
  int64_t split = wgs > 0 ? want / wgs : 1;
  const int64_t most = (keys + 4 * tk - 1) / (4 * tk);
  split = split < most ? split : most;
  split = split < kMaxSplit ? split : kMaxSplit;
  p.nsplit = (int32_t)(split > 1 ? split : 1);
  p.part_floats = p.nsplit > 1 ? (int64_t)a.B * a.Hkv * rows * p.nsplit * (d + 2) : 0;
  return p;
}

hipError_t launch_window_forward(int dtype, int d, const WindowArgs& args, hipStream_t s) {
  WindowArgs a = args;
  const ForwardPlan p = plan_forward(a, d);
  a.ntiles = p.ntiles;
  a.nsplit = p.nsplit;
  if (dtype == kBf16) return d == 128 ? launch<__bf16, 128>(a, p, s) : launch<__bf16, 64>(a, p, s);
  return d == 128 ? launch<_Float16, 128>(a, p, s) : launch<_Float16, 64>(a, p, s);
}

}  // namespace bsa_ops
