// Window attention forward for gfx950: a workgroup of NW waves owns 32 * NW rows
// (query tokens x the heads that share a key head), each wave 32 of them, and
// walks the keys that any of them sees - the first `sinks` and one contiguous
// range - in tiles of 8 or 16 KB of K and as much of V that come straight from memory
// to a ring in LDS.
//
// Scores are computed transposed, S^T = K Q^T (v_mfma 32x32x16): a lane then owns
// one row and 16 keys of each 32, so the softmax state is one number per lane and
// O^T += V^T P^T takes the lane's own probabilities as its operand.
//
// P is rounded to the tensors' type for that product, whose operands the matrix unit
// takes in 16 bits: each weight is off by half a step at most, which adds 0.001
// (relative, root mean square, bf16) to the 0.0017 of the rounding of O itself.  The sum
// is that of the weights before.
#include "window_common.h"

// (Kernel bodies are kept from the host's pass, which drops the launch stub of a
// template whose device builtins it cannot check.)

namespace bsa_ops {

namespace {

constexpr int kMaxSplit = 256;
constexpr float kSlack = 8.f;

// Inline asm must not read a matrix instruction's result too early: the compiler
// keeps the required distance for its own instructions only.
template <int N>
__device__ inline void settle(f32x16 (&x)[N]) {
  static_assert(N == 1 || N == 2, "score blocks of a tile");
  if constexpr (N == 1) asm volatile("s_nop 15\n\ts_nop 7" : "+v"(x[0]));
  else asm volatile("s_nop 15\n\ts_nop 7" : "+v"(x[0]), "+v"(x[1]));
}

// Maximum of three numbers; of NaN and a number, the number.
__device__ inline float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// O of the rows `mine` of a wave again, unnormalised, in place of o.  The products of a
// tile add 0 times V for the keys that a row does not see, which is NaN where V is not
// finite; rows that come out so are formed again here, with such values taken out of the
// products (0 in their place).  What a row sees of them is added from a product of its own:
// 1 for a visible key, else 0, times 1 for infinity, 32 for -infinity and 33 for NaN.  Its
// sums over 16 keys are whole numbers that both types and 32 bits hold, and tell the three
// apart.  (A key whose score is -inf has no weight and adds nothing.)
//
// A lane reads its own elements of K and V from memory: the other waves of the workgroup
// may have ended, so there is no barrier, and the ring is not touched.  (28800 queries, 24
// heads of 128, 14401 keys around each and 3600 sinks: 4.9 ms, with one infinity in the
// first value of every head 34 ms, with one in every value 39, of infinities alone 55.)
template <typename T, int D, int TK>
__device__ inline void rows_again(const WindowArgs& a, const KeyTiles& kt, int t_begin, int t_end, int b, int kvh, int qi,
                                  int qh, int lo, int hi, float m, bool mine, int lane, f32x16* o) {
  using E = Elem<T>;
  using R = Rows<D>;
  typedef typename E::x8 x8;
  const int n = lane & 31, hh = lane >> 5;
  const T* q = static_cast<const T*>(a.q) + b * a.qs.b + qh * a.qs.h + qi * a.qs.n + 8 * hh;
  const T* k = static_cast<const T*>(a.k) + b * a.ks.b + kvh * a.ks.h + 8 * hh;
  const T* v = static_cast<const T*>(a.v) + b * a.vs.b + kvh * a.vs.h + n;
  const float ref = m == kNegInf ? 0.f : m;
#pragma unroll
  for (int d = 0; d < R::kBlocks; ++d) {
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = mine ? 0.f : o[d][i];
  }
  for (int t = t_begin; t < t_end; ++t) {
    const int end = kt.limit(t);  // of the tile's keys
    for (int j0 = kt.key<TK>(t), jt = min(j0 + TK, end); j0 < jt; j0 += 32) {
      const uint32_t bits = mine ? visible_bits(j0, lo, min(hi, end - 1), a.sinks) : 0u;
      if (__ballot(bits != 0) == 0) continue;
      f32x16 s = {};
#pragma unroll
      for (int c = 0; c < R::kSteps; ++c) {
        x8 kf = {};
        if (j0 + n < end) kf = *reinterpret_cast<const x8*>(k + (j0 + n) * a.ks.n + 16 * c);
        s = E::mfma(kf, *reinterpret_cast<const x8*>(q + 16 * c), s);
      }
      u32x4 p[2], one[2];
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const uint32_t see = bits >> (4 * hh + (i >> 2) * 8 + (i & 3));
        const bool s0 = (see & 1u) && s[i] > kNegInf, s1 = (see & 2u) && s[i + 1] > kNegInf;
        p[i / 8][(i % 8) / 2] = pack2<T>(s0 ? fast_exp2(__builtin_fmaf(s[i], a.scale_log2, -ref)) : 0.f,
                                         s1 ? fast_exp2(__builtin_fmaf(s[i + 1], a.scale_log2, -ref)) : 0.f);
        one[i / 8][(i % 8) / 2] = pack2<T>(s0 ? 1.f : 0.f, s1 ? 1.f : 0.f);
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        x8 x[R::kBlocks];  // V by columns, its 16 keys in the order that the probabilities have
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int key = j0 + 16 * c + 8 * (e >> 2) + 4 * hh + (e & 3);
#pragma unroll
          for (int d = 0; d < R::kBlocks; ++d) x[d][e] = key < end ? v[key * a.vs.n + 32 * d] : (T)0.f;
        }
#pragma unroll
        for (int d = 0; d < R::kBlocks; ++d) {
          bool bad = false;
#pragma unroll
          for (int e = 0; e < 8; ++e) bad |= !(fabsf((float)x[d][e]) < __builtin_huge_valf());
          if (__ballot(bad) != 0) {
            x8 code;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float f = (float)x[d][e];
              const bool fin = fabsf(f) < __builtin_huge_valf();
              code[e] = (T)(fin ? 0.f : f > 0.f ? 1.f : f < 0.f ? 32.f : 33.f);
              x[d][e] = fin ? x[d][e] : (T)0.f;
            }
            const f32x16 sees = E::mfma(code, __builtin_bit_cast(x8, one[c]), f32x16{});
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int w = (int)sees[i];
              if (w & 31) o[d][i] += __builtin_huge_valf();
              if (w >> 5) o[d][i] += kNegInf;
            }
          }
          o[d] = E::mfma(x[d], __builtin_bit_cast(x8, p[c]), o[d]);
        }
      }
    }
  }
}

// Ends a wave's work: O and LSE of its rows, or the state of its slice of the keys
// for the join.
template <typename T, int D, int TK>
__device__ inline void store_rows(const WindowArgs& a, const KeyTiles& kt, int t_begin, int t_end, f32x16* o, float m,
                                  float l, bool live, int lo, int hi, int b, int bh, int qi, int qh, int row, int split,
                                  int lane) {
  using R = Rows<D>;
  const int hh = lane >> 5;
  l += other_half(l, lane);
  float zero = 0.f;  // NaN where a column is not finite
#pragma unroll
  for (int d = 0; d < R::kBlocks; ++d) {
#pragma unroll
    for (int i = 0; i < 16; ++i) zero = __builtin_fmaf(o[d][i], 0.f, zero);
  }
  // (a sum that is not finite itself says that the row saw such a key)
  const uint64_t again = __ballot(live && zero != 0.f && l < __builtin_huge_valf());
  if (__builtin_expect(again != 0, 0)) {
    const uint32_t rows = (uint32_t)again | (uint32_t)(again >> 32);
    rows_again<T, D, TK>(a, kt, t_begin, t_end, b, bh % a.Hkv, qi, qh, lo, hi, m, (rows >> (lane & 31)) & 1u, lane, o);
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int64_t rows = (int64_t)a.B * a.Hkv * a.Nq * a.group;
  // state of a slice: [row][slice] of O, then of (m, l)
  const int64_t at = ((int64_t)bh * a.Nq * a.group + row) * a.nsplit + split;
  T* op = static_cast<T*>(a.o) + b * a.os.b + qh * a.os.h + qi * a.os.n;
  float* po = a.part + at * D;
  if (live) {
    if (a.nsplit == 1) {
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
      if (a.lse && hh == 0) a.lse[((int64_t)b * a.H + qh) * a.Nq + qi] = l == 0.f ? kNegInf : (m + __log2f(l)) * kLn2;
    } else {
#pragma unroll
      for (int d = 0; d < R::kBlocks; ++d) {
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<f32x4*>(po + d * 32 + 8 * g + 4 * hh) =
              f32x4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
      }
      if (hh == 0) *reinterpret_cast<f32x2*>(a.part + rows * a.nsplit * D + 2 * at) = f32x2{m, l};
    }
  }
}

// One wave: single tokens and few rows, bound by the memory that K and V come from (64
// streams of 4096 visible keys, 8 key heads of 128: 188 us, 5.6 TB/s).  Four waves: head
// dim 64, where the exponentials take the vector unit 26 cycles for the 16 that the
// products take the matrix unit; four waves per SIMD overlap the two.
template <typename T, int D, int NW>
__global__ __launch_bounds__(64 * NW, NW == 4 ? 4 : 1) void window_fwd_kernel(WindowArgs a) {
#ifdef __HIP_DEVICE_COMPILE__
  using E = Elem<T>;
  using R = Rows<D>;
  typedef typename E::x8 x8;
  constexpr int TK = kTileKeys<D>, TQ = 32 * NW, kStages = 2;
  constexpr int kNKB = TK / 32, kTile = TK * R::kBytes;
  static_assert(kTile == 8192, "K and V tiles are 8 KB");
  using Load = TileLoad<D, TK, NW>;
  constexpr int kGroup = 2 * Load::kLoads;  // loads of one tile pair per wave
  // each slot is an array of its own: the compiler then sees that reads of one
  // never alias the loads that fill another, and leaves those in flight
  __shared__ __attribute__((aligned(1024))) uint8_t ring0[2 * kTile];
  __shared__ __attribute__((aligned(1024))) uint8_t ring1[2 * kTile];
  auto slot = [&](int i) -> uint8_t* { return i == 0 ? ring0 : ring1; };

  int b;
  const uint32_t item = item_of_slot(a, blockIdx.x, (uint32_t)a.ntiles * a.nsplit, &b);
  const int split = (int)(item % a.nsplit), rest = (int)(item / a.nsplit);
  const int tile = tile_of(a, rest % a.ntiles), kvh = rest / a.ntiles, bh = b * a.Hkv + kvh;
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
      const int last = kt.limit(t) - 1;
      const bool full = (j0 >= full_lo || j0 + TK <= a.sinks) && j0 + TK - 1 <= min(full_hi, last);
      if (!full) {
#pragma unroll
        for (int kb2 = 0; kb2 < kNKB; ++kb2) {
          const uint32_t bits = visible_bits(j0 + 32 * kb2, lo, min(hi, last), a.sinks) >> (4 * hh);
#pragma unroll
          for (int i = 0; i < 16; ++i) s[kb2][i] = (bits >> ((i >> 2) * 8 + (i & 3))) & 1u ? s[kb2][i] : kNegInf;
        }
      }
      // The reference is raised only where the maximum passes it by more than 2^8:
      // below that, sums in 32 bits and 16-bit probabilities hold them as well.
      float mx = kNegInf;
      settle(s);
#pragma unroll
      for (int kb2 = 0; kb2 < kNKB; ++kb2) {
#pragma unroll
        for (int i = 0; i < 16; i += 2) mx = max3(mx, s[kb2][i], s[kb2][i + 1]);
      }
      mx = max3(mx, mx, other_half(mx, lane)) * a.scale_log2;
      if (__ballot(mx > m + kSlack) != 0) {
        const float m_new = mx > m + kSlack ? mx : m;  // (-inf + 8 is -inf: the first key counts)
        const float alpha = m_new == m ? 1.f : fast_exp2(m - m_new);
        m = m_new;
        l *= alpha;
#pragma unroll
        for (int d = 0; d < R::kBlocks; ++d) o[d] *= alpha;
      }
      const float ref = m == kNegInf ? 0.f : m;
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
      l += sum;
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

  store_rows<T, D, TK>(a, kt, t_begin, t_end, o, m, l, live, lo, hi, b, bh, qi, qh, row, split, lane_now());
#endif
}

// x = keep ? x : -inf, in place (keep is per lane).  The tied operand pins the
// result to its register: written plainly, the compiler copies the scores on the
// common path, where nothing is masked.  (The condition may have been written by the
// instruction before: the compiler adds no wait states for inline asm.)
__device__ inline void mask_inplace(float& x, bool keep) {
  const float ninf = kNegInf;
  asm volatile("s_nop 1\n\tv_cndmask_b32_e64 %0, %1, %0, %2" : "+v"(x) : "v"(ninf), "s"(__ballot(keep)));
}

// The kernel for 128-row tiles of head dim 128: four waves of 32 rows, tiles of 64
// keys, two workgroups per CU.  The vector unit has nearly as much to do as the
// matrix unit (per score an fma, an exponential at a quarter of the rate, an add
// and half a conversion: 26 of the 32 cycles of its share of the products), so the
// two overlap within a wave: an iteration computes the scores of tile t + 1 and
// O += P V of tile t - 1 while it forms the probabilities of tile t, one
// exponential per matrix instruction.
//
// The reference that a row's probabilities are formed against is not moved tile by
// tile: they are formed against the current one, and their sum is checked before
// any product uses them.  Only where it passes 2^8 (or is NaN), or the row meets its
// first key, the reference is raised to the row's maximum, O is rescaled and the
// probabilities are formed again.  That and the masking of the next tile's scores
// share one rare branch: with one for each, the state no longer fits the registers.
//
// Slot j of the ring holds K of a tile x = j (mod 2) and V of tile x - 2: iteration
// t reads slot t + 1 (mod 2) and refills the other.
//
// 115200 queries, 24 heads, 14401 keys around each and 3600 sinks: 20.6 ms (1190
// TFLOP/s of visible pairs; the same work without the overlap within a wave 23.2 ms;
// eight waves and 256 rows 21.1; two groups of 32 rows per wave, which halve the LDS
// reads but leave one wave per SIMD, 23.7; 32-key tiles 21.6).
template <typename T, int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2)))
void window_fwd_piped_kernel(WindowArgs a) {
#ifdef __HIP_DEVICE_COMPILE__
  using E = Elem<T>;
  using R = Rows<D>;
  typedef typename E::x8 x8;
  constexpr int NW = 4, TQ = 32 * NW, TK = 64, kStages = 2;
  constexpr int kNKB = TK / 32, kTile = TK * R::kBytes;
  using Load = TileLoad<D, TK, NW>;
  constexpr int kLoads = Load::kLoads, kGroup = 2 * kLoads;
  __shared__ __attribute__((aligned(1024))) uint8_t ring0[2 * kTile];
  __shared__ __attribute__((aligned(1024))) uint8_t ring1[2 * kTile];
  auto kslot = [&](int i) BSA_INLINE -> uint8_t* { return i == 0 ? ring0 : ring1; };
  auto vslot = [&](int i) BSA_INLINE -> uint8_t* { return kslot(i) + kTile; };

  int b;
  const uint32_t item = item_of_slot(a, blockIdx.x, (uint32_t)a.ntiles * a.nsplit, &b);
  const int split = (int)(item % a.nsplit), rest = (int)(item / a.nsplit);
  const int tile = tile_of(a, rest % a.ntiles), kvh = rest / a.ntiles, bh = b * a.Hkv + kvh;
  const Seq sq(a, b);
  const int nrows = sq.q_len * a.group, r0 = tile * TQ;
  if (r0 >= nrows) return;
  KeyTiles kt;
  kt.init<TK>(a, sq, r0 / a.group, (min(r0 + TQ, nrows) - 1) / a.group);
  const int t_begin = (int)((int64_t)kt.nt * split / a.nsplit), t_end = (int)((int64_t)kt.nt * (split + 1) / a.nsplit);

  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, hh = lane >> 5;
  const int rw = r0 + 32 * w;  // the wave's first row
  const int row = rw + n;
  const bool live = row < nrows;
  const int qi = live ? row / a.group : 0, qh = kvh * a.group + (live ? row % a.group : 0);
  const int lo = sq.lo(a, qi), hi = live ? sq.hi(a, qi) : -1;
  x8 qf[R::kSteps];
  {
    const T* qp = static_cast<const T*>(a.q) + b * a.qs.b + qh * a.qs.h + qi * a.qs.n;
#pragma unroll
    for (int c = 0; c < R::kSteps; ++c) qf[c] = *reinterpret_cast<const x8*>(qp + 16 * c + 8 * hh);
  }
  // tiles that need no mask for any row of the wave
  const int wave_last = min(rw + 31, nrows - 1);
  const int full_lo = wave_last >= rw ? sq.lo(a, wave_last / a.group) : kFar;
  const int full_hi = wave_last >= rw ? sq.hi(a, rw / a.group) : -1;
  auto all_seen = [&](int t) BSA_INLINE -> bool {
    const int j0 = kt.key<TK>(t);
    return (j0 >= full_lo || j0 + TK <= a.sinks) && j0 + TK - 1 <= min(full_hi, kt.limit(t) - 1);
  };

  Load lk, lv;
  lk.init(a.ks.n, w, lane);
  lv.init(a.vs.n, w, lane);
  const char* kb = reinterpret_cast<const char*>(static_cast<const T*>(a.k) + b * a.ks.b + kvh * a.ks.h);
  const char* vb = reinterpret_cast<const char*>(static_cast<const T*>(a.v) + b * a.vs.b + kvh * a.vs.h);
  // tiles past the last load no row
  auto k_rsrc = [&](int t) BSA_INLINE {
    const int j = kt.key<TK>(t);
    return lk.rsrc(kb + (int64_t)j * a.ks.n * 2, t < t_end ? kt.limit(t) - j : 0);
  };
  auto v_rsrc = [&](int t) BSA_INLINE {
    const int j = kt.key<TK>(t);
    return lv.rsrc(vb + (int64_t)j * a.vs.n * 2, t < t_end ? kt.limit(t) - j : 0);
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
  float m_run = kNegInf, l_run = 0.f;

  // Operands of one iteration: units [0, kNA) are the scores of the next tile,
  // [kNA, kNU) O += P V of the previous one.
  constexpr int kNA = R::kSteps * kNKB, kNB = R::kBlocks * (TK / 16), kNU = kNA + kNB;
  auto load_op = [&](int u, const uint8_t* ks, const uint8_t* vs) BSA_INLINE -> x8 {
    if (u < kNA) return *reinterpret_cast<const x8*>(ks + (u % kNKB) * 32 * R::kBytes + koff[u / kNKB]);
    const int j = u - kNA, c = j / R::kBlocks, d = j % R::kBlocks;
    return read_tr_pair<T>(vs + c * 16 * R::kBytes + voff[0][d], vs + c * 16 * R::kBytes + voff[1][d]);
  };
  constexpr int kE = 16 * kNKB, kChunks = TK / 16;  // scores of a lane, chunks of 8 probabilities
  constexpr int kDmaEvery = kNU / kGroup;
  static_assert(kDmaEvery >= 1, "refill loads must fit the units");
  constexpr int kAhead = 3;
  auto a_end = [&](int u) BSA_INLINE -> int { return u < 0 ? 0 : u < kNU - 1 ? (u + 1) * kE / (kNU - 1) : kE; };
  constexpr float kSumMax = 256.f;
  const float c_log2 = a.scale_log2;

  auto apply_mask = [&](f32x16* s, int t) BSA_INLINE {
    const int j0 = kt.key<TK>(t), last = kt.limit(t) - 1;
#pragma unroll
    for (int kb2 = 0; kb2 < kNKB; ++kb2) {
      const uint32_t mine = visible_bits(j0 + 32 * kb2, lo, min(hi, last), a.sinks) >> (4 * hh);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float x = s[kb2][i];
        mask_inplace(x, (mine >> ((i >> 2) * 8 + (i & 3))) & 1u);
        s[kb2][i] = x;
      }
    }
  };
  auto exponent = [&](float sv, float nm) BSA_INLINE { return fast_exp2(__builtin_fmaf(sv, c_log2, nm)); };

  // Scores of tile t + 1 into s_nxt, O += P V of tile t - 1, the probabilities of
  // tile t (scores s_cur) into pw_cur; returns the lane's sum of them.
  auto iteration = [&](const f32x16* s_cur, f32x16* s_nxt, const uint8_t* ks_next, const uint8_t* vs_prev, u32x4* pw_cur,
                       const u32x4* pw_prev, int t, uint8_t* k_refill, uint8_t* v_refill) BSA_INLINE -> float {
    const float nm = m_run == kNegInf ? 0.f : -m_run;
    const __amdgpu_buffer_rsrc_t kr = k_rsrc(t + kStages), vr = v_rsrc(t + kStages - 2);
    float ls[2] = {0.f, 0.f};
    float pf[kE];
    auto stage_a = [&](int e) BSA_INLINE { pf[e] = exponent(s_cur[e / 16][e % 16], nm); };
    auto stage_b = [&](int pr) BSA_INLINE {
      const int e0 = 2 * pr;
      uint32_t pair = pack2<T>(pf[e0], pf[e0 + 1]);
      float& acc = ls[pr & 1];
      acc += pf[e0] + pf[e0 + 1];
      // keep both here: otherwise they are sunk past the check of the sum, and every
      // probability is held in 32 bits until then
      asm volatile("" : "+v"(acc), "+v"(pair));
      pw_cur[e0 / 8][(e0 % 8) / 2] = pair;
    };
    x8 op[kAhead + 1];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) op[u] = load_op(u, ks_next, vs_prev);
#pragma unroll
    for (int u = 0; u < kNU; ++u) {
      if (u + kAhead < kNU) op[(u + kAhead) % (kAhead + 1)] = load_op(u + kAhead, ks_next, vs_prev);
      if (u % kDmaEvery == 0 && u / kDmaEvery < kGroup) {
        const int i = u / kDmaEvery;
        if (i < kLoads) lk.one(kr, i, k_refill, w);
        else lv.one(vr, i - kLoads, v_refill, w);
      }
      if (u < kNA) {
        f32x16& acc = s_nxt[u % kNKB];
        acc = E::mfma(op[u % (kAhead + 1)], qf[u / kNKB], u < kNKB ? f32x16{} : acc);
      } else {
        const int j = u - kNA, d = j % R::kBlocks;
        o[d] = E::mfma(op[u % (kAhead + 1)], __builtin_bit_cast(x8, pw_prev[j / R::kBlocks]), o[d]);
      }
      // a pair is packed one step after its exponentials, so nothing waits for one
#pragma unroll
      for (int pr = a_end(u - 2) / 2; pr < a_end(u - 1) / 2; ++pr) stage_b(pr);
#pragma unroll
      for (int e = a_end(u - 1); e < a_end(u); ++e) stage_a(e);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int pr = a_end(kNU - 2) / 2; pr < kE / 2; ++pr) stage_b(pr);
    return ls[0] + ls[1];
  };

  // For the flagged rows: raise the reference to the maximum so far, rescale O and
  // l, and form the tile's probabilities again.  Other rows keep theirs to the bit.
  auto raise_reference = [&](const f32x16* s_cur, u32x4* pw_cur, bool mine, float sum_old) BSA_INLINE -> float {
    float mx = kNegInf;
#pragma unroll
    for (int kb2 = 0; kb2 < kNKB; ++kb2) {
#pragma unroll
      for (int i = 0; i < 16; i += 2) mx = max3(mx, s_cur[kb2][i], s_cur[kb2][i + 1]);
    }
    mx = max3(mx, mx, other_half(mx, lane)) * c_log2;
    const float m_new = mine ? max3(m_run, m_run, mx) : m_run;
    const float alpha = m_new == m_run ? 1.f : fast_exp2(m_run - m_new);
    m_run = m_new;
    l_run *= alpha;
#pragma unroll
    for (int d = 0; d < R::kBlocks; ++d) o[d] *= alpha;
    const float nm = m_new == kNegInf ? 0.f : -m_new;
    float ls[2] = {0.f, 0.f};
#pragma unroll
    for (int pr = 0; pr < kE / 2; ++pr) {
      const int e0 = 2 * pr;
      const float p0 = exponent(s_cur[e0 / 16][e0 % 16], nm), p1 = exponent(s_cur[e0 / 16][e0 % 16 + 1], nm);
      pw_cur[e0 / 8][(e0 % 8) / 2] = pack2<T>(p0, p1);
      ls[pr & 1] += p0 + p1;
    }
    return mine ? ls[0] + ls[1] : sum_old;
  };

  f32x16 sA[kNKB], sB[kNKB];
  u32x4 pwA[kChunks], pwB[kChunks];
#pragma unroll
  for (int c = 0; c < kChunks; ++c) pwB[c] = u32x4{};  // P of the tile before the first
  if (t_begin < t_end) {
    // slot 0 <- K of the first tile; slot 1 <- K of the next one, and the first V, which
    // the zeros of pwB multiply
    lk.issue(kb + (int64_t)kt.key<TK>(t_begin) * a.ks.n * 2, kt.limit(t_begin) - kt.key<TK>(t_begin), kslot(0), w);
    const __amdgpu_buffer_rsrc_t kr = k_rsrc(t_begin + 1), vr = v_rsrc(t_begin);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) lk.one(kr, j, kslot(1), w);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) lv.one(vr, j, vslot(1), w);
    wait_vm_lgkm<kGroup>();
    block_sync();
#pragma unroll
    for (int u = 0; u < kNA; ++u) {
      f32x16& acc = sA[u % kNKB];
      acc = E::mfma(load_op(u, kslot(0), nullptr), qf[u / kNKB], u < kNKB ? f32x16{} : acc);
    }
    settle(sA);
    apply_mask(sA, t_begin);
    wait_vm_lgkm<0>();
    block_sync();  // every wave has read slot 0 before it is refilled
  }
  for (int t0 = t_begin; t0 < t_end; t0 += kStages) {
    each_slot<kStages>([&](auto slot) BSA_INLINE -> bool {
      constexpr int u = decltype(slot)::value;
      const int t = t0 + u;
      if (t >= t_end) return false;
      f32x16* s_cur = u == 0 ? sA : sB;
      f32x16* s_nxt = u == 0 ? sB : sA;
      u32x4* pw_cur = u == 0 ? pwA : pwB;
      float sum = iteration(s_cur, s_nxt, kslot(1 - u), vslot(1 - u), pw_cur, u == 0 ? pwB : pwA, t, kslot(u), vslot(u));
      // (the sum is >= 0 or NaN, which as an integer is above every number)
      const int j0 = kt.key<TK>(t);
      const bool raise = __float_as_uint(sum) > __float_as_uint(kSumMax) ||
                         (m_run == kNegInf && j0 <= hi && (j0 + TK > lo || j0 < a.sinks));
      if (__builtin_expect(__ballot(raise) != 0 || !all_seen(t + 1), 0)) {
        // both halves of a row take the same decision
        const float mine = raise ? 1.f : 0.f;
        sum = raise_reference(s_cur, pw_cur, mine + other_half(mine, lane) > 0.f, sum);
        apply_mask(s_nxt, t + 1);
      }
      l_run += sum;
      wait_vm_lgkm<0>();
      block_sync();
      return true;
    });
  }
  if (t_begin < t_end) {
    // O += P V of the last tile
    const bool even = (t_end - 1 - t_begin) % 2 == 0;
    const u32x4* pw_last = even ? pwA : pwB;
    const uint8_t* vs = even ? vslot(0) : vslot(1);
#pragma unroll
    for (int j = 0; j < kNB; ++j)
      o[j % R::kBlocks] = E::mfma(load_op(kNA + j, nullptr, vs), __builtin_bit_cast(x8, pw_last[j / R::kBlocks]), o[j % R::kBlocks]);
  }
  wait_vm_lgkm<0>();  // no load may still write LDS when the workgroup ends
  store_rows<T, D, TK>(a, kt, t_begin, t_end, o, m_run, l_run, live, lo, hi, b, bh, qi, qh, row, split, lane_now());
#endif
}

// Joins the slices of a row: W waves per row, D / 4 threads a slice, with the loads of
// four slices in flight per thread.  One wave does for eight slices; more are shared by
// the four waves of a workgroup (one row of 256 slices: 28 us with a wave per row, 12 with
// four; 128 rows of 16: 5.8 and 4.4; 1024 rows of eight: 4.7 and 4.8; 2048 rows of two:
// 4.1 and 5.4).
//
// A slice whose weight is 0 in 32 bits hands on what is not finite in it: its keys are
// seen, and their weight is above 0.  (Slices of no visible key hold zeros.)
template <typename T, int D, int W>
__global__ __launch_bounds__(256) void window_join_kernel(WindowArgs a) {
  constexpr int kCols = D / 4, kPar = 64 * W / kCols, kBatch = 4;
  __shared__ f32x4 red[W][kCols];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = a.Nq * a.group;
  const int64_t rows = (int64_t)a.B * a.Hkv * per;
  const int64_t r = (int64_t)blockIdx.x * (4 / W) + (W == 1 ? wave : 0);
  if (r >= rows) return;
  const int bh = (int)(r / per), row = (int)(r % per);
  const int b = bh / a.Hkv, kvh = bh % a.Hkv;
  const Seq sq(a, b);
  if (row >= sq.q_len * a.group) return;
  const float* ml = a.part + rows * a.nsplit * D + 2 * (r * a.nsplit);
  // every wave forms the common maximum and sum for itself
  float top = kNegInf, sum = 0.f;
  for (int s = lane; s < a.nsplit; s += 64) top = fmaxf(top, ml[2 * s]);
#pragma unroll
  for (int x = 32; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
  auto weight = [&](float m) { return m == kNegInf ? 0.f : fast_exp2(m - top); };  // (NaN where top is infinite)
  for (int s = lane; s < a.nsplit; s += 64) sum += weight(ml[2 * s]) * ml[2 * s + 1];
#pragma unroll
  for (int x = 32; x; x >>= 1) sum += __shfl_xor(sum, x);
  const int in_row = W == 1 ? lane : tid, par = in_row / kCols, col = in_row % kCols;
  const float* po = a.part + r * a.nsplit * D + 4 * col;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = par; s0 < a.nsplit; s0 += kBatch * kPar) {
    f32x4 v[kBatch];
    float f[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int s = s0 + i * kPar;
      f[i] = 0.f;
      if (s < a.nsplit) {
        f[i] = weight(ml[2 * s]);
        v[i] = *reinterpret_cast<const f32x4*>(po + (int64_t)s * D);
      }
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      if (f[i] != 0.f) {
        acc += f[i] * v[i];
      } else if (s0 + i * kPar < a.nsplit) {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += fabsf(v[i][e]) < __builtin_huge_valf() ? 0.f : v[i][e];
      }
  }
#pragma unroll
  for (int x = kCols; x < 64; x <<= 1) {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], x);
  }
  if constexpr (W > 1) {
    if (lane < kCols) red[wave][col] = acc;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int i = 1; i < W; ++i) acc += red[i][col];
  }
  if (lane >= kCols) return;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  const int qi = row / a.group, qh = kvh * a.group + row % a.group;
  const u32x2 v = {pack2<T>(acc[0] * inv, acc[1] * inv), pack2<T>(acc[2] * inv, acc[3] * inv)};
  *reinterpret_cast<u32x2*>(static_cast<T*>(a.o) + b * a.os.b + qh * a.os.h + qi * a.os.n + 4 * col) = v;
  if (a.lse && col == 0)
    a.lse[((int64_t)b * a.H + qh) * a.Nq + qi] = sum == 0.f ? kNegInf : (top + __log2f(sum)) * kLn2;
}

template <typename T, int D>
hipError_t launch(const WindowArgs& a, const ForwardPlan& p, hipStream_t s) {
  const int64_t n = (int64_t)p.ntiles * p.nsplit * a.B * a.Hkv;
  if (n == 0) return hipSuccess;
  const int64_t rows = (int64_t)a.B * a.Hkv * a.Nq * a.group;
  if (!fits_launch(n, p.tile_rows * 2) || (p.nsplit > 1 && !fits_launch(rows, 256))) return hipErrorInvalidConfiguration;
  if (p.tile_rows == 32)
    hipLaunchKernelGGL((window_fwd_kernel<T, D, 1>), dim3((unsigned)n), dim3(64), 0, s, a);
  else if constexpr (D == 128)
    hipLaunchKernelGGL((window_fwd_piped_kernel<T, D>), dim3((unsigned)n), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((window_fwd_kernel<T, D, 4>), dim3((unsigned)n), dim3(256), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.nsplit == 1) return e;
  if (p.nsplit <= 8) hipLaunchKernelGGL((window_join_kernel<T, D, 1>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((window_join_kernel<T, D, 4>), dim3((unsigned)rows), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

// A row tile of 32 rows (one wave) where no key head has more, else of 128 (four
// waves that share every K and V tile).  Where that gives too few workgroups for the
// card, each row tile's keys are cut into slices.
//
// One-wave kernel: five workgroups share a CU (32 KB rings).  1024 of them keep memory
// busy, and more only cost in the join, unless there are 256 without slices, which 2048
// even out better (64 streams of 4096 keys, 8 key heads: 203 us with 1024, 195 with
// 2048; 8 streams: 27 and 29).  A slice of two tiles is worth its part of the join where
// there are few (1027 keys, 8 key heads: 8.7 us, with four tiles 9.7), eight where there
// are many.
//
// Four-wave kernels: a slice's partial rows are written and read again, 66 KB each at
// head dim 128, so slices are weighed: a tile of 64 keys takes a workgroup 1.2 us (1.74
// with two on a CU), the join 4 us and 27 ns a slice and workgroup.  (96 row tiles of 504
// keys: 16.5 us whole, 29.7 in five slices; 3 row tiles of 8000 keys: 65 us in two
// slices, 20 in forty.)  These are head dim 128's; at 64 a tile takes 1.1 us (1.3 with two
// on a CU, 1.8 with three, 2.3 with four), near enough that the same weighing serves.
ForwardPlan plan_forward(const WindowArgs& a, int d) {
  ForwardPlan p{};
  const int64_t rows = (int64_t)a.Nq * a.group;
  p.tile_rows = rows <= 32 ? 32 : 128;
  p.ntiles = (int32_t)((rows + p.tile_rows - 1) / p.tile_rows);
  const int64_t wgs = (int64_t)p.ntiles * a.B * a.Hkv;
  int64_t keys = (int64_t)a.left + a.right + 1 + (p.tile_rows + a.group - 1) / a.group;
  keys = keys < a.Nkv ? keys + (a.sinks < a.Nkv - keys ? a.sinks : a.Nkv - keys) : a.Nkv;
  int64_t split = 1;
  if (p.tile_rows == 32 && wgs > 0) {
    const int64_t least = (wgs < 256 ? 2 : 8) * (4096 / d), most = (keys + least - 1) / least;
    split = (wgs < 256 ? 1024 : 2048) / wgs;
    split = split < most ? split : most;
  } else if (wgs > 0) {
    const int64_t tiles = (keys + 63) / 64;
    int64_t best = tiles * (wgs <= 256 ? 1200 : 1740);  // ns
    for (int64_t s = 2; s * wgs <= 512 && s <= tiles; ++s) {
      const int64_t t = (tiles + s - 1) / s * (s * wgs <= 256 ? 1200 : 1740) + 4000 + 27 * s * wgs * d / 128;
      if (t < best) {
        best = t;
        split = s;
      }
    }
  }
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
