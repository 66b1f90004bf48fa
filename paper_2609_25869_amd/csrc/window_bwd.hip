// Window attention backward for gfx950, in two kernels and without atomics:
//
//   dQ    walks the keys of 128 rows as the forward kernel does, forming the
//         probabilities again from the scores and the LSE, and also leaves every
//         row's D = sum(dO o O) and base-2 LSE in the workspace;
//   dK/dV walks, for 128 keys, the queries that see any of them, head by head.
//         Sinks are seen by every later query: a tile with sinks is cut into
//         slices of its queries, of about the length of the other tiles' walks,
//         and a third kernel adds the slices' sums up in order.  (8192 queries, 16
//         heads over 4 key heads, window 1024, 4 sinks: 1626 us in one piece, 190 so.)
//
//   P = exp(S - LSE), dS = P o (dO V^T - D)
//   dQ = scale dS K, dV = P^T dO, dK = scale dS^T Q
//
// In both a wave holds 32 of its own rows (queries, or keys) as operands in
// registers, and the products over the head dim come out with one of those per
// lane, which is the layout that the products over the walked rows need.  Two
// workgroups of four waves share a CU; walked rows come in tiles of 64 through two
// ring slots (with 32 and four slots, twice the barriers: dK/dV 6.9 ms for 6.3).
// Where there are too few workgroups for two on a CU, a second form of the dK/dV kernel
// makes up for the missing wave within one.
//
// P, and dS after its subtraction, are rounded to the tensors' type for the products
// (float16 holds dS below 2^-14 to 2^-25: scale the loss where gradients are that
// small), whose operands the matrix unit takes in 16 bits; D is formed from O as it was
// stored, which saves O in 32 bits between the passes.  Everything else is 32 bits.
//
// 28800 queries and keys, 24 heads, 7201 keys around each and 3600 sinks: dQ 4.4 ms
// (1160 TFLOP/s of its three products), dK/dV 6.3 ms (1090 of its four), where a large
// library product reaches 1381.
#include "window_common.h"

// (Kernel bodies are kept from the host's pass, which drops the launch stub of a
// template whose device builtins it cannot check.)

namespace bsa_ops {

namespace {

constexpr int kWaves = 4;

// ---------------------------------------------------------------- dQ
template <typename T, int D>
__global__ __launch_bounds__(64 * kWaves) void window_dq_kernel(WindowArgs a) {
#ifdef __HIP_DEVICE_COMPILE__
  using E = Elem<T>;
  using R = Rows<D>;
  typedef typename E::x8 x8;
  constexpr int TK = 64, TQ = 32 * kWaves, kStages = 2;
  constexpr int kTile = TK * R::kBytes;
  using Load = TileLoad<D, TK, kWaves>;
  constexpr int kGroup = 2 * Load::kLoads;
  __shared__ __attribute__((aligned(1024))) uint8_t ring0[2 * kTile];
  __shared__ __attribute__((aligned(1024))) uint8_t ring1[2 * kTile];
  auto slot = [&](int i) -> uint8_t* { return i == 0 ? ring0 : ring1; };

  int b;
  const uint32_t item = item_of_slot(a, blockIdx.x, (uint32_t)a.ntiles, &b);
  const int tile = tile_of(a, (int)(item % a.ntiles)), kvh = (int)(item / a.ntiles);
  const Seq sq(a, b);
  const int nrows = sq.q_len * a.group, r0 = tile * TQ;
  if (r0 >= nrows) return;
  KeyTiles kt;
  kt.init<TK>(a, sq, r0 / a.group, (min(r0 + TQ, nrows) - 1) / a.group);

  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, hh = lane >> 5;
  const int row = r0 + 32 * w + n;
  const bool live = row < nrows;
  const int qi = live ? row / a.group : 0, qh = kvh * a.group + (live ? row % a.group : 0);
  const int lo = sq.lo(a, qi), hi = live ? sq.hi(a, qi) : -1;

  x8 qf[R::kSteps], df[R::kSteps];
  float delta = 0.f;
  {
    const T* qp = static_cast<const T*>(a.q) + b * a.qs.b + qh * a.qs.h + qi * a.qs.n;
    const T* dp = static_cast<const T*>(a.dout) + b * a.dos.b + qh * a.dos.h + qi * a.dos.n;
    const T* op = static_cast<const T*>(a.o) + b * a.os.b + qh * a.os.h + qi * a.os.n;
#pragma unroll
    for (int c = 0; c < R::kSteps; ++c) {
      qf[c] = *reinterpret_cast<const x8*>(qp + 16 * c + 8 * hh);
      df[c] = *reinterpret_cast<const x8*>(dp + 16 * c + 8 * hh);
      const x8 of = *reinterpret_cast<const x8*>(op + 16 * c + 8 * hh);
#pragma unroll
      for (int e = 0; e < 8; ++e) delta += (float)df[c][e] * (float)of[e];
    }
    delta += other_half(delta, lane);
  }
  const float lse = a.lse[((int64_t)b * a.H + qh) * a.Nq + qi] * kLog2e;
  if (live && hh == 0) {
    float* st = a.stats + ((int64_t)b * a.H + qh) * 2 * a.stat_rows + qi;
    st[0] = lse;
    st[a.stat_rows] = delta;
  }

  Load lk, lv;
  lk.init(a.ks.n, w, lane);
  lv.init(a.vs.n, w, lane);
  const char* kb = reinterpret_cast<const char*>(static_cast<const T*>(a.k) + b * a.ks.b + kvh * a.ks.h);
  const char* vb = reinterpret_cast<const char*>(static_cast<const T*>(a.v) + b * a.vs.b + kvh * a.vs.h);
  auto issue = [&](int t, uint8_t* s) BSA_INLINE {
    const int j = kt.key<TK>(t), rows = t < kt.nt ? kt.limit(t) - j : 0;
    lk.issue(kb + (int64_t)j * a.ks.n * 2, rows, s, w);
    lv.issue(vb + (int64_t)j * a.vs.n * 2, rows, s + kTile, w);
  };
  // (chunk c of a row, and column block d, differ from the first by bits that the
  // swizzle only flips)
  const int roff = R::row_read(lane, 0), toff0 = R::tr_read(lane, 0, 0), toff1 = R::tr_read(lane, 1, 0);
  f32x16 acc[R::kBlocks];
#pragma unroll
  for (int d = 0; d < R::kBlocks; ++d) acc[d] = f32x16{};
  const int wave_last = min(r0 + 32 * w + 31, nrows - 1);
  const int full_lo = wave_last >= r0 + 32 * w ? sq.lo(a, wave_last / a.group) : kFar;
  const int full_hi = wave_last >= r0 + 32 * w ? sq.hi(a, (r0 + 32 * w) / a.group) : -1;

  if (kt.nt > 0) {
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) issue(s, slot(s));
  }
  for (int tb = 0; tb < kt.nt; tb += kStages) {
    each_slot<kStages>([&](auto at) BSA_INLINE -> bool {
      constexpr int u = decltype(at)::value;
      const int t = tb + u;
      if (t >= kt.nt) return false;
      wait_vm_lgkm<(kStages - 2) * kGroup>();
      block_sync();
      issue(t + kStages - 1, slot((u + kStages - 1) % kStages));
      auto half = [&](auto blk) BSA_INLINE {
        const uint8_t* ks = slot(u) + decltype(blk)::value * 32 * R::kBytes;
        const uint8_t* vs = ks + kTile;
        int ro = roff, t0 = toff0, t1 = toff1;
        asm volatile("" : "+v"(ro), "+v"(t0), "+v"(t1));  // formed again per tile: sixteen addresses would not fit
        const int j0 = kt.key<TK>(t) + decltype(blk)::value * 32;
        // operands in the order of their use: K and V in turn, then K again by columns
        constexpr int kAhead = 3, kRowUnits = 2 * R::kSteps, kTrUnits = 2 * R::kBlocks;
        auto load_op = [&](int i) BSA_INLINE -> x8 {
          if (i < kRowUnits) return *reinterpret_cast<const x8*>((i % 2 ? vs : ks) + (ro ^ ((i / 2) << 5)));
          const int j = i - kRowUnits, c = j / R::kBlocks, d = j % R::kBlocks;
          const uint8_t* rows = ks + c * 16 * R::kBytes;
          return read_tr_pair<T>(rows + (t0 ^ (d << 6)), rows + (t1 ^ (d << 6)));
        };
        x8 op[kAhead + 1];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) op[i] = load_op(i);
        f32x16 s = {}, dp = {};
#pragma unroll
        for (int i = 0; i < kRowUnits; ++i) {
          op[(i + kAhead) % (kAhead + 1)] = load_op(i + kAhead);
          if (i % 2 == 0) s = E::mfma(op[i % (kAhead + 1)], qf[i / 2], s);
          else dp = E::mfma(op[i % (kAhead + 1)], df[i / 2], dp);
          __builtin_amdgcn_sched_barrier(0);
        }
        float ds[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) ds[i] = fast_exp2(__builtin_fmaf(s[i], a.scale_log2, -lse)) * (dp[i] - delta);
        const int last = kt.limit(t) - 1;
        const bool full = (j0 >= full_lo || j0 + 32 <= a.sinks) && j0 + 31 <= min(full_hi, last);
        if (__builtin_expect(!full, 0)) {
          const uint32_t bits = visible_bits(j0, lo, min(hi, last), a.sinks) >> (4 * hh);
#pragma unroll
          for (int i = 0; i < 16; ++i) zero_unless(ds[i], (bits >> ((i >> 2) * 8 + (i & 3))) & 1u);
        }
        u32x4 p[2];
#pragma unroll
        for (int i = 0; i < 16; i += 2) p[i / 8][(i % 8) / 2] = pack2<T>(ds[i], ds[i + 1]);
#pragma unroll
        for (int i = 0; i < kTrUnits; ++i) {
          const int u_at = kRowUnits + i, c = i / R::kBlocks, d = i % R::kBlocks;
          if (i + kAhead < kTrUnits) op[(u_at + kAhead) % (kAhead + 1)] = load_op(u_at + kAhead);
          acc[d] = E::mfma(op[u_at % (kAhead + 1)], __builtin_bit_cast(x8, p[c]), acc[d]);
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      half(std::integral_constant<int, 0>{});
      half(std::integral_constant<int, 1>{});
      return true;
    });
  }
  wait_vm_lgkm<0>();
  if (!live) return;
  T* gp = static_cast<T*>(a.dq) + b * a.dqs.b + qh * a.dqs.h + qi * a.dqs.n;
#pragma unroll
  for (int d = 0; d < R::kBlocks; ++d) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      u32x2 v;
      v[0] = pack2<T>(acc[d][4 * g] * a.scale, acc[d][4 * g + 1] * a.scale);
      v[1] = pack2<T>(acc[d][4 * g + 2] * a.scale, acc[d][4 * g + 3] * a.scale);
      *reinterpret_cast<u32x2*>(gp + d * 32 + 8 * g + 4 * hh) = v;
    }
  }
#endif
}

// ---------------------------------------------------------------- dK, dV
// The queries that see key j: i from first(j) to last(j).
struct Seen {
  int off, q_last, left, right, sinks, kv_len;
  __device__ Seen(const WindowArgs& a, const Seq& s)
      : off(s.off), q_last(s.q_len - 1), left(a.left), right(a.right), sinks(a.sinks), kv_len(s.kv_len) {}
  __device__ int first(int j) const { return (int)min(max((int64_t)j - right - off, (int64_t)0), (int64_t)kFar); }
  __device__ int last(int j) const {
    if (j >= kv_len) return -1;
    return j < sinks ? q_last : (int)max(min((int64_t)j + left - off, (int64_t)q_last), (int64_t)-1);
  }
};

// Deep: one wave per SIMD with all the registers, three ring slots, and the products of
// a tile in one sequence that nothing interrupts: operands are read four products ahead,
// and the probabilities of one half are formed between the products of the other.  A tile
// of 64 rows takes a workgroup 2.3 us, where the plain kernel takes 3.3 alone on its CU
// and 3.9 with another beside it.  (Operands six ahead: the same.)
// Three workgroups share a CU at head dim 64 (16384 tokens, 16 heads, window 1024: 386 us
// for dQ, dK and dV with two, 357 with three).
template <typename T, int D, bool Deep>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(Deep ? 1 : D == 64 ? 3 : 2, Deep ? 1 : D == 64 ? 3 : 2)))
void window_dkv_kernel(WindowArgs a) {
#ifdef __HIP_DEVICE_COMPILE__
  using E = Elem<T>;
  using R = Rows<D>;
  typedef typename E::x8 x8;
  constexpr int TR = 64, TKEY = 32 * kWaves, kStages = Deep ? 3 : 2;
  constexpr int kTile = TR * R::kBytes, kStat = 512;
  using Load = TileLoad<D, TR, kWaves>;
  constexpr int kGroup = 2 * Load::kLoads + 2;
  constexpr int kSlot = 2 * kTile + kWaves * kStat;  // Q, dO, and LSE and D of the rows, a copy per wave
  __shared__ __attribute__((aligned(1024))) uint8_t ring0[kSlot];
  __shared__ __attribute__((aligned(1024))) uint8_t ring1[kSlot];
  __shared__ __attribute__((aligned(1024))) uint8_t ring2[Deep ? kSlot : 16];
  auto slot = [&](int i) -> uint8_t* { return i == 0 ? ring0 : i == 1 ? ring1 : ring2; };

  // The tiles without sinks of every head come first, then the others: each kind is
  // spread over the XCDs by itself (in one list, where some XCDs get most of the sinks'
  // slices: 270 us for 239 at 8192 queries, 16 heads over 4, window 1024, 4 sinks).
  const int plain = (a.nktiles - a.nsink) * a.slices;  // items per key head
  const uint32_t all_plain = (uint32_t)plain * a.Hkv * a.B;
  const bool sink = blockIdx.x >= all_plain;
  const int of_kind = sink ? a.nsink * a.sink_slices : plain, nslice = sink ? a.sink_slices : a.slices;
  int b;
  const uint32_t item = item_of_slot(a, blockIdx.x - (sink ? all_plain : 0), (uint32_t)of_kind, &b);
  const int kvh = (int)(item / of_kind), in_kind = (int)(item % of_kind), bh = b * a.Hkv + kvh;
  const int tile = in_kind / nslice + (sink ? 0 : a.nsink), slice = in_kind % nslice;
  const Seq sq(a, b);
  const int k0 = tile * TKEY;
  if (k0 >= sq.kv_len) return;
  const Seen seen(a, sq);
  // queries that see any key of the tile (a sink's last query is the sequence's last)
  const int i_lo = seen.first(k0);
  const int i_hi = k0 < a.sinks ? sq.q_len - 1 : seen.last(min(k0 + TKEY, sq.kv_len) - 1);
  const int per_head = max(i_hi - i_lo + TR, 0) / TR;  // row tiles
  const int64_t all = (int64_t)per_head * a.group;
  const int64_t t_begin = all * slice / nslice;
  const int nt = (int)(all * (slice + 1) / nslice - t_begin);

  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);

  x8 kf[R::kSteps], vf[R::kSteps];
  {
    const int own = k0 + 32 * w + (lane & 31), at = own < sq.kv_len ? own : k0, hh = lane >> 5;
    const T* kp = static_cast<const T*>(a.k) + b * a.ks.b + kvh * a.ks.h + at * a.ks.n;
    const T* vp = static_cast<const T*>(a.v) + b * a.vs.b + kvh * a.vs.h + at * a.vs.n;
#pragma unroll
    for (int c = 0; c < R::kSteps; ++c) {
      kf[c] = *reinterpret_cast<const x8*>(kp + 16 * c + 8 * hh);
      vf[c] = *reinterpret_cast<const x8*>(vp + 16 * c + 8 * hh);
    }
  }

  Load lq, ld;
  lq.init(a.qs.n, w, lane);
  ld.init(a.dos.n, w, lane);
  // the row tile that is loaded next, and the one that is worked on
  int g_in = per_head ? (int)(t_begin / per_head) : 0, i_in = i_lo + (per_head ? (int)(t_begin % per_head) : 0) * TR;
  int i_now = i_in;
  auto issue = [&](uint8_t* s) BSA_INLINE {
    const bool any = g_in < a.group;
    const int qh = kvh * a.group + (any ? g_in : 0), rows = any ? i_hi + 1 - i_in : 0;
    lq.issue(reinterpret_cast<const char*>(static_cast<const T*>(a.q) + b * a.qs.b + qh * a.qs.h + i_in * a.qs.n), rows, s, w);
    ld.issue(reinterpret_cast<const char*>(static_cast<const T*>(a.dout) + b * a.dos.b + qh * a.dos.h + i_in * a.dos.n), rows,
             s + kTile, w);
    const uint32_t stat_off = (uint32_t)lane_now() * 4;
    const float* st = a.stats + ((int64_t)b * a.H + qh) * 2 * a.stat_rows + i_in;
    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<float*>(st), 0, any ? (int)((a.stat_rows + TR) * 4) : 0, 0x00020000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        rsrc, (__attribute__((address_space(3))) void*)(s + 2 * kTile + w * kStat), 4, stat_off, 0, 0, 0);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        rsrc, (__attribute__((address_space(3))) void*)(s + 2 * kTile + w * kStat + 256), 4, stat_off, (int)(a.stat_rows * 4), 0, 0);
    i_in += TR;
    if (i_in > i_hi) {
      i_in = i_lo;
      ++g_in;
    }
  };

  // (chunk c of a row, and column block d, differ from the first by bits that the
  // swizzle only flips)
  const int roff = R::row_read(lane, 0), toff0 = R::tr_read(lane, 0, 0), toff1 = R::tr_read(lane, 1, 0);
  f32x16 dk[R::kBlocks], dv[R::kBlocks];
#pragma unroll
  for (int d = 0; d < R::kBlocks; ++d) {
    dk[d] = f32x16{};
    dv[d] = f32x16{};
  }
  // rows of a tile that every key of the wave is seen by
  const int kw = k0 + 32 * w;
  const int full_lo = seen.first(kw + 31);
  const int full_hi = kw + 31 >= sq.kv_len ? -1 : min(seen.last(kw), kw < a.sinks && kw + 31 >= a.sinks ? seen.last(a.sinks) : kFar);

  if (nt > 0) {
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) issue(slot(s));
  }
  for (int tb = 0; tb < nt; tb += kStages) {
    each_slot<kStages>([&](auto at) BSA_INLINE -> bool {
      constexpr int u = decltype(at)::value;
      const int t = tb + u;
      if (t >= nt) return false;
      wait_vm_lgkm<(kStages - 2) * kGroup>();
      block_sync();
      issue(slot((u + kStages - 1) % kStages));
      if constexpr (Deep) {
        int ro = roff, t0 = toff0, t1 = toff1;
        asm volatile("" : "+v"(ro), "+v"(t0), "+v"(t1));  // formed again per tile
        // Products in their order, kP of them a phase: scores (S, dP in turn) of half 0, of
        // half 1, then dV and dK in turn of half 0, of half 1.
        constexpr int kP = 2 * R::kSteps, kUnits = 4 * kP;
        static_assert(kP == 16, "a phase forms one of a lane's 16 probabilities per product");
        const uint8_t* qs = slot(u);
        const uint8_t* gs = qs + kTile;
        auto load_op = [&](int i) BSA_INLINE -> x8 {
          const int ph = i / kP, j = i % kP, rows = (ph & 1) * 32 * R::kBytes;
          if (ph < 2) return *reinterpret_cast<const x8*>((j % 2 ? gs : qs) + rows + (ro ^ ((j / 2) << 5)));
          const int c = j / (2 * R::kBlocks), d = j / 2 % R::kBlocks, o = rows + c * 16 * R::kBytes;
          const uint8_t* x = j % 2 ? qs : gs;
          return read_tr_pair<T>(x + o + (t0 ^ (d << 6)), x + o + (t1 ^ (d << 6)));
        };
        const uint8_t* st = slot(u) + 2 * kTile + w * kStat + 16 * (lane_now() >> 5);
        constexpr int kAhead = 4;
        x8 op[kAhead + 1];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) op[i] = load_op(i);
        f32x16 s[2] = {}, dp[2] = {};
        u32x4 p[2][2], q[2][2];
        float pv[16], ds[16];
        f32x4 lse[2], delta[2];
        auto load_stat = [&](int h, int r4) BSA_INLINE {
          lse[r4 & 1] = *reinterpret_cast<const f32x4*>(st + 128 * h + 32 * r4);
          delta[r4 & 1] = *reinterpret_cast<const f32x4*>(st + 128 * h + 256 + 32 * r4);
        };
        auto form = [&](int h, int e) BSA_INLINE {
          const int r4 = e / 4;
          if (e % 4 == 0 && r4 < 3) load_stat(h, r4 + 1);
          pv[e] = fast_exp2(__builtin_fmaf(s[h][e], a.scale_log2, -lse[r4 & 1][e % 4]));
          ds[e] = dp[h][e] - delta[r4 & 1][e % 4];
        };
        auto pack = [&](int h, int e) BSA_INLINE {
          p[h][e / 8][(e % 8) / 2] = pack2<T>(pv[e], pv[e + 1]);
          q[h][e / 8][(e % 8) / 2] = pack2<T>(pv[e] * ds[e], pv[e + 1] * ds[e + 1]);
        };
        auto mask = [&](int h) BSA_INLINE {
          const int i_blk = i_now + 32 * h;
          if (__builtin_expect(i_blk >= full_lo && i_blk + 31 <= full_hi, 1)) return;
          const int l = lane_now(), key = kw + (l & 31);
          const uint32_t bits = (bits_below(seen.last(key) - i_blk + 1) & ~bits_below(seen.first(key) - i_blk)) >> (4 * (l >> 5));
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            const uint32_t b2 = bits >> (8 * (i >> 2) + (i & 3));
            const uint32_t keep = (b2 & 1u ? 0xffffu : 0u) | (b2 & 2u ? 0xffff0000u : 0u);
            uint32_t x = p[h][i / 8][(i % 8) / 2], y = q[h][i / 8][(i % 8) / 2];
            asm volatile("v_and_b32 %0, %2, %0\n\tv_and_b32 %1, %2, %1" : "+v"(x), "+v"(y) : "v"(keep));
            p[h][i / 8][(i % 8) / 2] = x;
            q[h][i / 8][(i % 8) / 2] = y;
          }
        };
        each_slot<kUnits>([&](auto unit) BSA_INLINE -> bool {
          constexpr int i = decltype(unit)::value, ph = i / kP, j = i % kP;
          if (i + kAhead < kUnits) op[(i + kAhead) % (kAhead + 1)] = load_op(i + kAhead);
          const x8 x = op[i % (kAhead + 1)];
          if (j == kP - 1 && ph < 2) load_stat(ph, 0);
          if (ph < 2) {
            if (j % 2 == 0) s[ph] = E::mfma(x, kf[j / 2], s[ph]);
            else dp[ph] = E::mfma(x, vf[j / 2], dp[ph]);
          } else {
            const int c = j / (2 * R::kBlocks), d = j / 2 % R::kBlocks, h = ph - 2;
            if (j % 2 == 0) dv[d] = E::mfma(x, __builtin_bit_cast(x8, p[h][c]), dv[d]);
            else dk[d] = E::mfma(x, __builtin_bit_cast(x8, q[h][c]), dk[d]);
          }
          // half 0's probabilities beside the scores of half 1, half 1's beside the
          // products of half 0
          if (ph == 1 || ph == 2) {
            const int h = ph - 1;
            if (j > 0 && j % 2 == 0) pack(h, j - 2);
            form(h, j);
            if (j == kP - 1) {
              pack(h, 14);
              mask(h);
            }
          }
          __builtin_amdgcn_sched_barrier(0);
          return true;
        });
      } else {
        auto half = [&](auto blk) BSA_INLINE {
          constexpr int rb = decltype(blk)::value;
          const int i_blk = i_now + 32 * rb;
          const uint8_t* qs = slot(u) + rb * 32 * R::kBytes;
          const uint8_t* gs = qs + kTile;
          int ro = roff, t0 = toff0, t1 = toff1;
          asm volatile("" : "+v"(ro), "+v"(t0), "+v"(t1));  // formed again per tile: sixteen addresses would not fit
          const uint8_t* st = slot(u) + 2 * kTile + w * kStat + 128 * rb + 16 * (lane_now() >> 5);
          f32x16 s = {}, dp = {};
#pragma unroll
          for (int c = 0; c < R::kSteps; ++c) {
            s = E::mfma(*reinterpret_cast<const x8*>(qs + (ro ^ (c << 5))), kf[c], s);
            dp = E::mfma(*reinterpret_cast<const x8*>(gs + (ro ^ (c << 5))), vf[c], dp);
          }
          const bool full = i_blk >= full_lo && i_blk + 31 <= full_hi;
          float pv[16], ds[16];
#pragma unroll
          for (int r4 = 0; r4 < 4; ++r4) {
            const f32x4 lse = *reinterpret_cast<const f32x4*>(st + 32 * r4);
            const f32x4 delta = *reinterpret_cast<const f32x4*>(st + 256 + 32 * r4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int i = 4 * r4 + e;
              pv[i] = fast_exp2(__builtin_fmaf(s[i], a.scale_log2, -lse[e]));
              ds[i] = pv[i] * (dp[i] - delta[e]);
            }
            __builtin_amdgcn_sched_barrier(0);
          }
          if (__builtin_expect(!full, 0)) {
            const int l = lane_now(), key = kw + (l & 31);
            const uint32_t bits =
                (bits_below(seen.last(key) - i_blk + 1) & ~bits_below(seen.first(key) - i_blk)) >> (4 * (l >> 5));
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const bool see = (bits >> (8 * (i >> 2) + (i & 3))) & 1u;
              zero_unless(pv[i], see);
              zero_unless(ds[i], see);
            }
          }
          u32x4 p[2], q[2];
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            p[i / 8][(i % 8) / 2] = pack2<T>(pv[i], pv[i + 1]);
            q[i / 8][(i % 8) / 2] = pack2<T>(ds[i], ds[i + 1]);
          }
#pragma unroll
          for (int c = 0; c < 2; ++c) {
#pragma unroll
            for (int d = 0; d < R::kBlocks; ++d) {
              const int o0 = c * 16 * R::kBytes + (t0 ^ (d << 6)), o1 = c * 16 * R::kBytes + (t1 ^ (d << 6));
              dv[d] = E::mfma(read_tr_pair<T>(gs + o0, gs + o1), __builtin_bit_cast(x8, p[c]), dv[d]);
              dk[d] = E::mfma(read_tr_pair<T>(qs + o0, qs + o1), __builtin_bit_cast(x8, q[c]), dk[d]);
            }
          }
        };
        half(std::integral_constant<int, 0>{});
        half(std::integral_constant<int, 1>{});
      }
      i_now += TR;
      if (i_now > i_hi) i_now = i_lo;
      return true;
    });
  }
  wait_vm_lgkm<0>();
  const int end_lane = lane_now(), key = kw + (end_lane & 31), hh = end_lane >> 5;
  if (key >= sq.kv_len) return;
  if (nslice > 1) {
    // [slice][dK, dV][key][column]
    const int64_t first_part = sink && a.slices > 1 ? plain : 0;
    float* part = a.part + ((int64_t)bh * dkv_parts(a) + first_part + in_kind) * (2 * TKEY * D) + (key - k0) * D;
#pragma unroll
    for (int d = 0; d < R::kBlocks; ++d) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int c = d * 32 + 8 * g + 4 * hh;
        *reinterpret_cast<f32x4*>(part + c) = f32x4{dk[d][4 * g], dk[d][4 * g + 1], dk[d][4 * g + 2], dk[d][4 * g + 3]};
        *reinterpret_cast<f32x4*>(part + TKEY * D + c) =
            f32x4{dv[d][4 * g], dv[d][4 * g + 1], dv[d][4 * g + 2], dv[d][4 * g + 3]};
      }
    }
    return;
  }
  T* kp = static_cast<T*>(a.dk) + b * a.dks.b + kvh * a.dks.h + key * a.dks.n;
  T* vp = static_cast<T*>(a.dv) + b * a.dvs.b + kvh * a.dvs.h + key * a.dvs.n;
#pragma unroll
  for (int d = 0; d < R::kBlocks; ++d) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      u32x2 x, y;
      x[0] = pack2<T>(dk[d][4 * g] * a.scale, dk[d][4 * g + 1] * a.scale);
      x[1] = pack2<T>(dk[d][4 * g + 2] * a.scale, dk[d][4 * g + 3] * a.scale);
      y[0] = pack2<T>(dv[d][4 * g], dv[d][4 * g + 1]);
      y[1] = pack2<T>(dv[d][4 * g + 2], dv[d][4 * g + 3]);
      *reinterpret_cast<u32x2*>(kp + d * 32 + 8 * g + 4 * hh) = x;
      *reinterpret_cast<u32x2*>(vp + d * 32 + 8 * g + 4 * hh) = y;
    }
  }
#endif
}

// Adds up the slices of the key tiles that are cut: one workgroup per 1024 elements of a
// tile's dK or dV (8 keys of 128), four columns a thread, eight slices in flight (64
// slices of four tiles: 9 us, one by one 18).
template <typename T, int D>
__global__ __launch_bounds__(256) void window_dkv_sum_kernel(WindowArgs a) {
  constexpr int TKEY = 32 * kWaves;
  const int cut_plain = a.slices > 1 ? a.nktiles - a.nsink : 0, cut = cut_plain + (a.sink_slices > 1 ? a.nsink : 0);
  const int bh = blockIdx.x / cut, c = blockIdx.x % cut;
  const bool sink = c >= cut_plain;
  const int tile = sink ? c - cut_plain : c + a.nsink, nslice = sink ? a.sink_slices : a.slices;
  const int b = bh / a.Hkv, kvh = bh % a.Hkv;
  const Seq sq(a, b);
  const int at = ((int)blockIdx.y * 256 + (int)threadIdx.x) * 4;  // in the tile's [key][column]
  const int key = tile * TKEY + at / D, col = at % D;
  if (key >= sq.kv_len) return;
  const int64_t p0 = sink ? (int64_t)cut_plain * a.slices + (int64_t)(c - cut_plain) * a.sink_slices : (int64_t)c * a.slices;
  const float* part = a.part + ((int64_t)bh * dkv_parts(a) + p0) * (2 * TKEY * D) + blockIdx.z * (TKEY * D) + at;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  constexpr int kBatch = 8;  // loads in flight
  for (int s0 = 0; s0 < nslice; s0 += kBatch) {
    f32x4 v[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      v[i] = s0 + i < nslice ? *reinterpret_cast<const f32x4*>(part + (int64_t)(s0 + i) * (2 * TKEY * D)) : f32x4{};
#pragma unroll
    for (int i = 0; i < kBatch; ++i) sum += v[i];
  }
  const float f = blockIdx.z == 0 ? a.scale : 1.f;
  const Strides& st = blockIdx.z == 0 ? a.dks : a.dvs;
  T* out = static_cast<T*>(blockIdx.z == 0 ? a.dk : a.dv) + b * st.b + kvh * st.h + key * st.n + col;
  *reinterpret_cast<u32x2*>(out) = u32x2{pack2<T>(sum[0] * f, sum[1] * f), pack2<T>(sum[2] * f, sum[3] * f)};
}

template <typename T, int D>
hipError_t launch(const WindowArgs& a, hipStream_t s) {
  const int64_t bh = (int64_t)a.B * a.Hkv, nq = a.ntiles * bh, nk = dkv_items(a) * bh;
  if (!fits_launch(nq, 64 * kWaves) || !fits_launch(nk, 64 * kWaves)) return hipErrorInvalidConfiguration;
  if (nq > 0) {
    hipLaunchKernelGGL((window_dq_kernel<T, D>), dim3((unsigned)nq), dim3(64 * kWaves), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (nk == 0) return hipSuccess;
  if (D == 128 && a.deep) hipLaunchKernelGGL((window_dkv_kernel<T, 128, true>), dim3((unsigned)nk), dim3(64 * kWaves), 0, s, a);
  else hipLaunchKernelGGL((window_dkv_kernel<T, D, false>), dim3((unsigned)nk), dim3(64 * kWaves), 0, s, a);
  hipError_t e = hipGetLastError();
  const int64_t cut = (a.sink_slices > 1 ? a.nsink : 0) + (a.slices > 1 ? a.nktiles - a.nsink : 0);
  if (e != hipSuccess || cut == 0) return e;
  hipLaunchKernelGGL((window_dkv_sum_kernel<T, D>), dim3((unsigned)(cut * bh), 32 * kWaves * D / 1024, 2), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

int64_t plan_backward(WindowArgs* a, int d) {
  constexpr int kKeys = 32 * kWaves;
  const int64_t rows = (int64_t)a->Nq * a->group;
  a->ntiles = (int32_t)((rows + 32 * kWaves - 1) / (32 * kWaves));
  a->nktiles = (a->Nkv + kKeys - 1) / kKeys;
  a->stat_rows = ((int64_t)a->Nq + 127) / 64 * 64;  // whole tiles of 64 rows may be read
  // Row tiles (of 64) that a key tile walks.  Every query that lies behind a tile may
  // see its sinks; others are seen from `right` before to `left` behind.
  auto min64 = [](int64_t x, int64_t y) { return x < y ? x : y; };
  auto max64 = [](int64_t x, int64_t y) { return x > y ? x : y; };
  const int64_t walk_sink = ((int64_t)a->Nq + 63) / 64 * a->group;
  const int64_t walk = min64(walk_sink, ((int64_t)a->left + a->right + kKeys + 63) / 64 * a->group);
  a->nsink = (int32_t)((a->sinks + kKeys - 1) / kKeys);
  // Which dK/dV kernel.  Two workgroups of the plain one share a CU, one of the deep one
  // has a CU to itself: deep where no CU would get two (8192 queries, window 1024, 3
  // heads: 91 us for dQ, dK and dV with the plain kernel, 77 with the deep one; 6 heads:
  // 128 and 139), and up to twice that where walks span much of the sequence and so are
  // of very different lengths (all keys before, 8 heads: 566 and 479; 12: 700 and 714).
  //
  // Slices.  A slice costs 128 KB (head dim 128) written and read again.  Tiles without
  // sinks are cut only where they are few: less than three quarters of the CUs, or half
  // for the deep kernel (twice that where walks are uneven; one key head, 4096 tokens, all
  // keys before, in shares: 300 us with 256 workgroups, 238 with 512).  Tiles with sinks
  // come last, to fill the gaps behind the longer ones: they are cut to the others' walk,
  // to a quarter of it where there are few workgroups, and for the deep kernel to one more
  // workgroup for every CU.  No slice is shorter than four row tiles, and the slices of
  // sinks take half a gigabyte at most.
  const int64_t bh = max64((int64_t)a->B * a->Hkv, 1), plain = bh * (a->nktiles - a->nsink);
  const int64_t want = 2 * walk > walk_sink ? 512 : 256;
  a->deep = d == 128 && bh * a->nktiles <= want;
  const int64_t cut = plain <= 0             ? 1
                      : a->deep              ? want / plain
                      : 4 * plain < 3 * want ? (want + plain - 1) / plain
                                             : 1;
  const int64_t goal = max64((walk + cut - 1) / cut, 4);
  const int64_t goal_sink = a->deep                  ? max64((walk_sink * a->nsink * bh + 255) / 256, 4)
                            : bh * a->nktiles < 1024 ? max64((goal + 3) / 4, 4)
                                                     : goal;
  const int64_t most_sink = max64(4096 / (bh * max64(a->nsink, 1)), 1);
  a->slices = (int32_t)max64(1, min64((walk + goal - 1) / goal, 256));
  a->sink_slices = (int32_t)max64(1, min64((walk_sink + goal_sink - 1) / goal_sink, min64(most_sink, 256)));
  return 2 * (int64_t)a->B * a->H * a->stat_rows + dkv_parts(*a) * a->B * a->Hkv * (2 * kKeys * d);
}

hipError_t launch_window_backward(int dtype, int d, const WindowArgs& args, hipStream_t s) {
  WindowArgs a = args;
  plan_backward(&a, d);
  a.part = a.stats + 2 * (int64_t)a.B * a.H * a.stat_rows;
  if (dtype == kBf16) return d == 128 ? launch<__bf16, 128>(a, s) : launch<__bf16, 64>(a, s);
  return d == 128 ? launch<_Float16, 128>(a, s) : launch<_Float16, 64>(a, s);
}

}  // namespace bsa_ops
