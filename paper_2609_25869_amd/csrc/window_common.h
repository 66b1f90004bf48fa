// Device helpers of the window attention kernels: element types, matrix
// instructions, tiles in LDS and the visibility of keys.
//
// A tile is 8 or 16 KB of token rows (32 or 64 of them), row-major, 2 * D bytes a row,
// filled by loads that go straight from memory to LDS.  The 16-byte chunks of row r are
// stored at chunk ^ swizzle(r), so that both ways of reading it - 32 rows at one
// chunk for the operands that contract over the head dim, and four rows of
// four chunks through the transposing read for those that contract over the
// rows - touch every bank.
#pragma once

#include <type_traits>
#include <utility>

#include "ops_internal.h"

#define BSA_INLINE __attribute__((always_inline))

namespace bsa_ops {
namespace {

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

template <typename T>
struct Elem;

template <>
struct Elem<__bf16> {
  typedef __bf16 x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 x4 __attribute__((ext_vector_type(4)));
  typedef __bf16 x8 __attribute__((ext_vector_type(8)));
  __device__ static f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};

template <>
struct Elem<_Float16> {
  typedef _Float16 x2 __attribute__((ext_vector_type(2)));
  typedef _Float16 x4 __attribute__((ext_vector_type(4)));
  typedef _Float16 x8 __attribute__((ext_vector_type(8)));
  __device__ static f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

template <typename T>
__device__ inline uint32_t pack2(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, typename Elem<T>::x2));
}

__device__ inline float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Value of the same register in the other half of the wave.
__device__ inline float other_half(float x, int lane) {
  const uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float((lane & 32) ? r[0] : r[1]);
}

// At most N of this wave's vector-memory operations are outstanding, and none of
// its LDS reads (gfx9 s_waitcnt encoding: vmcnt in bits 3:0 and 15:14, expcnt 6:4
// at its maximum, lgkmcnt 11:8 = 0).
template <int N>
__device__ inline void wait_vm_lgkm() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | ((N >> 4) << 14));
}

// Workgroup barrier without a memory fence: what the LDS loads wrote is complete
// once vmcnt says so, and a fence would also wait for the loads that are meant
// to stay in flight.
__device__ inline void block_sync() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Rows of D elements in LDS.
template <int D>
struct Rows {
  static constexpr int kBytes = 2 * D;           // of a row
  static constexpr int kChunks = D / 8;          // of 16 bytes in a row
  static constexpr int kPerLoad = 64 / kChunks;  // rows that one load instruction of a wave brings (1 KB)
  static constexpr int kSteps = D / 16;          // MFMAs that contract the head dim
  static constexpr int kBlocks = D / 32;         // 32-column blocks of the head dim

  __device__ static int swizzle(int r) {
    return D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : ((r & 2) << 1) | ((r >> 1) & 2) | ((r >> 3) & 1);
  }
  // Operand that contracts over the head dim: row `lane % 32` of a 32-row block,
  // elements 16 c + 8 (lane / 32) on.
  __device__ static int row_read(int lane, int c) {
    const int r = lane & 31;
    return r * kBytes + (((2 * c + (lane >> 5)) ^ swizzle(r & 15)) << 4);
  }
  // Operand that contracts over 16 rows: column 32 * blk + lane % 32 of the
  // transposed tile; part r (0, 1) holds rows 8 r + 4 (lane / 32) .. + 3, the order
  // in which a result of the other product holds them.
  __device__ static int tr_read(int lane, int r, int blk) {
    const int s16 = lane & 15, g = lane >> 4, mh = g & 1, gh = g >> 1;
    const int row = 8 * r + 4 * gh + (s16 >> 2);
    const int col = blk * 32 + 16 * mh + 4 * (s16 & 3);
    return row * kBytes + (((col >> 3) ^ swizzle(row & 15)) << 4) + (col & 7) * 2;
  }
};

__device__ inline i16x4 lds_read_tr(const uint8_t* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(p));
}

template <typename T>
__device__ inline typename Elem<T>::x8 read_tr_pair(const uint8_t* p0, const uint8_t* p1) {
  return __builtin_bit_cast(typename Elem<T>::x8,
                            __builtin_shufflevector(lds_read_tr(p0), lds_read_tr(p1), 0, 1, 2, 3, 4, 5, 6, 7));
}

// Loads of TR token rows into LDS by NW waves.  The buffer descriptor starts at
// the tile's first row and ends with its last valid one, so rows behind it read
// as zeros, and no offset passes 32 bits however long the sequence is.
template <int D, int TR, int NW>
struct TileLoad {
  using R = Rows<D>;
  static constexpr int kLoads = TR / (R::kPerLoad * NW);  // per wave
  static_assert(kLoads >= 1 && TR % (R::kPerLoad * NW) == 0, "rows split over the waves");
  static constexpr int kRep = 16 / (R::kPerLoad * NW) < 1 ? 1 : 16 / (R::kPerLoad * NW);  // loads until the swizzle repeats
  static constexpr int kOffs = kRep < kLoads ? kRep : kLoads;

  uint32_t offs[kOffs];
  uint32_t stride;  // bytes from a row to the next
  __device__ void init(int64_t row_stride, int w, int lane) {
    stride = (uint32_t)(row_stride * 2);
#pragma unroll
    for (int j = 0; j < kOffs; ++j) {
      const int r = R::kPerLoad * (w + j * NW) + lane / R::kChunks;
      offs[j] = (uint32_t)r * stride + (((lane % R::kChunks) ^ R::swizzle(r & 15)) << 4);
    }
  }
  // descriptor of `rows` valid rows (may be 0 or less, or more than TR) from `base` on
  __device__ __amdgpu_buffer_rsrc_t rsrc(const char* base, int rows) const {
    const int n = rows < TR ? rows : TR;
    const uint32_t bytes = n > 0 ? (uint32_t)(n - 1) * stride + R::kBytes : 0;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, (int)bytes, 0x00020000);
  }
  __device__ void one(__amdgpu_buffer_rsrc_t r, int j, uint8_t* lds, int w) const {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        r, (__attribute__((address_space(3))) void*)(lds + 1024 * (w + j * NW)), 16,
        offs[j % kOffs] + (uint32_t)((j / kOffs) * kOffs * NW * R::kPerLoad) * stride, 0, 0, 0);
  }
  __device__ void issue(const char* base, int rows, uint8_t* lds, int w) const {
    const __amdgpu_buffer_rsrc_t r = rsrc(base, rows);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) one(r, j, lds, w);
  }
};

// Lengths of one sequence, and the keys a query of it sees: [lo, hi] and the
// first `sinks` up to hi.
struct Seq {
  int q_len, kv_len, off;  // off: position of query 0
  __device__ Seq(const WindowArgs& a, int b) {
    q_len = a.q_len ? min(max(a.q_len[b], 0), a.Nq) : a.Nq;
    kv_len = a.kv_len ? min(max(a.kv_len[b], 0), a.Nkv) : a.Nkv;
    off = kv_len - q_len;
  }
  __device__ int lo(const WindowArgs& a, int i) const { return max(i + off - a.left, 0); }
  __device__ int hi(const WindowArgs& a, int i) const { return min(i + off + a.right, kv_len - 1); }
};

// f(0), f(1), ... f(N - 1) with constant arguments, as long as f returns true.  A
// large loop body under #pragma unroll may be unrolled in part only, and ring
// slots that are not constants make the compiler wait for every load in flight.
template <class F, int... I>
__device__ BSA_INLINE inline bool each_slot(F&& f, std::integer_sequence<int, I...>) {
  return (f(std::integral_constant<int, I>{}) && ...);
}
template <int N, class F>
__device__ BSA_INLINE inline bool each_slot(F&& f) {
  return each_slot(f, std::make_integer_sequence<int, N>{});
}

// Bits below x of a 32-bit word.
__device__ inline uint32_t bits_below(int x) { return x <= 0 ? 0u : x >= 32 ? ~0u : (1u << x) - 1u; }

// Which of the 32 keys from j on lie in [lo, hi], or below `sinks` and not above
// hi.
__device__ inline uint32_t visible_bits(int j, int lo, int hi, int sinks) {
  return bits_below(hi - j + 1) & (~bits_below(lo - j) | bits_below(sinks - j));
}

template <int D>
constexpr int kTileKeys = 4096 / D;  // window_fwd_kernel's, 8 KB of K: 32 keys of 128 elements, 64 of 64

// The keys of one row tile as a list of tiles: `ns` tiles of sinks from key 0, then
// tiles from key w0 on.  Keys that no row of the tile sees are in none: rows from
// limit() on are not loaded, and a tile of sinks masks from there, since the window may
// begin in it.
struct KeyTiles {
  int ns, nt, w0, sink_end, end;
  template <int TK>
  __device__ void init(const WindowArgs& a, const Seq& sq, int ia, int ib) {
    const int lo = sq.lo(a, ia);
    end = max(sq.hi(a, ib) + 1, 0);
    sink_end = min(a.sinks, min(lo, end));
    ns = (sink_end + TK - 1) / TK;
    w0 = lo;
    if (sink_end >= lo) {  // the sinks reach the window: one range
      ns = 0;
      w0 = 0;
    }
    nt = ns + max(end - w0 + TK - 1, 0) / TK;
  }
  template <int TK>
  __device__ int key(int t) const { return t < ns ? t * TK : w0 + (t - ns) * TK; }
  __device__ int limit(int t) const { return t < ns ? sink_end : end; }
};

// The lane index, formed again where it is used: rare paths and the ends of kernels
// then keep no register for it through the loop.
__device__ inline int lane_now() {
  int l = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
  asm volatile("" : "+v"(l));
  return l;
}

// x = keep ? x : 0 in place (keep is per lane), in a branch that is rarely taken: the
// tied operand pins the result to its register, and the compiler cannot turn the
// branch into selections that run every time.  (The condition may have been written by
// the instruction before: the compiler adds no wait states for inline asm.)
__device__ inline void zero_unless(float& x, bool keep) {
  asm volatile("s_nop 1\n\tv_cndmask_b32_e64 %0, 0, %0, %1" : "+v"(x) : "s"(__ballot(keep)));
}

// Dispatch order: the work item (of per_head in every key head, the heads of a sequence
// one after the other) and the sequence that a slot runs.  The eight XCDs take consecutive
// workgroups in turn.
//
// Every XCD gets a contiguous share of a sequence's items, in order: neighbouring row
// tiles of a head read nearly the same keys through one L2.  Every sequence is shared out
// by itself (with one list for the batch, XCDs that get the short ones run dry: three
// sequences of up to 5001 tokens, 16 heads of 64, window 701: 73 us with one list, 63 so),
// and the shares move on by one XCD from sequence to sequence.
//
// `deal`: the tiles are dealt out one by one instead, the first tile of every head and
// sequence before the second, and the row of eight turned by one each time.
__device__ inline uint32_t item_of_slot(const WindowArgs& a, uint32_t slot, uint32_t per_head, int* b) {
  const uint32_t n = per_head * a.Hkv;
  if (a.deal) {
    const uint32_t k = slot / 8, i = 8 * k + 8 <= n * a.B ? 8 * k + (slot + k) % 8 : slot;
    *b = (int)(i % a.B);
    return i / a.B % a.Hkv * per_head + i / a.B / a.Hkv;
  }
  *b = (int)(slot / n);
  const uint32_t s = slot % n, share = n / 8, more = n % 8, x = more ? s % 8 : (s + *b) % 8;
  return x * share + (x < more ? x : more) + s / 8;
}

// The i-th row tile of a head: where later rows see more keys, the last one first.
__device__ inline int tile_of(const WindowArgs& a, int i) { return a.later_longer ? a.ntiles - 1 - i : i; }

}  // namespace
}  // namespace bsa_ops
