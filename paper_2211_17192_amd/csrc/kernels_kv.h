// The paged key-value cache apart from a model: rows written into it (in 8 bits or bf16), rows read back, and the attention
// of a few query rows per sequence over it.
//
// Layout, as the models' caches: [page][K|V][kv head][slot][d_head]; a sequence's keys at positions 16 i .. 16 i + 15 are
// consecutive slots of one page (pages hold a power of two of at least 16 positions).  In 8 bits a row x of d_head values is
// kept as e4m3 codes c and one exponent, exps[page][K|V][kv head][slot] = E + 127, x = c 2^E, with E the smallest for which
// max |x| <= 448 2^E.  A power of two costs a floating-point format nothing but range, of which e4m3 has 17 binades: codes and exponents
// follow from x exactly (no quotient is rounded), and c 2^E is exact in bf16, whose matrix instructions the attention uses.
#pragma once
#include <type_traits>
#include "common.h"
#include "kernels_attn.h"

namespace sd {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr int KV_EXP_MIN = -111, KV_EXP_MAX = 120;   // E of a row: c 2^E stays a normal bf16 / fp32 number (the least code is 2^-9)

struct KvCacheArgs {
  void* pool;
  unsigned char* exps;      // e4m3 only
  const int* table;         // [n_seq][table_stride] pages
  int n_pages, n_seq, table_stride, page_shift, Hkv;
};

// ---------------------------------------------------------------------------
// Rows in and out
// ---------------------------------------------------------------------------
// Row i is position pos[i] (pos == nullptr: i % per_seq) of sequence seq[i] (seq == nullptr: i / per_seq).  What lies outside the
// table, or on a page outside the pool, is not written, and read as zeros.
struct KvRowsArgs {
  KvCacheArgs c;
  const int *seq, *pos;
  int rows, per_seq;
  void *k, *v;              // rows [i][head][d_head] at these distances, in elements; or (paged) a pool of the cache's geometry
  long long k_row, k_head, v_row, v_head;
  int paged;
};

// The row of the pool (of d_head elements) where K of head 0 of row i lies; -1: nowhere.
__device__ __forceinline__ long long kv_place(const KvRowsArgs& a, int i) {
  const int s = a.seq ? a.seq[i] : i / a.per_seq, p = a.pos ? a.pos[i] : i % a.per_seq;
  const int entry = p >> a.c.page_shift;
  const bool in = p >= 0 && (unsigned)s < (unsigned)a.c.n_seq && entry < a.c.table_stride;
  const int page = a.c.table[in ? (size_t)s * a.c.table_stride + entry : 0];
  if (!in || (unsigned)page >= (unsigned)a.c.n_pages) return -1;
  return ((long long)page * 2 * a.c.Hkv << a.c.page_shift) + (p & ((1 << a.c.page_shift) - 1));
}

struct OpMaxU { __device__ unsigned operator()(unsigned a, unsigned b) const { return max(a, b); } };
// The maximum over groups of 4, 8, 16 or 32 consecutive lanes, in each of them: quads by quad permutes, then the mirror images inside
// 8 and 16 lanes (the quads hold one value each by then).
template <int LANES> __device__ __forceinline__ unsigned group_max(unsigned v) {
  v = max(v, dpp_partner<1>(v));
  v = max(v, dpp_partner<2>(v));
  if (LANES >= 8) v = max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xf, 0xf, true));
  if (LANES >= 16) v = max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xf, 0xf, true));
  if (LANES == 32) v = lane_combine<16>(v, OpMaxU());
  return v;
}

__device__ __forceinline__ float two_to(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }

// 16 bytes of a row as they were loaded (rows come past the L2s: nobody reads them again, and what they would push out is
// wanted: 134 MB into an e4m3 cache 41.4 us, 44.1 with plain loads).
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
// Two floats rounded to bf16, the first in the low half.
__device__ __forceinline__ unsigned bf16_pair(float x, float y) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2{x, y}), bf16x2));
}
template <typename T> struct KvRaw;
template <> struct KvRaw<float> {
  typedef unsigned Codes;                            // their codes
  typedef u32x2 Bf16;                                // they in bf16
  f32x4 a;
  __device__ __forceinline__ void load(const float* p) { a = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p)); }
  __device__ __forceinline__ Bf16 rounded() const { return Bf16{bf16_pair(a[0], a[1]), bf16_pair(a[2], a[3])}; }
  // the largest magnitude, as the bits of a float
  __device__ __forceinline__ unsigned top() const {
    unsigned m = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) m = max(m, __float_as_uint(a[e]) & 0x7fffffffu);
    return m;
  }
  // codes of x / s
  __device__ __forceinline__ Codes codes(float s) const {
    s16x2 v = {0, 0};
    v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, a[0], a[1], s, false);
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, a[2], a[3], s, true));
  }
  // what is not finite becomes NaN, the rest at most `most`
  __device__ __forceinline__ void limit(float most) {
#pragma unroll
    for (int e = 0; e < 4; ++e) a[e] = ((__float_as_uint(a[e]) & 0x7fffffffu) >= 0x7f800000u) ? __uint_as_float(0x7fc00000u) : __builtin_amdgcn_fmed3f(a[e], -most, most);
  }
  __device__ __forceinline__ unsigned finite_top() const {
    unsigned m = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const unsigned x = __float_as_uint(a[e]) & 0x7fffffffu;
      m = max(m, x < 0x7f800000u ? x : 0u);
    }
    return m;
  }
};
template <> struct KvRaw<bf16> {
  typedef u32x2 Codes;
  typedef u32x4 Bf16;
  u32x4 a;
  __device__ __forceinline__ void load(const bf16* p) { a = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)); }
  __device__ __forceinline__ Bf16 rounded() const { return a; }
  __device__ __forceinline__ unsigned top() const {  // (two at a time in 16-bit integers)
    u16x2 m = {0, 0};
#pragma unroll
    for (int w = 0; w < 4; ++w) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, a[w] & 0x7fff7fffu));
    return (unsigned)max(m[0], m[1]) << 16;
  }
  __device__ __forceinline__ Codes codes(float s) const {
    unsigned c[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const unsigned lo = a[2 * h], hi = a[2 * h + 1];        // (a bit_cast of a vector's element takes its first)
      s16x2 v = {0, 0};
      v = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(v, __builtin_bit_cast(bf16x2, lo), s, false);
      c[h] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(v, __builtin_bit_cast(bf16x2, hi), s, true));
    }
    return Codes{c[0], c[1]};
  }
  __device__ __forceinline__ void limit(float most) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      unsigned r = 0;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const unsigned bits = h ? a[w] & 0xffff0000u : a[w] << 16;
        const float x = ((bits & 0x7fffffffu) >= 0x7f800000u) ? __uint_as_float(0x7fc00000u) : __builtin_amdgcn_fmed3f(__uint_as_float(bits), -most, most);
        r |= h ? __float_as_uint(x) & 0xffff0000u : __float_as_uint(x) >> 16;
      }
      a[w] = r;
    }
  }
  __device__ __forceinline__ unsigned finite_top() const {
    unsigned m = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const unsigned x = (h ? a[w] & 0xffff0000u : a[w] << 16) & 0x7fffffffu;
        m = max(m, x < 0x7f800000u ? x : 0u);
      }
    return m;
  }
};

// Calls that write 8 MB or more (PAST; in a model's prompt, whose attention reads it next, what the L2s cannot hold): their stores go past the L2s too, and an append waits for a row's place before it asks for the row, so that rows which are absent
// cost nothing; in smaller calls that wait would be seen.  (us, not / PAST: 134 MB read from an e4m3 cache into bf16 rows 41.3 / 25.4; 16 x 2047 rows of 8 heads of 128 into one 40.4 / 39.2,
// with 3 of 8 absent 36.6 / 27.3; 8 x 700 9.7 / 8.9, 8.4 / 6.8; 2 x 1200, 5 MB, 5.0 / 5.3; into a bf16 cache 16 x 2047 51.0 / 48.8.)
template <bool PAST, typename V> __device__ __forceinline__ void kv_store(V* p, const V& v) {
  if (PAST) __builtin_nontemporal_store(v, p);
  else *p = v;
}

// Rows in and out: 16 bytes of the rows' side of K and of V per thread, so that a wavefront's accesses are whole lines (fp32 rows by 32 bytes a thread: 131 us for
// 268 MB read into them past the L2s, 85 through them), a workgroup per KV_ROW_BYTES / row rows of one head.  A workgroup's neighbours take the other heads of its rows.
// Many rows are bound by memory (16 x 2047 rows of 8 heads of 128 in bf16: in 39.2 us, 5.1 TB/s as a copy; out 24.9), few by the chain position - page - row (80 rows 3.2 us).
constexpr int KV_ROW_BYTES = 256 * 16;
__device__ __forceinline__ void kv_rows_block(const KvRowsArgs& a, int& block, int& head) {
  block = (int)(blockIdx.x / (unsigned)a.c.Hkv);
  head = (int)(blockIdx.x - (unsigned)block * (unsigned)a.c.Hkv);
}

template <typename T, int DH, bool E4M3, bool PAST>
static __global__ __launch_bounds__(256) void kv_append_kernel(const KvRowsArgs a) {
  constexpr int EPT = 16 / sizeof(T), LPR = DH / EPT;
  int block, head;
  kv_rows_block(a, block, head);
  const int piece = threadIdx.x % LPR, i = block * (256 / LPR) + (int)threadIdx.x / LPR, ic = min(i, a.rows - 1);
  const long long apart = (long long)a.c.Hkv << a.c.page_shift;                // rows of the pool from K to V
  const long long head_row = (long long)head << a.c.page_shift;
  long long place = 0;
  if (a.paged || PAST) place = kv_place(a, ic);      // (paged: the rows come from such places themselves)
  if (PAST && place < 0) return;                     // (all lanes of the row)
  const long long from = (max(place, 0ll) + head_row) * DH;
  KvRaw<T> x[2];
  x[0].load(static_cast<const T*>(a.k) + (a.paged ? from : ic * a.k_row + head * a.k_head) + piece * EPT);
  x[1].load(static_cast<const T*>(a.v) + (a.paged ? from + apart * DH : ic * a.v_row + head * a.v_head) + piece * EPT);
  if (!a.paged && !PAST) place = kv_place(a, ic);
  const bool there = i < a.rows && place >= 0;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const long long to = place + head_row + w * apart;
    if constexpr (!E4M3) {
      if (!there) continue;
      kv_store<PAST>(reinterpret_cast<typename KvRaw<T>::Bf16*>(static_cast<bf16*>(a.c.pool) + to * DH + piece * EPT), x[w].rounded());
    } else {
      unsigned top = group_max<LPR>(x[w].top());
      if (__builtin_amdgcn_ballot_w64(top >= 0x7f000000u) != 0ull) {           // rare: NaN, infinities, and what would be read as infinity (256 * 2^120)
        top = group_max<LPR>(x[w].finite_top());
        x[w].limit(240.0f * 0x1p120f);
      }
      // 448 = 1.75 * 2^8
      const int E = min(max((int)(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0), KV_EXP_MIN), KV_EXP_MAX);
      typedef typename KvRaw<T>::Codes Codes;
      if (there) {
        kv_store<PAST>(reinterpret_cast<Codes*>(static_cast<unsigned char*>(a.c.pool) + to * DH + piece * EPT), x[w].codes(two_to(E)));
        if (piece == 0) a.c.exps[to] = (unsigned char)(E + 127);
      }
    }
  }
}

// Four codes times a power of two, in bf16 (exact).
__device__ __forceinline__ u32x2 e4m3_values(unsigned c, float s) {
  return u32x2{__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, s, false)), __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, s, true))};
}
__device__ __forceinline__ u32x4 e4m3_values(u32x2 c, float s) {
  const u32x2 lo = e4m3_values(c[0], s), hi = e4m3_values(c[1], s);
  return u32x4{lo[0], lo[1], hi[0], hi[1]};
}

template <typename T, int DH, bool E4M3, bool PAST>
static __global__ __launch_bounds__(256) void kv_read_kernel(const KvRowsArgs a) {
  constexpr int EPT = 16 / sizeof(T), LPR = DH / EPT;
  typedef typename KvRaw<T>::Codes Codes;
  typedef typename KvRaw<T>::Bf16 Bf16;
  int block, head;
  kv_rows_block(a, block, head);
  const int piece = threadIdx.x % LPR, i = block * (256 / LPR) + (int)threadIdx.x / LPR, ic = min(i, a.rows - 1);
  const long long apart = (long long)a.c.Hkv << a.c.page_shift, place = kv_place(a, ic);
  const long long row = max(place, 0ll) + ((long long)head << a.c.page_shift);
  Bf16 x[2];
  if constexpr (E4M3) {
    Codes c[2];
    unsigned e[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      c[w] = *reinterpret_cast<const Codes*>(static_cast<const unsigned char*>(a.c.pool) + (row + w * apart) * DH + piece * EPT);
      e[w] = a.c.exps[row + w * apart];
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) x[w] = e4m3_values(c[w], __uint_as_float(e[w] << 23));
  } else {
#pragma unroll
    for (int w = 0; w < 2; ++w) x[w] = *reinterpret_cast<const Bf16*>(static_cast<const bf16*>(a.c.pool) + (row + w * apart) * DH + piece * EPT);
  }
  if (i >= a.rows || (a.paged && place < 0)) return;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    if (place < 0) x[w] = x[w] ^ x[w];
    T* to = static_cast<T*>(w ? a.v : a.k) + (a.paged ? (row + w * apart) * DH : i * (w ? a.v_row : a.k_row) + head * (w ? a.v_head : a.k_head)) + piece * EPT;
    if constexpr (sizeof(T) == 2) kv_store<PAST>(reinterpret_cast<u32x4*>(to), x[w]);
    else kv_store<PAST>(reinterpret_cast<f32x4*>(to), f32x4{__uint_as_float(x[w][0] << 16), __uint_as_float(x[w][0] & 0xffff0000u),
                                                           __uint_as_float(x[w][1] << 16), __uint_as_float(x[w][1] & 0xffff0000u)});
  }
}

// ---------------------------------------------------------------------------
// Attention
// ---------------------------------------------------------------------------
constexpr int KV_MAX_RANGES = 128;                   // key ranges of a context at most
constexpr int KV_MAX_RANGE_KEYS = 4096;              // a wavefront holds the page entries of its keys in one register: 64 lanes x 16 keys x 4 wavefronts (or more)
constexpr int KV_ROWS = 16;                          // (row, head) pairs of a tile: one side of a matrix instruction; a workgroup takes one or two

// x / d for x, d < 2^16: with m = ceil(2^32 / d), x m is at most x d / 2^32 < 1 / d above x 2^32 / d.
struct KvDivisor {
  unsigned long long m;
  __host__ __device__ void set(int d) { m = ((1ull << 32) + (unsigned)d - 1) / (unsigned)d; }
  __device__ __forceinline__ int quotient(int x) const { return (int)((unsigned)x * m >> 32); }
};
struct KvAttnArgs {
  KvCacheArgs c;
  const void* q;            // T: row i, query head h at i * q_row + h * q_head
  long long q_row, q_head;
  void* out;                // T [rows][H][dh]
  float* lse;               // [rows][H], optional
  const int* pos;           // [n_seq * R]: the last key that a row sees, < 0: none
  int R, H, G, seq0;        // rows per sequence, query heads, query heads per kv head; the first sequence's row of the table
  int groups, rows_wg;      // a workgroup takes rows_wg of the R * G (row, head) pairs of a kv head
  int n_seq;
  KvDivisor by_g, by_groups, by_hkv;
  int max_len;              // positions count as max_len - 1 at most
  int range_keys, n_ranges;
  float c_log2;             // scale * log2(e)
  float* partial;           // [sequence][group][kv head][range][rows_wg][dh + 2]
  unsigned* tickets;        // [sequence][group][kv head], zero between launches
  bf16* out_frag;           // the output in the fragment order of a product over many rows instead
  int frag_ks, frag_slab;
};

// One pass over the keys with the running maximum and sum of the softmax; both products on the matrix cores in bf16, with exact
// operands: codes times their power of two, bf16 queries, fp32 queries and the probabilities as sums of bf16 numbers (NQ, NP of them).
//   S^T = K Q^T   16x16x32, A = 16 keys, B = 16 (row, head) pairs.  A lane takes 16 bytes of its key's row; which features of the row a lane
//                 of the fragment holds is free as long as K and Q agree.  The conversion from e4m3 multiplies by the key's power of two.  Loaded like
//                 this, 16 lanes touch 16 lines, so a CU gets through fewer bytes; calls that memory bounds load whole rows and turn them in LDS, which
//                 costs the others more than they wait (64 sequences of up to 8192, 1 row, 8 kv heads of 128: 137 us directly, 125 through LDS, in bf16 half as
//                 many 148 and 122; 16 of 2048 15.6 and 16.1).  Rows under 128 bytes are taken directly (heads of 32 47 us, 50 through LDS).
//   O^T = V^T P   A = 16 features x 32 keys: V's rows go through the wavefront's own part of LDS and come back transposed
//                 (ds_read_b64_tr_b8 / _b16), B = the probabilities as the lane has them, times V's powers of two.
// The wavefronts take turns of 32 keys, each with its own maximum, sum and output; they are joined
// through LDS.  The keys of a context are cut into ranges, a workgroup each; the last of a (sequence, group, kv head) to arrive
// joins them in range order (posts past the L2s, a relaxed ticket), so a result does not depend on which one that is.
// What a step's loads need is known before the loop: the page entries of all a wavefront's keys lie in one register, a lane each, and a
// tile of 16 keys has one uniform base address.  Loads run one step ahead and are never behind a branch; whole pages are in the pool, so
// slots behind the last key may be read, and whatever lies there (NaN too) is replaced by zeros before the product.
// Rows that see fewer keys than others of the same workgroup: where V of a key that some row does not see is not finite, zeros enter the product
// and a product of ones marks the rows that see it (0 * NaN would reach the others).
// Every sum is spelled out (fmaf), so that all builds of this kernel give a row the same bits.
// What bounds it: memory for large calls (64 sequences of 8192, 1.08 GB: 176 us, 6.1 TB/s; 5 rows 200).  A small call is a chain: launch, positions (1.2 us), first rows (0.6), the
// steps (0.9 each where a SIMD has one wavefront), the join (0.9): one sequence of 500 with 4 wavefronts 7.1 us.  Between: 16 of 2048 take 15.5, of which 10 are steps in
// which 128 CUs read 6.7 TB/s.  (Loads two steps ahead: 17.0; 64 keys a step: 17.8.)
// grid = (pairs of sequence and kv head x groups, ranges).  Workgroups take turns on the XCDs, so the groups of a pair, which read the same keys and
// values at about the same time, lie eight apart: one of them comes from memory, the others find the lines in their L2.
template <typename T, int DH, int NW, int NRT, bool E4M3, bool ONCE> struct KvShape {
  static constexpr int ES = E4M3 ? 1 : 2;            // bytes of an element of the cache
  static constexpr int KT = 2;                       // key tiles of a step
  static constexpr int STEP = 16 * KT;
  static constexpr int RB = DH * ES;                 // bytes of a row
  static constexpr int FPL = (E4M3 && DH >= 64) ? 16 : 8;                    // features a lane loads of a key at once
  static constexpr int KL = DH / (4 * FPL);          // ... and how often
  static constexpr int PPR = RB / 16;                // 16-byte pieces of a row of V
  static constexpr int RPL = 64 / PPR;               // rows of V per load of the wavefront
  static constexpr int NV = STEP / RPL;
  static constexpr int NQ = sizeof(T) == 4 ? 3 : 1, NP = sizeof(T) == 4 ? 3 : 2;
  static constexpr bool LDS_K = (ONCE || NRT == 2) && RB >= 128;            // K goes through LDS too
  static constexpr int STAGE = (LDS_K ? 2 : 1) * STEP * RB;                  // LDS of a wavefront: V, then K
  static constexpr int most(int a, int b) { return a > b ? a : b; }
  static constexpr int ML = KV_MAX_RANGES * KV_ROWS * NRT * 8;               // the ranges' (m, l)
  static constexpr int LDS = most(most(NW * STAGE, NW * KV_ROWS * (DH + 4) * 4), ML + 64 * NW * 16);
};

// Where 16-byte piece `p` of row `row` lies in a wavefront's part of LDS: rows without padding, the 16-feature chunks of a row exchanged so
// that the rows one transposing read takes at a time (e4m3: 8 of each 16-key half; bf16: 8) lie in different banks.
template <int DH, bool E4M3> __device__ __forceinline__ int kv_swizzle(int row) {
  constexpr int RP = 256 / (DH * (E4M3 ? 1 : 2));    // rows a pass over the banks holds
  const int id = E4M3 ? ((row & 7) | ((row >> 4 & 1) << 3)) : (row & 7);
  return id / RP;                                    // (below DH / 16)
}

// ... and for K, of which lanes read the same piece of 16 rows: the pieces of a row exchanged so that those of rows next to each other differ in their banks.
template <int DH, bool E4M3> __device__ __forceinline__ int kv_swizzle_k(int row) {
  constexpr int PPR = DH * (E4M3 ? 1 : 2) / 16;
  return PPR >= 8 ? row & 7 : row / (8 / PPR) & (PPR - 1);
}

template <bool ONCE, typename V> __device__ __forceinline__ V kv_load(const V* p) { return ONCE ? __builtin_nontemporal_load(p) : *p; }

template <typename T, int DH, int NW, int NRT, bool E4M3, bool ONCE>
static __global__ __launch_bounds__(64 * NW, 2) void kv_attention_kernel(const KvAttnArgs a) {
  using S = KvShape<T, DH, NW, NRT, E4M3, ONCE>;
  constexpr int KT = S::KT, KL = S::KL, NV = S::NV, NQ = S::NQ, NP = S::NP, STEP = S::STEP, TURN = NW * STEP, RB = S::RB, DT = DH / 16, KSQ = DH / 32;
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  typedef int i32x2 __attribute__((ext_vector_type(2)));
  __shared__ __align__(256) unsigned char lds[S::LDS];
  __shared__ int last_wg;
  __shared__ float row_m[KV_ROWS * NRT], row_l[KV_ROWS * NRT];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j = lane & 15, kq = lane >> 4;
  // x: (sequence, kv head) pairs by eights, then the groups of each eight
  const int eight = a.by_groups.quotient(blockIdx.x >> 3), grp = (int)(blockIdx.x >> 3) - eight * a.groups, pair = eight * 8 + (int)(blockIdx.x & 7);
  const int seq = a.by_hkv.quotient(pair), hkv = pair - seq * a.c.Hkv, range = blockIdx.y;
  if (seq >= a.n_seq) return;
  const int G = a.G, rg0 = grp * a.rows_wg, RG = min(a.rows_wg, a.R * G - rg0);       // this workgroup's (row, head) pairs
  const int range0 = range * a.range_keys;
  const int kb0 = range0 + wave * STEP;

  // ---- positions, page entries, queries: one round of loads ----
  const int* table = a.c.table + (size_t)(a.seq0 + seq) * a.c.table_stride;
  int pos[NRT];
  constexpr int QL = sizeof(T) / 2;                   // loads of eight queries
  u32x4 q_raw[NRT][KSQ][QL];
  const T* qp[NRT];
#pragma unroll
  for (int rt = 0; rt < NRT; ++rt) {                 // (lanes past the last pair repeat it; nobody reads them)
    const int rg = rg0 + min(rt * 16 + j, RG - 1), r = a.by_g.quotient(rg), row = seq * a.R + r;
    pos[rt] = a.pos[row];
    qp[rt] = static_cast<const T*>(a.q) + (long long)row * a.q_row + (long long)(hkv * G + rg - r * G) * a.q_head + kq * S::FPL;
  }
  // lane i: the page of the keys of tile i % KT of step i / KT
  const int my_page = table[min((kb0 + (lane / KT) * TURN + (lane % KT) * 16) >> a.c.page_shift, a.c.table_stride - 1)];
#pragma unroll
  for (int rt = 0; rt < NRT; ++rt)
#pragma unroll
    for (int s = 0; s < KSQ; ++s)
#pragma unroll
      for (int l = 0; l < QL; ++l) {
        constexpr int U = S::FPL / 8;
        q_raw[rt][s][l] = reinterpret_cast<const u32x4*>(qp[rt] + (s / U) * 4 * S::FPL + (s % U) * 8)[l];
      }
  const int capacity = (int)min((long long)a.max_len, (long long)a.c.table_stride << a.c.page_shift);
  const bool page_ok = (unsigned)my_page < (unsigned)a.c.n_pages;
  const unsigned long long ok_tiles = __builtin_amdgcn_ballot_w64(page_ok);
  const int safe_page = page_ok ? my_page : 0;

  // ---- loads ----
  const unsigned page_rows = 2u * (unsigned)a.c.Hkv << a.c.page_shift, v_rows = (unsigned)a.c.Hkv << a.c.page_shift;
  const unsigned slot_mask = (1u << a.c.page_shift) - 1u;
  const int k_lane = j * RB + kq * S::FPL * S::ES;   // this lane's bytes of a key tile, as the product takes them
  const int vpiece = lane % S::PPR, vrow = lane / S::PPR;      // ... of rows loaded whole
  // first row of the pool of tile kt of step i (its K); what lies behind the end re-reads a tile that was just read (the step's first, or that of the
  // step before it), which costs no memory traffic
  auto tile_row = [&](int i, int kt, int end) -> unsigned long long {
    const int step = kb0 + i * TURN;
    const int ii = (step < end) ? i : max(i - 1, 0), t = (step + kt * 16 < end) ? kt : 0;
    const unsigned page = (unsigned)__builtin_amdgcn_readlane(safe_page, ii * KT + t);
    return (unsigned long long)page * page_rows + ((unsigned)hkv << a.c.page_shift) + ((unsigned)(kb0 + ii * TURN + t * 16) & slot_mask);
  };
  const unsigned char* pool = static_cast<const unsigned char*>(a.c.pool);
  u32x4 kr[S::most(KT * KL, NV)], vr[NV];
  unsigned ke[KT], ve[KT];
  auto load_rows = [&](u32x4* to, const unsigned long long (&row)[KT]) {           // RPL rows a load: within a tile of 16, or two of them
#pragma unroll
    for (int c = 0; c < NV; ++c) {
      constexpr int RPL = S::RPL;
      if constexpr (RPL <= 16) to[c] = kv_load<ONCE>(reinterpret_cast<const u32x4*>(pool + (row[c * RPL / 16] + (c * RPL) % 16) * RB + vrow * RB + vpiece * 16));
      else to[c] = kv_load<ONCE>(reinterpret_cast<const u32x4*>(pool + (vrow < 16 ? row[2 * c] : row[2 * c + 1]) * RB + (vrow & 15) * RB + vpiece * 16));
    }
  };
  auto load_k = [&](int i, int end) {
    unsigned long long row[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) row[kt] = tile_row(i, kt, end);
    if constexpr (S::LDS_K) load_rows(kr, row);
    else {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int l = 0; l < KL; ++l) {
          const unsigned char* p = pool + row[kt] * RB + k_lane + l * 4 * S::FPL * S::ES;
          if constexpr (S::FPL * S::ES == 16) kr[kt * KL + l] = kv_load<ONCE>(reinterpret_cast<const u32x4*>(p));
          else { const u32x2 x = kv_load<ONCE>(reinterpret_cast<const u32x2*>(p)); kr[kt * KL + l] = u32x4{x[0], x[1], 0u, 0u}; }
        }
    }
    if (E4M3) {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) ke[kt] = *(a.c.exps + row[kt] + j);
    }
  };
  auto load_v = [&](int i, int end) {
    unsigned long long row[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) row[kt] = tile_row(i, kt, end) + v_rows;
    load_rows(vr, row);
    if (E4M3) {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) ve[kt] = *reinterpret_cast<const unsigned*>(a.c.exps + row[kt] + kq * 4);
    }
  };

  // The first range of a context is hardly ever empty: its first step is asked for before the positions have arrived.
  if (range == 0 && kb0 < capacity) { load_v(0, capacity); load_k(0, capacity); }

  bf16x8 qf[NRT][NQ][KSQ];                           // (fp32: three bf16 numbers hold 24 bits)
#pragma unroll
  for (int rt = 0; rt < NRT; ++rt)
#pragma unroll
    for (int s = 0; s < KSQ; ++s) {
      if constexpr (sizeof(T) == 2) qf[rt][0][s] = __builtin_bit_cast(bf16x8, q_raw[rt][s][0]);
      else {
        f32x4 x[2] = {__builtin_bit_cast(f32x4, q_raw[rt][s][0]), __builtin_bit_cast(f32x4, q_raw[rt][s][QL - 1])};
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          u32x4 w;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int h = e >> 1, r = (e & 1) * 2;
            w[e] = bf16_pair(x[h][r], x[h][r + 1]);
            x[h][r] -= __uint_as_float(w[e] << 16);
            x[h][r + 1] -= __uint_as_float(w[e] & 0xffff0000u);
          }
          qf[rt][n][s] = __builtin_bit_cast(bf16x8, w);
        }
      }
    }
  float m_run[NRT], l_run[NRT];
  f32x4 o[DT][NRT];
#pragma unroll
  for (int rt = 0; rt < NRT; ++rt) {
    m_run[rt] = -INFINITY; l_run[rt] = 0.0f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt][rt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  unsigned char *vt = lds + wave * S::STAGE, *kt_lds = vt + STEP * RB;
  // where this lane's transposing reads begin: e4m3 row s / 2 of the eight keys 4 kq + {0..3, 16..19}, bf16 row s / 4 of four keys
  const int tr_row = E4M3 ? ((j >> 3) * 16 + kq * 4 + (j >> 1 & 3)) : (kq * 4 + (j >> 2));
  const int tr_at = tr_row * RB + (E4M3 ? 8 * (j & 1) : 8 * (j & 3)), tr_swz = kv_swizzle<DH, E4M3>(tr_row);
  // features dt 16 + j of the 32 keys of a half of the step, as the product takes them: slot 8 kq + e is key (e / 4) 16 + 4 kq + e % 4
  auto v_frag = [&](int half, int dt) {
    bf16x8 vf;
    if constexpr (E4M3) {
      typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
      const i32x2 x = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)(vt + half * 32 * RB + (tr_at + ((dt ^ tr_swz) << 4))));
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)x[w], 1.0f, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)x[w], 1.0f, true);
        vf[4 * w] = lo[0]; vf[4 * w + 1] = lo[1]; vf[4 * w + 2] = hi[0]; vf[4 * w + 3] = hi[1];
      }
    } else {
      typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
      const unsigned char* vp = vt + half * 32 * RB + (tr_at + ((dt ^ tr_swz) << 5));           // (rows 16 apart are swizzled alike)
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)vp);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vp + 16 * RB));
      const s16x8 vb = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      vf = __builtin_bit_cast(bf16x8, vb);
    }
    return vf;
  };
  auto v_to_lds = [&](const u32x4 (&x)[NV]) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");     // what was read before is done
#pragma unroll
    for (int c = 0; c < NV; ++c) {
      const int row = c * S::RPL + vrow, sw = kv_swizzle<DH, E4M3>(row);
      const int at = E4M3 ? ((vpiece ^ sw) * 16) : (((vpiece >> 1) ^ sw) * 32 + (vpiece & 1) * 16);
      *reinterpret_cast<u32x4*>(vt + row * RB + at) = x[c];
    }
  };

  auto k_to_lds = [&](const u32x4* x) {
#pragma unroll
    for (int c = 0; c < NV; ++c) {
      const int row = c * S::RPL + vrow;
      *reinterpret_cast<u32x4*>(kt_lds + row * RB + (vpiece ^ kv_swizzle_k<DH, E4M3>(row)) * 16) = x[c];
    }
  };

  int far = pos[0], near = pos[0] < 0 ? 0x7fffffff : pos[0];
#pragma unroll
  for (int rt = 1; rt < NRT; ++rt) { far = max(far, pos[rt]); near = min(near, pos[rt] < 0 ? 0x7fffffff : pos[rt]); }
  const int kv_len = __builtin_amdgcn_readfirstlane(min(wave_max(far), capacity - 1)) + 1;      // keys that some row sees
  const int pos_min = __builtin_amdgcn_readfirstlane(min(wave_min(near), capacity - 1));        // every row that sees any sees these
  const int n_act = max(1, (kv_len + a.range_keys - 1) / a.range_keys);
  if (range >= n_act) return;
  const int end = min(kv_len, range0 + a.range_keys);
  if (range > 0 && kb0 < end) { load_v(0, end); load_k(0, end); }
  for (int i = 0, kb = kb0; kb < end; ++i, kb += TURN) {
    const unsigned tiles_ok = (unsigned)(ok_tiles >> ((i * KT) & 63)) & ((1u << KT) - 1u);
    const bool clean = kb + STEP - 1 <= pos_min && tiles_ok == (1u << KT) - 1u;        // uniform: every row sees every key of the step
    // ---- K and V into LDS; their registers take the next step's ----
    if (!clean) {
      unsigned bad = 0;
#pragma unroll
      for (int c = 0; c < NV; ++c) {
        const int row = c * S::RPL + vrow;
        const bool gone = kb + row >= end || !(tiles_ok >> (row >> 4) & 1u);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          if (gone) vr[c][w] = 0u;
          bad |= E4M3 ? ((vr[c][w] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u : ((vr[c][w] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
        }
      }
      if (E4M3) {                                    // (an exponent that nobody wrote may be that of an infinity)
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) ve[kt] -= (((ve[kt] & 0x7f7f7f7fu) + 0x01010101u) & ve[kt] & 0x80808080u) >> 7;
      }
      if (pos_min + 1 < kv_len && __builtin_amdgcn_ballot_w64(bad != 0u) != 0ull) {      // rare: some V that not every row sees is not finite
        // ones in its place, and a mark for the rows that see one; then zeros in its place
        u32x4 odd[NV];
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            if (E4M3) {
              const unsigned no = (((vr[c][w] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7;
              odd[c][w] = no * 0x38u;
              vr[c][w] &= ~(no * 0xffu);
            } else {
              const unsigned no = (((vr[c][w] & 0x7f807f80u) + 0x00800080u) & 0x80008000u) >> 15;
              odd[c][w] = no * 0x3f80u;
              vr[c][w] &= ~(no * 0xffffu);
            }
          }
        v_to_lds(odd);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
#pragma unroll
        for (int half = 0; half < KT / 2; ++half)
#pragma unroll
          for (int rt = 0; rt < NRT; ++rt) {
            u32x4 sees;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              const int key = kb + half * 32 + (w >> 1) * 16 + kq * 4 + (w & 1) * 2;
              sees[w] = (key <= pos[rt] ? 0x3f80u : 0u) | (key + 1 <= pos[rt] ? 0x3f800000u : 0u);
            }
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
              const f32x4 n = mma_bf16(v_frag(half, dt), __builtin_bit_cast(bf16x8, sees), f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
              for (int r = 0; r < 4; ++r) o[dt][rt][r] += (n[r] > 0.0f) ? __uint_as_float(0x7fc00000u) : 0.0f;
            }
          }
      }
    }
    v_to_lds(vr);
    if constexpr (S::LDS_K) k_to_lds(kr);
    unsigned ks[KT], vs[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) { ks[kt] = E4M3 ? ke[kt] : 0u; vs[kt] = E4M3 ? ve[kt] : 0u; }
    load_v(i + 1, end);
    if constexpr (S::LDS_K) {
      load_k(i + 1, end);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");   // this step's rows have landed in LDS
    }
    // ---- scores: sc[kt][rt][r] = S[key kb + kt 16 + kq 4 + r][pair rt 16 + j] ----
    f32x4 sc[KT][NRT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      u32x4 kx[KL];
#pragma unroll
      for (int l = 0; l < KL; ++l) {
        if constexpr (!S::LDS_K) kx[l] = kr[kt * KL + l];
        else {
          const int row = kt * 16 + j, at = (l * 4 + kq) * S::FPL * S::ES;
          const unsigned char* from = kt_lds + row * RB + ((at >> 4) ^ kv_swizzle_k<DH, E4M3>(row)) * 16;
          if constexpr (S::FPL * S::ES == 16) kx[l] = *reinterpret_cast<const u32x4*>(from);
          else { const u32x2 x = *reinterpret_cast<const u32x2*>(from + (at & 15)); kx[l] = u32x4{x[0], x[1], 0u, 0u}; }
        }
      }
      bf16x8 kf[KSQ];
      if constexpr (E4M3) {
        const float s2 = __uint_as_float(ks[kt] << 23);
#pragma unroll
        for (int s = 0; s < KSQ; ++s) {
          constexpr int U = S::FPL / 8;
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            const unsigned x = kx[s / U][(s % U) * 2 + w];
            const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, s2, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, s2, true);
            kf[s][4 * w] = lo[0]; kf[s][4 * w + 1] = lo[1]; kf[s][4 * w + 2] = hi[0]; kf[s][4 * w + 3] = hi[1];
          }
        }
      } else {
#pragma unroll
        for (int s = 0; s < KSQ; ++s) kf[s] = __builtin_bit_cast(bf16x8, kx[s]);
      }
#pragma unroll
      for (int rt = 0; rt < NRT; ++rt) {
        sc[kt][rt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int n = NQ - 1; n >= 0; --n)
#pragma unroll
          for (int s = 0; s < KSQ; ++s) sc[kt][rt] = mma_bf16(kf[s], qf[rt][n][s], sc[kt][rt]);
      }
    }
    if constexpr (!S::LDS_K) load_k(i + 1, end);
    // ---- softmax: the reference m_run only moves when scores outgrow it by 2^8 ----
    float f[NRT];
    bool rescale = false;
#pragma unroll
    for (int rt = 0; rt < NRT; ++rt) {
      if (!clean) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int key = kb + kt * 16 + kq * 4 + r;
            if (key >= end || key > pos[rt] || !(tiles_ok >> kt & 1u)) sc[kt][rt][r] = -INFINITY;
          }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, sc[kt][rt][r]);
      mx = lane_combine<16>(mx, OpMaxF());
      mx = lane_combine<32>(mx, OpMaxF());
      mx *= a.c_log2;
      const float m_old = m_run[rt], m_new = (mx > m_old + 8.0f || m_old == -INFINITY) ? fmaxf(m_old, mx) : m_old;
      f[rt] = (m_new == m_old) ? 1.0f : __builtin_amdgcn_exp2f(m_old - m_new);
      rescale = rescale || f[rt] != 1.0f;
      const float ref = (m_new == -INFINITY) ? 0.0f : m_new;
      float sum = 0.0f;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          sc[kt][rt][r] = __builtin_amdgcn_exp2f(fmaf(sc[kt][rt][r], a.c_log2, -ref));
          sum += sc[kt][rt][r];
        }
      l_run[rt] = fmaf(l_run[rt], f[rt], sum);       // this lane's keys; the quarters are added at the end
      m_run[rt] = m_new;
    }
    if (__builtin_amdgcn_ballot_w64(rescale) != 0ull) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int rt = 0; rt < NRT; ++rt)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[dt][rt][r] *= f[rt];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");     // this step's V has landed in LDS
    // ---- O^T += V^T P, 32 keys at a time ----
#pragma unroll
    for (int half = 0; half < KT / 2; ++half) {
      u32x4 pf[NRT][NP];
#pragma unroll
      for (int rt = 0; rt < NRT; ++rt)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const int kt = half * 2 + (w >> 1), r = (w & 1) * 2;
          float x = sc[kt][rt][r], y = sc[kt][rt][r + 1];
          if (E4M3) {
            x *= __uint_as_float((vs[kt] >> (8 * r) & 0xffu) << 23);
            y *= __uint_as_float((vs[kt] >> (8 * r + 8) & 0xffu) << 23);
          }
#pragma unroll
          for (int n = 0; n < NP; ++n) {
            const unsigned both = bf16_pair(x, y);
            pf[rt][n][w] = both;
            x -= __uint_as_float(both << 16);
            y -= __uint_as_float(both & 0xffff0000u);
          }
        }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const bf16x8 vf = v_frag(half, dt);
#pragma unroll
        for (int rt = 0; rt < NRT; ++rt)
#pragma unroll
          for (int n = NP - 1; n >= 0; --n) o[dt][rt] = mma_bf16(vf, __builtin_bit_cast(bf16x8, pf[rt][n]), o[dt][rt]);
      }
    }
  }

  // ---- join the wavefronts: each leaves O, m, l of its keys in LDS, rows of DH + 4 ----
  constexpr int D4 = DH / 4, NT = 64 * NW;
  float* mg = reinterpret_cast<float*>(lds);
  const size_t apart = (size_t)a.rows_wg * (DH + 2);            // floats from one range's results to the next's
  float* first = (n_act > 1) ? a.partial + (((size_t)seq * a.groups + grp) * a.c.Hkv + hkv) * a.n_ranges * apart : nullptr;
  auto write = [&](int g, int d, const f32x4& x, float m, float l) {           // the finished features d .. d + 3 of pair g
    const int r = a.by_g.quotient(rg0 + g), h = hkv * G + rg0 + g - r * G, row = seq * a.R + r;
    const bool none = l == 0.0f;
    if (a.lse != nullptr && d == 0) a.lse[(size_t)row * a.H + h] = none ? -INFINITY : fmaf(m, 0.6931471805599453f, logf(l));
    f32x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = none ? 0.0f : x[e] / l;
    size_t at = ((size_t)row * a.H + h) * DH + d;
    if constexpr (sizeof(T) == 2) {
      bf16* to = static_cast<bf16*>(a.out);
      if (a.out_frag != nullptr) {
        const int n = h * DH + d;
        to = a.out_frag;
        at = (((size_t)(n >> 5) * a.frag_ks + (size_t)(row >> 4) * a.frag_slab) * 64 + (row & 15) + 16 * ((n & 31) >> 3)) * 8 + (n & 7);
      }
      *reinterpret_cast<uint2*>(to + at) = make_uint2(bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3]));
    } else *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + at) = y;
  };
#pragma unroll
  for (int rt = 0; rt < NRT; ++rt) {
    __syncthreads();                                 // (V's region, or the tile before, is no longer in use)
    float l = lane_combine<16>(l_run[rt], OpSumF());
    l = lane_combine<32>(l, OpSumF());
    float* mine = mg + (wave * KV_ROWS + j) * (DH + 4);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4*>(mine + dt * 16 + kq * 4) = o[dt][rt];
    // (a row that sees nothing was carried along in the steps that need no mask)
    if (kq == 0) *reinterpret_cast<float2*>(mine + DH) = (pos[rt] < 0) ? make_float2(-INFINITY, 0.0f) : make_float2(m_run[rt], l);
    __syncthreads();
    for (int i = tid; i < min(RG - rt * KV_ROWS, KV_ROWS) * D4; i += NT) {
      const int g = i / D4, d = (i % D4) * 4;
      float mw[NW], lw[NW], m = -INFINITY, L = 0.0f;
      f32x4 ow[NW], acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float* from = mg + (w * KV_ROWS + g) * (DH + 4);
        const float2 x = *reinterpret_cast<const float2*>(from + DH);
        mw[w] = x.x; lw[w] = x.y; ow[w] = *reinterpret_cast<const f32x4*>(from + d);
        m = fmaxf(m, mw[w]);
      }
#pragma unroll
      for (int w = 0; w < NW; ++w) {                 // (a wavefront without keys, and a row without any, count as nothing)
        const float e = (mw[w] == -INFINITY) ? 0.0f : __builtin_amdgcn_exp2f(mw[w] - m);
        L = fmaf(lw[w], e, L);
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[r] = (mw[w] == -INFINITY && lw[w] == 0.0f) ? acc[r] : fmaf(ow[w][r], e, acc[r]);
      }
      const int rg = rt * KV_ROWS + g;
      if (n_act == 1) write(rg, d, acc, m, L);
      else {
        float* to = first + range * apart + rg * DH + d;
        post8(to, acc[0], acc[1]); post8(to + 2, acc[2], acc[3]);
        if (d == 0) post8(first + range * apart + a.rows_wg * DH + rg * 2, m, L);
      }
    }
  }
  if (n_act == 1) return;
  unsigned* ticket = a.tickets + ((size_t)seq * a.groups + grp) * a.c.Hkv + hkv;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this wavefront's posts have reached memory
  __syncthreads();
  if (tid == 0) {
    const int last = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (unsigned)n_act - 1u;
    last_wg = last;
    if (last) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (last_wg == 0) return;
  // ---- join the ranges: weights 2^(m_s - m) of every range and row, then the sum of the ranges' outputs.  A thread takes four features of a
  //      pair, and where the pairs leave threads over a part of the ranges (part, part + parts, ..); NB of them are asked for at once, the first ahead of the (m, l) ----
  const int items = RG * D4, parts = max(1, NT / items), part = (parts > 1) ? tid / items : 0, item = (parts > 1) ? tid - part * items : tid;
  constexpr int NB = 8;
  float2 lo[NB], hi[NB];
  auto ask = [&](int x0, int it) {
#pragma unroll
    for (int u = 0; u < NB; ++u) {
      const float* from = first + min(x0 + u * parts, n_act - 1) * apart + min(it, items - 1) * 4;
      lo[u] = collect8(from); hi[u] = collect8(from + 2);
    }
  };
  float2* ml = reinterpret_cast<float2*>(lds);       // [range][RG]
  for (int i = tid; i < n_act * RG; i += NT) {
    const int x = i / RG, g = i - x * RG;
    ml[i] = collect8(first + x * apart + a.rows_wg * DH + g * 2);
  }
  ask(part, item);
  __syncthreads();
  for (int g = tid >> 4; g < RG; g += NT / 16) {     // 16 lanes a row
    float m = -INFINITY, L = 0.0f;
    for (int x = j; x < n_act; x += 16) m = fmaxf(m, ml[x * RG + g].x);
    m = lane_combine<1>(m, OpMaxF()); m = lane_combine<2>(m, OpMaxF()); m = lane_combine<4>(m, OpMaxF()); m = lane_combine<8>(m, OpMaxF());
    for (int x = j; x < n_act; x += 16) {
      const float2 p = ml[x * RG + g];
      const float e = (p.x == -INFINITY) ? 0.0f : __builtin_amdgcn_exp2f(p.x - m);
      L = fmaf(p.y, e, L);
      ml[x * RG + g].x = e;
    }
    L = lane_combine<1>(L, OpSumF()); L = lane_combine<2>(L, OpSumF()); L = lane_combine<4>(L, OpSumF()); L = lane_combine<8>(L, OpSumF());
    if (j == 0) { row_m[g] = m; row_l[g] = L; }
  }
  __syncthreads();
  f32x4* sums = reinterpret_cast<f32x4*>(lds + S::ML);                         // [part][item]
  for (int it = item; it < items; it += NT) {        // (several items a thread: one part)
    const int g = it / D4, d = (it % D4) * 4;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (part < parts) {
      for (int x0 = part; x0 < n_act; x0 += NB * parts) {
        if (x0 != part || it != item) ask(x0, it);
#pragma unroll
        for (int u = 0; u < NB; ++u)
          if (x0 + u * parts < n_act) {
            const float w = ml[(x0 + u * parts) * RG + g].x;
            acc[0] = fmaf(lo[u].x, w, acc[0]); acc[1] = fmaf(lo[u].y, w, acc[1]); acc[2] = fmaf(hi[u].x, w, acc[2]); acc[3] = fmaf(hi[u].y, w, acc[3]);
          }
      }
    }
    if (parts == 1) write(g, d, acc, row_m[g], row_l[g]);
    else if (part < parts) sums[part * items + it] = acc;
  }
  if (parts == 1) return;
  __syncthreads();
  if (part == 0) {
    f32x4 acc = sums[item];
    for (int p = 1; p < parts; ++p) acc += sums[p * items + item];
    write(item / D4, (item % D4) * 4, acc, row_m[item / D4], row_l[item / D4]);
  }
}

// ---------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------
constexpr int KV_TICKETS = 65536;                    // (sequence, group, kv head)s of a call
constexpr size_t KV_TICKET_BYTES = (size_t)KV_TICKETS * sizeof(unsigned);

// How a call is cut into workgroups.  `pairs`: (row, query head) pairs of a kv head.  Measured in graphs over three sets of inputs, us a call; 8 kv heads
// of 128 in e4m3 and 4 query heads each unless said.
//   Calls over 128 MB of keys and values or more are bound by memory: loads past the L2s where one workgroup reads a line (64 sequences of 8192, one row 198 -> 184; what
//   several groups read is left in them: two groups of two tiles 335 -> 350), and two tiles of pairs a workgroup (64 of 8192, 5 rows 298 -> 200, 64 of 2048 81 -> 56).  Below
//   that one tile and more workgroups (16 of 2048, 5 rows 16.3 against 22; one of 500 7.8 against 10.5), and plain loads (16 of 2048, one row 15.3 against 17.3: the
//   memory-side cache holds them from call to call).   In bf16 caches of heads of 128 also below it, where the
//   groups of one tile are more than the CUs (18 of 1000 25.2 -> 17.9, 60 of 200 19.4 -> 15.3, 30 of 500 16.6 -> 15.9; in e4m3 17.3 -> 16.3, 24.1 -> 25.3, 22.3 -> 22.9).  fp32 queries have no
//   registers for two tiles.
//   Ranges: where there are fewer workgroups than CUs, as many as fill those, or twice as many where a row is under 128 bytes (2 sequences of 108567, 2 heads of 32
//   24.1 -> 16.7; 4 of 6874, 12 of 64 14.7 -> 13.5; with rows of 128 bytes 4 of 8192 20.8 -> 21.7).  Not for short contexts, where the join (2.6 us for heads of 128) costs more than
//   the steps that it saves: a step takes 0.9 us for heads of 128, 0.69 for 64, 0.56 for 32 (one sequence of 500 7.2 against 8.4 in two ranges, of 1000 10.4 against 8.4 in
//   four; 12 heads of 64: 1500 11.2 against 8.4 in six; 2 of 32: 1000 7.8 against 7.4, 3000 16.7 against 7.3 in twelve), later where eight wavefronts can take them (16 of 2048 15.3,
//   16.8 in two; one of 1200 with 64 heads of 64 8.7, 9.2 in five); nor more than the join is worth, which is the less the shorter the rows (one of 8192 in 8, 16, 32 ranges 13.9, 11.7,
//   13.3; of 32768 in 16, 32, 64 20.9, 19.0, 23.9; 2 heads of 32, 16384 in 16, 43, 64 10.7, 9.0, 9.0).  At most 4096 keys (64 of 8192 in ranges of 1024, 2048, 4096 199, 180, 176;
//   contexts of all lengths up to that 127, 123, 125).
//   Eight wavefronts for 512 keys or more where a CU has at most one workgroup (16 of 2048 15.3, 17.3 with four; 64 of 1200 with 2 heads of 32 7.9, 9.2; 64 of 2048 56.8, 52.6), and where
//   workgroups are few only for contexts in one range (one of 700 8.3, 8.8, with 12 heads of 64 6.7, 7.4; 4 of 8192 18.7, 17.6), and of
//   bf16 caches only for heads of 32 (16 of 1000 15.9, 14.4; 8 of 1000 with 12 heads of 64 9.6, 9.3; 64 of 2000 with 2 of 32 9.5, 11.3).
struct KvPlan { int rows_wg, groups, range_keys, n_ranges, waves; bool large, once; };
constexpr bool kv_eight_waves(int d_head, bool e4m3) { return e4m3 || d_head == 32; }
// What the sums of a row depend on: the ranges and the wavefronts.  wgs: (sequence, kv head, group)s.
inline void kv_plan_ranges(KvPlan& p, long long wgs, long long heads, int max_len, int d_head, bool e4m3) {
  p.large = heads * max_len * 2 * d_head * (e4m3 ? 1 : 2) >= 128ll << 20;
  const long long per_cu = wgs < 256 ? 256 / wgs : 1;
  long long ranges = 1;
  if (p.large) ranges = per_cu;
  else if (wgs < 64 ? (long long)max_len * (d_head + 128) >= 768 * 256 : (long long)max_len * d_head >= (per_cu > 2 ? 768 : 2560) * 128) {
    const long long most = per_cu > 2 && d_head * (e4m3 ? 1 : 2) < 128 ? 512 / wgs : per_cu, parts = (max_len + 255) / 256;
    ranges = most < parts ? most : parts;
    while (ranges > 1 && 100 * ranges * ranges * d_head > 3 * 128 * (long long)max_len) --ranges;
  }
  long long keys = (max_len + ranges - 1) / ranges;
  p.waves = (kv_eight_waves(d_head, e4m3) && !p.large && wgs <= 256 && (wgs >= 64 || ranges == 1) && keys >= 512 && p.rows_wg <= KV_ROWS) ? 8 : 4;
  const long long unit = 32 * p.waves, least = ((long long)max_len + KV_MAX_RANGES - 1) / KV_MAX_RANGES, longest = KV_MAX_RANGE_KEYS;
  if (keys > longest) keys = longest;
  if (keys < least) keys = least;
  p.range_keys = (int)((keys + unit - 1) / unit * unit);
  p.n_ranges = (max_len + p.range_keys - 1) / p.range_keys;
}
// What they do not depend on: how the rows are grouped.
inline void kv_plan_rows(KvPlan& p, long long heads, int pairs, int max_len, int d_head, bool e4m3, bool f32) {
  p.large = heads * max_len * 2 * d_head * (e4m3 ? 1 : 2) >= 128ll << 20;
  const bool many = heads * ((pairs + KV_ROWS - 1) / KV_ROWS) > 256 && !e4m3 && d_head == 128;
  const int most = ((p.large || many) && !f32) ? 2 * KV_ROWS : KV_ROWS;
  p.groups = (pairs + most - 1) / most;
  p.rows_wg = (pairs + p.groups - 1) / p.groups;
  p.once = p.large && p.groups == 1;
}
inline KvPlan kv_plan(int n_seq, int Hkv, int pairs, int max_len, int d_head, bool e4m3, bool f32) {
  KvPlan p{};
  const long long heads = (long long)n_seq * Hkv;
  kv_plan_rows(p, heads, pairs, max_len, d_head, e4m3, f32);
  kv_plan_ranges(p, heads * p.groups, heads, max_len, d_head, e4m3);
  return p;
}
inline size_t kv_scratch_bytes(int n_seq, int Hkv, int d_head, const KvPlan& p) {
  const size_t partial = p.n_ranges > 1 ? (size_t)n_seq * p.groups * Hkv * p.n_ranges * p.rows_wg * (d_head + 2) * sizeof(float) : 0;
  return KV_TICKET_BYTES + partial;
}

template <typename F> void kv_with_head(int d_head, F&& f) {
  if (d_head == 32) f(std::integral_constant<int, 32>());
  else if (d_head == 64) f(std::integral_constant<int, 64>());
  else f(std::integral_constant<int, 128>());
}
template <typename T> void launch_kv_rows(hipStream_t s, const KvRowsArgs& a, int d_head, bool e4m3, bool append) {
  kv_with_head(d_head, [&](auto dh) {
    constexpr int DH = decltype(dh)::value;
    constexpr int ROWS = KV_ROW_BYTES / (DH * (int)sizeof(T));                 // of a workgroup
    const dim3 grid((unsigned)((a.rows + ROWS - 1) / ROWS) * (unsigned)a.c.Hkv);
    auto launch = [&](auto past) {
      constexpr bool P = decltype(past)::value;
      if (append && e4m3) hipLaunchKernelGGL((kv_append_kernel<T, DH, true, P>), grid, dim3(256), 0, s, a);
      else if (append) hipLaunchKernelGGL((kv_append_kernel<T, DH, false, P>), grid, dim3(256), 0, s, a);
      else if (e4m3) hipLaunchKernelGGL((kv_read_kernel<T, DH, true, P>), grid, dim3(256), 0, s, a);
      else hipLaunchKernelGGL((kv_read_kernel<T, DH, false, P>), grid, dim3(256), 0, s, a);
    };
    const size_t written = (size_t)a.rows * a.c.Hkv * 2 * DH * (append ? (e4m3 ? 1 : 2) : sizeof(T));
    if (written >= (size_t)(a.paged ? 32 : 8) << 20) launch(std::true_type());
    else launch(std::false_type());
  });
}
inline void kv_set_plan(KvAttnArgs& a, const KvPlan& p) {          // (a.G, a.c and a.n_seq are set)
  a.groups = p.groups; a.rows_wg = p.rows_wg; a.range_keys = p.range_keys; a.n_ranges = p.n_ranges;
  a.by_g.set(a.G); a.by_groups.set(a.groups); a.by_hkv.set(a.c.Hkv);
}
template <typename T> void launch_kv_attention(hipStream_t s, const KvAttnArgs& a, int d_head, bool e4m3, int n_seq, const KvPlan& p) {
  kv_with_head(d_head, [&](auto dh) {
    constexpr int DH = decltype(dh)::value;
    const dim3 grid((unsigned)((n_seq * a.c.Hkv + 7) / 8 * 8 * p.groups), (unsigned)p.n_ranges), block(64 * p.waves);
    auto launch = [&](auto nw, auto nrt, auto codes, auto once) {
      hipLaunchKernelGGL((kv_attention_kernel<T, DH, decltype(nw)::value, decltype(nrt)::value, decltype(codes)::value, decltype(once)::value>), grid, block, 0, s, a);
    };
    const auto one = std::integral_constant<int, 1>();
    const auto two = std::integral_constant<int, 2>();
    auto with_cache = [&](auto codes) {
      if constexpr (kv_eight_waves(DH, decltype(codes)::value)) {
        if (p.waves == 8) { launch(std::integral_constant<int, 8>(), one, codes, std::false_type()); return; }
      }
      if (p.rows_wg <= KV_ROWS) {
        if (p.once) launch(std::integral_constant<int, 4>(), one, codes, std::true_type());
        else launch(std::integral_constant<int, 4>(), one, codes, std::false_type());
      } else if constexpr (sizeof(T) == 2) {         // (fp32 queries: one tile)
        if (p.once) launch(std::integral_constant<int, 4>(), two, codes, std::true_type());
        else launch(std::integral_constant<int, 4>(), two, codes, std::false_type());
      }
    };
    if (e4m3) with_cache(std::true_type());
    else with_cache(std::false_type());
  });
}

}  // namespace sd
