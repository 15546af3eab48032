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

// The maximum over groups of 4, 8 or 16 consecutive lanes, in each of them: quads by quad permutes, then the mirror images inside
// 8 and 16 lanes (the quads hold one value each by then).
template <int LANES> __device__ __forceinline__ unsigned group_max(unsigned v) {
  v = max(v, dpp_partner<1>(v));
  v = max(v, dpp_partner<2>(v));
  if (LANES >= 8) v = max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xf, 0xf, true));
  if (LANES >= 16) v = max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xf, 0xf, true));
  return v;
}

__device__ __forceinline__ float two_to(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }

// Eight consecutive elements per thread, DH / 8 threads per row; a thread takes the same row of K and of V.
// grid = (rows / (256 * 8 / DH), kv heads).
template <typename T, int DH, bool E4M3>
static __global__ __launch_bounds__(256) void kv_append_kernel(const KvRowsArgs a) {
  constexpr int LPR = DH / 8;
  const int piece = threadIdx.x % LPR, head = blockIdx.y;
  const int i = (int)(blockIdx.x * (256 / LPR) + threadIdx.x / LPR);
  const int ic = min(i, a.rows - 1);
  const long long at = kv_place(a, ic);
  const long long apart = (long long)a.c.Hkv << a.c.page_shift;                // rows of the pool from K to V
  const long long row = max(at, 0ll) + ((long long)head << a.c.page_shift);
  const T* from[2] = {static_cast<const T*>(a.k) + (a.paged ? row * DH : ic * a.k_row + head * a.k_head),
                      static_cast<const T*>(a.v) + (a.paged ? (row + apart) * DH : ic * a.v_row + head * a.v_head)};
  float x[2][8];
  load8<T>(from[0] + piece * 8, x[0]);
  load8<T>(from[1] + piece * 8, x[1]);
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const long long to = row + w * apart;
    if (!E4M3) {
      if (i < a.rows && at >= 0) store8<bf16>(static_cast<bf16*>(a.c.pool) + to * DH + piece * 8, x[w]);
      continue;
    }
    unsigned top = 0;                                // the largest finite magnitude, as bits
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const unsigned m = __float_as_uint(x[w][e]) & 0x7fffffffu;
      if (m >= 0x7f800000u) x[w][e] = __uint_as_float(0x7fc00000u);            // (infinities are kept as NaN)
      else top = max(top, m);
    }
    top = group_max<LPR>(top);
    // 448 = 1.75 * 2^8
    const int E = min(max((int)(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0), KV_EXP_MIN), KV_EXP_MAX);
    const float s = two_to(-E);
    const float most = (E == KV_EXP_MAX) ? 240.0f : 448.0f;                    // (256 * 2^120 would be read as infinity)
#pragma unroll
    for (int e = 0; e < 8; ++e) x[w][e] = (x[w][e] != x[w][e]) ? x[w][e] : __builtin_amdgcn_fmed3f(x[w][e] * s, -most, most);
    unsigned c[2] = {0, 0};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int v = __builtin_amdgcn_cvt_pk_fp8_f32(x[w][4 * h], x[w][4 * h + 1], 0, false);
      c[h] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(x[w][4 * h + 2], x[w][4 * h + 3], v, true);
    }
    if (i < a.rows && at >= 0) {
      *reinterpret_cast<uint2*>(static_cast<unsigned char*>(a.c.pool) + to * DH + piece * 8) = make_uint2(c[0], c[1]);
      if (piece == 0) a.c.exps[to] = (unsigned char)(E + 127);
    }
  }
}

// Eight codes as floats.
__device__ __forceinline__ void e4m3_values(const uint2 c, float scale, float (&x)[8]) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const unsigned w = h ? c.y : c.x;
    const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true);
    x[4 * h] = (float)lo[0]; x[4 * h + 1] = (float)lo[1]; x[4 * h + 2] = (float)hi[0]; x[4 * h + 3] = (float)hi[1];
  }
}

// grid as kv_append_kernel's.
template <typename T, int DH, bool E4M3>
static __global__ __launch_bounds__(256) void kv_read_kernel(const KvRowsArgs a) {
  constexpr int LPR = DH / 8;
  const int piece = threadIdx.x % LPR, head = blockIdx.y;
  const int i = (int)(blockIdx.x * (256 / LPR) + threadIdx.x / LPR);
  const int ic = min(i, a.rows - 1);
  const long long at = kv_place(a, ic);
  const long long apart = (long long)a.c.Hkv << a.c.page_shift;
  const long long row = max(at, 0ll) + ((long long)head << a.c.page_shift);
  float x[2][8];
  if (E4M3) {
    uint2 c[2];
    unsigned e[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      c[w] = *reinterpret_cast<const uint2*>(static_cast<const unsigned char*>(a.c.pool) + (row + w * apart) * DH + piece * 8);
      e[w] = a.c.exps[row + w * apart];
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) e4m3_values(c[w], __uint_as_float(e[w] << 23), x[w]);
  } else {
    load8<bf16>(static_cast<const bf16*>(a.c.pool) + row * DH + piece * 8, x[0]);
    load8<bf16>(static_cast<const bf16*>(a.c.pool) + (row + apart) * DH + piece * 8, x[1]);
  }
  if (at < 0) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[0][e] = x[1][e] = 0.0f;
    if (a.paged) return;
  }
  if (i >= a.rows) return;
  store8<T>(static_cast<T*>(a.k) + (a.paged ? row * DH : i * a.k_row + head * a.k_head) + piece * 8, x[0]);
  store8<T>(static_cast<T*>(a.v) + (a.paged ? (row + apart) * DH : i * a.v_row + head * a.v_head) + piece * 8, x[1]);
}

// ---------------------------------------------------------------------------
// Attention
// ---------------------------------------------------------------------------
constexpr int KV_NW = 4;                             // wavefronts of a workgroup
constexpr int KV_MAX_RANGES = 128;                   // key ranges of a context at most
constexpr int KV_MAX_RANGE_KEYS = 4096;              // a wavefront holds the page entries of its keys in one register: 64 lanes x 16 keys x 4 wavefronts

struct KvAttnArgs {
  KvCacheArgs c;
  const void* q;            // T: row i, query head h at i * q_row + h * q_head
  long long q_row, q_head;
  void* out;                // T [rows][H][dh]
  float* lse;               // [rows][H], optional
  const int* pos;           // [n_seq * R]: the last key that a row sees, < 0: none
  int R, H, G, seq0;        // rows per sequence, query heads, query heads per kv head; the first sequence's row of the table
  int groups, rows_wg;      // a workgroup takes rows_wg of the R * G (row, head) pairs of a kv head
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
//   S^T = K Q^T   16x16x32, A = 16 keys, B = 16 (row, head) pairs.  A lane loads 16 bytes of its key's row; which features of the row a lane
//                 of the fragment holds is free as long as K and Q agree.  The conversion from e4m3 multiplies by the key's power of two.
//   O^T = V^T P   A = 16 features x 32 keys: V's rows go through the wavefront's own part of LDS and come back transposed
//                 (ds_read_b64_tr_b8 / _b16), B = the probabilities as the lane has them, times V's powers of two.
// Four wavefronts take turns of 64 keys (32 in bf16: 8 KB of K and 8 of V either way), each with its own maximum, sum and output; they are joined
// through LDS.  The keys of a context are cut into ranges, a workgroup each; the last of a (sequence, group, kv head) to arrive
// joins them in range order (posts past the L2s, a relaxed ticket), so a result does not depend on which one that is.
// What a step's loads need is known before the loop: the page entries of all a wavefront's keys lie in one register, a lane each, and a
// tile of 16 keys has one uniform base address.  Loads run one step ahead and are never behind a branch; whole pages are in the pool, so
// slots behind the last key may be read, and whatever lies there (NaN too) is replaced by zeros before the product.
// Rows that see fewer keys than others of the same workgroup: where V of a key that some row does not see is not finite, its product is replaced
// by a mark for the rows that see it (0 * NaN would reach the others).
// grid = (kv heads, sequences, ranges x groups).
template <typename T, int DH, int NRT, bool E4M3> struct KvShape {
  static constexpr int ES = E4M3 ? 1 : 2;            // bytes of an element of the cache
  static constexpr int KT = E4M3 ? 4 : 2;            // key tiles of a step
  static constexpr int STEP = 16 * KT;
  static constexpr int RB = DH * ES;                 // bytes of a row
  static constexpr int FPL = (E4M3 && DH >= 64) ? 16 : 8;                    // features a lane loads of a key at once
  static constexpr int KL = DH / (4 * FPL);          // ... and how often
  static constexpr int PPR = RB / 16;                // 16-byte pieces of a row of V
  static constexpr int RPL = 64 / PPR;               // rows of V per load of the wavefront
  static constexpr int NV = STEP / RPL;
  static constexpr int NQ = sizeof(T) == 4 ? 3 : 1, NP = sizeof(T) == 4 ? 3 : 2;
  static constexpr int STAGE = STEP * RB;            // LDS of a wavefront
  static constexpr int MERGE = KV_NW * 16 * (DH + 4) * 4;
  static constexpr int LDS = (KV_NW * STAGE > MERGE ? KV_NW * STAGE : MERGE) > KV_MAX_RANGES * 16 * NRT * 8
                               ? (KV_NW * STAGE > MERGE ? KV_NW * STAGE : MERGE) : KV_MAX_RANGES * 16 * NRT * 8;
  // registers: of two workgroups a CU, one where two row tiles of split fp32 queries need more
  static constexpr int WGS = (sizeof(T) == 4 && NRT == 2) ? 1 : 2;
};

// Where 16-byte piece `p` of row `row` lies in a wavefront's part of LDS: rows without padding, the 16-feature chunks of a row exchanged so
// that the rows one transposing read takes at a time (e4m3: 8 of each 16-key half; bf16: 8) lie in different banks.
template <int DH, bool E4M3> __device__ __forceinline__ int kv_swizzle(int row) {
  constexpr int RP = 256 / (DH * (E4M3 ? 1 : 2));    // rows a pass over the banks holds
  const int id = E4M3 ? ((row & 7) | ((row >> 4 & 1) << 3)) : (row & 7);
  return id / RP;                                    // (below DH / 16)
}

// Two floats rounded to bf16, the first in the low half.
__device__ __forceinline__ unsigned bf16_pair(float x, float y) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2{x, y}), bf16x2));
}

template <typename T, int DH, int NRT, bool E4M3>
static __global__ __launch_bounds__(64 * KV_NW, (KvShape<T, DH, NRT, E4M3>::WGS)) void kv_attention_kernel(const KvAttnArgs a) {
  using S = KvShape<T, DH, NRT, E4M3>;
  constexpr int KT = S::KT, KL = S::KL, NV = S::NV, NQ = S::NQ, NP = S::NP, STEP = S::STEP, RB = S::RB, DT = DH / 16, KSQ = DH / 32;
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  typedef int i32x2 __attribute__((ext_vector_type(2)));
  __shared__ __align__(256) unsigned char lds[S::LDS];
  __shared__ int last_wg;
  __shared__ float row_m[32], row_l[32];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j = lane & 15, kq = lane >> 4;
  const int hkv = blockIdx.x, seq = blockIdx.y;
  const int range = (int)blockIdx.z / a.groups, grp = (int)blockIdx.z - range * a.groups;
  const int G = a.G, rg0 = grp * a.rows_wg, RG = min(a.rows_wg, a.R * G - rg0);       // this workgroup's (row, head) pairs
  const int range0 = range * a.range_keys;
  const int kb0 = range0 + wave * STEP;

  // ---- positions, page entries, queries: one round of loads ----
  const int* table = a.c.table + (size_t)(a.seq0 + seq) * a.c.table_stride;
  const int my_row = (rg0 + min(lane, RG - 1)) / G;
  const int my_pos = a.pos[seq * a.R + my_row];
  // lane i: the page of the keys of tile i % KT of step i / KT
  const int my_entry = min((kb0 + (lane / KT) * (KV_NW * STEP) + (lane % KT) * 16) >> a.c.page_shift, a.c.table_stride - 1);
  const int my_page = table[my_entry];
  bf16x8 qf[NRT][NQ][KSQ];
  int pos[NRT];
#pragma unroll
  for (int rt = 0; rt < NRT; ++rt) {
    const int rg = rg0 + min(rt * 16 + j, RG - 1), r = rg / G, h = hkv * G + rg - r * G;
    pos[rt] = a.pos[seq * a.R + r];
    const T* qp = static_cast<const T*>(a.q) + (long long)(seq * a.R + r) * a.q_row + (long long)h * a.q_head;
#pragma unroll
    for (int s = 0; s < KSQ; ++s) {
      constexpr int U = S::FPL / 8;
      const T* from = qp + (s / U) * 4 * S::FPL + kq * S::FPL + (s % U) * 8;
      if constexpr (sizeof(T) == 2) qf[rt][0][s] = ld_frag(from);
      else {
        float x[8];
        load8<float>(from, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          qf[rt][0][s][e] = (bf16)x[e];
          const float r1 = x[e] - (float)qf[rt][0][s][e];
          qf[rt][1][s][e] = (bf16)r1;
          qf[rt][2][s][e] = (bf16)(r1 - (float)qf[rt][1][s][e]);
        }
      }
    }
  }
  const int capacity = (int)min((long long)a.max_len, (long long)a.c.table_stride << a.c.page_shift);
  const int kv_len = __builtin_amdgcn_readfirstlane(min(wave_max(my_pos), capacity - 1)) + 1;     // keys that some row sees
  const int pos_min = __builtin_amdgcn_readfirstlane(min(wave_min(my_pos < 0 ? 0x7fffffff : my_pos), capacity - 1));     // every row that sees any sees these
  const int n_act = max(1, (kv_len + a.range_keys - 1) / a.range_keys);
  if (range >= n_act) return;
  const int end = min(kv_len, range0 + a.range_keys);
  const bool page_ok = (unsigned)my_page < (unsigned)a.c.n_pages;
  const unsigned long long ok_tiles = __builtin_amdgcn_ballot_w64(page_ok);
  const int safe_page = page_ok ? my_page : 0;

  // ---- loads ----
  const unsigned page_rows = 2u * (unsigned)a.c.Hkv << a.c.page_shift, v_rows = (unsigned)a.c.Hkv << a.c.page_shift;
  const unsigned slot_mask = (1u << a.c.page_shift) - 1u;
  const int k_lane = j * RB + kq * S::FPL * S::ES;   // this lane's bytes of a key tile
  const int vpiece = lane % S::PPR, vrow = lane / S::PPR;
  // first row of the pool of tile kt of step i (its K); what lies behind the end re-reads a tile that was just read (the step's first, or that of the
  // step before it), which costs no memory traffic
  auto tile_row = [&](int i, int kt) -> unsigned long long {
    const int step = kb0 + i * (KV_NW * STEP);
    const int ii = (step < end) ? i : max(i - 1, 0), t = (step + kt * 16 < end) ? kt : 0;
    const unsigned page = (unsigned)__builtin_amdgcn_readlane(safe_page, ii * KT + t);
    return (unsigned long long)page * page_rows + ((unsigned)hkv << a.c.page_shift) + ((unsigned)(kb0 + ii * (KV_NW * STEP) + t * 16) & slot_mask);
  };
  const unsigned char* pool = static_cast<const unsigned char*>(a.c.pool);
  u32x4 kr[KT][KL], vr[NV];
  unsigned ke[KT], ve[KT];
  auto load_k = [&](int i) {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      const unsigned long long row = tile_row(i, kt);
      const unsigned char* base = pool + row * RB;
#pragma unroll
      for (int l = 0; l < KL; ++l) {
        const unsigned char* p = base + k_lane + l * 4 * S::FPL * S::ES;
        if constexpr (S::FPL * S::ES == 16) kr[kt][l] = *reinterpret_cast<const u32x4*>(p);
        else { const uint2 x = *reinterpret_cast<const uint2*>(p); kr[kt][l] = u32x4{x.x, x.y, 0u, 0u}; }
      }
      if (E4M3) ke[kt] = *(a.c.exps + row + j);
    }
  };
  auto load_v = [&](int i) {
    unsigned long long row[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) row[kt] = tile_row(i, kt) + v_rows;
#pragma unroll
    for (int c = 0; c < NV; ++c) {
      // RPL rows a load: within a tile of 16, or two of them
      constexpr int RPL = S::RPL;
      if constexpr (RPL <= 16) vr[c] = *reinterpret_cast<const u32x4*>(pool + (row[c * RPL / 16] + (c * RPL) % 16) * RB + vrow * RB + vpiece * 16);
      else vr[c] = *reinterpret_cast<const u32x4*>(pool + (vrow < 16 ? row[2 * c] : row[2 * c + 1]) * RB + (vrow & 15) * RB + vpiece * 16);
    }
    if (E4M3) {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) ve[kt] = *reinterpret_cast<const unsigned*>(a.c.exps + row[kt] + kq * 4);
    }
  };

  float m_run[NRT], l_run[NRT];
  f32x4 o[DT][NRT];
#pragma unroll
  for (int rt = 0; rt < NRT; ++rt) {
    m_run[rt] = -INFINITY; l_run[rt] = 0.0f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt][rt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  unsigned char* vt = lds + wave * S::STAGE;
  // where this lane's transposing reads begin: e4m3 row s / 2 of the eight keys 4 kq + {0..3, 16..19}, bf16 row s / 4 of four keys
  const int tr_row = E4M3 ? ((j >> 3) * 16 + kq * 4 + (j >> 1 & 3)) : (kq * 4 + (j >> 2));
  const int tr_at = tr_row * RB + (E4M3 ? 8 * (j & 1) : 8 * (j & 3)), tr_swz = kv_swizzle<DH, E4M3>(tr_row);

  if (kb0 < end) { load_v(0); load_k(0); }
  for (int i = 0, kb = kb0; kb < end; ++i, kb += KV_NW * STEP) {
    const unsigned tiles_ok = (unsigned)(ok_tiles >> ((i * KT) & 63)) & ((1u << KT) - 1u);
    const bool clean = kb + STEP - 1 <= pos_min && tiles_ok == (1u << KT) - 1u;        // uniform: every row sees every key of the step
    bool marks = false;                              // some V that not every row sees is not finite
    // ---- V into LDS; its registers take the next step's ----
    if (!clean) {
      unsigned bad = 0;
#pragma unroll
      for (int c = 0; c < NV; ++c) {
        const int row = c * S::RPL + vrow;
        const bool gone = kb + row >= end || !(tiles_ok >> (row >> 4) & 1u);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          if (gone) vr[c][w] = 0u;
          if (E4M3) bad |= ((vr[c][w] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
          else bad |= (((vr[c][w] & 0x7f807f80u) + 0x00800080u) & 0x80008000u);
        }
      }
      marks = pos_min + 1 < kv_len && __builtin_amdgcn_ballot_w64(bad != 0u) != 0ull;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");     // the reads of the previous step are done
#pragma unroll
    for (int c = 0; c < NV; ++c) {
      const int row = c * S::RPL + vrow, sw = kv_swizzle<DH, E4M3>(row);
      const int at = E4M3 ? ((vpiece ^ sw) * 16) : (((vpiece >> 1) ^ sw) * 32 + (vpiece & 1) * 16);
      *reinterpret_cast<u32x4*>(vt + row * RB + at) = vr[c];
    }
    unsigned vs[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) vs[kt] = E4M3 ? ve[kt] : 0u;
    load_v(i + 1);
    // ---- scores: sc[kt][rt][r] = S[key kb + kt 16 + kq 4 + r][pair rt 16 + j] ----
    f32x4 sc[KT][NRT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      bf16x8 kf[KSQ];
      if constexpr (E4M3) {
        const float s2 = __uint_as_float(ke[kt] << 23);
#pragma unroll
        for (int s = 0; s < KSQ; ++s) {
          constexpr int U = S::FPL / 8;
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            const unsigned x = kr[kt][s / U][(s % U) * 2 + w];
            const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, s2, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, s2, true);
            kf[s][4 * w] = lo[0]; kf[s][4 * w + 1] = lo[1]; kf[s][4 * w + 2] = hi[0]; kf[s][4 * w + 3] = hi[1];
          }
        }
      } else {
#pragma unroll
        for (int s = 0; s < KSQ; ++s) kf[s] = __builtin_bit_cast(bf16x8, kr[kt][s]);
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
    load_k(i + 1);
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
          const float e = __builtin_amdgcn_exp2f(fmaf(sc[kt][rt][r], a.c_log2, -ref));
          sc[kt][rt][r] = e;
          sum += e;
        }
      l_run[rt] = l_run[rt] * f[rt] + sum;           // this lane's keys; the quarters are added at the end
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
    // ---- O^T += V^T P, 32 keys at a time: slot 8 kq + e of the product is key (e / 4) 16 + 4 kq + e % 4 of them ----
#pragma unroll
    for (int half = 0; half < KT / 2; ++half) {
      u32x4 pf[NRT][NP];
#pragma unroll
      for (int rt = 0; rt < NRT; ++rt)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const int kt = half * 2 + (w >> 1), r = (w & 1) * 2;
          float x = sc[kt][rt][r], y = sc[kt][rt][r + 1];
          if (E4M3) {                                // (a power of two that nobody wrote may be anything)
            const float sx = __uint_as_float((vs[kt] >> (8 * r) & 0xffu) << 23), sy = __uint_as_float((vs[kt] >> (8 * r + 8) & 0xffu) << 23);
            x = (clean || x != 0.0f) ? x * sx : 0.0f;
            y = (clean || y != 0.0f) ? y * sy : 0.0f;
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
          const unsigned char* vp = vt + half * 32 * RB + (tr_at + ((dt ^ tr_swz) << 5));       // (rows 16 apart are swizzled alike)
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)vp);
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vp + 16 * RB));
          const s16x8 vb = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
          vf = __builtin_bit_cast(bf16x8, vb);
        }
        if (marks) {                                 // uniform, rare
          u32x4 x = __builtin_bit_cast(u32x4, vf), odd;
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const unsigned no = ((x[w] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((x[w] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
            odd[w] = no & 0x3f803f80u;
            x[w] &= ~no;
          }
          vf = __builtin_bit_cast(bf16x8, x);
#pragma unroll
          for (int rt = 0; rt < NRT; ++rt) {
            u32x4 sees;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              const int key = kb + half * 32 + (w >> 1) * 16 + kq * 4 + (w & 1) * 2;
              sees[w] = (key <= pos[rt] ? 0x3f80u : 0u) | (key + 1 <= pos[rt] ? 0x3f800000u : 0u);
            }
            const f32x4 n = mma_bf16(__builtin_bit_cast(bf16x8, odd), __builtin_bit_cast(bf16x8, sees), f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
            for (int r = 0; r < 4; ++r) o[dt][rt][r] += (n[r] > 0.0f) ? __uint_as_float(0x7fc00000u) : 0.0f;
          }
        }
#pragma unroll
        for (int rt = 0; rt < NRT; ++rt)
#pragma unroll
          for (int n = NP - 1; n >= 0; --n) o[dt][rt] = mma_bf16(vf, __builtin_bit_cast(bf16x8, pf[rt][n]), o[dt][rt]);
      }
    }
  }

  // ---- join the wavefronts, a row tile at a time: each leaves O, m, l of its keys in LDS, rows of DH + 4 ----
  constexpr int D4 = DH / 4;
  float* mg = reinterpret_cast<float*>(lds);
  float* part = (n_act > 1) ? a.partial + ((((size_t)seq * a.groups + grp) * a.c.Hkv + hkv) * a.n_ranges + range) * a.rows_wg * (DH + 2) : nullptr;
  auto write = [&](int rg, int d, const f32x4& x, float m, float l) {        // the finished features d .. d + 3 of pair rg
    const int r = (rg0 + rg) / G, h = hkv * G + rg0 + rg - r * G, row = seq * a.R + r;
    const bool none = l == 0.0f;
    if (a.lse != nullptr && d == 0) a.lse[(size_t)row * a.H + h] = none ? -INFINITY : m * 0.6931471805599453f + logf(l);
    T res[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) res[e] = (T)(none ? 0.0f : x[e] / l);
    T* to = static_cast<T*>(a.out) + ((size_t)row * a.H + h) * DH + d;
    if constexpr (sizeof(T) == 2)
      if (a.out_frag != nullptr) {
        const int n = h * DH + d;
        to = reinterpret_cast<T*>(a.out_frag) + (((size_t)(n >> 5) * a.frag_ks + (size_t)(row >> 4) * a.frag_slab) * 64 + (row & 15) + 16 * ((n & 31) >> 3)) * 8 + (n & 7);
      }
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(to) = *reinterpret_cast<const uint2*>(res);
    else *reinterpret_cast<float4*>(to) = make_float4(res[0], res[1], res[2], res[3]);
  };
#pragma unroll
  for (int rt = 0; rt < NRT; ++rt) {
    __syncthreads();                                 // (V's region, or the tile before, is no longer in use)
    float l = lane_combine<16>(l_run[rt], OpSumF());
    l = lane_combine<32>(l, OpSumF());
    float* mine = mg + (wave * 16 + j) * (DH + 4);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4*>(mine + dt * 16 + kq * 4) = o[dt][rt];
    // (a row that sees nothing was carried along in the steps that need no mask)
    if (kq == 0) *reinterpret_cast<float2*>(mine + DH) = (pos[rt] < 0) ? make_float2(-INFINITY, 0.0f) : make_float2(m_run[rt], l);
    __syncthreads();
    for (int i = tid; i < 16 * D4; i += 64 * KV_NW) {
      const int rr = i / D4, rg = rt * 16 + rr, d = (i % D4) * 4;
      if (rg >= RG) continue;
      float mw[KV_NW], lw[KV_NW], m = -INFINITY, L = 0.0f;
      f32x4 ow[KV_NW], acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < KV_NW; ++w) {
        const float* from = mg + (w * 16 + rr) * (DH + 4);
        const float2 x = *reinterpret_cast<const float2*>(from + DH);
        mw[w] = x.x; lw[w] = x.y; ow[w] = *reinterpret_cast<const f32x4*>(from + d);
        m = fmaxf(m, mw[w]);
      }
#pragma unroll
      for (int w = 0; w < KV_NW; ++w) {              // (a wavefront without keys, and a row without any, count as nothing)
        const float e = (mw[w] == -INFINITY) ? 0.0f : __builtin_amdgcn_exp2f(mw[w] - m);
        L += lw[w] * e;
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[r] += (mw[w] == -INFINITY && lw[w] == 0.0f) ? 0.0f : ow[w][r] * e;
      }
      if (n_act == 1) write(rg, d, acc, m, L);
      else {
        float* to = part + rg * DH + d;
        post8(to, acc[0], acc[1]); post8(to + 2, acc[2], acc[3]);
        if (d == 0) post8(part + a.rows_wg * DH + rg * 2, m, L);
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
  // ---- join the ranges: weights 2^(m_s - m) of every range and row, then the sum of the ranges' outputs ----
  const float* first = part - (size_t)range * a.rows_wg * (DH + 2);
  const size_t apart = (size_t)a.rows_wg * (DH + 2);
  float2* ml = reinterpret_cast<float2*>(lds);       // [range][RG]
  for (int i = tid; i < n_act * RG; i += 64 * KV_NW) {
    const int x = i / RG, rg = i - x * RG;
    ml[i] = collect8(first + x * apart + a.rows_wg * DH + rg * 2);
  }
  __syncthreads();
  for (int rg = tid >> 4; rg < RG; rg += 4 * KV_NW) {                          // 16 lanes a row
    float m = -INFINITY, L = 0.0f;
    for (int x = j; x < n_act; x += 16) m = fmaxf(m, ml[x * RG + rg].x);
    m = lane_combine<1>(m, OpMaxF()); m = lane_combine<2>(m, OpMaxF()); m = lane_combine<4>(m, OpMaxF()); m = lane_combine<8>(m, OpMaxF());
    for (int x = j; x < n_act; x += 16) {
      const float2 p = ml[x * RG + rg];
      const float e = (p.x == -INFINITY) ? 0.0f : __builtin_amdgcn_exp2f(p.x - m);
      L += p.y * e;
      ml[x * RG + rg].x = e;
    }
    L = lane_combine<1>(L, OpSumF()); L = lane_combine<2>(L, OpSumF()); L = lane_combine<4>(L, OpSumF()); L = lane_combine<8>(L, OpSumF());
    L = row_first(L);
    if (j == 0) { row_m[rg] = m; row_l[rg] = L; }
  }
  __syncthreads();
  constexpr int NB = 16;                             // ranges asked for at once
  for (int i = tid; i < RG * D4; i += 64 * KV_NW) {
    const int rg = i / D4, d = (i % D4) * 4;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int x0 = 0; x0 < n_act; x0 += NB) {
      float2 lo[NB], hi[NB];
#pragma unroll
      for (int u = 0; u < NB; ++u) {
        const float* from = first + min(x0 + u, n_act - 1) * apart + rg * DH + d;
        lo[u] = collect8(from); hi[u] = collect8(from + 2);
      }
#pragma unroll
      for (int u = 0; u < NB; ++u) {
        const float w = (x0 + u < n_act) ? ml[(x0 + u) * RG + rg].x : 0.0f;
        if (x0 + u < n_act) { acc[0] += lo[u].x * w; acc[1] += lo[u].y * w; acc[2] += hi[u].x * w; acc[3] += hi[u].y * w; }
      }
    }
    write(rg, d, acc, row_m[rg], row_l[rg]);
  }
}

// ---------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------
constexpr int KV_TICKETS = 65536;                    // (sequence, group, kv head)s of a call
constexpr size_t KV_TICKET_BYTES = (size_t)KV_TICKETS * sizeof(unsigned);

// How a call is cut into workgroups.  `pairs`: (row, query head) pairs of a kv head.
struct KvPlan { int rows_wg, groups, range_keys, n_ranges; };
inline KvPlan kv_plan(int n_seq, int Hkv, int pairs, int max_len) {
  KvPlan p;
  p.rows_wg = pairs < 32 ? pairs : 32;
  p.groups = (pairs + 31) / 32;
  const long long wgs = (long long)n_seq * Hkv * p.groups;
  const long long want = (768 + wgs - 1) / wgs;                                // ranges for three workgroups a CU
  const long long keys = ((max_len + want - 1) / want + 255) / 256 * 256;
  long long least = ((long long)max_len + KV_MAX_RANGES - 1) / KV_MAX_RANGES;
  least = (least + 255) / 256 * 256;
  p.range_keys = (int)(keys > 2048 ? 2048 : keys);
  if (p.range_keys < least) p.range_keys = (int)least;
  p.n_ranges = (max_len + p.range_keys - 1) / p.range_keys;
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
    const dim3 grid((unsigned)((a.rows + 2048 / DH - 1) / (2048 / DH)), (unsigned)a.c.Hkv);
    if (append && e4m3) hipLaunchKernelGGL((kv_append_kernel<T, DH, true>), grid, dim3(256), 0, s, a);
    else if (append) hipLaunchKernelGGL((kv_append_kernel<T, DH, false>), grid, dim3(256), 0, s, a);
    else if (e4m3) hipLaunchKernelGGL((kv_read_kernel<T, DH, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((kv_read_kernel<T, DH, false>), grid, dim3(256), 0, s, a);
  });
}
// a.groups, rows_wg, range_keys, n_ranges: kv_plan's.
template <typename T> void launch_kv_attention(hipStream_t s, const KvAttnArgs& a, int d_head, bool e4m3, int n_seq) {
  kv_with_head(d_head, [&](auto dh) {
    constexpr int DH = decltype(dh)::value;
    const dim3 grid((unsigned)a.c.Hkv, (unsigned)n_seq, (unsigned)(a.n_ranges * a.groups)), block(64 * KV_NW);
    if (e4m3 && a.rows_wg <= 16) hipLaunchKernelGGL((kv_attention_kernel<T, DH, 1, true>), grid, block, 0, s, a);
    else if (e4m3) hipLaunchKernelGGL((kv_attention_kernel<T, DH, 2, true>), grid, block, 0, s, a);
    else if (a.rows_wg <= 16) hipLaunchKernelGGL((kv_attention_kernel<T, DH, 1, false>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((kv_attention_kernel<T, DH, 2, false>), grid, block, 0, s, a);
  });
}

}  // namespace sd
