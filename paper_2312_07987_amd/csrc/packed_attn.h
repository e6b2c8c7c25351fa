// Attention over packed sequences with grouped heads (packed_fwd.hip, packed_few.hip, packed_bwd.hip): arguments, geometry, and the
// operand helpers that let one kernel text serve bf16 and fp32 storage.
//
// Rows.  A sequence's queries of one kv head are the rows (token, head of the group): row = token * G + head % G.  All rows of a tile
// read the same keys and values, whatever G is, so short sequences fill tiles G times better and the tile under a causal mask
// ends at its last token.
//
// Slots.  The lengths are on the device, so the host launches an upper bound of the tiles: with tiles of BM rows sequence i owns the
// slots from first(i) = floor(rows before i / BM) + i on, which are at least ceil(rows / BM) many before first(i + 1).  first() rises by
// one or more, a wave finds the slot's sequence with one probe per lane and round (64 sequences one round, 4096 two).  At most one
// slot per sequence is empty.
//
// Levels.  Under a causal mask the tiles differ in length, and a launch that ends with a long one waits for it.  Where the longest sequence is not so
// much longer than the others that the grid would be mostly empty, work-groups are numbered by the tile's distance from the light end of its sequence,
// farthest first: (level, sequence) with as many levels as the longest sequence has tiles.  Tiles then start in falling order of length, and the
// sequence needs no search.  Work-group ids are dealt to the eight XCDs in turn whatever their load, so a sequence's place within a level moves by one
// from level to level (level_seq): with it standing still the longest sequence's tiles met on half of the XCDs (dK / dV of 16384 tokens 365 us
// against 170 by slots).
//
// Operands.  32 x 32 products over 16 reduction indices: lane = 32 g + r holds A[row r][k = 8 g .. 8 g + 7] and B[k][column r], register q of
// the result is D[8 (q / 4) + 4 g + q % 4][column r].  fp32 takes the same 8 values per lane through eight 32x32x2 instructions (the i-th
// multiplies k = i and k = 8 + i), so both types share every index below.
#pragma once
#include "mfma_util.h"

namespace sh {

struct PackedAttn {
  const void *Q, *K, *V, *KP, *VP;
  void* O;
  float* lse;                          // [H][total_q] or NULL
  const int *qoff, *qlen, *koff, *klen;   // qlen, klen may be NULL: the offsets' differences
  int nseq, H, Hk, G, dh, causal, prefix, max_q, max_k;
  int total_q, total_k;
  long q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head, kp_row, kp_head, vp_row, vp_head;
  float scale;
  unsigned g_inv;                      // div_magic(G)
  // Key ranges that other work-groups take as well leave normalised fp32 rows and their log-sum-exp (natural logarithm, -inf: nothing seen):
  // `dense` parts [part][total_q * H] and, from the few-row kernel, [slot * Hk + kv head][frows].
  int nsplit, part0;                   // this launch's parts of the keys, the first one's number; nsplit 0: O is written
  int levels;                          // tiles of the longest sequence: work-groups numbered by level; 0: by slot
  int groups, tall;                    // wave groups of a work-group of 128 rows, 1 or 2; tall: 256 rows (packed_fwd.hip)
  int flat, own;                       // flat: rows of all tokens over the prefix alone; own: the sequence's own keys alone
  float *po, *pl;
  int dhp;                             // part row length: dh rounded up to 4
  int nparts;                          // dense parts in all (the joining kernel)
  int chunk;                           // keys of a few-row work-group (0: all)
  int frows;                           // rows of its parts: max_q * G
  float *fo, *fl;
};

struct PackedAttnBwd {
  PackedAttn f;
  const void* dO;
  const float* delta;                  // [H][total_q]
  void *dQ, *dK, *dV;
  // bf16, head widths of 65 .. 128: score gradients dS^T [kv head][key][row of the sequence], rows of ds_ld, or NULL: computed again for dQ
  void* dS;
  long ds_ld;
  // rows of a dK / dV work-group (a multiple of PACKED_QT): key tiles that see more leave fp32 parts, [part][slot * Hk + kv head][dV, dK] of
  // dkv_floats each, for a second kernel
  int rchunk, rparts;
  int klevels;                         // as levels, of the key tiles
  float* dkv;
  long dkv_floats, kslots;             // (slots * Hk)
};

struct SeqGeom {
  int qbeg, lq, kbeg, lk;
};
__device__ __forceinline__ int clamp_to(int v, int lo, int hi) { return min(max(v, lo), hi); }
// (offsets and lengths come from device memory that the host has not seen: whatever they hold, every row stays inside the tensors)
__device__ __forceinline__ SeqGeom seq_geom(const PackedAttn& a, int i) {
  SeqGeom s;
  s.qbeg = clamp_to(a.qoff[i], 0, a.total_q);
  s.lq = clamp_to(a.qoff[i + 1], s.qbeg, a.total_q) - s.qbeg;
  if (a.qlen) s.lq = clamp_to(a.qlen[i], 0, s.lq);
  s.lq = min(s.lq, a.max_q);
  s.kbeg = clamp_to(a.koff[i], 0, a.total_k);
  s.lk = clamp_to(a.koff[i + 1], s.kbeg, a.total_k) - s.kbeg;
  if (a.klen) s.lk = clamp_to(a.klen[i], 0, s.lk);
  s.lk = min(s.lk, a.max_k);
  return s;
}
__device__ __forceinline__ int first_slot(const int* off, int total, int mul, int tile, int i) {
  return (int)((unsigned)(clamp_to(off[i], 0, total) * mul) / (unsigned)tile) + i;
}
// The sequence of a slot, the slot's number within it and the sequence's places; false for slots that hold nothing: ahead of the first sequence, behind
// the last tile of theirs, and, where offsets fall and the slots' order means nothing, any that is no tile of the sequence it leads to (its number may
// be negative or past 2^31 / tile).  KEYS: slots of `tile` keys, else of `tile` rows of G per query.  In the last round, where the lanes' sequences are neighbours, every lane reads its
// sequence's places along with the offset, so that up to 64 sequences cost one trip to memory.  All 64 lanes must take part.
template <bool KEYS>
__device__ __forceinline__ bool find_slot(const PackedAttn& a, int tile, int slot, int& nth, SeqGeom& s) {
  const int* off = KEYS ? a.koff : a.qoff;
  const int total = KEYS ? a.total_k : a.total_q, mul = KEYS ? 1 : a.G, lane = threadIdx.x & 63;
  int lo = 0, n = a.nseq;
  while (n > 64) {
    const int step = (n + 63) >> 6;
    const unsigned long long m = __ballot(lane * step < n && first_slot(off, total, mul, tile, lo + min(lane * step, n - 1)) <= slot);
    if (!m) return false;
    const int k = __popcll(m) - 1;
    lo += k * step;
    n = min(step, n - k * step);
  }
  const int i = lo + min(lane, n - 1);
  const int f = first_slot(off, total, mul, tile, i);
  const SeqGeom mine = seq_geom(a, i);
  const unsigned long long m = __ballot(lane < n && f <= slot);
  if (!m) return false;
  const int k = __builtin_amdgcn_readfirstlane(__popcll(m) - 1);
  nth = slot - __builtin_amdgcn_readlane(f, k);
  s.qbeg = __builtin_amdgcn_readlane(mine.qbeg, k);
  s.lq = __builtin_amdgcn_readlane(mine.lq, k);
  s.kbeg = __builtin_amdgcn_readlane(mine.kbeg, k);
  s.lk = __builtin_amdgcn_readlane(mine.lk, k);
  return nth >= 0 && (long)nth * tile < (KEYS ? s.lk : s.lq * mul);
}

__device__ __forceinline__ int level_seq(int id, int nseq) { return (id % nseq + id / nseq) % nseq; }

// ---- 16-byte pieces of rows -----------------------------------------------------------------------------------------------
// AL: alignment in bytes of every row (16, 8, or the element): how a piece may be read and written.
template <typename T>
struct Elem;
template <>
struct Elem<bf16_t> {
  typedef unsigned short raw;
  static constexpr int PER = 8;
};
template <>
struct Elem<float> {
  typedef float raw;
  static constexpr int PER = 4;
};

// The piece at element d of a row of dh elements; what lies past dh is read from inside the row and cut off by cut_piece.
template <typename T, int AL>
__device__ __forceinline__ uint4 load_row_piece(const typename Elem<T>::raw* row, int d, int dh) {
  if constexpr (AL == 16) {
    return *(const uint4*)(row + (d < dh ? d : 0));
  } else if constexpr (AL == 8) {
    constexpr int H = Elem<T>::PER / 2;
    const uint2 lo = *(const uint2*)(row + (d < dh ? d : 0)), hi = *(const uint2*)(row + (d + H < dh ? d + H : 0));
    return make_uint4(lo.x, lo.y, hi.x, hi.y);
  } else if constexpr (sizeof(T) == 2) {
    unsigned w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned lo = row[d + 2 * j < dh ? d + 2 * j : 0], hi = row[d + 2 * j + 1 < dh ? d + 2 * j + 1 : 0];
      w[j] = lo | hi << 16;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  } else {
    unsigned w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = __float_as_uint(row[d + j < dh ? d + j : 0]);
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
}
template <typename T, int AL>
__device__ __forceinline__ uint4 cut_piece(uint4 v, int d, int dh) {
  if constexpr (AL == 16) {
    if (d >= dh) v = make_uint4(0, 0, 0, 0);
  } else {
    constexpr int PW = 4 / sizeof(T);   // elements of a word
    unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (d + j * PW >= dh) w[j] = 0;
      if constexpr (AL < 4) {
        if (d + j * PW + 1 >= dh) w[j] &= 0xffffu;
      }
    }
    v = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return v;
}

// NROWS rows on their way from memory to LDS.  load() carries no tests: a row past the last valid one repeats it and a column past dh
// repeats column 0; store() puts zeros in both places (a key that no query sees has probability 0, and 0 times what lies behind a
// sequence need not be 0).  The pieces' places within a tile are worked out once (place): a tile is a uniform base and 32-bit offsets.
template <typename T, int DH, int AL, int NROWS, int NT>
struct PieceTile {
  typedef typename Elem<T>::raw raw;
  static constexpr int PER = Elem<T>::PER, CPR = DH / PER, TOTAL = NROWS * CPR, NCH = (TOTAL + NT - 1) / NT;
  uint4 r[NCH];
  unsigned ro[NCH];   // byte offset of the piece's row
  __device__ __forceinline__ void place(long row_stride, int tid) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) ro[i] = (unsigned)min((tid + i * NT) / CPR, NROWS - 1) * (unsigned)row_stride * (unsigned)sizeof(raw);
  }
  __device__ __forceinline__ void load(const raw* src, long row_stride, int valid, int dh, int tid) {
    const unsigned last = (unsigned)(min(valid, NROWS) - 1) * (unsigned)row_stride * (unsigned)sizeof(raw);   // uniform
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int d = (tid + i * NT) % CPR * PER;
      const unsigned o = min(ro[i], last);
      if constexpr (AL == 16)
        r[i] = *(const uint4*)((const char*)src + (o + (unsigned)(d < dh ? d : 0) * (unsigned)sizeof(raw)));
      else
        r[i] = load_row_piece<T, AL>((const raw*)((const char*)src + o), d, dh);
    }
  }
  __device__ __forceinline__ void store(raw* t, int ld, int valid, int dh, int tid) const {
    const bool whole = valid >= NROWS && dh == DH;   // uniform
    if (whole) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const int c = tid + i * NT;
        if (TOTAL % NT == 0 || c < TOTAL) *(uint4*)(t + c / CPR * ld + c % CPR * PER) = r[i];
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = tid + i * NT, row = c / CPR, d = c % CPR * PER;
      uint4 v = cut_piece<T, AL>(r[i], d, dh);
      const unsigned keep = row < valid ? 0xffffffffu : 0u;
      if (TOTAL % NT == 0 || c < TOTAL) *(uint4*)(t + row * ld + d) = make_uint4(v.x & keep, v.y & keep, v.z & keep, v.w & keep);
    }
  }
};

// ---- operand fragments ----------------------------------------------------------------------------------------------------
struct f32x8 {
  f32x4 lo, hi;
};
template <typename T>
struct FragOf;
template <>
struct FragOf<bf16_t> {
  typedef bf16x8 type;
};
template <>
struct FragOf<float> {
  typedef f32x8 type;
};
template <typename T>
using frag_t = typename FragOf<T>::type;

// LDS row strides in elements.  row_ld: rows 4 banks apart (of 64), the 16 rows that a fragment read touches at a time fall on all banks.  col_ld: rows 16
// banks apart, so the 4 rows x 64 bytes that two groups of 16 lanes of a transposing read touch do (bf16); the two lane halves' rows 32 banks apart (fp32).
// tile_ld: for tiles that are read both ways, twofold conflicts in either.
template <typename T, int DH>
constexpr int tile_ld() {
  return sizeof(T) == 2 ? DH + 16 : DH + 8;
}
template <typename T, int DH>
constexpr int row_ld() {
  return sizeof(T) == 2 ? DH + 8 : DH + 4;
}
template <typename T, int DH>
constexpr int col_ld() {
  return sizeof(T) == 4 ? DH + 8 : DH % 128 == 96 ? DH : DH / 128 * 128 + (DH % 128 ? 96 : 32);
}

__device__ __forceinline__ bf16x8 row_frag(const unsigned short* p) { return *(const bf16x8*)p; }
__device__ __forceinline__ f32x8 row_frag(const float* p) { return f32x8{*(const f32x4*)p, *(const f32x4*)(p + 4)}; }

// rows k0 .. k0 + 3 and k1 .. k1 + 3 of column nb + lane % 32 of a tile stored [row][column]
__device__ __forceinline__ bf16x8 col_frag(const unsigned short* tile, int ld, int k0, int k1, int nb, int lane) {
  const int s = lane & 15, col = nb + ((lane >> 4) & 1) * 16 + (s & 3) * 4;
  union {
    s16x4 half[2];
    bf16x8 v;
  } u;
  u.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, tile + (k0 + (s >> 2)) * ld + col));
  u.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, tile + (k1 + (s >> 2)) * ld + col));
  return u.v;
}
__device__ __forceinline__ f32x8 col_frag(const float* tile, int ld, int k0, int k1, int nb, int lane) {
  const float* p = tile + nb + (lane & 31);
  f32x8 f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    f.lo[j] = p[(k0 + j) * ld];
    f.hi[j] = p[(k1 + j) * ld];
  }
  return f;
}

// The fragments d = 16 kk + 8 g (STEP 16) of a row in memory, zeros from dh on; zeros altogether for a row that is not there (the address must be
// that of some row).  All loads are under way before the first is looked at: a test around each would make it a trip to memory of its own.
template <typename T, int AL, int N, int STEP>
__device__ __forceinline__ void mem_frags(frag_t<T>* f, const typename Elem<T>::raw* row, int d0, int dh, bool valid) {
  union U {
    uint4 q[sizeof(T) / 2];
    frag_t<T> v;
  } u[N];
#pragma unroll
  for (int kk = 0; kk < N; ++kk)
#pragma unroll
    for (int j = 0; j < (int)sizeof(T) / 2; ++j) u[kk].q[j] = load_row_piece<T, AL>(row, kk * STEP + d0 + j * Elem<T>::PER, dh);
#pragma unroll
  for (int kk = 0; kk < N; ++kk) {
#pragma unroll
    for (int j = 0; j < (int)sizeof(T) / 2; ++j) {
      u[kk].q[j] = cut_piece<T, AL>(u[kk].q[j], kk * STEP + d0 + j * Elem<T>::PER, dh);
      if (!valid) u[kk].q[j] = make_uint4(0, 0, 0, 0);
    }
    f[kk] = u[kk].v;
  }
}

__device__ __forceinline__ void pack_frag(bf16x8& o, const float* v) {
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = (__bf16)v[i];
}
__device__ __forceinline__ void pack_frag(f32x8& o, const float* v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    o.lo[i] = v[i];
    o.hi[i] = v[4 + i];
  }
}

__device__ __forceinline__ f32x16 mma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mma32(f32x8 a, f32x8 b, f32x16 c) {
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.lo[i], b.lo[i], c, 0, 0, 0);
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.hi[i], b.hi[i], c, 0, 0, 0);
  return c;
}

__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}

// acc[d] holds X^T[32 d + 8 (i / 4) + 4 g + i % 4][this lane's row]: stores them to that row
template <typename T, int AL, int NDB>
__device__ __forceinline__ void store_row(typename Elem<T>::raw* dst, const f32x16* acc, float mul, int g, int dh) {
#pragma unroll
  for (int d = 0; d < NDB; ++d)
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) {
      const int dd = d * 32 + 8 * i4 + 4 * g;
      const float x0 = acc[d][4 * i4] * mul, x1 = acc[d][4 * i4 + 1] * mul, x2 = acc[d][4 * i4 + 2] * mul, x3 = acc[d][4 * i4 + 3] * mul;
      if constexpr (sizeof(T) == 2 && AL >= 8) {
        if (dd < dh) *(uint2*)(dst + dd) = make_uint2(pack_bf16x2(x0, x1), pack_bf16x2(x2, x3));
      } else if constexpr (sizeof(T) == 4 && AL == 16) {
        if (dd < dh) *(float4*)(dst + dd) = make_float4(x0, x1, x2, x3);
      } else {
        const float x[4] = {x0, x1, x2, x3};
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (dd + j < dh) st((T*)dst, dd + j, x[j]);
      }
    }
}

// Norms and rotation of queries (0) and keys (1): qk_norm.hip
struct QkNormArgs {
  const void* x[2];
  const void* w[2];        // [dh] or NULL: ones
  const int* positions;    // [tokens] or NULL: the token's index
  int gaps;                // negative positions mark tokens that take no part: y and dx stay as they are, dw has nothing of them
  void* y[2];
  const void* dy[2];
  void* dx[2];
  float* dw[2];
  float* part;             // [work-groups][dh]
  long tokens, x_row[2], x_head[2], y_row[2], y_head[2];   // gradients lie as their tensors do
  int H[2], dh, rope_dim, hchunk;
  int norm;                // 0: rotation alone
  float eps;
  double rate[7];          // theta^(-2 2^k / rope_dim)
};
struct QkNormGrid {
  int x, y, yq, hchunk;   // y: head ranges of the queries (yq) and of the keys
};
QkNormGrid qk_norm_grid(long tokens, int H0, int H1, int dh, int bf16);
void launch_qk_norm_rope(QkNormArgs a, int bf16, int align, bool backward, hipStream_t s);
// for the layer (one side, dense rows): rates and alignment are filled in
void launch_layer_norm_rope(QkNormArgs a, int bf16, bool backward, hipStream_t s);
size_t packed_norm_bytes(long tokens, int heads, int dh, int bf16);
// pos[r] = r for the prefix' rows, prefix + the row's place in its sequence for the others, -1 for rows of no sequence
void launch_packed_positions(const int* offsets, int nseq, int max_len, int T, int prefix, int* pos, hipStream_t s);
// zeros in the rows that belong to no sequence of up to three tensors (NULL: none)
void launch_packed_clear(const int* offsets, int nseq, int max_len, int rows, int row_bytes, void* p0, void* p1, void* p2, hipStream_t s);

// launchers
void launch_packed_fwd(const PackedAttn& a, int bf16, int align, hipStream_t s);
void launch_packed_few(const PackedAttn& a, int bf16, int align, hipStream_t s);
void launch_packed_prefix(const PackedAttn& f, const PackedAttn& o, bool few, int bf16, int align, hipStream_t s);
void launch_packed_join(const PackedAttn& a, int bf16, hipStream_t s);
void launch_packed_bwd(const PackedAttnBwd& a, int bf16, int align, float* delta, hipStream_t s);

enum { PACKED_BM = 128, PACKED_BM2 = 256, PACKED_FEW = 16, PACKED_KB = 128, PACKED_QT = 64, PACKED_EXACT = 32 };
// head width that a work-group's tiles are laid out for
static inline int packed_width(int dh) { return dh <= 32 ? 32 : dh <= 64 ? 64 : dh <= 96 ? 96 : dh <= 128 ? 128 : 256; }
// lanes that share a row of the backward pass' <dO, O>: 16 bytes each
static inline int packed_delta_lanes(int dh, int esz) {
  int l = 8;
  while (l * 16 < dh * esz) l *= 2;
  return l;
}
// slots of `rows` rows in tiles of bm over nseq sequences
static inline long packed_slots(long rows, int bm, int nseq) { return rows / bm + nseq; }

}  // namespace sh
