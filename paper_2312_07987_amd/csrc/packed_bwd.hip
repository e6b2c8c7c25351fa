// Backward attention over packed sequences with grouped heads.  With P = exp(s Q K^T - lse) and delta = <dO, O> per row:
//   dS = P (dO V^T - delta),  dQ = s dS K,  dK = s dS^T Q,  dV = P^T dO,
// dK and dV summed over the rows of every head of the group inside one accumulator: no atomics, so results repeat bit for bit.
#include "packed_attn.h"

namespace sh {

typedef unsigned short raw16;

// A work-group's 128 rows: those that see most keys first
__device__ __forceinline__ bool row_tile(const PackedAttn& a, int id, int& row0, SeqGeom& s) {
  if (a.levels) {
    s = seq_geom(a, level_seq(id, a.nseq));
    row0 = (a.levels - 1 - id / a.nseq) * PACKED_BM;
    return row0 < s.lq * a.G;
  }
  int nth;
  if (!find_slot<false>(a, PACKED_BM, id, nth, s)) return false;
  row0 = ((s.lq * a.G + PACKED_BM - 1) / PACKED_BM - 1 - nth) * PACKED_BM;
  return true;
}

// delta[head][token] = <dO, O>, from the rows as they are stored: LR lanes hold a row in 16-byte pieces.  (Rows of no sequence are summed too; nothing reads those sums.)
//
// O's rounding to bf16 is an error of P delta in dS = P (dP - delta) that a form with O in 32 bits has not.  It counts where a row sees few keys: the more keys a row averages
// over, the smaller its O, and the smaller its P beside dP.  So for bf16 rows that see up to PACKED_EXACT (32) keys the kernels below take delta = sum P dP instead, which
// needs no O: all those keys are one block of their products.  Relative 2-norm error of dQ and dK with the results' and dS's roundings alone / with delta exact up to
// 32, 16 and no keys (float64 arithmetic, roundings put in one at a time): 96 sequences of 20 to 256 tokens, heads of 76, 2.35e-3 / 2.37, 2.40, 2.62; 1500 tokens, heads of
// 128, 2.36e-3 / 2.38, 2.39, 2.57.  It costs 1.4 to 2.8 us of a step over 96 such short sequences (44 and 52 us), 1 per cent of one over long ones; in the
// kernels below the block with such rows is a branch of its own, element after element, so that the others keep their registers.  (In a launch of its own, or tile by tile with <dO, O>:
// 4 to 5 us.)  Exact for all rows would be the forward pass' operations once more.
template <typename T, int LR, int AL>
__global__ __launch_bounds__(256) void packed_delta_kernel(PackedAttn a, const void* dO_, float* delta) {
  typedef typename Elem<T>::raw raw;
  const int d = threadIdx.x % LR * Elem<T>::PER;
  const long id = (long)blockIdx.x * (256 / LR) + threadIdx.x / LR;
  if (id >= (long)a.total_q * a.H) return;
  const int tok = (int)(id / a.H), head = (int)(id - (long)tok * a.H);
  const long at = (long)tok * a.o_row + (long)head * a.o_head;
  const uint4 o = cut_piece<T, AL>(load_row_piece<T, AL>((const raw*)a.O + at, d, a.dh), d, a.dh);
  const uint4 g = cut_piece<T, AL>(load_row_piece<T, AL>((const raw*)dO_ + at, d, a.dh), d, a.dh);
  const unsigned ow[4] = {o.x, o.y, o.z, o.w}, gw[4] = {g.x, g.y, g.z, g.w};
  float x = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (sizeof(T) == 2) {
      x = fmaf(__uint_as_float(ow[j] << 16), __uint_as_float(gw[j] << 16), x);
      x = fmaf(__uint_as_float(ow[j] & 0xffff0000u), __uint_as_float(gw[j] & 0xffff0000u), x);
    } else {
      x = fmaf(__uint_as_float(ow[j]), __uint_as_float(gw[j]), x);
    }
  }
#pragma unroll
  for (int k = 1; k < LR; k <<= 1) x += __shfl_xor(x, k, 64);
  if (d == 0) delta[(long)head * a.total_q + tok] = x;
}

// The first rows of a sequence, which see up to PACKED_EXACT keys: how many they are
__device__ __forceinline__ int exact_rows(const PackedAttn& a, const SeqGeom& s) {
  if (a.causal) return min(max(PACKED_EXACT - (s.lk - s.lq), 0), s.lq) * a.G;
  return s.lk <= PACKED_EXACT ? s.lq * a.G : 0;
}
// the sum of a lane half's 32 values, in all of its lanes
__device__ __forceinline__ float half_sum(float x) {
  x += __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), 0xB1, 0xF, 0xF, true));    // lane ^ 1
  x += __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), 0x4E, 0xF, 0xF, true));    // ^ 2
  x += __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), 0x141, 0xF, 0xF, true));   // the other four of eight
  x += __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), 0x140, 0xF, 0xF, true));   // the other eight of sixteen
  const auto v = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(v[0]) + __uint_as_float(v[1]);
}

// dK and dV of 128 keys of one (sequence, kv head): 4 waves x 32 keys, whose K and V rows are registers; tiles of 32 rows of Q and dO go
// through LDS.  PASS 0: both; 1: dV alone, 2: dK alone (fp32 heads wider than 128: both accumulators do not fit the registers).
template <typename T, int DH, int AL, int PASS>
__global__ __launch_bounds__(256, 1) void packed_dkv_kernel(PackedAttnBwd b) {
  const PackedAttn& a = b.f;
  typedef typename Elem<T>::raw raw;
  constexpr int QT = 32, KB = 128, LD = tile_ld<T, DH>(), NKD = DH / 16, NDB = DH / 32, PER = Elem<T>::PER, CPR = DH / PER;
  constexpr int TOTAL = QT * CPR, NCH = (TOTAL + 255) / 256;
  constexpr bool DV = PASS != 2, DK = PASS != 1;
  __shared__ __attribute__((aligned(16))) raw Qs[QT * LD], Gs[QT * LD];
  __shared__ float lse_s[QT], del_s[QT];

  const int hk = blockIdx.x % a.Hk, slot = blockIdx.x / a.Hk;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 31, g = lane >> 5, dh = a.dh;
  int nth;
  SeqGeom s;
  if (!find_slot<true>(a, KB, slot, nth, s)) return;
  const int k0 = nth * KB;
  const int off = s.lk - s.lq, rows = s.lq * a.G, key = k0 + wave * 32 + r;
  frag_t<T> kf[NKD], vf[DK ? NKD : 1];
  {
    const raw* K = (const raw*)a.K + (long)(s.kbeg + min(key, s.lk - 1)) * a.k_row + (long)hk * a.k_head;
    const raw* V = (const raw*)a.V + (long)(s.kbeg + min(key, s.lk - 1)) * a.v_row + (long)hk * a.v_head;
    mem_frags<T, AL, NKD, 16>(kf, K, 8 * g, dh, key < s.lk);
    if constexpr (DK) mem_frags<T, AL, NKD, 16>(vf, V, 8 * g, dh, key < s.lk);
  }
  f32x16 accK[DK ? NDB : 1], accV[DV ? NDB : 1];
#pragma unroll
  for (int d = 0; d < NDB; ++d) {
    if constexpr (DK) accK[d] = zero16();
    if constexpr (DV) accV[d] = zero16();
  }
  const float sc = a.scale * 1.44269504088896340736f;
  const int exact = exact_rows(a, s);
  // the first row that sees one of the keys
  const int rbeg = a.causal ? max(k0 - off, 0) * a.G / QT * QT : 0;

  uint4 tq[NCH], tg[NCH];
  float nlse = 0.f, ndel = 0.f;
  auto prefetch = [&](int r0) {   // (rows past the end repeat the last one)
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = tid + i * 256, row = min(r0 + c / CPR, rows - 1), d = c % CPR * PER;
      const int tok = div_by(row, a.g_inv), head = hk * a.G + row - tok * a.G;
      tq[i] = load_row_piece<T, AL>((const raw*)a.Q + (long)(s.qbeg + tok) * a.q_row + (long)head * a.q_head, d, dh);
      tg[i] = load_row_piece<T, AL>((const raw*)b.dO + (long)(s.qbeg + tok) * a.o_row + (long)head * a.o_head, d, dh);
    }
    const int row = min(r0 + (tid & (QT - 1)), rows - 1), tok = div_by(row, a.g_inv), head = hk * a.G + row - tok * a.G;
    nlse = a.lse[(long)head * a.total_q + s.qbeg + tok];
    ndel = b.delta[(long)head * a.total_q + s.qbeg + tok];
  };
  if (rbeg < rows) prefetch(rbeg);
  __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): what was loaded before the loop is not waited for again inside it
  for (int r0 = rbeg; r0 < rows; r0 += QT) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = tid + i * 256, row = c / CPR, d = c % CPR * PER;
      if (TOTAL % 256 != 0 && c >= TOTAL) continue;
      uint4 q = tq[i], x = tg[i];
      if (dh != DH) {
        q = cut_piece<T, AL>(q, d, dh);
        x = cut_piece<T, AL>(x, d, dh);
      }
      if (r0 + row >= rows) q = x = make_uint4(0, 0, 0, 0);
      *(uint4*)(Qs + row * LD + d) = q;
      *(uint4*)(Gs + row * LD + d) = x;
    }
    if (tid < QT) {
      lse_s[tid] = nlse * 1.44269504088896340736f;
      del_s[tid] = ndel;
    }
    __syncthreads();
    if (r0 + QT < rows) prefetch(r0 + QT);

    f32x16 S = zero16(), dP = zero16();
#pragma unroll
    for (int kk = 0; kk < NKD; ++kk) {
      S = mma32(row_frag(&Qs[r * LD + kk * 16 + 8 * g]), kf[kk], S);
      if constexpr (DK) dP = mma32(row_frag(&Gs[r * LD + kk * 16 + 8 * g]), vf[kk], dP);
    }
    float p[16], ds[16];
    const bool few = r0 < exact && k0 + wave == 0;   // uniform: the block has all keys of some of its rows
    const bool masked = r0 + QT > rows || k0 + wave * 32 + 32 > s.lk || (a.causal && k0 + wave * 32 + 31 > div_by(r0, a.g_inv) + off);
    auto visible = [&](int rr) { return r0 + rr < rows && key < s.lk && (!a.causal || key <= div_by(r0 + rr, a.g_inv) + off); };
    if (sizeof(T) == 2 && DK && few) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int rr = 8 * (i >> 2) + 4 * g + (i & 3);
        p[i] = visible(rr) ? __builtin_amdgcn_exp2f(fmaf(S[i], sc, -lse_s[rr])) : 0.f;
        const float t = half_sum(visible(rr) ? p[i] * dP[i] : 0.f);
        ds[i] = visible(rr) ? p[i] * (dP[i] - (r0 + rr < exact ? t : del_s[rr])) : 0.f;
        asm volatile("" : "+v"(ds[i]));
        __builtin_amdgcn_sched_barrier(0);   // (one after the other: the registers are full)
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int rr = 8 * (i >> 2) + 4 * g + (i & 3);
        float arg = fmaf(S[i], sc, -lse_s[rr]);
        if (masked) arg = visible(rr) ? arg : -INFINITY;
        p[i] = __builtin_amdgcn_exp2f(arg);
        if constexpr (DK) {
          ds[i] = p[i] * (dP[i] - del_s[rr]);
          if (masked && arg == -INFINITY) ds[i] = 0.f;   // (what a hidden row or key holds stays out)
        }
      }
    }
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      frag_t<T> pb, db;
      if constexpr (DV) pack_frag(pb, &p[8 * st]);
      if constexpr (DK) pack_frag(db, &ds[8 * st]);
      const int kb0 = 16 * st + 4 * g;
#pragma unroll
      for (int d = 0; d < NDB; ++d) {
        if constexpr (DV) accV[d] = mma32(col_frag(Gs, LD, kb0, kb0 + 8, d * 32, lane), pb, accV[d]);
        if constexpr (DK) accK[d] = mma32(col_frag(Qs, LD, kb0, kb0 + 8, d * 32, lane), db, accK[d]);
      }
    }
  }
  if (key < s.lk) {
    if constexpr (DK) store_row<T, AL, NDB>((raw*)b.dK + (long)(s.kbeg + key) * a.k_row + (long)hk * a.k_head, accK, a.scale, g, dh);
    if constexpr (DV) store_row<T, AL, NDB>((raw*)b.dV + (long)(s.kbeg + key) * a.v_row + (long)hk * a.v_head, accV, 1.f, g, dh);
  }
}

// A work-group's key tile: its number in the sequence, and the slot that its parts go to.  By level: the first tiles, which most rows see, first.
__device__ __forceinline__ bool key_tile(const PackedAttnBwd& b, int id, int& nth, int& slot, SeqGeom& s) {
  const PackedAttn& a = b.f;
  if (!b.klevels) {
    slot = id;
    return find_slot<true>(a, PACKED_KB, id, nth, s);
  }
  const int seq = level_seq(id, a.nseq);
  s = seq_geom(a, seq);
  nth = (s.lk + PACKED_KB - 1) / PACKED_KB - b.klevels + id / a.nseq;
  slot = first_slot(a.koff, a.total_k, 1, PACKED_KB, seq) + nth;
  return nth >= 0;
}

// The same for bf16 heads of up to 128 elements with two kinds of waves.  A single wave per SIMD, which is all that the kernel above has registers
// for, leaves the matrix cores idle during exponentials, conversions and LDS traffic.  Here waves 0 .. 3 (score) hold K and V fragments,
// form P and dS of a tile of 64 rows and leave both as bf16 operand fragments in LDS (and dS^T in memory for dQ); waves
// 4 .. 7 (gradient) hold the dK and dV accumulators, add the previous tile's products, and move the row tiles from memory to LDS.  One of each
// kind per SIMD; three stages for the row tiles (written a trip ahead, read by the score waves in the next trip and by the gradient waves
// in the one after), two hand-over buffers, one barrier per 64 rows.  A score wave has four chains of products in flight (S and dP of two blocks of 32 x 32):
// with one block per trip the chain barrier, fragment reads, products, exponentials, barrier was what a trip waited for.  Up to 96 elements the two
// blocks are of two key blocks, so that a fragment of the rows serves both (6600 tokens, 20 heads of 80 over 4, a backward pass 492 -> 472 us); of 128 the K and V fragments
// of two do not fit the registers (163 -> 190), and they are of two row blocks.
// A gradient wave owns dK or dV of 64 keys, so that a fragment of the rows serves two products there.
// (Q and dO straight from memory in operand order for the score waves: 32 rows of 32 bytes an instruction are more than the vector memory path
// carries, dK / dV of 16384 tokens 180 -> 329 us.)
// Heads of 97 .. 128: rows of 256 bytes whose 16-byte pieces are permuted by the row (swizzle), so that both the 16 rows of a fragment read and the
// 4 rows x 64 bytes of a transposing read fall on all banks, and three stages and two buffers fill the 160 KB.  Narrower ones are padded.
// Under a causal mask the first keys of a sequence are seen by all of its rows, the last by few, so rows are cut into ranges of rchunk
// and a (key tile, range) is a work-group; ranges that are the only one of their tile write dK and dV, others fp32 parts.
// Measured: 16 x 2048 tokens, 8 heads of 128, 485 us, 566 TFLOP/s; without the exponentials 453, without storing dS^T 413, without moving the row tiles 431,
// without all three 316: a trip is the sum of what its two kinds of waves cannot hide from each other, half of it matrix instructions.
template <int DH, int AL>
__global__ __launch_bounds__(512, 1) void packed_dkv_ws_kernel(PackedAttnBwd b) {
  const PackedAttn& a = b.f;
  constexpr int QT = PACKED_QT, KB = PACKED_KB, LD = DH == 128 ? 128 : DH + 16, NST = 3, NKD = DH / 16, NDB = DH / 32, CPR = DH / 8, TOTAL = QT * CPR, NCH = (TOTAL + 255) / 256;
  constexpr int SK = DH <= 96 ? 2 : 1, SR = QT / 32 / SK;   // key blocks and row blocks of a score wave
  constexpr int STAGE = 2 * QT * LD;
  constexpr bool KEEP = DH > 64;   // (narrower heads keep no score gradients: plan_backward)
  __shared__ __attribute__((aligned(16))) unsigned short tiles[NST * STAGE];
  __shared__ __attribute__((aligned(16))) uint4 hand[2][4][8][64];   // [buffer][key block][P, dS of 16 rows in turn][lane]
  static_assert(sizeof tiles + sizeof hand <= 160 * 1024, "fits a CU");

  int bid = blockIdx.x;
  const int hk = bid % a.Hk;
  bid /= a.Hk;
  const int nslot = gridDim.x / (a.Hk * b.rparts), part = b.rparts - 1 - bid / nslot, slot_ = bid % nslot;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 31, g = lane >> 5, dh = a.dh;
  int nth, slot;
  SeqGeom s;
  if (!key_tile(b, slot_, nth, slot, s)) return;
  const int k0 = nth * KB;
  const int off = s.lk - s.lq, rows = s.lq * a.G;
  const int first = a.causal ? max(k0 - off, 0) * a.G / QT * QT : 0;   // the first row tile that sees one of the keys
  // this range of the rows, and whether it is the only one
  const int p0 = min(first, max(rows - 1, 0)) / b.rchunk, p1 = max(rows - 1, 0) / b.rchunk;
  if (part < p0 || part > p1) return;
  const int rbeg = max(first, part * b.rchunk), rend = min(rows, (part + 1) * b.rchunk);
  const int n = rbeg < rend ? (rend - rbeg + QT - 1) / QT : 0;
  auto place = [&](int row, int& tok, int& head) {
    tok = div_by(row, a.g_inv);
    head = hk * a.G + row - tok * a.G;
    tok += s.qbeg;
  };

  // where piece p of a tile's row lies
  auto piece = [](int row, int p) { return DH == 128 ? p ^ ((row & 3) << 2 | (row >> 2 & 1) << 1 | (row >> 3 & 1)) : p; };

  if (wave < 4) {
    const int kb0 = SK == 2 ? (wave & 1) * 2 : wave, b0 = SK == 2 ? wave >> 1 : 0;   // the wave's key blocks, and its blocks of 32 of a tile's rows
    bf16x8 kf[SK][NKD], vf[SK][NKD];
    // (keys past the sequence have no row of dS^T: they repeat the last key's address and do not store)
    raw16* dsrow[SK];
#pragma unroll
    for (int k = 0; k < SK; ++k) {
      const int key = k0 + (kb0 + k) * 32 + r, kc = s.kbeg + min(key, s.lk - 1);
      mem_frags<bf16_t, AL, NKD, 16>(kf[k], (const raw16*)a.K + (long)kc * a.k_row + (long)hk * a.k_head, 8 * g, dh, key < s.lk);
      mem_frags<bf16_t, AL, NKD, 16>(vf[k], (const raw16*)a.V + (long)kc * a.v_row + (long)hk * a.v_head, 8 * g, dh, key < s.lk);
      dsrow[k] = (raw16*)b.dS + (b.dS ? ((long)hk * a.total_k + kc) * b.ds_ld + 8 * g : 0);
    }
    const float sc = a.scale * 1.44269504088896340736f;
    const int exact = exact_rows(a, s);
    // the statistics of the next tile's rows (lane half 0: lse, 1: delta; rows past the end repeat the last one)
    float st[SR];
    auto statistics = [&](int r0) {
#pragma unroll
      for (int blk = 0; blk < SR; ++blk) {
        int tok, head;
        place(min(r0 + (b0 + blk) * 32 + r, rows - 1), tok, head);
        st[blk] = (g ? b.delta : a.lse)[(long)head * a.total_q + tok];
      }
    };
    if (n > 0) statistics(rbeg);
    for (int it = 0; it <= n; ++it) {
      __syncthreads();
      if (it == n) break;
      const raw16* Qr = tiles + it % NST * STAGE;
      const raw16* Gr = Qr + QT * LD;
      // the statistics go through the start of the wave's own hand-over place, which is not written before they are read
      float* const sl = (float*)hand[it & 1][kb0][b0 * 4];
#pragma unroll
      for (int blk = 0; blk < SR; ++blk) sl[(blk * 2 + g) * 32 + r] = g ? st[blk] : st[blk] * 1.44269504088896340736f;
      if (it + 1 < n) statistics(rbeg + (it + 1) * QT);
      f32x16 S_[SR][SK], dP_[SR][SK];
#pragma unroll
      for (int blk = 0; blk < SR; ++blk)
#pragma unroll
        for (int k = 0; k < SK; ++k) S_[blk][k] = dP_[blk][k] = zero16();
#pragma unroll
      for (int kk = 0; kk < NKD; ++kk)
#pragma unroll
        for (int blk = 0; blk < SR; ++blk) {
          const int at = ((b0 + blk) * 32 + r) * LD + piece(r, 2 * kk + g) * 8;
          const bf16x8 q = row_frag(Qr + at), x = row_frag(Gr + at);
#pragma unroll
          for (int k = 0; k < SK; ++k) {
            S_[blk][k] = mma32(q, kf[k][kk], S_[blk][k]);
            dP_[blk][k] = mma32(x, vf[k][kk], dP_[blk][k]);
          }
        }
      wave_order();
      f32x4 L_[SR][4], D_[SR][4];
#pragma unroll
      for (int blk = 0; blk < SR; ++blk)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
          L_[blk][i4] = *(const f32x4*)&sl[blk * 64 + 8 * i4 + 4 * g];
          D_[blk][i4] = *(const f32x4*)&sl[blk * 64 + 32 + 8 * i4 + 4 * g];
        }
      wave_order();
#pragma unroll
      for (int blk = 0; blk < SR; ++blk) {
        const int r0 = rbeg + it * QT + (b0 + blk) * 32;
        if (r0 >= rend) break;   // uniform
#pragma unroll
        for (int k = 0; k < SK; ++k) {
          const int wk = k0 + (kb0 + k) * 32, key = wk + r;
          const f32x16 S = S_[blk][k], dP = dP_[blk][k];
          float p[16], ds[16];
          if (wk == 0 && r0 < exact) {   // uniform: the block has all keys of some of its rows
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int rr = r0 + 8 * (i >> 2) + 4 * g + (i & 3);
              const bool vis = rr < rend && key < s.lk && (!a.causal || key <= div_by(rr, a.g_inv) + off);
              p[i] = __builtin_amdgcn_exp2f(fmaf(S[i], sc, -L_[blk][i / 4][i % 4]));
              const float t = half_sum(vis ? p[i] * dP[i] : 0.f);
              ds[i] = p[i] * (dP[i] - (rr < exact ? t : D_[blk][i / 4][i % 4]));
              asm volatile("" : "+v"(ds[i]));
              __builtin_amdgcn_sched_barrier(0);   // (one after the other: the registers are full)
            }
          } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              p[i] = __builtin_amdgcn_exp2f(fmaf(S[i], sc, -L_[blk][i / 4][i % 4]));
              ds[i] = p[i] * (dP[i] - D_[blk][i / 4][i % 4]);
            }
          }
          // wave-uniform: most blocks lie wholly inside the visible region
          if (r0 + 32 > rend || wk + 32 > s.lk || (a.causal && wk + 31 > div_by(r0, a.g_inv) + off)) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int rr = r0 + 8 * (i >> 2) + 4 * g + (i & 3);
              const bool vis = rr < rend && key < s.lk && (!a.causal || key <= div_by(rr, a.g_inv) + off);
              p[i] = vis ? p[i] : 0.f;
              ds[i] = vis ? ds[i] : 0.f;
            }
          }
          // P and dS are rounded to bf16 here, once, for their products
          uint4* hd = hand[it & 1][kb0 + k][(b0 + blk) * 4] + lane;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            union {
              bf16x8 v;
              uint4 q;
            } up, ud;
            pack_frag(up.v, &p[8 * h]);
            pack_frag(ud.v, &ds[8 * h]);
            hd[2 * h * 64] = up.q;
            hd[(2 * h + 1) * 64] = ud.q;
            // elements 0..3 / 4..7: rows r0 + 16 h + 4 g + {0..3} / + 8 + {0..3} of this lane's key; the lane halves trade, so that each has 8 rows side by side
            const auto lo = __builtin_amdgcn_permlane32_swap(ud.q.x, ud.q.z, false, false), hi = __builtin_amdgcn_permlane32_swap(ud.q.y, ud.q.w, false, false);
            if (KEEP && b.dS && key < s.lk) *(uint4*)(dsrow[k] + r0 + 16 * h) = make_uint4(lo[0], hi[0], lo[1], hi[1]);
          }
        }
      }
    }
    return;
  }

  const int gt = tid - 256, gw = wave - 4;
  const int kb0 = (gw >> 1) * 2, of_k = gw & 1;   // the wave's two key blocks; dK or dV
  uint4 tq[NCH], tg[NCH];
  auto prefetch = [&](int r0) {   // (rows past the end repeat the last one)
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = gt + i * 256, d = c % CPR * 8;
      int tok, head;
      place(min(r0 + c / CPR, rows - 1), tok, head);
      tq[i] = load_row_piece<bf16_t, AL>((const raw16*)a.Q + (long)tok * a.q_row + (long)head * a.q_head, d, dh);
      tg[i] = load_row_piece<bf16_t, AL>((const raw16*)b.dO + (long)tok * a.o_row + (long)head * a.o_head, d, dh);
    }
  };
  auto stage = [&](raw16* t, int r0) {
    const bool whole = r0 + QT <= rows && dh == DH;   // uniform
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = gt + i * 256, row = c / CPR, d = c % CPR * 8;
      if (TOTAL % 256 != 0 && c >= TOTAL) continue;
      uint4 q = tq[i], x = tg[i];
      if (!whole) {
        q = cut_piece<bf16_t, AL>(q, d, dh);
        x = cut_piece<bf16_t, AL>(x, d, dh);
        if (r0 + row >= rows) q = x = make_uint4(0, 0, 0, 0);
      }
      *(uint4*)(t + row * LD + piece(row, d / 8) * 8) = q;
      *(uint4*)(t + (QT + row) * LD + piece(row, d / 8) * 8) = x;
    }
  };
  // rows k .. k + 3 and k + 8 .. k + 11 (k = 16 h + 4 g) of column 32 d + lane % 32
  auto columns = [&](const raw16* tile, int h, int d) {
    const int q = lane & 15, row = 16 * h + 4 * g + (q >> 2), p = 4 * d + (lane >> 4 & 1) * 2 + (q >> 1 & 1), in = (q & 1) * 4;
    union {
      s16x4 half[2];
      bf16x8 v;
    } u;
    u.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, tile + row * LD + piece(row, p) * 8 + in));
    u.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, tile + (row + 8) * LD + piece(row + 8, p) * 8 + in));
    return u.v;
  };
  f32x16 acc[2][NDB];
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int d = 0; d < NDB; ++d) acc[k][d] = zero16();
  if (n > 0) {
    prefetch(rbeg);
    stage(tiles, rbeg);
    if (n > 1) prefetch(rbeg + QT);
  }
  for (int it = 0; it <= n; ++it) {
    __syncthreads();
    // the tile it + 1 (requested a trip ago) goes into its stage and the tile it + 2 starts to travel
    if (it + 1 < n) {
      stage(tiles + (it + 1) % NST * STAGE, rbeg + (it + 1) * QT);
      if (it + 2 < n) prefetch(rbeg + (it + 2) * QT);
    }
    if (it == 0) continue;
    const raw16* tile = tiles + (it - 1) % NST * STAGE + (of_k ? 0 : QT * LD);   // dK: Q, dV: dO
    const int left = rend - (rbeg + (it - 1) * QT);   // rows of the tile that exist
#pragma unroll
    for (int h = 0; h < QT / 16; ++h) {
      if ((h & ~1) * 16 >= left) break;   // uniform: blocks of 32 rows that the score waves left out
      union {
        uint4 q;
        bf16x8 v;
      } w[2];   // dK: dS, dV: P
#pragma unroll
      for (int k = 0; k < 2; ++k) w[k].q = hand[(it - 1) & 1][kb0 + k][2 * h + of_k][lane];
#pragma unroll
      for (int d = 0; d < NDB; ++d) {
        const bf16x8 f = columns(tile, h, d);
#pragma unroll
        for (int k = 0; k < 2; ++k) acc[k][d] = mma32(f, w[k].v, acc[k][d]);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int key = k0 + (kb0 + k) * 32 + r;
    if (p0 == p1) {
      if (key < s.lk) {
        raw16* const out = of_k ? (raw16*)b.dK + (long)(s.kbeg + key) * a.k_row + (long)hk * a.k_head : (raw16*)b.dV + (long)(s.kbeg + key) * a.v_row + (long)hk * a.v_head;
        store_row<bf16_t, AL, NDB>(out, acc[k], of_k ? a.scale : 1.f, g, dh);
      }
      continue;
    }
    // a part: accumulators in register order, 16 bytes per lane, by key block and d block, dV first
    f32x4* out = (f32x4*)(b.dkv + ((long)part * b.kslots + (long)slot * a.Hk + hk) * b.dkv_floats) + (of_k * 4 + kb0 + k) * NDB * 4 * 64 + lane;
#pragma unroll
    for (int d = 0; d < NDB; ++d)
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) out[(d * 4 + i4) * 64] = f32x4{acc[k][d][4 * i4], acc[k][d][4 * i4 + 1], acc[k][d][4 * i4 + 2], acc[k][d][4 * i4 + 3]};
  }
}

// Adds the parts of the key tiles that have several, in range order: waves 0 .. 3 dV, 4 .. 7 dK, 32 keys each
template <int DH, int AL>
__global__ __launch_bounds__(512) void packed_dkv_join_kernel(PackedAttnBwd b) {
  const PackedAttn& a = b.f;
  constexpr int NDB = DH / 32;
  const int hk = blockIdx.x % a.Hk, slot = blockIdx.x / a.Hk;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, blk = wave & 3, r = lane & 31, g = lane >> 5, dh = a.dh;
  int nth;
  SeqGeom s;
  if (!find_slot<true>(a, PACKED_KB, slot, nth, s)) return;
  const int k0 = nth * PACKED_KB;
  const int off = s.lk - s.lq, rows = s.lq * a.G, first = a.causal ? max(k0 - off, 0) * a.G / PACKED_QT * PACKED_QT : 0;
  const int p0 = min(first, max(rows - 1, 0)) / b.rchunk, p1 = max(rows - 1, 0) / b.rchunk;
  if (p0 == p1) return;
  f32x16 acc[NDB];
#pragma unroll
  for (int d = 0; d < NDB; ++d) acc[d] = zero16();
  for (int p = p0; p <= p1; ++p) {
    const f32x4* in = (const f32x4*)(b.dkv + ((long)p * b.kslots + (long)slot * a.Hk + hk) * b.dkv_floats) + ((wave >= 4 ? 4 : 0) + blk) * NDB * 4 * 64 + lane;
#pragma unroll
    for (int d = 0; d < NDB; ++d)
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        const f32x4 v = in[(d * 4 + i4) * 64];
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[d][4 * i4 + j] += v[j];
      }
  }
  const int key = k0 + blk * 32 + r;
  if (key >= s.lk) return;
  if (wave < 4)
    store_row<bf16_t, AL, NDB>((unsigned short*)b.dV + (long)(s.kbeg + key) * a.v_row + (long)hk * a.v_head, acc, 1.f, g, dh);
  else
    store_row<bf16_t, AL, NDB>((unsigned short*)b.dK + (long)(s.kbeg + key) * a.k_row + (long)hk * a.k_head, acc, a.scale, g, dh);
}

// dQ from the kept score gradients: dQ^T[d][row] = s sum_key K^T[d][key] dS^T[key][row], a plain product.  128 rows of one (sequence, kv head),
// tiles of 128 keys of K and of dS^T through LDS, both read by columns (of 64 keys 124 us, of 128 109: 6600 tokens, 20 heads of 80 over 4); a wave owns 64 rows and half of d (96: 32 rows and all of d).
// What the dK / dV work-groups of a key tile did not write (rows that see none of its keys) is replaced by zeros.  Bound by its chain of trips (a register stage, two
// barriers, products: some 2.4 us a trip of 128 keys, so that the longest rows' work-groups end last), not by memory: 16 x 2048 tokens, 8 heads of 128, 537 MB of dS^T
// in 190 us are 2.8 TB/s, the case of one sequence of 4096 among shorter ones 2.1, a large copy 5.06.
template <int DH, int AL>
__global__ __launch_bounds__(256, 2) void packed_dq_ds_kernel(PackedAttnBwd b) {
  const PackedAttn& a = b.f;
  constexpr int KT = 128, LD = DH + 16, BM = PACKED_BM, LDD = BM + 16, NDB = DH / 32, NP = KT * BM / 8 / 256;
  constexpr bool SPLIT = NDB % 2 == 0;
  constexpr int NJ = SPLIT ? 2 : 1, ND = SPLIT ? NDB / 2 : NDB;
  __shared__ __attribute__((aligned(16))) unsigned short Ks[KT * LD], Ds[KT * LDD];
  const int hk = blockIdx.x % a.Hk, slot = blockIdx.x / a.Hk;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 31, g = lane >> 5, dh = a.dh;
  SeqGeom s;
  int row0;
  if (!row_tile(a, slot, row0, s)) return;
  const int rows = s.lq * a.G;
  const int off = s.lk - s.lq;
  const int wr = row0 + (SPLIT ? (wave & 1) * 64 : wave * 32), d0 = SPLIT ? (wave >> 1) * ND : 0;
  const int last_tok = div_by(min(row0 + BM, rows) - 1, a.g_inv), wq_last = div_by(min(wr + 32 * NJ, rows) - 1, a.g_inv) + off;
  const int kend = max(0, a.causal ? min(s.lk, last_tok + off + 1) : s.lk);
  const raw16* const K = (const raw16*)a.K + (long)s.kbeg * a.k_row + (long)hk * a.k_head;
  const raw16* const D = (const raw16*)b.dS + ((long)hk * a.total_k + s.kbeg) * b.ds_ld + row0;
  f32x16 acc[NJ][ND];
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int d = 0; d < ND; ++d) acc[j][d] = zero16();
  PieceTile<bf16_t, DH, AL, KT, 256> tk;
  // dS^T tile: 16 pieces of 8 rows per key
  uint4 td[NP];
  const int dk = tid / 16, dr = tid % 16 * 8;
  auto load_d = [&](int k0) {
#pragma unroll
    for (int i = 0; i < NP; ++i) td[i] = *(const uint4*)(D + (long)min(k0 + dk + 16 * i, kend - 1) * b.ds_ld + dr);
  };
  tk.place(a.k_row, tid);
  if (kend > 0) {
    tk.load(K, a.k_row, kend, dh, tid);
    load_d(0);
  }
  for (int k0 = 0; k0 < kend; k0 += KT) {
    // the first row written for this tile's keys, and the keys that exist
    const int written = a.causal ? max(k0 / PACKED_KB * PACKED_KB - off, 0) * a.G / PACKED_QT * PACKED_QT : 0;
    const bool keep = row0 + dr >= written && row0 + dr < (rows + 31) / 32 * 32;
    __syncthreads();
    tk.store(Ks, LD, kend - k0, dh, tid);
#pragma unroll
    for (int i = 0; i < NP; ++i) *(uint4*)(Ds + (dk + 16 * i) * LDD + dr) = keep && k0 + dk + 16 * i < kend ? td[i] : make_uint4(0, 0, 0, 0);
    __syncthreads();
    if (k0 + KT < kend) {
      tk.load(K + (long)(k0 + KT) * a.k_row, a.k_row, kend - k0 - KT, dh, tid);
      load_d(k0 + KT);
    }
    if (wr >= rows || (a.causal && k0 > wq_last)) continue;   // wave-uniform
#pragma unroll
    for (int kb = 0; kb < KT / 32; ++kb)
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        const int kr = kb * 32 + 16 * st + 4 * g;
        bf16x8 bq[NJ];
#pragma unroll
        for (int j = 0; j < NJ; ++j) bq[j] = col_frag(Ds, LDD, kr, kr + 8, wr - row0 + j * 32, lane);
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          const bf16x8 ka = col_frag(Ks, LD, kr, kr + 8, (d0 + d) * 32, lane);
#pragma unroll
          for (int j = 0; j < NJ; ++j) acc[j][d] = mma32(ka, bq[j], acc[j][d]);
        }
      }
  }
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int row = wr + j * 32 + r;
    if (row >= rows) continue;
    const int tok = div_by(row, a.g_inv), head = hk * a.G + row - tok * a.G;
    store_row<bf16_t, AL, ND>((raw16*)b.dQ + (long)(s.qbeg + tok) * a.q_row + (long)head * a.q_head + d0 * 32, acc[j], a.scale, g, dh - d0 * 32);
  }
}

// dQ of 128 rows of one (sequence, kv head): 4 waves x 32 rows, whose Q and dO are registers; K and V tiles go through LDS.
//   S^T[key][row] = K Q^T,  dP^T = V dO^T,  dQ^T[d][row] += K^T dS^T
template <typename T, int DH, int AL>
__global__ __launch_bounds__(256, DH* sizeof(T) > 256 ? 1 : 2) void packed_dq_kernel(PackedAttnBwd b) {
  const PackedAttn& a = b.f;
  typedef typename Elem<T>::raw raw;
  constexpr int KT = DH * sizeof(T) > 256 ? 32 : 64, LD = tile_ld<T, DH>(), NKD = DH / 16, NDB = DH / 32, BM = PACKED_BM;
  __shared__ __attribute__((aligned(16))) raw kv[2 * KT * LD];
  raw *const Ks = kv, *const Vs = kv + KT * LD;
  const int hk = blockIdx.x % a.Hk, slot = blockIdx.x / a.Hk;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 31, g = lane >> 5, dh = a.dh;
  SeqGeom s;
  int row0;
  if (!row_tile(a, slot, row0, s)) return;
  const int rows = s.lq * a.G;
  const int off = s.lk - s.lq, row = row0 + wave * 32 + r;
  const int tok = div_by(min(row, rows - 1), a.g_inv), head = hk * a.G + min(row, rows - 1) - tok * a.G;
  const int qpos = tok + off;
  const int wq_first = div_by(min(row0 + wave * 32, rows - 1), a.g_inv) + off;
  const int wq_last = div_by(min(row0 + wave * 32 + 31, rows - 1), a.g_inv) + off;
  const int last_tok = div_by(min(row0 + BM, rows) - 1, a.g_inv);
  const int kend = max(0, a.causal ? min(s.lk, last_tok + off + 1) : s.lk), exact = exact_rows(a, s);

  frag_t<T> qf[NKD], gf[NKD];
  const raw* Q = (const raw*)a.Q + (long)(s.qbeg + tok) * a.q_row + (long)head * a.q_head;
  const raw* G = (const raw*)b.dO + (long)(s.qbeg + tok) * a.o_row + (long)head * a.o_head;
  const float lse2 = a.lse[(long)head * a.total_q + s.qbeg + tok] * 1.44269504088896340736f;
  float del = b.delta[(long)head * a.total_q + s.qbeg + tok];
  f32x16 acc[NDB];
#pragma unroll
  for (int d = 0; d < NDB; ++d) acc[d] = zero16();
  const float sc = a.scale * 1.44269504088896340736f;
  const raw* const K = (const raw*)a.K + (long)s.kbeg * a.k_row + (long)hk * a.k_head;
  const raw* const V = (const raw*)a.V + (long)s.kbeg * a.v_row + (long)hk * a.v_head;
  PieceTile<T, DH, AL, KT, 256> tk, tv;
  tk.place(a.k_row, tid);
  tv.place(a.v_row, tid);
  if (kend > 0) {
    tk.load(K, a.k_row, kend, dh, tid);
    tv.load(V, a.v_row, kend, dh, tid);
  }
  mem_frags<T, AL, NKD, 16>(qf, Q, 8 * g, dh, row < rows);
  mem_frags<T, AL, NKD, 16>(gf, G, 8 * g, dh, row < rows);
  __builtin_amdgcn_s_waitcnt(0x0F70);
  for (int k0 = 0; k0 < kend; k0 += KT) {
    __syncthreads();
    tk.store(Ks, LD, kend - k0, dh, tid);
    tv.store(Vs, LD, kend - k0, dh, tid);
    __syncthreads();
    if (k0 + KT < kend) {
      tk.load(K + (long)(k0 + KT) * a.k_row, a.k_row, kend - k0 - KT, dh, tid);
      tv.load(V + (long)(k0 + KT) * a.v_row, a.v_row, kend - k0 - KT, dh, tid);
    }
    if (row0 + wave * 32 >= rows || (a.causal && k0 > wq_last)) continue;
    const bool masked = kend - k0 < KT || (a.causal && k0 + KT - 1 > wq_first);
#pragma unroll
    for (int kb = 0; kb < KT / 32; ++kb) {
      f32x16 S = zero16(), dP = zero16();
#pragma unroll
      for (int kk = 0; kk < NKD; ++kk) {
        S = mma32(row_frag(&Ks[(kb * 32 + r) * LD + kk * 16 + 8 * g]), qf[kk], S);
        dP = mma32(row_frag(&Vs[(kb * 32 + r) * LD + kk * 16 + 8 * g]), gf[kk], dP);
      }
      float ds[16];
      const int lim = (a.causal ? min(kend - 1, qpos) : kend - 1) - (k0 + kb * 32 + 4 * g);
      if (sizeof(T) == 2 && k0 + kb == 0 && row0 + wave * 32 < exact) {   // uniform; a row is a lane of either half
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          if (8 * (i >> 2) + (i & 3) <= lim) t = fmaf(__builtin_amdgcn_exp2f(fmaf(S[i], sc, -lse2)), dP[i], t);
          __builtin_amdgcn_sched_barrier(0);
        }
        t += __shfl_xor(t, 32, 64);
        del = row < exact ? t : del;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        ds[i] = __builtin_amdgcn_exp2f(fmaf(S[i], sc, -lse2)) * (dP[i] - del);
        if (masked && 8 * (i >> 2) + (i & 3) > lim) ds[i] = 0.f;
      }
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        frag_t<T> db;
        pack_frag(db, &ds[8 * st]);
        const int kb0 = kb * 32 + 16 * st + 4 * g;
#pragma unroll
        for (int d = 0; d < NDB; ++d) acc[d] = mma32(col_frag(Ks, LD, kb0, kb0 + 8, d * 32, lane), db, acc[d]);
      }
    }
  }
  if (row < rows) store_row<T, AL, NDB>((raw*)b.dQ + (long)(s.qbeg + tok) * a.q_row + (long)head * a.q_head, acc, a.scale, g, dh);
}

template <typename T, int DH, int AL>
static void launch_bwd_al(const PackedAttnBwd& b, hipStream_t s) {
  const PackedAttn& a = b.f;
  const long kslots = packed_slots(a.total_k, PACKED_KB, a.nseq) * a.Hk, qslots = packed_slots((long)a.total_q * a.G, PACKED_BM, a.nseq) * a.Hk;
  const dim3 gk((unsigned)kslots), gq((unsigned)(a.levels ? (long)a.levels * a.nseq * a.Hk : qslots));
  prof_mark(s, "attention.dkv");
  if constexpr (sizeof(T) == 4 && DH > 128) {
    packed_dkv_kernel<T, DH, AL, 1><<<gk, 256, 0, s>>>(b);
    packed_dkv_kernel<T, DH, AL, 2><<<gk, 256, 0, s>>>(b);
  } else if constexpr (sizeof(T) == 2 && DH <= 128) {
    packed_dkv_ws_kernel<DH, AL><<<dim3((unsigned)((b.klevels ? (long)b.klevels * a.nseq * a.Hk : kslots) * b.rparts)), 512, 0, s>>>(b);
    if (b.rparts > 1) packed_dkv_join_kernel<DH, AL><<<gk, 512, 0, s>>>(b);
    if constexpr (DH > 64) {
      if (b.dS && a.total_q > 0) {
        prof_mark(s, "attention.dq");
        packed_dq_ds_kernel<DH, AL><<<gq, 256, 0, s>>>(b);
        return;
      }
    }
  } else {
    packed_dkv_kernel<T, DH, AL, 0><<<gk, 256, 0, s>>>(b);
  }
  prof_mark(s, "attention.dq");
  packed_dq_kernel<T, DH, AL><<<gq, 256, 0, s>>>(b);
}
template <typename T, int DH>
static void launch_bwd(const PackedAttnBwd& b, int align, hipStream_t s) {
  if (align == 16) return launch_bwd_al<T, DH, 16>(b, s);
  if constexpr (sizeof(T) == 2) {
    if (align == 8) return launch_bwd_al<T, DH, 8>(b, s);
  }
  launch_bwd_al<T, DH, sizeof(T)>(b, s);
}
template <typename T, int LR>
static void launch_delta(const PackedAttnBwd& b, int align, float* delta, hipStream_t s) {
  const PackedAttn& a = b.f;
  const dim3 grid((unsigned)(((long)a.total_q * a.H + 256 / LR - 1) / (256 / LR)));
  if (align == 16) {
    packed_delta_kernel<T, LR, 16><<<grid, 256, 0, s>>>(a, b.dO, delta);
    return;
  }
  if constexpr (sizeof(T) == 2) {
    if (align == 8) {
      packed_delta_kernel<T, LR, 8><<<grid, 256, 0, s>>>(a, b.dO, delta);
      return;
    }
  }
  packed_delta_kernel<T, LR, sizeof(T)><<<grid, 256, 0, s>>>(a, b.dO, delta);
}
template <typename T>
static void launch_bwd_t(const PackedAttnBwd& b, int align, float* delta, hipStream_t s) {
  const PackedAttn& a = b.f;
  prof_mark(s, "attention.delta");
  if (a.total_q > 0) {   // (keys without a query get zeros below)
    const int lanes = packed_delta_lanes(a.dh, sizeof(T));
    if (lanes == 8)
      launch_delta<T, 8>(b, align, delta, s);
    else if (lanes == 16)
      launch_delta<T, 16>(b, align, delta, s);
    else if (lanes == 32)
      launch_delta<T, 32>(b, align, delta, s);
    else if constexpr (sizeof(T) == 4)
      launch_delta<T, 64>(b, align, delta, s);
  }
  if (a.dh <= 32)
    launch_bwd<T, 32>(b, align, s);
  else if (a.dh <= 64)
    launch_bwd<T, 64>(b, align, s);
  else if (a.dh <= 96)
    launch_bwd<T, 96>(b, align, s);
  else if (a.dh <= 128)
    launch_bwd<T, 128>(b, align, s);
  else
    launch_bwd<T, 256>(b, align, s);
}
void launch_packed_bwd(const PackedAttnBwd& b, int bf16, int align, float* delta, hipStream_t s) {
  if (bf16)
    launch_bwd_t<bf16_t>(b, align, delta, s);
  else
    launch_bwd_t<float>(b, align, delta, s);
}

}  // namespace sh
