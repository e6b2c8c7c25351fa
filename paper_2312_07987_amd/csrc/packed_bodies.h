// The bodies of the forward kernels over packed sequences, which stand alone (packed_fwd.hip, packed_few.hip) and side by side in one launch
// (packed_prefix.hip).
#pragma once
#include "packed_attn.h"

namespace sh {

// LDS of the bodies, in elements
template <typename T, int DH, int NG>
constexpr int packed_fwd_lds() {
  return NG * NG * (DH * (int)sizeof(T) > 256 ? 32 : 64) * (row_ld<T, DH>() + col_ld<T, DH>());
}
template <typename T, int DH>
constexpr int packed_few_lds() {
  return 4 * 32 * tile_ld<T, DH>();
}

// One work-group: 128 rows of one (sequence, kv head), four waves of 32, key tiles of KT.  NG = 2: two such groups of waves take
// alternate tiles of the same rows and merge their (o, m, l) through LDS at the end.  That halves the chain of a long row of tiles, which is what a
// batch of few long and many short sequences waits for, and the group has the CU to itself, so its two buffers per group (one barrier per trip)
// fit.  3 sequences of 4096 tokens, 4 heads of 128: 117 us with one group, 84 with two.
// Bound by the chain of a tile of keys, products, softmax, products, where few waves share a SIMD (64 x 512 tokens, 8 heads of 128, 80 us: 430 TFLOP/s), by the
// longest tile of rows where lengths differ.
template <typename T, int DH, int AL, int NG>
__device__ __forceinline__ void packed_fwd_body(const PackedAttn& a, int b, typename Elem<T>::raw* kv_) {
  typedef typename Elem<T>::raw raw;
  constexpr int KT = DH * sizeof(T) > 256 ? 32 : 64, LDK = row_ld<T, DH>(), LDV = col_ld<T, DH>(), NKD = DH / 16, NDB = DH / 32, BM = PACKED_BM;
  constexpr int NBUF = NG, TILE = KT * (LDK + LDV);
  const int hk = b % a.Hk;
  b /= a.Hk;
  const int ns = max(a.nsplit, 1), split = b % ns, slot = b / ns;
  const int grp = NG > 1 ? threadIdx.x >> 8 : 0;
  const int tid = threadIdx.x & 255, lane = tid & 63, wave = tid >> 6, r = lane & 31, g = lane >> 5, dh = a.dh;
  raw* const kv = kv_ + grp * NBUF * TILE;

  SeqGeom s;
  int row0;
  if (a.flat) {
    s.qbeg = 0;
    s.lq = a.total_q;
    s.kbeg = s.lk = 0;
    row0 = slot * BM;
  } else if (a.levels) {
    s = seq_geom(a, level_seq(slot, a.nseq));
    row0 = (a.levels - 1 - slot / a.nseq) * BM;
  } else {
    int nth;
    if (!find_slot<false>(a, BM, slot, nth, s)) return;
    // the last tiles, which see most keys, first
    row0 = ((s.lq * a.G + BM - 1) / BM - 1 - nth) * BM;
  }
  const int rows = s.lq * a.G;
  if (row0 >= rows) return;
  const int off = s.lk - s.lq;   // query i sees own keys <= off + i
  const int row = row0 + wave * 32 + r;
  const int tok = div_by(min(row, rows - 1), a.g_inv), head = hk * a.G + min(row, rows - 1) - tok * a.G;
  const int qpos = tok + off;
  const int wq_first = div_by(min(row0 + wave * 32, rows - 1), a.g_inv) + off;
  const int wq_last = div_by(min(row0 + wave * 32 + 31, rows - 1), a.g_inv) + off;
  const int last_tok = div_by(min(row0 + BM, rows) - 1, a.g_inv);
  const int prefix = a.own ? 0 : a.prefix;
  const int kend = a.flat ? 0 : max(0, a.causal ? min(s.lk, last_tok + off + 1) : s.lk);   // own keys that some row sees

  f32x16 o[NDB];
#pragma unroll
  for (int d = 0; d < NDB; ++d) o[d] = zero16();
  float m = -INFINITY, l = 0.f;
  const float sc = a.scale * 1.44269504088896340736f;   // logits in log2 units

  // tiles of the prefix, then of the own keys; this work-group's even share of them
  const int np = (prefix + KT - 1) / KT, nt = np + (kend + KT - 1) / KT;
  // (prefix below 2^30 rows, own keys below 2^31: less than 3 * 2^25 tiles, times up to 32 parts below 2^32)
  const int t0 = (int)((unsigned)nt * (unsigned)split / (unsigned)ns), t1 = (int)((unsigned)nt * (unsigned)(split + 1) / (unsigned)ns);
  PieceTile<T, DH, AL, KT, 256> tk, tv;
  const raw* const KP = (const raw*)a.KP + (long)hk * a.kp_head;
  const raw* const VP = (const raw*)a.VP + (long)hk * a.vp_head;
  const raw* const K = (const raw*)a.K + (long)s.kbeg * a.k_row + (long)hk * a.k_head;
  const raw* const V = (const raw*)a.V + (long)s.kbeg * a.v_row + (long)hk * a.v_head;
  auto valid_of = [&](int t) { return t < np ? prefix - t * KT : kend - (t - np) * KT; };
  // (the prefix may have other strides: the pieces are placed again at the border)
  tk.place(t0 + grp < np ? a.kp_row : a.k_row, tid);
  tv.place(t0 + grp < np ? a.vp_row : a.v_row, tid);
  auto load = [&](int t) {
    if (t >= np && t < np + NG) {
      tk.place(a.k_row, tid);
      tv.place(a.v_row, tid);
    }
    if (t < np) {
      tk.load(KP + (long)t * KT * a.kp_row, a.kp_row, valid_of(t), dh, tid);
      tv.load(VP + (long)t * KT * a.vp_row, a.vp_row, valid_of(t), dh, tid);
    } else {
      tk.load(K + (long)(t - np) * KT * a.k_row, a.k_row, valid_of(t), dh, tid);
      tv.load(V + (long)(t - np) * KT * a.v_row, a.v_row, valid_of(t), dh, tid);
    }
  };
  auto store = [&](int t, raw* buf) {
    tk.store(buf, LDK, valid_of(t), dh, tid);
    tv.store(buf + KT * LDK, LDV, valid_of(t), dh, tid);
  };
  if (t0 + grp < t1) load(t0 + grp);
  frag_t<T> qf[NKD];   // (behind the tile's loads: what is done with them waits for them)
  mem_frags<T, AL, NKD, 16>(qf, (const raw*)a.Q + (long)(s.qbeg + tok) * a.q_row + (long)head * a.q_head, 8 * g, dh, row < rows);
  __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): what was loaded before the loop is not waited for again inside it
  if constexpr (NG == 2) {
    if (t0 + grp < t1) store(t0 + grp, kv);
    if (t0 + grp + 2 < t1) load(t0 + grp + 2);
    __syncthreads();
  }
  // NG = 2, one barrier per trip: while a tile is multiplied out of one buffer the next one (requested a trip ago) is written into the other and
  // the one after that starts to travel.  NG = 1: the tile in the registers is written between two barriers.  All waves make the same trips.
  int cur = 0;
  for (int tb = t0; tb < t1; tb += NG, cur ^= NBUF - 1) {
    const int t = tb + grp, valid = valid_of(t), k0 = (t - np) * KT;
    const raw *const Ks = kv + cur * TILE, *const Vs = Ks + KT * LDK;
    if constexpr (NG == 2) {
      if (t + 2 < t1) {
        store(t + 2, kv + (cur ^ 1) * TILE);
        if (t + 4 < t1) load(t + 4);
      }
    } else {
      __syncthreads();
      store(t, kv);
      __syncthreads();
      if (t + 1 < t1) load(t + 1);
    }
    const bool masked = a.causal && t >= np;
    // wave-uniform: a tile past the end, no rows, or nothing that they see
    if (t < t1 && row0 + wave * 32 < rows && !(masked && k0 > wq_last)) {
      f32x16 sv[KT / 32];
#pragma unroll
      for (int kb = 0; kb < KT / 32; ++kb) {
        sv[kb] = zero16();
#pragma unroll
        for (int kk = 0; kk < NKD; ++kk) sv[kb] = mma32(row_frag(&Ks[(kb * 32 + r) * LDK + kk * 16 + 8 * g]), qf[kk], sv[kb]);
      }
      if (valid < KT || (masked && k0 + KT - 1 > wq_first)) {
        const int lim = (masked ? min(valid - 1, qpos - k0) : valid - 1) - 4 * g;
#pragma unroll
        for (int kb = 0; kb < KT / 32; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (kb * 32 + 8 * (i >> 2) + (i & 3) > lim) sv[kb][i] = -INFINITY;
      }
      float mt = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < KT / 32; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) mt = fmaxf(mt, sv[kb][i]);
      mt = fmaxf(mt, __shfl_xor(mt, 32, 64)) * sc;   // sc > 0
      const float mn = fmaxf(m, mt);
      if (__ballot(mn > m)) {   // most tiles move no maximum
        const float alpha = mn > m ? __builtin_amdgcn_exp2f(m - mn) : 1.f;   // m = -inf: 0
        l *= alpha;
#pragma unroll
        for (int d = 0; d < NDB; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[d][i] *= alpha;
      }
      m = mn;
      const float mb = mn == -INFINITY ? 0.f : mn;   // (a row that has seen no key yet)
      float ps = 0.f;
#pragma unroll
      for (int kb = 0; kb < KT / 32; ++kb)
#pragma unroll
        for (int st = 0; st < 2; ++st) {
          float p8[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            p8[i] = __builtin_amdgcn_exp2f(fmaf(sv[kb][8 * st + i], sc, -mb));   // masked: 0
            ps += p8[i];
          }
          // P is rounded to the storage type for its product; the sum keeps 32 bits
          frag_t<T> pb;
          pack_frag(pb, p8);
          const int kr = kb * 32 + 16 * st + 4 * g;
#pragma unroll
          for (int d = 0; d < NDB; ++d) o[d] = mma32(col_frag(Vs, LDV, kr, kr + 8, d * 32, lane), pb, o[d]);
        }
      l += ps;
    }
    if constexpr (NG == 2) __syncthreads();
  }
  l += __shfl_xor(l, 32, 64);
  if constexpr (NG == 2) {
    // group 1 parks its partial results over the tiles; group 0 of the same wave and lane holds the same row and elements
    static_assert(4 * (NDB * 16 + 2) * 64 * 4 <= NG * NBUF * TILE * (int)sizeof(raw), "the parked accumulators fit over the tiles");
    float* park = (float*)kv_ + wave * (NDB * 16 + 2) * 64 + lane;
    if (grp == 1) {
#pragma unroll
      for (int d = 0; d < NDB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) park[(d * 16 + i) * 64] = o[d][i];
      park[NDB * 16 * 64] = m;
      park[(NDB * 16 + 1) * 64] = l;
    }
    __syncthreads();
    if (grp == 1) return;
    const float m1 = park[NDB * 16 * 64], l1 = park[(NDB * 16 + 1) * 64], mn = fmaxf(m, m1), mb = mn == -INFINITY ? 0.f : mn;
    const float f0 = __builtin_amdgcn_exp2f(m - mb), f1 = __builtin_amdgcn_exp2f(m1 - mb);   // a group that saw no key: 0
#pragma unroll
    for (int d = 0; d < NDB; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] = o[d][i] * f0 + park[(d * 16 + i) * 64] * f1;
    l = l * f0 + l1 * f1;
    m = mn;
  }
  if (row >= rows) return;
  const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);   // nothing seen: zeros; NaN stays
  const float lse = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994530942f;
  if (a.nsplit) {
    const long at = (long)(a.part0 + split) * a.total_q * a.H + (long)(s.qbeg + tok) * a.H + head;
    if (g == 0) a.pl[at] = lse;
    store_row<float, 16, NDB>(a.po + at * a.dhp, o, inv, g, dh);
  } else {
    if (g == 0 && a.lse) a.lse[(long)head * a.total_q + s.qbeg + tok] = lse;
    store_row<T, AL, NDB>((raw*)a.O + (long)(s.qbeg + tok) * a.o_row + (long)head * a.o_head, o, inv, g, dh);
  }
}

// ---------------------------------------------------------------------------------------------------------------------------
// Attention of a few rows per sequence and kv head over many keys: single tokens (or a few) over a cache, with the heads of a group as
// further rows, at most 16 in all.  A work-group takes one (sequence, kv head) and a chunk of its keys; chunks have one length
// for all sequences, so ragged lengths make more work-groups, not longer ones.
//
// 16 x 16 products, lane = 16 g + r:
//   S^T[key][row] = K Q^T       K straight from memory in operand order (16 rows of 64 or 128 contiguous bytes an instruction)
//   O^T[d][row] += V^T P^T      a lane's scores of a piece's two blocks of 16 keys (4 g .. 4 g + 3 of each) are its operand as they are; V goes
//                               through the wave's own LDS and is read by columns in that key order
// The waves take every fourth piece of 32 keys without barriers; a piece's registers are requested again as soon as they are free and
// travel during the softmax and the second product.  Bound by reading K and V once: 32 tokens over 2000 .. 32768 keys, 8 kv heads of 128, 220 us,
// 4.5 TB/s (a large copy 5.06); 16 over 500 .. 4000, 4 kv heads, 14 us, 4.4 TB/s.
// ---------------------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ f32x4 mma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma16(f32x8 a, f32x8 b, f32x4 c) {
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.lo[i], b.lo[i], c, 0, 0, 0);
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.hi[i], b.hi[i], c, 0, 0, 0);
  return c;
}
// rows 4 g .. 4 g + 3 and 16 + 4 g .. of column nb + lane % 16 of a tile stored [row][column]
__device__ __forceinline__ bf16x8 col_frag16(const unsigned short* tile, int ld, int nb, int r, int g) {
  const unsigned short* p = tile + (4 * g + (r >> 2)) * ld + nb + (r & 3) * 4;
  union {
    s16x4 half[2];
    bf16x8 v;
  } u;
  u.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, p));
  u.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, p + 16 * ld));
  return u.v;
}
__device__ __forceinline__ f32x8 col_frag16(const float* tile, int ld, int nb, int r, int g) {
  const float* p = tile + 4 * g * ld + nb + r;
  f32x8 f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    f.lo[j] = p[j * ld];
    f.hi[j] = p[(16 + j) * ld];
  }
  return f;
}

template <typename T, int DH, int AL>
__device__ __forceinline__ void packed_few_body(const PackedAttn& a, int block, typename Elem<T>::raw* fsm, float (*ms)[PACKED_FEW], float (*ls)[PACKED_FEW]) {
  typedef typename Elem<T>::raw raw;
  constexpr int W = 4, KP = 32, PER = Elem<T>::PER, FP = 8 / PER;   // waves; keys of a piece; pieces of a fragment
  constexpr int NK = DH / 32, ND = DH / 16, LDV = tile_ld<T, DH>(), CPR = DH / PER, NV = KP * CPR / 64, LDO = DH + 4;
  // fsm: a piece of V per wave, then its output in fp32
  static_assert(PACKED_FEW * LDO * 4 <= KP * LDV * (int)sizeof(raw), "a wave's output fits over its V piece");

  const int hk = block % a.Hk, slot = block / a.Hk;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 15, g = lane >> 4, dh = a.dh;
  int nth = 0;
  SeqGeom s;
  if (a.chunk) {
    if (!find_slot<true>(a, a.chunk, slot, nth, s)) return;
  } else {
    s = seq_geom(a, slot);
  }
  const int rows = s.lq * a.G;   // at most frows = max_q * G <= 16
  const int key0 = nth * a.chunk, kend = a.chunk ? min(s.lk, key0 + a.chunk) : s.lk;
  if (rows <= 0) return;   // (unsplit, a sequence without keys still gets its zeros)
  const int off = s.lk - s.lq;
  const int rc = min(r, rows - 1), tok = div_by(rc, a.g_inv), head = hk * a.G + rc - tok * a.G;
  const raw* const K = (const raw*)a.K + (long)s.kbeg * a.k_row + (long)hk * a.k_head;
  const raw* const V = (const raw*)a.V + (long)s.kbeg * a.v_row + (long)hk * a.v_head;
  raw* const vl = fsm + wave * KP * LDV;

  union KF {
    uint4 q[FP];
    frag_t<T> f;
  };
  KF kf[2][NK];
  uint4 vf[NV];
  auto load = [&](int k0) {   // (a key past the end repeats the last one, at probability zero)
#pragma unroll
    for (int blk = 0; blk < 2; ++blk) {
      const raw* row = K + (long)min(k0 + 16 * blk + r, kend - 1) * a.k_row;
#pragma unroll
      for (int kk = 0; kk < NK; ++kk)
#pragma unroll
        for (int j = 0; j < FP; ++j) kf[blk][kk].q[j] = load_row_piece<T, AL>(row, kk * 32 + 8 * g + j * PER, dh);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = lane + 64 * i;
      vf[i] = load_row_piece<T, AL>(V + (long)min(k0 + c / CPR, kend - 1) * a.v_row, c % CPR * PER, dh);
    }
  };
  if (key0 + wave * KP < kend) load(key0 + wave * KP);
  frag_t<T> qf[NK];
  mem_frags<T, AL, NK, 32>(qf, (const raw*)a.Q + (long)(s.qbeg + tok) * a.q_row + (long)head * a.q_head, 8 * g, dh, r < rows);
  f32x4 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = f32x4{};
  float m = -INFINITY, l = 0.f;
  const float sc = a.scale * 1.44269504088896340736f;
  const bool cut = dh != DH;
  for (int k0 = key0 + wave * KP; k0 < kend; k0 += W * KP) {
    f32x4 sv[2];
#pragma unroll
    for (int blk = 0; blk < 2; ++blk) {
      sv[blk] = f32x4{};
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) {
        if (cut) {
#pragma unroll
          for (int j = 0; j < FP; ++j) kf[blk][kk].q[j] = cut_piece<T, AL>(kf[blk][kk].q[j], kk * 32 + 8 * g + j * PER, dh);
        }
        sv[blk] = mma16(kf[blk][kk].f, qf[kk], sv[blk]);
      }
    }
    wave_order();
    const bool whole = k0 + KP <= kend;   // uniform
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = lane + 64 * i;
      uint4 v = vf[i];
      if (cut) v = cut_piece<T, AL>(v, c % CPR * PER, dh);
      if (!whole && k0 + c / CPR >= kend) v = make_uint4(0, 0, 0, 0);
      *(uint4*)(vl + (c / CPR) * LDV + c % CPR * PER) = v;
    }
    wave_order();
    if (k0 + W * KP < kend) load(k0 + W * KP);   // uniform
    if (!whole || (a.causal && k0 + KP - 1 > off)) {
      const int lim = (a.causal ? min(kend - 1, tok + off) : kend - 1) - k0 - 4 * g;
#pragma unroll
      for (int blk = 0; blk < 2; ++blk)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          if (16 * blk + v > lim) sv[blk][v] = -INFINITY;
    }
    float mt = fmaxf(fmaxf(fmaxf(sv[0][0], sv[0][1]), fmaxf(sv[0][2], sv[0][3])), fmaxf(fmaxf(sv[1][0], sv[1][1]), fmaxf(sv[1][2], sv[1][3])));
    mt = fmaxf(mt, __shfl_xor(mt, 16, 64));
    mt = fmaxf(mt, __shfl_xor(mt, 32, 64)) * sc;   // sc > 0
    const float mn = fmaxf(m, mt), mb = mn == -INFINITY ? 0.f : mn;   // (a piece that the row does not see)
    const float alpha = __builtin_amdgcn_exp2f(m - mb);               // m = -inf: 0
    m = mn;
    float p8[8], ps = 0.f;
#pragma unroll
    for (int blk = 0; blk < 2; ++blk)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        p8[4 * blk + v] = __builtin_amdgcn_exp2f(fmaf(sv[blk][v], sc, -mb));   // masked: 0
        ps += p8[4 * blk + v];
      }
    l = l * alpha + ps;
    frag_t<T> pb;
    pack_frag(pb, p8);
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      o[d] *= alpha;
      o[d] = mma16(col_frag16(vl, LDV, d * 16, r, g), pb, o[d]);
    }
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  wave_order();
  float* const po = (float*)vl;
#pragma unroll
  for (int d = 0; d < ND; ++d) *(f32x4*)(po + r * LDO + d * 16 + 4 * g) = o[d];
  if (g == 0) {
    ms[wave][r] = m;
    ls[wave][r] = l;
  }
  __syncthreads();
  // four output columns a thread; a wave that saw no key has m = -inf, l = 0 and counts for nothing
  const long base = ((long)slot * a.Hk + hk) * a.frows;
  for (int t = tid; t < rows * (DH / 4); t += 256) {
    const int q = t / (DH / 4), d = t % (DH / 4) * 4;
    float mx = ms[0][q];
#pragma unroll
    for (int w = 1; w < W; ++w) mx = fmaxf(mx, ms[w][q]);
    const float mb = mx == -INFINITY ? 0.f : mx;
    float lt = 0.f;
    f32x4 x = f32x4{};
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = __builtin_amdgcn_exp2f(ms[w][q] - mb);
      lt += f * ls[w][q];
      x += f * *(const f32x4*)((const float*)(fsm + w * KP * LDV) + q * LDO + d);
    }
    const float inv = lt == 0.f ? 0.f : 1.f / lt, lse = lt == 0.f ? -INFINITY : (mb + log2f(lt)) * 0.69314718055994530942f;
    if (a.fo) {
      if (d < a.dhp) *(f32x4*)(a.fo + (base + q) * a.dhp + d) = x * inv;
      if (d == 0) a.fl[base + q] = lse;
    } else {
      const int qt = div_by(q, a.g_inv), h = hk * a.G + q - qt * a.G;
      raw* O = (raw*)a.O + (long)(s.qbeg + qt) * a.o_row + (long)h * a.o_head;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (d + j < dh) st((T*)O, d + j, x[j] * inv);
      if (d == 0 && a.lse) a.lse[(long)h * a.total_q + s.qbeg + qt] = lse;
    }
  }
}

}  // namespace sh
