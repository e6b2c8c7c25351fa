// Backward attention over packed sequences with grouped heads.  With P = exp(s Q K^T - lse) and delta = <dO, O> per row:
//   dS = P (dO V^T - delta),  dQ = s dS K,  dK = s dS^T Q,  dV = P^T dO,
// dK and dV summed over the rows of every head of the group inside one accumulator: no atomics, so results repeat bit for bit.
#include "packed_attn.h"

namespace sh {

// delta[head][token]: a wave takes one (token, head) per 16, 32 or 64 lanes
template <typename T, int LR>
__global__ __launch_bounds__(256) void packed_delta_kernel(PackedAttn a, const void* dO_, float* delta) {
  typedef typename Elem<T>::raw raw;
  const int sub = threadIdx.x / LR, c = threadIdx.x % LR * 4;
  const long id = (long)blockIdx.x * (256 / LR) + sub;
  if (id >= (long)a.total_q * a.H) return;
  const int tok = (int)(id / a.H), head = (int)(id % a.H);
  const T* O = (const T*)((const raw*)a.O + (long)tok * a.o_row + (long)head * a.o_head);
  const T* dO = (const T*)((const raw*)dO_ + (long)tok * a.o_row + (long)head * a.o_head);
  float x = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (c + j < a.dh) x += ld(O, c + j) * ld(dO, c + j);
#pragma unroll
  for (int d = 1; d < LR; d <<= 1) x += __shfl_xor(x, d, 64);
  if (c == 0) delta[(long)head * a.total_q + tok] = x;
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
  int seq, nth;
  if (!find_slot(a.koff, a.total_k, a.nseq, 1, KB, slot, seq, nth)) return;
  const SeqGeom s = seq_geom(a, seq);
  const int k0 = nth * KB;
  if (k0 >= s.lk) return;
  const int off = s.lk - s.lq, rows = s.lq * a.G, key = k0 + wave * 32 + r;
  frag_t<T> kf[NKD], vf[DK ? NKD : 1];
  {
    const raw* K = (const raw*)a.K + (long)(s.kbeg + min(key, s.lk - 1)) * a.k_row + (long)hk * a.k_head;
    const raw* V = (const raw*)a.V + (long)(s.kbeg + min(key, s.lk - 1)) * a.v_row + (long)hk * a.v_head;
#pragma unroll
    for (int kk = 0; kk < NKD; ++kk) {
      kf[kk] = mem_frag<T, AL>(K, kk * 16 + 8 * g, dh, key < s.lk);
      if constexpr (DK) vf[kk] = mem_frag<T, AL>(V, kk * 16 + 8 * g, dh, key < s.lk);
    }
  }
  f32x16 accK[DK ? NDB : 1], accV[DV ? NDB : 1];
#pragma unroll
  for (int d = 0; d < NDB; ++d) {
    if constexpr (DK) accK[d] = zero16();
    if constexpr (DV) accV[d] = zero16();
  }
  const float sc = a.scale * 1.44269504088896340736f;
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
    const bool masked = r0 + QT > rows || k0 + wave * 32 + 32 > s.lk || (a.causal && k0 + wave * 32 + 31 > div_by(r0, a.g_inv) + off);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int rr = 8 * (i >> 2) + 4 * g + (i & 3);
      float arg = fmaf(S[i], sc, -lse_s[rr]);
      if (masked) {
        const bool vis = r0 + rr < rows && key < s.lk && (!a.causal || key <= div_by(r0 + rr, a.g_inv) + off);
        arg = vis ? arg : -INFINITY;
      }
      p[i] = __builtin_amdgcn_exp2f(arg);
      if constexpr (DK) {
        ds[i] = p[i] * (dP[i] - del_s[rr]);
        if (masked && arg == -INFINITY) ds[i] = 0.f;   // (what a hidden row or key holds stays out)
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
  int seq, nth;
  if (!find_slot(a.qoff, a.total_q, a.nseq, a.G, BM, slot, seq, nth)) return;
  const SeqGeom s = seq_geom(a, seq);
  const int rows = s.lq * a.G, nt = (rows + BM - 1) / BM;
  if (nth >= nt) return;
  const int row0 = (nt - 1 - nth) * BM;
  const int off = s.lk - s.lq, row = row0 + wave * 32 + r;
  const int tok = div_by(min(row, rows - 1), a.g_inv), head = hk * a.G + min(row, rows - 1) - tok * a.G;
  const int qpos = tok + off;
  const int wq_first = div_by(min(row0 + wave * 32, rows - 1), a.g_inv) + off;
  const int wq_last = div_by(min(row0 + wave * 32 + 31, rows - 1), a.g_inv) + off;
  const int last_tok = div_by(min(row0 + BM, rows) - 1, a.g_inv);
  const int kend = max(0, a.causal ? min(s.lk, last_tok + off + 1) : s.lk);

  frag_t<T> qf[NKD], gf[NKD];
  const raw* Q = (const raw*)a.Q + (long)(s.qbeg + tok) * a.q_row + (long)head * a.q_head;
  const raw* G = (const raw*)b.dO + (long)(s.qbeg + tok) * a.o_row + (long)head * a.o_head;
#pragma unroll
  for (int kk = 0; kk < NKD; ++kk) {
    qf[kk] = mem_frag<T, AL>(Q, kk * 16 + 8 * g, dh, row < rows);
    gf[kk] = mem_frag<T, AL>(G, kk * 16 + 8 * g, dh, row < rows);
  }
  const float lse2 = a.lse[(long)head * a.total_q + s.qbeg + tok] * 1.44269504088896340736f;
  const float del = b.delta[(long)head * a.total_q + s.qbeg + tok];
  f32x16 acc[NDB];
#pragma unroll
  for (int d = 0; d < NDB; ++d) acc[d] = zero16();
  const float sc = a.scale * 1.44269504088896340736f;
  const raw* const K = (const raw*)a.K + (long)s.kbeg * a.k_row + (long)hk * a.k_head;
  const raw* const V = (const raw*)a.V + (long)s.kbeg * a.v_row + (long)hk * a.v_head;
  PieceTile<T, DH, AL, KT, 256> tk, tv;
  if (kend > 0) {
    tk.load(K, a.k_row, kend, dh, tid);
    tv.load(V, a.v_row, kend, dh, tid);
  }
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
  const dim3 gk((unsigned)(packed_slots(a.total_k, 128, a.nseq) * a.Hk));
  const dim3 gq((unsigned)(packed_slots((long)a.total_q * a.G, PACKED_BM, a.nseq) * a.Hk));
  if constexpr (sizeof(T) == 4 && DH > 128) {
    packed_dkv_kernel<T, DH, AL, 1><<<gk, 256, 0, s>>>(b);
    packed_dkv_kernel<T, DH, AL, 2><<<gk, 256, 0, s>>>(b);
  } else {
    packed_dkv_kernel<T, DH, AL, 0><<<gk, 256, 0, s>>>(b);
  }
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
template <typename T>
static void launch_bwd_t(const PackedAttnBwd& b, int align, float* delta, hipStream_t s) {
  const PackedAttn& a = b.f;
  const int lr = a.dh <= 64 ? 16 : a.dh <= 128 ? 32 : 64;
  const dim3 gd((unsigned)(((long)a.total_q * a.H + 256 / lr - 1) / (256 / lr)));
  if (a.total_q == 0) {   // (keys without a query get zeros below)
  } else if (lr == 16)
    packed_delta_kernel<T, 16><<<gd, 256, 0, s>>>(a, b.dO, delta);
  else if (lr == 32)
    packed_delta_kernel<T, 32><<<gd, 256, 0, s>>>(a, b.dO, delta);
  else
    packed_delta_kernel<T, 64><<<gd, 256, 0, s>>>(a, b.dO, delta);
  if (a.dh <= 64)
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
