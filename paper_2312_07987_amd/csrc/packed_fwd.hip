// Forward attention over packed sequences with grouped heads: O = softmax(s Q K^T + mask) V of every sequence by itself, with rows that
// all sequences see in front of their own keys where there is a shared prefix.
//
// Transposed products, S^T[key][row] = K Q^T and O^T[d][row] += V^T P^T: a row (token, head) is a lane column, so the running maximum
// and sum of its softmax are lane-local up to one exchange between the lane halves, and exp(S^T) is the second product's operand as it
// stands.  K and V tiles go through LDS once for all rows of the work-group.
#include "packed_attn.h"

namespace sh {

// One work-group: 4 waves x 32 rows of one (sequence, kv head), key tiles of KT.
template <typename T, int DH, int AL>
__global__ __launch_bounds__(256, DH <= 128 ? 2 : 1) void packed_fwd_kernel(PackedAttn a) {
  typedef typename Elem<T>::raw raw;
  constexpr int KT = DH * sizeof(T) > 256 ? 32 : 64, LD = tile_ld<T, DH>(), NKD = DH / 16, NDB = DH / 32, BM = PACKED_BM;
  __shared__ __attribute__((aligned(16))) raw kv[2 * KT * LD];
  raw *const Ks = kv, *const Vs = kv + KT * LD;

  int b = blockIdx.x;
  const int hk = b % a.Hk;
  b /= a.Hk;
  const int ns = max(a.nsplit, 1), split = b % ns, slot = b / ns;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 31, g = lane >> 5, dh = a.dh;

  SeqGeom s;
  int row0;
  if (a.flat) {
    s.qbeg = 0;
    s.lq = a.total_q;
    s.kbeg = s.lk = 0;
    row0 = slot * BM;
  } else {
    int nth;
    if (!find_slot<false>(a, BM, slot, nth, s)) return;
    // the last tiles, which see most keys, first
    const int nt = (s.lq * a.G + BM - 1) / BM;
    if (nth >= nt) return;
    row0 = (nt - 1 - nth) * BM;
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

  frag_t<T> qf[NKD];
  const raw* Q = (const raw*)a.Q + (long)(s.qbeg + tok) * a.q_row + (long)head * a.q_head;
#pragma unroll
  for (int kk = 0; kk < NKD; ++kk) qf[kk] = mem_frag<T, AL>(Q, kk * 16 + 8 * g, dh, row < rows);

  f32x16 o[NDB];
#pragma unroll
  for (int d = 0; d < NDB; ++d) o[d] = zero16();
  float m = -INFINITY, l = 0.f;
  const float sc = a.scale * 1.44269504088896340736f;   // logits in log2 units

  // tiles of the prefix, then of the own keys; this work-group's even share of them
  const int np = (prefix + KT - 1) / KT, nt = np + (kend + KT - 1) / KT;
  const int t0 = (int)((long)nt * split / ns), t1 = (int)((long)nt * (split + 1) / ns);
  PieceTile<T, DH, AL, KT, 256> tk, tv;
  const raw* const KP = (const raw*)a.KP + (long)hk * a.kp_head;
  const raw* const VP = (const raw*)a.VP + (long)hk * a.vp_head;
  const raw* const K = (const raw*)a.K + (long)s.kbeg * a.k_row + (long)hk * a.k_head;
  const raw* const V = (const raw*)a.V + (long)s.kbeg * a.v_row + (long)hk * a.v_head;
  auto valid_of = [&](int t) { return t < np ? prefix - t * KT : kend - (t - np) * KT; };
  auto load = [&](int t) {
    if (t < np) {
      tk.load(KP + (long)t * KT * a.kp_row, a.kp_row, valid_of(t), dh, tid);
      tv.load(VP + (long)t * KT * a.vp_row, a.vp_row, valid_of(t), dh, tid);
    } else {
      tk.load(K + (long)(t - np) * KT * a.k_row, a.k_row, valid_of(t), dh, tid);
      tv.load(V + (long)(t - np) * KT * a.v_row, a.v_row, valid_of(t), dh, tid);
    }
  };
  if (t0 < t1) load(t0);
  __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): what was loaded before the loop is not waited for again inside it
  for (int t = t0; t < t1; ++t) {
    const int valid = valid_of(t), k0 = (t - np) * KT;
    __syncthreads();
    tk.store(Ks, LD, valid, dh, tid);
    tv.store(Vs, LD, valid, dh, tid);
    __syncthreads();
    if (t + 1 < t1) load(t + 1);
    const bool masked = a.causal && t >= np;
    if (row0 + wave * 32 >= rows || (masked && k0 > wq_last)) continue;   // wave-uniform: no rows, or nothing that they see

    float sv[KT / 32][16];
#pragma unroll
    for (int kb = 0; kb < KT / 32; ++kb) {
      f32x16 acc = zero16();
#pragma unroll
      for (int kk = 0; kk < NKD; ++kk) acc = mma32(row_frag(&Ks[(kb * 32 + r) * LD + kk * 16 + 8 * g]), qf[kk], acc);
#pragma unroll
      for (int i = 0; i < 16; ++i) sv[kb][i] = acc[i];
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
    const bool moved = mn > m;
    const float alpha = moved ? __builtin_amdgcn_exp2f(m - mn) : 1.f;   // m = -inf: 0
    m = mn;
    const float mb = mn == -INFINITY ? 0.f : mn;   // (a row that has seen no key yet)
    float ps = 0.f;
#pragma unroll
    for (int kb = 0; kb < KT / 32; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        sv[kb][i] = __builtin_amdgcn_exp2f(fmaf(sv[kb][i], sc, -mb));   // masked: 0
        ps += sv[kb][i];
      }
    l = l * alpha + ps;
    if (__ballot(moved)) {
#pragma unroll
      for (int d = 0; d < NDB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= alpha;
    }
#pragma unroll
    for (int kb = 0; kb < KT / 32; ++kb)
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        frag_t<T> pb;
        pack_frag(pb, &sv[kb][8 * st]);
        const int kr = kb * 32 + 16 * st + 4 * g;
#pragma unroll
        for (int d = 0; d < NDB; ++d) o[d] = mma32(col_frag(Vs, LD, kr, kr + 8, d * 32, lane), pb, o[d]);
      }
  }
  l += __shfl_xor(l, 32, 64);
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

template <typename T, int DH>
static void launch_fwd(const PackedAttn& a, int align, dim3 grid, hipStream_t s) {
  if (align == 16) {
    packed_fwd_kernel<T, DH, 16><<<grid, 256, 0, s>>>(a);
    return;
  }
  if constexpr (sizeof(T) == 2) {
    if (align == 8) {
      packed_fwd_kernel<T, DH, 8><<<grid, 256, 0, s>>>(a);
      return;
    }
  }
  packed_fwd_kernel<T, DH, sizeof(T)><<<grid, 256, 0, s>>>(a);
}
template <typename T>
static void launch_fwd_t(const PackedAttn& a, int align, dim3 grid, hipStream_t s) {
  if (a.dh <= 64)
    launch_fwd<T, 64>(a, align, grid, s);
  else if (a.dh <= 96)
    launch_fwd<T, 96>(a, align, grid, s);
  else if (a.dh <= 128)
    launch_fwd<T, 128>(a, align, grid, s);
  else
    launch_fwd<T, 256>(a, align, grid, s);
}
void launch_packed_fwd(const PackedAttn& a, int bf16, int align, hipStream_t s) {
  const long rows = (long)a.total_q * a.G;
  const long slots = a.flat ? (rows + PACKED_BM - 1) / PACKED_BM : packed_slots(rows, PACKED_BM, a.nseq);
  const dim3 grid((unsigned)(slots * a.Hk * (a.nsplit > 0 ? a.nsplit : 1)));
  if (bf16)
    launch_fwd_t<bf16_t>(a, align, grid, s);
  else
    launch_fwd_t<float>(a, align, grid, s);
}

// ---------------------------------------------------------------------------------------------------------------------------
// Joining of the parts: lse = log sum exp lse_p, O = sum_p exp(lse_p - lse) o_p, in part order within each of the lane groups that read parts
// side by side.  A wave per (token, head); LR lanes hold a row in pieces of four, 64 / LR parts are read at a time.  Reads each part once: bytes,
// and in small calls the latency of offsets -> lse -> rows, so the parts' lse are read once, a lane each, and handed out by shuffles.
// ---------------------------------------------------------------------------------------------------------------------------
template <typename T, int LR>
__global__ __launch_bounds__(256) void packed_join_kernel(PackedAttn a) {
  typedef typename Elem<T>::raw raw;
  constexpr int NP = 64 / LR;
  const int lane = threadIdx.x & 63;
  const long id = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (id >= (long)a.total_q * a.H) return;   // wave-uniform
  const int tokg = (int)(id / a.H), head = (int)(id - (long)tokg * a.H), hk = head / a.G;
  // the token's sequence: the last one that begins at or before it (empty sequences share a begin with the next)
  int lo = 0, n = a.nseq;
  while (n > 64) {
    const int step = (n + 63) >> 6;
    const unsigned long long m = __ballot(lane * step < n && a.qoff[lo + min(lane * step, n - 1)] <= tokg);
    if (!m) return;
    const int k = __popcll(m) - 1;
    lo += k * step;
    n = min(step, n - k * step);
  }
  const int i = lo + min(lane, n - 1);
  const SeqGeom mine = seq_geom(a, i);
  const int few = a.chunk ? first_slot(a.koff, a.total_k, 1, a.chunk, i) : i;
  const unsigned long long m = __ballot(lane < n && a.qoff[i] <= tokg);
  if (!m) return;
  const int k = __builtin_amdgcn_readfirstlane(__popcll(m) - 1);
  const int lq = __builtin_amdgcn_readlane(mine.lq, k), lk = __builtin_amdgcn_readlane(mine.lk, k), few0 = __builtin_amdgcn_readlane(few, k);
  const int tok = tokg - __builtin_amdgcn_readlane(mine.qbeg, k);
  if (tok < 0 || tok >= lq) return;
  const int row = tok * a.G + head - hk * a.G;
  const int nfew = a.fo ? (a.chunk ? (lk + a.chunk - 1) / a.chunk : 1) : 0, nall = a.nparts + nfew;
  const long rows = (long)a.total_q * a.H;
  float mx = -INFINITY, tot = 0.f;
  f32x4 acc = f32x4{};
  const int c = lane % LR * 4, sub = lane / LR, cc = min(c, a.dhp - 4);
  for (int b = 0; b < nall; b += 64) {   // 64 parts at a time
    const int p = b + lane;
    const float lp = p >= nall ? -INFINITY : p < a.nparts ? a.pl[p * rows + id] : a.fl[((long)(few0 + p - a.nparts) * a.Hk + hk) * a.frows + row];
    float mn = lp;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) mn = fmaxf(mn, __shfl_xor(mn, d, 64));
    mn = fmaxf(mn, mx);
    if (mn == -INFINITY) continue;
    const float w = __builtin_amdgcn_exp2f((lp - mn) * 1.44269504088896340736f), alpha = __builtin_amdgcn_exp2f((mx - mn) * 1.44269504088896340736f);
    mx = mn;
    acc *= alpha;
    tot *= alpha;
    const int many = min(64, nall - b);
#pragma unroll 4
    for (int q = 0; q < many; q += NP) {
      const int p = b + min(q + sub, many - 1);
      const float wp = q + sub < many ? __shfl(w, q + sub, 64) : 0.f;
      const float* o = p < a.nparts ? a.po + (p * rows + id) * a.dhp : a.fo + (((long)(few0 + p - a.nparts) * a.Hk + hk) * a.frows + row) * a.dhp;
      const f32x4 v = *(const f32x4*)(o + cc);
      tot += wp;
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = wp > 0.f ? fmaf(wp, v[j], acc[j]) : acc[j];   // (a part that saw nothing of the row is not written)
    }
  }
#pragma unroll
  for (int d = LR; d < 64; d <<= 1) {
    tot += __shfl_xor(tot, d, 64);
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] += __shfl_xor(acc[j], d, 64);
  }
  const float inv = tot == 0.f ? 0.f : 1.f / tot;
  if (lane == 0 && a.lse) a.lse[(long)head * a.total_q + tokg] = tot == 0.f ? -INFINITY : mx + log2f(tot) * 0.69314718055994530942f;
  if (sub == 0) {
    raw* O = (raw*)a.O + (long)tokg * a.o_row + (long)head * a.o_head;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (c + j < a.dh) st((T*)O, c + j, acc[j] * inv);
  }
}

void launch_packed_join(const PackedAttn& a, int bf16, hipStream_t s) {
  const dim3 grid((unsigned)(((long)a.total_q * a.H + 3) / 4));
  if (bf16) {
    if (a.dh <= 64)
      packed_join_kernel<bf16_t, 16><<<grid, 256, 0, s>>>(a);
    else if (a.dh <= 128)
      packed_join_kernel<bf16_t, 32><<<grid, 256, 0, s>>>(a);
    else
      packed_join_kernel<bf16_t, 64><<<grid, 256, 0, s>>>(a);
  } else {
    if (a.dh <= 64)
      packed_join_kernel<float, 16><<<grid, 256, 0, s>>>(a);
    else if (a.dh <= 128)
      packed_join_kernel<float, 32><<<grid, 256, 0, s>>>(a);
    else
      packed_join_kernel<float, 64><<<grid, 256, 0, s>>>(a);
  }
}

}  // namespace sh
