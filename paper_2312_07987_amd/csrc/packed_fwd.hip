// Forward attention over packed sequences with grouped heads: O = softmax(s Q K^T + mask) V of every sequence by itself, with rows that
// all sequences see in front of their own keys where there is a shared prefix.
//
// Transposed products, S^T[key][row] = K Q^T and O^T[d][row] += V^T P^T: a row (token, head) is a lane column, so the running maximum
// and sum of its softmax are lane-local up to one exchange between the lane halves, and exp(S^T) is the second product's operand as it
// stands.  K and V tiles go through LDS once for all rows of the work-group.
#include <type_traits>

#include "packed_bodies.h"

namespace sh {

template <typename T, int DH, int AL, int NG>
__global__ __launch_bounds__(256 * NG, DH <= 128 && NG == 1 ? 2 : 1) void packed_fwd_kernel(PackedAttn a) {
  __shared__ __attribute__((aligned(16))) typename Elem<T>::raw kv[packed_fwd_lds<T, DH, NG>()];
  packed_fwd_body<T, DH, AL, NG>(a, blockIdx.x, kv);
}

// the larger of the two lane halves' values, in both
__device__ __forceinline__ float half_max(float x) {
  const auto v = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(v[0]), __uint_as_float(v[1]));
}
// ---------------------------------------------------------------------------------------------------------------------------
// The same for bf16, heads of 97 .. 128 elements and long rows of keys: 256 rows, eight waves of 32, one work-group per CU.
//
// A wave of the kernel above does one thing at a time, products, softmax, products, and counts on the other wave of its SIMD to fill the matrix cores
// meanwhile.  Here the loop is a pipeline over steps of 32 keys whose three parts do not depend on each other: in step s the products
// S(s + 1) = K Q^T, the softmax of S(s) and the products O += V^T P(s - 1)^T, 16 matrix instructions (512 cycles) with the vector instructions of 16
// exponentials a lane issued between them.  K and V tiles of 64 keys, read once for 256 rows, lie in three LDS stages each: one barrier per tile.
// The running maximum moves only where a tile's exceeds it by more than 2^8 in the exponent's base (P then stays below 2^8, which costs bf16
// nothing), so the accumulators are hardly ever scaled.
// Bound by what the vector and LDS pipes take between the products: 8192 tokens, 32 heads over 8 600 us, 916 TFLOP/s; with the matrix instructions alone
// 433, without staging the tiles 550, without the exponentials 625 of 690 on the card where these were timed.  (64 rows a wave, one wave per SIMD, is no
// help: a lone wave issues vector instructions at half rate.)  Narrower heads have fewer products to hide the same softmax behind: of 64, 4 x 2048
// tokens, 128 us against 101 with the kernel above.
// ---------------------------------------------------------------------------------------------------------------------------
template <int AL>
__global__ __launch_bounds__(512, 1) void packed_fwd_long_kernel(PackedAttn a) {
  typedef unsigned short raw;
  constexpr int DH = 128, KT = 64, LDK = row_ld<bf16_t, DH>(), LDV = col_ld<bf16_t, DH>(), NKD = DH / 16, NDB = DH / 32, BM = PACKED_BM2, NT = 512, TK = KT * LDK, TV = KT * LDV;
  __shared__ __attribute__((aligned(16))) raw Ks[3 * TK], Vs[3 * TV];
  const int hk = blockIdx.x % a.Hk, slot = blockIdx.x / a.Hk;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 31, g = lane >> 5, dh = a.dh;
  SeqGeom s;
  int row0;
  if (a.levels) {
    s = seq_geom(a, level_seq(slot, a.nseq));
    row0 = (a.levels - 1 - slot / a.nseq) * BM;
  } else {
    int nth;
    if (!find_slot<false>(a, BM, slot, nth, s)) return;
    row0 = ((s.lq * a.G + BM - 1) / BM - 1 - nth) * BM;
  }
  const int rows = s.lq * a.G;
  if (row0 >= rows) return;
  const int off = s.lk - s.lq, wr = row0 + wave * 32, row = wr + r;
  const int wq_first = div_by(min(wr, rows - 1), a.g_inv) + off, wq_last = div_by(min(wr + 31, rows - 1), a.g_inv) + off;
  const int last_tok = div_by(min(row0 + BM, rows) - 1, a.g_inv);
  const int prefix = a.prefix;
  const int kend = max(0, a.causal ? min(s.lk, last_tok + off + 1) : s.lk);
  const int tok = div_by(min(row, rows - 1), a.g_inv), head = hk * a.G + min(row, rows - 1) - tok * a.G;
  bf16x8 qf[NKD];
  f32x16 o[NDB];
#pragma unroll
  for (int d = 0; d < NDB; ++d) o[d] = zero16();
  float m = -INFINITY, l = 0.f;
  const float sc = a.scale * 1.44269504088896340736f;

  const int np = (prefix + KT - 1) / KT, nt = np + (kend + KT - 1) / KT;
  // this wave's tiles: up to the last one with a key that one of its rows sees
  const int seen = !a.causal ? nt : np + (wq_last >= 0 ? wq_last / KT + 1 : 0);
  const int tend = wr < rows ? min(nt, seen) : 0;
  PieceTile<bf16_t, DH, AL, KT, NT> tk, tv;
  const raw* const KP = (const raw*)a.KP + (long)hk * a.kp_head;
  const raw* const VP = (const raw*)a.VP + (long)hk * a.vp_head;
  const raw* const K = (const raw*)a.K + (long)s.kbeg * a.k_row + (long)hk * a.k_head;
  const raw* const V = (const raw*)a.V + (long)s.kbeg * a.v_row + (long)hk * a.v_head;
  auto valid_of = [&](int t) { return t < np ? prefix - t * KT : kend - (t - np) * KT; };
  tk.place(0 < np ? a.kp_row : a.k_row, tid);   // (the prefix may have other strides: placed again at the border)
  tv.place(0 < np ? a.vp_row : a.v_row, tid);
  auto load_k = [&](int t) {
    const bool p = t < np;
    if (t == np) tk.place(a.k_row, tid);
    tk.load((p ? KP : K) + (long)(p ? t : t - np) * KT * (p ? a.kp_row : a.k_row), p ? a.kp_row : a.k_row, valid_of(t), dh, tid);
  };
  auto load_v = [&](int t) {
    const bool p = t < np;
    if (t == np) tv.place(a.v_row, tid);
    tv.load((p ? VP : V) + (long)(p ? t : t - np) * KT * (p ? a.vp_row : a.v_row), p ? a.vp_row : a.v_row, valid_of(t), dh, tid);
  };
  f32x16 S[2];      // [step parity]
  bf16x8 P[2][2];   // [step parity][16 keys]
  P[1][0] = P[1][1] = bf16x8{};

  if (nt > 0) {
    // tile 0 of both, tile 1 of K; zeros where the first step's products with P = 0 read V
    load_k(0);
    load_v(0);
    // (behind the tile's loads: what is done with them waits for them)
    mem_frags<bf16_t, AL, NKD, 16>(qf, (const raw*)a.Q + (long)(s.qbeg + tok) * a.q_row + (long)head * a.q_head, 8 * g, dh, row < rows);
    for (int i = tid; i < TV / 8; i += NT) *(uint4*)(Vs + 2 * TV + i * 8) = make_uint4(0, 0, 0, 0);
    tk.store(Ks, LDK, valid_of(0), dh, tid);
    tv.store(Vs, LDV, valid_of(0), dh, tid);
    if (nt > 1) {
      load_k(1);
      load_v(1);
      tk.store(Ks + TK, LDK, valid_of(1), dh, tid);
    }
    if (nt > 2) load_k(2);
    __syncthreads();
    S[0] = zero16();
#pragma unroll
    for (int kk = 0; kk < NKD; ++kk) S[0] = mma32(row_frag(&Ks[r * LDK + kk * 16 + 8 * g]), qf[kk], S[0]);
  }
  // one step: PAR its parity; Kn the next step's 32 keys, Vp the previous step's.  The matrix instructions' fragments are read AHEAD ones before them, and a
  // share of the softmax is issued behind each: first the maximum, over the first SM instructions, then the exponentials.
  constexpr int NF = NKD + 2 * NDB, SM = NF / 4, AHEAD = 3;
  auto step = [&](int st_, auto par, const raw* Kn, const raw* Vp) {
    constexpr int PAR = decltype(par)::value;
    const int t = st_ >> 1, valid = valid_of(t) - 32 * PAR, k0 = (t - np) * KT + 32 * PAR;
    const bool masked = a.causal && t >= np;
    f32x16 sv = S[PAR];
    if (valid < 32 || (masked && k0 + 31 > wq_first)) {   // wave-uniform
      const int lim = (masked ? min(valid - 1, tok + off - k0) : valid - 1) - 4 * g;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (8 * (i >> 2) + (i & 3) > lim) sv[i] = -INFINITY;
    }
    auto fragment = [&](int q) {
      const int i = q / 2;   // in turn: the score products are one chain, each waits for the one before it
      return q % 2 == 0 ? row_frag(&Kn[r * LDK + i * 16 + 8 * g]) : col_frag(Vp, LDV, 16 * (i / NDB) + 4 * g, 16 * (i / NDB) + 4 * g + 8, i % NDB * 32, lane);
    };
    bf16x8 f[NF];
    float mt, mb, alpha, ps = 0.f, p[16];
    bool moved = false;
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) f[q] = fragment(q);
#pragma unroll
    for (int q = 0; q < NF; ++q) {
      if (q + AHEAD < NF) f[q + AHEAD] = fragment(q + AHEAD);
      const int i = q / 2;
      if (q % 2 == 0)
        S[PAR ^ 1] = mma32(f[q], qf[i], i == 0 ? zero16() : S[PAR ^ 1]);
      else
        o[i % NDB] = mma32(f[q], P[PAR ^ 1][i / NDB], o[i % NDB]);
      if (q < SM) {
        if (q == 0) mt = sv[0];
#pragma unroll
        for (int e = 16 * q / SM; e < 16 * (q + 1) / SM; ++e) mt = fmaxf(mt, sv[e]);
        if (q == SM - 1) {
          mt = half_max(mt) * sc;
          moved = mt > m + 8.f;
          const float mn = moved ? mt : m;
          mb = mn == -INFINITY ? 0.f : mn;
          alpha = moved ? __builtin_amdgcn_exp2f(m - mn) : 1.f;   // m = -inf: 0
          m = mn;
        }
      } else {
#pragma unroll
        for (int e = 16 * (q - SM) / (NF - SM); e < 16 * (q + 1 - SM) / (NF - SM); ++e) {
          p[e] = __builtin_amdgcn_exp2f(fmaf(sv[e], sc, -mb));   // masked: 0
          ps += p[e];
          // P is rounded to bf16 for its product; the sum keeps 32 bits
          if (e % 8 == 7) {
            pack_frag(P[PAR][e / 8], &p[e - 7]);
            asm volatile("" : "+v"(P[PAR][e / 8]));   // here, not where the next step reads it
          }
        }
      }
      asm volatile("" : "+v"(ps));
      __builtin_amdgcn_sched_barrier(0);
    }
    l = fmaf(l, alpha, ps);
    if (__ballot(moved)) {
#pragma unroll
      for (int d = 0; d < NDB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= alpha;
    }
  };
  // tile t + 1 of V and t + 2 of K (requested a trip ago) go into their stages, and the next ones start to travel
  int s0 = 0, s1 = 1, s2 = 2;   // the stages of the tiles t, t + 1, t + 2 (and t - 1)
  auto move = [&](int t) {
    if (t > 0) __syncthreads();
    if (t + 1 < nt) tv.store(Vs + s1 * TV, LDV, valid_of(t + 1), dh, tid);
    if (t + 2 < nt) {
      tk.store(Ks + s2 * TK, LDK, valid_of(t + 2), dh, tid);
      load_v(t + 2);
    }
    if (t + 3 < nt) load_k(t + 3);
  };
  auto turn = [&] {
    const int x = s0;
    s0 = s1;
    s1 = s2;
    s2 = x;
  };
  for (int t = 0; t < tend; ++t) {
    move(t);
    const raw *const Kt = Ks + s0 * TK, *const Vt = Vs + s0 * TV;
    step(2 * t, std::integral_constant<int, 0>{}, Kt + 32 * LDK, Vs + s2 * TV + 32 * LDV);
    step(2 * t + 1, std::integral_constant<int, 1>{}, Ks + s1 * TK, Vt);
    turn();
  }
  if (tend > 0) {   // the last step's products with V
    const raw* Vp = Vs + s2 * TV + 32 * LDV;
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int d = 0; d < NDB; ++d) o[d] = mma32(col_frag(Vp, LDV, 16 * st + 4 * g, 16 * st + 4 * g + 8, d * 32, lane), P[1][st], o[d]);
  }
  for (int t = tend; t < nt; ++t) {   // (tiles that only the other waves' rows see)
    move(t);
    turn();
  }
  l += __shfl_xor(l, 32, 64);
  if (row >= rows) return;
  const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);   // nothing seen: zeros; NaN stays
  const float lse = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994530942f;
  if (g == 0 && a.lse) a.lse[(long)head * a.total_q + s.qbeg + tok] = lse;
  store_row<bf16_t, AL, NDB>((raw*)a.O + (long)(s.qbeg + tok) * a.o_row + (long)head * a.o_head, o, inv, g, dh);
}

template <typename T, int DH, int AL>
static void launch_fwd_al(const PackedAttn& a, dim3 grid, hipStream_t s) {
  if constexpr (DH == 128 && sizeof(T) == 2) {
    if (a.tall) {
      packed_fwd_long_kernel<AL><<<grid, 512, 0, s>>>(a);
      return;
    }
  }
  if constexpr (DH <= 128) {
    if (a.groups == 2) {
      packed_fwd_kernel<T, DH, AL, 2><<<grid, 512, 0, s>>>(a);
      return;
    }
  }
  packed_fwd_kernel<T, DH, AL, 1><<<grid, 256, 0, s>>>(a);
}
template <typename T, int DH>
static void launch_fwd(const PackedAttn& a, int align, dim3 grid, hipStream_t s) {
  if (align == 16) return launch_fwd_al<T, DH, 16>(a, grid, s);
  if constexpr (sizeof(T) == 2) {
    if (align == 8) return launch_fwd_al<T, DH, 8>(a, grid, s);
  }
  launch_fwd_al<T, DH, sizeof(T)>(a, grid, s);
}
template <typename T>
static void launch_fwd_t(const PackedAttn& a, int align, dim3 grid, hipStream_t s) {
  if (a.dh <= 32)
    launch_fwd<T, 32>(a, align, grid, s);
  else if (a.dh <= 64)
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
  const int bm = a.tall ? PACKED_BM2 : PACKED_BM;
  const long slots = a.levels ? (long)a.levels * a.nseq : packed_slots(rows, bm, a.nseq);
  const dim3 grid((unsigned)(slots * a.Hk * (a.nsplit > 0 ? a.nsplit : 1)));
  if (bf16)
    launch_fwd_t<bf16_t>(a, align, grid, s);
  else
    launch_fwd_t<float>(a, align, grid, s);
}

// ---------------------------------------------------------------------------------------------------------------------------
// Joining of the parts: lse = log sum exp lse_p, O = sum_p exp(lse_p - lse) o_p, in one fixed order.  LR lanes hold a row in pieces of four, so a wave
// reads 64 / LR parts at a time; WV waves share a (token, head) and meet in LDS.  Reads each part once: bytes, and in small calls the latency of
// offsets -> lse -> rows, so the parts' lse are read once, a lane each, and handed out by shuffles.
// ---------------------------------------------------------------------------------------------------------------------------
template <typename T, int LR, int WV>
__global__ __launch_bounds__(256) void packed_join_kernel(PackedAttn a) {
  typedef typename Elem<T>::raw raw;
  constexpr int NP = 64 / LR;
  __shared__ float sm_o[WV > 1 ? 4 : 1][LR * 4], sm_s[WV > 1 ? 4 : 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long id = WV > 1 ? (long)blockIdx.x : (long)blockIdx.x * 4 + wave;
  if (id >= (long)a.total_q * a.H) return;   // uniform among the waves of a row, as all returns below
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
    const float mb = mn == -INFINITY ? 0.f : mn;   // (nothing seen yet, or NaN alone, which has to stay)
    const float w = __builtin_amdgcn_exp2f((lp - mb) * 1.44269504088896340736f), alpha = __builtin_amdgcn_exp2f((mx - mb) * 1.44269504088896340736f);
    mx = mn;
    acc *= alpha;
    tot *= alpha;
    const int many = min(64, nall - b);
#pragma unroll 4
    for (int q = WV > 1 ? wave * NP : 0; q < many; q += NP * WV) {
      const int p = b + min(q + sub, many - 1);
      const float wq = __shfl(w, min(q + sub, 63), 64);   // (of all lanes: a lane that takes no part hands nothing out)
      const float wp = q + sub < many ? wq : 0.f;
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
  if constexpr (WV > 1) {   // (all waves of the row hold the same mx)
    if (sub == 0) *(f32x4*)&sm_o[wave][c] = acc;
    if (lane == 0) sm_s[wave] = tot;
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int x = 1; x < WV; ++x) {
      tot += sm_s[x];
      acc += *(const f32x4*)&sm_o[x][c];
    }
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

template <typename T, int LR>
static void launch_join(const PackedAttn& a, hipStream_t s) {
  // Four waves a row where there are few rows, and latency counts: 64 / 1920 rows in 12 / 3 parts 20.0 -> 17.9 / 24.4 -> 20.6 us (with what makes the
  // parts); 4096 / 7680 rows 23.4 -> 26.1 / 33.8 -> 38.0
  const long rows = (long)a.total_q * a.H;
  if (rows < 2048)
    packed_join_kernel<T, LR, 4><<<dim3((unsigned)rows), 256, 0, s>>>(a);
  else
    packed_join_kernel<T, LR, 1><<<dim3((unsigned)((rows + 3) / 4)), 256, 0, s>>>(a);
}
template <typename T>
static void launch_join_t(const PackedAttn& a, hipStream_t s) {
  if (a.dh <= 64)
    launch_join<T, 16>(a, s);
  else if (a.dh <= 128)
    launch_join<T, 32>(a, s);
  else
    launch_join<T, 64>(a, s);
}
void launch_packed_join(const PackedAttn& a, int bf16, hipStream_t s) {
  if (bf16)
    launch_join_t<bf16_t>(a, s);
  else
    launch_join_t<float>(a, s);
}

}  // namespace sh
