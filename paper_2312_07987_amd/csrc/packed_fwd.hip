// Forward attention over packed sequences with grouped heads: O = softmax(s Q K^T + mask) V of every sequence by itself, with rows that
// all sequences see in front of their own keys where there is a shared prefix.
//
// Transposed products, S^T[key][row] = K Q^T and O^T[d][row] += V^T P^T: a row (token, head) is a lane column, so the running maximum
// and sum of its softmax are lane-local up to one exchange between the lane halves, and exp(S^T) is the second product's operand as it
// stands.  K and V tiles go through LDS once for all rows of the work-group.
#include <type_traits>

#include "packed_bodies.h"

namespace sh {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

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
// The same for bf16 and long rows of tiles: 4 waves x 64 rows, one wave per SIMD with all of its registers.
//
// What bounds the kernel above is that its waves read every K and V fragment for 32 rows only (the LDS pipe is then as busy as the matrix cores)
// and do one thing at a time: products, then the softmax, then products, with LDS latency in front of each.  Here a fragment serves 64 rows, and the
// loop is a pipeline over steps of 32 keys whose three parts do not depend on each other: in step s the products S(s + 1) = K Q^T, the softmax of S(s)
// and the products O += V^T P(s - 1)^T, 32 matrix instructions (1024 cycles) beside the vector instructions of 32 exponentials a lane (about
// 800), interleaved by the scheduling groups.  K and V tiles of 64 keys lie in three LDS stages each: one barrier per tile.
// The running maximum moves only where a tile's exceeds it by more than 2^8 in the exponent's base (P then stays below 2^8, which costs bf16
// nothing), so the accumulators are hardly ever scaled.
// ---------------------------------------------------------------------------------------------------------------------------
template <int DH, int AL, int NJ, int NW>
__global__ __launch_bounds__(64 * NW, 1) void packed_fwd_long_kernel(PackedAttn a) {
  typedef unsigned short raw;
  constexpr int KT = 64, LDK = row_ld<bf16_t, DH>(), LDV = col_ld<bf16_t, DH>(), NKD = DH / 16, NDB = DH / 32, BM = NW * 32 * NJ, NT = 64 * NW, TK = KT * LDK, TV = KT * LDV;
  constexpr bool ACC = NW == 4;   // one wave per SIMD: 256 more registers that only matrix instructions and moves reach
  __shared__ __attribute__((aligned(16))) raw Ks[3 * TK], Vs[3 * TV];
  int b = blockIdx.x;
  const int hk = b % a.Hk;
  b /= a.Hk;
  const int ns = max(a.nsplit, 1), split = b % ns, slot = b / ns;
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
  if (row0 < 0 || row0 >= rows) return;
  const int off = s.lk - s.lq, wr = row0 + wave * 32 * NJ;
  const int wq_first = div_by(min(wr, rows - 1), a.g_inv) + off, wq_last = div_by(min(wr + 32 * NJ - 1, rows - 1), a.g_inv) + off;
  const int last_tok = div_by(min(row0 + BM, rows) - 1, a.g_inv);
  const int prefix = a.own ? 0 : a.prefix;
  const int kend = max(0, a.causal ? min(s.lk, last_tok + off + 1) : s.lk);
  int tok[NJ], head[NJ];
  bf16x8 qf[NJ][NKD];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int row = min(wr + j * 32 + r, rows - 1);
    tok[j] = div_by(row, a.g_inv);
    head[j] = hk * a.G + row - tok[j] * a.G;
  }
  f32x16 o[NJ][NDB];
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int d = 0; d < NDB; ++d) o[j][d] = zero16();
  float m[NJ], l[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    m[j] = -INFINITY;
    l[j] = 0.f;
  }
  const float sc = a.scale * 1.44269504088896340736f;

  const int np = (prefix + KT - 1) / KT, nt = np + (kend + KT - 1) / KT;
  const int t0 = (int)((unsigned)(nt * split) / (unsigned)ns), t1 = (int)((unsigned)(nt * (split + 1)) / (unsigned)ns);
  // this wave's tiles: up to the last one with a key that one of its rows sees
  const int seen = !a.causal ? nt : np + (wq_last >= 0 ? wq_last / KT + 1 : 0);
  const int tend = wr < rows ? min(t1, seen) : 0;
  PieceTile<bf16_t, DH, AL, KT, NT> tk, tv;
  const raw* const KP = (const raw*)a.KP + (long)hk * a.kp_head;
  const raw* const VP = (const raw*)a.VP + (long)hk * a.vp_head;
  const raw* const K = (const raw*)a.K + (long)s.kbeg * a.k_row + (long)hk * a.k_head;
  const raw* const V = (const raw*)a.V + (long)s.kbeg * a.v_row + (long)hk * a.v_head;
  auto valid_of = [&](int t) { return t < np ? prefix - t * KT : kend - (t - np) * KT; };
  tk.place(t0 < np ? a.kp_row : a.k_row, tid);   // (the prefix may have other strides: placed again at the border)
  tv.place(t0 < np ? a.vp_row : a.v_row, tid);
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
  auto stage = [&](int t) { return (t - t0) % 3; };
  auto hold = [](auto& tile) {   // a tile on its way waits in the accumulation registers
#pragma unroll
    for (int i = 0; i < tile.NCH; ++i)
      if constexpr (ACC) asm volatile("" : "+a"(*(u32x4*)&tile.r[i]));
  };
  f32x16 S[2][NJ];   // [step parity][row block]
  bf16x8 P[2][NJ][2];   // [step parity][row block][16 keys]
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int st = 0; st < 2; ++st) P[1][j][st] = bf16x8{};

  if (t0 < t1) {
    // tile t0 of both, tile t0 + 1 of K; zeros where the first step's products with P = 0 read V
    load_k(t0);
    load_v(t0);
#pragma unroll
    for (int j = 0; j < NJ; ++j)   // (behind the tile's loads: what is done with them waits for them)
      mem_frags<bf16_t, AL, NKD, 16>(qf[j], (const raw*)a.Q + (long)(s.qbeg + tok[j]) * a.q_row + (long)head[j] * a.q_head, 8 * g, dh, wr + j * 32 + r < rows);
    for (int i = tid; i < TV / 8; i += NT) *(uint4*)(Vs + 2 * TV + i * 8) = make_uint4(0, 0, 0, 0);
    tk.store(Ks, LDK, valid_of(t0), dh, tid);
    tv.store(Vs, LDV, valid_of(t0), dh, tid);
    if (t0 + 1 < t1) {
      load_k(t0 + 1);
      load_v(t0 + 1);
      tk.store(Ks + TK, LDK, valid_of(t0 + 1), dh, tid);
    }
    if (t0 + 2 < t1) load_k(t0 + 2);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < NJ; ++j) S[0][j] = zero16();
#pragma unroll
    for (int kk = 0; kk < NKD; ++kk) {
      const bf16x8 kf = row_frag(&Ks[r * LDK + kk * 16 + 8 * g]);
#pragma unroll
      for (int j = 0; j < NJ; ++j) S[0][j] = mma32(kf, qf[j][kk], S[0][j]);
    }
  }
  // one step: PAR its parity; Kn the next step's 32 keys, Vp the previous step's.  The matrix instructions come in slots of two (the row blocks)
  // that share a fragment, read three slots ahead; a slot's share of the softmax is issued behind them.  First the maximum, over the first SM
  // slots, then the exponentials.
  constexpr int NF = NKD + 2 * NDB, NS = NJ * NF, SM = NS / 4, AHEAD = 3;
  auto step = [&](int st_, auto par, const raw* Kn, const raw* Vp) {
    constexpr int PAR = decltype(par)::value;
    const int t = st_ >> 1, valid = valid_of(t) - 32 * PAR, k0 = (t - np) * KT + 32 * PAR;
    const bool masked = a.causal && t >= np;
    // the products leave S in accumulation registers; Q and O stay there, which leaves the others to the softmax
    f32x16 sv[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      sv[j] = S[PAR][j];
      if constexpr (ACC) {
        asm volatile("" : "+v"(sv[j]));
#pragma unroll
        for (int kk = 0; kk < NKD; ++kk) asm volatile("" : "+a"(qf[j][kk]));
#pragma unroll
        for (int d = 0; d < NDB; ++d) asm volatile("" : "+a"(o[j][d]));
      }
    }
    if (valid < 32 || (masked && k0 + 31 > wq_first)) {   // wave-uniform
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const int lim = (masked ? min(valid - 1, tok[j] + off - k0) : valid - 1) - 4 * g;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (8 * (i >> 2) + (i & 3) > lim) sv[j][i] = -INFINITY;
      }
    }
    auto fragment = [&](int q) {
      const int i = q / 2;   // in turn: the score products are one chain, each waits for the one before it
      return q % 2 == 0 ? row_frag(&Kn[r * LDK + i * 16 + 8 * g]) : col_frag(Vp, LDV, 16 * (i / NDB) + 4 * g, 16 * (i / NDB) + 4 * g + 8, i % NDB * 32, lane);
    };
    bf16x8 f[NF];
    float mt[NJ], mb[NJ], alpha[NJ], ps[NJ], p[NJ][16];
    bool any = false;
#pragma unroll
    for (int j = 0; j < NJ; ++j) ps[j] = 0.f;
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) f[q] = fragment(q);
#pragma unroll
    for (int u = 0; u < NS; ++u) {
      const int q = u / NJ, h = u % NJ;
      if (h == 0 && q + AHEAD < NF) f[q + AHEAD] = fragment(q + AHEAD);
      const int i = q / 2;
      if (q % 2 == 0)
        S[PAR ^ 1][h] = mma32(f[q], qf[h][i], i == 0 ? zero16() : S[PAR ^ 1][h]);
      else
        o[h][i % NDB] = mma32(f[q], P[PAR ^ 1][h][i / NDB], o[h][i % NDB]);
      if (u < SM) {
        // maximum over elements 16 u / SM .. of both row blocks
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          if (u == 0) mt[j] = sv[j][0];
#pragma unroll
          for (int e = 16 * u / SM; e < 16 * (u + 1) / SM; ++e) mt[j] = fmaxf(mt[j], sv[j][e]);
          if (u == SM - 1) {
            mt[j] = half_max(mt[j]) * sc;
            const bool moved = mt[j] > m[j] + 8.f;
            any |= moved;
            const float mn = moved ? mt[j] : m[j];
            mb[j] = mn == -INFINITY ? 0.f : mn;
            alpha[j] = moved ? __builtin_amdgcn_exp2f(m[j] - mn) : 1.f;   // m = -inf: 0
            m[j] = mn;
          }
        }
      } else {
#pragma unroll
        for (int e = 16 * NJ * (u - SM) / (NS - SM); e < 16 * NJ * (u + 1 - SM) / (NS - SM); ++e) {
          const int j = e / 16, c = e % 16;
          p[j][c] = __builtin_amdgcn_exp2f(fmaf(sv[j][c], sc, -mb[j]));   // masked: 0
          ps[j] += p[j][c];
          // P is rounded to bf16 for its product; the sum keeps 32 bits
          if (c % 8 == 7) {
            pack_frag(P[PAR][j][c / 8], &p[j][c - 7]);
            asm volatile("" : "+v"(P[PAR][j][c / 8]));   // here, not where the next step reads it
          }
        }
      }
#pragma unroll
      for (int j = 0; j < NJ; ++j) asm volatile("" : "+v"(ps[j]));
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) l[j] = fmaf(l[j], alpha[j], ps[j]);
    if (__ballot(any)) {
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int d = 0; d < NDB; ++d) {
#pragma unroll
          for (int i = 0; i < 16; ++i) o[j][d][i] *= alpha[j];
          if constexpr (ACC) asm volatile("" : "+a"(o[j][d]));   // 16 at a time, or the compiler asks for 128 registers at once
        }
    }
  };
  // tile t + 1 of V and t + 2 of K (requested a trip ago) go into their stages, and the next ones start to travel
  auto move = [&](int t) {
    if (t > t0) __syncthreads();
    if (t + 1 < t1) {
      hold(tv);
      tv.store(Vs + stage(t + 1) * TV, LDV, valid_of(t + 1), dh, tid);
    }
    if (t + 2 < t1) {
      hold(tk);
      tk.store(Ks + stage(t + 2) * TK, LDK, valid_of(t + 2), dh, tid);
      load_v(t + 2);
    }
    if (t + 3 < t1) load_k(t + 3);
  };
  for (int t = t0; t < tend; ++t) {
    move(t);
    const raw *const Kt = Ks + stage(t) * TK, *const Vt = Vs + stage(t) * TV;
    step(2 * t, std::integral_constant<int, 0>{}, Kt + 32 * LDK, Vs + (t - t0 + 2) % 3 * TV + 32 * LDV);
    step(2 * t + 1, std::integral_constant<int, 1>{}, Ks + stage(t + 1) * TK, Vt);
  }
  if (tend > t0) {   // the last step's products with V
    const raw* Vp = Vs + stage(tend - 1) * TV + 32 * LDV;
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int d = 0; d < NDB; ++d) {
        const bf16x8 vf = col_frag(Vp, LDV, 16 * st + 4 * g, 16 * st + 4 * g + 8, d * 32, lane);
#pragma unroll
        for (int j = 0; j < NJ; ++j) o[j][d] = mma32(vf, P[1][j][st], o[j][d]);
      }
  }
  for (int t = max(tend, t0); t < t1; ++t) move(t);   // (tiles that only the other waves' rows see)
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    float lt = l[j];
    lt += __shfl_xor(lt, 32, 64);
    if (wr + j * 32 + r >= rows) continue;
    const float inv = lt > 0.f ? 1.f / lt : (lt == 0.f ? 0.f : lt);
    const float lse = lt == 0.f ? -INFINITY : (m[j] + log2f(lt)) * 0.69314718055994530942f;
    if (a.nsplit) {
      const long at = (long)(a.part0 + split) * a.total_q * a.H + (long)(s.qbeg + tok[j]) * a.H + head[j];
      if (g == 0) a.pl[at] = lse;
      store_row<float, 16, NDB>(a.po + at * a.dhp, o[j], inv, g, dh);
    } else {
      if (g == 0 && a.lse) a.lse[(long)head[j] * a.total_q + s.qbeg + tok[j]] = lse;
      store_row<bf16_t, AL, NDB>((raw*)a.O + (long)(s.qbeg + tok[j]) * a.o_row + (long)head[j] * a.o_head, o[j], inv, g, dh);
    }
  }
}

template <typename T, int DH, int AL>
static void launch_fwd_al(const PackedAttn& a, dim3 grid, hipStream_t s) {
  if constexpr (DH >= 64 && DH <= 128 && sizeof(T) == 2) {
    if (a.groups == 4) {
      packed_fwd_long_kernel<DH, AL, 1, 8><<<grid, 512, 0, s>>>(a);
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
  const int bm = a.groups == 4 ? PACKED_BM2 : PACKED_BM;
  const long slots = a.flat ? (rows + bm - 1) / bm : a.levels ? (long)a.levels * a.nseq : packed_slots(rows, bm, a.nseq);
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
