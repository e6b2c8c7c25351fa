// Attention of a few rows per sequence and kv head over many keys: single tokens (or a few) over a cache, with the heads of a group as
// further rows, at most 16 in all.  A work-group takes one (sequence, kv head) and a chunk of its keys; chunks have one length
// for all sequences, so ragged lengths make more work-groups, not longer ones.
//
// 16 x 16 products, lane = 16 g + r:
//   S^T[key][row] = K Q^T       K straight from memory in operand order (16 rows of 64 or 128 contiguous bytes an instruction)
//   O^T[d][row] += V^T P^T      a lane's scores of a piece's two blocks of 16 keys (4 g .. 4 g + 3 of each) are its operand as they are; V goes
//                               through the wave's own LDS and is read by columns in that key order
// The waves take every fourth piece of 32 keys without barriers; a piece's registers are requested again as soon as they are free and
// travel during the softmax and the second product.  Bound by reading K and V once.
#include "packed_attn.h"

namespace sh {

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
__global__ __launch_bounds__(256, 1) void packed_few_kernel(PackedAttn a) {
  typedef typename Elem<T>::raw raw;
  constexpr int W = 4, KP = 32, PER = Elem<T>::PER, FP = 8 / PER;   // waves; keys of a piece; pieces of a fragment
  constexpr int NK = DH / 32, ND = DH / 16, LDV = tile_ld<T, DH>(), CPR = DH / PER, NV = KP * CPR / 64, LDO = DH + 4;
  __shared__ __attribute__((aligned(16))) raw fsm[W * KP * LDV];   // a piece of V per wave, then its output in fp32
  __shared__ float ms[W][PACKED_FEW], ls[W][PACKED_FEW];
  static_assert(PACKED_FEW * LDO * 4 <= KP * LDV * (int)sizeof(raw), "a wave's output fits over its V piece");

  const int hk = blockIdx.x % a.Hk, slot = blockIdx.x / a.Hk;
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
  if (rows <= 0 || (a.chunk && key0 >= s.lk)) return;   // (unsplit, a sequence without keys still gets its zeros)
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

template <typename T, int DH>
static void launch_few(const PackedAttn& a, int align, dim3 grid, hipStream_t s) {
  if (align == 16) {
    packed_few_kernel<T, DH, 16><<<grid, 256, 0, s>>>(a);
    return;
  }
  if constexpr (sizeof(T) == 2) {
    if (align == 8) {
      packed_few_kernel<T, DH, 8><<<grid, 256, 0, s>>>(a);
      return;
    }
  }
  packed_few_kernel<T, DH, sizeof(T)><<<grid, 256, 0, s>>>(a);
}
template <typename T>
static void launch_few_t(const PackedAttn& a, int align, dim3 grid, hipStream_t s) {
  if (a.dh <= 64)
    launch_few<T, 64>(a, align, grid, s);
  else if (a.dh <= 128)
    launch_few<T, 128>(a, align, grid, s);
  else
    launch_few<T, 256>(a, align, grid, s);
}
void launch_packed_few(const PackedAttn& a, int bf16, int align, hipStream_t s) {
  const long slots = a.chunk ? packed_slots(a.total_k, a.chunk, a.nseq) : a.nseq;
  const dim3 grid((unsigned)(slots * a.Hk));
  if (bf16)
    launch_few_t<bf16_t>(a, align, grid, s);
  else
    launch_few_t<float>(a, align, grid, s);
}

}  // namespace sh
