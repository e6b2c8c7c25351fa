// Norms of queries and keys for each head with the position rotation in the same pass:
//   n = x r w,  r = (mean x^2 + eps)^(-1/2) over the head's d elements,  y = n with the pair (2 i, 2 i + 1) turned by
//   position * theta^(-2 i / rope_dim) for 2 i < rope_dim.
// Backward (r is computed again from x: keeping it would save nothing, x is read anyway):
//   dn = dy turned back,  dw = sum over rows of dn x r,  g = dn w,  dx = r (g - x r mean(g x r)).
//
// Bound by bytes: x (and dy) read once, y (dx) written once.  A group of LR lanes holds a head's row in 16-byte pieces (the
// sums over it are a butterfly), takes one token and walks that token's heads, so the token's sines and cosines are computed once for all
// of its heads: angles in 64 bits down to a fraction of a turn and a remainder, so positions of millions keep their place to the last bit of fp32.
#include "packed_attn.h"

namespace sh {

// cos and sin of 2 pi * turns
__device__ __forceinline__ void turn_cos_sin(double turns, float& c, float& s) {
  const double f = turns - rint(turns);   // exact
  const float hi = (float)f, lo = (float)(f - (double)hi) * 6.28318530717958647692f;   // lo: below 2^-25 turns
  float s0, c0;
  sincospif(2.f * hi, &s0, &c0);
  c = fmaf(-lo, s0, c0);
  s = fmaf(lo, c0, s0);
}

template <typename T>
struct Lane {   // a lane's elements of a row
  static constexpr int N = Elem<T>::PER;
  float v[N];
  __device__ __forceinline__ void from(uint4 q) {
    const unsigned w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (sizeof(T) == 2)
        v[i] = __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
      else
        v[i] = __uint_as_float(w[i]);
    }
  }
};

template <typename T, int AL>
__device__ __forceinline__ uint4 lane_piece(const typename Elem<T>::raw* row, int d, int dh) {
  return cut_piece<T, AL>(load_row_piece<T, AL>(row, d, dh), d, dh);
}
template <typename T, int AL>
__device__ __forceinline__ void store_piece(typename Elem<T>::raw* row, int d, int dh, const float* v) {
  constexpr int N = Elem<T>::PER;
  if constexpr (AL == 16) {
    if (d >= dh) return;
    if constexpr (sizeof(T) == 2)
      *(uint4*)(row + d) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
    else
      *(float4*)(row + d) = make_float4(v[0], v[1], v[2], v[3]);
  } else if constexpr (AL == 8) {
    if (d < dh) *(uint2*)(row + d) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    if (d + 4 < dh) *(uint2*)(row + d + 4) = make_uint2(pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (d + i < dh) st((T*)row, d + i, v[i]);
  }
}

// What a lane keeps for all heads of a token: its columns' weights and its pairs' angle rates in turns per position
template <typename T, int AL>
struct NormCols {
  static constexpr int N = Elem<T>::PER;
  float w[2][N];
  double rate[N / 2];
  __device__ __forceinline__ void init(const QkNormArgs& a, int d) {
    Lane<T> l;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const typename Elem<T>::raw* w_ = (const typename Elem<T>::raw*)a.w[k];
      if (w_) l.from(lane_piece<T, AL>(w_, d, a.dh));
#pragma unroll
      for (int i = 0; i < N; ++i) w[k][i] = w_ ? l.v[i] : 1.f;
    }
    // theta^(-2 i / rope_dim) / 2 pi from its binary powers: pair i = d / 2 + j
#pragma unroll
    for (int j = 0; j < N / 2; ++j) {
      const int i = d / 2 + j;
      double x = 0.15915494309189533577;
#pragma unroll
      for (int k = 0; k < 7; ++k)
        if (i >> k & 1) x *= a.rate[k];
      rate[j] = 2 * i < a.rope_dim ? x : 0.;
    }
  }
};

template <typename T, int LR, int AL>
__global__ __launch_bounds__(256) void qk_norm_rope_fwd_kernel(QkNormArgs a) {
  typedef typename Elem<T>::raw raw;
  constexpr int N = Elem<T>::PER;
  const int d = threadIdx.x % LR * N, heads = a.H[0] + a.H[1];
  const int h0 = blockIdx.y * a.hchunk, h1 = min(h0 + a.hchunk, heads);
  NormCols<T, AL> c;
  c.init(a, d);
  const float inv_d = 1.f / a.dh;
  for (long t = (long)blockIdx.x * (256 / LR) + threadIdx.x / LR; t < a.tokens; t += (long)gridDim.x * (256 / LR)) {
    auto row = [&](int h) { return h < a.H[0] ? (const raw*)a.x[0] + t * a.x_row[0] + h * a.x_head[0] : (const raw*)a.x[1] + t * a.x_row[1] + (h - a.H[0]) * a.x_head[1]; };
    uint4 next = load_row_piece<T, AL>(row(h0), d, a.dh);
    float cs[N / 2], sn[N / 2];
    const double pos = a.positions ? a.positions[t] : (double)t;
#pragma unroll
    for (int j = 0; j < N / 2; ++j) turn_cos_sin(pos * c.rate[j], cs[j], sn[j]);
    for (int h = h0; h < h1; ++h) {
      Lane<T> x;
      x.from(cut_piece<T, AL>(next, d, a.dh));
      if (h + 1 < h1) next = load_row_piece<T, AL>(row(h + 1), d, a.dh);
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) sum = fmaf(x.v[i], x.v[i], sum);
#pragma unroll
      for (int k = 1; k < LR; k <<= 1) sum += __shfl_xor(sum, k, 64);
      const float r = 1.f / sqrtf(fmaf(sum, inv_d, a.eps));
      const int k = h >= a.H[0];
      float y[N];
#pragma unroll
      for (int j = 0; j < N / 2; ++j) {
        const float u = x.v[2 * j] * r * c.w[k][2 * j], v = x.v[2 * j + 1] * r * c.w[k][2 * j + 1];
        y[2 * j] = u * cs[j] - v * sn[j];
        y[2 * j + 1] = u * sn[j] + v * cs[j];
      }
      raw* out = k ? (raw*)a.y[1] + t * a.y_row[1] + (h - a.H[0]) * a.y_head[1] : (raw*)a.y[0] + t * a.y_row[0] + h * a.y_head[0];
      store_piece<T, AL>(out, d, a.dh, y);
    }
  }
}

template <typename T, int LR, int AL>
__global__ __launch_bounds__(256) void qk_norm_rope_bwd_kernel(QkNormArgs a) {
  typedef typename Elem<T>::raw raw;
  constexpr int N = Elem<T>::PER, NG = 256 / LR;
  __shared__ float part[2][NG][LR * N + 1];
  const int d = threadIdx.x % LR * N, grp = threadIdx.x / LR, heads = a.H[0] + a.H[1];
  const int h0 = blockIdx.y * a.hchunk, h1 = min(h0 + a.hchunk, heads);
  NormCols<T, AL> c;
  c.init(a, d);
  const float inv_d = 1.f / a.dh;
  float dw[2][N];
#pragma unroll
  for (int i = 0; i < N; ++i) dw[0][i] = dw[1][i] = 0.f;
  for (long t = (long)blockIdx.x * NG + grp; t < a.tokens; t += (long)gridDim.x * NG) {
    auto row = [&](int h) { return h < a.H[0] ? (const raw*)a.x[0] + t * a.x_row[0] + h * a.x_head[0] : (const raw*)a.x[1] + t * a.x_row[1] + (h - a.H[0]) * a.x_head[1]; };
    auto drow = [&](int h) { return h < a.H[0] ? (const raw*)a.dy[0] + t * a.y_row[0] + h * a.y_head[0] : (const raw*)a.dy[1] + t * a.y_row[1] + (h - a.H[0]) * a.y_head[1]; };
    uint4 nx = load_row_piece<T, AL>(row(h0), d, a.dh), nd = load_row_piece<T, AL>(drow(h0), d, a.dh);
    float cs[N / 2], sn[N / 2];
    const double pos = a.positions ? a.positions[t] : (double)t;
#pragma unroll
    for (int j = 0; j < N / 2; ++j) turn_cos_sin(pos * c.rate[j], cs[j], sn[j]);
    for (int h = h0; h < h1; ++h) {
      Lane<T> x, dy;
      x.from(cut_piece<T, AL>(nx, d, a.dh));
      dy.from(cut_piece<T, AL>(nd, d, a.dh));
      if (h + 1 < h1) {
        nx = load_row_piece<T, AL>(row(h + 1), d, a.dh);
        nd = load_row_piece<T, AL>(drow(h + 1), d, a.dh);
      }
      const bool k = h >= a.H[0];
      float dn[N], g[N], sum = 0.f, dot = 0.f;
#pragma unroll
      for (int j = 0; j < N / 2; ++j) {
        dn[2 * j] = dy.v[2 * j] * cs[j] + dy.v[2 * j + 1] * sn[j];
        dn[2 * j + 1] = dy.v[2 * j + 1] * cs[j] - dy.v[2 * j] * sn[j];
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        g[i] = dn[i] * (k ? c.w[1][i] : c.w[0][i]);
        sum = fmaf(x.v[i], x.v[i], sum);
        dot = fmaf(g[i], x.v[i], dot);
      }
#pragma unroll
      for (int q = 1; q < LR; q <<= 1) {
        sum += __shfl_xor(sum, q, 64);
        dot += __shfl_xor(dot, q, 64);
      }
      const float r = 1.f / sqrtf(fmaf(sum, inv_d, a.eps)), coef = dot * inv_d * r * r;
      float dx[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        dx[i] = r * (g[i] - x.v[i] * coef);
        const float e = dn[i] * x.v[i] * r;
        dw[0][i] += k ? 0.f : e;
        dw[1][i] += k ? e : 0.f;
      }
      raw* out = k ? (raw*)a.dx[1] + t * a.x_row[1] + (h - a.H[0]) * a.x_head[1] : (raw*)a.dx[0] + t * a.x_row[0] + h * a.x_head[0];
      store_piece<T, AL>(out, d, a.dh, dx);
    }
  }
  // the work-group's sums in group order, then one row of partial sums per work-group
#pragma unroll
  for (int i = 0; i < N; ++i) {
    part[0][grp][d + i] = dw[0][i];
    part[1][grp][d + i] = dw[1][i];
  }
  __syncthreads();
  const long b = (long)blockIdx.y * gridDim.x + blockIdx.x;
  for (int i = threadIdx.x; i < 2 * a.dh; i += 256) {
    const int k = i / a.dh, col = i % a.dh;
    float s = 0.f;
    for (int q = 0; q < NG; ++q) s += part[k][q][col];
    a.part[b * 2 * a.dh + i] = s;
  }
}

// dw[k][col] = the work-groups' partial sums, 32 strands of them in order, then the strands in order
__global__ __launch_bounds__(256) void qk_norm_dw_kernel(const float* part, int blocks, int dh, float* dw0, float* dw1) {
  __shared__ float s[32][9];
  const int c = threadIdx.x & 7, q = threadIdx.x >> 3, i = blockIdx.x * 8 + c;
  float x = 0.f;
  if (i < 2 * dh) {
#pragma unroll 8
    for (int b = q; b < blocks; b += 32) x += part[(long)b * 2 * dh + i];
  }
  s[q][c] = x;
  __syncthreads();
  if (q == 0 && i < 2 * dh) {
    float t = 0.f;
#pragma unroll
    for (int j = 0; j < 32; ++j) t += s[j][c];
    float* dw = i < dh ? dw0 : dw1;
    if (dw) dw[i % dh] = t;
  }
}

// Lanes of a row: a power of two of 16-byte pieces
static int row_lanes(int dh, int bf16) {
  const int n = bf16 ? 8 : 4;
  int l = 8;
  while (l * n < dh) l *= 2;
  return l;
}
// Work-groups along the tokens, and heads a group of lanes walks.  All heads of a token by one group computes its angles once; with few tokens the
// heads are spread over more groups until the chip has 8 waves on every SIMD of a quarter of its CUs
QkNormGrid qk_norm_grid(long tokens, int heads, int dh, int bf16) {
  const int per = 256 / row_lanes(dh, bf16);
  QkNormGrid g;
  const long blocks = (tokens + per - 1) / per;
  g.x = (int)(blocks < 1024 ? blocks : 1024);
  int parts = (int)(1024 / g.x);
  parts = parts < 1 ? 1 : parts > heads ? heads : parts;
  g.hchunk = (heads + parts - 1) / parts;
  g.y = (heads + g.hchunk - 1) / g.hchunk;
  return g;
}

template <typename T, int LR, int AL>
static void launch_norm_al(const QkNormArgs& a, dim3 grid, bool backward, hipStream_t s) {
  if (backward)
    qk_norm_rope_bwd_kernel<T, LR, AL><<<grid, 256, 0, s>>>(a);
  else
    qk_norm_rope_fwd_kernel<T, LR, AL><<<grid, 256, 0, s>>>(a);
}
template <typename T, int LR>
static void launch_norm_lr(const QkNormArgs& a, int align, dim3 grid, bool backward, hipStream_t s) {
  if (align == 16) return launch_norm_al<T, LR, 16>(a, grid, backward, s);
  if constexpr (sizeof(T) == 2) {
    if (align == 8) return launch_norm_al<T, LR, 8>(a, grid, backward, s);
  }
  launch_norm_al<T, LR, sizeof(T)>(a, grid, backward, s);
}
void launch_qk_norm_rope(QkNormArgs a, int bf16, int align, bool backward, hipStream_t s) {
  const QkNormGrid g = qk_norm_grid(a.tokens, a.H[0] + a.H[1], a.dh, bf16);
  const dim3 grid(g.x, g.y);
  a.hchunk = g.hchunk;
  const int lr = row_lanes(a.dh, bf16);
  if (bf16) {
    if (lr == 8)
      launch_norm_lr<bf16_t, 8>(a, align, grid, backward, s);
    else if (lr == 16)
      launch_norm_lr<bf16_t, 16>(a, align, grid, backward, s);
    else
      launch_norm_lr<bf16_t, 32>(a, align, grid, backward, s);
  } else {
    if (lr == 8)
      launch_norm_lr<float, 8>(a, align, grid, backward, s);
    else if (lr == 16)
      launch_norm_lr<float, 16>(a, align, grid, backward, s);
    else if (lr == 32)
      launch_norm_lr<float, 32>(a, align, grid, backward, s);
    else
      launch_norm_lr<float, 64>(a, align, grid, backward, s);
  }
  if (backward && (a.dw[0] || a.dw[1])) qk_norm_dw_kernel<<<dim3((2 * a.dh + 7) / 8), 256, 0, s>>>(a.part, g.x * g.y, a.dh, a.dw[0], a.dw[1]);
}

}  // namespace sh
