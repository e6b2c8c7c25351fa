// Norms of queries and keys for each head with the position rotation in the same pass:
//   n = x r w,  r = (mean x^2 + eps)^(-1/2) over the head's d elements,  y = n with the pair (2 i, 2 i + 1) turned by
//   position * theta^(-2 i / rope_dim) for 2 i < rope_dim.
// Backward (r is computed again from x: keeping it would save nothing, x is read anyway):
//   dn = dy turned back,  dw = sum over rows of dn x r,  g = dn w,  dx = r (g - x r mean(g x r)).
//
// Bound by bytes: x (and dy) read once, y (dx) written once (16384 tokens, 40 heads of 128 in bf16: forward 72 us, 4.7 TB/s, backward 120, 4.2, as a large copy's 5.06).  A group of LR lanes holds a head's row in 16-byte pieces (the
// sums over it are a butterfly), takes one token and walks up to 16 of its heads, for which the token's sines and cosines are computed
// once: angles in 64 bits down to a fraction of a turn and a remainder, so positions of millions keep their place to the last bit of fp32.
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
  float w[N];
  double rate[N / 2];
  __device__ __forceinline__ void init(const QkNormArgs& a, int side, int d) {
    Lane<T> l;
    const typename Elem<T>::raw* w_ = (const typename Elem<T>::raw*)a.w[side];
    if (w_) l.from(lane_piece<T, AL>(w_, d, a.dh));
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = w_ ? l.v[i] : 1.f;
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

// blockIdx.y: a range of hchunk heads of the queries, then of the keys
template <typename T, int LR, int AL>
__global__ __launch_bounds__(256) void qk_norm_rope_fwd_kernel(QkNormArgs a) {
  typedef typename Elem<T>::raw raw;
  constexpr int N = Elem<T>::PER;
  const int d = threadIdx.x % LR * N, yq = (a.H[0] + a.hchunk - 1) / a.hchunk, side = (int)blockIdx.y >= yq;
  const int h0 = (blockIdx.y - (side ? yq : 0)) * a.hchunk, h1 = min(h0 + a.hchunk, a.H[side]);
  const long xh = a.x_head[side], yh = a.y_head[side];
  NormCols<T, AL> c;
  c.init(a, side, d);
  const float inv_d = 1.f / a.dh;
  for (long t = (long)blockIdx.x * (256 / LR) + threadIdx.x / LR; t < a.tokens; t += (long)gridDim.x * (256 / LR)) {
    const raw* x_ = (const raw*)a.x[side] + t * a.x_row[side] + h0 * xh;
    raw* y_ = (raw*)a.y[side] + t * a.y_row[side] + h0 * yh;
    uint4 next = load_row_piece<T, AL>(x_, d, a.dh);
    float cs[N / 2], sn[N / 2];
    const double pos = a.positions ? a.positions[t] : (double)t;
    if (a.gaps && pos < 0.) continue;
#pragma unroll
    for (int j = 0; j < N / 2; ++j) turn_cos_sin(pos * c.rate[j], cs[j], sn[j]);
    for (int h = h0; h < h1; ++h, y_ += yh) {
      Lane<T> x;
      x.from(cut_piece<T, AL>(next, d, a.dh));
      x_ += xh;
      if (h + 1 < h1) next = load_row_piece<T, AL>(x_, d, a.dh);
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) sum = fmaf(x.v[i], x.v[i], sum);
#pragma unroll
      for (int k = 1; k < LR; k <<= 1) sum += __shfl_xor(sum, k, 64);
      const float r = a.norm ? 1.f / sqrtf(fmaf(sum, inv_d, a.eps)) : 1.f;
      float y[N];
#pragma unroll
      for (int j = 0; j < N / 2; ++j) {
        const float u = x.v[2 * j] * r * c.w[2 * j], v = x.v[2 * j + 1] * r * c.w[2 * j + 1];
        y[2 * j] = u * cs[j] - v * sn[j];
        y[2 * j + 1] = u * sn[j] + v * cs[j];
      }
      store_piece<T, AL>(y_, d, a.dh, y);
    }
  }
}

template <typename T, int LR, int AL>
__global__ __launch_bounds__(256) void qk_norm_rope_bwd_kernel(QkNormArgs a) {
  typedef typename Elem<T>::raw raw;
  constexpr int N = Elem<T>::PER, NG = 256 / LR;
  __shared__ float part[NG][LR * N + 1];
  const int d = threadIdx.x % LR * N, grp = threadIdx.x / LR, yq = (a.H[0] + a.hchunk - 1) / a.hchunk, side = (int)blockIdx.y >= yq;
  const int h0 = (blockIdx.y - (side ? yq : 0)) * a.hchunk, h1 = min(h0 + a.hchunk, a.H[side]);
  const long xh = a.x_head[side], yh = a.y_head[side];
  NormCols<T, AL> c;
  c.init(a, side, d);
  const float inv_d = 1.f / a.dh;
  float dw[N];
#pragma unroll
  for (int i = 0; i < N; ++i) dw[i] = 0.f;
  for (long t = (long)blockIdx.x * NG + grp; t < a.tokens; t += (long)gridDim.x * NG) {
    const raw* x_ = (const raw*)a.x[side] + t * a.x_row[side] + h0 * xh;
    raw* dx_ = (raw*)a.dx[side] + t * a.x_row[side] + h0 * xh;
    const raw* dy_ = (const raw*)a.dy[side] + t * a.y_row[side] + h0 * yh;
    uint4 nx = load_row_piece<T, AL>(x_, d, a.dh), nd = load_row_piece<T, AL>(dy_, d, a.dh);
    float cs[N / 2], sn[N / 2];
    const double pos = a.positions ? a.positions[t] : (double)t;
    if (a.gaps && pos < 0.) continue;
#pragma unroll
    for (int j = 0; j < N / 2; ++j) turn_cos_sin(pos * c.rate[j], cs[j], sn[j]);
    for (int h = h0; h < h1; ++h, dx_ += xh) {
      Lane<T> x, dy;
      x.from(cut_piece<T, AL>(nx, d, a.dh));
      dy.from(cut_piece<T, AL>(nd, d, a.dh));
      x_ += xh;
      dy_ += yh;
      if (h + 1 < h1) {
        nx = load_row_piece<T, AL>(x_, d, a.dh);
        nd = load_row_piece<T, AL>(dy_, d, a.dh);
      }
      float dn[N], g[N], sum = 0.f, dot = 0.f;
#pragma unroll
      for (int j = 0; j < N / 2; ++j) {
        dn[2 * j] = dy.v[2 * j] * cs[j] + dy.v[2 * j + 1] * sn[j];
        dn[2 * j + 1] = dy.v[2 * j + 1] * cs[j] - dy.v[2 * j] * sn[j];
      }
      if (!a.norm) {   // uniform
        store_piece<T, AL>(dx_, d, a.dh, dn);
        continue;
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        g[i] = dn[i] * c.w[i];
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
        dw[i] = fmaf(dn[i], x.v[i] * r, dw[i]);
      }
      store_piece<T, AL>(dx_, d, a.dh, dx);
    }
  }
  // the work-group's sums in group order, then one row of partial sums per work-group
#pragma unroll
  for (int i = 0; i < N; ++i) part[grp][d + i] = dw[i];
  __syncthreads();
  const long b = (long)blockIdx.y * gridDim.x + blockIdx.x;
  for (int i = threadIdx.x; i < a.dh; i += 256) {
    float s = 0.f;
    for (int q = 0; q < NG; ++q) s += part[q][i];
    a.part[b * a.dh + i] = s;
  }
}

// dw[k][col] = the work-groups' partial sums (yq rows of `blocks` for the queries, the rest for the keys), 32 strands of them in order, then the strands in order
__global__ __launch_bounds__(256) void qk_norm_dw_kernel(const float* part, int blocks, int yq, int yk, int dh, float* dw0, float* dw1) {
  __shared__ float s[32][9];
  const int c = threadIdx.x & 7, q = threadIdx.x >> 3, k = blockIdx.y, i = blockIdx.x * 8 + c;
  const int n = blocks * (k ? yk : yq);
  const float* p = part + (long)(k ? yq : 0) * blocks * dh;
  float x = 0.f;
  if (i < dh) {
#pragma unroll 8
    for (int b = q; b < n; b += 32) x += p[(long)b * dh + i];
  }
  s[q][c] = x;
  __syncthreads();
  if (q == 0 && i < dh) {
    float t = 0.f;
#pragma unroll
    for (int j = 0; j < 32; ++j) t += s[j][c];
    float* dw = k ? dw1 : dw0;
    if (dw) dw[i] = t;
  }
}

// Lanes of a row: a power of two of 16-byte pieces
static int row_lanes(int dh, int bf16) {
  const int n = bf16 ? 8 : 4;
  int l = 8;
  while (l * n < dh) l *= 2;
  return l;
}
// Work-groups along the tokens, and heads that a group of lanes walks (of one side: its columns' weights and sums are then one register each).  A
// group's angles serve its heads, so it takes 16 of them, fewer where there are few tokens (some 2048 work-groups: 8 waves on every SIMD).
QkNormGrid qk_norm_grid(long tokens, int H0, int H1, int dh, int bf16) {
  const int per = 256 / row_lanes(dh, bf16);
  QkNormGrid g;
  const long blocks = (tokens + per - 1) / per;
  g.x = (int)(blocks < 1024 ? blocks : 1024);
  const int want = 2048 / g.x, heads = H0 + H1;
  g.hchunk = (heads + want - 1) / want;
  if (g.hchunk > 16) g.hchunk = 16;
  g.yq = (H0 + g.hchunk - 1) / g.hchunk;
  g.y = g.yq + (H1 + g.hchunk - 1) / g.hchunk;
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
  const QkNormGrid g = qk_norm_grid(a.tokens, a.H[0], a.H[1], a.dh, bf16);
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
  if (backward && (a.dw[0] || a.dw[1])) qk_norm_dw_kernel<<<dim3((a.dh + 7) / 8, 2), 256, 0, s>>>(a.part, g.x, g.yq, g.y - g.yq, a.dh, a.dw[0], a.dw[1]);
}

void launch_layer_norm_rope(QkNormArgs a, int bf16, bool backward, hipStream_t s) {
  for (int k = 0; k < 7; ++k) a.rate[k] = a.rope_dim ? pow(10000., -2. * (1 << k) / a.rope_dim) : 0.;
  const int esz = bf16 ? 2 : 4;
  const unsigned long bits = (unsigned long)a.dh * esz | (unsigned long)(uintptr_t)a.w[0];   // (the workspace's rows begin at multiples of 256)
  launch_qk_norm_rope(a, bf16, bits % 16 == 0 ? 16 : bf16 && bits % 8 == 0 ? 8 : esz, backward, s);
}
size_t packed_norm_bytes(long tokens, int heads, int dh, int bf16) {
  const QkNormGrid g = qk_norm_grid(tokens, heads, 0, dh, bf16);
  return (size_t)g.x * g.y * dh * 4;
}

// The place of row q in its sequence, -1 if it belongs to none
__device__ __forceinline__ int place_in_sequence(const int* offsets, int nseq, int max_len, int q) {
  int lo = 0, hi = nseq;   // the last sequence that begins at or before q
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (offsets[mid] <= q)
      lo = mid;
    else
      hi = mid;
  }
  const int beg = max(offsets[lo], 0);
  return q >= beg && q < offsets[lo + 1] && q - beg < max_len ? q - beg : -1;
}

__global__ __launch_bounds__(256) void packed_positions_kernel(const int* offsets, int nseq, int max_len, int T, int prefix, int* pos) {
  const int row = blockIdx.x * 256 + threadIdx.x;
  if (row >= T) return;
  const int at = row < prefix ? -1 : place_in_sequence(offsets, nseq, max_len, row - prefix);
  pos[row] = row < prefix ? row : at < 0 ? -1 : prefix + at;
}

// zeros in the rows of up to three tensors that belong to no sequence: a wave per row
__global__ __launch_bounds__(256) void packed_clear_kernel(const int* offsets, int nseq, int max_len, int rows, int shorts, unsigned short* p0, unsigned short* p1, unsigned short* p2) {
  const int row = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= rows || place_in_sequence(offsets, nseq, max_len, row) >= 0) return;
  for (int i = threadIdx.x & 63; i < shorts; i += 64) {
    const long at = (long)row * shorts + i;
    if (p0) p0[at] = 0;
    if (p1) p1[at] = 0;
    if (p2) p2[at] = 0;
  }
}
void launch_packed_clear(const int* offsets, int nseq, int max_len, int rows, int row_bytes, void* p0, void* p1, void* p2, hipStream_t s) {
  packed_clear_kernel<<<dim3((rows + 3) / 4), 256, 0, s>>>(offsets, nseq, max_len, rows, row_bytes / 2, (unsigned short*)p0, (unsigned short*)p1, (unsigned short*)p2);
}
void launch_packed_positions(const int* offsets, int nseq, int max_len, int T, int prefix, int* pos, hipStream_t s) {
  packed_positions_kernel<<<dim3((T + 255) / 256), 256, 0, s>>>(offsets, nseq, max_len, T, prefix, pos);
}

}  // namespace sh
