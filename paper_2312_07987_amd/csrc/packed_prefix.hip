// Sequences that share a prefix, where each has few rows: the prefix in tiles of the rows of all sequences, read once for all, and the sequences' own keys
// as parts of their own, both in one launch: the first work-groups take the prefix, the others the sequences (one after the other in two launches the
// smaller one leaves most of the chip idle: 64 single tokens over 4096 shared keys and up to 500 of their own 17 + 11 us,
// together 21).  Bound by the chain of key tiles that a wave walks, and for few rows by the prefix' bytes.
#include "packed_bodies.h"

namespace sh {

template <typename T, int DH, int AL, bool FEW>
__global__ __launch_bounds__(256, DH * sizeof(T) <= 256 ? 2 : 1) void packed_prefix_kernel(PackedAttn f, PackedAttn o, int flat_blocks) {
  typedef typename Elem<T>::raw raw;
  constexpr int A = packed_fwd_lds<T, DH, 1>(), B = FEW ? packed_few_lds<T, DH>() : 0;
  __shared__ __attribute__((aligned(16))) raw lds[A > B ? A : B];
  if ((int)blockIdx.x < flat_blocks) return packed_fwd_body<T, DH, AL, 1>(f, blockIdx.x, lds);
  if constexpr (FEW) {
    __shared__ float ms[4][PACKED_FEW], ls[4][PACKED_FEW];
    packed_few_body<T, DH, AL>(o, blockIdx.x - flat_blocks, lds, ms, ls);
  } else {
    packed_fwd_body<T, DH, AL, 1>(o, blockIdx.x - flat_blocks, lds);
  }
}

template <typename T, int DH, int AL>
static void launch_prefix_al(const PackedAttn& f, const PackedAttn& o, bool few, int flat, int own, hipStream_t s) {
  const dim3 grid((unsigned)(flat + own));
  if (few)
    packed_prefix_kernel<T, DH, AL, true><<<grid, 256, 0, s>>>(f, o, flat);
  else
    packed_prefix_kernel<T, DH, AL, false><<<grid, 256, 0, s>>>(f, o, flat);
}
template <typename T, int DH>
static void launch_prefix(const PackedAttn& f, const PackedAttn& o, bool few, int flat, int own, int align, hipStream_t s) {
  if (align == 16) return launch_prefix_al<T, DH, 16>(f, o, few, flat, own, s);
  if constexpr (sizeof(T) == 2) {
    if (align == 8) return launch_prefix_al<T, DH, 8>(f, o, few, flat, own, s);
  }
  launch_prefix_al<T, DH, sizeof(T)>(f, o, few, flat, own, s);
}
template <typename T>
static void launch_prefix_t(const PackedAttn& f, const PackedAttn& o, bool few, int flat, int own, int align, hipStream_t s) {
  if (f.dh <= 64)
    launch_prefix<T, 64>(f, o, few, flat, own, align, s);
  else if (f.dh <= 128)
    launch_prefix<T, 128>(f, o, few, flat, own, align, s);
  else
    launch_prefix<T, 256>(f, o, few, flat, own, align, s);
}
// f: the prefix (flat), o: the own keys, by packed_few_body or in tiles
void launch_packed_prefix(const PackedAttn& f, const PackedAttn& o, bool few, int bf16, int align, hipStream_t s) {
  const long rows = (long)f.total_q * f.G;
  const long flat = (rows + PACKED_BM - 1) / PACKED_BM * f.Hk * f.nsplit;
  const long slots = few ? (o.chunk ? packed_slots(o.total_k, o.chunk, o.nseq) : o.nseq) : (o.levels ? (long)o.levels * o.nseq : packed_slots(rows, PACKED_BM, o.nseq)) * o.nsplit;
  if (bf16)
    launch_prefix_t<bf16_t>(f, o, few, (int)flat, (int)(slots * o.Hk), align, s);
  else
    launch_prefix_t<float>(f, o, few, (int)flat, (int)(slots * o.Hk), align, s);
}

}  // namespace sh
