// Launches of packed_few_body (packed_bodies.h): a few rows per sequence and kv head over many keys.
#include "packed_bodies.h"

namespace sh {

template <typename T, int DH, int AL>
__global__ __launch_bounds__(256, 1) void packed_few_kernel(PackedAttn a) {
  __shared__ __attribute__((aligned(16))) typename Elem<T>::raw fsm[packed_few_lds<T, DH>()];
  __shared__ float ms[4][PACKED_FEW], ls[4][PACKED_FEW];
  packed_few_body<T, DH, AL>(a, blockIdx.x, fsm, ms, ls);
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
