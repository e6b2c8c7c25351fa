// C ABI of the operators beside the layer (include/switchhead.h): argument checks, the choice of kernels and of how the keys are split,
// workspace carving and launches.  Nothing here allocates or synchronises.
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <initializer_list>

#include "../../include/switchhead.h"
#include "packed_attn.h"

using namespace sh;

namespace {

sh_status fail(sh_status code, const char* fmt, ...) {
  char text[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(text, sizeof text, fmt, ap);
  va_end(ap);
  return (sh_status)report(code, text);
}

sh_status check_launch(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(SH_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return SH_OK;
}

size_t align_up(size_t v) { return (v + 255) & ~(size_t)255; }
long ceil_div(long a, long b) { return (a + b - 1) / b; }

// The largest of 16, 8 and the element's size that divides every address and every stride: how rows are read and written
int alignment(std::initializer_list<const void*> ptrs, std::initializer_list<int64_t> strides, int dh, int esz) {
  uint64_t bits = (uint64_t)dh * esz;
  for (const void* p : ptrs) bits |= (uint64_t)(uintptr_t)p;
  for (int64_t s : strides) bits |= (uint64_t)s * esz;
  return bits % 16 == 0 ? 16 : (esz == 2 && bits % 8 == 0) ? 8 : esz;
}
bool elements_aligned(std::initializer_list<const void*> ptrs, int esz) {
  for (const void* p : ptrs)
    if ((uintptr_t)p % esz) return false;
  return true;
}

bool any_same(std::initializer_list<const void*> outs, std::initializer_list<const void*> ins) {
  for (const void* o : outs)
    for (const void* i : ins)
      if (o && o == i) return true;
  return false;
}

// Rows of a tensor [rows, heads, d] in memory: dense where the strides are 0.  Limits: a tile's rows are addressed by 32-bit byte offsets.
bool fill_strides(int64_t& row, int64_t& head, int64_t heads, int64_t d) {
  if (row < 0 || head < 0) return false;
  if (head == 0) head = d;
  if (row == 0) row = heads * head;
  return row < (1ll << 23) && head < (1ll << 40);
}
// ... an output's rows must not lie over each other
bool disjoint(int64_t rows, int64_t heads, int64_t row, int64_t head, int64_t d) {
  const bool by_row = (heads == 1 || head >= d) && (rows <= 1 || row >= (heads - 1) * head + d);
  const bool by_head = (rows <= 1 || row >= d) && (heads == 1 || head >= (rows - 1) * row + d);
  return by_row || by_head;
}

// ---- attention ------------------------------------------------------------------------------------------------------------
struct AttnPlan {
  sh_attention a;             // strides filled in
  int G, esz;
  bool few, two_parts;        // few rows per sequence: packed_few.hip; the prefix as a part of its own, for the rows of all sequences together
  int chunk, nsplit, nflat;   // keys of a few-row work-group (0: all); key ranges of the own keys and of the prefix
  int groups, tall;           // wave groups of a tile's work-group; tiles of 256 rows
  int levels, levels128, klevels;   // levels of the row tiles (the forward's, the backward's) and of the key tiles, 0: by slot
  int dhp;
  size_t po, pl, fo, fl, total;
};

constexpr double MAX_THREADS = 4294967296.;   // of a launch

// (the sizes that 32-bit row arithmetic and 24-bit reciprocals cover)
sh_status plan_attention(AttnPlan& p, const sh_attention* d) {
  if (!d) return fail(SH_ERR_INVALID_ARG, "the attention's description is NULL");
  p.a = *d;
  sh_attention& a = p.a;
  if (a.nseq < 0 || a.total_q < 0 || a.total_k < 0 || a.max_q < 0 || a.max_k < 0 || a.prefix < 0)
    return fail(SH_ERR_INVALID_ARG, "negative size (nseq=%d total_q=%d total_k=%d max_q=%d max_k=%d prefix=%d)", a.nseq, a.total_q, a.total_k,
                a.max_q, a.max_k, a.prefix);
  if (a.nheads < 1 || a.nkv_heads < 1 || a.d_head < 1)
    return fail(SH_ERR_INVALID_ARG, "nheads, nkv_heads and d_head must be >= 1 (%d, %d, %d)", a.nheads, a.nkv_heads, a.d_head);
  if (a.nheads % a.nkv_heads) return fail(SH_ERR_INVALID_ARG, "nheads=%d is no multiple of nkv_heads=%d", a.nheads, a.nkv_heads);
  if (a.causal != 0 && a.causal != 1) return fail(SH_ERR_INVALID_ARG, "causal must be 0 or 1");
  if (a.dtype != SH_F32 && a.dtype != SH_BF16) return fail(SH_ERR_INVALID_ARG, "unknown dtype %d", a.dtype);
  if (!(a.scale >= 0.f) || !std::isfinite(a.scale)) return fail(SH_ERR_INVALID_ARG, "scale must be positive and finite, or 0 for 1 / sqrt(d_head)");
  if (a.d_head > 256) return fail(SH_ERR_UNSUPPORTED, "d_head=%d exceeds the limit of 256", a.d_head);
  if (a.nheads > 4096) return fail(SH_ERR_UNSUPPORTED, "nheads=%d exceeds the limit of 4096", a.nheads);
  if (a.scale == 0.f) a.scale = 1.0f / sqrtf((float)a.d_head);
  p.G = a.nheads / a.nkv_heads;
  p.esz = a.dtype == SH_BF16 ? 2 : 4;
  if (a.max_q > a.total_q) a.max_q = a.total_q;
  if (a.max_k > a.total_k) a.max_k = a.total_k;
  if (!fill_strides(a.q_row, a.q_head, a.nheads, a.d_head) || !fill_strides(a.k_row, a.k_head, a.nkv_heads, a.d_head) ||
      !fill_strides(a.v_row, a.v_head, a.nkv_heads, a.d_head) || !fill_strides(a.o_row, a.o_head, a.nheads, a.d_head) ||
      !fill_strides(a.kp_row, a.kp_head, a.nkv_heads, a.d_head) || !fill_strides(a.vp_row, a.vp_head, a.nkv_heads, a.d_head))
    return fail(SH_ERR_UNSUPPORTED, "strides must not be negative, row strides must stay below 2^23 and head strides below 2^40 elements");
  if (!disjoint(a.total_q, a.nheads, a.o_row, a.o_head, a.d_head)) return fail(SH_ERR_INVALID_ARG, "the strides of O lay rows over each other");
  const long G = p.G, rows = (long)a.total_q * G, most = (long)a.max_q * G;
  if ((long)a.total_q * a.nheads >= (1l << 31) || (long)a.total_k * G >= (1l << 31) - 128 * G || most * G >= (1l << 32) || a.nseq >= (1 << 24))
    return fail(SH_ERR_UNSUPPORTED, "too large: total_q * nheads and total_k * group must stay below 2^31, max_q * group^2 below 2^32, nseq below 2^24");
  if (a.prefix >= 1 << 30) return fail(SH_ERR_UNSUPPORTED, "prefix=%d: must stay below 2^30", a.prefix);

  p.dhp = (a.d_head + 3) / 4 * 4;
  p.few = most <= PACKED_FEW;
  p.two_parts = false;
  p.chunk = 0;
  p.nsplit = p.nflat = 0;
  p.groups = 1;
  p.tall = 0;
  // levels where their grid is at most twice that of slots, or small: 16 sequences of 512 tokens 25.3 us by slots, 19.4 by levels; 3 of 4096 104 and 84
  auto levels = [&](long most, long all, int tile) {
    const long n = ceil_div(most, tile);
    return a.causal && n * a.nseq <= 2 * packed_slots(all, tile, a.nseq) + 1024 / a.nkv_heads ? (int)n : 0;
  };
  p.levels = p.levels128 = levels(most, rows, PACKED_BM);
  p.klevels = levels(a.max_k, a.total_k, PACKED_KB);
  const long seqs = a.nseq > 0 ? a.nseq : 1;
  // A prefix: either every sequence's tiles walk it ahead of their own keys, or the rows of all sequences go into common tiles over it and
  // the own keys are a second part.  The second saves what the first wastes in tiles that rows of one sequence do not fill (a sequence's last tile is
  // half full on average), times the prefix, and pays for writing and joining two fp32 parts per row, about as long as 900 keys of a tile.
  // Alone / in common, us, 4 heads of 128: 2048 shared keys, 64 sequences of 30 rows 44.1 / 33.8, of 100 rows 51 / 80; 500 shared keys (32 heads over 8),
  // 64 sequences of 64 rows 34 / 43, of 4 rows 155 / 47 (4096 shared).
  if (a.prefix > 0) {
    const double tiles = std::fmin(std::fmax((double)seqs, rows / 128. + 0.5 * seqs), (double)ceil_div(most, PACKED_BM) * seqs);
    p.two_parts = (p.few || a.prefix * (128. * tiles - rows) > 900. * rows) && rows * G < (1l << 32) && 64. * a.total_q * a.nheads < MAX_THREADS;
    if (!p.two_parts) p.few = false;
  }
  const int kt = (a.d_head <= 64 || (p.esz == 2 && a.d_head <= 128)) ? 64 : 32;
  if (p.few) {
    // Chunks that make some 1500 work-groups of the keys there are, of 512 keys or more where that makes 512 of them; where a sequence's keys are few, one
    // work-group takes them all.  Chunks of 256 / 512: a token of 8192 keys, 32 heads over 8 (128 work-groups of 512) 14.2 / 16.8 us; 8 tokens of 32768 keys, 8
    // heads over 1 (512) 35.9 / 30.3.  Unsplit, 32 tokens of 2000 .. 32768 keys take 428 instead of 317, 64 of 4000 each 185 instead of 197.
    const long keys = (long)a.max_k * seqs < a.total_k ? (long)a.max_k * seqs : a.total_k;
    const long least = keys * a.nkv_heads >= 512 * 512 ? 512 : 256;
    long chunk = ceil_div(keys * a.nkv_heads, 1536);
    chunk = ceil_div(chunk < least ? least : chunk > 1024 ? 1024 : chunk, 128) * 128;
    if (a.max_k > 2 * chunk || (a.max_k > chunk && seqs * a.nkv_heads < 256)) p.chunk = (int)chunk;
  } else {
    const long tiles = (rows / PACKED_BM + seqs) * a.nkv_heads;
    const long kts = ceil_div((long)(p.two_parts ? 0 : a.prefix) + a.max_k, kt);
    // Two wave groups where there is less than one round of work-groups, and tiles of keys for both.  One / two: 4 sequences of 2048 tokens, 4 heads, 62 / 49 us
    // (272 tiles); 64 of 512 tokens, 4 heads, 48 / 65 (1280).
    p.groups = a.d_head <= 128 && kts >= 8 && tiles < 1024 && !p.two_parts ? 2 : 1;
    // 256-row tiles, one work-group per CU, for long rows of keys and three rounds of work-groups or more: 8192 tokens, 32 heads over 8 (1024 tiles) 623 -> 596 us, 2
    // of them, 16 heads 632 -> 603, 3 of 4096, 20 heads over 4 (960) 310 -> 302; but 16 of 2048, 8 heads (1024) 186 -> 198, and 8192 tokens, 20 heads over 4
    // (640 tiles, whose last round is half empty) 404 -> 414.
    if (!p.two_parts && p.esz == 2 && a.d_head > 96 && a.d_head <= 128 && (long)a.prefix + a.max_k >= 4096 && most >= 4096 &&
        ceil_div(rows, PACKED_BM2) * a.nkv_heads >= 768) {
      p.tall = 1;
      p.groups = 1;
      p.levels = levels(most, rows, PACKED_BM2);
    }
    // Few tiles and many keys: several work-groups share a tile's keys, some 512 in all (256 of two wave groups) with 8 tiles of keys each or more.  17 queries over 8000 keys, 4
    // heads, 141 us unsplit, 23 split; 512, 300, 64 over 2500, 300, 4000 77 and 28 (36 with half as many parts).
    long ns = 512 / p.groups / tiles;
    if (ns > kts / 8) ns = kts / 8;
    if (ns > 32) ns = 32;
    p.nsplit = !p.tall && (ns >= 2 || p.two_parts) ? (int)(ns > 0 ? ns : 1) : 0;
  }
  if (p.two_parts) {
    const long tiles = ceil_div(rows, PACKED_BM) * a.nkv_heads, kts = ceil_div(a.prefix, kt);
    // Some 256 work-groups beside those of the own keys; more parts cost more to join than they save: 64 tokens behind 4096 shared keys, 32 heads over 8, 29 us with 256,
    // 38 with 512; 64 times 4 behind 8192 78 and 71, 131 with 128.
    long ns = 256 / (tiles > 0 ? tiles : 1);
    if (ns > kts / 2) ns = kts / 2;
    if (ns > 32) ns = 32;
    p.nflat = (int)(ns < 1 ? 1 : ns);
  }
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += align_up(bytes);
    return o;
  };
  const size_t dense = (size_t)(p.nsplit + p.nflat) * a.total_q * a.nheads;
  p.po = take(dense * p.dhp * 4);
  p.pl = take(dense * 4);
  p.fo = p.fl = 0;
  if (p.few && (p.chunk || p.two_parts)) {
    const size_t slots = (size_t)(p.chunk ? packed_slots(a.total_k, p.chunk, a.nseq) : a.nseq) * a.nkv_heads * most;
    p.fo = take(slots * p.dhp * 4);
    p.fl = take(slots * 4);
  }
  p.total = off > 256 ? off : 256;
  // (a launch has less than 2^32 threads)
  const long nqs = p.levels ? (long)p.levels * a.nseq : packed_slots(rows, p.tall ? PACKED_BM2 : PACKED_BM, a.nseq);
  const double own = p.few ? 256. * (p.chunk ? packed_slots(a.total_k, p.chunk, a.nseq) : a.nseq) : (p.tall || p.groups == 2 ? 512. : 256.) * nqs * (p.nsplit > 0 ? p.nsplit : 1);
  const double flat = p.two_parts ? 256. * ceil_div(rows, PACKED_BM) * p.nflat : 0.;
  if ((own + flat) * a.nkv_heads >= MAX_THREADS || ((p.nsplit || p.nflat || p.chunk) && 64. * a.total_q * a.nheads >= MAX_THREADS))
    return fail(SH_ERR_UNSUPPORTED, "too large: the work-groups of nseq=%d, total_q=%d, total_k=%d, nheads=%d do not fit one launch", a.nseq, a.total_q, a.total_k, a.nheads);
  return SH_OK;
}

// Workspace of a backward pass: delta, the parts of dK and dV, and the score gradients where they are kept
struct BwdPlan {
  size_t dkv, ds, total;   // ds 0: not kept
  int rchunk, rparts;
  long ds_ld, dkv_floats;
  double threads;          // of its largest launch
};
// Kept score gradients, for heads of 65 .. 128 elements, in up to 2 GiB.  A backward pass with them / with scores worked out again for dQ, us, 16 heads over 4 and
// over 16:
//   d    32 x 256 tokens        4 x 2048                 1 x 8192                   4096 and 20 of 300
//   128  94 / 113, 128 / 139    353 / 380, 333 / 320     1287 / 1381, 1007 / 1030   597 / 663, 381 / 420
//   96   79 / 87,  118 / 124    292 / 311, 298 / 267     1060 / 1124, 889 / 827     490 / 527, 343 / 333
//   76   78 / 84,  122 / 134    314 / 334, 315 / 289     1162 / 1227, 959 / 882     547 / 584, 365 / 371
//   64   66 / 68,   90 / 89     248 / 239, 232 / 194      932 / 857,  752 / 608     423 / 426, 295 / 269
//   32   56 / 54,   75 / 74     222 / 207, 221 / 160      848 / 748,  728 / 495     376 / 384, 267 / 228
// A pair of query and key costs its two bytes there and back whatever the width, but 8 d operations again: below 65 those are the cheaper ones.  The limit is
// for the memory, which is laid out for the longest sequence: 4 x 4096 tokens of 32 heads of 128 over 8 would take 4 GiB for 2049 us against 2175.
constexpr size_t MAX_DS_BYTES = (size_t)2 << 30;
BwdPlan plan_backward(const AttnPlan& p) {
  const sh_attention& a = p.a;
  BwdPlan b{};
  const long rows = (long)a.max_q * p.G, w = packed_width(a.d_head);
  size_t off = align_up((size_t)a.total_q * a.nheads * 4) + 256;
  b.rchunk = (int)(rows > 0 ? ceil_div(rows, PACKED_QT) * PACKED_QT : PACKED_QT);
  b.rparts = 1;
  if (a.dtype == SH_BF16 && a.d_head <= 128 && rows > 0) {
    // Rows of a dK / dV work-group: what a CU would get if every key tile were seen by the longest rows there are.  Parts cost their writing and a second
    // kernel, so they are for launches with a few tiles far longer than the rest.  Forward and backward with 100 / 50 / 35 / 20 per cent of this and without parts, us: 6600
    // tokens of 20 heads of 80 over 4, longest 4096, 598 / 630 / 622 / 639 and 745; 4096 tokens of 8 heads of 128 over 2 308 / 321 / 326 / 345 and 646; 16384 tokens of 4
    // heads of 128, longest 4096 (no parts at 100 and 50 per cent, whose ranges hold all rows) 305 / 306 / 328 / 340 and 307.  At least 512, where a work-group is about as
    // long as its start and the extra parts.
    const long tiles = ceil_div(a.total_k, PACKED_KB) * a.nkv_heads;
    long chunk = tiles * rows / 256;
    chunk = ceil_div(chunk < 512 ? 512 : chunk, PACKED_QT) * PACKED_QT;
    if (chunk < rows) {
      b.rparts = (int)ceil_div(rows, chunk);
      b.rchunk = (int)(ceil_div(ceil_div(rows, b.rparts), PACKED_QT) * PACKED_QT);
      b.rparts = (int)ceil_div(rows, b.rchunk);
    }
    if (b.rparts > 1) {
      b.dkv = off;
      b.dkv_floats = 2l * PACKED_KB * w;
      off += align_up((size_t)b.rparts * packed_slots(a.total_k, PACKED_KB, a.nseq) * a.nkv_heads * b.dkv_floats * 4);
    }
    b.ds_ld = ceil_div(rows, PACKED_BM) * PACKED_BM;
    const size_t ds = (size_t)a.nkv_heads * a.total_k * b.ds_ld * 2;
    if (a.d_head > 64 && ds > 0 && ds <= MAX_DS_BYTES) {
      b.ds = off;
      off += align_up(ds);
    }
  }
  const double kb = p.klevels ? (double)p.klevels * a.nseq : packed_slots(a.total_k, PACKED_KB, a.nseq);
  const double qb = p.levels128 ? (double)p.levels128 * a.nseq : packed_slots((long)a.total_q * p.G, PACKED_BM, a.nseq);
  b.threads = 512. * std::fmax(kb * b.rparts, std::fmax((double)packed_slots(a.total_k, PACKED_KB, a.nseq), qb)) * a.nkv_heads;
  b.threads = std::fmax(b.threads, (double)packed_delta_lanes(a.d_head, p.esz) * a.total_q * a.nheads + 256.);
  b.total = off;
  return b;
}

sh_status check_workspace(const void* ws, size_t have, size_t need) {
  if (!ws) return fail(SH_ERR_INVALID_ARG, "workspace is NULL");
  if (((uintptr_t)ws & 255) != 0) return fail(SH_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  if (have < need) return fail(SH_ERR_WORKSPACE_TOO_SMALL, "workspace has %zu bytes, %zu needed", have, need);
  return SH_OK;
}

PackedAttn packed_args(const AttnPlan& p, const int32_t* qoff, const int32_t* qlen, const int32_t* koff, const int32_t* klen) {
  const sh_attention& d = p.a;
  PackedAttn a{};
  a.qoff = qoff;
  a.qlen = qlen;
  a.koff = koff;
  a.klen = klen;
  a.nseq = d.nseq;
  a.H = d.nheads;
  a.Hk = d.nkv_heads;
  a.G = p.G;
  a.g_inv = p.G > 1 ? 0xFFFFFFFFu / (unsigned)p.G + 1u : 0u;
  a.dh = d.d_head;
  a.causal = d.causal;
  a.prefix = d.prefix;
  a.max_q = d.max_q;
  a.max_k = d.max_k;
  a.total_q = d.total_q;
  a.total_k = d.total_k;
  a.q_row = d.q_row;
  a.q_head = d.q_head;
  a.k_row = d.k_row;
  a.k_head = d.k_head;
  a.v_row = d.v_row;
  a.v_head = d.v_head;
  a.o_row = d.o_row;
  a.o_head = d.o_head;
  a.kp_row = d.kp_row;
  a.kp_head = d.kp_head;
  a.vp_row = d.vp_row;
  a.vp_head = d.vp_head;
  a.scale = d.scale;
  a.dhp = p.dhp;
  a.groups = p.groups;
  a.tall = p.tall;
  a.levels = p.levels;
  return a;
}

// ---- norms ----------------------------------------------------------------------------------------------------------------
// An output over its input: every element must lie where it lay (strides along one row or one head mean nothing)
bool same_places(int64_t tokens, int64_t heads, int64_t row0, int64_t head0, int64_t row1, int64_t head1) {
  return (tokens <= 1 || row0 == row1) && (heads <= 1 || head0 == head1);
}
sh_status plan_norm(sh_qk_norm& a, const sh_qk_norm* d) {
  if (!d) return fail(SH_ERR_INVALID_ARG, "the norms' description is NULL");
  a = *d;
  if (a.tokens < 0 || a.nheads < 1 || a.nkv_heads < 0 || a.d_head < 1)
    return fail(SH_ERR_INVALID_ARG, "tokens and nkv_heads must be >= 0, nheads and d_head >= 1 (%d, %d, %d, %d)", a.tokens, a.nkv_heads, a.nheads, a.d_head);
  if (a.rope_dim < 0 || a.rope_dim % 2 || a.rope_dim > a.d_head)
    return fail(SH_ERR_INVALID_ARG, "rope_dim=%d must be even and lie in 0..d_head=%d", a.rope_dim, a.d_head);
  if (a.dtype != SH_F32 && a.dtype != SH_BF16) return fail(SH_ERR_INVALID_ARG, "unknown dtype %d", a.dtype);
  if (!(a.eps >= 0.f) || !std::isfinite(a.eps)) return fail(SH_ERR_INVALID_ARG, "eps must be finite and >= 0");
  if (!(a.theta >= 0.f) || !std::isfinite(a.theta)) return fail(SH_ERR_INVALID_ARG, "theta must be positive and finite, or 0 for 10000");
  if (a.d_head > 256) return fail(SH_ERR_UNSUPPORTED, "d_head=%d exceeds the limit of 256", a.d_head);
  if (a.nheads > 4096 || a.nkv_heads > 4096) return fail(SH_ERR_UNSUPPORTED, "more than 4096 heads");
  if (a.theta == 0.f) a.theta = 10000.f;
  if (!fill_strides(a.q_row, a.q_head, a.nheads, a.d_head) || !fill_strides(a.k_row, a.k_head, a.nkv_heads, a.d_head) ||
      !fill_strides(a.yq_row, a.yq_head, a.nheads, a.d_head) || !fill_strides(a.yk_row, a.yk_head, a.nkv_heads, a.d_head))
    return fail(SH_ERR_UNSUPPORTED, "strides must not be negative, row strides must stay below 2^23 and head strides below 2^40 elements");
  return SH_OK;
}

QkNormArgs norm_args(const sh_qk_norm& a, const void* Q, const void* K, const void* w_Q, const void* w_K, const int32_t* positions) {
  QkNormArgs n{};
  n.x[0] = Q;
  n.x[1] = K;
  n.w[0] = w_Q;
  n.w[1] = w_K;
  n.positions = positions;
  n.tokens = a.tokens;
  n.x_row[0] = a.q_row;
  n.x_row[1] = a.k_row;
  n.x_head[0] = a.q_head;
  n.x_head[1] = a.k_head;
  n.y_row[0] = a.yq_row;
  n.y_row[1] = a.yk_row;
  n.y_head[0] = a.yq_head;
  n.y_head[1] = a.yk_head;
  n.H[0] = a.nheads;
  n.H[1] = a.nkv_heads;
  n.dh = a.d_head;
  n.rope_dim = a.rope_dim;
  n.eps = a.eps;
  n.norm = 1;
  for (int k = 0; k < 7; ++k) n.rate[k] = a.rope_dim ? pow((double)a.theta, -2.0 * (1 << k) / a.rope_dim) : 0.;
  return n;
}
size_t norm_bytes(const sh_qk_norm& a) {
  const QkNormGrid g = qk_norm_grid(a.tokens > 0 ? a.tokens : 1, a.nheads, a.nkv_heads, a.d_head, a.dtype == SH_BF16);
  return align_up((size_t)g.x * g.y * a.d_head * 4);
}

}  // namespace

extern "C" {

size_t switchhead_attention_workspace_bytes(const sh_attention* d, int32_t backward) {
  AttnPlan p;
  if (plan_attention(p, d) != SH_OK) return 0;
  const size_t b = backward ? plan_backward(p).total : 0;
  return b > p.total ? b : p.total;
}

sh_status switchhead_attention_forward(const sh_attention* d, const void* Q, const void* K, const void* V, const void* K_prefix, const void* V_prefix,
                                       const int32_t* q_offsets, const int32_t* q_lengths, const int32_t* k_offsets, const int32_t* k_lengths,
                                       void* O, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
  AttnPlan p;
  sh_status r = plan_attention(p, d);
  if (r != SH_OK) return r;
  const sh_attention& s = p.a;
  // (a tensor without rows may be NULL)
  if (((!Q || !O) && s.total_q) || ((!K || !V) && s.total_k) || !q_offsets || !k_offsets)
    return fail(SH_ERR_INVALID_ARG, "Q, K, V, O, q_offsets, k_offsets must not be NULL");
  if (s.prefix > 0 && (!K_prefix || !V_prefix)) return fail(SH_ERR_INVALID_ARG, "prefix=%d but K_prefix or V_prefix is NULL", s.prefix);
  if (!elements_aligned({Q, K, V, O, K_prefix, V_prefix}, p.esz) || !elements_aligned({lse, q_offsets, q_lengths, k_offsets, k_lengths}, 4))
    return fail(SH_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
  if ((r = check_workspace(workspace, workspace_bytes, p.total)) != SH_OK) return r;
  if (s.nseq == 0 || s.total_q == 0 || s.max_q == 0) return SH_OK;
  const void *const k = s.total_k ? K : nullptr, *const v = s.total_k ? V : nullptr, *const kp = s.prefix ? K_prefix : nullptr, *const vp = s.prefix ? V_prefix : nullptr;
  if (any_same({O}, {k, v, kp, vp})) return fail(SH_ERR_INVALID_ARG, "O lies over keys or values");
  const hipStream_t st = (hipStream_t)hip_stream;
  const int bf16 = s.dtype == SH_BF16;
  const int align = alignment({Q, K, V, O, K_prefix, V_prefix}, {s.q_row, s.q_head, s.k_row, s.k_head, s.v_row, s.v_head, s.o_row, s.o_head, s.kp_row, s.kp_head, s.vp_row, s.vp_head},
                              s.d_head, p.esz);
  PackedAttn a = packed_args(p, q_offsets, q_lengths, k_offsets, k_lengths);
  a.Q = Q;
  a.K = K;
  a.V = V;
  a.KP = K_prefix;
  a.VP = V_prefix;
  a.O = O;
  a.lse = lse;
  char* const ws = (char*)workspace;
  a.po = (float*)(ws + p.po);
  a.pl = (float*)(ws + p.pl);
  a.nparts = p.nsplit + p.nflat;
  a.frows = s.max_q * p.G;
  if (p.few) {
    a.chunk = p.chunk;
    if (p.chunk || p.two_parts) {
      a.fo = (float*)(ws + p.fo);
      a.fl = (float*)(ws + p.fl);
    }
  }
  PackedAttn t = a;   // in tiles: this launch's parts
  t.nsplit = p.nsplit;
  t.part0 = p.nflat;
  t.own = p.two_parts;
  if (p.two_parts) {
    prof_mark(st, "attention.prefix");
    PackedAttn f = a;
    f.flat = 1;
    f.nsplit = p.nflat;
    launch_packed_prefix(f, p.few ? a : t, p.few, bf16, align, st);
  } else if (p.few) {
    prof_mark(st, "attention.few");
    launch_packed_few(a, bf16, align, st);
  } else {
    prof_mark(st, "attention.tiles");
    launch_packed_fwd(t, bf16, align, st);
  }
  if (a.nparts || a.fo) {
    prof_mark(st, "attention.join");
    launch_packed_join(a, bf16, st);
  }
  prof_mark(st, nullptr);
  return check_launch("switchhead_attention_forward");
}

sh_status switchhead_attention_backward(const sh_attention* d, const void* Q, const void* K, const void* V, const void* O, const void* dO, const float* lse,
                                        const int32_t* q_offsets, const int32_t* q_lengths, const int32_t* k_offsets, const int32_t* k_lengths,
                                        void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes, void* hip_stream) {
  AttnPlan p;
  sh_status r = plan_attention(p, d);
  if (r != SH_OK) return r;
  const sh_attention& s = p.a;
  if (((!Q || !O || !dO || !lse || !dQ) && s.total_q) || ((!K || !V || !dK || !dV) && s.total_k) || !q_offsets || !k_offsets)
    return fail(SH_ERR_INVALID_ARG, "Q, K, V, O, dO, lse, dQ, dK, dV, q_offsets, k_offsets must not be NULL");
  if (s.prefix > 0) return fail(SH_ERR_UNSUPPORTED, "the backward pass takes no shared prefix");
  if (!elements_aligned({Q, K, V, O, dO, dQ, dK, dV}, p.esz) || !elements_aligned({lse, q_offsets, q_lengths, k_offsets, k_lengths}, 4))
    return fail(SH_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
  if (!disjoint(s.total_q, s.nheads, s.q_row, s.q_head, s.d_head) || !disjoint(s.total_k, s.nkv_heads, s.k_row, s.k_head, s.d_head) ||
      !disjoint(s.total_k, s.nkv_heads, s.v_row, s.v_head, s.d_head))
    return fail(SH_ERR_INVALID_ARG, "the strides of Q, K or V lay the rows of a gradient over each other");
  const BwdPlan w = plan_backward(p);
  if (w.threads >= MAX_THREADS)
    return fail(SH_ERR_UNSUPPORTED, "too large: the work-groups of nseq=%d, total_q=%d, total_k=%d, nheads=%d do not fit one launch", s.nseq, s.total_q, s.total_k, s.nheads);
  if ((r = check_workspace(workspace, workspace_bytes, w.total)) != SH_OK) return r;
  if (s.nseq == 0 || (s.total_q == 0 && s.total_k == 0)) return SH_OK;
  // dK and dV are written before dQ reads K (and, where score gradients are not kept, Q, V and dO), and by other work-groups than those that still read
  const void *const oq = s.total_q ? dQ : nullptr, *const ok = s.total_k ? dK : nullptr, *const ov = s.total_k ? dV : nullptr;
  if (any_same({ok, ov}, {Q, K, V, dO}) || any_same({oq}, {K, V, ok, ov}) || any_same({ok}, {ov}))
    return fail(SH_ERR_INVALID_ARG, "a gradient lies over a tensor that is still read, or over another gradient");
  const hipStream_t st = (hipStream_t)hip_stream;
  const int bf16 = s.dtype == SH_BF16;
  const int align = alignment({Q, K, V, O, dO, dQ, dK, dV}, {s.q_row, s.q_head, s.k_row, s.k_head, s.v_row, s.v_head, s.o_row, s.o_head}, s.d_head, p.esz);
  PackedAttnBwd b{};
  b.f = packed_args(p, q_offsets, q_lengths, k_offsets, k_lengths);
  b.f.levels = p.levels128;
  b.f.Q = Q;
  b.f.K = K;
  b.f.V = V;
  b.f.O = (void*)O;
  b.f.lse = (float*)lse;
  b.dO = dO;
  b.dQ = dQ;
  b.dK = dK;
  b.dV = dV;
  float* delta = (float*)workspace;
  b.delta = delta;
  b.rchunk = w.rchunk;
  b.rparts = w.rparts;
  b.kslots = packed_slots(s.total_k, PACKED_KB, s.nseq) * s.nkv_heads;
  b.klevels = p.klevels;
  b.dkv = (float*)((char*)workspace + w.dkv);
  b.dkv_floats = w.dkv_floats;
  b.ds_ld = w.ds_ld;
  b.dS = w.ds ? (char*)workspace + w.ds : nullptr;
  launch_packed_bwd(b, bf16, align, delta, st);
  prof_mark(st, nullptr);
  return check_launch("switchhead_attention_backward");
}

size_t switchhead_qk_norm_workspace_bytes(const sh_qk_norm* d) {
  sh_qk_norm a;
  if (plan_norm(a, d) != SH_OK) return 0;
  return norm_bytes(a);
}

sh_status switchhead_qk_norm_rope_forward(const sh_qk_norm* d, const void* Q, const void* K, const void* w_Q, const void* w_K, const int32_t* positions,
                                          void* Y_Q, void* Y_K, void* hip_stream) {
  sh_qk_norm a;
  sh_status r = plan_norm(a, d);
  if (r != SH_OK) return r;
  const int esz = a.dtype == SH_BF16 ? 2 : 4;
  if (a.tokens && (!Q || !Y_Q || (a.nkv_heads && (!K || !Y_K)))) return fail(SH_ERR_INVALID_ARG, "Q, K, Y_Q, Y_K must not be NULL");
  if (!elements_aligned({Q, K, w_Q, w_K, Y_Q, Y_K}, esz) || !elements_aligned({positions}, 4)) return fail(SH_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
  if (!disjoint(a.tokens, a.nheads, a.yq_row, a.yq_head, a.d_head) || (a.nkv_heads && !disjoint(a.tokens, a.nkv_heads, a.yk_row, a.yk_head, a.d_head)))
    return fail(SH_ERR_INVALID_ARG, "the strides of Y_Q or Y_K lay rows over each other");
  if ((Q == Y_Q && !same_places(a.tokens, a.nheads, a.q_row, a.q_head, a.yq_row, a.yq_head)) ||
      (a.nkv_heads && K == Y_K && !same_places(a.tokens, a.nkv_heads, a.k_row, a.k_head, a.yk_row, a.yk_head)))
    return fail(SH_ERR_INVALID_ARG, "an output over its input needs the input's strides");
  if (a.tokens == 0) return SH_OK;
  if (a.nkv_heads && (any_same({Y_Q}, {K, Y_K}) || any_same({Y_K}, {Q}))) return fail(SH_ERR_INVALID_ARG, "Y_Q or Y_K lies over the other side's tensor");
  QkNormArgs n = norm_args(a, Q, K, w_Q, w_K, positions);
  n.y[0] = Y_Q;
  n.y[1] = Y_K;
  const int align = alignment({Q, K, w_Q, w_K, Y_Q, Y_K}, {a.q_row, a.q_head, a.k_row, a.k_head, a.yq_row, a.yq_head, a.yk_row, a.yk_head}, a.d_head, esz);
  prof_mark((hipStream_t)hip_stream, "qk_norm_rope");
  launch_qk_norm_rope(n, a.dtype == SH_BF16, align, false, (hipStream_t)hip_stream);
  prof_mark((hipStream_t)hip_stream, nullptr);
  return check_launch("switchhead_qk_norm_rope_forward");
}

sh_status switchhead_qk_norm_rope_backward(const sh_qk_norm* d, const void* Q, const void* K, const void* w_Q, const void* w_K, const int32_t* positions,
                                           const void* dY_Q, const void* dY_K, void* dQ, void* dK, float* dw_Q, float* dw_K, void* workspace,
                                           size_t workspace_bytes, void* hip_stream) {
  sh_qk_norm a;
  sh_status r = plan_norm(a, d);
  if (r != SH_OK) return r;
  const int esz = a.dtype == SH_BF16 ? 2 : 4;
  if (a.tokens && (!Q || !dY_Q || !dQ || (a.nkv_heads && (!K || !dY_K || !dK)))) return fail(SH_ERR_INVALID_ARG, "Q, K, dY_Q, dY_K, dQ, dK must not be NULL");
  if (!elements_aligned({Q, K, w_Q, w_K, dY_Q, dY_K, dQ, dK}, esz) || !elements_aligned({positions, dw_Q, dw_K}, 4))
    return fail(SH_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
  if (!disjoint(a.tokens, a.nheads, a.q_row, a.q_head, a.d_head) || (a.nkv_heads && !disjoint(a.tokens, a.nkv_heads, a.k_row, a.k_head, a.d_head)))
    return fail(SH_ERR_INVALID_ARG, "the strides of Q or K lay the rows of a gradient over each other");
  if ((dQ == dY_Q && !same_places(a.tokens, a.nheads, a.q_row, a.q_head, a.yq_row, a.yq_head)) ||
      (a.nkv_heads && dK == dY_K && !same_places(a.tokens, a.nkv_heads, a.k_row, a.k_head, a.yk_row, a.yk_head)))
    return fail(SH_ERR_INVALID_ARG, "a gradient over its upstream gradient needs the same strides");
  if ((r = check_workspace(workspace, workspace_bytes, norm_bytes(a))) != SH_OK) return r;
  const hipStream_t st = (hipStream_t)hip_stream;
  if (a.tokens == 0) {   // (the sums of no rows)
    if (dw_Q) launch_fill_f32(dw_Q, a.d_head, 0.f, st);
    if (dw_K) launch_fill_f32(dw_K, a.d_head, 0.f, st);
    return check_launch("switchhead_qk_norm_rope_backward");
  }
  if (a.nkv_heads && (any_same({dQ}, {K, dY_K, dK}) || any_same({dK}, {Q, dY_Q}))) return fail(SH_ERR_INVALID_ARG, "dQ or dK lies over the other side's tensor");
  QkNormArgs n = norm_args(a, Q, K, w_Q, w_K, positions);
  n.dy[0] = dY_Q;
  n.dy[1] = dY_K;
  n.dx[0] = dQ;
  n.dx[1] = dK;
  n.dw[0] = dw_Q;
  n.dw[1] = dw_K;
  n.part = (float*)workspace;
  const int align = alignment({Q, K, w_Q, w_K, dY_Q, dY_K, dQ, dK}, {a.q_row, a.q_head, a.k_row, a.k_head, a.yq_row, a.yq_head, a.yk_row, a.yk_head}, a.d_head, esz);
  prof_mark(st, "qk_norm_rope_bwd");
  launch_qk_norm_rope(n, a.dtype == SH_BF16, align, true, st);
  prof_mark(st, nullptr);
  return check_launch("switchhead_qk_norm_rope_backward");
}

}  // extern "C"
