// Copies of whole sequences inside a decode cache or from one cache to another: forks, compaction of a batch, a move to a
// cache with other capacities, and slots made empty.
//
// HBM-bound: 5.1 to 5.8 TB/s, read and written together.  A region's or ring's rows lie one behind the other, so a unit of work (kUnitBytes of
// one head's K rows and of its V rows) is a piece of memory.  It is requested whole into registers and stored to every copy that the launch makes of
// its sequence, so that a fork reads its source once.  The host does not know how full a region is: there is a unit for every
// kUnitBytes of the smaller capacity, and those behind the last row return at once.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <vector>

#include "tca_cache.h"

namespace tca {

constexpr int kCopyThreads = 256;
constexpr int kUnitBytes = 32 << 10;            // of K, and as many of V
constexpr int kMaxCopies = 64;                  // of one launch (the tables are kernel arguments)
constexpr int kMaxTargets = 8;                  // that one workgroup serves

struct CopyPlan {
  int64_t src_offs[TCA_MAX_HEADS + 1], dst_offs[TCA_MAX_HEADS + 1];
  int32_t unit0[TCA_MAX_HEADS + 1];             // first unit of each head's region
  int32_t ring_units, unit_rows;
  int32_t src[kMaxCopies];                      // sequence of each turn (grid.y); -1: its targets are made empty
  int32_t first[kMaxCopies + 1];                // its targets: dst[first[i]] .. dst[first[i + 1] - 1]
  int32_t dst[kMaxCopies];
};

// Rows pass through once, so they are stored past the caches, and where a sequence has one copy loaded past them too.  us with plain
// accesses / stores only / both: a sequence of 30000 tokens to seven places (0.86 GB moved) 323 / 157 / 173, twelve of 20000 on the FP8
// cache to a second one (0.96 GB) 284 / 182 / 168.
__device__ __forceinline__ void stream_out(uint4* p, uint4 v) {
  __builtin_nontemporal_store(raw16_t{v.x, v.y, v.z, v.w}, reinterpret_cast<raw16_t*>(p));
}
__device__ __forceinline__ uint4 stream_in(const uint4* p) {
  const raw16_t v = __builtin_nontemporal_load(reinterpret_cast<const raw16_t*>(p));
  return make_uint4(v.x, v.y, v.z, v.w);
}
__device__ __forceinline__ void stream_out(uint8_t* p, uint8_t v) { *p = v; }
__device__ __forceinline__ uint8_t stream_in(const uint8_t* p) { return *p; }

// `bytes`, at most kUnitBytes, of each of two arrays to n targets.  Chunk: what is copied at a time.
template <typename Chunk, typename Target>
__device__ __forceinline__ void copy_pieces(const void* k, const void* v, int bytes, int n, Target target) {
  constexpr int kPer = kUnitBytes / (kCopyThreads * 16);                   // chunks of a thread in flight, of K and of V
  const Chunk* const ks = (const Chunk*)k;
  const Chunk* const vs = (const Chunk*)v;
  const int chunks = bytes / (int)sizeof(Chunk);
  for (int c0 = threadIdx.x; c0 < chunks; c0 += kPer * kCopyThreads) {
    Chunk a[kPer], b[kPer];
    auto load = [&](auto get) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int at = c0 + i * kCopyThreads;
        if (at < chunks) { a[i] = get(ks + at); b[i] = get(vs + at); }
      }
    };
    if (n == 1) load([](const Chunk* p) { return stream_in(p); });
    else load([](const Chunk* p) { return *p; });
    for (int d = 0; d < n; ++d) {
      Chunk *kd, *vd;
      target(d, (void**)&kd, (void**)&vd);
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int at = c0 + i * kCopyThreads;
        if (at < chunks) { stream_out(kd + at, a[i]); stream_out(vd + at, b[i]); }
      }
    }
  }
}

// grid (units of a sequence, turns); block 256
template <typename Chunk>
__global__ __launch_bounds__(kCopyThreads) void copy_sequences_kernel(tca_cache from, tca_cache to, CopyPlan cp, int Hs, int Hkv, int w,
                                                                     int row_bytes) {
  const int turn = blockIdx.y, u = blockIdx.x, tid = threadIdx.x;
  const int src = cp.src[turn], first = cp.first[turn], n = cp.first[turn + 1] - first;
  if (u == 0) {                                  // the counters
    for (int d = 0; d < n; ++d) {
      const size_t dst = cp.dst[first + d];
      for (int h = tid; h < Hs; h += kCopyThreads) {
        const int64_t cap = cp.dst_offs[h + 1] - cp.dst_offs[h];
        const int rows = src < 0 ? 0 : from.n_rows[(size_t)src * Hs + h];
        to.n_rows[dst * Hs + h] = (int32_t)(rows < cap ? rows : cap);
      }
      if (tid == 0) to.length[dst] = src < 0 ? 0 : from.length[src];
    }
  }
  if (src < 0) return;
  const int ring_all = Hkv * cp.ring_units;
  if (u < ring_all) {
    const int kvh = u / cp.ring_units, r0 = (u - kvh * cp.ring_units) * cp.unit_rows;
    const int64_t T = from.length[src];
    const int rows = (int)min((int64_t)min(r0 + cp.unit_rows, w), T) - r0;
    if (rows <= 0) return;
    const size_t at = ((size_t)src * Hkv + kvh) * w + r0;
    auto to_row = [&](int d) { return ((size_t)cp.dst[first + d] * Hkv + kvh) * w + r0; };
    copy_pieces<Chunk>((const char*)from.ringK + at * row_bytes, (const char*)from.ringV + at * row_bytes, rows * row_bytes, n,
                       [&](int d, void** k, void** v) {
                         *k = (char*)to.ringK + to_row(d) * row_bytes;
                         *v = (char*)to.ringV + to_row(d) * row_bytes;
                       });
    if (from.kv_format == TCA_KV_FP8) {
      for (int r = tid; r < rows; r += kCopyThreads) {
        const float ks = from.ringK_scale[at + r], vs = from.ringV_scale[at + r];
        for (int d = 0; d < n; ++d) { to.ringK_scale[to_row(d) + r] = ks; to.ringV_scale[to_row(d) + r] = vs; }
      }
    }
    return;
  }
  // the head whose region holds the unit, found by all lanes at once
  const int ru = u - ring_all, lane = tid & 63;
  const int end0 = lane < Hs ? cp.unit0[lane + 1] : INT32_MAX, end1 = lane + 64 < Hs ? cp.unit0[lane + 65] : INT32_MAX;
  const int hs = __popcll(__ballot(end0 <= ru)) + __popcll(__ballot(end1 <= ru));
  const int r0 = (ru - cp.unit0[hs]) * cp.unit_rows;
  const int64_t room = cp.dst_offs[hs + 1] - cp.dst_offs[hs];
  const int64_t held = min((int64_t)from.n_rows[(size_t)src * Hs + hs], room);
  const int rows = (int)min((int64_t)cp.unit_rows, held - r0);
  if (rows <= 0) return;
  const size_t at = (size_t)src * from.cap_rows + cp.src_offs[hs] + r0;
  auto to_row = [&](int d) { return (size_t)cp.dst[first + d] * to.cap_rows + cp.dst_offs[hs] + r0; };
  copy_pieces<Chunk>((const char*)from.Kg + at * row_bytes, (const char*)from.Vg + at * row_bytes, rows * row_bytes, n,
                     [&](int d, void** k, void** v) {
                       *k = (char*)to.Kg + to_row(d) * row_bytes;
                       *v = (char*)to.Vg + to_row(d) * row_bytes;
                     });
  const bool scales = from.kv_format == TCA_KV_FP8;
  for (int r = tid; r < rows; r += kCopyThreads) {
    const int32_t pos = from.idx[at + r];
    float ks = 0.f, vs = 0.f;
    if (scales) { ks = from.Kg_scale[at + r]; vs = from.Vg_scale[at + r]; }
    for (int d = 0; d < n; ++d) {
      to.idx[to_row(d) + r] = pos;
      if (scales) { to.Kg_scale[to_row(d) + r] = ks; to.Vg_scale[to_row(d) + r] = vs; }
    }
  }
}

struct Span { uintptr_t begin, end; };

// Whether one of `reads` meets one of `writes`, or two of `writes` each other (both are sorted here).
static bool spans_meet(std::vector<Span>& reads, std::vector<Span>& writes) {
  auto less = [](const Span& a, const Span& b) { return a.begin < b.begin; };
  std::sort(reads.begin(), reads.end(), less);
  std::sort(writes.begin(), writes.end(), less);
  for (size_t i = 0; i + 1 < writes.size(); ++i)
    if (writes[i].end > writes[i + 1].begin) return true;
  size_t j = 0;
  uintptr_t reach = 0;                           // how far the reads that begin before a write's end go
  for (const Span& x : writes) {
    while (j < reads.size() && reads[j].begin < x.end) reach = std::max(reach, reads[j++].end);
    if (reach > x.begin) return true;
  }
  return false;
}

static int check_copy(const tca_params* prm, const tca_cache* c, const int64_t* offs, const char* which) {
  const int rc = check_cache(prm, c);
  if (rc) return rc;
  if (!offs) return fail(TCA_ERR_INVALID, "tca_cache_copy: NULL pointer argument");
  const int Hs = sel_heads(prm);
  if (offs[0] != 0 || offs[Hs] != c->cap_rows)
    return fail(TCA_ERR_INVALID, "tca_cache_copy: %s offs[0] must be 0 and offs[Hs] must equal cap_rows", which);
  for (int h = 0; h < Hs; ++h) {
    if (offs[h + 1] < offs[h]) return fail(TCA_ERR_INVALID, "tca_cache_copy: %s offs not ascending at %d", which, h);
    if (offs[h + 1] - offs[h] > INT32_MAX) return fail(TCA_ERR_UNSUPPORTED, "tca_cache_copy: head region beyond int32 rows");
  }
  return TCA_OK;
}

static int cache_copy(const tca_params* prm, const tca_cache* from, const int64_t* src_offs, const int32_t* src_seq, const tca_cache* to,
                      const int64_t* dst_offs, const int32_t* dst_seq, int n_copies, hipStream_t st) {
  int rc = check_params(prm);
  if (rc) return rc;
  rc = check_copy(prm, from, src_offs, "source");
  if (rc) return rc;
  rc = check_copy(prm, to, dst_offs, "target");
  if (rc) return rc;
  if (n_copies < 0) return fail(TCA_ERR_INVALID, "tca_cache_copy: n_copies=%d", n_copies);
  if (n_copies == 0) return TCA_OK;
  if (!src_seq || !dst_seq) return fail(TCA_ERR_INVALID, "tca_cache_copy: NULL pointer argument");
  if (from->kv_format != to->kv_format)
    return fail(TCA_ERR_INVALID, "tca_cache_copy: kv_format=%d into kv_format=%d", from->kv_format, to->kv_format);
  if (n_copies > to->batch) return fail(TCA_ERR_INVALID, "tca_cache_copy: n_copies=%d into %d sequences", n_copies, to->batch);
  const int Hs = sel_heads(prm), Hkv = prm->n_kv_heads, w = prm->window;
  const size_t row_bytes = prm->head_dim * (from->kv_format == TCA_KV_FP8 ? 1 : elem_bytes(prm));
  struct Copy { int32_t src, dst; };
  std::vector<Copy> copies;
  std::vector<Span> reads, writes, region_reads, region_writes;
  copies.reserve(n_copies);
  auto span = [](const void* p, int64_t seq, size_t bytes) {
    const uintptr_t at = (uintptr_t)p + (size_t)seq * bytes;
    return Span{at, at + bytes};
  };
  const size_t ring_bytes = (size_t)Hkv * w * row_bytes, from_bytes = from->cap_rows * row_bytes, to_bytes = to->cap_rows * row_bytes;
  for (int i = 0; i < n_copies; ++i) {
    if (src_seq[i] < -1 || src_seq[i] >= from->batch || dst_seq[i] < 0 || dst_seq[i] >= to->batch)
      return fail(TCA_ERR_INVALID, "tca_cache_copy: copy %d of sequence %d to %d is outside the batch", i, src_seq[i], dst_seq[i]);
    // a sequence onto itself: nothing to do, as long as nothing else is written there (it counts as read)
    const bool self = src_seq[i] >= 0 && (char*)from->ringK + (size_t)src_seq[i] * ring_bytes == (char*)to->ringK + (size_t)dst_seq[i] * ring_bytes;
    if (self && ((char*)from->Kg + (size_t)src_seq[i] * from_bytes != (char*)to->Kg + (size_t)dst_seq[i] * to_bytes ||
                 from->cap_rows != to->cap_rows || !std::equal(src_offs, src_offs + Hs + 1, dst_offs)))
      return fail(TCA_ERR_INVALID, "tca_cache_copy: copy %d shares its source's memory", i);
    if (src_seq[i] >= 0) {
      reads.push_back(span(from->ringK, src_seq[i], ring_bytes));
      if (from_bytes) region_reads.push_back(span(from->Kg, src_seq[i], from_bytes));
    }
    if (self) continue;
    writes.push_back(span(to->ringK, dst_seq[i], ring_bytes));
    if (to_bytes) region_writes.push_back(span(to->Kg, dst_seq[i], to_bytes));
    copies.push_back({src_seq[i], dst_seq[i]});
  }
  if (spans_meet(reads, writes) || spans_meet(region_reads, region_writes))
    return fail(TCA_ERR_INVALID, "tca_cache_copy: a sequence is written twice, or written and read (a permutation takes a second cache)");

  CopyPlan cp;
  cp.unit_rows = (int32_t)(kUnitBytes / row_bytes);
  int64_t units = 0;
  for (int h = 0; h < Hs; ++h) {
    cp.src_offs[h] = src_offs[h];
    cp.dst_offs[h] = dst_offs[h];
    cp.unit0[h] = (int32_t)units;
    units += (std::min(src_offs[h + 1] - src_offs[h], dst_offs[h + 1] - dst_offs[h]) + cp.unit_rows - 1) / cp.unit_rows;
    if (units > INT32_MAX / 2) return fail(TCA_ERR_UNSUPPORTED, "tca_cache_copy: %lld rows", (long long)from->cap_rows);
  }
  cp.src_offs[Hs] = src_offs[Hs];
  cp.dst_offs[Hs] = dst_offs[Hs];
  cp.unit0[Hs] = (int32_t)units;
  cp.ring_units = (w + cp.unit_rows - 1) / cp.unit_rows;
  units += (int64_t)Hkv * cp.ring_units;
  if (units > INT32_MAX / 2) return fail(TCA_ERR_UNSUPPORTED, "tca_cache_copy: window=%d", w);
  // copies of one sequence next to each other, so that a workgroup serves several
  std::stable_sort(copies.begin(), copies.end(), [](const Copy& a, const Copy& b) { return a.src < b.src; });
  const bool wide = aligned16(from->Kg, from->Vg, from->ringK, from->ringV) && aligned16(to->Kg, to->Vg, to->ringK, to->ringV);
  for (size_t at = 0; at < copies.size();) {
    int turns = 0, n = 0;
    while (at < copies.size() && n < kMaxCopies) {
      const int32_t src = copies[at].src;
      cp.src[turns] = src;
      cp.first[turns] = n;
      for (int k = 0; at < copies.size() && copies[at].src == src && k < kMaxTargets && n < kMaxCopies; ++k) cp.dst[n++] = copies[at++].dst;
      cp.first[++turns] = n;
    }
    const dim3 grid((unsigned)units, turns);
    auto launch = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, grid, dim3(kCopyThreads), 0, st, *from, *to, cp, Hs, Hkv, w, (int)row_bytes);
    };
    if (wide) launch(copy_sequences_kernel<uint4>);
    else launch(copy_sequences_kernel<uint8_t>);
    TCA_HIP_CHECK(hipGetLastError());
  }
  return TCA_OK;
}

}  // namespace tca

using namespace tca;

extern "C" int tca_cache_copy(const tca_params* prm, const tca_cache* src, const int64_t* src_offs, const int32_t* src_seq,
                              const tca_cache* dst, const int64_t* dst_offs, const int32_t* dst_seq, int n_copies, void* stream) {
  try {
    return cache_copy(prm, src, src_offs, src_seq, dst, dst_offs, dst_seq, n_copies, (hipStream_t)stream);
  } catch (...) {                                // host memory for the lists
    return fail(TCA_ERR_INVALID, "tca_cache_copy: out of host memory for %d copies", n_copies);
  }
}
