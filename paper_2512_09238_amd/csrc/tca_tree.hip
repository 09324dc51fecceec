// Attention of a tree of drafted tokens over the compacted cache: per sequence up to 64 nodes, each of which attends to the
// regions' rows behind its window, to the ring's rows inside it, to its ancestors and to itself.
//
// Two launches.
//   partial : split-K attention.  A unit is a chunk of rows of one head's region, or of one KV head's ring (the last of them takes
//             the nodes' own rows too); a workgroup of four waves takes a unit and a group of up to 32, 64 or 128 of its queries (a
//             query: a node and one of the heads that read the unit).  With up to 32 each wave takes every fourth tile of 32
//             keys; with more, two or four waves, 32 queries each, share a tile, so that a row is read once for all of them.
//             Each wave keeps an online softmax of its own; they are merged into one (reference, sum, acc[D]) partial per query.
//   merge   : a wave per node and query head merges the partials of its region and of its KV head's ring.
//
// Up to 64 queries a row the memory is the bound: a row of K and V (512 bytes at d = 128, bf16) takes 64 x 768 flops, a fifth of
// what the matrix cores do in the time that its bytes take.  So the shape follows the loads: tiles are copied straight into LDS ahead
// of their use, a wave with a tile of its own needs no barrier, and two workgroups a CU cover each other's start and end.  32 heads,
// d = 128, budgets of 27 % on average: 64 nodes over 16 x 100000 tokens 1.01 to 1.02 ms, 4.8 to 4.9 TB/s; 8 over 16 x
// 60000 514 us, 5.8 TB/s; 32 over 8 x 30000 173 to 174 us, 4.4 TB/s (a tenth of it in the rings, whose rows meet 128 queries); 5 over
// 1 x 2000 15 to 17 us, of which the two launches, each a chain of waits, are all.  (A first shape, a wave with up to 64 queries and masks in
// every tile: 1730 us, 283 us and 21 us for the first, third and last.)
// With 128 queries a row, on the FP8 cache (half the bytes), the products and weights are the bound: 16 nodes of 8 heads over 12 x
// 60000 tokens 222 to 235 us, where their bytes take 85 and their products 95.  A round of 128 queries and 64 keys takes two
// workgroups of a CU 6200 cycles: products 3070, passage through LDS 2600, vector instructions 3600, each of them under the others of the
// other workgroup in part.
//
// Products as in the prefill kernel (v_mfma_f32_32x32x16_bf16; lane = (hh = lane / 32, c = lane % 32)):
//   S^T = K Q^T  : A = K rows (key = c, 8 consecutive d), B = Q (query = c, same 8 d), C[key = 8 (r/4) + 4 hh + r%4][query = c]
//   O^T = V^T P^T: B = P^T from the C registers, A = V^T (d = c, the same 8 keys) by transposing LDS reads; P^T as two bf16 numbers a
//   weight, a product each
// A lane holds 16 keys of one query: maximum and sum are in-register reductions and one exchange between the halves.
//
// Visibility.  Node of depth e sits at T + e.  Region: idx ascends, so a query sees a prefix; the prefix of depth 0 is counted
// once per wave, and each deeper node sees at most e rows more.  Ring: slot r holds the position T - w + ((r - T) mod w), which is
// inside the window iff that distance is over e.  Nodes: the path's bits.  Only tiles at these edges evaluate a mask.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "tca_tree.h"

namespace tca {

typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kTreeThreads = 256;
constexpr int kTreeWaves = kTreeThreads / 64;
// Keys of a tile: 32, or 64 where four waves share it (two independent chains of products and weights a wave, and half the barriers).
constexpr int tree_keys(int qg) { return qg == 4 ? 64 : 32; }
constexpr int kMinTreeChunk = 128;              // rows per unit of a short step, and of a long one: see choose_tree_chunk (at most 64 x 64: see probe)
constexpr int kMaxTreeChunk = 4096;
constexpr int kTreeSlots = 512;                 // workgroups at a time: two on a CU
constexpr int kTreeUnits = 2048, kTreeBusy = 1024;      // workgroups that short chunks may come to
constexpr int kMaxTreeSlots = 4096;             // units per head that a step is taken for

// Quotients of small numbers (number times divisor below 2^32) by one multiplication.
struct SmallDiv {
  uint32_t magic;                     // 2^32 / divisor rounded up; 0 for the divisor 1
  __host__ __device__ __forceinline__ void set(uint32_t d) { magic = d == 1 ? 0 : 0xFFFFFFFFu / d + 1; }
  __device__ __forceinline__ int operator()(int x) const { return magic ? (int)__umulhi((uint32_t)x, magic) : x; }
};

struct TreeTables {
  int64_t offs[TCA_MAX_HEADS + 1];
  int32_t unit0[TCA_MAX_HEADS + 1];   // first unit of each head's region; unit0[Hs]: their number
};
// What every workgroup reads before anything else: kernel arguments of their own, so that they come with one request (each line of the
// arguments that is asked for where it is used is a wait).
struct TreeShape {
  int n, Hq, Hkv, G, GS, w;                      // G: query heads of a KV head; GS: of a selection
  int chunk, ring_units, region_units;           // rows per unit, units of one ring, of all regions of a sequence
  int region_groups, kv_groups;                  // groups of queries of a region's unit, of a ring's
  SmallDiv by_region_groups, by_kv_groups, by_ring_units, by_GS, by_G;
};

// A partial of T results: its reference (fp32 rows: a double, see tree_partial_f32_kernel), its sum and D columns.
template <typename T> struct TreePartial {
  using ref_t = std::conditional_t<sizeof(T) == 4, double, float>;
  static constexpr int kSum = sizeof(ref_t) / 4, kColumns = 2 * kSum;      // where they lie, in floats
};
template <typename T, int D> constexpr int tree_partial_floats() { return D + TreePartial<T>::kColumns; }

// Partials of a sequence: region unit by region unit its n GS queries, then for each KV head the units of its ring (the
// last one with the nodes' own rows), n G queries each.  A query's number inside a unit: node * heads + head.
__host__ __device__ __forceinline__ int64_t partials_of(const TreeShape& t) {
  return (int64_t)t.n * ((int64_t)t.GS * t.region_units + (int64_t)t.Hq * t.ring_units);
}

// (restricted as in read_transposed)
__device__ __forceinline__ bf16x8_t tree_read16(const unsigned char* __restrict__ lds_src) { return *reinterpret_cast<const bf16x8_t*>(lds_src); }

// Waves of a workgroup, and its LDS: the tiles of its groups of waves, in stages (in their place at the end the waves' results); then
// references, sums, scales, flags.
constexpr int kNW = 4;
constexpr int tree_stages(int qg) { return qg == 1 ? 1 : 2; }
template <int D> constexpr int tree_tile_bytes(int qg) {
  const int tiles = kNW / qg * tree_stages(qg) * 4 * tree_keys(qg) * D, results = kNW * 32 * D * 4;
  return tiles > results ? tiles : results;
}
template <typename KV, int D> constexpr int tree_lds_bytes(int qg) {
  return tree_tile_bytes<D>(qg) + kNW * 32 * 8 + (sizeof(KV) == 1 ? kNW / qg * 16 * tree_keys(qg) : 0) + kNW / qg * 16;
}

// What a workgroup works on: blockIdx.x, the rings' units first.
struct TreeUnit {
  int head, heads, kvh, slot, group;             // first query head, heads that read the unit, KV head, chunk, group of queries
  bool ring;
  int hs;                                        // the region's head
  size_t first;                                  // its first partial
};
__device__ __forceinline__ TreeUnit tree_unit(const TreeShape& t, const int32_t* __restrict__ unit0, int s, int r) {
  const int G = t.G, lane = threadIdx.x & 63;
  const int kv_units = t.Hkv * t.ring_units, kv_all = kv_units * t.kv_groups;
  TreeUnit u = {};
  const size_t seq = (size_t)s * partials_of(t);
  if (r < kv_all) {
    const int v = t.by_kv_groups(r);
    u.group = r - v * t.kv_groups;
    u.kvh = t.by_ring_units(v);
    u.slot = v - u.kvh * t.ring_units;
    u.ring = true;
    u.heads = G;
    u.head = u.kvh * G;
    u.first = seq + (size_t)t.n * t.GS * t.region_units + (size_t)v * t.n * G;
    return u;
  }
  r -= kv_all;
  const int v = t.by_region_groups(r), Hs = t.by_GS(t.Hq);
  u.group = r - v * t.region_groups;
  const int end0 = lane < Hs ? unit0[lane + 1] : INT32_MAX, end1 = lane + 64 < Hs ? unit0[lane + 65] : INT32_MAX;
  u.hs = __popcll(__ballot(end0 <= v)) + __popcll(__ballot(end1 <= v));
  u.slot = v - unit0[u.hs];
  u.heads = t.GS;
  u.head = u.hs * t.GS;
  u.kvh = t.by_G(u.head);
  u.first = seq + (size_t)v * t.n * t.GS;
  return u;
}

// Rows of a region's chunk of `len` that a lane's query sees, up to `bound`, where the first `lo` are seen by all: at most 64 more, for
// positions are distinct and no node is deeper.  Called by whole waves.
__device__ __forceinline__ int more_seen(const int32_t* __restrict__ at, int len, int lo, int64_t bound) {
  const int lane = threadIdx.x & 63;
  const int next = lo + lane < len ? at[lo + lane] : INT32_MAX;
  int more = 0;
#pragma unroll
  for (int step = 32; step > 0; step >>= 1) more += (int64_t)__shfl(next, more + step - 1, kWave) <= bound ? step : 0;
  more += (int64_t)__shfl(next, more & 63, kWave) <= bound ? 1 : 0;
  return lo + more;
}

// T mod w (a 64-bit division takes a hundred instructions; positions are 32 bits as a rule)
__device__ __forceinline__ int oldest_slot(int64_t T, int w) { return T >> 32 ? (int)(T % w) : (int)((uint32_t)T % (uint32_t)w); }

template <typename KV> struct TreeCache {
  const int32_t* idx;
  const KV *Kg, *Vg;
  const int32_t* n_rows;
  const KV *ringK, *ringV;
  const int64_t* length;
  const float *Kg_scale, *Vg_scale, *ringK_scale, *ringV_scale;
  int64_t cap_rows;
};

// A unit's rows as its workgroup sees them, in tiles of TK: tiles that every query sees whole (two ranges of them), and the others, at the edges.
template <int TK> struct TreeRows {
  int n_rows;                                    // rows that some query sees
  int s0, e0, s1, e1;                            // tiles [s0, e0) and [s1, e1) are clear
  int hidden;                                    // ring: the slot of the oldest position, seen by nobody
  __device__ __forceinline__ int tiles() const { return (n_rows + TK - 1) / TK; }
  __device__ __forceinline__ int clear_tiles() const { return e0 - s0 + e1 - s1; }
  __device__ __forceinline__ int clear_tile(int i) const { return i < e0 - s0 ? s0 + i : s1 + (i - (e0 - s0)); }
  __device__ __forceinline__ int edge_tile(int i) const { return i < s0 ? i : i - s0 < s1 - e0 ? e0 + (i - s0) : e1 + (i - s0 - (s1 - e0)); }
};
template <int TK> __device__ __forceinline__ TreeRows<TK> ring_rows(int n_rows, int hidden, int deepest, int w) {
  TreeRows<TK> t;
  t.n_rows = n_rows;
  t.hidden = hidden;
  const int full = n_rows / TK;
  t.s0 = 0;
  t.e0 = t.s1 = t.e1 = full;
  // The slots of the oldest `deepest` + 1 positions, modulo w: at most two pieces of the chunk, and then one at either end.
  bool cut = false;
  for (int k = -1; k <= 1; ++k) {
    const int lo = max(0, hidden + k * w), hi = min(n_rows, hidden + k * w + deepest + 1);
    if (lo >= hi) continue;
    const int a = lo / TK, z = (hi + TK - 1) / TK;
    if (a == 0) t.s0 = min(z, full);
    else if (!cut) { t.e0 = min(a, full); t.s1 = min(z, full); cut = true; }
  }
  if (t.e0 < t.s0) t.e0 = t.s0;
  if (t.s1 < t.e0) t.s1 = t.e0;
  if (t.e1 < t.s1) t.e1 = t.s1;
  return t;
}

// One unit and one group of 32 QG queries: QG waves (32 queries each) share a tile, kNW / QG groups of them take every kNW / QG-th tile.
// KV: bf16_t, or fp8_t with a scale per row.
// What a workgroup waits for at its start is lost, so the parents, the length, the region's fill, probes of its positions and the queries
// are asked for at once, the first tile behind them, and which rows are seen is found out while the tile is on its way.  (In this
// order: loads return in the order of their requests.)
template <typename KV, int D, int QG>
__device__ __forceinline__ void tree_body(const TreeCache<KV>& c, const TreeShape& th, const TreeTables& tt, const TreeUnit& u, int s,
                                          float sl2e, const int32_t* __restrict__ parent, const bf16_t* __restrict__ q,
                                          const bf16_t* __restrict__ k_new, const bf16_t* __restrict__ v_new, float* __restrict__ part,
                                          unsigned char* lds) {
  constexpr bool kFp8 = sizeof(KV) == 1;
  constexpr int NW = kNW, KG = NW / QG;          // tiles at a time
  constexpr int KK = D / 16, DS = D / 32, CPR = D / 8;
  constexpr int TK = tree_keys(QG), SUB = TK / 32;
  constexpr int TB = TK * D * 2;                 // bytes of a K or V tile in LDS
  constexpr int STAGES = tree_stages(QG);
  constexpr int NL = TB / 1024 / QG;             // wave-loads of a bf16 tile, this wave's share
  const int n = th.n, Hkv = th.Hkv, w = th.w;
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hh = lane >> 5, cc = lane & 31;
  const int kg = wv / QG, qg = wv % QG;
  unsigned char* const mine = lds + kg * (STAGES * 2 * TB);
  float* const extra = reinterpret_cast<float*>(lds + tree_tile_bytes<D>(QG));
  float* const ms = extra;                       // [NW][32]
  float* const ls = ms + NW * 32;
  float* const scales = ls + NW * 32;            // FP8: [KG][2 stages][K (times sl2e), V][TK]
  unsigned long long* const odd = reinterpret_cast<unsigned long long*>(scales + (kFp8 ? KG * 4 * TK : 0));      // [2][KG]
  auto sync = [&] {                              // those who share a tile
    if constexpr (QG > 1) {
      __syncthreads();
    } else {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_s_waitcnt(0xC07F);        // lgkmcnt(0)
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  };

  // where the unit's rows lie, and how many there are room for
  const int64_t off = u.ring ? 0 : tt.offs[u.hs], end = u.ring ? 0 : tt.offs[u.hs + 1];
  const int r0 = u.slot * th.chunk;
  const size_t base = u.ring ? ((size_t)s * Hkv + u.kvh) * w + r0 : (size_t)s * c.cap_rows + off + r0;
  const int room = u.ring ? min(w - r0, th.chunk) : (int)min(end - off - r0, (int64_t)th.chunk);
  const KV* const kbase = (u.ring ? c.ringK : c.Kg) + base * D;
  const KV* const vbase = (u.ring ? c.ringV : c.Vg) + base * D;
  const float* const ksc = (u.ring ? c.ringK_scale : c.Kg_scale) + base;
  const float* const vsc = (u.ring ? c.ringV_scale : c.Vg_scale) + base;

  // ---- asked for first
  const int up = lane < n ? parent[(size_t)s * n + lane] : -2;
  const int64_t T = c.length[s];
  const int n_q = n * u.heads, q0 = u.group * (32 * QG);               // queries of the unit, the first one here
  int fill = 0, probe = 0;
  const int step = (room + kWave - 1) / kWave;   // region: rows of a piece whose last position is looked at
  if (!u.ring) {
    fill = c.n_rows[s * th.by_GS(th.Hq) + u.hs];
    probe = c.idx[base + min((lane + 1) * step, room) - 1];
  }
  bf16x8_t qf[KK];
  {
    const int x = min(q0 + qg * 32 + cc, n_q - 1), i = u.ring ? th.by_G(x) : th.by_GS(x);
    const bf16_t* const q_row = q + (((size_t)s * n + i) * th.Hq + u.head + (x - i * u.heads)) * D;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) qf[kk] = *reinterpret_cast<const bf16x8_t*>(q_row + kk * 16 + hh * 8);
  }
  __builtin_amdgcn_sched_barrier(0);

  // ---- tiles on their way.  bf16: straight into LDS.
  constexpr int kRsrcFlags = 0x00020000;         // raw buffer, 32-bit data format
  const int room_bytes = kFp8 ? 0 : __builtin_amdgcn_readfirstlane(room) * (D * 2);
  const __amdgpu_buffer_rsrc_t krs = __builtin_amdgcn_make_buffer_rsrc((void*)kbase, 0, room_bytes, kRsrcFlags);
  const __amdgpu_buffer_rsrc_t vrs = __builtin_amdgcn_make_buffer_rsrc((void*)vbase, 0, room_bytes, kRsrcFlags);
  int klo[NL], vlo[NL];                          // this lane's byte offsets inside a tile
#pragma unroll
  for (int j = 0; j < NL; ++j) {
    const int cid = (j * QG + qg) * 64 + lane, r = cid / CPR, ch = cid % CPR;
    klo[j] = k_off<D>(r, ch);
    vlo[j] = v_off<D>(r, ch);
  }
  auto copy_k = [&](int t, unsigned char* dst) {
#pragma unroll
    for (int j = 0; j < NL; ++j) copy16_to_lds(krs, klo[j], t * TB, dst + (j * QG + qg) * 1024);
  };
  auto copy_v = [&](int t, unsigned char* dst) {
#pragma unroll
    for (int j = 0; j < NL; ++j) copy16_to_lds(vrs, vlo[j], t * TB, dst + TB + (j * QG + qg) * 1024);
  };
  // FP8: as codes in registers, from there as bf16 numbers (which hold every code) into LDS
  auto bf16_of_codes = [](uint32_t lo, uint32_t hi) {
    return raw16_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true))};
  };
  // (two tiles ahead where waves share a tile; four with QG = 4 cost registers and brought nothing)
  constexpr int NC = (TK * D / 1024 + QG - 1) / QG, AHEAD = QG == 1 ? 1 : 2;
  struct Codes {
    raw16_t k[NC], v[NC];
    float rs;                                    // 32 keys: the lower lanes K's scale of a row, the upper ones V's; 64: wave 0 K's, wave 1 V's
  } codes[AHEAD];
  auto place = [&](int j) { return (j * QG + qg) * 64 + lane; };
  auto fetch = [&](int t, Codes& x) {
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int cid = place(j);
      if (NC * QG * 64 == TK * D / 16 || cid < TK * D / 16) {
        const size_t at = (size_t)t * (TK * D) + cid * 16;
        x.k[j] = load_raw16(kbase + at);
        x.v[j] = load_raw16(vbase + at);
      }
    }
    if constexpr (TK == 32) x.rs = (hh ? vsc : ksc)[t * TK + cc];
    else x.rs = ((qg & 1) ? vsc : ksc)[t * TK + lane];
  };
  auto store = [&](const Codes& x, unsigned char* dst, float* sc) {
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int cid = place(j), r = cid / (D / 16), ch = 2 * (cid % (D / 16));
      if (NC * QG * 64 == TK * D / 16 || cid < TK * D / 16) {
        *reinterpret_cast<raw16_t*>(dst + k_off<D>(r, ch)) = bf16_of_codes(x.k[j].x, x.k[j].y);
        *reinterpret_cast<raw16_t*>(dst + k_off<D>(r, ch + 1)) = bf16_of_codes(x.k[j].z, x.k[j].w);
        *reinterpret_cast<raw16_t*>(dst + TB + v_off<D>(r, ch)) = bf16_of_codes(x.v[j].x, x.v[j].y);
        *reinterpret_cast<raw16_t*>(dst + TB + v_off<D>(r, ch + 1)) = bf16_of_codes(x.v[j].z, x.v[j].w);
      }
    }
    if constexpr (TK == 32) {
      if (qg == 0) sc[lane] = hh ? x.rs : x.rs * sl2e;
    } else if (qg < 2) {
      sc[qg * TK + lane] = qg ? x.rs : x.rs * sl2e;
    }
  };
  // the first tile, as a rule: what it is by the rows there is room for
  const bool early = (kg + 1) * TK <= room;
  if (early) {
    if constexpr (kFp8) {
      fetch(kg, codes[0]);
    } else {
      copy_k(kg, mine);
      copy_v(kg, mine);
    }
  }
  __builtin_amdgcn_sched_barrier(0);

  // ---- the queries' nodes: this lane's, and the deepest of the workgroup's
  const TreeNode node = tree_node(up);
  int deepest = -1, depth = 0;
  uint64_t path = 0;
#pragma unroll
  for (int g = 0; g < QG; ++g) {
    const int x = min(q0 + g * 32 + cc, n_q - 1), i = u.ring ? th.by_G(x) : th.by_GS(x);
    const int exists = __shfl((int)node.there, i, kWave), d = __shfl(node.depth, i, kWave);         // (by all lanes)
    if (q0 + g * 32 + cc < n_q && exists) deepest = max(deepest, d);
    const uint64_t p = shfl64(node.path, i);
    if (g == qg) {
      depth = d;
      path = p;
    }
  }
  for (int o = 16; o > 0; o >>= 1) deepest = max(deepest, __shfl_xor(deepest, o, kWave));
  deepest = __builtin_amdgcn_readfirstlane(deepest);
  float* const out = part + (u.first + q0) * (D + 2);
  // (a copy into LDS must not outlive the workgroup)
  auto leave = [&] { __builtin_amdgcn_s_waitcnt(0x0F70); };
  if (deepest < 0) { leave(); return; }          // no node among them: nobody reads these partials

  // ---- the unit's rows that are seen
  int seen = 0;                                  // region: those that this lane's query sees
  TreeRows<TK> rows;
  const int node_rows = u.ring && u.slot == th.ring_units - 1 ? n : 0;
  if (!u.ring) {
    const int len = min(fill - r0, room);
    int n_clear = 0, most = 0;
    if (len > 0) {
      // pieces that are seen whole by all, then the rows of the first one that is not
      const int last = min((lane + 1) * step, room) - 1;
      const bool whole = lane * step < room && last < len && (int64_t)probe <= T - w;
      n_clear = min(__popcll(__ballot(whole)) * step, len);
      if (n_clear < len) n_clear += __popcll(__ballot(lane < step && n_clear + lane < len && (int64_t)c.idx[base + min(n_clear + lane, len - 1)] <= T - w));
      most = seen = n_clear;
      if (deepest > 0 && n_clear < len) {
        seen = more_seen(c.idx + base, len, n_clear, T - w + depth);
        most = more_seen(c.idx + base, len, n_clear, T - w + deepest);
      }
    }
    rows.n_rows = __builtin_amdgcn_readfirstlane(most);
    rows.s0 = 0;
    rows.e0 = rows.s1 = rows.e1 = __builtin_amdgcn_readfirstlane(n_clear) / TK;
    rows.hidden = 0;
  } else {
    rows = ring_rows<TK>(max(0, __builtin_amdgcn_readfirstlane((int)(min((int64_t)(r0 + room), T) - r0))),
                     __builtin_amdgcn_readfirstlane(oldest_slot(T, w) - r0), deepest, w);
  }
  if (rows.n_rows <= 0 && node_rows == 0) {
    for (int x = tid; x < min(n_q - q0, 32 * QG); x += NW * 64) { out[(size_t)x * (D + 2)] = -INFINITY; out[(size_t)x * (D + 2) + 1] = 0.f; }
    leave();
    return;
  }

  // per-lane LDS offsets of the fragments inside a tile
  int kfa[KK], vfa[DS];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) kfa[kk] = k_off<D>(cc, 2 * kk + hh);
  const int vr = 4 * hh + ((cc >> 2) & 3);       // what a lane addresses: 4 columns of a key; what it receives: a column of 4 keys
#pragma unroll
  for (int sl = 0; sl < DS; ++sl) vfa[sl] = v_off<D>(vr, 4 * sl + 2 * (cc >> 4) + ((cc >> 1) & 1)) + (cc & 1) * 8;

  f32x16_t o[DS];
  float m = -INFINITY, l = 0.f;                  // m: as the scores are (FP8: in base-2 units; bf16: before the factor sl2e)
  const float unit = kFp8 ? 1.f : sl2e;
#pragma unroll
  for (int sl = 0; sl < DS; ++sl)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[sl][r] = 0.f;

  // A tile in LDS against this wave's queries.  sc: its rows' scales (FP8); edge: keys that sees(key) says no to are masked;
  // between: called when K has been read, before V is.
  auto work_tile = [&](const unsigned char* kb, const float* sc, auto edge_tag, auto sees, auto between) {
    constexpr bool kEdge = decltype(edge_tag)::value;
    const unsigned char* const vb = kb + TB;
    f32x16_t sv[SUB];
#pragma unroll
    for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
      for (int r = 0; r < 16; ++r) sv[sub][r] = 0.f;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int sub = 0; sub < SUB; ++sub)
        sv[sub] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tree_read16(kb + kfa[kk] + sub * (32 * D * 2)), qf[kk], sv[sub], 0, 0, 0);
    if constexpr (kFp8) {
#pragma unroll
      for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          const f32x4_t ks = *reinterpret_cast<const f32x4_t*>(sc + sub * 32 + 8 * r4 + 4 * hh);
#pragma unroll
          for (int e = 0; e < 4; ++e) sv[sub][4 * r4 + e] *= ks[e];
        }
    }
    if constexpr (kEdge) {
#pragma unroll
      for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
        for (int r = 0; r < 16; ++r) sv[sub][r] = sees(sub * 32 + 8 * (r >> 2) + 4 * hh + (r & 3)) ? sv[sub][r] : -INFINITY;
    }
    float m4[4 * SUB];
#pragma unroll
    for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
      for (int r = 0; r < 4; ++r) m4[4 * sub + r] = fmaxf(fmaxf(sv[sub][r], sv[sub][r + 4]), fmaxf(sv[sub][r + 8], sv[sub][r + 12]));
#pragma unroll
    for (int r = 1; r < 4 * SUB; ++r) m4[0] = fmaxf(m4[0], m4[r]);
    const float mx = half_max(m4[0]);
    const float m_new = fmaxf(m, mx);
    if (__any(m_new > m)) {
      const float alpha = m_new > m ? __builtin_amdgcn_exp2f((m - m_new) * unit) : 1.f;          // 0 while m = -inf
      l *= alpha;
#pragma unroll
      for (int sl = 0; sl < DS; ++sl)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[sl][r] *= alpha;
      m = m_new;
    }
    const float top = m_new == -INFINITY ? 0.f : m_new;                // (keys of -inf only: no weight)
    // bf16: a weight is exp2(fma(score, sl2e, -ref)), one instruction less than from the difference to the maximum.  ref is rounded, which
    // is up to 2^-15 of a unit for references up to 2^10; those beyond take the difference (from 2^31 on a weight came out infinite,
    // or none was left).
    float ref = top * unit;
    if constexpr (!kFp8) {
      if (__any(fabsf(ref) > 0x1p10f)) {
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
          for (int r = 0; r < 16; ++r) sv[sub][r] -= top;
        ref = 0.f;
      }
    }
    // The sum takes the fp32 terms; the product takes each as two bf16 numbers, its leading bits and what they leave, together off by
    // 2^-17 of it at most, so that an element whose terms cancel is as exact as from a decode step's fp32 weights.  (Leading bits alone:
    // up to 50 times that error.  us without / with the second product: 32 nodes over 8 x 30000 tokens 172 / 173, 64 over 16 x 100000
    // 985 / 1006; where products bind, 16 of 64 heads over 12 x 60000, FP8 and a shared selection, 189 / 222, 48 over 8 x 50000 247 / 291.)
    bf16x8_t pf[SUB][2], pl[SUB][2];
    float lt[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int sub = 0; sub < SUB; ++sub) {
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        f32x4_t vs;
        if constexpr (kFp8) vs = *reinterpret_cast<const f32x4_t*>(sc + TK + sub * 32 + 8 * r4 + 4 * hh);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 4 * r4 + e;
          const float x = sv[sub][r], p = __builtin_amdgcn_exp2f(kFp8 ? x - ref : fmaf(x, sl2e, -ref));
          lt[e] += p;
          float pv = p;
          if constexpr (kFp8) pv = kEdge && x == -INFINITY ? 0.f : p * vs[e];           // the V row's scale rides on the weight
          const __bf16 hi = (__bf16)pv;
          pf[sub][r >> 3][r & 7] = hi;
          pl[sub][r >> 3][r & 7] = (__bf16)(pv - (float)hi);
        }
      }
    }
    l += (lt[0] + lt[1]) + (lt[2] + lt[3]);
    between();
#pragma unroll
    for (int g = 0; g < 2 * SUB; ++g)
#pragma unroll
      for (int s2 = 0; s2 < DS; s2 += 2) {             // (two slices: a product waits for the one before it on the same sums)
        bf16x8_t vt[2];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const unsigned char* at = vb + vfa[s2 + y] + g * (16 * D * 2);
          const bf16x4_t lo = read_transposed(at), hi = read_transposed(at + 8 * D * 2);
          vt[y] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
#pragma unroll
        for (int y = 0; y < 2; ++y) o[s2 + y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vt[y], pl[g >> 1][g & 1], o[s2 + y], 0, 0, 0);
#pragma unroll
        for (int y = 0; y < 2; ++y) o[s2 + y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vt[y], pf[g >> 1][g & 1], o[s2 + y], 0, 0, 0);
      }
  };

  // ---- the clear tiles.  A group without a tile in the last round copies the last one once more and works on none.
  const int n_clear = rows.clear_tiles(), rounds = (n_clear + KG - 1) / KG;
  auto tile_of = [&](int i) { return rows.clear_tile(min(i * KG + kg, n_clear - 1)); };
  const bool first_in = early && kg < n_clear && tile_of(0) == kg;     // what is on its way is the tile to begin with
  const auto nothing = [] {};
  const auto all = [](int) { return true; };
  if constexpr (kFp8) {
    // The next tiles as codes in registers, while this one is worked on; where several waves share a tile, the next one is on its way into
    // LDS meanwhile.
    float* const sc = scales + kg * (4 * TK);
    if (rounds > 0) {
      if (!first_in) fetch(tile_of(0), codes[0]);
#pragma unroll
      for (int a = 1; a < AHEAD; ++a) fetch(tile_of(a), codes[a]);
      if constexpr (QG > 1) {
        store(codes[0], mine, sc);
        fetch(tile_of(AHEAD), codes[0]);
      }
    }
#pragma unroll 1
    for (int i0 = 0; i0 < rounds; i0 += AHEAD) {
#pragma unroll
      for (int a = 0; a < AHEAD; ++a) {
        const int i = i0 + a, st = a % STAGES;
        if (i >= rounds) break;
        sync();
        if constexpr (QG == 1) {
          store(codes[0], mine, sc);
          fetch(tile_of(i + 1), codes[0]);
          sync();
        } else if (i + 1 < rounds) {
          store(codes[(a + 1) % AHEAD], mine + (st ^ 1) * (2 * TB), sc + (st ^ 1) * (2 * TK));
          fetch(tile_of(i + 1 + AHEAD), codes[(a + 1) % AHEAD]);
        }
        if (i * KG + kg < n_clear) work_tile(mine + st * (2 * TB), sc + st * (2 * TK), std::false_type{}, all, nothing);
      }
    }
  } else {
    if (!first_in) {                             // (in another order than it was asked for, the wrong one could land last)
      __builtin_amdgcn_s_waitcnt(0x0F70);
      if (rounds > 0) {
        copy_k(tile_of(0), mine);
        copy_v(tile_of(0), mine);
      }
    }
    if constexpr (QG == 1) {
      // One stage: the next tile's K is asked for when this one's has been read, V likewise; the other waves of the SIMD work meanwhile.
      static_assert(NL < 16, "four bits");
#pragma unroll 1
      for (int t = kg, i = 0; t < n_clear; t += KG, ++i) {
        __builtin_amdgcn_s_waitcnt(0x0F70 | NL); // K is in
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        work_tile(mine, nullptr, std::false_type{}, all, [&] {
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          copy_k(tile_of(i + 1), mine);
          __builtin_amdgcn_s_waitcnt(0x0F70 | NL);                     // V is in
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        });
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_s_waitcnt(0xC07F);
        copy_v(tile_of(i + 1), mine);
      }
    } else {
      static_assert(STAGES == 2, "the next tile into the other one");
#pragma unroll 1
      for (int i = 0, st = 0; i < rounds; ++i, st ^= 1) {
        __builtin_amdgcn_s_waitcnt(0x0F70);
        sync();                                  // this tile has landed, and the one before has been worked on
        copy_k(tile_of(i + 1), mine + (st ^ 1) * (2 * TB));
        copy_v(tile_of(i + 1), mine + (st ^ 1) * (2 * TB));
        if (i * KG + kg < n_clear) work_tile(mine + st * (2 * TB), nullptr, std::false_type{}, all, nothing);
      }
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);          // nothing more is on its way into LDS
  }

  // ---- the tiles at the edges and those of the nodes' own rows, through registers.  A masked key has the weight 0, which the product
  // turns into NaN where its V row is not finite: such elements are left out of the tile and added for the queries that see them.
  // (What they add is what they are, whatever the weight: an infinity, or NaN.)
  const int n_ring = rows.tiles() - n_clear, n_edge = n_ring + (node_rows + TK - 1) / TK, edge_rounds = (n_edge + KG - 1) / KG;
  sync();                                        // the last clear tile has been worked on
  if (edge_rounds > 0) {
    if (qg == 0 && lane < 2) odd[lane * KG + kg] = 0;
    sync();
  }
#pragma unroll 1
  for (int i = 0; i < edge_rounds; ++i) {
    const int e = i * KG + kg;
    const bool some = e < n_edge, own = e >= n_ring;
    const int t = own ? e - n_ring : rows.edge_tile(e);
    const int here = own ? n : rows.n_rows;
    float* const sc = scales + kg * (4 * TK);
    constexpr int NB = NL < 4 ? NL : 4;          // requests of K and of V at a time
    if (some) {
#pragma unroll 1
      for (int j0 = 0; j0 < NL; j0 += NB) {
        raw16_t kr[NB], vw[NB];
        float s0[NB], s1[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          const int cid = ((j0 + j) * QG + qg) * 64 + lane, row = t * TK + cid / CPR, ch = cid % CPR;
          kr[j] = vw[j] = raw16_t{0, 0, 0, 0};
          s0[j] = s1[j] = 0.f;
          if (row < here) {
            if (own) {
              const size_t at = (((size_t)s * n + row) * Hkv + u.kvh) * D + ch * 8;
              kr[j] = load_raw16(k_new + at);
              vw[j] = load_raw16(v_new + at);
            } else {
              const size_t at = (size_t)row * D + ch * 8;
              if constexpr (kFp8) {
                const uint2 a = *reinterpret_cast<const uint2*>(kbase + at), b = *reinterpret_cast<const uint2*>(vbase + at);
                kr[j].x = a.x; kr[j].y = a.y;
                vw[j].x = b.x; vw[j].y = b.y;
                s0[j] = ksc[row];
                s1[j] = vsc[row];
              } else {
                kr[j] = load_raw16(kbase + at);
                vw[j] = load_raw16(vbase + at);
              }
            }
          }
        }
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          const int cid = ((j0 + j) * QG + qg) * 64 + lane, r = cid / CPR, ch = cid % CPR;
          if constexpr (kFp8) {
            if (own) {                           // through codes and scales, as the cache would give them back
              float f[8];
              uint32_t codes[2];
              widen_raw16<bf16_t>(kr[j], f);
              s0[j] = fp8_codes<8, CPR>(f, codes);
              kr[j].x = codes[0]; kr[j].y = codes[1];
              widen_raw16<bf16_t>(vw[j], f);
              s1[j] = fp8_codes<8, CPR>(f, codes);
              vw[j].x = codes[0]; vw[j].y = codes[1];
            }
            kr[j] = bf16_of_codes(kr[j].x, kr[j].y);
            vw[j] = bf16_of_codes(vw[j].x, vw[j].y);
          }
          bool bad = false;
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const bool lo = (vw[j][x] & 0x7F80u) == 0x7F80u, hi = (vw[j][x] & 0x7F800000u) == 0x7F800000u;
            bad |= lo | hi;
            vw[j][x] &= (lo ? 0xFFFF0000u : 0xFFFFFFFFu) & (hi ? 0x0000FFFFu : 0xFFFFFFFFu);
          }
          if (bad) atomicOr(&odd[(i & 1) * KG + kg], 1ull << r);
          *reinterpret_cast<raw16_t*>(mine + k_off<D>(r, ch)) = kr[j];
          *reinterpret_cast<raw16_t*>(mine + TB + v_off<D>(r, ch)) = vw[j];
          if (kFp8 && ch == 0) { sc[r] = s0[j] * sl2e; sc[TK + r] = s1[j]; }
        }
      }
    }
    sync();
    if (some) {
      const int key0 = t * TK;
      auto sees = [&](int r) {
        const int key = key0 + r;
        const int x = key - rows.hidden, dist = x < 0 ? x + w : x >= w ? x - w : x;     // from the oldest position's slot, in [0, w)
        const bool in_ring = key < rows.n_rows && dist > depth, in_tree = key < n && (path >> (key & 63) & 1) != 0;
        return own ? in_tree : u.ring ? in_ring : key < seen;
      };
      work_tile(mine, sc, std::true_type{}, sees, nothing);
      const unsigned long long marked = odd[(i & 1) * KG + kg];
      uint64_t left = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(marked >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)marked);
#pragma unroll 1
      while (left) {
        const int r = __builtin_ctzll(left), row = key0 + r;
        left &= left - 1;
        const bool mine_too = sees(r);
#pragma unroll
        for (int sl = 0; sl < DS; ++sl)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            const int d = sl * 32 + 8 * q4 + 4 * hh;
            float v[4];
            if (kFp8 && !own) fp8x4_to_f32(*reinterpret_cast<const uint32_t*>((const char*)vbase + (size_t)row * D + d), v[0], v[1], v[2], v[3]);
            else load_slice<bf16_t, 4>(own ? v_new + (((size_t)s * n + row) * Hkv + u.kvh) * D + d
                                           : reinterpret_cast<const bf16_t*>(vbase) + (size_t)row * D + d, v);
#pragma unroll
            for (int x = 0; x < 4; ++x)
              if (mine_too && (__float_as_uint(v[x]) & 0x7F800000u) == 0x7F800000u) o[sl][4 * q4 + x] += v[x];
          }
      }
    }
    sync();
    if (qg == 0 && lane == 0) odd[(i & 1) * KG + kg] = 0;              // (the round after the next one's)
  }

  // ---- the groups' results
  f32x4_t* const po = reinterpret_cast<f32x4_t*>(lds);
  const float lt = half_sum(l);
  __syncthreads();
  if (hh == 0) { ms[wv * 32 + cc] = m * unit; ls[wv * 32 + cc] = lt; }
#pragma unroll
  for (int sl = 0; sl < DS; ++sl)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4)
      po[((wv * DS + sl) * 4 + q4) * 64 + lane] = f32x4_t{o[sl][4 * q4], o[sl][4 * q4 + 1], o[sl][4 * q4 + 2], o[sl][4 * q4 + 3]};
  __syncthreads();
  const int query = q0 + qg * 32 + cc;
  float M = -INFINITY, L = 0.f, wgt[KG];
#pragma unroll
  for (int k = 0; k < KG; ++k) M = fmaxf(M, ms[(k * QG + qg) * 32 + cc]);
#pragma unroll
  for (int k = 0; k < KG; ++k) {
    const float lk = ls[(k * QG + qg) * 32 + cc];
    wgt[k] = lk != 0.f ? __builtin_amdgcn_exp2f(ms[(k * QG + qg) * 32 + cc] - M) : 0.f;      // (a sum that is NaN takes part)
    if (lk != 0.f) L += lk * wgt[k];
  }
#pragma unroll
  for (int y = 0; y < DS * 4 / KG; ++y) {
    const int x = y * KG + kg;
    f32x4_t a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < KG; ++k) {
      const f32x4_t v = po[((k * QG + qg) * DS * 4 + x) * 64 + lane];
#pragma unroll
      for (int e = 0; e < 4; ++e) a[e] += v[e] * wgt[k];
    }
    if (query < n_q) {
      float* const row = out + (size_t)(qg * 32 + cc) * (D + 2);
      float* const at = row + 2 + 32 * (x >> 2) + 8 * (x & 3) + 4 * hh;
      *reinterpret_cast<float2*>(at) = make_float2(a[0], a[1]);
      *reinterpret_cast<float2*>(at + 2) = make_float2(a[2], a[3]);
      if (x == 0 && hh == 0) *reinterpret_cast<float2*>(row) = make_float2(M, L);
    }
  }
}

// grid (units of a sequence, sequences); block 64 kNW.  QGR, QGK: groups of 32 queries that a region's unit is taken by, and a ring's.
template <typename KV, int D, int QGR, int QGK>
__global__ __launch_bounds__(kNW * 64, 2) void tree_partial_kernel(
    const int32_t* __restrict__ parent, const bf16_t* __restrict__ q, const bf16_t* __restrict__ k_new, const bf16_t* __restrict__ v_new,
    float* __restrict__ part, const int32_t* __restrict__ idx, const KV* __restrict__ Kg, const KV* __restrict__ Vg,
    const int32_t* __restrict__ n_rows, const KV* __restrict__ ringK, const KV* __restrict__ ringV, const int64_t* __restrict__ length,
    const float* __restrict__ Kg_scale, const float* __restrict__ Vg_scale, const float* __restrict__ ringK_scale,
    const float* __restrict__ ringV_scale, int64_t cap_rows, float sl2e, int n, int Hq, int Hkv, int G, int GS, int w, int chunk,
    int ring_units, int region_units, int region_groups, int kv_groups, SmallDiv by_region_groups, SmallDiv by_kv_groups,
    SmallDiv by_ring_units, SmallDiv by_GS, SmallDiv by_G, TreeTables tt) {
  constexpr int kR = tree_lds_bytes<KV, D>(QGR), kK = tree_lds_bytes<KV, D>(QGK);
  __shared__ __attribute__((aligned(16))) unsigned char lds[kR > kK ? kR : kK];
  const TreeShape th = {n, Hq, Hkv, G, GS, w, chunk, ring_units, region_units, region_groups, kv_groups,
                        by_region_groups, by_kv_groups, by_ring_units, by_GS, by_G};
  const TreeCache<KV> c = {idx, Kg, Vg, n_rows, ringK, ringV, length, Kg_scale, Vg_scale, ringK_scale, ringV_scale, cap_rows};
  const int s = blockIdx.y;
  const TreeUnit u = tree_unit(th, tt.unit0, s, blockIdx.x);
  if (QGR == QGK || !u.ring) tree_body<KV, D, QGR>(c, th, tt, u, s, sl2e, parent, q, k_new, v_new, part, lds);
  else tree_body<KV, D, QGK>(c, th, tt, u, s, sl2e, parent, q, k_new, v_new, part, lds);
}

// The same for fp32 rows, which come from memory to the operands: a wave has tiles of 16 keys and the workgroup 16 queries.  Logits
// (in units of ln 2) fp64 from v_mfma_f64_16x16x4; references whole numbers, fp64 too, from the first tile to the last merge (the fp32
// number next to a logit of 2^31 may be 128 away from it, and the weights with it infinite or nothing); the
// product with V on v_mfma_f32_16x16x4, of tiles at the edges key by key on the vector ALU (a masked key's V row may be
// anything).  lane = (kb = lane / 16, c = lane % 16): scores of the keys kb + 4 r against query c; of O^T the elements (D / 16) (4 kb + r) + s.
// grid (units of all sequences, of 16 queries each); block 256
template <int D>
__global__ __launch_bounds__(kTreeThreads) void tree_partial_f32_kernel(
    TreeCache<float> c, TreeShape th, double scale2, const int32_t* __restrict__ parent, const float* __restrict__ q,
    const float* __restrict__ k_new, const float* __restrict__ v_new, float* __restrict__ part, TreeTables tt) {
  typedef double f64x4_t __attribute__((ext_vector_type(4)));
  constexpr int TK = 16, SB = D / 16;
  constexpr int PF = tree_partial_floats<float, D>(), kSum = TreePartial<float>::kSum, kColumns = TreePartial<float>::kColumns;
  __shared__ float acc_s[kTreeWaves][16][D];
  __shared__ double ms[kTreeWaves][16];
  __shared__ float ls[kTreeWaves][16];
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), s = blockIdx.y;
  const int kb = lane >> 4, cq = lane & 15, n = th.n, w = th.w, Hkv = th.Hkv;
  const TreeUnit u = tree_unit(th, tt.unit0, s, blockIdx.x);
  const int64_t T = c.length[s];
  const TreeNode node = tree_node(lane < n ? parent[(size_t)s * n + lane] : -2);
  const int n_q = n * u.heads, q0 = u.group * 16;
  float* const out = part + (u.first + q0) * PF;
  const int x = min(q0 + cq, n_q - 1), i = u.ring ? th.by_G(x) : th.by_GS(x);
  const int exists = __shfl((int)node.there, i, kWave);                // (by all lanes)
  const bool there = q0 + cq < n_q && exists != 0;
  const int depth = __shfl(node.depth, i, kWave);
  const uint64_t path = shfl64(node.path, i);
  const float* const q_row = q + (((size_t)s * n + i) * th.Hq + u.head + (x - i * u.heads)) * D;
  int deepest = there ? depth : -1;
  for (int o = 8; o > 0; o >>= 1) deepest = max(deepest, __shfl_xor(deepest, o, kWave));
  deepest = __builtin_amdgcn_readfirstlane(deepest);
  if (deepest < 0) return;

  const int r0 = u.slot * th.chunk;
  const size_t base = u.ring ? ((size_t)s * Hkv + u.kvh) * w + r0 : (size_t)s * c.cap_rows + tt.offs[u.hs] + r0;
  const float* const kbase = (u.ring ? c.ringK : c.Kg) + base * D;
  const float* const vbase = (u.ring ? c.ringV : c.Vg) + base * D;
  const float* const k_node = k_new + ((size_t)s * n * Hkv + u.kvh) * D;
  const float* const v_node = v_new + ((size_t)s * n * Hkv + u.kvh) * D;
  int n_rows = 0, n_clear = 0, seen = 0;
  const int hidden = oldest_slot(T, w) - r0, node_rows = u.ring && u.slot == th.ring_units - 1 ? n : 0;
  if (!u.ring) {
    const int len = min(c.n_rows[s * th.by_GS(th.Hq) + u.hs] - r0, th.chunk);
    if (len > 0) {
      n_clear = count_le_wave(c.idx + base, len, T - w);
      seen = more_seen(c.idx + base, len, n_clear, T - w + depth);
      n_rows = more_seen(c.idx + base, len, n_clear, T - w + deepest);
    }
  } else {
    n_rows = max(0, (int)(min((int64_t)min(w, r0 + th.chunk), T) - r0));
  }
  n_rows = __builtin_amdgcn_readfirstlane(n_rows);
  if (n_rows <= 0 && node_rows == 0) {
    if (tid < min(n_q - q0, 16)) { *reinterpret_cast<double*>(out + (size_t)tid * PF) = -INFINITY; out[(size_t)tid * PF + kSum] = 0.f; }
    return;
  }
  auto distance = [&](int r) { const int y = r - hidden; return y < 0 ? y + w : y >= w ? y - w : y; };

  double qd[D / 4];
#pragma unroll
  for (int t = 0; t < SB; ++t) {
    const f32x4_t v = *reinterpret_cast<const f32x4_t*>(q_row + kb * (D / 4) + 4 * t);
#pragma unroll
    for (int e = 0; e < 4; ++e) qd[4 * t + e] = (double)v[e];
  }
  double m = -INFINITY;
  float l = 0.f;
  f32x4_t o[SB];
#pragma unroll
  for (int s = 0; s < SB; ++s) o[s] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const int row_tiles = (n_rows + TK - 1) / TK, n_tiles = row_tiles + (node_rows + TK - 1) / TK;
  for (int t = wv; t < n_tiles; t += kTreeWaves) {
    const bool own = t >= row_tiles;               // the nodes' rows
    const int key0 = (own ? t - row_tiles : t) * TK, here = own ? node_rows : n_rows;
    const float *kt = own ? k_node : kbase, *vt = own ? v_node : vbase;
    const size_t stride = own ? (size_t)Hkv * D : D;
    const int d0 = distance(key0);
    const bool clear = !own && key0 + TK <= here && (u.ring ? d0 > deepest && d0 + TK <= w : key0 + TK <= n_clear);
    auto sees = [&](int key) {
      if (own) return key < n && (path >> (key & 63) & 1) != 0;
      return u.ring ? key < n_rows && distance(key) > depth : key < seen;
    };
    f32x4_t kf[SB], vd[4][SB / 4];
    const float* const krow = kt + min(key0 + cq, here - 1) * stride + kb * (D / 4);
#pragma unroll
    for (int s = 0; s < SB; ++s) kf[s] = *reinterpret_cast<const f32x4_t*>(krow + 4 * s);
    if (clear) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int y = 0; y < SB / 4; ++y) vd[r][y] = *reinterpret_cast<const f32x4_t*>(vt + (key0 + kb + 4 * r) * stride + 4 * (cq * (SB / 4) + y));
    }
    f64x4_t acc = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
    for (int s = 0; s < SB; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f64_16x16x4f64((double)kf[s][e], qd[4 * s + e], acc, 0, 0, 0);
    double xs[4], mx = -INFINITY;
    bool see[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      see[r] = clear || sees(key0 + kb + 4 * r);
      xs[r] = see[r] ? acc[r] * scale2 : -INFINITY;
      mx = fmax(mx, xs[r]);
    }
    mx = fmax(mx, __shfl_xor(mx, 16, kWave));
    mx = fmax(mx, __shfl_xor(mx, 32, kWave));
    const double m_new = fmax(m, ceil(mx));
    const float corr = m_new > m ? __builtin_amdgcn_exp2f((float)(m - m_new)) : 1.f;
    m = m_new;
    const double ref = m == -INFINITY ? 0.0 : m;
    float p[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) p[r] = see[r] && xs[r] != -INFINITY ? exp2_diff(xs[r] - ref) : 0.f;
    l = fmaf(l, corr, (p[0] + p[1]) + (p[2] + p[3]));
    f32x4_t ot[SB];
#pragma unroll
    for (int s = 0; s < SB; ++s) ot[s] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    if (clear) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int y = 0; y < SB / 4; ++y)
#pragma unroll
          for (int e = 0; e < 4; ++e) ot[4 * y + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vd[r][y][e], p[r], ot[4 * y + e], 0, 0, 0);
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
#pragma unroll 1
        for (int k = 0; k < 4; ++k) {            // the key that the lanes 16 k .. hold
          const float pk = __shfl(p[r], 16 * k + cq, kWave);
          const int key = key0 + k + 4 * r;
          if (!sees(key)) continue;
          const float* const vrow = vt + key * stride + kb * (D / 4);
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int s4 = 0; s4 < SB / 4; ++s4) {
              const f32x4_t v = *reinterpret_cast<const f32x4_t*>(vrow + j * SB + 4 * s4);
#pragma unroll
              for (int e = 0; e < 4; ++e) ot[4 * s4 + e][j] = fmaf(pk, v[e], ot[4 * s4 + e][j]);
            }
        }
      }
    }
#pragma unroll
    for (int s = 0; s < SB; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[s][e] = fmaf(o[s][e], corr, ot[s][e]);
  }
  l += __shfl_xor(l, 16, kWave);
  l += __shfl_xor(l, 32, kWave);
  if (kb == 0) { ms[wv][cq] = m; ls[wv][cq] = l; }
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int s = 0; s < SB; ++s) acc_s[wv][cq][SB * (4 * kb + j) + s] = o[s][j];
  __syncthreads();
  for (int y = tid; y < 16 * D; y += kTreeThreads) {
    const int qi = y / D, d = y % D;
    if (q0 + qi >= n_q) continue;
    double M = -INFINITY;
#pragma unroll
    for (int k = 0; k < kTreeWaves; ++k) M = fmax(M, ms[k][qi]);
    double L = 0, a = 0;                         // (in fp32 the four parts' sums would add their roundings)
#pragma unroll
    for (int k = 0; k < kTreeWaves; ++k)
      if (ls[k][qi] != 0.f) {
        const float wgt = __builtin_amdgcn_exp2f((float)(ms[k][qi] - M));
        L += (double)ls[k][qi] * wgt;
        a += (double)acc_s[k][qi][d] * wgt;
      }
    float* const row = out + (size_t)qi * PF;
    row[kColumns + d] = (float)a;
    if (d == 0) { *reinterpret_cast<double*>(row) = M; row[kSum] = (float)L; }
  }
}

// grid (ceil(n Hq / 4), B); block 256: a wave per node and query head, D / 64 columns a lane.  Up to 64 partials at a time: the lanes
// take a reference and a sum each, then the weights go round.
template <typename T, int D>
__global__ __launch_bounds__(256) void tree_merge_kernel(const int32_t* __restrict__ parent, const float* __restrict__ part, T* __restrict__ O,
                                                         TreeShape th, SmallDiv by_Hq, TreeTables tt) {
  using sum_t = std::conditional_t<sizeof(T) == 4, double, float>;         // (as in the merge of a decode step)
  using ref_t = typename TreePartial<T>::ref_t;
  constexpr int C = D / 64, PF = tree_partial_floats<T, D>(), kColumns = TreePartial<T>::kColumns;
  const int lane = threadIdx.x & 63, s = blockIdx.y, n = th.n;
  const int x = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (x >= n * th.Hq) return;
  const int up = lane < n ? parent[(size_t)s * n + lane] : -2;
  const int i = by_Hq(x), h = x - i * th.Hq, hs = th.by_GS(h), kvh = th.by_G(h);
  const int first = tt.unit0[hs], ns = tt.unit0[hs + 1] - first, n_slots = ns + th.ring_units;
  const float* const seq = part + (size_t)s * partials_of(th) * PF;
  const float* const p_region = seq + ((size_t)first * n * th.GS + (size_t)i * th.GS + (h - hs * th.GS)) * PF;
  const float* const p_kv = seq + ((size_t)n * th.GS * th.region_units + (size_t)kvh * th.ring_units * n * th.G + (size_t)i * th.G + (h - kvh * th.G)) * PF;
  const size_t step_region = (size_t)n * th.GS * PF, step_kv = (size_t)n * th.G * PF;
  auto partial_at = [&](int k) { return k < ns ? p_region + k * step_region : p_kv + (size_t)(k - ns) * step_kv; };
  T* const row = O + (((size_t)s * n + i) * th.Hq + h) * D + lane * C;
  ref_t M = -INFINITY;
  sum_t L = 0, a[C];
#pragma unroll
  for (int e = 0; e < C; ++e) a[e] = 0;
  for (int k0 = 0; k0 < n_slots; k0 += 64) {
    struct __attribute__((aligned(8))) { ref_t m; float l; } ml = {-INFINITY, 0.f};
    if (k0 + lane < n_slots) ml = *reinterpret_cast<const decltype(ml)*>(partial_at(k0 + lane));
    if (k0 == 0 && !__shfl((int)tree_node(up).there, i, kWave)) return;           // (while they are on their way)
    const bool some = ml.l != 0.f;                                      // (a NaN sum is no empty partial)
    ref_t top = some ? ml.m : -INFINITY;
    for (int o = 32; o > 0; o >>= 1) top = fmax(top, __shfl_xor(top, o, kWave));
    const ref_t m_new = fmax(M, top);
    const float corr = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((float)(M - m_new));
    const float wgt = some ? __builtin_amdgcn_exp2f((float)(ml.m - m_new)) : 0.f;
    L = L * corr + group_sum(some ? (sum_t)ml.l * wgt : (sum_t)0, kWave);
#pragma unroll
    for (int e = 0; e < C; ++e) a[e] *= corr;
    M = m_new;
    unsigned long long left = __ballot(some);
    constexpr int UN = 4;
    while (left) {
      float v[UN][C], wk[UN];
#pragma unroll
      for (int y = 0; y < UN; ++y) {
        wk[y] = 0.f;
#pragma unroll
        for (int e = 0; e < C; ++e) v[y][e] = 0.f;
        if (left) {
          const int k = __builtin_ctzll(left);
          left &= left - 1;
          wk[y] = __shfl(wgt, k, kWave);
          const float* const src = partial_at(k0 + k) + kColumns + lane * C;
          if constexpr (C == 2) { const float2 z = *reinterpret_cast<const float2*>(src); v[y][0] = z.x; v[y][1] = z.y; }
          else v[y][0] = *src;
        }
      }
#pragma unroll
      for (int y = 0; y < UN; ++y)
#pragma unroll
        for (int e = 0; e < C; ++e) a[e] += (sum_t)v[y][e] * wk[y];
    }
  }
#pragma unroll
  for (int e = 0; e < C; ++e) store_f32(row + e, (float)(a[e] / L));
}

// ------------------------------------------------------------------ host side --
// Groups of 32 queries (fp32: of 16, always one) that `queries` of a unit are taken by, and what a workgroup takes of them.
static int groups_of(const tca_params* prm, int64_t queries) { return prm->dtype == TCA_F32 || queries <= 32 ? 1 : queries <= 64 ? 2 : 4; }
static int queries_of(const tca_params* prm, int64_t queries) { return prm->dtype == TCA_F32 ? 16 : 32 * groups_of(prm, queries); }

static int64_t chunks_of(int64_t rows, int chunk) { return (rows + chunk - 1) / chunk; }

// Fills the shape for chunks of `chunk` rows; the workgroups per sequence.
static int64_t set_tree_chunk(TreeShape& th, TreeTables& tt, const tca_params* prm, int n, int chunk) {
  const int Hs = sel_heads(prm);
  int64_t run = 0;
  for (int h = 0; h < Hs; ++h) {
    tt.unit0[h] = (int32_t)run;
    run += chunks_of(tt.offs[h + 1] - tt.offs[h], chunk);
  }
  tt.unit0[Hs] = (int32_t)run;
  th.n = n;
  th.Hq = prm->n_q_heads;
  th.Hkv = prm->n_kv_heads;
  th.G = th.Hq / th.Hkv;
  th.GS = sel_group(prm);
  th.w = prm->window;
  th.chunk = chunk;
  th.ring_units = (int32_t)chunks_of(prm->window, chunk);
  th.region_units = (int32_t)run;
  th.region_groups = (int32_t)chunks_of((int64_t)n * th.GS, queries_of(prm, n * th.GS));
  th.kv_groups = (int32_t)chunks_of((int64_t)n * th.G, queries_of(prm, n * th.G));
  th.by_region_groups.set(th.region_groups);
  th.by_kv_groups.set(th.kv_groups);
  th.by_ring_units.set(th.ring_units);
  th.by_GS.set(th.GS);
  th.by_G.set(th.G);
  return run * th.region_groups + (int64_t)th.Hkv * th.ring_units * th.kv_groups;
}

static size_t tree_bytes(const tca_params* prm, int64_t partials) {
  const int head = prm->dtype == TCA_F32 ? TreePartial<float>::kColumns : TreePartial<bf16_t>::kColumns;
  return align_up((size_t)partials * (prm->head_dim + head) * sizeof(float), 256);
}

// The chunk length of a step, as far as its partials have room: the shortest with which all units run at a time, two on a CU, or if none
// does the shortest that comes to kTreeUnits, or the full one.  A unit's start and end take about 8 us, as long as 160 rows of its share of
// the memory's rate, so that many short units lose; one round of long ones has no last round, and where there are several
// the last one should be short.  us with at most 512 / 1024 / 2048 units (32 heads, 8 KV heads, d = 128, bf16): 1 x 30000 tokens
// and 16 nodes 29 / 37 / 53, 2 x 100000 and 64 141 / 152 / 155, 4 x 30000 and 8 82 / 84 / 89; more than 512 in any case: 8 x 30000
// and 32 199 / 180 / 174, 16 x 8000 and 24 (FP8) 221 / 143 / 134.  Where a region's rows meet more than 64 queries units are bound by
// their products, and those of one round do not end together as those that share the memory do: kTreeBusy in any case.  Shared selection,
// 512 / 1024 / 2048: 4 x 20000 and 16 (64 heads, FP8) 70 / 57 / 69, 8 x 50000 and 48 (FP8) 225 / 218 / 228, on bf16 rows 189 / 202 / 220.
// fp32 rows take the same numbers, whose units of 16 queries are one on a CU at d = 128: 1 x 5000 and 8 54 / 61 / 60, 1 x 20000 and 24 123 / 139 / 160,
// 16 x 20000 and 8 765 / 765 / 691; 512 are enough for 4 x 12000 and 20, 369 / 304 / 289, and for 8 x 8000 and 16, 438 / 353 / 326, which more
// would suit.
static int64_t choose_tree_chunk(TreeShape& th, TreeTables& tt, const tca_params* prm, int batch, int n, size_t ws_bytes) {
  const bool busy = groups_of(prm, n * sel_group(prm)) == 4;
  for (const int most : {busy ? kTreeBusy : kTreeSlots, busy ? kTreeBusy : kTreeUnits})
    for (int c = kMinTreeChunk; c <= kMaxTreeChunk; c *= 2) {
      const int64_t units = set_tree_chunk(th, tt, prm, n, c);
      if (units * batch <= most && tree_bytes(prm, batch * partials_of(th)) <= ws_bytes) return units;
    }
  return set_tree_chunk(th, tt, prm, n, kMaxTreeChunk);
}

}  // namespace tca

using namespace tca;

extern "C" size_t tca_decode_tree_workspace_bytes(const tca_params* prm, int batch, int n_nodes, int64_t max_head_rows) {
  if (check_params(prm) != TCA_OK || batch < 1 || n_nodes < 1 || n_nodes > kMaxNodes || max_head_rows < 0) return 0;
  // chunks of full length, every head as long as the longest; or what short ones can come to: a group of queries a workgroup
  const int64_t full = (int64_t)batch * n_nodes * prm->n_q_heads * (chunks_of(max_head_rows, kMaxTreeChunk) + chunks_of(prm->window, kMaxTreeChunk));
  const int64_t most = (int64_t)batch * n_nodes * prm->n_q_heads * (chunks_of(max_head_rows, kMinTreeChunk) + chunks_of(prm->window, kMinTreeChunk));
  int64_t few = (int64_t)kTreeUnits * queries_of(prm, n_nodes * (prm->n_q_heads / prm->n_kv_heads));
  if (few > most) few = most;
  return tree_bytes(prm, full > few ? full : few);
}

extern "C" int tca_decode_tree(const tca_params* prm, const tca_cache* cache, const int64_t* offs, int n_nodes,
                               const int32_t* parent, const void* q, const void* k_new, const void* v_new, void* O, void* ws,
                               size_t ws_bytes, void* stream) {
  int rc = check_tree_args(prm, cache, offs, n_nodes, "tca_decode_tree");
  if (rc) return rc;
  if (!parent || !q || !k_new || !v_new || !O || !ws) return fail(TCA_ERR_INVALID, "tca_decode_tree: NULL pointer argument");
  if (!aligned16(q, k_new, v_new, nullptr)) return fail(TCA_ERR_INVALID, "tca_decode_tree: q, k_new and v_new must be 16-byte aligned");
  const int Hs = sel_heads(prm), Hq = prm->n_q_heads, B = cache->batch, n = n_nodes;
  TreeShape th;
  TreeTables tt;
  int64_t max_rows = 0;
  for (int h = 0; h <= Hs; ++h) {
    tt.offs[h] = offs[h];
    if (h && offs[h] - offs[h - 1] > max_rows) max_rows = offs[h] - offs[h - 1];
  }
  if (chunks_of(max_rows, kMaxTreeChunk) + chunks_of(prm->window, kMaxTreeChunk) > kMaxTreeSlots)
    return fail(TCA_ERR_UNSUPPORTED, "tca_decode_tree: more than %d split-K slots per head", kMaxTreeSlots);
  set_tree_chunk(th, tt, prm, n, kMaxTreeChunk);
  const size_t need = tree_bytes(prm, B * partials_of(th));
  if (ws_bytes < need || ((uintptr_t)ws & 255))
    return fail(TCA_ERR_WORKSPACE, "tca_decode_tree: scratch needs %zu bytes, 256-byte aligned; %zu available", need, ws_bytes);
  const dim3 grid((unsigned)choose_tree_chunk(th, tt, prm, B, n, ws_bytes), B);
  hipStream_t st = (hipStream_t)stream;
  const double sl2e = logit_scale(prm) * 1.44269504088896340736;
  float* const part = (float*)ws;
  SmallDiv by_Hq;
  by_Hq.set(Hq);
  auto merge = [&](auto kernel, auto tag) {
    using TT = decltype(tag);
    hipLaunchKernelGGL(kernel, dim3((unsigned)((n * Hq + 3) / 4), B), dim3(256), 0, st, parent, (const float*)part, (TT*)O, th, by_Hq, tt);
  };
  auto with = [&](auto d_tag) {
    constexpr int D = decltype(d_tag)::value;
    if (prm->dtype == TCA_F32) {
      const TreeCache<float> c = {cache->idx, (const float*)cache->Kg, (const float*)cache->Vg, cache->n_rows, (const float*)cache->ringK,
                                  (const float*)cache->ringV, cache->length, nullptr, nullptr, nullptr, nullptr, cache->cap_rows};
      hipLaunchKernelGGL(tree_partial_f32_kernel<D>, grid, dim3(kTreeThreads), 0, st, c, th, sl2e, parent, (const float*)q, (const float*)k_new,
                         (const float*)v_new, part, tt);
      merge(tree_merge_kernel<float, D>, float{});
      return;
    }
    auto rows = [&](auto kv_tag) {
      using KV = decltype(kv_tag);
      auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(kNW * 64), 0, st, parent, (const bf16_t*)q, (const bf16_t*)k_new, (const bf16_t*)v_new, part,
                           (const int32_t*)cache->idx, (const KV*)cache->Kg, (const KV*)cache->Vg, (const int32_t*)cache->n_rows,
                           (const KV*)cache->ringK, (const KV*)cache->ringV, (const int64_t*)cache->length, (const float*)cache->Kg_scale,
                           (const float*)cache->Vg_scale, (const float*)cache->ringK_scale, (const float*)cache->ringV_scale, cache->cap_rows,
                           std::max((float)sl2e, FLT_MIN), th.n, th.Hq, th.Hkv, th.G, th.GS, th.w, th.chunk, th.ring_units, th.region_units, th.region_groups,
                           th.kv_groups, th.by_region_groups, th.by_kv_groups, th.by_ring_units, th.by_GS, th.by_G, tt);
      };
      switch (groups_of(prm, n * th.GS) * 8 + groups_of(prm, n * th.G)) {
        case 9: go(tree_partial_kernel<KV, D, 1, 1>); break;
        case 10: go(tree_partial_kernel<KV, D, 1, 2>); break;
        case 12: go(tree_partial_kernel<KV, D, 1, 4>); break;
        case 18: go(tree_partial_kernel<KV, D, 2, 2>); break;
        case 20: go(tree_partial_kernel<KV, D, 2, 4>); break;
        case 36: go(tree_partial_kernel<KV, D, 4, 4>); break;
      }
    };
    if (cache->kv_format == TCA_KV_FP8) rows(fp8_t{});
    else rows(bf16_t{});
    merge(tree_merge_kernel<bf16_t, D>, bf16_t{});
  };
  if (prm->head_dim == 128) with(std::integral_constant<int, 128>{});
  else with(std::integral_constant<int, 64>{});
  TCA_HIP_CHECK(hipGetLastError());
  return TCA_OK;
}
