// Keys and values in pages: appending new rows (with the position rotation applied on the way) and attention that reads
// them - prompts, chunks of prompts and single tokens, whole contexts or a sliding window with a few first tokens that stay
// visible, with or without a prefix that all sequences share.
//
// A page holds page_size rows of every KV head, [Hkv][page_size][D]: the layout of a prompt or compressed cache of that many
// rows.  Row r of sequence b is row r % page_size of page table[b][r / page_size].
#pragma once
#include "cd_common.h"
#include "cd_score.h"

namespace cd {

// ---- where a row is ---------------------------------------------------------------------------------------------------

// x / d for 0 <= x < 2^31 as one 64-bit product and shift: magic = ceil(2^shift / d), shift = 31 + ceil(log2 d).  magic < 2^32
// and x * (magic * d - 2^shift) < 2^31 * d <= 2^shift, so the quotient is exact.
struct PageDiv { uint32_t magic; int shift; };
__device__ __forceinline__ int page_div(int x, PageDiv d) {
  return static_cast<int>((static_cast<uint64_t>(static_cast<uint32_t>(x)) * d.magic) >> d.shift);
}

struct Pages {
  const int32_t* table;      // entries of sequence b at table + b * table_stride
  int64_t table_stride;
  int page_size, n_pages, Hkv;
  PageDiv div;
};

// Row `pos` of KV head g as a row number of the page buffers (rows of D elements; below 2^32 for every buffer that fits the
// card).  An entry that names no page is read as the nearest one that exists.
__device__ __forceinline__ uint32_t page_row(const Pages& pg, const int32_t* table, int g, int pos) {
  const int e = page_div(pos, pg.div);
  const int page = min(max(table[e], 0), pg.n_pages - 1);
  return (static_cast<uint32_t>(page) * pg.Hkv + g) * pg.page_size + (pos - e * pg.page_size);
}

// ---- append -------------------------------------------------------------------------------------------------------------

struct PagedAppendArgs {
  const char* q; const char* k; const char* v;      // [total][heads][D], tokens q_stride / k_stride / v_stride bytes apart
  int64_t q_stride, k_stride, v_stride;
  const int32_t* new_off;                           // [batch+1] tokens of a sequence, or NULL: one each
  const int32_t* positions;                         // [total] place in the text, or NULL: the row in the cache
  const float* rot_table;                           // [n_positions][rot]: cosines, then sines
  char* k_pages; char* v_pages; char* q_out;
  const int32_t* lens; int32_t* new_lens;
  Pages pages;
  int64_t total_new;
  int batch, Hq, max_new, max_pages, rot, n_positions, tokens_per_group, write_lens;
};

// 16 bytes of a row as 32-bit floats, and back.
template <typename T> __device__ __forceinline__ void unpack16(const u32x4& x, float (&f)[Elem<T>::kPer16B]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t u = x[e];
    if constexpr (sizeof(T) == 2) {
      f[2 * e] = as_f32(u << 16);
      f[2 * e + 1] = as_f32(u & 0xffff0000u);
    } else {
      f[e] = as_f32(u);
    }
  }
}
template <typename T> __device__ __forceinline__ u32x4 pack16(const float (&f)[Elem<T>::kPer16B]) {
  u32x4 x;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (sizeof(T) == 2) x[e] = pack_bf16x2(f[2 * e], f[2 * e + 1]);
    else x[e] = __builtin_bit_cast(uint32_t, f[e]);
  }
  return x;
}
template <int N> __device__ __forceinline__ void load_floats(const float* p, float (&f)[N]) {
#pragma unroll
  for (int e = 0; e < N; e += 4) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(p + e);
    f[e] = x[0]; f[e + 1] = x[1]; f[e + 2] = x[2]; f[e + 3] = x[3];
  }
}

// A workgroup takes tokens_per_group tokens of one sequence; a thread 16 bytes of one head (two pieces of 16 bytes, the two
// elements of its pairs, where those lie half the rotated part apart).  The rotation is in 32 bits, rounded once to the
// storage type.  Bound by the bytes of the heads, read and written once.
template <typename T, int D, bool kHalves>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedAppendArgs a) {
  constexpr int E = Elem<T>::kPer16B;
  constexpr int kChunks = D / E;
  const int b = blockIdx.y;
  int64_t t0 = b, t1 = b + 1;
  if (a.new_off) { t0 = a.new_off[b]; t1 = a.new_off[b + 1]; }
  t0 = min(max(t0, static_cast<int64_t>(0)), a.total_new);
  t1 = min(max(t1, t0), a.total_new);
  const int n = static_cast<int>(min(t1 - t0, static_cast<int64_t>(a.max_new)));
  const int len = a.lens[b];
  const bool fits = len >= 0 && static_cast<int64_t>(len) + n <= static_cast<int64_t>(a.max_pages) * a.pages.page_size;
  const int first = static_cast<int>(blockIdx.x) * a.tokens_per_group;
  __syncthreads();                                  // everyone has read the length before it changes
  if (a.write_lens && blockIdx.x == 0 && threadIdx.x == 0) a.new_lens[b] = fits ? len + n : len;
  const int here = min(a.tokens_per_group, n - first);
  if (here <= 0) return;
  const int32_t* table = a.pages.table + b * a.pages.table_stride;
  const int Hq = a.q ? a.Hq : 0, Hkv = a.pages.Hkv, rot = a.rot;
  const int turned_units = kHalves ? (D - rot / 2) / E : kChunks;      // threads of a turned head: a pair of pieces, or a piece
  const int turned = (Hq + Hkv) * turned_units, per_token = turned + Hkv * kChunks;
  for (int item = threadIdx.x; item < here * per_token; item += 256) {
    const int tt = item / per_token, r = item - tt * per_token;
    const int t = first + tt;
    const int64_t token = t0 + t;
    const char* src; char* dst;
    int u; bool turn = false;
    if (r < turned) {
      const int h = r / turned_units;
      u = r - h * turned_units;
      turn = u < (kHalves ? rot / 2 : rot) / E;
      if (kHalves && !turn) u += rot / 2 / E;       // the pieces behind the pairs
      if (h < Hq) {
        src = a.q + token * a.q_stride + static_cast<int64_t>(h) * D * sizeof(T);
        dst = a.q_out + (token * Hq + h) * D * sizeof(T);
      } else {
        src = a.k + token * a.k_stride + static_cast<int64_t>(h - Hq) * D * sizeof(T);
        dst = a.k_pages;
      }
      if (h >= Hq) {
        if (!fits) continue;
        const int e = page_div(len + t, a.pages.div), page = table[e];
        if (page < 0 || page >= a.pages.n_pages) continue;
        dst += ((static_cast<int64_t>(page) * Hkv + (h - Hq)) * a.pages.page_size + (len + t - e * a.pages.page_size)) * D * sizeof(T);
      }
    } else {
      const int h = (r - turned) / kChunks;
      u = (r - turned) - h * kChunks;
      if (!fits) continue;
      const int e = page_div(len + t, a.pages.div), page = table[e];
      if (page < 0 || page >= a.pages.n_pages) continue;
      src = a.v + token * a.v_stride + static_cast<int64_t>(h) * D * sizeof(T);
      dst = a.v_pages + ((static_cast<int64_t>(page) * Hkv + h) * a.pages.page_size + (len + t - e * a.pages.page_size)) * D * sizeof(T);
    }
    if (!turn) { st16(dst + u * 16, ld16(src + u * 16)); continue; }
    const int pos = min(max(a.positions ? a.positions[token] : len + t, 0), a.n_positions - 1);
    const float* cs = a.rot_table + static_cast<int64_t>(pos) * rot;
    if constexpr (kHalves) {
      const int far = rot / 2 * static_cast<int>(sizeof(T));
      float x[E], y[E], c[E], s[E], p[E], q[E];
      unpack16<T>(ld16(src + u * 16), x);
      unpack16<T>(ld16(src + u * 16 + far), y);
      load_floats(cs + u * E, c);
      load_floats(cs + rot / 2 + u * E, s);
#pragma unroll
      for (int e = 0; e < E; ++e) { p[e] = x[e] * c[e] - y[e] * s[e]; q[e] = y[e] * c[e] + x[e] * s[e]; }
      st16(dst + u * 16, pack16<T>(p));
      st16(dst + u * 16 + far, pack16<T>(q));
    } else {
      float x[E], p[E];
      unpack16<T>(ld16(src + u * 16), x);
#pragma unroll
      for (int e = 0; e < E / 2; ++e) {
        const float c = cs[u * (E / 2) + e], s = cs[rot / 2 + u * (E / 2) + e];
        p[2 * e] = x[2 * e] * c - x[2 * e + 1] * s;
        p[2 * e + 1] = x[2 * e + 1] * c + x[2 * e] * s;
      }
      st16(dst + u * 16, pack16<T>(p));
    }
  }
}

// new_lens of calls whose sequences have several workgroups, where it is the array the lengths are read from.
__global__ __launch_bounds__(256) void paged_lens_kernel(PagedAppendArgs a) {
  const int b = blockIdx.x * 256 + threadIdx.x;
  if (b >= a.batch) return;
  int64_t t0 = min(max(static_cast<int64_t>(a.new_off[b]), static_cast<int64_t>(0)), a.total_new);
  int64_t t1 = min(max(static_cast<int64_t>(a.new_off[b + 1]), t0), a.total_new);
  const int n = static_cast<int>(min(t1 - t0, static_cast<int64_t>(a.max_new)));
  const int len = a.lens[b];
  const bool fits = len >= 0 && static_cast<int64_t>(len) + n <= static_cast<int64_t>(a.max_pages) * a.pages.page_size;
  a.new_lens[b] = fits ? len + n : len;
}

// ---- attention ------------------------------------------------------------------------------------------------------------

struct PagedAttendArgs {
  const void* q;             // [total_q][Hq][D]
  const int32_t* q_off;      // [batch+1], or NULL: one token each
  const void* k; const void* v;
  const int32_t* lens;       // rows of each sequence's cache, or NULL: fixed_len rows
  Pages pages;
  int fixed_len, max_len;
  int64_t total_q;
  int batch, Hq, G, max_q_len;
  int window, sinks;         // window 0: no limit
  int all_see_all;           // a prefix: every query sees every row
  float sl2;                 // scale * log2(e)
  void* out; float* lse;     // one split: the results
  float* part_o;             // several: [total_q][Hq][slots][D] unnormalised outputs
  float2* part_ml;           // [total_q][Hq][slots] (maximum in log2 units, sum)
  int NS, tiles_per_split;   // splits of this launch, tiles of one
  int slots, slot0;          // partials of a row, and the first of this launch
};

// The tokens of sequence b: first token and number.
__device__ __forceinline__ int query_range(const PagedAttendArgs& a, int b, int64_t& q0) {
  if (a.all_see_all) { q0 = 0; return static_cast<int>(a.total_q); }
  int64_t q1;
  if (a.q_off) { q0 = a.q_off[b]; q1 = a.q_off[b + 1]; } else { q0 = b; q1 = b + 1; }
  q0 = min(max(q0, static_cast<int64_t>(0)), a.total_q);
  q1 = min(max(q1, q0), a.total_q);
  return static_cast<int>(min(q1 - q0, static_cast<int64_t>(a.max_q_len)));
}
__device__ __forceinline__ int cache_rows(const PagedAttendArgs& a, int b) {
  return a.lens ? min(max(a.lens[b], 0), a.max_len) : a.fixed_len;
}

// The tiles of TK rows that a block of queries needs: those that hold one of the first `sinks` rows, then those from the
// oldest query's window to the newest query.  A tile takes part with the rows of its range only, so that a tile of both
// ranges counts no row twice, and rows outside (freed pages, rows behind the end) are never read.
template <int TK>
struct KeyTiles {
  int n_sink, n, first, sink_end, lo, hi;
  __device__ __forceinline__ KeyTiles(int len, int pos_min, int pos_max, int window, int sinks) {
    hi = min(len, pos_max + 1);
    lo = window ? max(0, pos_min - window + 1) : 0;
    sink_end = window ? min(sinks, hi) : 0;
    if (lo <= sink_end) { lo = 0; sink_end = 0; }      // one range
    n_sink = (sink_end + TK - 1) / TK;
    first = lo / TK;
    n = hi > 0 ? n_sink + (hi + TK - 1) / TK - first : 0;
  }
  __device__ __forceinline__ void tile(int u, int& base, int& from, int& to) const {
    const bool s = u < n_sink;
    base = (s ? u : first + u - n_sink) * TK;
    from = s ? 0 : lo;
    to = s ? sink_end : hi;
  }
};

// Few queries: a workgroup owns the queries of one (sequence, KV head) - up to 16 NT (token, head) rows of its group - and a
// stretch of the cache; its 4 waves take 32-row tiles in turn.  S^T = K Q^T on the matrix cores puts a query into a column,
// so that its softmax weights stay in the lanes that made them and are the B operand of O^T += V^T P^T as they are: the rows
// of a tile are dealt to the K operand in the order in which the products want the weights.  K and V go from memory to
// registers without LDS.  Bound by the bytes of K and V.
template <typename T, int D, int NT>
struct PagedWave {
  static constexpr int EPL = Elem<T>::kPer16B, KD = Elem<T>::kStepK, NK = D / KD;
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int NP = kBf16 ? 1 : D / 64;            // 16-byte pieces of a V row per lane (bf16, D = 64: 8 bytes)
  static constexpr int NX = kBf16 ? D / 16 : 4;            // elements of a piece
  static constexpr int NACC = NP * NX;                     // O^T tiles: 16 rows (slots of D) x 16 queries
  typedef uint32_t VPiece __attribute__((ext_vector_type(kBf16 && D == 64 ? 2 : 4)));

  u32x4 qf[NT][NK];
  f32x4 o[NT][NACC];
  float m[NT], l[NT];                                      // running maximum (log2 units) and this lane's share of the sum

  // row of a tile that lane (i, c) loads for K group t, and for slot e of V
  static __device__ __forceinline__ int k_row(int t, int i) { return kBf16 ? 8 * (i >> 2) + 4 * t + (i & 3) : 16 * t + i; }
  static __device__ __forceinline__ int v_row(int e, int c) { return kBf16 ? 8 * c + e : 16 * (e >> 2) + 4 * c + (e & 3); }
  // row of a tile of weight r of K group t in lane group c
  static __device__ __forceinline__ int p_row(int t, int c, int r) { return kBf16 ? 8 * c + 4 * t + r : 16 * t + 4 * c + r; }
  // first of the elements of D that lane group c holds of output piece p: o[.][p NX + x][r] is element d_first + r NX + x
  static __device__ __forceinline__ int d_first(int p, int c) { return p * 64 + c * 4 * NX; }

  __device__ __forceinline__ void load_k(const T* k, uint32_t rid, int i, int c, u32x4 (&kf)[2][NK]) const {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const T* kp = k + static_cast<int64_t>(static_cast<uint32_t>(__shfl(static_cast<int>(rid), k_row(t, i)))) * D + c * EPL;
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) kf[t][kk] = ld16_stream(kp + kk * KD);
    }
  }
  __device__ __forceinline__ void load_v(const T* v, uint32_t rid, int i, int c, VPiece (&vf)[8][NP]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const T* vp = v + static_cast<int64_t>(static_cast<uint32_t>(__shfl(static_cast<int>(rid), v_row(e, c)))) * D + i * NX;
#pragma unroll
      for (int p = 0; p < NP; ++p) vf[e][p] = __builtin_nontemporal_load(reinterpret_cast<const VPiece*>(vp + p * 64));
    }
  }
  // A operand of output tile (p, x): slot i holds element p 64 + i NX + x of the rows of lane group c
  __device__ __forceinline__ u32x4 v_operand(const VPiece (&vf)[8][NP], int p, int x, int t) const {
    u32x4 f;
    if constexpr (kBf16) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t lo = vf[2 * j][0][x >> 1], hi = vf[2 * j + 1][0][x >> 1];
        f[j] = __builtin_amdgcn_perm(hi, lo, x & 1 ? 0x07060302u : 0x05040100u);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = vf[4 * t + j][p][x];
    }
    return f;
  }
};

template <typename T, int D, int NT>
__global__ __launch_bounds__(256) void paged_stream_kernel(PagedAttendArgs a) {
  using W = PagedWave<T, D, NT>;
  constexpr int TK = 32, kWaves = 4;
  // workgroups go to the XCDs in turn and the late splits of short caches are empty: the splits are rotated from head to head
  const int rb = blockIdx.x / a.NS, g = blockIdx.y, b = blockIdx.z;
  const int split = static_cast<int>((blockIdx.x - rb * a.NS + g + gridDim.y * b) % a.NS);
  const int lane = threadIdx.x & 63, i = lane & 15, c = lane >> 4, wave = wave_index();
  int64_t q0;
  const int nq = query_range(a, b, q0), R = nq * a.G, r0 = rb * 16 * NT;
  if (r0 >= R) return;
  const int len = cache_rows(a, b);
  const int past = len - nq;
  const int pos_min = a.all_see_all ? len - 1 : past + r0 / a.G;
  const int pos_max = a.all_see_all ? len - 1 : past + (min(r0 + 16 * NT, R) - 1) / a.G;
  const KeyTiles<TK> kt(len, pos_min, pos_max, a.window, a.sinks);
  const int u_end = min(kt.n, (split + 1) * a.tiles_per_split);
  const int32_t* table = a.pages.table + b * a.pages.table_stride;
  const T* K = static_cast<const T*>(a.k);
  const T* V = static_cast<const T*>(a.v);

  W w;
  int64_t row[NT];                                         // (token, head) of this lane's column, -1: none
  int pos[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = r0 + 16 * nt + i;
    const bool valid = r < R;
    const int t = valid ? r / a.G : 0;
    row[nt] = valid ? (q0 + t) * a.Hq + g * a.G + (r - t * a.G) : -1;
    pos[nt] = !valid ? -1 : a.all_see_all ? len - 1 : past + t;
    const T* qp = static_cast<const T*>(a.q) + (valid ? row[nt] : 0) * D + c * W::EPL;
#pragma unroll
    for (int kk = 0; kk < W::NK; ++kk) w.qf[nt][kk] = valid ? ld16(qp + kk * W::KD) : zero16();
#pragma unroll
    for (int x = 0; x < W::NACC; ++x) w.o[nt][x] = f32x4{0.f, 0.f, 0.f, 0.f};
    w.m[nt] = -INFINITY;
    w.l[nt] = 0.f;
  }
  auto row_of = [&](int u) -> uint32_t {                   // of row lane % 32 of the tile
    int base, from, to;
    kt.tile(u, base, from, to);
    return page_row(a.pages, table, g, min(max(base + (lane & 31), from), to - 1));
  };
  int u = split * a.tiles_per_split + wave;
  uint32_t rid = u < u_end ? row_of(u) : 0;
  while (u < u_end) {
    u32x4 kf[2][W::NK];
    typename W::VPiece vf[8][W::NP];
    w.load_k(K, rid, i, c, kf);
    w.load_v(V, rid, i, c, vf);
    int base, from, to;
    kt.tile(u, base, from, to);
    u += kWaves;
    if (u < u_end) rid = row_of(u);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int kk = 0; kk < W::NK; ++kk)
#pragma unroll
        for (int t = 0; t < 2; ++t) mma_step<T>(s[t], kf[t][kk], w.qf[nt][kk]);
      float top = -INFINITY;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int j = base + W::p_row(t, c, r);
          const bool see = j >= from && j < to && j <= pos[nt] && (a.window == 0 || j > pos[nt] - a.window || j < a.sinks);
          s[t][r] = see ? s[t][r] * a.sl2 : -INFINITY;
          top = fmaxf(top, s[t][r]);
        }
      const float mn = fmaxf(w.m[nt], col4_max(top));
      const float ref = mn == -INFINITY ? 0.f : mn;
      const float f = mn == w.m[nt] ? 1.f : fast_exp2(w.m[nt] - ref);
      w.m[nt] = mn;
      float sum = 0.f;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) { s[t][r] = fast_exp2(s[t][r] - ref); sum += s[t][r]; }
      w.l[nt] = w.l[nt] * f + sum;
      if (__any(f != 1.f)) {
#pragma unroll
        for (int x = 0; x < W::NACC; ++x) w.o[nt][x] *= f;
      }
      // The weights are rounded to the type of V, the precision the matrix cores take them in.
      if constexpr (W::kBf16) {
        const u32x4 pf = {pack_bf16x2(s[0][0], s[0][1]), pack_bf16x2(s[0][2], s[0][3]), pack_bf16x2(s[1][0], s[1][1]), pack_bf16x2(s[1][2], s[1][3])};
#pragma unroll
        for (int x = 0; x < W::NX; ++x) mma_step<T>(w.o[nt][x], w.v_operand(vf, 0, x, 0), pf);
      } else {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const u32x4 pf = __builtin_bit_cast(u32x4, s[t]);
#pragma unroll
          for (int p = 0; p < W::NP; ++p)
#pragma unroll
            for (int x = 0; x < W::NX; ++x) mma_step<T>(w.o[nt][p * W::NX + x], w.v_operand(vf, p, x, t), pf);
        }
      }
    }
  }

  // The four waves' shares, joined pairwise through LDS: (2, 3) into (0, 1), then 1 into 0.
  __shared__ f32x4 so[2][NT][W::NACC][64];
  __shared__ float sm[2][NT][64], sl[2][NT][64];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) w.l[nt] = col4_sum(w.l[nt]);
#pragma unroll
  for (int half = 2; half >= 1; half >>= 1) {
    if (wave >= half && wave < 2 * half) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int x = 0; x < W::NACC; ++x) so[wave - half][nt][x][lane] = w.o[nt][x];
        sm[wave - half][nt][lane] = w.m[nt];
        sl[wave - half][nt][lane] = w.l[nt];
      }
    }
    __syncthreads();
    if (wave < half) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float m2 = sm[wave][nt][lane], mn = fmaxf(w.m[nt], m2), ref = mn == -INFINITY ? 0.f : mn;
        const float f = fast_exp2(w.m[nt] - ref), f2 = fast_exp2(m2 - ref);
        w.m[nt] = mn;
        w.l[nt] = w.l[nt] * f + sl[wave][nt][lane] * f2;
#pragma unroll
        for (int x = 0; x < W::NACC; ++x) w.o[nt][x] = w.o[nt][x] * f + so[wave][nt][x][lane] * f2;
      }
    }
    __syncthreads();
  }
  if (wave != 0) return;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    if (row[nt] < 0) continue;
    if (a.slots > 1) {
      const int64_t at = row[nt] * a.slots + a.slot0 + split;
      if (c == 0) a.part_ml[at] = float2{w.m[nt], w.l[nt]};
      if (w.l[nt] == 0.f) continue;
#pragma unroll
      for (int p = 0; p < W::NP; ++p)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int x = 0; x < W::NX; ++x) a.part_o[at * D + W::d_first(p, c) + r * W::NX + x] = w.o[nt][p * W::NX + x][r];
    } else {
      const float inv = w.l[nt] > 0.f ? 1.f / w.l[nt] : 0.f;
#pragma unroll
      for (int p = 0; p < W::NP; ++p)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int x = 0; x < W::NX; ++x)
            store_elem(static_cast<T*>(a.out), row[nt] * D + W::d_first(p, c) + r * W::NX + x, w.o[nt][p * W::NX + x][r] * inv);
      if (c == 0) a.lse[row[nt]] = w.l[nt] > 0.f ? (w.m[nt] + fast_log2(w.l[nt])) * kLn2 : -INFINITY;
    }
  }
}

// Many queries: the tiles of 64 rows go through LDS, where the 4 waves of a workgroup share them, 32 (token, head) rows of a
// group to a wave.  The next tile is on its way (straight into LDS, two buffers) while one is worked on.
//
// S^T = K Q^T in products of 32 x 32 x 16: a lane has one query (l % 32) and of 32 rows the 16 rows 8 (r / 4) + 4 h + r % 4,
// h = l / 32.  Its weights are the B operand of O^T += V^T P^T as they are, since the order of the contraction is free: step s
// of 32 rows takes 16 s + 4 h + {0..3, 8..11} from lane half h.  V^T comes from LDS by transposing reads: 16 lanes name 4 rows
// x 4 pieces of 4 elements (lane i: row i / 4, piece i % 4) and get a column of 4 each; which elements of D make up the pieces
// is free too, and is taken so that a lane ends with 8 neighbouring elements of its query's output.  16-byte pieces of a row
// are permuted by XOR with the row in LDS (K: row % 8, V: 2 (row % 4)), which makes both kinds of reads free of conflicts.
//
// Sums are taken against a reference that follows the maximum only when a tile exceeds it by 2^8 (any reference gives the
// same result while nothing overflows), so that the outputs are rarely rescaled.
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4;

template <int D>
struct PagedTile {
  static constexpr int TK = 64, kRows = 128, kWaves = 4;
  static constexpr int kRowBytes = 2 * D, kChunks = D / 8;         // 16-byte pieces of a row
  static constexpr int kPerLoad = 64 / kChunks;                    // rows of one load instruction
  static constexpr int kLoads = TK / kWaves / kPerLoad;
  static constexpr int kTileBytes = TK * kRowBytes;
  static constexpr int NS = D / 16, ND = D / 32;
};

__device__ __forceinline__ f32x16 mma32(const u32x4& a, const u32x4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

template <int D>
__global__ __launch_bounds__(256, 2) void paged_tile_kernel(PagedAttendArgs a) {
  using P = PagedTile<D>;
  constexpr int TK = P::TK;
  __shared__ __attribute__((aligned(16))) char s_k[2][P::kTileBytes], s_v[2][P::kTileBytes];
  // workgroups of a (sequence, KV head) behind one L2, the heads of every sequence spread over the XCDs; the longest rows of a
  // prompt first
  int x = blockIdx.x, gb = blockIdx.y + gridDim.y * blockIdx.z;
  if ((gridDim.y * gridDim.z) % 8 == 0) {
    const int64_t at = x + static_cast<int64_t>(gridDim.x) * gb;
    const int64_t slot = at / 8;
    x = static_cast<int>(slot % gridDim.x);
    gb = static_cast<int>(slot / gridDim.x) * 8 + static_cast<int>(at % 8);
  }
  const int g = gb % a.pages.Hkv, b = gb / a.pages.Hkv;
  const int blocks = static_cast<int>(gridDim.x) / a.NS;
  const int split = x % a.NS, rb = blocks - 1 - x / a.NS;
  const int lane = threadIdx.x & 63, wave = wave_index(), col = lane & 31, h = lane >> 5;
  int64_t q0;
  const int nq = query_range(a, b, q0), R = nq * a.G, r0 = rb * P::kRows;
  if (r0 >= R) return;
  const int len = cache_rows(a, b), past = len - nq;
  const int pos_min = a.all_see_all ? len - 1 : past + r0 / a.G;
  const int pos_max = a.all_see_all ? len - 1 : past + (min(r0 + P::kRows, R) - 1) / a.G;
  const KeyTiles<TK> kt(len, pos_min, pos_max, a.window, a.sinks);
  const int u0 = split * a.tiles_per_split, u_end = min(kt.n, u0 + a.tiles_per_split);

  // this wave's rows
  const int wr0 = r0 + 32 * wave, r = wr0 + col;
  const bool valid = r < R, any_rows = wr0 < R;
  const int t = valid ? r / a.G : 0;
  const int64_t row = (q0 + t) * a.Hq + g * a.G + (r - t * a.G);       // where valid
  const int pos = !valid ? -1 : a.all_see_all ? len - 1 : past + t;
  const int wave_min = a.all_see_all ? len - 1 : past + wr0 / a.G;
  const int wave_max = a.all_see_all ? len - 1 : past + (min(wr0 + 32, R) - 1) / a.G;
  u32x4 qf[P::NS];
#pragma unroll
  for (int s = 0; s < P::NS; ++s)
    qf[s] = valid ? ld16(static_cast<const uint16_t*>(a.q) + row * D + s * 16 + h * 8) : zero16();
  f32x16 o[P::ND];
#pragma unroll
  for (int d = 0; d < P::ND; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
  float ref = -INFINITY, l = 0.f;                      // reference (unscaled logits), this lane's share of the sum

  // a tile's rows on their way: this wave brings 16 of them, lane % 16 looks up the page of one
  const int32_t* table = a.pages.table + b * a.pages.table_stride;
  int entry = 0, at_row = 0;
  auto look_up = [&](int u) {
    int base, from, to;
    kt.tile(u, base, from, to);
    const int p = min(max(base + 16 * wave + (lane & 15), from), to - 1);
    const int e = page_div(p, a.pages.div);
    at_row = p - e * a.pages.page_size;
    entry = table[e];
  };
  auto row_number = [&]() -> uint32_t {
    const int page = min(max(entry, 0), a.pages.n_pages - 1);
    return (static_cast<uint32_t>(page) * a.pages.Hkv + g) * a.pages.page_size + at_row;
  };
  const int sub = lane / P::kChunks, piece = lane % P::kChunks;
  auto issue = [&](uint32_t rid, char* kd, char* vd) {
#pragma unroll
    for (int n = 0; n < P::kLoads; ++n) {
      const int in_wave = n * P::kPerLoad + sub;                     // row of the wave's 16
      const int64_t off = static_cast<int64_t>(static_cast<uint32_t>(__shfl(static_cast<int>(rid), in_wave))) * D;
      load_to_lds16(static_cast<const uint16_t*>(a.k) + off + ((piece ^ (in_wave & 7)) * 8), kd + (16 * wave + n * P::kPerLoad) * P::kRowBytes);
      load_to_lds16(static_cast<const uint16_t*>(a.v) + off + ((piece ^ (2 * (in_wave & 3))) * 8), vd + (16 * wave + n * P::kPerLoad) * P::kRowBytes);
    }
  };

  // offsets of this lane's reads
  uint32_t k_off[4], v_off[2];
#pragma unroll
  for (int s = 0; s < 4; ++s) k_off[s] = col * P::kRowBytes + (((2 * s) ^ (h ^ (lane & 7))) * 16);
  const int li = lane & 15, dh = (lane >> 4) & 1;
#pragma unroll
  for (int d = 0; d < 2; ++d)
    v_off[d] = (4 * h + (li >> 2)) * P::kRowBytes + (((4 * d) ^ (2 * dh + (li & 1)) ^ (2 * (li >> 2))) * 16) + ((li & 3) >> 1) * 8;

  auto step = [&](int u, const char* __restrict kc, const char* __restrict vc, char* __restrict kn, char* __restrict vn) __attribute__((always_inline)) {
    const bool more = u + 1 < u_end;
    if (more) {
      const uint32_t rid = row_number();
      if (u + 2 < u_end) look_up(u + 2);
      issue(rid, kn, vn);
    }
    int base, from, to;
    kt.tile(u, base, from, to);
    if (any_rows && base <= wave_max) {
      f32x16 s[2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[kb][e] = 0.f;
#pragma unroll
        for (int st = 0; st < P::NS; ++st) {
          const u32x4 kf = *reinterpret_cast<const u32x4*>(kc + k_off[st & 3] + (st >> 2) * 128 + kb * 32 * P::kRowBytes);
          s[kb] = mma32(kf, qf[st], s[kb]);
        }
      }
      const bool full = base >= from && base + TK <= to && base + TK - 1 <= wave_min &&
                        (a.window == 0 || base > wave_max - a.window || base + TK <= a.sinks);
      if (!full) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int j = base + 32 * kb + 8 * (e >> 2) + 4 * h + (e & 3);
            const bool see = j >= from && j < to && j <= pos && (a.window == 0 || j > pos - a.window || j < a.sinks);
            if (!see) s[kb][e] = -INFINITY;
          }
      }
      float top = s[0][0];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, s[kb][e]);
      float lo, hi;
      pair32(top, lo, hi);
      top = fmaxf(lo, hi);
      if (__any((top - ref) * a.sl2 > 8.f)) {          // -inf - -inf is no number and asks for nothing
        const float mn = fmaxf(ref, top), f = mn == ref ? 1.f : fast_exp2((ref - mn) * a.sl2);
        ref = mn;
        l *= f;
#pragma unroll
        for (int d = 0; d < P::ND; ++d)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[d][e] *= f;
      }
      const float shift = ref == -INFINITY ? 0.f : ref * a.sl2;
      u32x4 pf[2][2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int e = 0; e < 16; ++e) { s[kb][e] = fast_exp2(s[kb][e] * a.sl2 - shift); l += s[kb][e]; }
        // rounded to bf16, what the matrix cores take
#pragma unroll
        for (int sh = 0; sh < 2; ++sh)
#pragma unroll
          for (int j = 0; j < 4; ++j) pf[kb][sh][j] = pack_bf16x2(s[kb][8 * sh + 2 * j], s[kb][8 * sh + 2 * j + 1]);
      }
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int sh = 0; sh < 2; ++sh)
#pragma unroll
          for (int d = 0; d < P::ND; ++d) {
            const char* vp = vc + v_off[d & 1] + (d >> 1) * 128 + (32 * kb + 16 * sh) * P::kRowBytes;
            typedef __attribute__((address_space(3))) s16x4* LdsPtr;
            const s16x4 lo4 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)vp);
            const s16x4 hi4 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(vp + 8 * P::kRowBytes));
            typedef __attribute__((ext_vector_type(8))) short s16x8;
            const s16x8 vf = __builtin_shufflevector(lo4, hi4, 0, 1, 2, 3, 4, 5, 6, 7);
            o[d] = mma32(__builtin_bit_cast(u32x4, vf), pf[kb][sh], o[d]);
          }
    }
    stage_barrier();
    asm volatile("" : "+v"(entry));                    // looked at behind the wait of the barrier only
  };
  if (u0 < u_end) {
    look_up(u0);
    const uint32_t rid = row_number();
    if (u0 + 1 < u_end) look_up(u0 + 1);
    issue(rid, s_k[0], s_v[0]);
    stage_barrier();
    asm volatile("" : "+v"(entry));
    int u = u0;
    for (; u + 1 < u_end; u += 2) {
      step(u, s_k[0], s_v[0], s_k[1], s_v[1]);
      step(u + 1, s_k[1], s_v[1], s_k[0], s_v[0]);
    }
    if (u < u_end) step(u, s_k[0], s_v[0], s_k[1], s_v[1]);
  }
  if (!valid) return;
  float lo, hi;
  pair32(l, lo, hi);
  l = lo + hi;
  const float m = ref * a.sl2;                           // log2 units
  if (a.slots > 1) {
    const int64_t at = row * a.slots + a.slot0 + split;
    if (h == 0) a.part_ml[at] = float2{m, l};
    if (l == 0.f) return;
#pragma unroll
    for (int d = 0; d < P::ND; ++d)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<f32x4*>(a.part_o + at * D + 32 * d + 16 * (e >> 3) + 8 * h + (e & 4)) = f32x4{o[d][e], o[d][e + 1], o[d][e + 2], o[d][e + 3]};
  } else {
    const float inv = l > 0.f ? 1.f / l : 0.f;
    uint16_t* out = static_cast<uint16_t*>(a.out) + row * D;
#pragma unroll
    for (int d = 0; d < P::ND; ++d)
#pragma unroll
      for (int e = 0; e < 16; e += 8) {
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = pack_bf16x2(o[d][e + 2 * j] * inv, o[d][e + 2 * j + 1] * inv);
        st16(out + 32 * d + 2 * e + 8 * h, w);
      }
    if (h == 0) a.lse[row] = l > 0.f ? (m + fast_log2(l)) * kLn2 : -INFINITY;
  }
}

// The partial results of a (token, head) joined, by W waves: 1 where a workgroup joins four rows, 4 where the rows are few and
// their partials many.  A partial without any row has no output, only its (maximum, sum).  Tokens that no sequence owns are left
// as they are.
constexpr int kJoinSlots = 256;                            // most partials of a row

template <typename T, int D, int W>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttendArgs a) {
  constexpr int N = D / 64, NJ = kJoinSlots / 64, U = 4;
  const int lane = threadIdx.x & 63, wave = wave_index(), part = wave % W;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * (4 / W) + wave / W;
  const int64_t q_first = a.q_off ? a.q_off[0] : 0, q_end = a.q_off ? min(static_cast<int64_t>(a.q_off[a.batch]), a.total_q) : a.total_q;
  const int64_t token = row / a.Hq;
  const bool owned = token >= q_first && token < q_end;
  if (W == 1 && !owned) return;
  const float2* ml = a.part_ml + (owned ? row : 0) * a.slots;
  float2 x[NJ];
  float top = -INFINITY;
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    x[j] = 64 * j + lane < a.slots ? ml[64 * j + lane] : float2{-INFINITY, 0.f};
    top = fmaxf(top, x[j].x);
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
  const float ref = top == -INFINITY ? 0.f : top;
  float l = 0.f, f[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    f[j] = x[j].y > 0.f ? fast_exp2(x[j].x - ref) : 0.f;
    l += x[j].y * f[j];
  }
  l = wave_sum(l);
  float o[N] = {};
  const float* po = a.part_o + (owned ? row : 0) * a.slots * D + lane * N;
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    if (64 * j >= a.slots) break;
    for (int s = part; s < min(64, a.slots - 64 * j); s += W * U) {
      float w[U];
      bool any = false;
#pragma unroll
      for (int y = 0; y < U; ++y) {
        w[y] = s + W * y < 64 ? __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f[j]), min(s + W * y, 63))) : 0.f;
        any |= w[y] != 0.f;
      }
      if (!any) continue;
      float v[U][N];
#pragma unroll
      for (int y = 0; y < U; ++y)
#pragma unroll
        for (int e = 0; e < N; ++e) v[y][e] = w[y] != 0.f ? po[static_cast<int64_t>(64 * j + s + W * y) * D + e] : 0.f;
#pragma unroll
      for (int y = 0; y < U; ++y)
#pragma unroll
        for (int e = 0; e < N; ++e) o[e] += v[y][e] * w[y];
    }
  }
  if constexpr (W > 1) {
    __shared__ float so[W][D];
#pragma unroll
    for (int e = 0; e < N; ++e) so[part][lane * N + e] = o[e];
    __syncthreads();
    if (part != 0 || !owned) return;
#pragma unroll
    for (int e = 0; e < N; ++e)
      for (int w = 1; w < W; ++w) o[e] += so[w][lane * N + e];
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int e = 0; e < N; ++e) store_elem(static_cast<T*>(a.out), row * D + lane * N + e, o[e] * inv);
  if (lane == 0) a.lse[row] = l > 0.f ? (ref + fast_log2(l)) * kLn2 : -INFINITY;
}

}  // namespace cd
