// Attention over the lists of a block: dci_attn_forward (dense rows) and dci_attn_cached (rows of the 8-bit cache).
//
// For a row i and a head h, over the entries e of the row's list:  z_e = scale (q_i . K_e) + bias_e,  out = sum exp(z_e) V_e / sum exp(z_e).
// One pass over the list: a running maximum m, the sum l of exp(z - m) and the accumulator of exp(z - m) V, the last two rescaled
// when m grows.  Every K and V row that an entry names is read once, straight into registers, 16 columns of an 8-bit row to a lane, 8 of others:
//   a head's columns lie in LH = 1 .. 32 adjacent lanes, in pieces of 16 bytes that follow each other from lane to lane, so that a load asks
//   for 128 bytes in one place wherever a head has them (a lane has one piece, of a 32-bit row two; the piece that a head ends in is its last 16
//   bytes, whichever of them the piece before has as well: those count once in a score, and are written twice alike), the heads of a row side by
//   side, P lanes in all (a power of two up to 64; more heads are shared out between wavefronts).  A score is a sum over LH lanes, and the lanes of
//   a head then hold what they need for their columns of the output: nothing passes through LDS.
//   The 64 / P groups of lanes of a wavefront work on rows of their own, or R of them on one row, each on every R-th entry, and join their
//   (m, l, acc) at the row's end.
//   A group's lanes look up P entries at a time, an entry to a lane, the next P while these are worked on; what an entry names then goes from its
//   lane to all of them.  An entry that is left out takes row 0's place and a score of -inf.
//   Query heads that share a key head are worked on together, up to four of them (GQ), from the same registers (24,576 rows of nine 32-bit entries,
//   16 query heads of 64 on four: 105 us; two at a time 112).
// Lists of more than 64 entries, and all where there is a handful of them, are worked on by chunks: a wavefront takes `chunk` entries of the whole
// array of entries, so that neither the number nor the length of lists needs to be known, and finds the rows they belong to (a 64-way search in
// indptr).  A list that lies within a chunk is done there; of others (m, l, acc) of the piece is left in the workspace, for k_attn_join to add up in
// order.  A chunk has at most two such pieces: that of a list that goes on from before or begins with the chunk (0), and that of one that begins
// inside and goes on behind it (1).
// What bounds it: the lines that entries name.  98,304 rows of 12 entries of four 8-bit heads of 64, with weights: 141 us (129 without them), 0.92 GB
// between L2 and memory by the counters, 6.5 TB/s; 0.6 GB of them are keys and values, 0.1 q and out, the rest lines of slots, scales and weights.
// Dense 32-bit rows, 24,576 by 8.5 entries of 2 KB: 72 us, 0.47 GB, 6.5 TB/s.  Where rows are few or entries narrow it is the chain of reads, bounds -
// source - slot - row, and the instructions: 10,007 rows of 36 entries of three heads of 41 with biases and weights take 47 us at 2.7 TB/s, of which
// 14.8 million vector instructions are 24.
#include "dci_kv.h"

namespace dci {
namespace {

constexpr int kAttnBlock = 256, kAttnWaves = kAttnBlock / kWave;
constexpr int kShort = 64;  // longer lists are worked on by chunks
constexpr float kLog2E = 1.44269504088896340736f;
// Wavefronts to a SIMD that the registers are shared out for: as many as there are with few registers spilled.  (Two query heads to a key head spill up
// to 36 with three wavefronts, of 8-bit and 32-bit rows.  With two wavefronts and none spilled, lists of nine to 2,000 entries of four such pairs
// take 2 % more on average: 10 to 1 % less with a bias where lists are short, 1 to 14 % more where rows are of 8 bits and lists long, 9 to 23 % more
// for 16-bit rows and short lists, which spill none.)
constexpr int waves_per_simd(int type, int gq) { return gq == 4 ? 2 : gq == 2 ? 3 : type == DCI_F32 || type == kE4M3 ? 3 : 4; }
// columns to a lane
template <int TYPE>
constexpr int kCols = TYPE == kE4M3 ? 16 : 8;
constexpr double kWeightUnit = 4294967296.0;  // 2^32

struct Attn {
  long long n_rows;
  const long long* n_dev;
  const long long* indptr;
  const int* src;
  long long n_edges;
  unsigned n_src, n_at;  // sources; rows of k and v (sources again, or slots)
  int type;              // of q and out
  int heads, dim, group;
  float scale;
  const char* q;
  char* out;
  long long q_stride, out_stride;  // bytes
  float* lse;
  const float* bias;
  int bias_heads;
  const char *k, *v;
  unsigned k_stride, v_stride;  // bytes
  const float* scales;           // the cache's, [block, kv head, 2]
  int block_log2, kv_heads;
  const int* slots;  // nullptr: src is the row of k and v
  float* scores;     // [n_edges, heads], accumulating only
  unsigned long long* weight;
  int lh_log2, p_log2, r_log2;  // lanes to a head, to an entry; lane groups to a row
  bool ragged;                  // dense rows whose heads do not fill those lanes: columns of others, or none, are read as well
  int wave_heads;               // key heads to a wavefront
  int passes;                   // wavefronts that share a row's key heads and their groups
  int gq_passes;                // of them, those that share a group
  int pass_heads;               // query heads to one of those, in k_attn_groups
  int chunk;
  int n_chunks;  // 0: there are no long lists
  int short_list;  // longer lists are worked on by chunks: kShort, or 0 where all are
  long long longest;  // entries of a list that count
  int stash_row;  // with weights: floats of LDS for the scores of an entry (an odd number, against bank conflicts), 0 without
  float* part_ml;   // [2 n_chunks, heads, 2]
  float* part_acc;  // [2 n_chunks, heads, W]
  float* all_lse;   // lse of the long lists by row, accumulating only
};

// What a lane of an attention wavefront is there for
struct Place {
  int sub;    // its group's number among those of a row
  int part;   // its number among the head's lanes
  bool on;    // whether there is a head for it
  int kv;     // its key head
  int head;   // its first query head
  int n_q;    // how many query heads
  int local;  // the first one's number within the wavefront
};

template <int GQ, int COLS>
struct State {
  float m[GQ], l[GQ], acc[GQ][COLS];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int g = 0; g < GQ; ++g) {
      m[g] = -INFINITY;
      l[g] = 0.f;
#pragma unroll
      for (int j = 0; j < COLS; ++j) acc[g][j] = 0.f;
    }
  }
};

__device__ __forceinline__ float exp_diff(float a, float b) { return __builtin_amdgcn_exp2f((a - b) * kLog2E); }
__device__ __forceinline__ float log_of(float x) { return __builtin_amdgcn_logf(x) * 0.69314718055994530942f; }
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.f ? -INFINITY : m + log_of(l); }
__device__ __forceinline__ float finite_or_0(float m) { return m == -INFINITY ? 0.f : m; }

// The last rows that begin at or before entries p and p2 >= p (so those that hold them, if any do); n >= 1, wavefront-wide
__device__ __forceinline__ void rows_holding(const long long* __restrict__ indptr, long long n, long long p, long long p2, long long* row, long long* row2) {
  long long lo = 0, hi = n, lo2 = 0, hi2 = n;
  while (hi - lo > 1 || hi2 - lo2 > 1) {
    const long long step = (hi - lo + kWave - 1) / kWave, step2 = (hi2 - lo2 + kWave - 1) / kWave;
    const long long at = lo + lane_id() * step, at2 = lo2 + lane_id() * step2;
    const bool before = at < hi && indptr[at] <= p, before2 = at2 < hi2 && indptr[at2] <= p2;
    const int c = __popcll(__ballot(before)), c2 = __popcll(__ballot(before2));  // prefixes of the lanes, as indptr ascends
    if (c) lo += (c - 1) * step;
    hi = min(hi, lo + (c ? step : 1));
    if (c2) lo2 += (c2 - 1) * step2;
    hi2 = min(hi2, lo2 + (c2 ? step2 : 1));
  }
  *row = lo;
  *row2 = lo2;
}

// do_piece(row, b, e) for every list [b, e) of more than short_list entries that has some in [c0, c1)
template <class F>
__device__ __forceinline__ void for_long_lists(const Attn& a, long long n, long long c0, long long c1, const F& do_piece) {
  long long first, last;
  rows_holding(a.indptr, n, c0, c1 - 1, &first, &last);
  for (long long row0 = first; row0 <= last; row0 += kWave) {
    const long long row = row0 + lane_id();
    long long b = 0, e = 0;
    if (row <= last) {
      b = a.indptr[row];
      e = min(min(a.n_edges, a.indptr[row + 1]), b + a.longest);
    }
    for (unsigned long long todo = __ballot(b >= 0 && e - b > a.short_list && e > c0 && b < c1); todo; todo &= todo - 1) {
      const int i = __builtin_ctzll(todo);
      do_piece(row0 + i, __shfl(b, i, kWave), __shfl(e, i, kWave));
    }
  }
}

// What entry-holding lane: the row of k and v that source s stands for, -1: none
__device__ __forceinline__ int named(const Attn& a, int s) {
  const bool in = (unsigned)s < a.n_src;
  const int at = a.slots ? a.slots[in ? s : 0] : s;
  return in && (unsigned)at < a.n_at ? at : -1;
}

// The columns of a lane: piece j, kPiece<TYPE> columns from first_column on, if there are any left for it (then `some`); all of them where
// heads are too narrow for a piece (!WIDE)
template <int TYPE>
constexpr int kPiece = 16 / type_bytes(TYPE);
template <int TYPE>
constexpr int kPieces = kCols<TYPE> / kPiece<TYPE>;
template <int TYPE, bool WIDE>
__device__ __forceinline__ int first_column(const Attn& a, const Place& pl, int j, bool* some, int* skip) {
  if (!WIDE) {
    *some = pl.part == 0 && j == 0;
    *skip = 0;
    return 0;
  }
  const int c = ((j << a.lh_log2) + pl.part) * kPiece<TYPE>, col = min(c, a.dim - kPiece<TYPE>);
  *some = c < a.dim;
  *skip = c - col;  // columns that are another piece's
  return col;
}
// A lane's columns of a row of the cache, whose heads are padded to whole pieces
__device__ __forceinline__ int cached_column(const Attn& a, const Place& pl) {
  return pl.part * kChunk < a.dim ? pl.part * kChunk : 0;
}

// Entries [e0, e1) that are gone through: none where nothing can be named
__device__ __forceinline__ int entries(const Attn& a, long long e0, long long e1) {
  return a.n_at > 0 && a.n_src > 0 ? (int)max(0ll, min(e1 - e0, 0x7FFFFFFFll - 8192)) : 0;
}
// The source of a lane's first entry of them
__device__ __forceinline__ int first_source(const Attn& a, const Place& pl, long long e0, long long e1, int r_log2) {
  const int t = ((lane_id() & ((1 << a.p_log2) - 1)) << r_log2) + pl.sub;
  return t < entries(a, e0, e1) ? a.src[e0 + t] : -1;
}

// Which columns of a piece of a dense row are the lane's own, as masks of its words.  (q has a 0 for the others, but 0 times an infinite key is no number.
// The masks cost 24,576 rows of nine entries up to 5 % where heads do not fill their lanes, eight 16-bit heads of 40 on four 36 -> 37 us, and 1 %
// on average where they do; made anew for each entry, as those of 32-bit rows are, they cost 16-bit ones up to 13 %.)
template <int TYPE>
struct Own {
  static constexpr int kMasks = TYPE == DCI_F32 ? 1 : 4;
  unsigned at[kMasks];  // of fp32 rows the first of them: a mask to a word would take registers that are not there

  __device__ __forceinline__ void set(const Attn& a, const Place& pl, int j) {
    bool some;
    int skip;
    (void)first_column<TYPE, true>(a, pl, j, &some, &skip);
    const int first = some ? skip : kPiece<TYPE>;
    if (TYPE == DCI_F32) at[0] = (unsigned)first;
#pragma unroll
    for (int i = 0; i < kMasks && TYPE != DCI_F32; ++i) {
      at[i] = first <= 2 * i ? ~0u : first == 2 * i + 1 ? 0xFFFF0000u : 0u;
      asm volatile("" : "+v"(at[i]));
    }
  }
  __device__ __forceinline__ uint4 of(uint4 w) const {
    if (TYPE != DCI_F32) return make_uint4(w.x & at[0], w.y & at[kMasks > 1 ? 1 : 0], w.z & at[kMasks > 2 ? 2 : 0], w.w & at[kMasks > 3 ? 3 : 0]);
    int first = (int)at[0];
    asm volatile("" : "+v"(first));
    auto own = [&](int i) { return (unsigned)((first - i - 1) >> 31); };
    return make_uint4(w.x & own(0), w.y & own(1), w.z & own(2), w.w & own(3));
  }
};

// Entries [e0, e1) of one row into st (source0: their first_source): those of group `sub` are every (1 << r_log2)-th from e0 + sub on.  Returns what the lane's entry of the last
// P << r_log2 named (there are no more where that is used).  stash (nullable): LDS for the scores, entry by entry of the wavefront; scores (nullable):
// memory for them, entry by entry of the call.
template <int TYPE, int GQ, bool BIAS, bool WIDE>
__device__ __forceinline__ int attend(const Attn& a, const Place& pl, long long e0, long long e1, int r_log2, int source0, const float (&q)[GQ][kCols<TYPE>],
                                      State<GQ, kCols<TYPE>>& st, float* stash, float* scores) {
  constexpr int U = WIDE || TYPE == kE4M3 ? 4 : 1, C = kCols<TYPE>;  // entries at a time
  const int n = entries(a, e0, e1);
  const int* __restrict__ src = a.src + e0;
  const int lane = lane_id(), in = lane & ((1 << a.p_log2) - 1), base = lane - in;
  const int batch = 1 << (a.p_log2 + r_log2), first = (in << r_log2) + pl.sub;
  auto source = [&](int t) { return t < n ? src[t] : -1; };
  int next = -1, after = source(first + batch);
  if (n > 0) next = named(a, source0);
  const int width = TYPE == kE4M3 ? (a.dim + kChunk - 1) / kChunk * kChunk : a.dim;
  const char *k0 = a.k + (long long)(pl.kv * width) * type_bytes(TYPE), *v0 = a.v + (long long)(pl.kv * width) * type_bytes(TYPE);
  int offset[Chunk<TYPE, C>::kWords];
#pragma unroll
  for (int j = 0; j < Chunk<TYPE, C>::kWords; ++j) {
    bool some;
    int skip;
    offset[j] = (TYPE == kE4M3 ? cached_column(a, pl) : first_column<TYPE, WIDE>(a, pl, j, &some, &skip)) * type_bytes(TYPE);
  }
  Own<TYPE> own[Chunk<TYPE, C>::kWords];
  if (TYPE != kE4M3 && WIDE) {
#pragma unroll
    for (int j = 0; j < Chunk<TYPE, C>::kWords; ++j) own[j].set(a, pl, j);
  }
  if (TYPE == kE4M3) {
    k0 += offset[0];
    v0 += offset[0];
  }
  const char* s0 = reinterpret_cast<const char*>(a.scales + 2 * pl.kv);
  const unsigned s_stride = 8u * a.kv_heads;
  int now = -1;
  for (int t0 = 0; t0 < n; t0 += batch) {
    now = next;
    next = named(a, after);
    after = source(t0 + 2 * batch + first);
    const int mine = min(1 << a.p_log2, (n - t0 - pl.sub + (1 << r_log2) - 1) >> r_log2);  // entries of this group
    for (int u0 = 0; u0 < mine; u0 += U) {
      Chunk<TYPE, C> kc[U], vc[U];
      float ks[U], vs[U], bias[U][GQ];
      bool there[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int at = __shfl(now, base + u0 + u, kWave);
        there[u] = at >= 0;
        const unsigned row = there[u] ? (unsigned)at : 0u;
        ks[u] = vs[u] = 1.f;
        const char *pk = k0 + (unsigned long long)row * a.k_stride, *pv = v0 + (unsigned long long)row * a.v_stride;
        if (TYPE == kE4M3) {
          kc[u].load(pk);
          vc[u].load(pv);
        } else if (WIDE) {
#pragma unroll
          for (int j = 0; j < Chunk<TYPE, C>::kWords; ++j) kc[u].w[j] = load_16(pk + offset[j]);
#pragma unroll
          for (int j = 0; j < Chunk<TYPE, C>::kWords; ++j) vc[u].w[j] = load_16(pv + offset[j]);
        } else {
          kc[u].load(pk, a.dim, false);
          vc[u].load(pv, a.dim, false);
        }
        if (TYPE == kE4M3) {
          const float2 s = *reinterpret_cast<const float2*>(s0 + (unsigned long long)(row >> a.block_log2) * s_stride);
          ks[u] = s.x;
          vs[u] = s.y;
        }
        if (BIAS) {
          const int t = t0 + ((u0 + u) << r_log2) + pl.sub;
#pragma unroll
          for (int g = 0; g < GQ; ++g)
            bias[u][g] = there[u] && g < pl.n_q ? a.bias[(e0 + t) * a.bias_heads + (a.bias_heads > 1 ? pl.head + g : 0)] : 0.f;
        }
      }
      // (an entry after the other: numbers made of all entries' bytes ahead of their use would not fit the registers)
      __builtin_amdgcn_sched_barrier(0);
      float z[U][GQ];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (TYPE != kE4M3 && WIDE && a.ragged) {  // q has a 0 for the others, but 0 times an infinity is no number
#pragma unroll
          for (int j = 0; j < Chunk<TYPE, C>::kWords; ++j) kc[u].w[j] = own[j].of(kc[u].w[j]);
        }
#pragma unroll
        for (int g = 0; g < GQ; ++g) z[u][g] = 0.f;
#pragma unroll
        for (int j = 0; j < C / 2; ++j) {
          float x, y;
          kc[u].pair(j, x, y);
#pragma unroll
          for (int g = 0; g < GQ; ++g) z[u][g] = fmaf(q[g][2 * j + 1], y, fmaf(q[g][2 * j], x, z[u][g]));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      sum_lanes<U * GQ>(&z[0][0], a.lh_log2);
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int g = 0; g < GQ; ++g) {
          z[u][g] *= a.scale * ks[u];
          if (BIAS) z[u][g] = bias[u][g] == -INFINITY ? -INFINITY : z[u][g] + bias[u][g];
          if (!there[u]) z[u][g] = -INFINITY;
        }
        if (!there[u]) vc[u].clear();
      }
      if ((stash || scores) && pl.part == 0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int t = t0 + ((u0 + u) << r_log2) + pl.sub;
#pragma unroll
          for (int g = 0; g < GQ; ++g) {
            if (g < pl.n_q) {
              if (stash) stash[(base + u0 + u) * a.stash_row + pl.local + g] = z[u][g];
              if (scores && t < n) scores[(e0 + t) * a.heads + pl.head + g] = z[u][g];
            }
          }
        }
      }
      float p[U][GQ];
#pragma unroll
      for (int g = 0; g < GQ; ++g) {
        float m = st.m[g];
#pragma unroll
        for (int u = 0; u < U; ++u) m = fmaxf(m, z[u][g]);
        const float top = finite_or_0(m), shrink = exp_diff(st.m[g], top);
        st.m[g] = m;
        st.l[g] *= shrink;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          p[u][g] = exp_diff(z[u][g], top);
          st.l[g] += p[u][g];
          p[u][g] *= vs[u];
        }
#pragma unroll
        for (int j = 0; j < C; ++j) st.acc[g][j] *= shrink;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        // with a bias an entry may be left out for one head and not for the next: its values, whatever they are, then add nothing
        bool with[GQ];
#pragma unroll
        for (int g = 0; g < GQ; ++g) with[g] = !BIAS || z[u][g] != -INFINITY;
#pragma unroll
        for (int j = 0; j < C / 2; ++j) {
          float x, y;
          vc[u].pair(j, x, y);
#pragma unroll
          for (int g = 0; g < GQ; ++g) {
            if (with[g]) {
              st.acc[g][2 * j] = fmaf(p[u][g], x, st.acc[g][2 * j]);
              st.acc[g][2 * j + 1] = fmaf(p[u][g], y, st.acc[g][2 * j + 1]);
            }
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  return now;
}

// (m, l, acc) of lanes `apart` away joined into st
template <int GQ, int COLS>
__device__ __forceinline__ void join_lanes(State<GQ, COLS>& st, int apart) {
#pragma unroll
  for (int g = 0; g < GQ; ++g) {
    const float m2 = __shfl_xor(st.m[g], apart, kWave), l2 = __shfl_xor(st.l[g], apart, kWave);
    const float m = fmaxf(st.m[g], m2), base = finite_or_0(m);
    const float f1 = exp_diff(st.m[g], base), f2 = exp_diff(m2, base);
    st.m[g] = m;
    st.l[g] = st.l[g] * f1 + l2 * f2;
#pragma unroll
    for (int j = 0; j < COLS; ++j) {
      const float other = __shfl_xor(st.acc[g][j], apart, kWave);
      st.acc[g][j] = st.acc[g][j] * f1 + other * f2;
    }
  }
}

__device__ __forceinline__ void add_weight(const Attn& a, int at, float p) {
  if (p > 0.f && at >= 0) atomicAdd(a.weight + at, (unsigned long long)((double)p * kWeightUnit + 0.5));
}

// What a lane is there for in pass `pass` over the heads
template <int GQ>
__device__ __forceinline__ Place place_of(const Attn& a, int pass, int r_log2, int* heads_here, int* n_q) {
  const int in = lane_id() & ((1 << a.p_log2) - 1), g_id = lane_id() >> a.p_log2, h = in >> a.lh_log2;
  const int gq_part = pass % a.gq_passes, wave_part = pass / a.gq_passes;
  *heads_here = min(a.wave_heads, a.kv_heads - wave_part * a.wave_heads);
  *n_q = min(GQ, a.group - gq_part * GQ);
  Place pl;
  pl.on = h < *heads_here;
  pl.sub = g_id & ((1 << r_log2) - 1);
  pl.part = in & ((1 << a.lh_log2) - 1);
  pl.kv = pl.on ? wave_part * a.wave_heads + h : 0;
  pl.n_q = pl.on ? *n_q : 0;
  pl.head = pl.kv * a.group + gq_part * GQ;
  pl.local = h * GQ;
  return pl;
}

template <int TYPE, int GQ, bool WIDE>
__device__ __forceinline__ void read_q(const Attn& a, const Place& pl, long long row, bool real, float (&q)[GQ][kCols<TYPE>]) {
#pragma unroll
  for (int g = 0; g < GQ; ++g) {
    const char* p = a.q + row * a.q_stride + (long long)((pl.head + g) * a.dim) * type_bytes(a.type);
    const bool here = real && g < pl.n_q;
#pragma unroll
    for (int j = 0; j < kCols<TYPE>; ++j) q[g][j] = 0.f;
    if (!WIDE) {
      if (here && pl.part == 0) read_chunk(a.type, p, a.dim, false, q[g]);
      continue;
    }
#pragma unroll
    for (int j = 0; j < kPieces<TYPE>; ++j) {
      bool some;
      int skip;
      const int col = first_column<TYPE, WIDE>(a, pl, j, &some, &skip);
      if (here && some) {
        if (TYPE == kE4M3) {
          read_chunk(a.type, p + col * type_bytes(a.type), kChunk, true, q[g]);  // columns `skip` before those of the row of the cache
        } else {
          Chunk<TYPE, kPiece<TYPE>> c;
          c.w[0] = load_16(p + col * type_bytes(TYPE));
#pragma unroll
          for (int i = 0; i < kPiece<TYPE> / 2; ++i) c.pair(i, q[g][j * kPiece<TYPE> + 2 * i], q[g][j * kPiece<TYPE> + 2 * i + 1]);
        }
      }
      if (TYPE == kE4M3) {
        if (a.dim % kChunk) shift_down(q[g], skip & (kChunk - 1));
        continue;
      }
#pragma unroll
      for (int i = 0; i < kPiece<TYPE>; ++i)
        if (i < skip) q[g][j * kPiece<TYPE> + i] = 0.f;
    }
  }
}

// A lane's columns of a head of the output
template <int TYPE, bool WIDE>
__device__ __forceinline__ void write_out(const Attn& a, const Place& pl, char* p, const float (&y)[kCols<TYPE>]) {
  if (!WIDE) {
    if (pl.part == 0) write_chunk(a.type, p, a.dim, false, y);
    return;
  }
#pragma unroll
  for (int j = 0; j < kPieces<TYPE>; ++j) {
    bool some;
    int skip;
    const int col = first_column<TYPE, WIDE>(a, pl, j, &some, &skip);
    if (TYPE == kE4M3) {
      if (a.dim % kChunk == 0) {
        if (some) write_chunk(a.type, p + col * type_bytes(a.type), kChunk, true, y);
        continue;
      }
      // the head's last 16 columns: `skip` of the lane before (every lane takes part in the exchange), then its own
      float both[2 * kChunk];
#pragma unroll
      for (int i = 0; i < kChunk; ++i) {
        both[i] = dpp<0x111>(y[i]);  // of the lane before, in sixteen
        both[kChunk + i] = y[i];
      }
      shift_down(both, (kChunk - skip) & (kChunk - 1));
      float z[kChunk];
#pragma unroll
      for (int i = 0; i < kChunk; ++i) z[i] = skip ? both[i] : y[i];
      if (some) write_chunk(a.type, p + col * type_bytes(a.type), kChunk, true, z);
    } else if (!some) {
      continue;
    } else if (TYPE == DCI_F32) {
      store_16(p + col * 4, make_uint4(__float_as_uint(y[4 * j]), __float_as_uint(y[4 * j + 1]), __float_as_uint(y[4 * j + 2]), __float_as_uint(y[4 * j + 3])));
    } else {
      const int i = j * kPiece<TYPE>;
      store_16(p + col * 2, make_uint4(two<TYPE>(y[i], y[i + 1]), two<TYPE>(y[i + 2], y[i + 3]), two<TYPE>(y[i + 4], y[i + 5]), two<TYPE>(y[i + 6], y[i + 7])));
    }
  }
}

__device__ __forceinline__ long long rows_of(const Attn& a) { return a.n_dev ? min(a.n_rows, max(0ll, *a.n_dev)) : a.n_rows; }

// A row's sum is its output
template <int TYPE, int GQ, bool WIDE>
__device__ __forceinline__ void finish_row(const Attn& a, const Place& pl, long long row, const State<GQ, kCols<TYPE>>& st) {
#pragma unroll
  for (int g = 0; g < GQ; ++g) {
    if (g < pl.n_q) {
      const float inv = st.l[g] == 0.f ? 0.f : __builtin_amdgcn_rcpf(st.l[g]);
      float y[kCols<TYPE>];
#pragma unroll
      for (int j = 0; j < kCols<TYPE>; ++j) y[j] = st.acc[g][j] * inv;
      write_out<TYPE, WIDE>(a, pl, a.out + row * a.out_stride + (long long)((pl.head + g) * a.dim) * type_bytes(a.type), y);
      if (pl.part == 0) {
        const float lse = lse_of(st.m[g], st.l[g]);
        if (a.lse) a.lse[row * a.heads + pl.head + g] = lse;
        if (a.all_lse) a.all_lse[row * a.heads + pl.head + g] = lse;
      }
    }
  }
}

// A chunk to a wavefront: what long lists have there
template <int TYPE, int GQ, bool BIAS, bool WIDE>
__global__ __launch_bounds__(kAttnBlock, waves_per_simd(TYPE, GQ)) void k_attn_chunks(const Attn a) {
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), p_lanes = 1 << a.p_log2;
  const unsigned unit = blockIdx.x * kAttnWaves + wave, c = unit / (unsigned)a.passes;  // wavefronts side by side read the same rows
  int heads_here, n_q;
  const Place pl = place_of<GQ>(a, (int)(unit - c * a.passes), 6 - a.p_log2, &heads_here, &n_q);
  const long long n = rows_of(a);
  if (c >= (unsigned)a.n_chunks || n == 0) return;
  const long long c0 = (long long)c * a.chunk, c1 = min(c0 + a.chunk, min(a.n_edges, a.indptr[n]));
  if (c0 >= c1) return;
  for_long_lists(a, n, c0, c1, [&](long long row, long long b, long long e) {
    const int source0 = first_source(a, pl, max(b, c0), min(e, c1), 6 - a.p_log2);
    float q[GQ][kCols<TYPE>];
    read_q<TYPE, GQ, WIDE>(a, pl, row, true, q);
    State<GQ, kCols<TYPE>> st;
    st.clear();
    (void)attend<TYPE, GQ, BIAS, WIDE>(a, pl, max(b, c0), min(e, c1), 6 - a.p_log2, source0, q, st, nullptr, a.scores);
    for (int apart = p_lanes; apart < kWave; apart <<= 1) join_lanes(st, apart);
    if (lane_id() >= p_lanes) return;
    if (b >= c0 && e <= c1) {
      finish_row<TYPE, GQ, WIDE>(a, pl, row, st);
      return;
    }
#pragma unroll
    for (int g = 0; g < GQ; ++g) {
      if (g < pl.n_q) {
        const long long at = (2 * (long long)c + (b > c0 ? 1 : 0)) * a.heads + pl.head + g;
        if (pl.part == 0) {
          a.part_ml[2 * at] = st.m[g];
          a.part_ml[2 * at + 1] = st.l[g];
        }
        float* acc = a.part_acc + at * ((a.dim + kChunk - 1) / kChunk * kChunk);
#pragma unroll
        for (int j = 0; j < kPieces<TYPE>; ++j) {
          bool some;
          int skip;
          int col = first_column<TYPE, WIDE>(a, pl, j, &some, &skip);
          if (!some) continue;
          if (TYPE == kE4M3) col = cached_column(a, pl);
#pragma unroll
          for (int i = 0; i < (WIDE ? kPiece<TYPE> : kCols<TYPE>); i += 4)
            store_16(reinterpret_cast<char*>(acc + col + i), make_uint4(__float_as_uint(st.acc[g][j * kPiece<TYPE> + i]), __float_as_uint(st.acc[g][j * kPiece<TYPE> + i + 1]),
                                                                        __float_as_uint(st.acc[g][j * kPiece<TYPE> + i + 2]), __float_as_uint(st.acc[g][j * kPiece<TYPE> + i + 3])));
        }
      }
    }
  });
}

// Rows, one or more to a wavefront, one set after the other; long lists are not its business
template <int TYPE, int GQ, bool BIAS, bool WIDE>
__global__ __launch_bounds__(kAttnBlock, waves_per_simd(TYPE, GQ)) void k_attn_rows(const Attn a) {
  extern __shared__ float stash_all[];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const int p_lanes = 1 << a.p_log2, groups = kWave >> a.p_log2, g_id = lane >> a.p_log2, r_log2 = a.r_log2;
  const unsigned unit = blockIdx.x * kAttnWaves + wave, turn = unit / (unsigned)a.passes;
  int heads_here, n_q;
  const Place pl = place_of<GQ>(a, (int)(unit - turn * a.passes), r_log2, &heads_here, &n_q);
  const long long n = rows_of(a);
  const int at_once = groups >> r_log2;
  const unsigned turns = (unsigned)((n + at_once - 1) / at_once), step = gridDim.x * kAttnWaves / (unsigned)a.passes;
  float* stash = stash_all + wave * (kWave + groups) * a.stash_row;
  // the bounds of the next rows are on their way while these are worked on, and so are, once these have been read, the next ones' sources
  auto bounds = [&](unsigned k, long long* b, long long* e) {
    const long long row = (long long)k * at_once + (g_id >> r_log2);
    *b = *e = 0;
    if (k < turns && row < n) {
      *b = a.indptr[row];
      *e = a.indptr[row + 1];
    }
  };
  auto settle = [&](long long* b, long long* e) {  // false for a long list
    *b = max(0ll, *b);
    *e = max(*b, min(min(a.n_edges, *e), *b + a.longest));
    const bool here = !(a.n_chunks && *e - *b > a.short_list);
    if (!here) *e = *b;
    return here;
  };
  long long b, e;
  bounds(turn, &b, &e);
  bool here = settle(&b, &e);
  int source0 = first_source(a, pl, b, e, r_log2);
  for (unsigned k = turn; k < turns; k += step) {
    const long long row = (long long)k * at_once + (g_id >> r_log2);
    const bool mine = row < n && here;
    long long next_b, next_e;
    bounds(k + step >= k ? k + step : turns, &next_b, &next_e);
    if (!__any(mine)) {  // long lists only
      here = settle(&next_b, &next_e);
      b = next_b;
      e = next_e;
      source0 = first_source(a, pl, b, e, r_log2);
      continue;
    }
    float q[GQ][kCols<TYPE>];
    read_q<TYPE, GQ, WIDE>(a, pl, row, mine, q);
    State<GQ, kCols<TYPE>> st;
    st.clear();
    const int names = attend<TYPE, GQ, BIAS, WIDE>(a, pl, b, e, r_log2, source0, q, st, a.stash_row ? stash : nullptr, nullptr);
    here = settle(&next_b, &next_e);
    b = next_b;
    e = next_e;
    source0 = first_source(a, pl, b, e, r_log2);
    for (int apart = p_lanes; apart < p_lanes << r_log2; apart <<= 1) join_lanes(st, apart);
    if (mine && pl.sub == 0) finish_row<TYPE, GQ, WIDE>(a, pl, row, st);
    if (!a.stash_row) continue;
    float* lses = stash + (kWave + g_id) * a.stash_row;
    if (pl.part == 0) {
#pragma unroll
      for (int g = 0; g < GQ; ++g)
        if (g < pl.n_q) lses[pl.local + g] = lse_of(st.m[g], st.l[g]);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (names >= 0) {  // every lane its own entry, over the wavefront's heads
      const float* zs = stash + lane * a.stash_row;
      float p = 0.f;
      for (int h = 0; h < heads_here; ++h) {
#pragma unroll
        for (int g = 0; g < GQ; ++g) {
          if (g < n_q) {
            const float z = zs[h * GQ + g];
            if (z != -INFINITY) p += exp_diff(z, lses[h * GQ + g]);
          }
        }
      }
      add_weight(a, names, p);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// ---- long lists of the cache whose query heads share key heads: matrix instructions ----------------------------------------------------
//
// A wavefront takes a chunk, one key head and up to eight of its query heads, 32 entries at a time, in two tiles of 16:
//   scores     S^T = K Q^T, 16 entries by 16 columns, v_mfma_f32_16x16x32_bf16.  A lane (j = lane % 16, b = lane / 16) brings 16-byte pieces of
//              entry j's key as they lie in memory, piece b of every 64 columns; the order of the columns in the sum is free, so the query's
//              operand is laid out to match.  8-bit keys, times their scale, are bf16 numbers exactly; so is a query in one part (bf16), two
//              (fp16) or three (fp32).  Column j is query head j % H, so every head comes 16 / H times.
//   softmax    the lane that is left with a score holds four consecutive entries (4 b ..) of either tile, which is how the second product wants
//              its operand: nothing is exchanged but the maximum over b.  Rescaling waits until a maximum grows.
//   values     O = P V, 16 rows (column j of before) by 16 columns of V, 32 entries deep.  P is a sum of three bf16 numbers (2^-27 of it is lost):
//              part j / H of head j % H is row j, so the parts cost no instruction of their own.  Where H > 5 there are rows for two.  16-bit outputs
//              have no use for the third (2^-18 of P is lost, a 128th of half a step of fp16), fp32 ones get it in a second product with the same
//              operand (620,000 entries of eight key heads of 128 with 64 query heads 295 -> 299 us, of four of 64 with 32 96 -> 100; in passes
//              over four heads half as many take 256 for 165, and 85 for 57).  The value's scale is P's.  A lane brings W / 16 bytes of eight entries' values, side by side over j, pairs two entries' bytes with v_perm
//              and converts.
// At the end the parts of O are added up through LDS.  It does a quarter of the vector instructions of k_attn_chunks for four heads to a group:
// 620,000 entries of eight key heads of 128 with 32 query heads take 280 to 299 us, 380 by k_attn_chunks.  What bounds it are the rows, 1.5 GB there
// by the counters, 5 to 5.4 TB/s; 950,000 entries of four heads of 64 take 116 us at 4.9 TB/s, with 82 requests to L2 a nanosecond.
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ unsigned bf16_pair(float a, float b) { return two<DCI_BF16>(a, b); }
// The leading eight bits of x as bf16 in the upper half; x becomes what they leave (0 of an infinity and of what is no number)
__device__ __forceinline__ unsigned leading(float& x) {
  const unsigned u = __float_as_uint(x), h = u & 0xFFFF0000u;
  if ((u & 0x7F800000u) == 0x7F800000u) {
    x = 0.f;
    return u & 0x7FFFFFu ? 0x7FC00000u : h;
  }
  x -= __uint_as_float(h);
  return h;
}
// Two neighbouring codes, the lower or the higher two of w, times a power of two
__device__ __forceinline__ unsigned pair_of_codes(unsigned w, float scale, bool high) {
  return __builtin_bit_cast(unsigned, high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
}
// What lane I of the 16 has
template <int I>
__device__ __forceinline__ int of_lane(int x) {
  return __builtin_amdgcn_update_dpp(0, x, 0x150 + I, 0xF, 0xF, true);
}
template <int I>
__device__ __forceinline__ float of_lane(float x) {
  return __int_as_float(of_lane<I>(__float_as_int(x)));
}

// 32 entries as they come: the bytes that a lane has of their keys and values, the scales, where the values of the entry that it looks up for the 16 are
template <int W>
struct GroupStep {
  uint4 kc[2][W / 64];
  unsigned vc[8][W / 64];
  float ks[2], vs;
  int at_v;
  bool gone;  // not all of the 32 name something
};

template <int W, int NQ>
__global__ __launch_bounds__(kAttnBlock, W == 64 ? 3 : 2) void k_attn_groups(const Attn a) {
  constexpr int kBlocks = W / 64, kSteps = W / 32, kWords = W / 64, kTiles = W / 16;
  __shared__ float sum[kAttnWaves][16][W + 4];
  const int lane = lane_id(), j = lane & 15, b4 = lane >> 4, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const unsigned unit = blockIdx.x * kAttnWaves + wave, c = unit / (unsigned)a.passes, pass = unit - c * a.passes;
  const int kv = (int)pass / a.gq_passes, heads = a.pass_heads, h0 = (int)pass % a.gq_passes * heads;
  const int parts = heads <= 5 ? 3 : 2, part = j / heads;
  const bool add_rest = NQ == 3 && parts == 2;
  const bool used = part < parts && h0 + j % heads < a.group;
  const int head = kv * a.group + min(h0 + j % heads, a.group - 1);
  const long long n = rows_of(a);
  if (c >= (unsigned)a.n_chunks || n == 0) return;
  const long long c0 = (long long)c * a.chunk, c1 = min(c0 + a.chunk, min(a.n_edges, a.indptr[n]));
  if (c0 >= c1) return;
  const float measure = a.scale * kLog2E;
  const char *k0 = a.k + kv * W + b4 * 16, *v0 = a.v + kv * W + j * (W / 16), *s0 = reinterpret_cast<const char*>(a.scales + 2 * kv);
  const unsigned s_stride = 8u * a.kv_heads;
  for_long_lists(a, n, c0, c1, [&](long long row, long long b, long long e) {
    const long long e0 = max(b, c0);
    const int entries = (int)(min(e, c1) - e0);
    const int* __restrict__ src = a.src + e0;
    int names = lane < entries ? src[lane] : -1;
    // the query: what multiplies bytes 8 (s % 2) .. of block s / 2
    bf16x8 q[NQ][kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = 0.f;
      if (used)
        read_chunk(a.type, a.q + row * a.q_stride + (long long)(head * a.dim + (s / 2) * 64 + b4 * 16 + (s & 1) * 8) * type_bytes(a.type), 8, true, x);
#pragma unroll
      for (int p = 0; p < NQ; ++p) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (leading(x[2 * i]) >> 16) | leading(x[2 * i + 1]);
        q[p][s] = __builtin_bit_cast(bf16x8, w);
      }
    }
    names = named(a, names);
    float m = -INFINITY, l = 0.f;
    f32x4 o[kTiles];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    int names_now = names, source_next = kWave + lane < entries ? src[kWave + lane] : -1;
    // (the next 32 entries' bytes on their way meanwhile would take registers from the third and the second wavefront of a SIMD: 303 -> 326 us)
    auto load = [&](GroupStep<W>& s, int half) {
      int at_k[2];
      s.at_v = __shfl(names_now, half + ((j & 4) << 2) + b4 * 4 + (j & 3), kWave);  // lane j < 8: entry 4 b + j % 4 of tile j / 4
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        at_k[t] = max(0, __shfl(names_now, half + t * 16 + j, kWave));
        const char* p = k0 + (unsigned long long)(unsigned)at_k[t] * a.k_stride;
#pragma unroll
        for (int x = 0; x < kBlocks; ++x) s.kc[t][x] = load_16(p + x * 64);
        s.ks[t] = *reinterpret_cast<const float*>(s0 + (unsigned long long)((unsigned)at_k[t] >> a.block_log2) * s_stride);
      }
      s.gone = __any(s.at_v < 0);
      const int row_v = max(0, s.at_v);
      s.vs = *reinterpret_cast<const float*>(s0 + 4 + (unsigned long long)((unsigned)row_v >> a.block_log2) * s_stride);
#define DCI_EIGHT(DO_) DO_(0) DO_(1) DO_(2) DO_(3) DO_(4) DO_(5) DO_(6) DO_(7)
#define DCI_LOAD(I_)                                                                                \
  {                                                                                                 \
    const char* p = v0 + (unsigned long long)(unsigned)of_lane<I_>(row_v) * a.v_stride;             \
    if (kWords == 1) s.vc[I_][0] = *reinterpret_cast<const unsigned*>(p);                             \
    else if (kWords == 2) {                                                                         \
      const uint2 u = *reinterpret_cast<const uint2*>(p);                                           \
      s.vc[I_][0] = u.x;                                                                              \
      s.vc[I_][kWords > 1 ? 1 : 0] = u.y;                                                             \
    } else {                                                                                        \
      const uint4 u = load_16(p);                                                                   \
      s.vc[I_][0] = u.x;                                                                              \
      s.vc[I_][kWords > 1 ? 1 : 0] = u.y;                                                             \
      s.vc[I_][kWords > 2 ? 2 : 0] = u.z;                                                             \
      s.vc[I_][kWords > 2 ? 3 : 0] = u.w;                                                             \
    }                                                                                               \
  }
      DCI_EIGHT(DCI_LOAD)
#undef DCI_LOAD
    };
    auto work = [&](GroupStep<W>& s, int t0) {
      float z[8];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        f32x4 sum_t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < kSteps; ++x) {
          const uint4 w = s.kc[t][x / 2];
          const unsigned lo = x & 1 ? w.z : w.x, hi = x & 1 ? w.w : w.y;
          const u32x4 u = {pair_of_codes(lo, s.ks[t], false), pair_of_codes(lo, s.ks[t], true), pair_of_codes(hi, s.ks[t], false), pair_of_codes(hi, s.ks[t], true)};
#pragma unroll
          for (int p = 0; p < NQ; ++p) sum_t = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, u), q[p][x], sum_t, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) z[4 * t + i] = sum_t[i];
      }
      if (s.gone) {
#define DCI_GONE(I_)                                     \
  if (of_lane<I_>(s.at_v) < 0) {                           \
    z[I_] = -INFINITY;                                   \
    _Pragma("unroll") for (int x = 0; x < kWords; ++x) s.vc[I_][x] = 0; \
  }
        DCI_EIGHT(DCI_GONE)
#undef DCI_GONE
      }
      if (a.scores && used && part == 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int t = t0 + (i >> 2) * 16 + b4 * 4 + (i & 3);
          if (t < entries) a.scores[(e0 + t) * a.heads + head] = z[i] == -INFINITY ? z[i] : z[i] * a.scale;
        }
      }
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        z[i] = z[i] == -INFINITY ? z[i] : z[i] * measure;
        top = fmaxf(top, z[i]);
      }
      top = fmaxf(top, __shfl_xor(top, 16, kWave));
      top = fmaxf(top, __shfl_xor(top, 32, kWave));
      if (__any(top > m)) {
        const float next = fmaxf(m, top), shrink = __builtin_amdgcn_exp2f(m - finite_or_0(next));
        m = next;
        l *= shrink;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float f = __shfl(shrink, b4 * 4 + r, kWave);
#pragma unroll
          for (int i = 0; i < kTiles; ++i) o[i][r] *= f;
        }
      }
      const float base = finite_or_0(m);
      unsigned pw[4];
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[i] = __builtin_amdgcn_exp2f(z[i] - base);
        l += p[i];
      }
#define DCI_SCALE(I_) p[I_] *= of_lane<I_>(s.vs);
      DCI_EIGHT(DCI_SCALE)
#undef DCI_SCALE
#undef DCI_EIGHT
      unsigned rest[4];  // what two parts leave, for fp32 outputs
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float x = p[2 * i], y = p[2 * i + 1];
        unsigned w = bf16_pair(x, y);
        rest[i] = 0;
        if (part > 0 || add_rest) {
          x -= __uint_as_float(w << 16);
          y -= __uint_as_float(w & 0xFFFF0000u);
          const unsigned w1 = bf16_pair(x, y);
          unsigned w2 = 0;
          if (NQ == 3 || part > 1) w2 = bf16_pair(x - __uint_as_float(w1 << 16), y - __uint_as_float(w1 & 0xFFFF0000u));
          if (add_rest) rest[i] = used && part == 0 ? w2 : 0;
          if (part > 0) w = part > 1 ? w2 : w1;
        }
        pw[i] = used ? w : 0;
      }
      const bf16x8 pa = __builtin_bit_cast(bf16x8, (u32x4{pw[0], pw[1], pw[2], pw[3]})), pr = __builtin_bit_cast(bf16x8, (u32x4{rest[0], rest[1], rest[2], rest[3]}));
#pragma unroll
      for (int x = 0; x < kWords; ++x) {
        unsigned low[4], high[4];  // two entries' bytes 0 0' 1 1', 2 2' 3 3'
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          low[i] = __builtin_amdgcn_perm(s.vc[2 * i + 1][x], s.vc[2 * i][x], 0x05010400u);
          high[i] = __builtin_amdgcn_perm(s.vc[2 * i + 1][x], s.vc[2 * i][x], 0x07030602u);
        }
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          u32x4 u;
#pragma unroll
          for (int i = 0; i < 4; ++i) u[i] = pair_of_codes(d < 2 ? low[i] : high[i], 1.f, d & 1);
          o[4 * x + d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pa, __builtin_bit_cast(bf16x8, u), o[4 * x + d], 0, 0, 0);
          if (add_rest) o[4 * x + d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pr, __builtin_bit_cast(bf16x8, u), o[4 * x + d], 0, 0, 0);
        }
      }
    };
    for (int t0 = 0; t0 < entries; t0 += 32) {
      if (t0 % kWave == 0 && t0) {
        names_now = named(a, source_next);
        source_next = t0 + kWave + lane < entries ? src[t0 + kWave + lane] : -1;
      }
      GroupStep<W> s;
      load(s, t0 & 32);
      work(s, t0);
    }
    l += __shfl_xor(l, 16, kWave);
    l += __shfl_xor(l, 32, kWave);
    const bool whole = b >= c0 && e <= c1;  // the list lies in the chunk
    const long long at0 = (2 * (long long)c + (b > c0 ? 1 : 0)) * a.heads;
    m *= 0.69314718055994530942f;
    if (used && part == 0 && b4 == 0) {
      if (whole) {
        if (a.lse) a.lse[row * a.heads + head] = lse_of(m, l);
        if (a.all_lse) a.all_lse[row * a.heads + head] = lse_of(m, l);
      } else {
        a.part_ml[2 * (at0 + head)] = m;
        a.part_ml[2 * (at0 + head) + 1] = l;
      }
    }
    // row 4 b + r, columns j (W / 16) + 4 x + d
#pragma unroll
    for (int r = 0; r < 4; ++r) {
#pragma unroll
      for (int x = 0; x < kWords; ++x)
        *reinterpret_cast<float4*>(&sum[wave][b4 * 4 + r][j * (W / 16) + 4 * x]) = make_float4(o[4 * x][r], o[4 * x + 1][r], o[4 * x + 2][r], o[4 * x + 3][r]);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    for (int h = 0; h < heads && h0 + h < a.group; ++h) {
      const float sum_h = __shfl(l, h, kWave), inv = sum_h == 0.f ? 0.f : __builtin_amdgcn_rcpf(sum_h);
      const int at_head = kv * a.group + h0 + h;
      for (int col = lane * 4; col < W; col += kWave * 4) {
        float4 y = *reinterpret_cast<const float4*>(&sum[wave][h][col]);
        for (int p = 1; p < parts; ++p) {
          const float4 x = *reinterpret_cast<const float4*>(&sum[wave][h + p * heads][col]);
          y = make_float4(y.x + x.x, y.y + x.y, y.z + x.z, y.w + x.w);
        }
        if (!whole) {
          *reinterpret_cast<float4*>(a.part_acc + (at0 + at_head) * W + col) = y;
        } else {
          const float out[4] = {y.x * inv, y.y * inv, y.z * inv, y.w * inv};
          write_chunk(a.type, a.out + row * a.out_stride + (long long)(at_head * W + col) * type_bytes(a.type), 4, false, out);
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  });
}

// One workgroup per row and head, or, where there are fewer of them, per chunk and head, for the long list that begins in the chunk and goes on behind
// it: the list's pieces added up in order.  Their weights exp(m - max) are made 256 at a time, in LDS; columns lie side by side, in as many slices of
// the pieces as the workgroup has room for.  11 to 16 us behind long lists, a third of that the launch.
__global__ __launch_bounds__(kAttnBlock) void k_attn_join(const Attn a, bool by_row) {
  const int head = (int)(blockIdx.x % (unsigned)a.heads);
  const long long n = rows_of(a);
  long long row = blockIdx.x / (unsigned)a.heads;
  if (by_row) {
    if (row >= n) return;
  } else {
    if (n == 0) return;
    const long long c0 = row * a.chunk, c1 = min(c0 + a.chunk, min(a.n_edges, a.indptr[n]));
    if (c0 >= c1) return;
    rows_holding(a.indptr, n, c1 - 1, c1 - 1, &row, &row);
    if (a.indptr[row] < c0) return;
  }
  const long long b = a.indptr[row], e = min(min(a.n_edges, a.indptr[row + 1]), b + a.longest);
  const bool nothing = e <= b && a.short_list == 0;  // no chunk has anything of it
  if (b < 0 || (e - b <= a.short_list && !nothing)) return;
  const long long c = b / a.chunk;
  if (!nothing && c == (e - 1) / a.chunk) return;  // done in its chunk
  const int width = (a.dim + kChunk - 1) / kChunk * kChunk;
  const int pieces = nothing ? 0 : (int)((e - 1) / a.chunk - c) + 1;
  auto place = [&](int k) { return (2 * (c + k) + (k == 0 && b != c * a.chunk ? 1 : 0)) * a.heads + head; };
  __shared__ float4 part[kAttnBlock];
  __shared__ float red[kAttnWaves], weights[kAttnBlock];
  const int lane = lane_id(), wave = (int)threadIdx.x / kWave;
  float m = -INFINITY;
  for (int k = (int)threadIdx.x; k < pieces; k += kAttnBlock) m = fmaxf(m, a.part_ml[2 * place(k)]);
  for (int d = kWave / 2; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, kWave));
  if (lane == 0) red[wave] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kAttnWaves; ++w) m = fmaxf(m, red[w]);
  const float top = finite_or_0(m);
  int lanes = 4;  // lanes to a piece, four columns to a lane
  while (lanes * 4 < width) lanes <<= 1;
  const int slices = kAttnBlock / lanes, col = ((int)threadIdx.x & (lanes - 1)) * 4, slice = (int)threadIdx.x / lanes;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  float l = 0.f;
  for (int k0 = 0; k0 < pieces; k0 += kAttnBlock) {
    const int k = k0 + (int)threadIdx.x;
    float w = 0.f;
    if (k < pieces) {
      const long long at = place(k);
      w = exp_diff(a.part_ml[2 * at], top);
      l += a.part_ml[2 * at + 1] * w;
    }
    __syncthreads();
    weights[threadIdx.x] = w;
    __syncthreads();
    if (col < width) {
      const int end = min(kAttnBlock, pieces - k0);
#pragma unroll 8
      for (int i = slice; i < end; i += slices) {
        const float4 x = *reinterpret_cast<const float4*>(a.part_acc + place(k0 + i) * width + col);
        const float f = weights[i];
        acc = make_float4(fmaf(x.x, f, acc.x), fmaf(x.y, f, acc.y), fmaf(x.z, f, acc.z), fmaf(x.w, f, acc.w));
      }
    }
  }
  for (int d = kWave / 2; d; d >>= 1) l += __shfl_xor(l, d, kWave);
  __syncthreads();
  if (lane == 0) red[wave] = l;
  part[threadIdx.x] = acc;
  __syncthreads();
  l = 0.f;
#pragma unroll
  for (int w = 0; w < kAttnWaves; ++w) l += red[w];
  if (slice == 0 && col < a.dim) {
    for (int s = 1; s < slices; ++s) {
      const float4 x = part[s * lanes + col / 4];
      acc = make_float4(acc.x + x.x, acc.y + x.y, acc.z + x.z, acc.w + x.w);
    }
    const float inv = l == 0.f ? 0.f : 1.f / l, y[4] = {acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv};
    write_chunk(a.type, a.out + row * a.out_stride + ((long long)head * a.dim + col) * type_bytes(a.type), min(4, a.dim - col), false, y);
  }
  if (threadIdx.x == 0) {
    const float lse = lse_of(m, l);
    if (a.lse) a.lse[row * a.heads + head] = lse;
    if (a.all_lse) a.all_lse[row * a.heads + head] = lse;
  }
}

// Accumulated weights of the long lists, an entry to a lane
__global__ __launch_bounds__(kAttnBlock) void k_attn_weights(const Attn a) {
  const long long c = (long long)blockIdx.x * kAttnWaves + threadIdx.x / kWave;
  const long long n = rows_of(a);
  if (c >= a.n_chunks || n == 0) return;
  const long long c0 = c * a.chunk, c1 = min(c0 + a.chunk, min(a.n_edges, a.indptr[n]));
  if (c0 >= c1) return;
  for_long_lists(a, n, c0, c1, [&](long long row, long long b, long long e) {
    const long long to = min(e, c1);
    for (long long t = max(b, c0) + lane_id(); t < to; t += kWave) {
      float p = 0.f;
      for (int h = 0; h < a.heads; ++h) {
        const float z = a.scores[t * a.heads + h];
        if (z != -INFINITY) p += exp_diff(z, a.all_lse[row * a.heads + h]);
      }
      add_weight(a, named(a, a.src[t]), p);
    }
  });
}

// How a call's work is cut, from its arguments alone (the workspace query has no context)
struct Split {
  bool matrix;  // long lists go to k_attn_groups
  int p_log2, lh_log2, wave_heads, gq, gq_passes, passes;
  bool wide;  // heads of 16 bytes at least: read and written 16 at a time
  int chunk;
  int64_t n_chunks;
  int64_t most_chunks;  // that this call or one of fewer entries has, which may be cut shorter
};
constexpr int64_t kMaxGroups = 0xFFFFFFFFll / kAttnBlock;  // workgroups to a launch: its lanes are counted in 32 bits, and one of more runs too few
constexpr int64_t kWantedWaves = 4096, kFewWaves = 1024;  // 16 and four to a compute unit
constexpr int kStashHeads = 32;  // query heads of a wavefront, at most, with weights: 40 KB of scores to a workgroup, four workgroups to a compute unit

// type: of k and v
Split split_of(const dci_attn& t, int type, bool accumulate) {
  Split s;
  const int cols = type == kE4M3 ? kCols<kE4M3> : kCols<DCI_F32>;
  const bool wide = t.head_dim * type_bytes(type) >= 16;
  s.wide = wide;
  const int group = t.n_heads / t.kv_heads, gq = group == 1 ? 1 : group == 2 ? 2 : 4;
  s.gq = wide ? gq : 1;
  s.gq_passes = (group + s.gq - 1) / s.gq;
  s.lh_log2 = log2_up((t.head_dim + cols - 1) / cols);
  s.wave_heads = kWave >> s.lh_log2;
  if (accumulate && s.wave_heads > kStashHeads / gq) s.wave_heads = kStashHeads / gq;
  if (s.wave_heads > t.kv_heads) s.wave_heads = t.kv_heads;
  s.p_log2 = log2_up((int64_t)s.wave_heads << s.lh_log2);
  if (s.p_log2 < 2) s.p_log2 = 2;  // entries are taken four at a time
  s.passes = (t.kv_heads + s.wave_heads - 1) / s.wave_heads * s.gq_passes;
  // To k_attn_groups from three query heads to a key head on: 620,000 entries of eight key heads of 128 take 297 us there for three to a group and 385 in
  // k_attn_chunks, 306 and 700 for eight; for two 294 and 261 (950,000 entries of four of 64: 132 and 169, 146 and 289; 127 and 114).
  s.matrix = type == kE4M3 && group >= 3 && !t.bias && (t.head_dim == 64 || t.head_dim == 128 || t.head_dim == 256);
  const int64_t waves = s.matrix ? (int64_t)t.kv_heads * ((group + 7) / 8) : ((int64_t)t.kv_heads * kv_width(t.head_dim) + 1023) / 1024 * ((group + gq - 1) / gq);
  // Chunks of 64 to 512 entries: as long as there are wavefronts enough (with half as many 620,000 entries of eight heads of 128, two query heads to
  // each, take 309 us for 261).  Shorter ones (16 or 32; a step of k_attn_groups is 32 entries) where that leaves only a few to a compute unit: 28,000
  // entries of seven 32-bit heads of 64 take 48 us in chunks of 32 and 55 in chunks of 64.  With more wavefronts the pieces cost more than they give:
  // 37,000 entries of eight 16-bit heads of 128 on two take 46 us in chunks of 16, 38 in 32, 37 in 64.
  int64_t most = 0;
  for (s.chunk = s.matrix ? 32 : 16; s.chunk < 512; s.chunk *= 2) {
    const int64_t wanted = s.chunk < 64 ? kFewWaves : kWantedWaves;
    if (t.n_edges / s.chunk * waves <= wanted) break;
    if (wanted / waves + 1 > most) most = wanted / waves + 1;
  }
  // Longer ones where the join, a workgroup to a chunk and head, would have more workgroups than a launch may have; no other launch has more.
  for (; (t.n_edges + s.chunk - 1) / s.chunk * t.n_heads > kMaxGroups; s.chunk *= 2) most = kMaxGroups / t.n_heads;
  const int64_t longest = t.max_list > 0 && t.max_list < t.n_edges ? t.max_list : t.n_edges;
  s.n_chunks = longest > kShort ? (t.n_edges + s.chunk - 1) / s.chunk : 0;
  s.most_chunks = s.n_chunks && most > s.n_chunks ? most : s.n_chunks;
  return s;
}

struct Parts {
  float *scores = nullptr, *all_lse = nullptr, *ml = nullptr, *acc = nullptr;
};
Parts take_parts(Arena& ar, const dci_attn& t, int64_t n_chunks, bool accumulate) {
  Parts p;
  if (n_chunks) {
    if (accumulate) p.scores = ar.take<float>((size_t)t.n_edges * t.n_heads);
    if (accumulate) p.all_lse = ar.take<float>((size_t)t.n_rows * t.n_heads);
    p.ml = ar.take<float>((size_t)n_chunks * 2 * t.n_heads * 2);
    p.acc = ar.take<float>((size_t)n_chunks * 2 * t.n_heads * kv_width(t.head_dim));
  }
  return p;
}

constexpr int64_t kMaxEdges = (int64_t)1 << 38;

// Whether the sizes are ones that the work can be cut for
bool sizes_ok(const dci_attn& t) {
  return t.n_rows >= 0 && t.n_edges >= 0 && t.n_src >= 0 && t.max_list >= 0 && t.kv_heads >= 1 && t.n_heads >= t.kv_heads &&
         t.n_heads <= DCI_MAX_HEADS && t.n_heads % t.kv_heads == 0 && t.head_dim >= 1 && t.head_dim <= DCI_MAX_HEAD_DIM;
}

int32_t check_attn(dci_ctx* ctx, const dci_attn* t) {
  if (!ctx) return DCI_ERR_INVALID_ARG;
  if (!t) return fail(ctx, DCI_ERR_INVALID_ARG, "attention: null arguments");
  if (!sizes_ok(*t))
    return fail(ctx, DCI_ERR_INVALID_ARG,
                "attention: n_rows %lld, n_edges %lld, n_src %lld, max_list %d, n_heads %d, kv_heads %d, head_dim %d: sizes must not be negative, "
                "n_heads (at most %d) a multiple of kv_heads, head_dim 1 .. %d",
                (long long)t->n_rows, (long long)t->n_edges, (long long)t->n_src, t->max_list, t->n_heads, t->kv_heads, t->head_dim,
                DCI_MAX_HEADS, DCI_MAX_HEAD_DIM);
  if (!known_type(t->dtype)) return fail(ctx, DCI_ERR_INVALID_ARG, "attention: unknown dtype %d", t->dtype);
  if (t->n_rows > 0x7FFFFFFFll || t->n_src > 0x7FFFFFFFll || t->n_edges > kMaxEdges)
    return fail(ctx, DCI_ERR_UNSUPPORTED, "attention: more than 2^31-1 rows or sources, or 2^38 list entries");
  if (t->n_rows > 0 && (!t->indptr || !t->q || !t->out || (t->n_edges > 0 && !t->src)))
    return fail(ctx, DCI_ERR_INVALID_ARG, "attention: null indptr, src, q or out");
  const int64_t row = (int64_t)t->n_heads * t->head_dim;
  if (t->q_stride < row || t->out_stride < row)
    return fail(ctx, DCI_ERR_INVALID_ARG, "attention: q and out rows are n_heads * head_dim = %lld numbers long, strides %lld and %lld", (long long)row,
                (long long)t->q_stride, (long long)t->out_stride);
  if (!aligned_rows(t->q, t->dtype) || !aligned_rows(t->out, t->dtype))
    return fail(ctx, DCI_ERR_INVALID_ARG, "attention: q and out must be aligned to their type");
  if (t->bias ? t->bias_heads != 1 && t->bias_heads != t->n_heads : t->bias_heads != 0 && t->n_edges > 0)  // (an array of nothing may be null)
    return fail(ctx, DCI_ERR_INVALID_ARG, "attention: bias_heads is 1 or n_heads with a bias and 0 without, not %d", t->bias_heads);
  return DCI_OK;
}

template <int TYPE, int GQ, bool BIAS, bool WIDE>
void launch_attn(const Attn& a, unsigned chunk_grid, unsigned row_grid, unsigned lds, hipStream_t stream) {
  if (chunk_grid) hipLaunchKernelGGL((k_attn_chunks<TYPE, GQ, BIAS, WIDE>), dim3(chunk_grid), dim3(kAttnBlock), 0, stream, a);
  if (row_grid) hipLaunchKernelGGL((k_attn_rows<TYPE, GQ, BIAS, WIDE>), dim3(row_grid), dim3(kAttnBlock), lds, stream, a);
}
template <int TYPE, int GQ, bool WIDE>
void launch_attn(const Attn& a, unsigned chunk_grid, unsigned row_grid, unsigned lds, hipStream_t stream) {
  if (a.bias) launch_attn<TYPE, GQ, true, WIDE>(a, chunk_grid, row_grid, lds, stream);
  else launch_attn<TYPE, GQ, false, WIDE>(a, chunk_grid, row_grid, lds, stream);
}
template <int TYPE>
void launch_attn(const Split& s, const Attn& a, unsigned chunk_grid, unsigned row_grid, unsigned lds, hipStream_t stream) {
  if (!s.wide) launch_attn<TYPE, 1, false>(a, chunk_grid, row_grid, lds, stream);
  else if (s.gq == 1) launch_attn<TYPE, 1, true>(a, chunk_grid, row_grid, lds, stream);
  else if (s.gq == 2) launch_attn<TYPE, 2, true>(a, chunk_grid, row_grid, lds, stream);
  else launch_attn<TYPE, 4, true>(a, chunk_grid, row_grid, lds, stream);
}

template <int W>
void launch_groups(const Attn& a, unsigned grid, hipStream_t stream) {
  if (a.type == DCI_BF16) hipLaunchKernelGGL((k_attn_groups<W, 1>), dim3(grid), dim3(kAttnBlock), 0, stream, a);
  else if (a.type == DCI_F16) hipLaunchKernelGGL((k_attn_groups<W, 2>), dim3(grid), dim3(kAttnBlock), 0, stream, a);
  else hipLaunchKernelGGL((k_attn_groups<W, 3>), dim3(grid), dim3(kAttnBlock), 0, stream, a);
}

int32_t attn(dci_ctx* ctx, const dci_attn& t, int type, Attn a, bool accumulate) {
  const Split s = split_of(t, type, accumulate);
  Arena ar(ctx->ws, ctx->ws_bytes);
  const Parts parts = take_parts(ar, t, s.n_chunks, accumulate);
  if (!ar.ok()) {
    ctx->req_workspace = ar.off;
    return fail(ctx, DCI_ERR_CAPACITY, "workspace holds %zu bytes, this attention call needs %zu", ctx->ws_bytes, ar.off);
  }
  const int64_t b = type_bytes(t.dtype);
  a.n_rows = t.n_rows;
  a.n_dev = reinterpret_cast<const long long*>(t.n_dev);
  a.indptr = reinterpret_cast<const long long*>(t.indptr);
  a.src = t.src;
  a.n_edges = t.n_edges;
  a.type = t.dtype;
  a.heads = t.n_heads;
  a.kv_heads = t.kv_heads;
  a.dim = t.head_dim;
  a.group = t.n_heads / t.kv_heads;
  a.scale = t.scale;
  a.q = static_cast<const char*>(t.q);
  a.out = static_cast<char*>(t.out);
  a.q_stride = t.q_stride * b;
  a.out_stride = t.out_stride * b;
  a.lse = t.lse;
  a.bias = t.bias;
  a.bias_heads = t.bias_heads;
  // with weights, LDS for 64 entries' scores and a row of lse to each lane group
  a.stash_row = accumulate && t.n_edges > 0 ? (s.wave_heads * s.gq) | 1 : 0;
  const unsigned lds = (unsigned)(kAttnWaves * (kWave + (kWave >> s.p_log2)) * a.stash_row * sizeof(float));
  a.scores = parts.scores;
  a.all_lse = parts.all_lse;
  a.part_ml = parts.ml;
  a.part_acc = parts.acc;
  a.lh_log2 = s.lh_log2;
  a.ragged = type != kE4M3 && s.wide && t.head_dim != kCols<DCI_F32> << s.lh_log2;
  a.p_log2 = s.p_log2;
  a.wave_heads = s.wave_heads;
  a.passes = s.passes;
  a.gq_passes = s.gq_passes;
  a.chunk = s.chunk;
  a.n_chunks = (int)s.n_chunks;
  a.longest = t.max_list > 0 ? t.max_list : t.n_edges;
  const bool by_row = t.n_rows <= s.n_chunks;
  // A handful of rows: all by chunks, which spares a launch, and a row that has nothing is the join's: 16 lists of 500 entries take 16 to 17 us and 17
  // of them 22 to 30, of 10,000 entries 35 to 63 and 41 to 71 (four key heads of 64; dense 32-bit rows, 8-bit ones, 8-bit ones of four query heads each).
  // With many rows a chunk might hold dozens of tiny lists, and a wavefront takes several microseconds for each; how many may go before that costs
  // more than the launch depends on their lengths, which are not known here, so 16 is a line on the safe side and not the best one.
  const bool all_by_chunks = by_row && t.n_rows <= 16;
  a.short_list = all_by_chunks ? 0 : kShort;
  // lane groups to a row: one, unless that leaves wavefronts to be had (no more then than there are entries in a list) or, with weights, the scores
  // of the longest list would not all be at hand at its end.  (12,000 rows of 12 entries of four heads of 64: 23 us, 27 with two groups to a row.)
  const int groups_log2 = 6 - s.p_log2;
  const int64_t mean = t.n_edges / t.n_rows, longest = s.n_chunks ? kShort : t.max_list > 0 ? t.max_list : t.n_edges;
  a.r_log2 = 0;
  while (a.r_log2 < groups_log2 && ((((t.n_rows * s.passes) << a.r_log2 >> groups_log2) < kWantedWaves && (2ll << a.r_log2) <= mean) ||
                                    (accumulate && (1ll << (s.p_log2 + a.r_log2)) < longest)))
    ++a.r_log2;
  const int64_t at_once = 1ll << (groups_log2 - a.r_log2);
  int64_t blocks = ((t.n_rows + at_once - 1) / at_once * s.passes + kAttnWaves - 1) / kAttnWaves;
  const int64_t at_a_time = (int64_t)ctx->num_cus * waves_per_simd(type, s.gq);
  if (blocks > at_a_time) blocks = at_a_time;
  blocks = (blocks + s.passes - 1) / s.passes * s.passes;  // a wavefront keeps its share of the heads from row to row
  unsigned chunk_grid = (unsigned)((s.n_chunks * s.passes + kAttnWaves - 1) / kAttnWaves), row_grid = all_by_chunks ? 0 : (unsigned)blocks, group_grid = 0;
  Attn by_group = a;
  if (s.matrix && s.n_chunks) {
    by_group.gq_passes = (a.group + 7) / 8;
    by_group.pass_heads = (a.group + by_group.gq_passes - 1) / by_group.gq_passes;
    by_group.passes = t.kv_heads * by_group.gq_passes;
    group_grid = (unsigned)((s.n_chunks * by_group.passes + kAttnWaves - 1) / kAttnWaves);
    chunk_grid = 0;
  }
  const OnDevice on(ctx->device);
  DCI_HIP(ctx, on.err);
  {
    Timed timed(ctx, DCI_K_ATTN);
    if (group_grid) {
      if (t.head_dim == 64) launch_groups<64>(by_group, group_grid, ctx->stream);
      else if (t.head_dim == 128) launch_groups<128>(by_group, group_grid, ctx->stream);
      else launch_groups<256>(by_group, group_grid, ctx->stream);
      DCI_LAUNCH_CHECK(ctx);
    }
    if (type == kE4M3) launch_attn<kE4M3>(s, a, chunk_grid, row_grid, lds, ctx->stream);
    else if (type == DCI_F32) launch_attn<DCI_F32>(s, a, chunk_grid, row_grid, lds, ctx->stream);
    else if (type == DCI_BF16) launch_attn<DCI_BF16>(s, a, chunk_grid, row_grid, lds, ctx->stream);
    else launch_attn<DCI_F16>(s, a, chunk_grid, row_grid, lds, ctx->stream);
    DCI_LAUNCH_CHECK(ctx);
    if (s.n_chunks) {
      hipLaunchKernelGGL(k_attn_join, dim3((unsigned)((by_row ? t.n_rows : s.n_chunks) * t.n_heads)), dim3(kAttnBlock), 0, ctx->stream, a, by_row);
      DCI_LAUNCH_CHECK(ctx);
      if (accumulate && a.n_src > 0) {  // (without sources nobody has written scores)
        hipLaunchKernelGGL(k_attn_weights, dim3((unsigned)((s.n_chunks + kAttnWaves - 1) / kAttnWaves)), dim3(kAttnBlock), 0, ctx->stream, a);
        DCI_LAUNCH_CHECK(ctx);
      }
    }
  }
  return DCI_OK;
}

}  // namespace
}  // namespace dci

extern "C" {

size_t dci_attn_workspace_bytes(const dci_attn* attn, int32_t accumulate) {
  if (!attn || !dci::sizes_ok(*attn) || attn->n_edges > dci::kMaxEdges) return 0;
  // for rows of the cache or dense ones, whichever need more
  size_t most = 0;
  for (int type : {(int)dci::kE4M3, (int)attn->dtype}) {
    if (type != dci::kE4M3 && !dci::known_type(type)) return 0;
    dci::Arena ar(nullptr, 0);
    (void)dci::take_parts(ar, *attn, dci::split_of(*attn, type, accumulate != 0).most_chunks, accumulate != 0);
    if (ar.off > most) most = ar.off;
  }
  return most;
}

int32_t dci_attn_forward(dci_ctx* ctx, const dci_attn* attn, const void* k, int64_t k_stride, const void* v, int64_t v_stride) {
  const int32_t rc = dci::check_attn(ctx, attn);
  if (rc != DCI_OK) return rc;
  const int64_t row = (int64_t)attn->kv_heads * attn->head_dim;
  if (k_stride < row || v_stride < row)
    return dci::fail(ctx, DCI_ERR_INVALID_ARG, "attention: k and v rows are kv_heads * head_dim = %lld numbers long, strides %lld and %lld",
                     (long long)row, (long long)k_stride, (long long)v_stride);
  if (k_stride >= 1ll << 30 || v_stride >= 1ll << 30) return dci::fail(ctx, DCI_ERR_UNSUPPORTED, "attention: k and v strides of 2^30 numbers and more");
  if (attn->n_src > 0 && (!k || !v)) return dci::fail(ctx, DCI_ERR_INVALID_ARG, "attention: null k or v");
  if (!dci::aligned_rows(k, attn->dtype) || !dci::aligned_rows(v, attn->dtype))
    return dci::fail(ctx, DCI_ERR_INVALID_ARG, "attention: k and v must be aligned to their type");
  if (attn->n_rows == 0) return DCI_OK;
  dci::Attn a = {};
  a.n_src = a.n_at = (unsigned)attn->n_src;
  a.k = static_cast<const char*>(k);
  a.v = static_cast<const char*>(v);
  a.k_stride = (unsigned)(k_stride * dci::type_bytes(attn->dtype));
  a.v_stride = (unsigned)(v_stride * dci::type_bytes(attn->dtype));
  return dci::attn(ctx, *attn, attn->dtype, a, false);
}

int32_t dci_attn_cached(dci_ctx* ctx, const dci_attn* attn, const dci_kv_cache* cache, const int32_t* slots, int32_t accumulate) {
  int32_t rc = dci::check_attn(ctx, attn);
  if (rc == DCI_OK) rc = dci::check_kv_cache(ctx, cache);
  if (rc != DCI_OK) return rc;
  if (attn->kv_heads != cache->kv_heads || attn->head_dim != cache->head_dim)
    return dci::fail(ctx, DCI_ERR_INVALID_ARG, "attention: %d key heads of %d columns, the cache has %d of %d", attn->kv_heads, attn->head_dim,
                     cache->kv_heads, cache->head_dim);
  if (accumulate && !cache->weight) return dci::fail(ctx, DCI_ERR_INVALID_ARG, "attention: the cache has no weights to accumulate");
  if (attn->n_rows == 0) return DCI_OK;
  const int width = dci::kv_width(cache->head_dim);
  dci::Attn a = {};
  // Lanes whose entry names no source read the first slot all the same; without sources there is none, and they read what is there instead.
  a.slots = slots && attn->n_src == 0 ? reinterpret_cast<const int32_t*>(attn->indptr) : slots;
  a.n_at = (unsigned)cache->n_slots;
  a.n_src = slots ? (unsigned)attn->n_src : a.n_at;
  a.k = reinterpret_cast<const char*>(cache->codes);
  a.v = a.k + (int64_t)cache->kv_heads * width;
  a.k_stride = a.v_stride = 2u * cache->kv_heads * width;
  a.scales = cache->scales;
  a.block_log2 = dci::log2_up(cache->block);
  a.weight = reinterpret_cast<unsigned long long*>(cache->weight);
  return dci::attn(ctx, *attn, dci::kE4M3, a, accumulate != 0);
}

}  // extern "C"
