// Attention over the lists of a block: dci_attn_forward (dense rows) and dci_attn_cached (rows of the 8-bit cache).
//
// For a row i and a head h, over the entries e of the row's list:  z_e = scale (q_i . K_e) + bias_e,  out = sum exp(z_e) V_e / sum exp(z_e).
// One pass over the list: a running maximum m, the sum l of exp(z - m) and the accumulator of exp(z - m) V, the last two rescaled
// when m grows.  Every K and V row that an entry names is read once, straight into registers, 16 columns to a lane:
//   a head's columns lie in LH = 1 .. 16 adjacent lanes, the heads of a row side by side, P lanes in all (a power of two up to 64; more
//   heads are shared out between wavefronts).  A score is a sum over LH lanes (DPP), and the lanes of a head then hold what they need
//   for their columns of the output: nothing passes through LDS.
//   The 64 / P groups of lanes of a wavefront work on rows of their own, or R of them on one row, each on every R-th entry, and join their
//   (m, l, acc) at the row's end.
//   Query heads that share a key head are worked on together, up to four of them (GQ), from the same registers.
// Lists longer than `chunk` entries are cut at multiples of it in the whole array of entries, so that neither the number nor the
// length of lists needs to be known: a wavefront takes `chunk` entries, finds the rows they belong to (a 64-way search in indptr) and
// leaves (m, l, acc) of its piece of a long list in the workspace.  At most two pieces of long lists meet in a chunk, as a list that lay between
// two others inside it would be no longer than it: the list that goes on from before (or begins with the chunk) is piece 0, one that begins
// inside is piece 1.  k_attn_join adds a list's pieces up in order.
// What bounds it: the rows' bytes.  A row of the cache is 2 * kv_heads * head_dim bytes in one place, so a gather of whole rows
// goes at nearly the rate of a copy.
#include "dci_kv.h"

namespace dci {
namespace {

constexpr int kAttnBlock = 256, kAttnWaves = kAttnBlock / kWave;
constexpr float kLog2E = 1.44269504088896340736f;
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
  bool q_wide, out_wide, kv_wide;
  float* lse;
  const float* bias;
  int bias_heads;
  const char *k, *v;
  long long k_stride, v_stride;  // bytes
  const float* scales;           // the cache's, [block, kv head, 2]
  int block_log2, kv_heads;
  const int* slots;  // nullptr: src is the row of k and v
  float* scores;     // [n_edges, heads], accumulating only
  unsigned long long* weight;
  int lh_log2, p_log2, r_log2;  // lanes to a head, to an entry; lane groups to a row
  int wave_heads;               // key heads to a wavefront
  int passes;                   // wavefronts that share a row's key heads and their groups
  int gq_passes;                // of them, those that share a group
  int chunk;
  int n_chunks;  // 0: no list is cut
  int chunk_blocks, row_blocks;
  float* part_ml;   // [2 n_chunks, heads, 2]
  float* part_acc;  // [2 n_chunks, heads, W]
  float* all_lse;   // lse of the cut lists by row, accumulating only
};

// What a lane of an attention wavefront is there for
struct Place {
  int sub;    // its group's number among those of a row
  int col;    // its first column
  int cols;   // its columns, 0: none
  int kv;     // its key head
  int head;   // its first query head
  int n_q;    // how many query heads
  bool on;
};

template <int GQ>
struct State {
  float m[GQ], l[GQ], acc[GQ][kChunk];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int g = 0; g < GQ; ++g) {
      m[g] = -INFINITY;
      l[g] = 0.f;
#pragma unroll
      for (int j = 0; j < kChunk; ++j) acc[g][j] = 0.f;
    }
  }
};

__device__ __forceinline__ float exp_diff(float a, float b) { return __builtin_amdgcn_exp2f((a - b) * kLog2E); }
__device__ __forceinline__ float finite_or_0(float m) { return m == -INFINITY ? 0.f : m; }

// The last row that begins at or before entry p (so the one that holds it, if one does); n >= 1, wavefront-wide
__device__ __forceinline__ long long row_of(const long long* __restrict__ indptr, long long n, long long p) {
  long long lo = 0, hi = n;
  while (hi - lo > 1) {
    const long long step = (hi - lo + kWave - 1) / kWave;
    const long long at = lo + lane_id() * step;
    const unsigned long long before = __ballot(at < hi && indptr[at] <= p);
    const int c = __popcll(before);  // a prefix of the lanes, as indptr ascends
    if (c == 0) return lo;
    lo += (c - 1) * step;
    hi = min(hi, lo + step);
  }
  return lo;
}

__device__ __forceinline__ int slot_of(const Attn& a, int s) {
  if ((unsigned)s >= a.n_src) return -1;
  return a.slots ? a.slots[s] : s;
}

// Entries [e0, e1) of one row, every (1 << r_log2)-th from e0 + sub on, into st
template <int TYPE, int GQ, bool BIAS>
__device__ __forceinline__ void attend(const Attn& a, const Place& pl, long long e0, long long e1, int r_log2, const float (&q)[GQ][kChunk],
                                       State<GQ>& st) {
  constexpr int U = TYPE == DCI_F32 ? 2 : 4;  // entries at a time
  const int n = (int)min(e1 - e0, (long long)0x7FFFFFFF - 1024);
  const int* __restrict__ src = a.src + e0;
  const int step = 1 << r_log2;
  const long long k_off = (long long)pl.kv * a.dim * type_bytes(TYPE) + pl.col * type_bytes(TYPE);
  const char* k0 = a.k + (TYPE == kE4M3 ? (long long)pl.kv * ((a.dim + kChunk - 1) / kChunk * kChunk) + pl.col : k_off);
  const char* v0 = a.v + (TYPE == kE4M3 ? (long long)pl.kv * ((a.dim + kChunk - 1) / kChunk * kChunk) + pl.col : k_off);
  int at[U], next[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int t = pl.sub + u * step;
    at[u] = t < n ? src[t] : -1;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int t = pl.sub + (U + u) * step;
    next[u] = t < n ? src[t] : -1;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) at[u] = slot_of(a, at[u]);
  for (int t0 = 0; t0 < n; t0 += U * step) {
    Chunk<TYPE> kc[U], vc[U];
    float ks[U], vs[U], bias[U][GQ];
    bool there[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + pl.sub + u * step;
      there[u] = (unsigned)at[u] < a.n_at;
      kc[u].clear();
      vc[u].clear();
      ks[u] = vs[u] = 1.f;
      if (there[u] && pl.on) {
        if (pl.cols > 0) {
          kc[u].load(k0 + at[u] * a.k_stride, pl.cols, a.kv_wide);
          vc[u].load(v0 + at[u] * a.v_stride, pl.cols, a.kv_wide);
        }
        if (TYPE == kE4M3) {
          const float2 s = *reinterpret_cast<const float2*>(a.scales + 2 * ((long long)(at[u] >> a.block_log2) * a.kv_heads + pl.kv));
          ks[u] = s.x;
          vs[u] = s.y;
        }
      }
      if (BIAS) {
#pragma unroll
        for (int g = 0; g < GQ; ++g)
          bias[u][g] = there[u] && pl.on && g < pl.n_q ? a.bias[(e0 + t) * a.bias_heads + (a.bias_heads > 1 ? pl.head + g : 0)] : 0.f;
      }
    }
    // the slots of the entries after these, and the sources of those after them, on their way while these are worked on
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + pl.sub + (2 * U + u) * step;
      at[u] = slot_of(a, next[u]);
      next[u] = t < n ? src[t] : -1;
    }
    float z[U][GQ];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float dot[GQ];
#pragma unroll
      for (int g = 0; g < GQ; ++g) dot[g] = 0.f;
#pragma unroll
      for (int j = 0; j < kChunk / 2; ++j) {
        float x, y;
        kc[u].pair(j, x, y);
#pragma unroll
        for (int g = 0; g < GQ; ++g) dot[g] = fmaf(q[g][2 * j + 1], y, fmaf(q[g][2 * j], x, dot[g]));
      }
#pragma unroll
      for (int g = 0; g < GQ; ++g) {
        z[u][g] = sum_lanes(dot[g], a.lh_log2) * (a.scale * ks[u]);
        if (BIAS) z[u][g] = bias[u][g] == -INFINITY ? -INFINITY : z[u][g] + bias[u][g];
        if (!there[u]) z[u][g] = -INFINITY;
      }
    }
    if (a.scores && pl.col == 0 && pl.on) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int t = t0 + pl.sub + u * step;
        if (t < n) {
#pragma unroll
          for (int g = 0; g < GQ; ++g)
            if (g < pl.n_q) a.scores[(e0 + t) * a.heads + pl.head + g] = z[u][g];
        }
      }
    }
    float p[U][GQ];
#pragma unroll
    for (int g = 0; g < GQ; ++g) {
      float m = st.m[g];
#pragma unroll
      for (int u = 0; u < U; ++u) m = fmaxf(m, z[u][g]);
      const float base = finite_or_0(m), shrink = exp_diff(st.m[g], base);
      st.m[g] = m;
      st.l[g] *= shrink;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        p[u][g] = exp_diff(z[u][g], base);
        st.l[g] += p[u][g];
        p[u][g] *= vs[u];
      }
#pragma unroll
      for (int j = 0; j < kChunk; ++j) st.acc[g][j] *= shrink;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      // with a bias an entry may be left out for one head and not for the next: its values, whatever they are, then add nothing
      bool in[GQ];
#pragma unroll
      for (int g = 0; g < GQ; ++g) in[g] = !BIAS || z[u][g] != -INFINITY;
#pragma unroll
      for (int j = 0; j < kChunk / 2; ++j) {
        float x, y;
        vc[u].pair(j, x, y);
#pragma unroll
        for (int g = 0; g < GQ; ++g) {
          if (in[g]) {
            st.acc[g][2 * j] = fmaf(p[u][g], x, st.acc[g][2 * j]);
            st.acc[g][2 * j + 1] = fmaf(p[u][g], y, st.acc[g][2 * j + 1]);
          }
        }
      }
    }
  }
}

// (m, l, acc) of lanes `apart` away joined into st
template <int GQ>
__device__ __forceinline__ void join_lanes(State<GQ>& st, int apart) {
#pragma unroll
  for (int g = 0; g < GQ; ++g) {
    const float m2 = __shfl_xor(st.m[g], apart, kWave), l2 = __shfl_xor(st.l[g], apart, kWave);
    const float m = fmaxf(st.m[g], m2), base = finite_or_0(m);
    const float f1 = exp_diff(st.m[g], base), f2 = exp_diff(m2, base);
    st.m[g] = m;
    st.l[g] = st.l[g] * f1 + l2 * f2;
#pragma unroll
    for (int j = 0; j < kChunk; ++j) {
      const float other = __shfl_xor(st.acc[g][j], apart, kWave);
      st.acc[g][j] = st.acc[g][j] * f1 + other * f2;
    }
  }
}

__device__ __forceinline__ void add_weight(const Attn& a, int s, float p) {
  const int at = slot_of(a, s);
  if (p > 0.f && (unsigned)at < a.n_at) atomicAdd(a.weight + at, (unsigned long long)((double)p * kWeightUnit + 0.5));
}

template <int TYPE, int GQ, bool BIAS>
__global__ __launch_bounds__(kAttnBlock, 2) void k_attn(const Attn a) {
  const int lane = lane_id(), wave = (int)threadIdx.x / kWave;
  const int p_lanes = 1 << a.p_log2, lh = 1 << a.lh_log2, groups = kWave >> a.p_log2;
  const bool chunks = (int)blockIdx.x < a.chunk_blocks;
  const long long unit0 = (long long)(chunks ? blockIdx.x : blockIdx.x - a.chunk_blocks) * kAttnWaves + wave;
  const int pass = (int)(unit0 % a.passes);  // wavefronts side by side read the same rows
  Place pl;
  {
    const int in = lane & (p_lanes - 1), h = in >> a.lh_log2;
    const int wave_part = pass / a.gq_passes, gq_part = pass % a.gq_passes;
    pl.col = (in & (lh - 1)) * kChunk;
    pl.kv = wave_part * a.wave_heads + h;
    pl.on = h < a.wave_heads && pl.kv < a.kv_heads;
    if (!pl.on) pl.kv = 0;
    pl.cols = min(kChunk, max(0, a.dim - pl.col));
    pl.n_q = pl.on ? min(GQ, a.group - gq_part * GQ) : 0;
    pl.head = pl.kv * a.group + gq_part * GQ;
  }
  const long long n = a.n_dev ? min(a.n_rows, max(0ll, *a.n_dev)) : a.n_rows;
  float q[GQ][kChunk];
  State<GQ> st;
  auto read_q = [&](long long row, bool real) {
#pragma unroll
    for (int g = 0; g < GQ; ++g) {
#pragma unroll
      for (int j = 0; j < kChunk; ++j) q[g][j] = 0.f;
      if (real && g < pl.n_q && pl.cols > 0)
        read_chunk(a.type, a.q + row * a.q_stride + ((long long)(pl.head + g) * a.dim + pl.col) * type_bytes(a.type), pl.cols, a.q_wide, q[g]);
    }
  };
  if (chunks) {
    const long long c = unit0 / a.passes;
    if (c >= a.n_chunks || n == 0) return;
    const long long c0 = c * a.chunk, c1 = min(c0 + a.chunk, min(a.n_edges, a.indptr[n]));
    if (c0 >= c1) return;
    pl.sub = lane >> a.p_log2;
    const long long first = row_of(a.indptr, n, c0), last = row_of(a.indptr, n, c1 - 1);
    for (int piece = 0; piece < 2; ++piece) {
      const long long row = piece ? last : first;
      if (piece && first == last) break;
      const long long b = a.indptr[row], e = a.indptr[row + 1];
      if (e - b <= a.chunk) continue;
      read_q(row, true);
      st.clear();
      attend<TYPE, GQ, BIAS>(a, pl, max(b, c0), min(e, c1), 6 - a.p_log2, q, st);
      for (int apart = p_lanes; apart < kWave; apart <<= 1) join_lanes<GQ>(st, apart);
      if (lane < p_lanes && pl.cols > 0) {
#pragma unroll
        for (int g = 0; g < GQ; ++g) {
          if (g < pl.n_q) {
            const long long at = (2 * c + (b > c0 ? 1 : 0)) * a.heads + pl.head + g;
            if (pl.col == 0) {
              a.part_ml[2 * at] = st.m[g];
              a.part_ml[2 * at + 1] = st.l[g];
            }
            float4* acc = reinterpret_cast<float4*>(a.part_acc + at * ((a.dim + kChunk - 1) / kChunk * kChunk) + pl.col);
#pragma unroll
            for (int j = 0; j < kChunk / 4; ++j)
              acc[j] = make_float4(st.acc[g][4 * j], st.acc[g][4 * j + 1], st.acc[g][4 * j + 2], st.acc[g][4 * j + 3]);
          }
        }
      }
    }
    return;
  }
  const int r_log2 = a.r_log2, r = 1 << r_log2, rows_at_once = groups >> r_log2;
  const int g_id = lane >> a.p_log2;
  pl.sub = g_id & (r - 1);
  const long long stride = (long long)a.row_blocks * kAttnWaves / a.passes * rows_at_once;
  for (long long row0 = unit0 / a.passes * rows_at_once; row0 < n; row0 += stride) {
    const long long row = row0 + (g_id >> r_log2);
    const bool real = row < n;
    long long b = 0, e = 0;
    if (real) {
      b = max(0ll, a.indptr[row]);
      e = min(a.n_edges, a.indptr[row + 1]);
      if (e < b) e = b;
    }
    const bool mine = real && (a.n_chunks == 0 || e - b <= a.chunk);
    if (!mine) e = b;
    read_q(row, mine);
    st.clear();
    attend<TYPE, GQ, BIAS>(a, pl, b, e, r_log2, q, st);
    for (int apart = p_lanes; apart < (p_lanes << r_log2); apart <<= 1) join_lanes<GQ>(st, apart);
    float lse[GQ];
#pragma unroll
    for (int g = 0; g < GQ; ++g) {
      lse[g] = st.l[g] == 0.f ? -INFINITY : st.m[g] + logf(st.l[g]);
      if (mine && pl.sub == 0 && g < pl.n_q) {
        const float inv = st.l[g] == 0.f ? 0.f : 1.f / st.l[g];
        float y[kChunk];
#pragma unroll
        for (int j = 0; j < kChunk; ++j) y[j] = st.acc[g][j] * inv;
        if (pl.cols > 0)
          write_chunk(a.type, a.out + row * a.out_stride + ((long long)(pl.head + g) * a.dim + pl.col) * type_bytes(a.type), pl.cols,
                      a.out_wide, y);
        if (a.lse && pl.col == 0) a.lse[row * a.heads + pl.head + g] = lse[g];
      }
    }
    if (a.scores) {
      __threadfence_block();  // the scores of this wavefront's other lanes
      const int len = (int)(e - b);
      for (int t0 = 0; t0 < len; t0 += r * lh) {
        const int t = t0 + pl.sub * lh + pl.col / kChunk;
        float p = 0.f;
        if (t < len && pl.on) {
#pragma unroll
          for (int g = 0; g < GQ; ++g) {
            if (g < pl.n_q) {
              const float z = a.scores[(b + t) * a.heads + pl.head + g];
              if (z != -INFINITY) p += exp_diff(z, lse[g]);
            }
          }
        }
        for (int apart = lh; apart < p_lanes; apart <<= 1) p += __shfl_xor(p, apart, kWave);
        if (t < len && (lane & (p_lanes - 1)) < lh) add_weight(a, a.src[b + t], p);
      }
    }
  }
}

// One workgroup per chunk and head: the list that begins in the chunk, if it is a long one
__global__ __launch_bounds__(kAttnBlock) void k_attn_join(const Attn a) {
  const int head = (int)(blockIdx.x % (unsigned)a.heads);
  const long long c = blockIdx.x / (unsigned)a.heads;
  const long long n = a.n_dev ? min(a.n_rows, max(0ll, *a.n_dev)) : a.n_rows;
  if (n == 0) return;
  const long long total = min(a.n_edges, a.indptr[n]);
  const long long c0 = c * a.chunk, c1 = min(c0 + a.chunk, total);
  if (c0 >= c1) return;
  const long long row = row_of(a.indptr, n, c1 - 1);
  const long long b = a.indptr[row], e = min(total, a.indptr[row + 1]);
  if (b < c0 || e - b <= a.chunk) return;
  const int width = (a.dim + kChunk - 1) / kChunk * kChunk;
  const int pieces = (int)((e - 1) / a.chunk - c) + 1;
  auto place = [&](int k) { return (2 * (c + k) + (k == 0 && b != c0 ? 1 : 0)) * a.heads + head; };
  __shared__ float part[kAttnBlock], red[kAttnWaves];
  const int lane = lane_id(), wave = (int)threadIdx.x / kWave;
  float m = -INFINITY;
  for (int k = (int)threadIdx.x; k < pieces; k += kAttnBlock) m = fmaxf(m, a.part_ml[2 * place(k)]);
  for (int d = kWave / 2; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, kWave));
  if (lane == 0) red[wave] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kAttnWaves; ++w) m = fmaxf(m, red[w]);
  const float base = finite_or_0(m);
  __syncthreads();
  float l = 0.f;
  for (int k = (int)threadIdx.x; k < pieces; k += kAttnBlock) {
    const long long at = place(k);
    l += a.part_ml[2 * at + 1] * exp_diff(a.part_ml[2 * at], base);
  }
  for (int d = kWave / 2; d; d >>= 1) l += __shfl_xor(l, d, kWave);
  if (lane == 0) red[wave] = l;
  __syncthreads();
  l = 0.f;
#pragma unroll
  for (int w = 0; w < kAttnWaves; ++w) l += red[w];
  // columns side by side, as many slices of the pieces as the workgroup has room for
  int cols = 16;
  while (cols < width) cols <<= 1;
  const int slices = kAttnBlock / cols, col = (int)threadIdx.x & (cols - 1), slice = (int)threadIdx.x / cols;
  float acc = 0.f;
  if (col < width) {
    for (int k = slice; k < pieces; k += slices) {
      const long long at = place(k);
      acc += a.part_acc[at * width + col] * exp_diff(a.part_ml[2 * at], base);
    }
  }
  part[threadIdx.x] = acc;
  __syncthreads();
  if (slice == 0 && col < a.dim) {
    for (int s = 1; s < slices; ++s) acc += part[s * cols + col];
    const float y = l == 0.f ? 0.f : acc / l;
    char* o = a.out + row * a.out_stride + ((long long)head * a.dim + col) * type_bytes(a.type);
    if (a.type == DCI_F32) *reinterpret_cast<float*>(o) = y;
    else if (a.type == DCI_BF16) *reinterpret_cast<unsigned short*>(o) = (unsigned short)two<DCI_BF16>(y, 0.f);
    else *reinterpret_cast<unsigned short*>(o) = (unsigned short)two<DCI_F16>(y, 0.f);
  }
  if (threadIdx.x == 0) {
    const float lse = l == 0.f ? -INFINITY : m + logf(l);
    if (a.lse) a.lse[row * a.heads + head] = lse;
    if (a.all_lse) a.all_lse[row * a.heads + head] = lse;
  }
}

// Accumulated weights of the long lists, an entry to a lane
__global__ __launch_bounds__(kAttnBlock) void k_attn_weights(const Attn a) {
  const long long c = (long long)blockIdx.x * kAttnWaves + threadIdx.x / kWave;
  const long long n = a.n_dev ? min(a.n_rows, max(0ll, *a.n_dev)) : a.n_rows;
  if (c >= a.n_chunks || n == 0) return;
  const long long c0 = c * a.chunk, c1 = min(c0 + a.chunk, min(a.n_edges, a.indptr[n]));
  if (c0 >= c1) return;
  const long long first = row_of(a.indptr, n, c0), last = row_of(a.indptr, n, c1 - 1);
  for (int piece = 0; piece < 2; ++piece) {
    const long long row = piece ? last : first;
    if (piece && first == last) break;
    const long long b = a.indptr[row], e = a.indptr[row + 1];
    if (e - b <= a.chunk) continue;
    const long long to = min(e, c1);
    for (long long t = max(b, c0) + lane_id(); t < to; t += kWave) {
      float p = 0.f;
      for (int h = 0; h < a.heads; ++h) {
        const float z = a.scores[t * a.heads + h];
        if (z != -INFINITY) p += exp_diff(z, a.all_lse[row * a.heads + h]);
      }
      add_weight(a, a.src[t], p);
    }
  }
}


// How a call's work is cut, from its arguments alone (the workspace query has no context)
struct Split {
  int p_log2, lh_log2, wave_heads, gq, gq_passes, passes;
  int chunk;
  int64_t n_chunks;
};
constexpr int64_t kWantedWaves = 4096;  // 16 to a compute unit

Split split_of(const dci_attn& t) {
  Split s;
  s.lh_log2 = log2_up((t.head_dim + kChunk - 1) / kChunk);
  s.p_log2 = log2_up((int64_t)t.kv_heads << s.lh_log2);
  if (s.p_log2 > 6) s.p_log2 = 6;
  s.wave_heads = (kWave >> s.lh_log2) < t.kv_heads ? (kWave >> s.lh_log2) : t.kv_heads;
  const int group = t.n_heads / t.kv_heads;
  s.gq = group == 1 ? 1 : group == 2 ? 2 : 4;
  s.gq_passes = (group + s.gq - 1) / s.gq;
  s.passes = (t.kv_heads + s.wave_heads - 1) / s.wave_heads * s.gq_passes;
  // chunks of 64 to 512 entries: as long as there are wavefronts enough
  s.chunk = 64;
  while (s.chunk < 512 && t.n_edges / s.chunk * s.passes > kWantedWaves) s.chunk *= 2;
  const int64_t longest = t.max_list > 0 && t.max_list < t.n_edges ? t.max_list : t.n_edges;
  s.n_chunks = longest > s.chunk ? (t.n_edges + s.chunk - 1) / s.chunk : 0;
  return s;
}

struct Parts {
  float *scores = nullptr, *all_lse = nullptr, *ml = nullptr, *acc = nullptr;
};
Parts take_parts(Arena& ar, const dci_attn& t, const Split& s, bool accumulate) {
  Parts p;
  if (accumulate) p.scores = ar.take<float>((size_t)t.n_edges * t.n_heads);
  if (s.n_chunks) {
    if (accumulate) p.all_lse = ar.take<float>((size_t)t.n_rows * t.n_heads);
    p.ml = ar.take<float>((size_t)s.n_chunks * 2 * t.n_heads * 2);
    p.acc = ar.take<float>((size_t)s.n_chunks * 2 * t.n_heads * kv_width(t.head_dim));
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
  if (t->bias ? t->bias_heads != 1 && t->bias_heads != t->n_heads : t->bias_heads != 0)
    return fail(ctx, DCI_ERR_INVALID_ARG, "attention: bias_heads is 1 or n_heads with a bias and 0 without, not %d", t->bias_heads);
  return DCI_OK;
}

template <int TYPE>
void launch_attn(int gq, const Attn& a, dim3 grid, hipStream_t stream) {
#define DCI_ATTN(GQ_)                                                                                             \
  do {                                                                                                            \
    if (a.bias) hipLaunchKernelGGL((k_attn<TYPE, GQ_, true>), grid, dim3(kAttnBlock), 0, stream, a);              \
    else hipLaunchKernelGGL((k_attn<TYPE, GQ_, false>), grid, dim3(kAttnBlock), 0, stream, a);                    \
  } while (0)
  if (gq == 1) DCI_ATTN(1);
  else if (gq == 2) DCI_ATTN(2);
  else DCI_ATTN(4);
#undef DCI_ATTN
}

int32_t attn(dci_ctx* ctx, const dci_attn& t, int type, Attn a, bool accumulate) {
  const Split s = split_of(t);
  Arena ar(ctx->ws, ctx->ws_bytes);
  const Parts parts = take_parts(ar, t, s, accumulate);
  if (!ar.ok()) {
    ctx->req_workspace = ar.off;
    return fail(ctx, DCI_ERR_CAPACITY, "workspace holds %zu bytes, this attention call needs %zu", ctx->ws_bytes, ar.off);
  }
  if (s.n_chunks * t.n_heads > 0x7FFFFFFFll || s.n_chunks * s.passes > 0x7FFFFFFFll)
    return fail(ctx, DCI_ERR_UNSUPPORTED, "attention: too many list entries and heads for one call");
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
  a.q_wide = by_16_bytes(t.q, t.q_stride, t.head_dim, t.dtype);
  a.out_wide = by_16_bytes(t.out, t.out_stride, t.head_dim, t.dtype);
  a.lse = t.lse;
  a.bias = t.bias;
  a.bias_heads = t.bias_heads;
  a.scores = parts.scores;
  a.all_lse = parts.all_lse;
  a.part_ml = parts.ml;
  a.part_acc = parts.acc;
  a.lh_log2 = s.lh_log2;
  a.p_log2 = s.p_log2;
  a.wave_heads = s.wave_heads;
  a.passes = s.passes;
  a.gq_passes = s.gq_passes;
  a.chunk = s.chunk;
  a.n_chunks = (int)s.n_chunks;
  a.chunk_blocks = (int)((s.n_chunks * s.passes + kAttnWaves - 1) / kAttnWaves);
  // lane groups to a row: one, unless that leaves wavefronts to be had; no more than there are entries in a list
  const int groups_log2 = 6 - s.p_log2;
  const int64_t mean = t.n_edges / t.n_rows;
  a.r_log2 = 0;
  while (a.r_log2 < groups_log2 && ((t.n_rows * s.passes) << a.r_log2 >> groups_log2) < kWantedWaves && (2ll << a.r_log2) <= mean) ++a.r_log2;
  const int64_t at_once = 1ll << (groups_log2 - a.r_log2);
  int64_t blocks = ((t.n_rows + at_once - 1) / at_once * s.passes + kAttnWaves - 1) / kAttnWaves;
  if (blocks > (int64_t)ctx->num_cus * 32) blocks = (int64_t)ctx->num_cus * 32;
  blocks = (blocks + s.passes - 1) / s.passes * s.passes;  // a wavefront keeps its share of the heads from row to row
  a.row_blocks = (int)blocks;
  const OnDevice on(ctx->device);
  DCI_HIP(ctx, on.err);
  {
    Timed timed(ctx, DCI_K_ATTN);
    const dim3 grid((unsigned)(a.chunk_blocks + a.row_blocks));
    if (type == kE4M3) launch_attn<kE4M3>(s.gq, a, grid, ctx->stream);
    else if (type == DCI_F32) launch_attn<DCI_F32>(s.gq, a, grid, ctx->stream);
    else if (type == DCI_BF16) launch_attn<DCI_BF16>(s.gq, a, grid, ctx->stream);
    else launch_attn<DCI_F16>(s.gq, a, grid, ctx->stream);
    DCI_LAUNCH_CHECK(ctx);
    if (s.n_chunks) {
      hipLaunchKernelGGL(k_attn_join, dim3((unsigned)(s.n_chunks * t.n_heads)), dim3(kAttnBlock), 0, ctx->stream, a);
      DCI_LAUNCH_CHECK(ctx);
      if (accumulate) {
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
  dci::Arena ar(nullptr, 0);
  (void)dci::take_parts(ar, *attn, dci::split_of(*attn), accumulate != 0);
  return ar.off;
}

int32_t dci_attn_forward(dci_ctx* ctx, const dci_attn* attn, const void* k, int64_t k_stride, const void* v, int64_t v_stride) {
  const int32_t rc = dci::check_attn(ctx, attn);
  if (rc != DCI_OK) return rc;
  const int64_t row = (int64_t)attn->kv_heads * attn->head_dim;
  if (k_stride < row || v_stride < row)
    return dci::fail(ctx, DCI_ERR_INVALID_ARG, "attention: k and v rows are kv_heads * head_dim = %lld numbers long, strides %lld and %lld",
                     (long long)row, (long long)k_stride, (long long)v_stride);
  if (attn->n_src > 0 && (!k || !v)) return dci::fail(ctx, DCI_ERR_INVALID_ARG, "attention: null k or v");
  if (!dci::aligned_rows(k, attn->dtype) || !dci::aligned_rows(v, attn->dtype))
    return dci::fail(ctx, DCI_ERR_INVALID_ARG, "attention: k and v must be aligned to their type");
  if (attn->n_rows == 0) return DCI_OK;
  dci::Attn a = {};
  a.n_src = a.n_at = (unsigned)attn->n_src;
  a.k = static_cast<const char*>(k);
  a.v = static_cast<const char*>(v);
  a.k_stride = k_stride * dci::type_bytes(attn->dtype);
  a.v_stride = v_stride * dci::type_bytes(attn->dtype);
  a.kv_wide = dci::by_16_bytes(k, k_stride, attn->head_dim, attn->dtype) && dci::by_16_bytes(v, v_stride, attn->head_dim, attn->dtype);
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
  a.slots = slots;
  a.n_at = (unsigned)cache->n_slots;
  a.n_src = slots ? (unsigned)attn->n_src : a.n_at;
  a.k = reinterpret_cast<const char*>(cache->codes);
  a.v = a.k + (int64_t)cache->kv_heads * width;
  a.k_stride = a.v_stride = 2ll * cache->kv_heads * width;
  a.kv_wide = true;
  a.scales = cache->scales;
  a.block_log2 = dci::log2_up(cache->block);
  a.weight = reinterpret_cast<unsigned long long*>(cache->weight);
  return dci::attn(ctx, *attn, dci::kE4M3, a, accumulate != 0);
}

}  // extern "C"
