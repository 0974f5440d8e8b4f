// The 8-bit key/value cache: clearing, writing and reading rows (dci_kv_clear, dci_kv_write, dci_kv_read) and finding slots for a batch's
// nodes by eviction (dci_kv_admit).
#include "dci_kv.h"

namespace dci {

int32_t check_kv_cache(dci_ctx* ctx, const dci_kv_cache* c) {
  if (!ctx) return DCI_ERR_INVALID_ARG;
  if (!c) return fail(ctx, DCI_ERR_INVALID_ARG, "key/value cache: null");
  if (c->n_slots < 1 || c->n_slots > 0x7FFFFFFFll || c->block < 1 || c->block > 64 || (c->block & (c->block - 1)) || c->kv_heads < 1 ||
      c->kv_heads > DCI_MAX_HEADS || c->head_dim < 1 || c->head_dim > DCI_MAX_HEAD_DIM)
    return fail(ctx, DCI_ERR_INVALID_ARG,
                "key/value cache: n_slots %lld (1 .. 2^31-1), block %d (a power of two, 1 .. 64), kv_heads %d (1 .. %d), head_dim %d (1 .. %d)",
                (long long)c->n_slots, c->block, c->kv_heads, DCI_MAX_HEADS, c->head_dim, DCI_MAX_HEAD_DIM);
  if (!c->codes || !c->scales) return fail(ctx, DCI_ERR_INVALID_ARG, "key/value cache: null codes or scales");
  if (reinterpret_cast<uintptr_t>(c->codes) % 16 || reinterpret_cast<uintptr_t>(c->scales) % 8)
    return fail(ctx, DCI_ERR_INVALID_ARG, "key/value cache: codes must be 16-byte and scales 8-byte aligned");
  return DCI_OK;
}

namespace {

constexpr int kKvBlock = 256, kKvWaves = kKvBlock / kWave;
constexpr int kMinExp = -100, kMaxExp = 119;  // of a scale: 2^-kMinExp and 448 * 2^kMaxExp are fp32 numbers

// ---- clearing -------------------------------------------------------------------------------------

__global__ __launch_bounds__(kKvBlock) void k_kv_clear(uint4* codes, long long n16, float* scales, long long n_scales,
                                                       unsigned long long* weight, long long* node, long long n_slots) {
  const long long at = blockIdx.x * (long long)kKvBlock + threadIdx.x, step = (long long)gridDim.x * kKvBlock;
  for (long long i = at; i < n16; i += step) codes[i] = make_uint4(0, 0, 0, 0);
  for (long long i = at; i < n_scales; i += step) scales[i] = 0.f;
  for (long long i = at; i < n_slots; i += step) {
    if (weight) weight[i] = 0;
    if (node) node[i] = -1;
  }
}

// ---- writing --------------------------------------------------------------------------------------

struct KvWrite {
  const int* slots;
  long long n_max;
  const long long* n_dev;
  int type;
  const char* from[2];  // keys, values
  long long stride[2];  // bytes
  bool wide[2];
  unsigned char* codes;
  float* scales;
  long long n_slots;
  int block_log2, kv_heads, dim, lh_log2;
  unsigned* host_flag;
};

constexpr int kWriteRows = 4;  // entries of the list that a wavefront looks for the beginnings of blocks in

__device__ __forceinline__ bool is_number(float x) { return (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u; }

// The least e with amax <= 448 * 2^e, 448 = 1.75 * 2^8
__device__ __forceinline__ int need_exp(float amax) {
  const unsigned u = __float_as_uint(amax);
  if (u == 0) return kMinExp;
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return min(max(e, kMinExp), kMaxExp);  // (an fp32 number below 2^-126 comes out below kMinExp all the same)
}
__device__ __forceinline__ float exp2_of(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }

// 16 numbers as codes, each divided by 2^e first; rounded to nearest even, at most 448
__device__ __forceinline__ uint4 encode(const float (&x)[kChunk], int e) {
  const float f = exp2_of(-e);
  unsigned w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float y[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float v = x[4 * j + k];
      y[k] = is_number(v) ? fminf(fmaxf(v * f, -448.f), 448.f) : __uint_as_float(0x7FC00000u);
    }
    int u = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    u = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], u, true);
    w[j] = (unsigned)u;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// A wavefront to four entries of the list, a key head and a kind (keys or values).  It writes the blocks whose first entry is among its
// four, whole: with 64 / LH rows at a time (LH lanes to a head of a row, 16 columns each) it takes the maximum of what is to be
// written, settles the scale, rounds the block's other rows anew where that grew, and writes.  The list ascends, so a block's entries are
// together, and no other wavefront touches this head and kind of the block.  What bounds it: the rows' bytes, read once where
// a block's rows fit the wavefront (64 columns and 16 rows, say), twice, the second time from the L2, where they do not.
__global__ __launch_bounds__(kKvBlock) void k_kv_write(const KvWrite a) {
  const int lane = lane_id();
  const long long unit = (long long)blockIdx.x * kKvWaves + threadIdx.x / kWave;
  const int parts = 2 * a.kv_heads;
  const int kind = (int)(unit % parts) & 1, head = (int)(unit % parts) >> 1;
  const long long i0 = unit / parts * kWriteRows;
  const long long n = a.n_dev ? min(a.n_max, max(0ll, *a.n_dev)) : a.n_max;
  if (i0 >= n) return;
  auto slot_at = [&](long long i) {
    const int s = i < n ? a.slots[i] : -1;
    return (unsigned)s < (unsigned long long)a.n_slots ? s : -1;
  };
  bool first = false;
  if (lane < kWriteRows) {
    const int s = slot_at(i0 + lane);
    const int before = i0 + lane > 0 ? slot_at(i0 + lane - 1) : -1;
    first = s >= 0 && (before < 0 || (before >> a.block_log2) != (s >> a.block_log2));
    if (s >= 0 && i0 + lane > 0 && (before < 0 || before >= s)) *a.host_flag = 2u;  // not ascending: dci_sync says so
  }
  unsigned long long firsts = __ballot(first);
  const int lh = 1 << a.lh_log2, at_once = kWave >> a.lh_log2;
  const int r = lane >> a.lh_log2, col = (lane & (lh - 1)) * kChunk, cols = min(kChunk, max(0, a.dim - col));
  const int width = (a.dim + kChunk - 1) / kChunk * kChunk;
  const char* from = a.from[kind] + ((long long)head * a.dim + col) * type_bytes(a.type);
  unsigned char* to = a.codes + (long long)(kind * a.kv_heads + head) * width + col;
  const long long row_bytes = 2ll * a.kv_heads * width;
  while (firsts) {
    const long long i = i0 + __builtin_ctzll(firsts);
    firsts &= firsts - 1;
    const int block_slots = 1 << a.block_log2;
    const int mine = lane < block_slots ? slot_at(i + lane) : -1;
    const int b = __shfl(mine, 0, kWave) >> a.block_log2;
    const unsigned long long with = __ballot(mine >= 0 && (mine >> a.block_log2) == b);
    const int rows = with == ~0ull ? kWave : __builtin_ctzll(~with);
    const long long slot0 = (long long)b << a.block_log2;
    const int block_rows = (int)min((long long)block_slots, a.n_slots - slot0);
    float amax = 0.f, x[kChunk];
    for (int t = r; t < rows + r; t += at_once) {  // (all lanes take the same turns)
#pragma unroll
      for (int j = 0; j < kChunk; ++j) x[j] = 0.f;
      if (t < rows && cols > 0) read_chunk(a.type, from + (i + t) * a.stride[kind], cols, a.wide[kind], x);
#pragma unroll
      for (int j = 0; j < kChunk; ++j) amax = fmaxf(amax, is_number(x[j]) ? fabsf(x[j]) : 0.f);
    }
    for (int d = kWave / 2; d; d >>= 1) amax = fmaxf(amax, __shfl_xor(amax, d, kWave));
    float* scale = a.scales + 2 * ((long long)b * a.kv_heads + head) + kind;
    const float old = *scale;
    int e = need_exp(amax);
    if (rows < block_rows && old != 0.f) {
      const int old_e = (int)(__float_as_uint(old) >> 23) - 127;
      if (e > old_e) {
        unsigned long long written = lane < rows ? 1ull << (mine & (block_slots - 1)) : 0ull;
        for (int d = kWave / 2; d; d >>= 1) written |= __shfl_xor(written, d, kWave);
        const float up = old * exp2_of(-e);  // 2^(old_e - e), or 0 far below
        for (int t = r; t < block_rows; t += at_once) {
          if (!((written >> t) & 1) && col < width) {
            Chunk<kE4M3> c;
            unsigned char* p = to + (slot0 + t) * row_bytes;
            c.load(reinterpret_cast<const char*>(p), kChunk, true);
            float y[kChunk];
#pragma unroll
            for (int j = 0; j < kChunk / 2; ++j) {
              c.pair(j, y[2 * j], y[2 * j + 1]);
              y[2 * j] *= up;
              y[2 * j + 1] *= up;
            }
            *reinterpret_cast<uint4*>(p) = encode(y, 0);
          }
        }
      } else {
        e = old_e;
      }
    }
    for (int t = r; t < rows + r; t += at_once) {
      if (rows > at_once) {
#pragma unroll
        for (int j = 0; j < kChunk; ++j) x[j] = 0.f;
        if (t < rows && cols > 0) read_chunk(a.type, from + (i + t) * a.stride[kind], cols, a.wide[kind], x);
      }
      const int s = __shfl(mine, min(t, kWave - 1), kWave);
      if (t < rows && col < width) *reinterpret_cast<uint4*>(to + (long long)s * row_bytes) = encode(x, e);
    }
    if (lane == 0) *scale = exp2_of(e);
  }
}

// ---- reading --------------------------------------------------------------------------------------

struct KvRead {
  const int* slots;
  long long n_max;
  const long long* n_dev;
  int type;
  char* to[2];
  long long stride[2];
  bool wide;
  const unsigned char* codes;
  const float* scales;
  long long n_slots;
  int block_log2, kv_heads, dim;
};

// 16 bytes of the output to a lane where that goes (4 or 8 columns), else a number; lanes side by side along a row.  What bounds it: the
// bytes written.
__global__ __launch_bounds__(kKvBlock) void k_kv_read(const KvRead a) {
  const int width = (a.dim + kChunk - 1) / kChunk * kChunk;
  const int per = a.wide ? 16 / type_bytes(a.type) : 1;
  const unsigned head_pieces = (unsigned)(a.dim / per), row_pieces = 2u * a.kv_heads * head_pieces;
  const long long n = a.n_dev ? min(a.n_max, max(0ll, *a.n_dev)) : a.n_max;
  const long long all = n * row_pieces, step = (long long)gridDim.x * kKvBlock;
  for (long long at = blockIdx.x * (long long)kKvBlock + threadIdx.x; at < all; at += step) {
    const long long i = at / row_pieces;
    const unsigned in = (unsigned)(at - i * row_pieces), part = in / head_pieces, col = (in - part * head_pieces) * per;
    const unsigned kind = part / (unsigned)a.kv_heads, head = part - kind * a.kv_heads;
    const int s = a.slots[i];
    if ((unsigned)s >= (unsigned long long)a.n_slots) continue;
    const unsigned char* p = a.codes + ((2ll * s + kind) * a.kv_heads + head) * width + col;
    const float scale = a.scales[2 * ((long long)(s >> a.block_log2) * a.kv_heads + head) + kind];
    char* o = a.to[kind] + i * a.stride[kind] + ((long long)head * a.dim + col) * type_bytes(a.type);
    if (a.wide) {
      Chunk<kE4M3> c;
      c.clear();
      c.w[0].x = *reinterpret_cast<const unsigned*>(p);
      if (per == 8) c.w[0].y = *reinterpret_cast<const unsigned*>(p + 4);
      float y[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        c.pair(j, y[2 * j], y[2 * j + 1]);
        y[2 * j] *= scale;
        y[2 * j + 1] *= scale;
      }
      if (a.type == DCI_F32) *reinterpret_cast<float4*>(o) = make_float4(y[0], y[1], y[2], y[3]);
      else if (a.type == DCI_BF16)
        *reinterpret_cast<uint4*>(o) = make_uint4(two<DCI_BF16>(y[0], y[1]), two<DCI_BF16>(y[2], y[3]), two<DCI_BF16>(y[4], y[5]), two<DCI_BF16>(y[6], y[7]));
      else
        *reinterpret_cast<uint4*>(o) = make_uint4(two<DCI_F16>(y[0], y[1]), two<DCI_F16>(y[2], y[3]), two<DCI_F16>(y[4], y[5]), two<DCI_F16>(y[6], y[7]));
    } else {
      Chunk<kE4M3> c;
      c.clear();
      c.w[0].x = *p;
      float y, unused;
      c.pair(0, y, unused);
      y *= scale;
      if (a.type == DCI_F32) *reinterpret_cast<float*>(o) = y;
      else if (a.type == DCI_BF16) *reinterpret_cast<unsigned short*>(o) = (unsigned short)two<DCI_BF16>(y, 0.f);
      else *reinterpret_cast<unsigned short*>(o) = (unsigned short)two<DCI_F16>(y, 0.f);
    }
  }
}

int32_t check_rows(dci_ctx* ctx, const dci_kv_cache* cache, const int32_t* slots, int64_t n_max, int32_t dtype, const void* k, int64_t k_stride,
                   const void* v, int64_t v_stride) {
  const int32_t rc = check_kv_cache(ctx, cache);
  if (rc != DCI_OK) return rc;
  if (!known_type(dtype)) return fail(ctx, DCI_ERR_INVALID_ARG, "key/value rows: unknown dtype %d", dtype);
  if (n_max < 0 || (n_max > 0 && (!slots || !k || !v))) return fail(ctx, DCI_ERR_INVALID_ARG, "key/value rows: null slots, k or v, or a negative count");
  if (n_max > 0x7FFFFFFFll) return fail(ctx, DCI_ERR_UNSUPPORTED, "key/value rows: more than 2^31-1 rows");
  const int64_t row = (int64_t)cache->kv_heads * cache->head_dim;
  if (k_stride < row || v_stride < row)
    return fail(ctx, DCI_ERR_INVALID_ARG, "key/value rows are kv_heads * head_dim = %lld numbers long, strides %lld and %lld", (long long)row,
                (long long)k_stride, (long long)v_stride);
  if (!aligned_rows(k, dtype) || !aligned_rows(v, dtype)) return fail(ctx, DCI_ERR_INVALID_ARG, "key/value rows must be aligned to their type");
  return DCI_OK;
}

// ---- admission ------------------------------------------------------------------------------------
//
// The m slots of least (weight, slot) among those that the batch does not use, by a radix selection over the weights: a first digit of 12 bits
// that is a floating-point code of the weight (six bits of exponent, six of mantissa: weights differ in their order of magnitude, and a
// digit of their highest bits would be the same for all), then as many digits of 12 bits of the rest as it takes until the slots
// at the border are all alike or all wanted; a digit's counts are added up by workgroup in LDS, then in memory, and the workgroup
// that ends last looks for the border.  Then slots and misses are numbered by prefix sums over tiles, and the j-th slot goes to the j-th
// miss.  What bounds it: launches, and 8 bytes per slot and digit that mostly come from the last-level cache.

constexpr int kDigit = 12, kBins = 1 << kDigit, kDigits = 6;  // 6 bits of exponent and mantissa each, then up to 57 others
constexpr int kAdmitBlock = 256, kNodeTile = 1024, kSlotTile = 2048;

struct AdmitState {
  unsigned ticket[kDigits + 2];
  unsigned hits, evicted;
  unsigned misses;
  unsigned want;  // m
  // the border: slots with weight >> shift == prefix; `need` of the `have` such slots are taken, and all with a smaller weight
  unsigned long long prefix;
  int shift;
  unsigned need, have;
  int done;
};

struct Admit {
  unsigned long long* weight;
  long long* node;
  int* remap;
  long long num_nodes;
  const long long* nodes;
  long long n_max;
  const long long* n_dev;
  int *slots, *fresh, *fresh_slots;
  long long* counts;
  unsigned n_slots;
  AdmitState* st;
  unsigned* hit;        // a bit per slot
  unsigned* hist;       // [kDigits][kBins]
  unsigned* node_tile;  // misses in a tile of nodes, then the sum of those before
  unsigned long long* slot_tile;  // (smaller, at the border) likewise
  int node_tiles, slot_tiles, hist_blocks;
};

constexpr int kClaim = (int)0x80000000;  // remap of a node that place i of the batch asks a slot for: kClaim + i, below -1

__device__ __forceinline__ unsigned first_digit(unsigned long long w) {
  if (w < 64) return (unsigned)w;
  const int e = 63 - __builtin_clzll(w);
  return (unsigned)((e - 5) * 64 + ((w >> (e - 6)) & 63));
}

template <class T>
__device__ __forceinline__ T peek(const T* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <class T>
__device__ __forceinline__ void put(T* p, T v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ long long batch_size(const Admit& a) { return a.n_dev ? min(a.n_max, max(0ll, *a.n_dev)) : a.n_max; }

// Sum of x over the threads before this one, workgroup-wide; total: over all
__device__ unsigned long long block_before(unsigned long long x, unsigned long long* total) {
  __shared__ unsigned long long sums[kAdmitBlock / kWave];
  const unsigned long long incl = (unsigned long long)wave_incl_scan64((long long)x);
  const int wave = (int)threadIdx.x / kWave;
  __syncthreads();
  if (lane_id() == kWave - 1) sums[wave] = incl;
  __syncthreads();
  unsigned long long before = incl - x, all = 0;
#pragma unroll
  for (int w = 0; w < kAdmitBlock / kWave; ++w) {
    if (w < wave) before += sums[w];
    all += sums[w];
  }
  *total = all;
  return before;
}

// True in the workgroup that gets here last of `of`; what the others wrote before (with put, or atomics) is there for it
__device__ bool last_here(unsigned* ticket, unsigned of) {
  __shared__ bool last;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == of - 1;
  __syncthreads();
  if (last) __threadfence();
  return last;
}

// Tile sums become sums of the tiles before; returns the total (one workgroup)
template <class T>
__device__ T scan_tiles(T* tile, int n) {
  unsigned long long carry = 0;
  for (int t0 = 0; t0 < n; t0 += kAdmitBlock) {
    const int t = t0 + (int)threadIdx.x;
    const unsigned long long x = t < n ? (unsigned long long)peek(tile + t) : 0;
    unsigned long long total;
    const unsigned long long before = block_before(x, &total);
    if (t < n) put(tile + t, (T)(carry + before));
    carry += total;
  }
  return (T)carry;
}

__global__ __launch_bounds__(kAdmitBlock) void k_admit_lookup(const Admit a) {
  const long long n = batch_size(a), i = blockIdx.x * (long long)kAdmitBlock + threadIdx.x;
  bool new_hit = false;
  if (i < n) {
    const long long v = a.nodes[i];
    if (v >= 0 && v < a.num_nodes) {
      const int s = peek(a.remap + v);
      if (s >= 0 && (unsigned)s < a.n_slots) {
        const unsigned bit = 1u << (s & 31);
        new_hit = !(atomicOr(a.hit + (s >> 5), bit) & bit);
      } else {
        atomicMin(a.remap + v, kClaim + (int)i);
      }
    }
  }
  const int hits = __popcll(__ballot(new_hit));
  if (lane_id() == 0 && hits) atomicAdd(&a.st->hits, (unsigned)hits);
}

// Place i of the batch is the first of a node without a slot
__device__ __forceinline__ bool is_miss(const Admit& a, long long i, long long n) {
  if (i >= n) return false;
  const long long v = a.nodes[i];
  return v >= 0 && v < a.num_nodes && a.remap[v] == kClaim + (int)i;
}

// One workgroup: the bin in which the need-th slot lies
__device__ void find_border(const Admit& a, const unsigned* hist, int digit) {
  AdmitState* st = a.st;
  __shared__ unsigned found_bin, found_before;
  if (threadIdx.x == 0) found_bin = 0xFFFFFFFFu;
  __syncthreads();
  const unsigned need = digit ? st->need : st->want;
  unsigned long long carry = 0;
  for (int b0 = 0; b0 < kBins; b0 += kAdmitBlock) {
    const unsigned x = peek(hist + b0 + threadIdx.x);
    unsigned long long total;
    const unsigned long long before = carry + block_before(x, &total);
    if (before < need && before + x >= need) {
      found_bin = b0 + threadIdx.x;
      found_before = (unsigned)before;
    }
    carry += total;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    if (need == 0) {
      st->prefix = 0;
      st->shift = 0;
      st->need = st->have = 0;
      st->done = 1;
    } else {
      const unsigned bin = found_bin;
      if (digit == 0) {
        if (bin < 64) {
          st->prefix = bin;
          st->shift = 0;
        } else {
          st->prefix = 64 + (bin & 63);
          st->shift = (int)(bin >> 6) - 1;
        }
      } else {
        const int shift = max(0, st->shift - kDigit);
        st->prefix = (st->prefix << (st->shift - shift)) + bin;
        st->shift = shift;
      }
      st->need = need - found_before;
      st->have = peek(hist + bin);
      st->done = st->shift == 0 || st->need == st->have;
    }
  }
}

// Digit `digit` of the slots at the border; with the first one, workgroups of their own count the misses
__global__ __launch_bounds__(kAdmitBlock) void k_admit_digit(const Admit a, int digit) {
  AdmitState* st = a.st;
  if (digit && st->done) return;
  __shared__ unsigned bins[kBins];
  unsigned* hist = a.hist + digit * kBins;
  if ((int)blockIdx.x < a.hist_blocks) {
    for (int b = (int)threadIdx.x; b < kBins; b += kAdmitBlock) bins[b] = 0;
    __syncthreads();
    const unsigned long long prefix = digit ? st->prefix : 0;
    const int shift = digit ? st->shift : 0, low = max(0, shift - kDigit);
    const unsigned step = (unsigned)a.hist_blocks * kAdmitBlock;
    for (unsigned long long s = blockIdx.x * kAdmitBlock + threadIdx.x; s < a.n_slots; s += step) {
      const unsigned long long w = a.weight[s];
      const bool taken = (a.hit[s >> 5] >> (s & 31)) & 1;
      if (!taken) {
        if (!digit) atomicAdd(&bins[first_digit(w)], 1u);
        else if (w >> shift == prefix) atomicAdd(&bins[(unsigned)(w >> low) & ((1u << (shift - low)) - 1)], 1u);
      }
    }
    __syncthreads();
    for (int b = (int)threadIdx.x; b < kBins; b += kAdmitBlock)
      if (bins[b]) atomicAdd(hist + b, bins[b]);
  } else {
    const long long n = batch_size(a), i0 = (long long)(blockIdx.x - a.hist_blocks) * kNodeTile;
    unsigned count = 0;
    for (int k = 0; k < kNodeTile / kAdmitBlock; ++k) count += is_miss(a, i0 + k * kAdmitBlock + threadIdx.x, n) ? 1 : 0;
    unsigned long long total;
    (void)block_before(count, &total);
    if (threadIdx.x == 0) put(a.node_tile + (blockIdx.x - a.hist_blocks), (unsigned)total);
  }
  if (!last_here(&st->ticket[digit], gridDim.x)) return;
  if (!digit) {
    const unsigned misses = scan_tiles(a.node_tile, a.node_tiles);
    if (threadIdx.x == 0) {
      st->misses = misses;
      st->want = min(misses, a.n_slots - peek(&st->hits));
    }
    __syncthreads();
  }
  find_border(a, hist, digit);
}

// (weight below the border, at it) of a slot, in the high and the low half
__device__ __forceinline__ unsigned long long side_of(const Admit& a, unsigned long long s, unsigned long long prefix, int shift) {
  if (s >= a.n_slots || ((a.hit[s >> 5] >> (s & 31)) & 1)) return 0;
  const unsigned long long p = a.weight[s] >> shift;
  return p < prefix ? 1ull << 32 : p == prefix ? 1ull : 0ull;
}

// How many slots of every tile are taken, and the list of the misses that get one
__global__ __launch_bounds__(kAdmitBlock) void k_admit_number(const Admit a) {
  AdmitState* st = a.st;
  if ((int)blockIdx.x < a.slot_tiles) {
    const unsigned long long s0 = (unsigned long long)blockIdx.x * kSlotTile, prefix = st->prefix;
    const int shift = st->shift;
    unsigned long long sum = 0, total;
    if (st->want)
      for (int k = 0; k < kSlotTile / kAdmitBlock; ++k) sum += side_of(a, s0 + k * kAdmitBlock + threadIdx.x, prefix, shift);
    (void)block_before(sum, &total);
    if (threadIdx.x == 0) put(a.slot_tile + blockIdx.x, total);
    if (last_here(&st->ticket[kDigits], (unsigned)a.slot_tiles)) (void)scan_tiles(a.slot_tile, a.slot_tiles);
    return;
  }
  const long long n = batch_size(a);
  const unsigned want = st->want, tile = blockIdx.x - a.slot_tiles;
  unsigned long long carry = a.node_tile[tile];
  for (int k = 0; k < kNodeTile / kAdmitBlock; ++k) {
    const long long i = (long long)tile * kNodeTile + k * kAdmitBlock + threadIdx.x;
    const bool miss = is_miss(a, i, n);
    unsigned long long total;
    const unsigned long long j = carry + block_before(miss ? 1 : 0, &total);
    if (miss && j < want) a.fresh[j] = (int)i;
    if (i >= want && i < a.n_max) {
      a.fresh[i] = -1;
      a.fresh_slots[i] = -1;
    }
    carry += total;
  }
}

// The j-th slot to the j-th miss
__global__ __launch_bounds__(kAdmitBlock) void k_admit_give(const Admit a) {
  AdmitState* st = a.st;
  const unsigned want = st->want;
  if (!want) return;
  const unsigned long long prefix = st->prefix;
  const int shift = st->shift;
  const unsigned need = st->need;
  constexpr int kPer = kSlotTile / kAdmitBlock;
  const unsigned long long s0 = (unsigned long long)blockIdx.x * kSlotTile + threadIdx.x * kPer;
  unsigned long long side[kPer], sum = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    side[k] = side_of(a, s0 + k, prefix, shift);
    sum += side[k];
  }
  unsigned long long total;
  unsigned long long before = a.slot_tile[blockIdx.x] + block_before(sum, &total);
  unsigned evicted = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const unsigned smaller = (unsigned)(before >> 32), equal = (unsigned)before;
    if (side[k] >> 32 || (side[k] && equal < need)) {
      const unsigned j = smaller + min(equal, need);
      const int s = (int)(s0 + k);
      const long long v = a.nodes[a.fresh[j]], old = a.node[s];
      if (old >= 0 && old < a.num_nodes) {
        a.remap[old] = -1;
        ++evicted;
      }
      a.node[s] = v;
      a.weight[s] = 1;
      a.remap[v] = s;
      a.fresh_slots[j] = s;
    }
    before += side[k];
  }
  (void)block_before(evicted, &total);
  if (threadIdx.x == 0 && total) atomicAdd(&st->evicted, (unsigned)total);
}

// The slots of the batch; claims that got none are taken back
__global__ __launch_bounds__(kAdmitBlock) void k_admit_slots(const Admit a) {
  const long long n = batch_size(a), i = blockIdx.x * (long long)kAdmitBlock + threadIdx.x;
  if (i == 0) {
    const AdmitState* st = a.st;
    a.counts[0] = st->want;
    a.counts[1] = st->misses;
    a.counts[2] = st->hits;
    a.counts[3] = st->evicted;
  }
  if (i >= n) return;
  const long long v = a.nodes[i];
  int s = -1;
  if (v >= 0 && v < a.num_nodes) {
    s = a.remap[v];
    if (s == kClaim + (int)i) a.remap[v] = -1;
    if (s < 0) s = -1;
  }
  a.slots[i] = s;
}

struct AdmitSpace {
  AdmitState* st;
  unsigned *hit, *hist, *node_tile;
  unsigned long long* slot_tile;
  size_t clear_bytes;  // from st on
};
AdmitSpace admit_space(Arena& ar, int64_t n_slots, int64_t n_max) {
  AdmitSpace s;
  s.st = ar.take<AdmitState>(1);
  s.hist = ar.take<unsigned>((size_t)kDigits * kBins);
  s.hit = ar.take<unsigned>((size_t)(n_slots + 31) / 32);
  s.clear_bytes = ar.off;
  s.node_tile = ar.take<unsigned>((size_t)(n_max + kNodeTile - 1) / kNodeTile);
  s.slot_tile = ar.take<unsigned long long>((size_t)(n_slots + kSlotTile - 1) / kSlotTile);
  return s;
}

}  // namespace
}  // namespace dci

extern "C" {

int32_t dci_kv_clear(dci_ctx* ctx, const dci_kv_cache* cache) {
  const int32_t rc = dci::check_kv_cache(ctx, cache);
  if (rc != DCI_OK) return rc;
  const dci::OnDevice on(ctx->device);
  DCI_HIP(ctx, on.err);
  const int64_t n16 = cache->n_slots * 2 * cache->kv_heads * (dci::kv_width(cache->head_dim) / dci::kChunk);
  const int64_t blocks = (cache->n_slots + cache->block - 1) / cache->block;
  int64_t grid = (n16 + dci::kKvBlock - 1) / dci::kKvBlock;
  if (grid > (int64_t)ctx->num_cus * 8) grid = (int64_t)ctx->num_cus * 8;
  dci::Timed timed(ctx, DCI_K_KV);
  hipLaunchKernelGGL(dci::k_kv_clear, dim3((unsigned)grid), dim3(dci::kKvBlock), 0, ctx->stream, reinterpret_cast<uint4*>(cache->codes), (long long)n16,
                     cache->scales, (long long)(blocks * cache->kv_heads * 2), reinterpret_cast<unsigned long long*>(cache->weight),
                     reinterpret_cast<long long*>(cache->node), (long long)cache->n_slots);
  DCI_LAUNCH_CHECK(ctx);
  return DCI_OK;
}

int32_t dci_kv_write(dci_ctx* ctx, const dci_kv_cache* cache, const int32_t* slots, int64_t n_max, const int64_t* n_dev, int32_t dtype,
                     const void* k, int64_t k_stride, const void* v, int64_t v_stride) {
  const int32_t rc = dci::check_rows(ctx, cache, slots, n_max, dtype, k, k_stride, v, v_stride);
  if (rc != DCI_OK) return rc;
  if (n_max == 0) return DCI_OK;
  const dci::OnDevice on(ctx->device);
  DCI_HIP(ctx, on.err);
  const int64_t bytes = dci::type_bytes(dtype);
  dci::KvWrite a = {};
  a.slots = slots;
  a.n_max = n_max;
  a.n_dev = reinterpret_cast<const long long*>(n_dev);
  a.type = dtype;
  a.from[0] = static_cast<const char*>(k);
  a.from[1] = static_cast<const char*>(v);
  a.stride[0] = k_stride * bytes;
  a.stride[1] = v_stride * bytes;
  a.wide[0] = dci::by_16_bytes(k, k_stride, cache->head_dim, dtype);
  a.wide[1] = dci::by_16_bytes(v, v_stride, cache->head_dim, dtype);
  a.codes = cache->codes;
  a.scales = cache->scales;
  a.n_slots = cache->n_slots;
  a.block_log2 = dci::log2_up(cache->block);
  a.kv_heads = cache->kv_heads;
  a.dim = cache->head_dim;
  a.lh_log2 = dci::log2_up((cache->head_dim + dci::kChunk - 1) / dci::kChunk);
  a.host_flag = ctx->host_flag;
  const int64_t waves = (n_max + dci::kWriteRows - 1) / dci::kWriteRows * 2 * cache->kv_heads;
  const int64_t grid = (waves + dci::kKvWaves - 1) / dci::kKvWaves;
  if (grid > 0x7FFFFFFFll) return dci::fail(ctx, DCI_ERR_UNSUPPORTED, "key/value rows: too many rows and heads for one call");
  dci::Timed timed(ctx, DCI_K_KV);
  hipLaunchKernelGGL(dci::k_kv_write, dim3((unsigned)grid), dim3(dci::kKvBlock), 0, ctx->stream, a);
  DCI_LAUNCH_CHECK(ctx);
  return DCI_OK;
}

int32_t dci_kv_read(dci_ctx* ctx, const dci_kv_cache* cache, const int32_t* slots, int64_t n_max, const int64_t* n_dev, int32_t dtype,
                    void* k, int64_t k_stride, void* v, int64_t v_stride) {
  const int32_t rc = dci::check_rows(ctx, cache, slots, n_max, dtype, k, k_stride, v, v_stride);
  if (rc != DCI_OK) return rc;
  if (n_max == 0) return DCI_OK;
  const dci::OnDevice on(ctx->device);
  DCI_HIP(ctx, on.err);
  const int64_t bytes = dci::type_bytes(dtype);
  dci::KvRead a = {};
  a.slots = slots;
  a.n_max = n_max;
  a.n_dev = reinterpret_cast<const long long*>(n_dev);
  a.type = dtype;
  a.to[0] = static_cast<char*>(k);
  a.to[1] = static_cast<char*>(v);
  a.stride[0] = k_stride * bytes;
  a.stride[1] = v_stride * bytes;
  a.wide = dci::by_16_bytes(k, k_stride, cache->head_dim, dtype) && dci::by_16_bytes(v, v_stride, cache->head_dim, dtype);
  a.codes = cache->codes;
  a.scales = cache->scales;
  a.n_slots = cache->n_slots;
  a.block_log2 = dci::log2_up(cache->block);
  a.kv_heads = cache->kv_heads;
  a.dim = cache->head_dim;
  const int64_t pieces = n_max * 2 * cache->kv_heads * (a.wide ? cache->head_dim * bytes / 16 : cache->head_dim);
  int64_t grid = (pieces + dci::kKvBlock - 1) / dci::kKvBlock;
  if (grid > (int64_t)ctx->num_cus * 64) grid = (int64_t)ctx->num_cus * 64;
  dci::Timed timed(ctx, DCI_K_KV);
  hipLaunchKernelGGL(dci::k_kv_read, dim3((unsigned)grid), dim3(dci::kKvBlock), 0, ctx->stream, a);
  DCI_LAUNCH_CHECK(ctx);
  return DCI_OK;
}

size_t dci_kv_admit_workspace_bytes(int64_t n_slots, int64_t n_max) {
  if (n_slots < 1 || n_max < 0) return 0;
  dci::Arena ar(nullptr, 0);
  (void)dci::admit_space(ar, n_slots, n_max);
  return ar.off;
}

int32_t dci_kv_admit(dci_ctx* ctx, const dci_kv_cache* cache, int32_t* remap, int64_t num_nodes, const int64_t* nodes, int64_t n_max,
                     const int64_t* n_dev, int32_t* slots, int32_t* fresh, int32_t* fresh_slots, int64_t* counts) {
  const int32_t rc = dci::check_kv_cache(ctx, cache);
  if (rc != DCI_OK) return rc;
  if (!cache->weight || !cache->node) return dci::fail(ctx, DCI_ERR_INVALID_ARG, "admission: the cache has no weights or nodes");
  if (!remap || num_nodes < 1 || !counts || n_max < 0 || (n_max > 0 && (!nodes || !slots || !fresh || !fresh_slots)))
    return dci::fail(ctx, DCI_ERR_INVALID_ARG, "admission: null remap, nodes, slots, fresh, fresh_slots or counts, or a negative size");
  if (n_max > 0x7FFFFFFFll - 1 || num_nodes > 0x7FFFFFFFll) return dci::fail(ctx, DCI_ERR_UNSUPPORTED, "admission: more than 2^31-1 nodes, or 2^31-2 in a batch");
  dci::Arena ar(ctx->ws, ctx->ws_bytes);
  const dci::AdmitSpace sp = dci::admit_space(ar, cache->n_slots, n_max);
  if (!ar.ok()) {
    ctx->req_workspace = ar.off;
    return dci::fail(ctx, DCI_ERR_CAPACITY, "workspace holds %zu bytes, admission needs %zu", ctx->ws_bytes, ar.off);
  }
  const dci::OnDevice on(ctx->device);
  DCI_HIP(ctx, on.err);
  dci::Admit a = {};
  a.weight = reinterpret_cast<unsigned long long*>(cache->weight);
  a.node = reinterpret_cast<long long*>(cache->node);
  a.remap = remap;
  a.num_nodes = num_nodes;
  a.nodes = reinterpret_cast<const long long*>(nodes);
  a.n_max = n_max;
  a.n_dev = reinterpret_cast<const long long*>(n_dev);
  a.slots = slots;
  a.fresh = fresh;
  a.fresh_slots = fresh_slots;
  a.counts = reinterpret_cast<long long*>(counts);
  a.n_slots = (unsigned)cache->n_slots;
  a.st = sp.st;
  a.hit = sp.hit;
  a.hist = sp.hist;
  a.node_tile = sp.node_tile;
  a.slot_tile = sp.slot_tile;
  a.node_tiles = (int)((n_max + dci::kNodeTile - 1) / dci::kNodeTile);
  a.slot_tiles = (int)((cache->n_slots + dci::kSlotTile - 1) / dci::kSlotTile);
  a.hist_blocks = a.slot_tiles < 128 ? a.slot_tiles : 128;
  const unsigned node_blocks = (unsigned)(n_max > 0 ? (n_max + dci::kAdmitBlock - 1) / dci::kAdmitBlock : 1);
  dci::Timed timed(ctx, DCI_K_KV);
  const int32_t filled = dci::fill_bytes(ctx, sp.st, sp.clear_bytes, 0);
  if (filled != DCI_OK) return filled;
#define DCI_ADMIT(kernel_, grid_, ...)                                                                                       \
  do {                                                                                                                       \
    hipLaunchKernelGGL(kernel_, dim3((unsigned)(grid_)), dim3(dci::kAdmitBlock), 0, ctx->stream, ##__VA_ARGS__);             \
    DCI_LAUNCH_CHECK(ctx);                                                                                                   \
  } while (0)
  DCI_ADMIT(dci::k_admit_lookup, node_blocks, a);
  for (int digit = 0; digit < dci::kDigits; ++digit) DCI_ADMIT(dci::k_admit_digit, a.hist_blocks + (digit ? 0 : a.node_tiles), a, digit);
  DCI_ADMIT(dci::k_admit_number, a.slot_tiles + a.node_tiles, a);
  DCI_ADMIT(dci::k_admit_give, a.slot_tiles, a);
  DCI_ADMIT(dci::k_admit_slots, node_blocks, a);
#undef DCI_ADMIT
  return DCI_OK;
}

}  // extern "C"
