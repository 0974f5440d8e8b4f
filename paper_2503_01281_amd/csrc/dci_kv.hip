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
  bool wide, odd;       // heads of 16 columns at least, or of a multiple of 16 bytes: read by 16 bytes; of those, heads that end inside 16 bytes
  unsigned char* codes;
  float* scales;
  long long n_slots;
  int block_log2, kv_heads, dim, lh_log2;
  unsigned first_turn;  // of this launch
  unsigned* host_flag;
};

__device__ __forceinline__ bool is_number(float x) { return (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u; }

// The least e with amax <= 448 * 2^e, 448 = 1.75 * 2^8
__device__ __forceinline__ int need_exp(float amax) {
  const unsigned u = __float_as_uint(amax);
  if (u == 0) return kMinExp;
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return min(max(e, kMinExp), kMaxExp);  // (an fp32 number below 2^-126 comes out below kMinExp all the same)
}
__device__ __forceinline__ float exp2_of(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }

// 16 numbers as codes, each divided by 2^e first; rounded to nearest even, at most 448.  (The conversion makes NaN of infinities by itself, but of
// numbers beyond 464 as well, and those only kMaxExp leaves.)
__device__ __forceinline__ uint4 encode(const float (&x)[kChunk], int e) {
  const float f = exp2_of(-e);
  float y[kChunk];
#pragma unroll
  for (int j = 0; j < kChunk; ++j) y[j] = x[j] * f;
  if (__builtin_expect(e == kMaxExp, 0)) {
#pragma unroll
    for (int j = 0; j < kChunk; ++j) y[j] = is_number(y[j]) ? fminf(fmaxf(y[j], -448.f), 448.f) : y[j];
  }
  unsigned w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    int u = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * j], y[4 * j + 1], 0, false);
    u = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * j + 2], y[4 * j + 3], u, true);
    w[j] = (unsigned)u;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// The greatest magnitude among the numbers that are some (infinities are rare, and looked for once one has shown)
__device__ __forceinline__ float peak_of(const float (&x)[kChunk]) {
  float amax = 0.f;
#pragma unroll
  for (int j = 0; j < kChunk; ++j) amax = fmaxf(amax, fabsf(x[j]));
  if (!is_number(amax)) {
    amax = 0.f;
#pragma unroll
    for (int j = 0; j < kChunk; ++j) amax = fmaxf(amax, is_number(x[j]) ? fabsf(x[j]) : 0.f);
  }
  return amax;
}

// A lane's 16 columns of a head, from `col` on.  Where the head ends inside 16 bytes of them (odd), its last 16 columns are read, wherever they
// lie: `skip` of those are the lane's before, and shift_down brings its own to their place, zeros behind them.  (Number by number, 200,000 rows of
// 16-bit heads of 97 take twice as long; heads of 72 take 8 % less as they are than with a shift.)
struct Piece {
  int from, cols, skip;
  __device__ __forceinline__ Piece(int col, int dim, bool odd) {
    from = odd ? min(col, dim - kChunk) : col;
    cols = col >= dim ? 0 : odd ? kChunk : min(kChunk, dim - col);
    skip = cols ? col - from : 0;
  }
};

// The block whose entries are rows [i, i + rows) of the list, for one head and kind, by a whole wavefront: first the maximum of what is to be
// written, then the scale, the block's other rows where that grew, the rows.  mine: lane t's slot, -1 where it is none of the block's.
template <int TYPE>
__device__ void write_block(const KvWrite& a, int kind, int head, long long i, int mine) {
  const int lane = lane_id(), lh = 1 << a.lh_log2, at_once = kWave >> a.lh_log2;
  const int r = lane >> a.lh_log2, col = (lane & (lh - 1)) * kChunk;
  const Piece piece(col, a.dim, a.odd);
  const int width = (a.dim + kChunk - 1) / kChunk * kChunk, block_slots = 1 << a.block_log2;
  const char* from = a.from[kind] + ((long long)head * a.dim + piece.from) * type_bytes(TYPE);
  unsigned char* to = a.codes + (long long)(kind * a.kv_heads + head) * width + col;
  const long long row_bytes = 2ll * a.kv_heads * width;
  const unsigned long long with = __ballot(mine >= 0);
  const int rows = with == ~0ull ? kWave : __builtin_ctzll(~with);
  const int b = __shfl(mine, 0, kWave) >> a.block_log2;
  const long long slot0 = (long long)b << a.block_log2;
  const int block_rows = (int)min((long long)block_slots, a.n_slots - slot0);
  float amax = 0.f, x[kChunk];
  for (int t0 = 0; t0 < rows; t0 += at_once) {
    const int t = t0 + r;
    if (t < rows && piece.cols > 0) {
      read_chunk_as<TYPE>(from + (i + t) * a.stride[kind], piece.cols, a.wide, x);
      amax = fmaxf(amax, peak_of(x));
    }
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
  for (int t0 = 0; t0 < rows; t0 += at_once) {
    const int t = t0 + r, s = __shfl(mine, min(t, kWave - 1), kWave);
    if (t < rows && col < width) {
#pragma unroll
      for (int j = 0; j < kChunk; ++j) x[j] = 0.f;
      if (piece.cols > 0) read_chunk_as<TYPE>(from + (i + t) * a.stride[kind], piece.cols, a.wide, x);
      if (a.odd) shift_down(x, piece.skip);
      *reinterpret_cast<uint4*>(to + (long long)s * row_bytes) = encode(x, e);
    }
  }
  if (lane == 0) *scale = exp2_of(e);
}

// A wavefront to T * 64 / LH entries of the list (LH lanes to a head of a row, 16 columns each) and a key head.  It writes the blocks whose first
// entry is among its own, whole; the list ascends, so a block's entries are together, and no other wavefront touches this head of the block.  Its
// slots come first, as entries outside the cache have no rows (0 to 3 % slower than all rows at once for half a million rows, 1 to 8 % quicker
// for fewer), then all rows, keys and values.  The blocks that end among the wavefront's entries are done side by side, their maxima joined in LDS; one that goes on behind them, and one whose other rows have to be rounded
// anew, is done on its own (write_block).  What bounds it: the rows' bytes, read and written once (half a million rows of 512 numbers in 16 bits:
// 142 to 176 us, by what the last-level cache has of them, 0.78 GB, 4.4 to 5.5 TB/s).
template <int TYPE, int T>
__global__ __launch_bounds__(kKvBlock) void k_kv_write(const KvWrite a) {
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const unsigned unit = blockIdx.x * (unsigned)kKvWaves + wave, turn = unit / (unsigned)a.kv_heads;
  const int head = (int)(unit - turn * a.kv_heads);
  const int lh = 1 << a.lh_log2, at_once = kWave >> a.lh_log2, tile = T * at_once;
  const long long i0 = ((long long)a.first_turn + turn) * tile;
  const long long n = a.n_dev ? min(a.n_max, max(0ll, *a.n_dev)) : a.n_max;
  __shared__ unsigned peaks[kKvWaves][2][kWave];
  if (i0 >= n) return;
  const int r = lane >> a.lh_log2, col = (lane & (lh - 1)) * kChunk;
  const Piece piece(col, a.dim, a.odd);
  const int width = (a.dim + kChunk - 1) / kChunk * kChunk;
  auto slot_at = [&](long long i) {
    const int s = i < n ? a.slots[i] : -1;
    return (unsigned)s < (unsigned long long)a.n_slots ? s : -1;
  };
  const int s = lane < tile ? slot_at(i0 + lane) : -1;
  const unsigned long long real = __ballot(s >= 0);
  const int count = real == ~0ull ? kWave : __builtin_ctzll(~real);  // entries before the first that is outside: behind them there need be no rows
  Chunk<TYPE> x[2][T];
#pragma unroll
  for (int kind = 0; kind < 2; ++kind) {
    const char* from = a.from[kind] + ((long long)head * a.dim + piece.from) * type_bytes(TYPE);
#pragma unroll
    for (int k = 0; k < T; ++k) {
      x[kind][k].clear();
      const long long i = i0 + k * at_once + r;
      if (k * at_once + r < count && piece.cols > 0) x[kind][k].load(from + i * a.stride[kind], piece.cols, a.wide);
    }
  }
  const int before = i0 + lane > 0 && lane < tile ? slot_at(i0 + lane - 1) : -1;
  const int behind = slot_at(i0 + tile);
  peaks[wave][0][lane] = peaks[wave][1][lane] = 0;
  const bool is_first = s >= 0 && (before < 0 || (before >> a.block_log2) != (s >> a.block_log2));
  if (s >= 0 && i0 + lane > 0 && (before < 0 || before >= s)) *a.host_flag = 1u;  // not ascending: dci_sync says so
  const unsigned long long firsts = __ballot(is_first);
  if (!firsts) return;
  const int last_first = kWave - 1 - __builtin_clzll(firsts);
  // the last block, if it goes on behind these entries
  const bool open = count == tile && behind >= 0 && behind >> a.block_log2 == __shfl(s, tile - 1, kWave) >> a.block_log2;
  const unsigned long long closed = open ? firsts & ((1ull << last_first) - 1) : firsts;
  auto first_of = [&](int row) {  // the first entry of a row's block, -1: not done here
    const unsigned long long up_to = firsts & ((2ull << row) - 1);
    if (!up_to || row >= count) return -1;
    const int f = kWave - 1 - __builtin_clzll(up_to);
    return (closed >> f) & 1 ? f : -1;
  };
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int kind = 0; kind < 2; ++kind) {
#pragma unroll
    for (int k = 0; k < T; ++k) {
      float y[kChunk];
#pragma unroll
      for (int j = 0; j < kChunk / 2; ++j) x[kind][k].pair(j, y[2 * j], y[2 * j + 1]);
      const float amax = max_lanes(peak_of(y), a.lh_log2);
      const int f = first_of(k * at_once + r);
      if (f >= 0 && col == 0) atomicMax(&peaks[wave][kind][f], __float_as_uint(amax));
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  // lane f settles the scales of the block that begins with entry f
  int e[2] = {0, 0};
  bool apart[2] = {false, false};
  if ((closed >> lane) & 1) {
    const unsigned long long later = firsts >> 1 >> lane;
    const int rows = (later ? lane + 1 + __builtin_ctzll(later) : count) - lane;
    const int b = s >> a.block_log2;
    const int block_rows = (int)min(1ll << a.block_log2, a.n_slots - ((long long)b << a.block_log2));
    float2* scales = reinterpret_cast<float2*>(a.scales) + (long long)b * a.kv_heads + head;
    float2 now = make_float2(0.f, 0.f);  // a block that is written whole keeps nothing
    if (rows < block_rows) now = *scales;
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
      const float old = kind ? now.y : now.x;
      e[kind] = need_exp(__uint_as_float(peaks[wave][kind][lane]));
      if (old != 0.f) {
        const int old_e = (int)(__float_as_uint(old) >> 23) - 127;
        apart[kind] = e[kind] > old_e;
        e[kind] = max(e[kind], old_e);
      }
    }
    *scales = make_float2(apart[0] ? now.x : exp2_of(e[0]), apart[1] ? now.y : exp2_of(e[1]));
  }
  const unsigned long long go_on = open ? 1ull << last_first : 0ull;
#pragma unroll
  for (int kind = 0; kind < 2; ++kind) {
    const unsigned long long alone = __ballot(apart[kind]) | go_on;
#pragma unroll
    for (int k = 0; k < T; ++k) {
      const int row = k * at_once + r, f = first_of(row);
      const int to_e = __shfl(e[kind], max(f, 0), kWave), to_s = __shfl(s, row, kWave);
      if (f >= 0 && !((alone >> f) & 1) && col < width) {
        float y[kChunk];
#pragma unroll
        for (int j = 0; j < kChunk / 2; ++j) x[kind][k].pair(j, y[2 * j], y[2 * j + 1]);
        if (a.odd) shift_down(y, piece.skip);
        *reinterpret_cast<uint4*>(a.codes + ((2ll * to_s + kind) * a.kv_heads + head) * width + col) = encode(y, to_e);
      }
    }
    for (unsigned long long todo = alone; todo; todo &= todo - 1) {
      const long long i = i0 + __builtin_ctzll(todo);
      int mine = lane < 1 << a.block_log2 ? slot_at(i + lane) : -1;
      if (mine >= 0 && mine >> a.block_log2 != __shfl(mine, 0, kWave) >> a.block_log2) mine = -1;
      write_block<TYPE>(a, kind, head, i, mine);
    }
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
  const unsigned char* codes;
  const float* scales;
  long long n_slots;
  int block_log2, kv_heads, dim;
  int lanes_log2;  // lanes to a row
};

// 16 bytes of the output to a lane (4 or 8 columns; a head's last piece ends with it, and has columns of the one before as well), a number where heads
// are narrower.  Lanes lie side by side along a row, `lanes` of them (a
// power of two up to a workgroup) to a row, and a lane keeps its place in the rows; four rows at a time.  What bounds it: the bytes
// written (PAST: past the caches; half a million rows of 512 numbers as fp32: 268 us, 1.3 GB, 4.9 TB/s).
template <int TYPE, bool WIDE, bool PAST>
__global__ __launch_bounds__(kKvBlock) void k_kv_read(const KvRead a) {
  constexpr int kPer = WIDE ? 16 / type_bytes(TYPE) : 1, kAtOnce = 4;
  const int width = (a.dim + kChunk - 1) / kChunk * kChunk;
  const unsigned head_pieces = (unsigned)(a.dim + kPer - 1) / kPer, row_pieces = 2u * a.kv_heads * head_pieces;
  const long long n = a.n_dev ? min(a.n_max, max(0ll, *a.n_dev)) : a.n_max;
  const int lanes = 1 << a.lanes_log2, rows = kKvBlock >> a.lanes_log2;
  const long long step = (long long)gridDim.x * rows;
  for (unsigned in = threadIdx.x & (lanes - 1); in < row_pieces; in += lanes) {
    const unsigned part = in / head_pieces, col = min((in - part * head_pieces) * kPer, (unsigned)(a.dim - kPer));
    const unsigned kind = part / (unsigned)a.kv_heads, head = part - kind * a.kv_heads;
    const unsigned char* codes = a.codes + (long long)part * width + col;
    const float* scales = a.scales + 2 * head + kind;
    char* to = (kind ? a.to[1] : a.to[0]) + ((long long)head * a.dim + col) * type_bytes(TYPE);
    const long long stride = kind ? a.stride[1] : a.stride[0];
    for (long long i0 = blockIdx.x * (long long)rows + (threadIdx.x >> a.lanes_log2); i0 < n; i0 += kAtOnce * step) {
      int s[kAtOnce];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        s[k] = i0 + k * step < n ? a.slots[i0 + k * step] : -1;
        if ((unsigned)s[k] >= (unsigned long long)a.n_slots) s[k] = -1;
      }
      Chunk<kE4M3> c[kAtOnce];
      float scale[kAtOnce];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        c[k].clear();
        scale[k] = 0.f;
        if (s[k] >= 0) {
          const unsigned char* p = codes + s[k] * (2ll * a.kv_heads * width);
          if (!WIDE) c[k].w[0].x = *p;
          else if (kPer == 4) c[k].w[0].x = *reinterpret_cast<const u32_any*>(p);
          else {
            const u32x2_any u = *reinterpret_cast<const u32x2_any*>(p);
            c[k].w[0].x = u.x;
            c[k].w[0].y = u.y;
          }
          scale[k] = scales[2ll * (s[k] >> a.block_log2) * a.kv_heads];
        }
      }
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        if (s[k] < 0) continue;
        float y[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          c[k].pair(j, y[2 * j], y[2 * j + 1]);
          y[2 * j] *= scale[k];
          y[2 * j + 1] *= scale[k];
        }
        char* o = to + (i0 + k * step) * stride;
        if (!WIDE) {
          if (TYPE == DCI_F32) *reinterpret_cast<float*>(o) = y[0];
          else *reinterpret_cast<unsigned short*>(o) = (unsigned short)two<TYPE>(y[0], 0.f);
        } else {
          const uint4 u = TYPE == DCI_F32 ? make_uint4(__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3]))
                                          : make_uint4(two<TYPE>(y[0], y[1]), two<TYPE>(y[2], y[3]), two<TYPE>(y[4], y[5]), two<TYPE>(y[6], y[7]));
          if (PAST) store_16_past(o, u);
          else store_16(o, u);
        }
      }
    }
  }
}

template <int TYPE>
void launch_write(int tiles, const KvWrite& a, unsigned grid, hipStream_t stream) {
  if (tiles == 1) hipLaunchKernelGGL((k_kv_write<TYPE, 1>), dim3(grid), dim3(kKvBlock), 0, stream, a);
  else if (tiles == 2) hipLaunchKernelGGL((k_kv_write<TYPE, 2>), dim3(grid), dim3(kKvBlock), 0, stream, a);
  else if (tiles == 4) hipLaunchKernelGGL((k_kv_write<TYPE, 4>), dim3(grid), dim3(kKvBlock), 0, stream, a);
  else hipLaunchKernelGGL((k_kv_write<TYPE, 8>), dim3(grid), dim3(kKvBlock), 0, stream, a);
}
template <int TYPE>
void launch_read(bool wide, bool past, const KvRead& a, unsigned grid, hipStream_t stream) {
  if (!wide) hipLaunchKernelGGL((k_kv_read<TYPE, false, false>), dim3(grid), dim3(kKvBlock), 0, stream, a);
  else if (past) hipLaunchKernelGGL((k_kv_read<TYPE, true, true>), dim3(grid), dim3(kKvBlock), 0, stream, a);
  else hipLaunchKernelGGL((k_kv_read<TYPE, true, false>), dim3(grid), dim3(kKvBlock), 0, stream, a);
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
// The m slots of least (weight, slot) among those that the batch does not use, by a radix selection over the weights: a first digit of 13 bits
// that is a floating-point code of the weight (six bits of exponent, seven of mantissa: weights differ in their order of magnitude, and a
// digit of their highest bits would be the same for all), then digits of 13 bits of the rest, until the slots at the border are all alike or
// all wanted.  A digit's counts are added up by workgroup in LDS, then in memory; every workgroup of the next kernel looks for the border in them.  Three
// digits tell weights apart that differ by 2^-33 of themselves (all of them below 16); what is left after that, one workgroup does by itself.
// Slots and misses are kept as bit masks, numbered by prefix sums over tiles of them, and the j-th slot goes to the j-th miss.  While the call
// runs, the slots that are hit have the highest bit of their weight set.
// Nothing waits for another workgroup: what a kernel leaves is looked through by every workgroup of the next (the counts of a digit, the sums of at
// most 1,024 tiles).  What bounds it: seven launches (eight for large caches) one after the other, each a few dependent reads long, and for large
// batches the random lines of remap, weights and nodes.  400,000 nodes on a million slots take 87 us: 21 of them the look-up (0.55 million lines that
// L2 does not have, 26 a nanosecond, and 0.24 million atomics), 11 the first digit, 12 the other two, 10 numbering, 15 giving, 8 the slots; 3,000 nodes
// on 65,536 slots take 37 us in launches of 3 to 7 us.

constexpr int kDigit = 13, kBins = 1 << kDigit, kDigits = 3;
constexpr int kMantissa = 7;  // of the first digit
constexpr int kDigitBlock = 1024, kDigitSlots = 8;  // lanes; slots to a lane at a time
constexpr int kAdmitBlock = 256, kStretch = 2048, kStretchWords = kStretch / 64;
constexpr int kTiles = 1024;  // at most, of slots and of the batch
constexpr int kHistBlocks = 256;

// Slots with weight >> shift == prefix are at the border: `need` of them are taken, and all with a smaller weight
struct Border {
  unsigned long long prefix;
  int shift;
  unsigned need;
  int done;
};
struct AdmitState {
  Border border[kDigits];  // after digit 0, 1, and all
  unsigned misses, hits;
  unsigned want;  // m
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
  unsigned* hist;                 // [kDigits][kBins]
  unsigned* hit_part;             // [kHistBlocks] slots hit
  unsigned long long* node_mask;  // a bit per place of the batch: a miss
  unsigned* node_tile;            // misses in a tile of the batch
  unsigned long long* slot_mask;  // [2] per 64 slots: weight below the border, at it
  unsigned long long* slot_tile;  // (below, at) in a tile of slots, in the high and the low half
  unsigned* gone_tile;            // nodes that lost their slot
  int node_tiles, node_tile_blocks;    // tiles of the batch, kDigitBlock places times that many each
  int slot_tiles, slot_tile_stretches; // tiles of slots, kStretch slots times that many each
  int hist_blocks;
};

constexpr int kClaim = (int)0x80000000;  // remap of a node that place i of the batch asks a slot for: kClaim + i, below -1

__device__ __forceinline__ unsigned first_digit(unsigned long long w) {
  if (w < 1u << kMantissa) return (unsigned)w;
  const int e = 63 - __builtin_clzll(w);
  return (unsigned)(((e - kMantissa + 1) << kMantissa) + ((w >> (e - kMantissa)) & ((1 << kMantissa) - 1)));
}

__device__ __forceinline__ long long batch_size(const Admit& a) { return a.n_dev ? min(a.n_max, max(0ll, *a.n_dev)) : a.n_max; }
constexpr unsigned long long kHit = 1ull << 63;  // in a weight

// Sum of x over the threads before this one, workgroup-wide; total: over all
template <int BLOCK>
__device__ unsigned long long block_before(unsigned long long x, unsigned long long* total) {
  __shared__ unsigned long long sums[BLOCK / kWave];
  const unsigned long long incl = (unsigned long long)wave_incl_scan64((long long)x);
  const int wave = (int)threadIdx.x / kWave;
  __syncthreads();
  if (lane_id() == kWave - 1) sums[wave] = incl;
  __syncthreads();
  unsigned long long before = incl - x, all = 0;
#pragma unroll
  for (int w = 0; w < BLOCK / kWave; ++w) {
    if (w < wave) before += sums[w];
    all += sums[w];
  }
  *total = all;
  return before;
}

// Sums of the tiles before `tile`, workgroup-wide
template <int BLOCK, class T>
__device__ unsigned long long tiles_before(const T* tiles, int tile) {
  unsigned long long sum = 0, total;
  for (int t = (int)threadIdx.x; t < tile; t += BLOCK) sum += tiles[t];
  (void)block_before<BLOCK>(sum, &total);
  return total;
}

// Hits are marked, misses claim their node; and the counts of the digits to come are cleared
__global__ __launch_bounds__(kAdmitBlock) void k_admit_lookup(const Admit a) {
  const long long n = batch_size(a), i = blockIdx.x * (long long)kAdmitBlock + threadIdx.x;
  for (long long k = i; k < kDigits * kBins / 4; k += (long long)gridDim.x * kAdmitBlock) reinterpret_cast<uint4*>(a.hist)[k] = make_uint4(0, 0, 0, 0);
  if (i >= n) return;
  const long long v = a.nodes[i];
  if (v < 0 || v >= a.num_nodes) return;
  const int s = a.remap[v];  // a claim that has just been made may or may not show: either way it is no slot
  if (s >= 0 && (unsigned)s < a.n_slots) a.weight[s] |= kHit;  // (whoever else has the node writes the same)
  else atomicMin(a.remap + v, kClaim + (int)i);
}

// Workgroup-wide: the bin of a digit's counts in which the need-th slot lies.  before: the border after the digit before, nullptr for the first.
template <int BLOCK>
__device__ Border find_border(const unsigned* hist, unsigned need, const Border* before) {
  constexpr int kPer = kBins / BLOCK;
  __shared__ Border found;
  unsigned x[kPer], sum = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) sum += x[k] = hist[threadIdx.x * kPer + k];
  unsigned long long total;
  unsigned smaller = (unsigned)block_before<BLOCK>(sum, &total);
  if (need == 0) {  // nothing is wanted: no weight is below 0, and none of those that are 0 is needed
    if (threadIdx.x == 0) found = Border{0, 0, 0, 1};
  } else if (smaller < need && smaller + sum >= need) {  // one lane
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      if (smaller < need && smaller + x[k] >= need) {
        const unsigned bin = threadIdx.x * kPer + k;
        Border b;
        if (!before) {
          b.shift = bin >> kMantissa ? (int)(bin >> kMantissa) - 1 : 0;
          b.prefix = bin >> kMantissa ? (1u << kMantissa) + (bin & ((1u << kMantissa) - 1)) : bin;
        } else {
          b.shift = max(0, before->shift - kDigit);
          b.prefix = (before->prefix << (before->shift - b.shift)) + bin;
        }
        b.need = need - smaller;
        b.done = b.shift == 0 || b.need == x[k];
        found = b;
        break;
      }
      smaller += x[k];
    }
  }
  __syncthreads();
  const Border b = found;
  __syncthreads();
  return b;
}

// Counts of one digit over slots s0, s0 + step, ... into LDS, `kDigitSlots` at a time; returns the slots hit that it met
template <bool FIRST>
__device__ unsigned count_digit(const Admit& a, unsigned* bins, unsigned long long s0, unsigned long long step, unsigned long long prefix, int shift) {
  const int low = max(0, shift - kDigit);
  const unsigned mask = (1u << (shift - low)) - 1;
  unsigned hits = 0;
  for (unsigned long long s = s0; s < a.n_slots; s += step * kDigitSlots) {
    unsigned long long w[kDigitSlots];
    bool real[kDigitSlots];
#pragma unroll
    for (int k = 0; k < kDigitSlots; ++k) {
      const unsigned long long at = s + k * step;
      real[k] = at < a.n_slots;
      w[k] = real[k] ? a.weight[at] : 0;
    }
#pragma unroll
    for (int k = 0; k < kDigitSlots; ++k) {
      if (w[k] & kHit) ++hits;
      else if (real[k]) {
        if (FIRST) atomicAdd(&bins[first_digit(w[k])], 1u);
        else if (w[k] >> shift == prefix) atomicAdd(&bins[(unsigned)(w[k] >> low) & mask], 1u);
      }
    }
  }
  return hits;
}

// The first digit of every slot's weight; workgroups beside mark the misses
__global__ __launch_bounds__(kDigitBlock) void k_admit_first_digit(const Admit a) {
  __shared__ unsigned bins[kBins];
  unsigned long long total;
  if ((int)blockIdx.x < a.hist_blocks) {
    for (int b = (int)threadIdx.x; b < kBins; b += kDigitBlock) bins[b] = 0;
    __syncthreads();
    const unsigned hits = count_digit<true>(a, bins, blockIdx.x * (unsigned long long)kDigitBlock + threadIdx.x, (unsigned long long)a.hist_blocks * kDigitBlock, 0, 0);
    (void)block_before<kDigitBlock>(hits, &total);
    if (threadIdx.x == 0) a.hit_part[blockIdx.x] = (unsigned)total;
    for (int b = (int)threadIdx.x; b < kBins; b += kDigitBlock)
      if (bins[b]) atomicAdd(a.hist + b, bins[b]);
    return;
  }
  const int tile = (int)blockIdx.x - a.hist_blocks;
  const long long n = batch_size(a);
  unsigned misses = 0;
  for (int k = 0; k < a.node_tile_blocks; ++k) {
    const long long i = ((long long)tile * a.node_tile_blocks + k) * kDigitBlock + threadIdx.x;
    bool miss = false;  // the first place of a node without a slot
    if (i < n) {
      const long long v = a.nodes[i];
      miss = v >= 0 && v < a.num_nodes && a.remap[v] == kClaim + (int)i;
    }
    const unsigned long long mask = __ballot(miss);
    if (lane_id() == 0) a.node_mask[i >> 6] = mask;
    misses += miss ? 1 : 0;
  }
  (void)block_before<kDigitBlock>(misses, &total);
  if (threadIdx.x == 0) a.node_tile[tile] = (unsigned)total;
}

// The border after digit 0, as all workgroups of a kernel find it; the first one notes it, and the batch's figures
__device__ Border first_border(const Admit& a) {
  const unsigned misses = (unsigned)tiles_before<kDigitBlock>(a.node_tile, a.node_tiles);
  const unsigned hits = (unsigned)tiles_before<kDigitBlock>(a.hit_part, a.hist_blocks);
  const unsigned want = min(misses, a.n_slots - hits);
  const Border b = find_border<kDigitBlock>(a.hist, want, nullptr);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.st->misses = misses;
    a.st->hits = hits;
    a.st->want = want;
    a.st->border[0] = b;
  }
  return b;
}

// Digit 1 or 2 of the slots at the border
__global__ __launch_bounds__(kDigitBlock) void k_admit_digit(const Admit a, int digit) {
  __shared__ unsigned bins[kBins];
  Border b;
  if (digit == 1) {
    b = first_border(a);
  } else {
    b = a.st->border[0];
    if (!b.done) b = find_border<kDigitBlock>(a.hist + kBins, b.need, &a.st->border[0]);
    if (blockIdx.x == 0 && threadIdx.x == 0) a.st->border[1] = b;
  }
  if (b.done) return;
  for (int k = (int)threadIdx.x; k < kBins; k += kDigitBlock) bins[k] = 0;
  __syncthreads();
  (void)count_digit<false>(a, bins, blockIdx.x * (unsigned long long)kDigitBlock + threadIdx.x, (unsigned long long)a.hist_blocks * kDigitBlock, b.prefix, b.shift);
  __syncthreads();
  for (int k = (int)threadIdx.x; k < kBins; k += kDigitBlock)
    if (bins[k]) atomicAdd(a.hist + digit * kBins + k, bins[k]);
}

// Workgroup-wide: the border after all digits
template <int BLOCK>
__device__ Border last_border(const Admit& a, unsigned* bins) {
  __shared__ Border last;
  Border b = a.st->border[1];
  if (!b.done) b = find_border<BLOCK>(a.hist + 2 * kBins, b.need, &a.st->border[1]);
  while (!b.done) {
    if (threadIdx.x == 0) last = b;
    for (int k = (int)threadIdx.x; k < kBins; k += BLOCK) bins[k] = 0;
    __syncthreads();
    (void)count_digit<false>(a, bins, threadIdx.x, BLOCK, b.prefix, b.shift);
    __syncthreads();
    b = find_border<BLOCK>(bins, b.need, &last);
  }
  return b;
}

__global__ __launch_bounds__(kDigitBlock) void k_admit_border(const Admit a) {
  __shared__ unsigned bins[kBins];
  const Border b = last_border<kDigitBlock>(a, bins);
  if (threadIdx.x == 0) a.st->border[2] = b;
}

// Marks the slots below and at the border, and writes the list of the misses that get a slot.  FIND: every workgroup looks for the border itself, which
// spares a launch (3 us); where digits are left over after all, each of them goes through all slots, so only for caches of up to kFindSlots, and
// the marks of hits stay until nobody looks for it any more (beyond, they are taken off here, in order: k_admit_slots takes twice as long with that).
constexpr int64_t kFindSlots = 1 << 18;
template <bool FIND>
__global__ __launch_bounds__(kAdmitBlock) void k_admit_number(const Admit a) {
  __shared__ unsigned bins[FIND ? kBins : 1];
  const unsigned want = a.st->want;
  if ((int)blockIdx.x < a.slot_tiles) {
    const Border b = FIND ? last_border<kAdmitBlock>(a, bins) : a.st->border[2];
    if (FIND && blockIdx.x == 0 && threadIdx.x == 0) a.st->border[2] = b;
    unsigned long long sum = 0, total;
    for (int stretch = 0; stretch < a.slot_tile_stretches; ++stretch) {
      const unsigned long long s0 = ((unsigned long long)blockIdx.x * a.slot_tile_stretches + stretch) * kStretch + threadIdx.x;
      unsigned long long p[kStretch / kAdmitBlock];
      bool open[kStretch / kAdmitBlock];
#pragma unroll
      for (int k = 0; k < kStretch / kAdmitBlock; ++k) {
        const unsigned long long s = s0 + k * kAdmitBlock;
        const unsigned long long w = s < a.n_slots ? a.weight[s] : 0;
        if (!FIND && (w & kHit)) a.weight[s] = w & ~kHit;
        open[k] = s < a.n_slots && want && !(w & kHit);
        p[k] = w >> b.shift;
      }
#pragma unroll
      for (int k = 0; k < kStretch / kAdmitBlock; ++k) {
        const unsigned long long below = __ballot(open[k] && p[k] < b.prefix), at = __ballot(open[k] && p[k] == b.prefix);
        if (lane_id() == 0) {
          const unsigned long long word = (s0 + k * kAdmitBlock) >> 6;
          a.slot_mask[2 * word] = below;
          a.slot_mask[2 * word + 1] = at;
          sum += ((unsigned long long)__popcll(below) << 32) + __popcll(at);
        }
      }
    }
    (void)block_before<kAdmitBlock>(sum, &total);
    if (threadIdx.x == 0) a.slot_tile[blockIdx.x] = total;
    return;
  }
  // places of the batch: as many as there are in a tile's workgroup
  const long long at = (long long)(blockIdx.x - a.slot_tiles) * kDigitBlock;
  const int tile = (int)(at / kDigitBlock / a.node_tile_blocks);
  unsigned long long before = tiles_before<kAdmitBlock>(a.node_tile, tile), total;
  {
    unsigned sum = 0;
    const long long w0 = (long long)tile * a.node_tile_blocks * (kDigitBlock / 64);
    for (long long w = w0 + threadIdx.x; w < at / 64; w += kAdmitBlock) sum += (unsigned)__popcll(a.node_mask[w]);
    (void)block_before<kAdmitBlock>(sum, &total);
    before += total;
  }
  for (int k = 0; k < kDigitBlock / kAdmitBlock; ++k) {
    const long long i = at + k * kAdmitBlock + threadIdx.x;
    if (i < a.n_max && i >= want) a.fresh[i] = a.fresh_slots[i] = -1;
    const unsigned long long mask = a.node_mask[i >> 6];
    const bool miss = (mask >> (i & 63)) & 1;
    unsigned long long j = before + __popcll(mask & ((1ull << (i & 63)) - 1));
    for (long long w = at / 64; w < i >> 6; ++w) j += __popcll(a.node_mask[w]);
    if (miss && j < want) a.fresh[j] = (int)i;
  }
}

// The j-th slot to the j-th miss
__global__ __launch_bounds__(kAdmitBlock) void k_admit_give(const Admit a) {
  const unsigned want = a.st->want, need = a.st->border[2].need;
  __shared__ unsigned long long words[kStretchWords][2], firsts[kStretchWords];  // masks; (below, at) before them
  unsigned long long carry = tiles_before<kAdmitBlock>(a.slot_tile, (int)blockIdx.x), total;
  unsigned lost = 0;
  for (int stretch = 0; stretch < a.slot_tile_stretches && want; ++stretch) {
    const unsigned long long s0 = ((unsigned long long)blockIdx.x * a.slot_tile_stretches + stretch) * kStretch;
    unsigned long long x = 0;
    const int w = (int)threadIdx.x;
    if (w < kStretchWords) {
      words[w][0] = a.slot_mask[2 * (s0 / 64 + w)];
      words[w][1] = a.slot_mask[2 * (s0 / 64 + w) + 1];
      x = ((unsigned long long)__popcll(words[w][0]) << 32) + __popcll(words[w][1]);
    }
    const unsigned long long before = block_before<kAdmitBlock>(x, &total);
    if (w < kStretchWords) firsts[w] = carry + before;
    carry += total;
    __syncthreads();
#pragma unroll 4
    for (int k = 0; k < kStretch / kAdmitBlock; ++k) {
      const int in = k * kAdmitBlock + (int)threadIdx.x, v_w = in >> 6;
      const unsigned long long bit = 1ull << (in & 63);
      const unsigned below = (unsigned)(firsts[v_w] >> 32) + (unsigned)__popcll(words[v_w][0] & (bit - 1));
      const unsigned at = (unsigned)firsts[v_w] + (unsigned)__popcll(words[v_w][1] & (bit - 1));
      if ((words[v_w][0] & bit) || ((words[v_w][1] & bit) && at < need)) {
        const unsigned j = below + min(at, need);
        const int s = (int)(s0 + in);
        const long long v = a.nodes[a.fresh[j]], old = a.node[s];
        if (old >= 0 && old < a.num_nodes) {
          a.remap[old] = -1;
          ++lost;
        }
        a.node[s] = v;
        a.weight[s] = 1;
        a.remap[v] = s;
        a.fresh_slots[j] = s;
      }
    }
    __syncthreads();
  }
  (void)block_before<kAdmitBlock>(lost, &total);
  if (threadIdx.x == 0) a.gone_tile[blockIdx.x] = (unsigned)total;
}

// The slots of the batch; claims that got none are taken back, and marks of hits that are still there
template <bool UNMARK>
__global__ __launch_bounds__(kAdmitBlock) void k_admit_slots(const Admit a) {
  const long long n = batch_size(a), i = blockIdx.x * (long long)kAdmitBlock + threadIdx.x;
  if (blockIdx.x == 0) {
    const unsigned long long total = tiles_before<kAdmitBlock>(a.gone_tile, a.slot_tiles);
    if (threadIdx.x == 0) {
      a.counts[0] = a.st->want;
      a.counts[1] = a.st->misses;
      a.counts[2] = a.st->hits;
      a.counts[3] = (long long)total;
    }
  }
  if (i >= n) return;
  const long long v = a.nodes[i];
  int s = -1;
  if (v >= 0 && v < a.num_nodes) {
    s = a.remap[v];
    if (s == kClaim + (int)i) a.remap[v] = -1;
    if (s < 0 || (unsigned)s >= a.n_slots) s = -1;
    else if (UNMARK) a.weight[s] &= ~kHit;  // (whoever else has the node writes the same)
  }
  a.slots[i] = s;
}

struct AdmitSpace {
  AdmitState* st;
  unsigned *hist, *hit_part, *node_tile, *gone_tile;
  unsigned long long *node_mask, *slot_mask, *slot_tile;
  int node_tiles, node_tile_blocks, slot_tiles, slot_tile_stretches;
};
AdmitSpace admit_space(Arena& ar, int64_t n_slots, int64_t n_max) {
  AdmitSpace s;
  const int64_t blocks = (n_max + kDigitBlock - 1) / kDigitBlock, stretches = (n_slots + kStretch - 1) / kStretch;
  s.node_tile_blocks = (int)((blocks + kTiles - 1) / kTiles);
  s.node_tiles = blocks ? (int)((blocks + s.node_tile_blocks - 1) / s.node_tile_blocks) : 0;
  s.slot_tile_stretches = (int)((stretches + kTiles - 1) / kTiles);
  s.slot_tiles = (int)((stretches + s.slot_tile_stretches - 1) / s.slot_tile_stretches);
  s.hist = ar.take<unsigned>((size_t)kDigits * kBins);
  s.st = ar.take<AdmitState>(1);
  s.hit_part = ar.take<unsigned>(kHistBlocks);
  s.node_mask = ar.take<unsigned long long>((size_t)s.node_tiles * s.node_tile_blocks * (kDigitBlock / 64));
  s.node_tile = ar.take<unsigned>(kTiles);
  s.slot_mask = ar.take<unsigned long long>((size_t)s.slot_tiles * s.slot_tile_stretches * kStretchWords * 2);
  s.slot_tile = ar.take<unsigned long long>(kTiles);
  s.gone_tile = ar.take<unsigned>(kTiles);
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
  a.wide = cache->head_dim >= dci::kChunk || cache->head_dim * bytes % 16 == 0;
  a.odd = a.wide && cache->head_dim * bytes % 16 != 0;
  a.codes = cache->codes;
  a.scales = cache->scales;
  a.n_slots = cache->n_slots;
  a.block_log2 = dci::log2_up(cache->block);
  a.kv_heads = cache->kv_heads;
  a.dim = cache->head_dim;
  a.lh_log2 = dci::log2_up((cache->head_dim + dci::kChunk - 1) / dci::kChunk);
  a.host_flag = ctx->host_flag + 1;
  // Entries to a wavefront: a block's, as far as four times the rows that it has lanes for go, eight times where many blocks may be written whole (a
  // block that does not fit is read twice).  Heads of 128, blocks of 64, 16-bit rows: 200,000 of 200,000 slots 469 us with eight and 611 with four,
  // 20,000 of them 270 and 256.
  const int at_once = dci::kWave >> a.lh_log2, most = n_max >= cache->n_slots / 2 ? 8 : 4;
  int tiles = 1;
  while (tiles < most && tiles * at_once < cache->block) tiles *= 2;
  // A launch's lanes are counted in 32 bits, and one of more runs what is left of their number beyond: turns go to as many launches as that takes, each
  // a whole number of workgroups.
  const int64_t turns = (n_max + tiles * at_once - 1) / (tiles * at_once);
  const int64_t most_turns = (0xFFFFFFFFll / dci::kKvBlock) / cache->kv_heads * dci::kKvWaves;
  dci::Timed timed(ctx, DCI_K_KV);
  for (int64_t first = 0; first < turns; first += most_turns) {
    a.first_turn = (unsigned)first;
    const int64_t waves = (turns - first < most_turns ? turns - first : most_turns) * cache->kv_heads;
    const unsigned grid = (unsigned)((waves + dci::kKvWaves - 1) / dci::kKvWaves);
    if (dtype == DCI_F32) dci::launch_write<DCI_F32>(tiles, a, grid, ctx->stream);
    else if (dtype == DCI_BF16) dci::launch_write<DCI_BF16>(tiles, a, grid, ctx->stream);
    else dci::launch_write<DCI_F16>(tiles, a, grid, ctx->stream);
    DCI_LAUNCH_CHECK(ctx);
  }
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
  const bool wide = cache->head_dim * bytes >= 16;
  a.codes = cache->codes;
  a.scales = cache->scales;
  a.n_slots = cache->n_slots;
  a.block_log2 = dci::log2_up(cache->block);
  a.kv_heads = cache->kv_heads;
  a.dim = cache->head_dim;
  const int64_t pieces = 2ll * cache->kv_heads * (wide ? (cache->head_dim * bytes + 15) / 16 : cache->head_dim);
  a.lanes_log2 = dci::log2_up(pieces);
  if (a.lanes_log2 > 8) a.lanes_log2 = 8;  // a workgroup
  // An output of more than the last-level cache holds (256 MB) is not there when it is read next, and only drives out what is.  Past it 184,000 rows of
  // 2 KB take 74 us for 98; half a million 268 for 254, but the write of their rows 149 for 181.  Below, 10,000 rows and attention over them take 43 for 41.
  const bool past = n_max * pieces * 16 > 256ll << 20;
  const int64_t rows = dci::kKvBlock >> a.lanes_log2;
  int64_t grid = (n_max + rows * 4 - 1) / (rows * 4);
  if (grid > (int64_t)ctx->num_cus * 32) grid = (int64_t)ctx->num_cus * 32;
  dci::Timed timed(ctx, DCI_K_KV);
  if (dtype == DCI_F32) dci::launch_read<DCI_F32>(wide, past, a, (unsigned)grid, ctx->stream);
  else if (dtype == DCI_BF16) dci::launch_read<DCI_BF16>(wide, past, a, (unsigned)grid, ctx->stream);
  else dci::launch_read<DCI_F16>(wide, past, a, (unsigned)grid, ctx->stream);
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
  a.hist = sp.hist;
  a.hit_part = sp.hit_part;
  a.node_mask = sp.node_mask;
  a.node_tile = sp.node_tile;
  a.slot_mask = sp.slot_mask;
  a.slot_tile = sp.slot_tile;
  a.gone_tile = sp.gone_tile;
  a.node_tiles = sp.node_tiles;
  a.node_tile_blocks = sp.node_tile_blocks;
  a.slot_tiles = sp.slot_tiles;
  a.slot_tile_stretches = sp.slot_tile_stretches;
  const int64_t per_block = dci::kDigitBlock * dci::kDigitSlots;
  a.hist_blocks = (int)((cache->n_slots + per_block - 1) / per_block);
  if (a.hist_blocks > dci::kHistBlocks) a.hist_blocks = dci::kHistBlocks;
  const unsigned node_blocks = (unsigned)(n_max > 0 ? (n_max + dci::kAdmitBlock - 1) / dci::kAdmitBlock : 1);
  dci::Timed timed(ctx, DCI_K_KV);
#define DCI_ADMIT(kernel_, grid_, block_, ...)                                                                               \
  do {                                                                                                                       \
    hipLaunchKernelGGL(kernel_, dim3((unsigned)(grid_)), dim3(block_), 0, ctx->stream, ##__VA_ARGS__);                       \
    DCI_LAUNCH_CHECK(ctx);                                                                                                   \
  } while (0)
  DCI_ADMIT(dci::k_admit_lookup, node_blocks < 24 ? 24 : node_blocks, dci::kAdmitBlock, a);
  DCI_ADMIT(dci::k_admit_first_digit, a.hist_blocks + a.node_tiles, dci::kDigitBlock, a);
  DCI_ADMIT(dci::k_admit_digit, a.hist_blocks, dci::kDigitBlock, a, 1);
  DCI_ADMIT(dci::k_admit_digit, a.hist_blocks, dci::kDigitBlock, a, 2);
  const int64_t number_blocks = a.slot_tiles + (n_max + dci::kDigitBlock - 1) / dci::kDigitBlock;
  if (cache->n_slots <= dci::kFindSlots) {
    DCI_ADMIT(dci::k_admit_number<true>, number_blocks, dci::kAdmitBlock, a);
  } else {
    DCI_ADMIT(dci::k_admit_border, 1, dci::kDigitBlock, a);
    DCI_ADMIT(dci::k_admit_number<false>, number_blocks, dci::kAdmitBlock, a);
  }
  DCI_ADMIT(dci::k_admit_give, a.slot_tiles, dci::kAdmitBlock, a);
  if (cache->n_slots <= dci::kFindSlots) DCI_ADMIT(dci::k_admit_slots<true>, node_blocks, dci::kAdmitBlock, a);
  else DCI_ADMIT(dci::k_admit_slots<false>, node_blocks, dci::kAdmitBlock, a);
#undef DCI_ADMIT
  return DCI_OK;
}

}  // extern "C"
