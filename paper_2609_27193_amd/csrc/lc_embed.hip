// Rows of a table by token, scaled, and the table's gradient.
//
//   out[t] = scale * W[token[t] - first]            (zeros for a token outside the table)
//   dW[v] (+)= scale * sum over t with token[t] - first = v of dout[t]
//
// Both are bound by memory; of the gradient's, most is the table itself, which
// is written whole.  The gradient sorts the tokens by row and position and sums
// a row's in fp32, in runs whose bounds and order go by the sizes and the sorted
// tokens alone: the result does not depend on how blocks are scheduled.
#include "lc_ops_device.h"

namespace lc {
namespace {

// Row of the table for token i, or `vocab` for a token outside it.
__device__ __forceinline__ uint32_t token_row(uint64_t tokens, int token64, uint64_t i, int64_t first, uint64_t vocab) {
  typedef const __attribute__((address_space(1))) int64_t gc_i64;
  typedef const __attribute__((address_space(1))) int32_t gc_i32;
  const int64_t t = token64 ? *(gc_i64*)(tokens + 8 * i) : *(gc_i32*)(tokens + 4 * i);
  const uint64_t r = static_cast<uint64_t>(t) - static_cast<uint64_t>(first);  // wraps below `first`: beyond the table
  return t >= first && r < vocab ? static_cast<uint32_t>(r) : static_cast<uint32_t>(vocab);
}

constexpr uint32_t kEmbedThreads = 256;
constexpr int kEmbedVecs = 4;  // groups of eight that a thread has in flight

// `lanes` threads (a power of two) take one token's row, 8 elements each at a
// time.  Bound by memory, 16384 rows of 4096 out of 128256 in bf16: 32.4 us, 8 TB/s
// with the rows that come again out of the caches; the output goes past them
// (through them 34.7 us).
template <int WDT, int ODT>
__global__ __launch_bounds__(kEmbedThreads) void embed_fwd_kernel(EmbedFwd a, uint32_t lanes_log2) {
  const uint32_t lanes = 1u << lanes_log2, per_block = kEmbedThreads >> lanes_log2;
  const uint32_t groups = (a.dim + 7) / 8, lane = threadIdx.x & (lanes - 1);
  const uint64_t items = (a.n + per_block - 1) / per_block;
  for (uint64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const uint64_t t = it * per_block + (threadIdx.x >> lanes_log2);
    if (t >= a.n) continue;
    const uint32_t row = token_row(a.tokens, a.token64, t, a.first, a.vocab);
    const bool held = row < a.vocab;
    const uint64_t src = a.w.data + static_cast<uint64_t>(row) * a.w.stride * kEsz<WDT>;
    const uint64_t dst = a.out.data + t * a.out.stride * kEsz<ODT>;
    for (uint32_t g0 = lane; g0 < groups; g0 += lanes * kEmbedVecs) {
      Raw8<WDT> r[kEmbedVecs];
#pragma unroll
      for (int i = 0; i < kEmbedVecs; ++i) {
        const uint32_t g = g0 + i * lanes;
        for (auto& q : r[i].v) q = u32x4{0, 0, 0, 0};
        if (held && g < groups) r[i] = load8_raw<WDT>(src + 8ull * kEsz<WDT> * g, in_group(a.dim, g));
      }
#pragma unroll
      for (int i = 0; i < kEmbedVecs; ++i) {
        const uint32_t g = g0 + i * lanes;
        if (g >= groups) break;
        float f[8];
        unpack8<WDT>(r[i], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = held ? f[e] * a.scale : 0.0f;
        store8<ODT, kStreams<ODT>>(dst + 8ull * kEsz<ODT> * g, f, in_group(a.dim, g));
      }
    }
  }
}

// ---- clearing the table -------------------------------------------------------------
// A block clears `per` rows, about 256 KB and 64 of them at most, or those of
// them that are not in `skip`; a wave's rows follow each other (16384 tokens into
// 128256 x 2048 bf16, whole: 112 us, the waves' rows in turn 116).
struct Fill {
  uint64_t data, pitch, first, rows;  // of the table: its first row, bytes a row; rows first to rows - 1
  uint64_t end;                       // no byte from here on is written
  uint64_t bytes;                     // of a row that count, even: up to 2^32
  uint32_t per;
};
__host__ inline uint64_t fill_blocks(const Fill& f) { return (f.rows - f.first + f.per - 1) / f.per; }
__device__ __forceinline__ void fill_rows(const Fill& f, uint64_t block, uint64_t skip) {
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x / 64;
  const uint64_t r0 = f.first + block * f.per;
  const uint32_t run = (f.per + waves - 1) / waves;
  for (uint32_t i = wave * run; i < (wave + 1) * run && i < f.per && r0 + i < f.rows; ++i) {
    if (skip >> i & 1) continue;
    const uint64_t p = f.data + (r0 + i) * f.pitch;
    const uint64_t bytes = f.end - p < f.bytes ? f.end - p : f.bytes;
    for (uint64_t at = lane * 16; at + 16 <= bytes; at += 64 * 16) st_any(reinterpret_cast<uint8_t*>(p + at), u32x4{0, 0, 0, 0});
    const uint64_t tail = bytes & ~15ull;
    if (tail + lane * 2 < bytes) *(g_u16*)(p + tail + lane * 2) = 0;
  }
}

// ---- sorting the tokens ------------------------------------------------------------
// Few tokens need no order (embed_direct_kernel, below).  Up to kRankTokens one
// launch counts, for every token, the tokens that come before it (a smaller row,
// or the same row at an earlier position); beyond that one block sorts, or, many,
// a radix sort of kDigitBits a pass, two launches a pass.  All are bound by
// latency: 4096 tokens, counted, about 8 us; a pass of 16384 tokens 2.5 to 4.7 and
// 4.5 to 5.3 us for its two launches.  Their few blocks leave the chip to others,
// which clear the table meanwhile, rows with a token and without: writing the
// former twice costs less than the sort's time alone (16384 tokens into 128256 x
// 2048 bf16, sorted by passes: 117 us, and 152 where the sums' launch cleared the
// rows without a token; one block sorts these now, 112).
constexpr uint32_t kRankTokens = 4096;
constexpr uint32_t kRankThreads = 256;
constexpr uint32_t kRankOwn = 8;  // tokens of a block; its 32 slices of threads share the others
constexpr uint32_t kDigitBits = 9, kDigits = 1u << kDigitBits;
constexpr uint32_t kSortThreads = 512;
constexpr uint32_t kSortWaves = kSortThreads / 64;
static_assert(kSortThreads == kDigits, "one thread a digit");

__global__ __launch_bounds__(kRankThreads) void embed_rank_kernel(EmbedBwd a, Fill fill, uint32_t fill_from,
                                                                  uint32_t* keys, uint32_t* pos) {
  __shared__ __align__(16) uint32_t all[kRankTokens];
  __shared__ uint32_t count[kRankThreads / kRankOwn][kRankOwn];
  if (blockIdx.x >= fill_from) {
    for (uint64_t b = blockIdx.x - fill_from; fill.first + b * fill.per < fill.rows; b += gridDim.x - fill_from)
      fill_rows(fill, b, 0);
    return;
  }
  const uint32_t n = static_cast<uint32_t>(a.n);
  const uint32_t padded = (n + kRankOwn - 1) / kRankOwn * kRankOwn;
  for (uint32_t i = threadIdx.x; i < padded; i += kRankThreads)
    all[i] = i < n ? token_row(a.tokens, a.token64, i, a.first, a.vocab) : 0xFFFFFFFFu;
  __syncthreads();
  const uint32_t own = threadIdx.x % kRankOwn, slice = threadIdx.x / kRankOwn;
  for (uint32_t base = blockIdx.x * kRankOwn; base < n; base += fill_from * kRankOwn) {
    const uint32_t i = base + own, key = all[i];
    uint32_t before = 0;
    // groups of kRankOwn tokens, dealt out to the slices
    for (uint32_t g = slice * kRankOwn; g < padded; g += kRankThreads) {
      if (g == base) {
        for (uint32_t j = 0; j < kRankOwn; ++j) {
          const uint32_t k = all[g + j];
          before += k < key || (k == key && j < own);
        }
      } else {
        // an equal row counts where it stands before: k < key + 1 there.  key
        // is at most 2^31 for a token; the padding's own rank is not used.
        const uint32_t limit = g < base ? key + 1 : key;
#pragma unroll
        for (uint32_t j = 0; j < kRankOwn; j += 4) {
          const u32x4 k = *reinterpret_cast<const u32x4*>(&all[g + j]);
          before += (k[0] < limit) + (k[1] < limit) + (k[2] < limit) + (k[3] < limit);
        }
      }
    }
    count[slice][own] = before;
    __syncthreads();
    if (slice == 0 && i < n) {
      uint32_t r = 0;
#pragma unroll
      for (uint32_t s = 0; s < kRankThreads / kRankOwn; ++s) r += count[s][own];
      keys[r] = key;
      pos[r] = i;
    }
    __syncthreads();
  }
}

// The tile of a radix pass: a multiple of kSortThreads that leaves at most
// kSortTiles of them, for every tile reads the counts of all.
constexpr uint32_t kSortTiles = 64;
__host__ __device__ inline uint32_t sort_tile(uint64_t n) {
  const uint64_t per = (n + kSortTiles - 1) / kSortTiles;
  return static_cast<uint32_t>((per + kSortThreads - 1) / kSortThreads * kSortThreads);
}

// Lanes of the wave that are `on` and have this lane's digit.
__device__ __forceinline__ uint64_t lanes_of_digit(bool on, uint32_t digit, uint32_t bits) {
  const uint64_t all = __ballot(on);
  uint32_t lo = static_cast<uint32_t>(all), hi = static_cast<uint32_t>(all >> 32);
#pragma unroll
  for (uint32_t bit = 0; bit < kDigitBits; ++bit) {
    if (bit >= bits) break;  // the same for the whole grid
    const uint32_t zero = (digit >> bit & 1) - 1;  // all ones where the bit is not set
    const uint64_t ones = __ballot(zero == 0);
    lo &= static_cast<uint32_t>(ones) ^ zero;
    hi &= static_cast<uint32_t>(ones >> 32) ^ zero;
  }
  return static_cast<uint64_t>(hi) << 32 | lo;
}

// keys null: the tokens themselves, at position i.
__device__ __forceinline__ uint32_t sort_key(const EmbedBwd& a, const uint32_t* keys, uint64_t i) {
  return keys ? keys[i] : token_row(a.tokens, a.token64, i, a.first, a.vocab);
}

__global__ __launch_bounds__(kSortThreads) void embed_count_kernel(EmbedBwd a, Fill fill, uint32_t fill_from,
                                                                   const uint32_t* keys, uint32_t shift, uint32_t tile,
                                                                   uint32_t* hist) {
  __shared__ uint32_t bins[kDigits];
  if (blockIdx.x >= fill_from) {
    for (uint64_t b = blockIdx.x - fill_from; fill.first + b * fill.per < fill.rows; b += gridDim.x - fill_from)
      fill_rows(fill, b, 0);
    return;
  }
  const uint64_t tiles = (a.n + tile - 1) / tile;
  for (uint64_t b = blockIdx.x; b < tiles; b += fill_from) {
    bins[threadIdx.x] = 0;
    __syncthreads();
    const uint64_t end = b * tile + tile < a.n ? b * tile + tile : a.n;
    for (uint64_t i = b * tile + threadIdx.x; i < end; i += kSortThreads)
      atomicAdd(&bins[(sort_key(a, keys, i) >> shift) % kDigits], 1u);  // whole numbers: any order gives the same
    __syncthreads();
    hist[b * kDigits + threadIdx.x] = bins[threadIdx.x];
    __syncthreads();
  }
}

__global__ __launch_bounds__(kSortThreads) void embed_scatter_kernel(EmbedBwd a, Fill fill, uint32_t fill_from,
                                                                     const uint32_t* keys, const uint32_t* pos,
                                                                     uint32_t shift, uint32_t tile, const uint32_t* hist,
                                                                     uint32_t* keys_out, uint32_t* pos_out) {
  __shared__ uint32_t next[kDigits];              // where a digit's next key goes
  __shared__ uint32_t wave_count[kSortWaves][kDigits];
  __shared__ uint32_t wave_total[kSortWaves];
  const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (blockIdx.x >= fill_from) {
    for (uint64_t b = blockIdx.x - fill_from; fill.first + b * fill.per < fill.rows; b += gridDim.x - fill_from)
      fill_rows(fill, b, 0);
    return;
  }
  const uint32_t tiles = static_cast<uint32_t>((a.n + tile - 1) / tile);
  for (uint64_t b = blockIdx.x; b < tiles; b += fill_from) {
    uint32_t total = 0, before = 0;
#pragma unroll 16
    for (uint32_t j = 0; j < tiles; ++j) {
      const uint32_t h = hist[j * kDigits + tid];
      total += h;
      before += j < b ? h : 0;
    }
    // exclusive sum of `total` over the digits
    uint32_t scan = total;
#pragma unroll
    for (uint32_t d = 1; d < 64; d <<= 1) {
      const uint32_t o = __shfl_up(scan, d, 64);
      if (lane >= d) scan += o;
    }
    if (lane == 63) wave_total[wave] = scan;
    __syncthreads();
    uint32_t base = scan - total;
    for (uint32_t w = 0; w < wave; ++w) base += wave_total[w];
    next[tid] = base + before;
#pragma unroll
    for (uint32_t w = 0; w < kSortWaves; ++w) wave_count[w][tid] = 0;
    __syncthreads();
    for (uint32_t r = 0; r < tile; r += kSortThreads) {
      const uint64_t i = b * tile + r + tid;
      const bool on = i < a.n;
      const uint32_t key = on ? sort_key(a, keys, i) : 0;
      const uint32_t digit = (key >> shift) % kDigits;
      const uint64_t same = lanes_of_digit(on, digit, kDigitBits);
      const uint32_t rank = __popcll(same & ((1ull << lane) - 1));
      if (on && rank == 0) wave_count[wave][digit] = __popcll(same);
      __syncthreads();
      uint32_t at = next[tid];
#pragma unroll
      for (uint32_t w = 0; w < kSortWaves; ++w) {  // thread tid owns digit tid
        const uint32_t c = wave_count[w][tid];
        wave_count[w][tid] = at;
        at += c;
      }
      next[tid] = at;
      __syncthreads();
      if (on) {
        const uint32_t to = wave_count[wave][digit] + rank;
        keys_out[to] = key;
        pos_out[to] = pos ? pos[i] : static_cast<uint32_t>(i);
      }
      __syncthreads();
#pragma unroll
      for (uint32_t w = 0; w < kSortWaves; ++w) wave_count[w][tid] = 0;
      __syncthreads();
    }
  }
}

// ---- sorting in one block -------------------------------------------------------------
// One block sorts alone, in one launch, while the others clear the table: KPT
// tokens a thread, up to kDigitBits a pass, exchanged through LDS.  A wave has
// 64 * KPT tokens that follow each other; a token's place within its wave's
// tokens of a digit comes from ballots and the wave's own counts, so that a pass
// keeps the order of what is equal.  Bound by that one CU's vector ALU: 13.7 us
// for 6000 tokens of 2000 rows, 28 for 16384 of 50257, where the passes over all
// blocks take 24 and 24.  So it sorts up to 8192 tokens (6000 into 2000 x 300
// fp32, whole, 29 us, by passes 38.6), and twice that where the table takes as long
// to clear (16384 into 32000 x 4096 bf16 83 us for 89, into 50257 x 1024, 103 MB,
// 46.5 for 43).
constexpr uint32_t kBlockThreads = 1024, kBlockWaves = kBlockThreads / 64;
constexpr uint32_t kBlockTokens = 8 * kBlockThreads;
constexpr uint64_t kBlockClears = 128ull << 20;  // bytes
bool sorts_in_block(uint64_t n, uint64_t table_bytes) {
  return n <= kBlockTokens || (n <= 2 * kBlockTokens && table_bytes >= kBlockClears);
}
template <uint32_t KPT>
__global__ __launch_bounds__(kBlockThreads) void embed_block_sort_kernel(EmbedBwd a, Fill fill, uint32_t passes, uint32_t bits,
                                                                         uint32_t* keys, uint32_t* pos) {
  __shared__ uint32_t key_lds[KPT * kBlockThreads];
  __shared__ uint16_t pos_lds[KPT * kBlockThreads];
  __shared__ uint16_t count[kBlockWaves][kDigits];  // a wave's tokens of a digit, then where the first of them goes
  __shared__ uint32_t wave_total[kDigits / 64];
  static_assert(2 * kBlockTokens <= 1u << 16, "positions and places in 16 bits");
  if (blockIdx.x > 0) {
    for (uint64_t b = blockIdx.x - 1; fill.first + b * fill.per < fill.rows; b += gridDim.x - 1) fill_rows(fill, b, 0);
    return;
  }
  const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = static_cast<uint32_t>(a.n);
  const uint32_t at0 = wave * 64 * KPT + lane;
  volatile uint16_t* const mine = count[wave];  // other lanes' writes are seen
  uint32_t key[KPT], from[KPT], place[KPT];
#pragma unroll
  for (uint32_t r = 0; r < KPT; ++r) {
    const uint32_t i = at0 + 64 * r;
    from[r] = i;
    key[r] = token_row(a.tokens, a.token64, i < n ? i : n - 1, a.first, a.vocab);
  }
  for (uint32_t pass = 0; pass < passes; ++pass) {
    const uint32_t shift = pass * bits, digits = 1u << bits;
    for (uint32_t d = lane; d < digits; d += 64) mine[d] = 0;
#pragma unroll
    for (uint32_t r = 0; r < KPT; ++r) {
      const bool on = at0 + 64 * r < n;
      const uint32_t digit = key[r] >> shift & (digits - 1);
      const uint64_t same = lanes_of_digit(on, digit, bits);
      const uint32_t before = __popcll(same & ((1ull << lane) - 1));
      const uint32_t had = mine[digit];
      __builtin_amdgcn_wave_barrier();
      if (on && before == 0) mine[digit] = static_cast<uint16_t>(had + __popcll(same));
      __builtin_amdgcn_wave_barrier();
      place[r] = had + before;
    }
    __syncthreads();
    uint32_t total = 0, scan = 0;
    if (tid < kDigits) {  // whole waves: a thread a digit; behind the last one, counts that no one reads
#pragma unroll
      for (uint32_t w = 0; w < kBlockWaves; ++w) {
        const uint32_t c = count[w][tid];
        count[w][tid] = static_cast<uint16_t>(total);
        total += c;
      }
      scan = total;
#pragma unroll
      for (uint32_t d = 1; d < 64; d <<= 1) {
        const uint32_t o = __shfl_up(scan, d, 64);
        if (lane >= d) scan += o;
      }
      if (lane == 63) wave_total[wave] = scan;
    }
    __syncthreads();
    if (tid < kDigits) {
      uint32_t base = scan - total;
      for (uint32_t w = 0; w < wave; ++w) base += wave_total[w];
#pragma unroll
      for (uint32_t w = 0; w < kBlockWaves; ++w) count[w][tid] = static_cast<uint16_t>(count[w][tid] + base);
    }
    __syncthreads();
#pragma unroll
    for (uint32_t r = 0; r < KPT; ++r) {
      if (at0 + 64 * r >= n) continue;
      const uint32_t to = count[wave][key[r] >> shift & (digits - 1)] + place[r];
      key_lds[to] = key[r];
      pos_lds[to] = static_cast<uint16_t>(from[r]);
    }
    __syncthreads();
#pragma unroll
    for (uint32_t r = 0; r < KPT; ++r) {  // behind the last token: whatever lies there, and is not used
      key[r] = key_lds[at0 + 64 * r];
      from[r] = pos_lds[at0 + 64 * r];
    }
    // the next pass's counts are written before its own barriers, and so are its keys after them
  }
#pragma unroll
  for (uint32_t r = 0; r < KPT; ++r) {
    const uint32_t i = at0 + 64 * r;
    if (i < n) {
      keys[i] = key[r];
      pos[i] = from[r];
    }
  }
}

// ---- sums of the sorted tokens ---------------------------------------------------------
// A wave takes `run` sorted positions and 512 columns.  A row whose tokens all
// lie in the tile is written at once; one that crosses into the next tile
// leaves fp32 partial sums: [tile][0] of the row that came in from the tile
// before, [tile][1] of one that begins here and goes on.  The join kernel adds
// those in the order of the tiles.  So a token that fills the batch is spread
// over the chip like any others.
constexpr uint32_t kSumThreads = 256;
constexpr uint32_t kSumCols = 512;

// Sorted positions of a tile: more leave fewer parts to join, fewer leave more
// waves; 16 at least, and beyond that some 512 tiles, or 2048 waves of few columns
// (131072 tokens into 32000 x 2048, all of one row: 2048 tiles 223 us, 512 153, as
// often as words 191 and 183; 16384 into 128256 x 2048 113 and 112).
__host__ inline uint32_t sum_run(uint64_t n, uint64_t chunks) {
  const uint64_t tiles = chunks < 4 ? 2048 / chunks : 512;
  uint64_t r = 16;
  while (r * tiles < n) r *= 2;
  return static_cast<uint32_t>(r);
}

// The eight columns that a lane sums.  Every load of a group of rows goes out
// without a condition, or the compiler waits for each: a lane without columns
// reads the row's last eight, and so does the lane of a row's last, smaller
// group, which moves its sums down at the end (WHOLE: rows of at least eight
// columns).
struct Cols {
  uint32_t g, at;  // the group of eight, and the first column that is read
  int in;          // columns of the group
};
__device__ __forceinline__ Cols sum_cols(uint32_t dim, uint32_t chunk) {
  const uint32_t g = chunk * (kSumCols / 8) + (threadIdx.x & 63);
  return Cols{g, dim >= 8 && 8 * g > dim - 8 ? dim - 8 : 8 * g, in_group(dim, g)};
}
template <int DT, bool WHOLE>
__device__ __forceinline__ Raw8<DT> load_cols(uint64_t row, const Cols& c) {
  if constexpr (WHOLE) return load8_raw<DT>(row + c.at * static_cast<uint64_t>(kEsz<DT>));
  else return load8_raw<DT>(row, c.in);
}
__device__ __forceinline__ void move_down(const Cols& c, float (&f)[8]) {
  const uint32_t s = 8 * c.g - c.at;
  if (c.in <= 0 || s == 0) return;
#pragma unroll
  for (int b = 4; b; b >>= 1)
    if (s & b)
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = e + b < 8 ? f[e + b] : 0.0f;
}

struct SumArgs {
  Rows dout, dw;
  const uint32_t* keys;
  const uint32_t* pos;
  float* part;       // [tiles][2][dim]
  uint64_t n, vocab;
  uint32_t dim, run, tiles, chunks;
  float scale;
  int accumulate;
};

__device__ __forceinline__ float* sum_part(const SumArgs& a, uint64_t tile, int which) {
  return a.part + (tile * 2 + which) * static_cast<uint64_t>(a.dim);
}

template <int GDT>
__device__ __forceinline__ void sum_write(const SumArgs& a, uint32_t row, uint32_t g, const float (&acc)[8], int n) {
  const uint64_t p = a.dw.data + (static_cast<uint64_t>(row) * a.dw.stride + 8ull * g) * kEsz<GDT>;
  float f[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = acc[e] * a.scale;
  if (a.accumulate) {
    float old[8];
    unpack8<GDT>(load8_raw<GDT>(p, n), old);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] += old[e];
  }
  store8<GDT>(p, f, n);
}

__device__ __forceinline__ void part_write(float* p, uint32_t g, const float (&acc)[8], int n) {
  store8<kF32>(reinterpret_cast<uint64_t>(p) + 32ull * g, acc, n);
}

template <int DDT, int GDT, bool WHOLE>
__device__ void sum_tile(const SumArgs& a, uint64_t item) {
  constexpr int U = 8;  // rows in flight; with 16, 28 us for 18 of 16384 x 2048 bf16
  const uint32_t lane = threadIdx.x & 63;
  const uint32_t tile = static_cast<uint32_t>(item / a.chunks), chunk = static_cast<uint32_t>(item % a.chunks);
  const Cols cols = sum_cols(a.dim, chunk);
  const uint64_t b0 = static_cast<uint64_t>(tile) * a.run;
  const uint64_t b1 = b0 + a.run < a.n ? b0 + a.run : a.n;
  const uint32_t none = static_cast<uint32_t>(a.vocab);
  const uint32_t left = b0 ? a.keys[b0 - 1] : none;   // `none` sorts last and is never summed
  const uint32_t right = b1 < a.n ? a.keys[b1] : none;
  float acc[8] = {};
  uint32_t cur = none;
  bool open_left = false;
  auto flush = [&](bool open_right) {
    if (cur == none || cols.in <= 0) return;
    if constexpr (WHOLE) move_down(cols, acc);
    if (open_left) part_write(sum_part(a, tile, 0), cols.g, acc, cols.in);
    else if (open_right) part_write(sum_part(a, tile, 1), cols.g, acc, cols.in);
    else sum_write<GDT>(a, cur, cols.g, acc, cols.in);
  };
  for (uint64_t c0 = b0; c0 < b1; c0 += 64) {
    const uint32_t m = static_cast<uint32_t>(b1 - c0 < 64 ? b1 - c0 : 64);
    const uint32_t key = lane < m ? a.keys[c0 + lane] : none;
    const uint32_t at = lane < m ? a.pos[c0 + lane] : 0;
    for (uint32_t u0 = 0; u0 < m; u0 += U) {
      Raw8<DDT> r[U];
      uint32_t k[U];
      if (static_cast<uint32_t>(__builtin_amdgcn_readlane(key, u0)) == none) break;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        k[u] = __builtin_amdgcn_readlane(key, u0 + u);  // `none` behind the last token, at position 0
        const uint32_t p = __builtin_amdgcn_readlane(at, u0 + u);
        r[u] = load_cols<DDT, WHOLE>(a.dout.data + static_cast<uint64_t>(p) * a.dout.stride * kEsz<DDT>, cols);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (k[u] == none) continue;  // behind the last token, or outside the table
        if (k[u] != cur) {
          flush(false);
          open_left = c0 == b0 && u0 + u == 0 && k[u] == left;
          cur = k[u];
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
        }
        float f[8];
        unpack8<DDT>(r[u], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += f[e];
      }
    }
  }
  flush(cur == right);
}

// The first of the n sorted keys that is not below `key`: the wave looks at 64
// of them at once, evenly spread over what is left.
__device__ __forceinline__ uint64_t first_not_below(const uint32_t* keys, uint64_t n, uint64_t key) {
  const uint32_t lane = threadIdx.x & 63;
  uint64_t lo = 0, hi = n;  // keys before lo are below, keys from hi on are not
  while (lo < hi) {
    const uint64_t step = (hi - lo + 63) / 64, at = lo + lane * step;
    const uint64_t below = __ballot(at < hi && keys[at < hi ? at : lo] < key);
    const uint32_t c = __popcll(below);  // the samples are sorted: the first c are below
    const uint64_t next = lo + c * step;
    lo = c ? lo + (c - 1) * step + 1 : lo;
    hi = next < hi ? next : hi;
  }
  return lo;
}

template <int DDT, int GDT>
__global__ __launch_bounds__(kSumThreads) void embed_sum_kernel(SumArgs a) {
  const uint64_t items = static_cast<uint64_t>(a.tiles) * a.chunks;
  for (uint64_t b = blockIdx.x; b * (kSumThreads / 64) < items; b += gridDim.x) {
    const uint64_t item = b * (kSumThreads / 64) + (threadIdx.x >> 6);
    if (item >= items) continue;
    if (a.dim >= 8) sum_tile<DDT, GDT, true>(a, item);
    else sum_tile<DDT, GDT, false>(a, item);
  }
}

// The row that begins in `tile` and goes on behind it.  Its four waves add a
// quarter of the tiles each, then the first adds the quarters in order.
template <int GDT>
__global__ __launch_bounds__(kSumThreads) void embed_join_kernel(SumArgs a) {
  constexpr uint32_t W = kSumThreads / 64;
  __shared__ float sums[W][kSumCols];
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t items = static_cast<uint64_t>(a.tiles - 1) * a.chunks;  // the last tile has none
  for (uint64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const uint32_t tile = static_cast<uint32_t>(item / a.chunks), chunk = static_cast<uint32_t>(item % a.chunks);
    const uint64_t b0 = static_cast<uint64_t>(tile) * a.run, b1 = b0 + a.run;  // b1 < n: not the last tile
    const uint32_t key = a.keys[b1 - 1];
    const uint64_t ahead = b1 + static_cast<uint64_t>(lane) * a.run;  // the next 64 tiles' first positions
    const uint32_t first = a.keys[ahead < a.n ? ahead : a.n - 1];
    if (key == a.vocab || a.keys[b1] != key || (b0 && a.keys[b0 - 1] == key)) continue;
    // the last tile that holds the row, mostly one of those
    const uint64_t others = __ballot(ahead >= a.n || first != key);
    uint32_t lo;
    if (others) {
      lo = tile + static_cast<uint32_t>(__builtin_ctzll(others));
    } else {
      const uint64_t behind = b1 + first_not_below(a.keys + b1, a.n - b1, static_cast<uint64_t>(key) + 1);
      lo = static_cast<uint32_t>((behind - 1) / a.run);
    }
    const uint32_t count = lo - tile + 1;  // [tile][1], then [tile + 1][0] to [lo][0]
    const uint32_t g = chunk * (kSumCols / 8) + lane;
    const int in = in_group(a.dim, g);
    float acc[8] = {};
    const uint32_t j1 = static_cast<uint32_t>(static_cast<uint64_t>(count) * (wave + 1) / W);
    constexpr uint32_t U = 8;  // parts in flight
    for (uint32_t j0 = static_cast<uint32_t>(static_cast<uint64_t>(count) * wave / W); j0 < j1; j0 += U) {
      Raw8<kF32> r[U];
#pragma unroll
      for (uint32_t u = 0; u < U; ++u) {
        const uint32_t j = j0 + u;
        const float* p = j ? sum_part(a, tile + j, 0) : sum_part(a, tile, 1);
        r[u] = load8_raw<kF32>(reinterpret_cast<uint64_t>(p) + 32ull * g, j < j1 ? in : 0);
      }
#pragma unroll
      for (uint32_t u = 0; u < U; ++u) {
        float f[8];
        unpack8<kF32>(r[u], f);
        if (j0 + u < j1) {
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e] += f[e];
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[wave][e * 64 + lane] = acc[e];
    __syncthreads();
    if (wave == 0 && in > 0) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        for (uint32_t w = 1; w < W; ++w) acc[e] += sums[w][e * 64 + lane];
      sum_write<GDT>(a, key, g, acc, in);
    }
    __syncthreads();
  }
}

// ---- few tokens: one launch ---------------------------------------------------------------
// A block takes a token and lists the positions of its row in their order.  A
// row of up to kDirectAlone tokens is summed by the block of the first of them,
// 512 columns a wave.  Of more, the block of token q takes columns 512 q and on:
// there each wave sums a run of the tokens and the first wave adds the others'
// sums.  Other blocks clear the rows without a token.
// Bound by the launch and the reads' latency: 1024 tokens, as often as words,
// added to rows of 2048 columns in bf16 5.8 us (sorted 20.2); all of one row
// 29.5 (sorted 15.7), for one block then reads a column's tokens.  Up to 1024
// tokens blocks of 256 threads (512: 8.8 and 18.6 us), to 2048 of 512, where the
// one row costs more (rows of 1024: 14.9, 256 threads 11.2, sorted 20.7; one row
// 33, 59 and 20).  4096 tokens: 36 us, sorted 25.
constexpr uint32_t kDirectTokens = 2048;
constexpr uint32_t kDirectSlots = 4;  // tokens of a thread: 256 threads up to 1024 tokens, then 512
constexpr uint32_t kDirectAlone = 8;

template <int DDT, int GDT, bool WHOLE, uint32_t THREADS>
__global__ __launch_bounds__(THREADS) void embed_direct_kernel(EmbedBwd a, Fill fill, uint64_t fills) {
  constexpr uint32_t W = THREADS / 64;
  constexpr int U = kDirectAlone;  // rows in flight
  __shared__ uint16_t list[kDirectSlots * THREADS];  // positions of the row's tokens
  __shared__ uint32_t found[W];
  __shared__ uint32_t own;  // where the block's token is in the list
  __shared__ unsigned long long touched;
  __shared__ float sums[W][kSumCols];
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t n = static_cast<uint32_t>(a.n), chunks = (a.dim + kSumCols - 1) / kSumCols;
  for (uint64_t b = blockIdx.x; b < n + fills; b += gridDim.x) {
    if (b >= n) {
      const uint64_t r0 = (b - n) * fill.per;
      if (threadIdx.x == 0) touched = 0;
      __syncthreads();
      for (uint32_t j = threadIdx.x; j < n; j += THREADS) {
        const uint64_t row = token_row(a.tokens, a.token64, j, a.first, a.vocab);
        if (row >= r0 && row < r0 + fill.per) atomicOr(&touched, 1ull << (row - r0));  // any order gives the same
      }
      __syncthreads();
      const uint64_t skip = touched;
      __syncthreads();
      fill_rows(fill, b - n, skip);
      continue;
    }
    const uint32_t i = static_cast<uint32_t>(b);
    const uint32_t row = token_row(a.tokens, a.token64, i, a.first, a.vocab);
    if (row >= a.vocab) continue;  // the same for the whole block
    const uint32_t j0 = wave * (64 * kDirectSlots) + lane;
    uint64_t same[kDirectSlots];
    uint32_t count = 0;
#pragma unroll
    for (uint32_t s = 0; s < kDirectSlots; ++s) {
      const uint32_t j = j0 + s * 64;
      same[s] = __ballot(j < n && token_row(a.tokens, a.token64, j < n ? j : 0, a.first, a.vocab) == row);
      count += __popcll(same[s]);
    }
    if (lane == 0) found[wave] = count;
    __syncthreads();
    uint32_t total = 0, at = 0;
#pragma unroll
    for (uint32_t w = 0; w < W; ++w) {
      total += found[w];
      at += w < wave ? found[w] : 0;
    }
#pragma unroll
    for (uint32_t s = 0; s < kDirectSlots; ++s) {
      const uint32_t to = at + __popcll(same[s] & ((1ull << lane) - 1));
      if (same[s] >> lane & 1) list[to] = static_cast<uint16_t>(j0 + s * 64);
      if (j0 + s * 64 == i) own = to;
      at += __popcll(same[s]);
    }
    __syncthreads();
    // the same for the whole block; the next list is written behind a barrier
    const bool shared = total > kDirectAlone;
    const uint32_t from = shared ? own : own * chunks + wave, step = shared ? total : W;
    const uint32_t run = shared ? (total + W - 1) / W : total;
    const uint32_t t0 = shared ? wave * run : 0, t1 = t0 + run < total ? t0 + run : total;
    for (uint32_t chunk = from; chunk < chunks; chunk += step) {
      const Cols cols = sum_cols(a.dim, chunk);
      const uint64_t to = a.dw.data + (static_cast<uint64_t>(row) * a.dw.stride + 8ull * cols.g) * kEsz<GDT>;
      const bool writes = !shared || wave == 0;
      Raw8<GDT> old = load8_raw<GDT>(to, a.accumulate && writes ? cols.in : 0);
      float acc[8] = {};
      for (uint32_t c0 = t0; c0 < t1; c0 += 64) {
        const uint32_t m = t1 - c0 < 64 ? t1 - c0 : 64;
        const uint32_t mine = list[lane < m ? c0 + lane : c0];
        for (uint32_t u0 = 0; u0 < m; u0 += U) {
          Raw8<DDT> r[U];
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const uint32_t p = __builtin_amdgcn_readlane(mine, u0 + u);
            r[u] = load_cols<DDT, WHOLE>(a.dout.data + p * a.dout.stride * kEsz<DDT>, cols);
          }
#pragma unroll
          for (int u = 0; u < U; ++u) {
            float f[8];
            unpack8<DDT>(r[u], f);
            if (u0 + u < m) {
#pragma unroll
              for (int e = 0; e < 8; ++e) acc[e] += f[e];
            }
          }
        }
      }
      if (shared) {
        __syncthreads();  // the sums before are read
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[wave][e * 64 + lane] = acc[e];
        __syncthreads();
        if (wave == 0)
          for (uint32_t w = 1; w < W; ++w)
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] += sums[w][e * 64 + lane];
      }
      if (!writes || cols.in <= 0) continue;
      if constexpr (WHOLE) move_down(cols, acc);
      float f[8];
      unpack8<GDT>(old, f);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = a.accumulate ? acc[e] * a.scale + f[e] : acc[e] * a.scale;
      store8<GDT>(to, f, cols.in);
    }
  }
}

uint64_t pad256(uint64_t x) { return (x + 255) / 256 * 256; }

struct BwdRegions {
  uint64_t keys[2], pos[2], hist, part, end;
  uint32_t run, tiles;
};
BwdRegions bwd_regions(uint64_t n, uint64_t dim) {
  BwdRegions r{};
  if (n <= kDirectTokens) return r;
  r.run = sum_run(n, (dim + kSumCols - 1) / kSumCols);
  r.tiles = static_cast<uint32_t>((n + r.run - 1) / r.run);
  const bool radix = n > kBlockTokens;  // up to twice that, by the table
  const uint64_t list = pad256(n * 4);
  uint64_t at = 0;
  for (int i = 0; i < (radix ? 2 : 1); ++i) {
    r.keys[i] = at;
    r.pos[i] = at + list;
    at += 2 * list;
  }
  r.hist = at;
  if (radix) at += pad256((n + sort_tile(n) - 1) / sort_tile(n) * kDigits * 4);
  r.part = at;
  if (r.tiles > 1) at += pad256(static_cast<uint64_t>(r.tiles) * 2 * dim * 4);
  r.end = at;
  return r;
}

template <int WDT>
hipError_t embed_fwd_of(const EmbedFwd& a, hipStream_t st) {
  const uint32_t groups = (a.dim + 7) / 8;
  uint32_t lg = 0;
  while ((1u << lg) < groups && (1u << lg) < kEmbedThreads) ++lg;
  const uint64_t per_block = kEmbedThreads >> lg;
  const uint32_t grid = grid_for((a.n + per_block - 1) / per_block, kEmbedThreads);
  return launch_op(a.out_dtype == kBf16 ? embed_fwd_kernel<WDT, kBf16> : embed_fwd_kernel<WDT, kF32>, grid,
                   kEmbedThreads, st, a, lg);
}

template <int DDT, int GDT>
hipError_t embed_sums(const SumArgs& s, hipStream_t st) {
  const uint64_t items = static_cast<uint64_t>(s.tiles) * s.chunks;
  const hipError_t e =
      launch_op(embed_sum_kernel<DDT, GDT>, grid_for((items + kSumThreads / 64 - 1) / (kSumThreads / 64), kSumThreads),
                kSumThreads, st, s);
  if (e != hipSuccess || s.tiles <= 1) return e;
  return launch_op(embed_join_kernel<GDT>, grid_for(static_cast<uint64_t>(s.tiles - 1) * s.chunks, kSumThreads),
                   kSumThreads, st, s);
}

Fill fill_of(uint64_t data, uint64_t pitch, uint64_t rows, uint64_t bytes) {
  const uint64_t per = bytes < 262144 ? 262144 / bytes : 1;
  return Fill{data, pitch, 0, rows, data + (rows ? (rows - 1) * pitch + bytes : 0), bytes, static_cast<uint32_t>(per < 64 ? per : 64)};
}
Fill whole_table(const EmbedBwd& a) {
  const uint64_t e = a.dw_dtype == kBf16 ? 2 : 4;
  return fill_of(a.dw.data, a.dw.stride * e, a.accumulate ? 0 : a.vocab, a.dim * e);
}
// The same where no row is left out: rows without a gap are cleared 4 KB at a time.
Fill whole_table_at_once(const EmbedBwd& a) {
  const Fill f = whole_table(a);
  if (f.pitch != f.bytes || f.rows == 0) return f;
  Fill g = fill_of(f.data, 4096, (f.end - f.data + 4095) / 4096, 4096);
  g.end = f.end;
  return g;
}

// Blocks for `work` items and behind them for the rows to clear; a capped grid
// leaves some of each.
struct SortGrid {
  uint32_t fill_from, blocks;
};
SortGrid sort_grid(uint64_t work, const Fill& f, uint32_t threads) {
  SortGrid g;
  const uint64_t fills = fill_blocks(f);
  const uint32_t cap = grid_for(~0ull >> 1, threads);
  g.fill_from = static_cast<uint32_t>(work < cap / 2 ? work : cap / 2);
  g.blocks = g.fill_from + static_cast<uint32_t>(fills < cap - g.fill_from ? fills : cap - g.fill_from);
  return g;
}

template <int DDT, int GDT, bool WHOLE>
hipError_t embed_direct(const EmbedBwd& a, hipStream_t st) {
  const Fill f = whole_table(a);
  const uint64_t fills = fill_blocks(f);
  if (a.n + fills == 0) return hipSuccess;
  if (a.n <= 256 * kDirectSlots)
    return launch_op(embed_direct_kernel<DDT, GDT, WHOLE, 256>, grid_for(a.n + fills, 256), 256, st, a, f, fills);
  return launch_op(embed_direct_kernel<DDT, GDT, WHOLE, 512>, grid_for(a.n + fills, 512), 512, st, a, f, fills);
}

template <int DDT, int GDT>
hipError_t embed_bwd_of(const EmbedBwd& a, const SumArgs& s, hipStream_t st) {
  if (a.n > kDirectTokens) return embed_sums<DDT, GDT>(s, st);
  return a.dim >= 8 ? embed_direct<DDT, GDT, true>(a, st) : embed_direct<DDT, GDT, false>(a, st);
}

}  // namespace

hipError_t launch_embed_fwd(const EmbedFwd& a, hipStream_t st) {
  return a.w_dtype == kBf16 ? embed_fwd_of<kBf16>(a, st) : embed_fwd_of<kF32>(a, st);
}

uint64_t embed_bwd_workspace(uint64_t n, uint64_t dim) { return bwd_regions(n, dim).end; }

hipError_t launch_embed_bwd(const EmbedBwd& a, hipStream_t st) {
  const BwdRegions r = bwd_regions(a.n, a.dim);
  uint32_t* keys[2] = {reinterpret_cast<uint32_t*>(a.ws + r.keys[0]), reinterpret_cast<uint32_t*>(a.ws + r.keys[1])};
  uint32_t* pos[2] = {reinterpret_cast<uint32_t*>(a.ws + r.pos[0]), reinterpret_cast<uint32_t*>(a.ws + r.pos[1])};
  int sorted = 0;
  const Fill table = whole_table_at_once(a);
  if (!sorts_in_block(a.n, table.rows * table.bytes)) {
    uint32_t* hist = reinterpret_cast<uint32_t*>(a.ws + r.hist);
    const uint32_t tile = sort_tile(a.n);
    const uint64_t tiles = (a.n + tile - 1) / tile;
    uint32_t launches = 0, launch = 0;
    for (uint32_t shift = 0; shift == 0 || a.vocab >> shift; shift += kDigitBits) launches += 2;  // keys 0 to vocab
    Fill f = table;
    const uint64_t rows = f.rows, share = (rows / launches + f.per) / f.per * f.per;
    auto next = [&] {  // the launch's share of the table
      f.first = share * launch < rows ? share * launch : rows;
      ++launch;
      f.rows = share * launch < rows ? share * launch : rows;
      return sort_grid(tiles, f, kSortThreads);
    };
    int from = -1;
    for (uint32_t shift = 0; shift == 0 || a.vocab >> shift; shift += kDigitBits) {
      const int to = from == 0 ? 1 : 0;
      const uint32_t* ki = from < 0 ? nullptr : keys[from];
      const uint32_t* pi = from < 0 ? nullptr : pos[from];
      SortGrid g = next();
      hipError_t e = launch_op(embed_count_kernel, g.blocks, kSortThreads, st, a, f, g.fill_from, ki, shift, tile, hist);
      if (e != hipSuccess) return e;
      g = next();
      e = launch_op(embed_scatter_kernel, g.blocks, kSortThreads, st, a, f, g.fill_from, ki, pi, shift, tile, hist, keys[to],
                    pos[to]);
      if (e != hipSuccess) return e;
      from = to;
    }
    sorted = from;
  } else if (a.n > kRankTokens) {
    const SortGrid g = sort_grid(1, table, kBlockThreads);
    uint32_t bits = 1;
    while (a.vocab >> bits) ++bits;  // keys 0 to vocab
    const uint32_t passes = (bits + kDigitBits - 1) / kDigitBits;
    const hipError_t e = launch_op(a.n > kBlockTokens ? embed_block_sort_kernel<16> : embed_block_sort_kernel<8>, g.blocks,
                                   kBlockThreads, st, a, table, passes, (bits + passes - 1) / passes, keys[0], pos[0]);
    if (e != hipSuccess) return e;
  } else if (a.n > kDirectTokens) {
    const SortGrid g = sort_grid((a.n + kRankOwn - 1) / kRankOwn, table, kRankThreads);
    const hipError_t e = launch_op(embed_rank_kernel, g.blocks, kRankThreads, st, a, table, g.fill_from, keys[0], pos[0]);
    if (e != hipSuccess) return e;
  }
  SumArgs s;
  s.dout = a.dout;
  s.dw = a.dw;
  s.keys = keys[sorted];
  s.pos = pos[sorted];
  s.part = reinterpret_cast<float*>(a.ws + r.part);
  s.n = a.n;
  s.vocab = a.vocab;
  s.dim = a.dim;
  s.run = r.run;
  s.tiles = r.tiles;
  s.chunks = (a.dim + kSumCols - 1) / kSumCols;
  s.scale = a.scale;
  s.accumulate = a.accumulate;
  if (a.dout_dtype == kBf16)
    return a.dw_dtype == kBf16 ? embed_bwd_of<kBf16, kBf16>(a, s, st) : embed_bwd_of<kBf16, kF32>(a, s, st);
  return a.dw_dtype == kBf16 ? embed_bwd_of<kF32, kBf16>(a, s, st) : embed_bwd_of<kF32, kF32>(a, s, st);
}

}  // namespace lc
