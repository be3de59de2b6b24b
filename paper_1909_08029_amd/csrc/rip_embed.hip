// Embedding lookup with scaling and its gradient by sorted tokens (gfx950).
//
//   out[t]  = scale * table[id_t]
//   grad[v] = scale * sum over {t : id_t = v}, ascending t, of dout[t]
//
// Both are bound by memory: the lookup reads and writes a row a token, the
// gradient reads a row a token and writes the whole table's gradient (P-Reduce
// reads every element of it).  65536 tokens, a table of 131072 x 2048, all bf16:
// the lookup takes 59 us (350 MB, 5.9 TB/s), the gradient 187: sort and two thirds
// of the zeros 68, merge and the other third 37 (537 MB, 5.1 TB/s), sums 70 (350
// MB, 5.0 TB/s), joins 12.
//
// The gradient runs over the tokens sorted by id, a fixed number of them to a
// wave, however often an id occurs: a frequent id is shared by many waves
// instead of making one wave long.  A wave adds a run of equal ids in
// registers and writes the row if the run is its own; a run that passes the
// wave's ends leaves its partial sums in the workspace, and a last launch adds
// those.  Nothing is added atomically, so the result is the same in every call.

#include "rip_ops_common.h"

namespace rip {
namespace {

constexpr int kWave = 64;
constexpr int kLookupBlock = 256;
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / kWave;
constexpr int kSortItems = 8;                          // tokens of a thread
constexpr int kChunk = kSortThreads * kSortItems;      // most tokens sorted by one workgroup
constexpr int kPart = kChunk / 2;                      // tokens of a chunk where there are several:
                                                       // 8192 at once take 21 us, 4096 14
constexpr int kMaxDigit = 8;                           // bits of a pass of the sort
constexpr int kMaxEntries = 32;                        // of the sorted list to a wave, below kWave
constexpr int kSumWaves = 4;                            // that share a row's columns in a workgroup
constexpr int kBatch = 4;                              // rows that a wave loads together
constexpr int kColumns = kWave * kLane;                // columns of a wave
constexpr int kMergeThreads = 256;

constexpr int kFillBytes = 1 << 16;                    // bytes zeroed by a workgroup of the fill

// A lane's columns: eight from `at` on, of which it owns those from skip on.  The
// last lane of a row whose width is no multiple of eight moves back so that its
// eight lie in the row: no load then needs a second look at the width.  NARROW rows,
// of fewer than eight columns, are taken element by element.
struct Columns {
  int at, skip, width;
  bool on;
};
__device__ __forceinline__ Columns columns_of(int c, int width) {
  const int at = min(c, max(width - kLane, 0));
  return {at, c - at, width, c < width};
}
template <int DT, bool NARROW, bool STREAM = false>
__device__ __forceinline__ void load_columns(const typename Elem<DT>::T* row, const Columns& k,
                                             float (&f)[kLane]) {
  if constexpr (NARROW)
    load_unit<DT>(row, 0, k.width, f);
  else
    Elem<DT>::template load8<STREAM>(row + k.at, f);
}
template <int DT>
__device__ __forceinline__ void store_columns(typename Elem<DT>::T* row, const Columns& k,
                                              const float (&f)[kLane]) {
  if (k.skip == 0 && k.width >= kLane) {
    Elem<DT>::store8(row + k.at, f);
  } else {
#pragma unroll
    for (int j = 0; j < kLane; ++j)
      if (j >= k.skip && k.at + j < k.width) Elem<DT>::store(row + k.at + j, f[j]);
  }
}

// A thread handles eight columns of ROWS consecutive tokens, whose rows it loads
// together.
template <int TD, int OD, int ROWS, bool NARROW>
__global__ __launch_bounds__(kLookupBlock) void lookup_kernel(
    const typename Elem<TD>::T* table, int64_t vocab, int width, int64_t ld, const void* ids,
    int wide, int64_t n, uint32_t units, FastDiv per_row, float scale, typename Elem<OD>::T* out,
    int64_t ld_out) {
  const uint32_t unit = blockIdx.x * kLookupBlock + threadIdx.x;
  if (unit >= units) return;
  const uint32_t group = per_row.div(unit);
  const Columns k = columns_of((int)(unit - group * per_row.d) * kLane, width);
  const int64_t t = (int64_t)group * ROWS;
  float f[ROWS][kLane];
  bool live[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {  // every row is loaded, row 0 for ids outside the table
    const int64_t id = load_id(ids, wide, t + r < n ? t + r : n - 1);
    live[r] = id >= 0 && id < vocab;
    load_columns<TD, NARROW>(table + (live[r] ? id : 0) * ld, k, f[r]);
  }
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    if (t + r >= n) break;
#pragma unroll
    for (int j = 0; j < kLane; ++j) f[r][j] = live[r] ? f[r][j] * scale : 0.0f;
    store_columns<OD>(out + (t + r) * ld_out, k, f[r]);
  }
}

// Sort of up to kChunk (id, position) pairs by id in one workgroup: passes over
// digits of `bits` bits from the lowest, each stable.  A wave holds consecutive
// elements; equal digits in a wave find each other with one ballot a bit.
struct SortShared {
  uint32_t key[kChunk];
  uint16_t pos[kChunk];
  uint32_t count[kSortWaves << kMaxDigit];
  uint32_t wave_sum[kSortWaves];
};

__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// `items` of each thread, the first items * kSortThreads of the chunk, take part.
__device__ void sort_chunk(SortShared& sh, int items, int passes, int bits) {
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  const int buckets = 1 << bits, cells = kSortWaves << bits;
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  for (int p = 0; p < passes; ++p) {
    for (int i = tid; i < cells; i += kSortThreads) sh.count[i] = 0;
    __syncthreads();
    uint32_t key[kSortItems], rank[kSortItems];
    uint16_t pos[kSortItems];
#pragma unroll
    for (int r = 0; r < kSortItems; ++r) {
      if (r >= items) break;
      const int i = (wave * items + r) * kWave + lane;
      key[r] = sh.key[i];
      pos[r] = sh.pos[i];
      const uint32_t d = (key[r] >> (p * bits)) & (buckets - 1);
      uint64_t same = ~(uint64_t)0;
      for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot((d >> b) & 1);
        same &= (d >> b) & 1 ? set : ~set;
      }
      // counters are laid out digit by digit, the waves of a digit in a row
      const uint32_t cell = d * kSortWaves + wave;
      const uint32_t before = sh.count[cell];
      rank[r] = before + __popcll(same & below);
      // a wave's accesses to LDS happen in order; the fences keep the compiler's
      wave_fence();
      if (!(same & below)) sh.count[cell] = before + __popcll(same);
      wave_fence();
    }
    __syncthreads();
    // exclusive sums of the counters, a run of them to each thread
    const int per = (cells + kSortThreads - 1) / kSortThreads;
    uint32_t sum = 0;
    for (int i = 0; i < per; ++i) {
      const int cell = tid * per + i;
      if (cell < cells) sum += sh.count[cell];
    }
    uint32_t scan = sum;
    for (int o = 1; o < kWave; o <<= 1) {
      const uint32_t up = __shfl_up(scan, o);
      if (lane >= o) scan += up;
    }
    if (lane == kWave - 1) sh.wave_sum[wave] = scan;
    __syncthreads();
    uint32_t base = scan - sum;
    for (int w = 0; w < wave; ++w) base += sh.wave_sum[w];
    for (int i = 0; i < per; ++i) {
      const int cell = tid * per + i;
      if (cell < cells) {
        const uint32_t c = sh.count[cell];
        sh.count[cell] = base;
        base += c;
      }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortItems; ++r) {
      if (r >= items) break;
      const uint32_t d = (key[r] >> (p * bits)) & (buckets - 1);
      const uint32_t to = sh.count[d * kSortWaves + wave] + rank[r];
      sh.key[to] = key[r];
      sh.pos[to] = pos[r];
    }
    __syncthreads();
  }
}

// Bytes [p, end) become zeros; both are even addresses.
template <bool STREAM>
__device__ __forceinline__ void zero_range(char* p, char* end, int thread, int threads) {
  const u32x4_any zero = {0, 0, 0, 0};
  char* body = (char*)(((uintptr_t)p + 15) & ~(uintptr_t)15);
  body = body < end ? body : end;
  for (char* q = p + 2 * thread; q < body; q += 2 * threads) *(uint16_t*)q = 0;
  char* q = body + 16 * thread;
  for (; q + 16 <= end; q += 16 * threads) {
    if constexpr (STREAM)
      store_stream((u32x4_any*)q, zero);
    else
      *(u32x4_any*)q = zero;
  }
  if (q < end)
    for (; q < end; q += 2) *(uint16_t*)q = 0;
}

// Rows of the gradient that a launch zeroes beside its other work, a run of them to
// a workgroup.
struct Fill {
  void* grad;
  int64_t vocab, ld;
  int width, rows;  // rows of a workgroup
  int stream;       // past the caches
  int64_t first;    // run of the launch's first such workgroup
};
template <int GD, int THREADS, bool STREAM>
__device__ __forceinline__ void zero_rows(const Fill& z, int64_t run) {
  const int64_t row0 = (z.first + run) * z.rows;
  const int64_t row1 = row0 + z.rows < z.vocab ? row0 + z.rows : z.vocab;
  constexpr int kSize = sizeof(typename Elem<GD>::T);
  char* grad = static_cast<char*>(z.grad);
  const int tid = threadIdx.x;
  if (z.ld == z.width) {  // rows without gaps are one range
    zero_range<STREAM>(grad + row0 * z.ld * kSize, grad + row1 * z.ld * kSize, tid, THREADS);
  } else {  // a wave a row
    for (int64_t r = row0 + tid / kWave; r < row1; r += THREADS / kWave) {
      char* p = grad + r * z.ld * kSize;
      zero_range<STREAM>(p, p + (int64_t)z.width * kSize, tid % kWave, kWave);
    }
  }
}
template <int GD, int THREADS>
__device__ __forceinline__ void zero_rows(const Fill& z, int64_t run) {
  if (z.stream)
    zero_rows<GD, THREADS, true>(z, run);
  else
    zero_rows<GD, THREADS, false>(z, run);
}

// Workgroups below `chunks` each sort `chunk` tokens (ids outside the vocabulary
// become `vocab` and go last); the others zero rows of the gradient meanwhile.
template <int GD>
__global__ __launch_bounds__(kSortThreads) void sort_kernel(
    const void* ids, int wide, int64_t n, uint32_t vocab, int passes, int bits, int chunks,
    int chunk, uint32_t* sorted_id, uint32_t* sorted_pos, Fill fill) {
  __shared__ SortShared sh;
  const int tid = threadIdx.x;
  if ((int)blockIdx.x >= chunks) {
    zero_rows<GD, kSortThreads>(fill, blockIdx.x - chunks);
    return;
  }
  const int64_t base = (int64_t)blockIdx.x * chunk;
  const int count = (int)(n - base < chunk ? n - base : chunk);
  const int items = (count + kSortThreads - 1) / kSortThreads;
  for (int i = tid; i < items * kSortThreads; i += kSortThreads) {
    int64_t id = i < count ? load_id(ids, wide, base + i) : (int64_t)vocab;
    if (id < 0 || id > (int64_t)vocab) id = vocab;
    sh.key[i] = (uint32_t)id;
    sh.pos[i] = (uint16_t)i;
  }
  __syncthreads();
  sort_chunk(sh, items, passes, bits);
  for (int i = tid; i < count; i += kSortThreads) {
    sorted_id[base + i] = sh.key[i];
    sorted_pos[base + i] = (uint32_t)base + sh.pos[i];
  }
}

// Groups of kWays sorted chunks become sorted runs: an entry's place is its place in
// its own chunk and its rank in every other (equal ids of earlier chunks go first).
// kSide chunks are searched side by side, a halving of all of them at a time, as
// the loads of one search wait for each other: first among every 64th entry of the
// chunks, in LDS, then among the 64 before it, which lie in two cache lines.
// Workgroups from `merges` on zero rows of the gradient.
constexpr int kWays = 16, kSide = 8, kEvery = 64, kSamples = kPart / kEvery;
template <int GD>
__global__ __launch_bounds__(kMergeThreads) void merge_kernel(
    const uint32_t* id_in, const uint32_t* pos_in, int64_t n, uint32_t* id_out, uint32_t* pos_out,
    int merges, Fill fill) {
  __shared__ uint32_t sample[kSide][kSamples];
  if ((int)blockIdx.x >= merges) {
    zero_rows<GD, kMergeThreads>(fill, blockIdx.x - merges);
    return;
  }
  const int last_entry = (int)n - 1;
  const int i = (int)blockIdx.x * kMergeThreads + threadIdx.x, mine = min(i, last_entry);
  const int own = mine / kPart;
  const uint32_t id = id_in[mine], pos = pos_in[mine];
  // a workgroup's entries are of one chunk; its group's chunks
  const int group = (int)blockIdx.x * kMergeThreads / (kWays * kPart) * kWays;
  const int chunks = min(group + kWays, last_entry / kPart + 1);
  int at = group * kPart + mine - own * kPart;
  for (int c0 = group; c0 < chunks; c0 += kSide) {
    __syncthreads();
    for (int j = threadIdx.x; j < kSide * kSamples; j += kMergeThreads) {
      const int64_t e = (int64_t)c0 * kPart + (int64_t)j * kEvery + kEvery - 1;
      sample[j / kSamples][j % kSamples] = e < n ? id_in[e] : ~0u;  // past the end: above all ids
    }
    __syncthreads();
    // rank = entries below `id`, or up to it in earlier chunks: of 2 * half left
    // to look at, the first half goes if its last entry does
    int rank[kSide];
#pragma unroll
    for (int u = 0; u < kSide; ++u) rank[u] = 0;
#pragma unroll
    for (int half = kSamples; half > 0; half /= 2)
#pragma unroll
      for (int u = 0; u < kSide; ++u) {
        const int to = rank[u] + half;
        const uint32_t x = sample[u][min(to, kSamples) - 1];
        const bool goes = x < id || (x == id && c0 + u < own);
        rank[u] = goes && to <= kSamples ? to : rank[u];
      }
#pragma unroll
    for (int u = 0; u < kSide; ++u) rank[u] *= kEvery;
#pragma unroll
    for (int half = kEvery / 2; half > 0; half /= 2) {
      uint32_t x[kSide];
      int e[kSide];
#pragma unroll
      for (int u = 0; u < kSide; ++u) {
        e[u] = (c0 + u) * kPart + rank[u] + half - 1;
        x[u] = id_in[min(e[u], last_entry)];
      }
#pragma unroll
      for (int u = 0; u < kSide; ++u) {
        const bool goes = x[u] < id || (x[u] == id && c0 + u < own);
        rank[u] += goes && rank[u] < kPart && e[u] <= last_entry ? half : 0;
      }
    }
#pragma unroll
    for (int u = 0; u < kSide; ++u)
      if (c0 + u < chunks && c0 + u != own) at += rank[u];
  }
  if (i <= last_entry) {
    id_out[at] = id;
    pos_out[at] = pos;
  }
}

// The same with runs of `run` entries, longer than a chunk (lists of more than
// kWays * kPart tokens), searched in memory.
__global__ __launch_bounds__(kMergeThreads) void merge_runs_kernel(
    const uint32_t* id_in, const uint32_t* pos_in, int64_t n, int run, uint32_t* id_out,
    uint32_t* pos_out) {
  const int i = (int)blockIdx.x * kMergeThreads + threadIdx.x, last_entry = (int)n - 1;
  if (i > last_entry) return;
  const int own = i / run, group = own / kWays * kWays;
  const int runs = min(group + kWays, last_entry / run + 1);
  const uint32_t id = id_in[i];
  int at = group * run + i - own * run;
  for (int c0 = group; c0 < runs; c0 += kSide) {
    int rank[kSide];
#pragma unroll
    for (int u = 0; u < kSide; ++u) rank[u] = 0;
    for (int half = run; half > 0; half /= 2) {
      uint32_t x[kSide];
      int64_t e[kSide];
#pragma unroll
      for (int u = 0; u < kSide; ++u) {
        e[u] = (int64_t)(c0 + u) * run + rank[u] + half - 1;
        x[u] = id_in[e[u] < last_entry ? e[u] : last_entry];
      }
#pragma unroll
      for (int u = 0; u < kSide; ++u) {
        const bool goes = x[u] < id || (x[u] == id && c0 + u < own);
        rank[u] += goes && rank[u] + half <= run && e[u] <= last_entry ? half : 0;
      }
    }
#pragma unroll
    for (int u = 0; u < kSide; ++u)
      if (c0 + u < runs && c0 + u != own) at += rank[u];
  }
  id_out[at] = id;
  pos_out[at] = pos_in[i];
}

template <int GD, bool NARROW>
__device__ __forceinline__ void write_row(typename Elem<GD>::T* row, const Columns& k, float scale,
                                          int accumulate, const float (&acc)[kLane]) {
  float f[kLane];
  if (accumulate) {
    load_columns<GD, NARROW>(row, k, f);
#pragma unroll
    for (int j = 0; j < kLane; ++j) f[j] = f[j] + scale * acc[j];
  } else {
#pragma unroll
    for (int j = 0; j < kLane; ++j) f[j] = scale * acc[j];
  }
  store_columns<GD>(row, k, f);
}

// Partial sums of a wave's two slots, a lane's eight columns in a row.
__device__ __forceinline__ float* partial_at(float* partial, int64_t wave, int slot, int lanes,
                                             int lane) {
  return partial + ((wave * 2 + slot) * lanes + lane) * kLane;
}

// One wave: entries [a, b) of the sorted list, 512 columns.  Partial sums of a
// run that began before `a` go to slot 0 of the wave's share, those of a run
// that begins here and goes on to slot 1.
template <int DD, int GD, bool NARROW>
__global__ __launch_bounds__(kWave* kSumWaves) void sum_kernel(
    const typename Elem<DD>::T* dout, int64_t ld_dout, const uint32_t* id, const uint32_t* pos,
    int64_t n, uint32_t vocab, int per, float scale, typename Elem<GD>::T* grad, int width,
    int64_t ld, int accumulate, float* partial) {
  const int64_t a = (int64_t)blockIdx.x * per;
  const int count = (int)(a + per < n ? per : n - a), lane = threadIdx.x % kWave;
  const int c = (blockIdx.y * blockDim.x + threadIdx.x) * kLane, lanes = (width + kLane - 1) / kLane;
  const Columns k = columns_of(c, width);
  // the wave's entries and the one after them, an entry a lane
  const int64_t mine = a + lane < n ? a + lane : n - 1;
  const uint32_t my_id = a + lane < n ? id[mine] : vocab, my_pos = pos[mine];
  const uint32_t before = id[a > 0 ? a - 1 : 0];
  const uint32_t head = __builtin_amdgcn_readfirstlane(my_id);
  if (head >= vocab) return;  // only ids outside the vocabulary from here on
  float acc[kLane] = {};
  bool begins = a == 0 || before != head;
  for (int i0 = 0; i0 < count; i0 += kBatch) {
    float f[kBatch][kLane];
    uint32_t v[kBatch + 1];
#pragma unroll
    for (int u = 0; u <= kBatch; ++u) v[u] = __builtin_amdgcn_readlane(my_id, i0 + u);
    // all of them are loaded, by all lanes, and not all are used
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int64_t t = (uint32_t)__builtin_amdgcn_readlane(my_pos, min(i0 + u, count - 1));
      load_columns<DD, NARROW, true>(dout + t * ld_dout, k, f[u]);
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (i0 + u >= count || v[u] >= vocab) break;
#pragma unroll
      for (int j = 0; j < kLane; ++j) acc[j] += f[u][j];
      const bool ends = v[u + 1] != v[u];
      if (!ends && i0 + u + 1 < count) continue;
      if (k.on) {
        if (begins && ends)
          write_row<GD, NARROW>(grad + (int64_t)v[u] * ld, k, scale, accumulate, acc);
        else
          Elem<RIP_FP32>::store8(partial_at(partial, blockIdx.x, begins ? 1 : 0, lanes, c / kLane), acc);
      }
#pragma unroll
      for (int j = 0; j < kLane; ++j) acc[j] = 0.0f;
      begins = true;
    }
  }
}

constexpr int kJoinWaves = 8;
constexpr int kShortRun = 16;  // partial sums that one wave adds

// Runs that pass the end of a wave's entries: a workgroup looks at the ends of
// kJoinWaves waves of the sum, one each of its own, and adds up the partial sums of
// the runs that begin in those: slot 1 of the wave where a run begins and slot 0 of
// those that it passes through.  A wave adds a short run alone; a long one is
// shared by all waves of the workgroup.
template <int GD, bool NARROW>
__global__ __launch_bounds__(kWave* kJoinWaves) void join_kernel(
    const uint32_t* id, int64_t n, uint32_t vocab, int per, int waves, float* partial,
    float scale, typename Elem<GD>::T* grad, int width, int64_t ld, int accumulate) {
  __shared__ float part[kJoinWaves][kColumns];
  __shared__ int run_last[kJoinWaves];
  __shared__ uint32_t run_id[kJoinWaves];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int c = blockIdx.y * kColumns + lane * kLane, lanes = (width + kLane - 1) / kLane;
  const Columns k = columns_of(c, width);
  {
    const int64_t own = (int64_t)blockIdx.x * kJoinWaves + wave, a = own * per, b = a + per;
    int last = -1;  // last wave that the run reaches
    uint32_t v = 0;
    if (b < n) {
      v = id[b - 1];
      const bool goes_on = id[b] == v, began = id[a] != v || a == 0 || id[a - 1] != v;
      if (v < vocab && goes_on && began) {
        last = (int)own + 1;
        for (;; last += kWave) {  // the first whose own last entry ends the run
          const int w = last + lane;
          const int64_t end = ((int64_t)w + 1) * per;
          const bool on = w < waves - 1 && id[end - 1] == v && id[end] == v;
          const uint64_t stop = ~__ballot(on);
          if (stop) {
            last += __ffsll((unsigned long long)stop) - 1;
            break;
          }
        }
      }
    }
    const int count = last - (int)own;
    if (last >= 0 && count <= kShortRun) {
      if (k.on) {
        float acc[kLane], f[kLane];
        Elem<RIP_FP32>::load8(partial_at(partial, own, 1, lanes, c / kLane), acc);
#pragma unroll 4
        for (int w = 1; w <= count; ++w) {
          Elem<RIP_FP32>::load8(partial_at(partial, own + w, 0, lanes, c / kLane), f);
#pragma unroll
          for (int j = 0; j < kLane; ++j) acc[j] += f[j];
        }
        write_row<GD, NARROW>(grad + (int64_t)v * ld, k, scale, accumulate, acc);
      }
      last = -1;
    }
    if (lane == 0) {
      run_last[wave] = last;
      run_id[wave] = v;
    }
  }
  __syncthreads();
  for (int r = 0; r < kJoinWaves; ++r) {
    const int last = run_last[r], first = blockIdx.x * kJoinWaves + r;
    if (last < 0) continue;
    const int count = last - first;  // partial sums after the first
    float acc[kLane] = {}, f[kLane];
    if (k.on) {
      if (wave == 0) Elem<RIP_FP32>::load8(partial_at(partial, first, 1, lanes, c / kLane), acc);
      const int w1 = (wave + 1) * count / kJoinWaves;
#pragma unroll 4
      for (int w = wave * count / kJoinWaves; w < w1; ++w) {
        Elem<RIP_FP32>::load8(partial_at(partial, (int64_t)first + 1 + w, 0, lanes, c / kLane), f);
#pragma unroll
        for (int j = 0; j < kLane; ++j) acc[j] += f[j];
      }
    }
#pragma unroll
    for (int j = 0; j < kLane; ++j) part[wave][lane * kLane + j] = acc[j];
    __syncthreads();
    if (wave == 0 && k.on) {
      for (int w = 1; w < kJoinWaves; ++w)
#pragma unroll
        for (int j = 0; j < kLane; ++j) acc[j] += part[w][lane * kLane + j];
      write_row<GD, NARROW>(grad + (int64_t)run_id[r] * ld, k, scale, accumulate, acc);
    }
    __syncthreads();
  }
}

// The gradient of up to kFewTokens tokens in one launch, without a sort: each
// workgroup has a run of the table's rows, and each wave has all ids in registers,
// two to a lane, and finds a row's tokens with two ballots.  (40 tokens, a table of
// 50257 x 512 fp32: 21 us through the sort, 14.5 so.)
constexpr int kFewTokens = 2 * kWave, kFewThreads = 256, kFewBatch = 8;
template <int DD, int GD, bool NARROW>
__global__ __launch_bounds__(kFewThreads) void few_kernel(
    const typename Elem<DD>::T* dout, int64_t ld_dout, const void* ids, int wide, int n,
    float scale, int accumulate, Fill fill) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, width = fill.width;
  const int64_t id0 = lane < n ? load_id(ids, wide, lane) : -1;
  const int64_t id1 = lane + kWave < n ? load_id(ids, wide, lane + kWave) : -1;
  const int64_t row0 = (int64_t)blockIdx.x * fill.rows;
  const int64_t row1 = row0 + fill.rows < fill.vocab ? row0 + fill.rows : fill.vocab;
  if (!__ballot((id0 >= row0 && id0 < row1) || (id1 >= row0 && id1 < row1))) {
    if (!accumulate) zero_rows<GD, kFewThreads>(fill, blockIdx.x);
    return;
  }
  typename Elem<GD>::T* grad = static_cast<typename Elem<GD>::T*>(fill.grad);
  // a wave takes 512 columns of a row at a time
  const int parts = (width + kColumns - 1) / kColumns, units = (int)(row1 - row0) * parts;
  for (int unit = wave; unit < units; unit += kFewThreads / kWave) {
    const int64_t r = row0 + unit / parts;
    const int c0 = unit % parts * kColumns, c = c0 + lane * kLane;
    uint64_t in0 = __ballot(id0 == r), in1 = __ballot(id1 == r);
    typename Elem<GD>::T* row = grad + r * fill.ld;
    if (!(in0 | in1)) {
      if (!accumulate)
        zero_range<false>((char*)(row + c0), (char*)(row + min(c0 + kColumns, width)), lane, kWave);
      continue;
    }
    const Columns k = columns_of(c, width);
    float acc[kLane] = {};
    while (in0 | in1) {  // kFewBatch of the row's tokens at a time, ascending
      float f[kFewBatch][kLane];
      int64_t t = 0;
      int got = 0;
#pragma unroll
      for (int u = 0; u < kFewBatch; ++u) {
        if (in0) {
          t = __ffsll((unsigned long long)in0) - 1;
          in0 &= in0 - 1;
          got = u + 1;
        } else if (in1) {
          t = kWave + __ffsll((unsigned long long)in1) - 1;
          in1 &= in1 - 1;
          got = u + 1;
        }
        load_columns<DD, NARROW>(dout + t * ld_dout, k, f[u]);
      }
#pragma unroll
      for (int u = 0; u < kFewBatch; ++u)
#pragma unroll
        for (int j = 0; j < kLane; ++j)
          if (u < got) acc[j] += f[u][j];
    }
    if (k.on) write_row<GD, NARROW>(row, k, scale, accumulate, acc);
  }
}

// Entries of the sorted list that a wave adds up.
int entries_per_wave(int64_t n, int64_t width) {
  const int64_t columns = ceil_div(width, kColumns);
  int per = 4;
  while (per < kMaxEntries && ceil_div(n, 2 * per) * columns >= 2048) per *= 2;
  return per;
}

struct GradPlan {
  int per, waves, chunk, chunks;
  int64_t id_bytes, partial_bytes, total;
};
GradPlan grad_plan(int64_t n, int64_t width) {
  GradPlan p{};
  p.per = entries_per_wave(n, width);
  p.waves = (int)ceil_div(n, p.per);
  p.chunk = n <= kChunk ? kChunk : kPart;
  p.chunks = (int)ceil_div(n, p.chunk);
  p.id_bytes = ceil_div(n * 4, 256) * 256;
  p.partial_bytes = (int64_t)p.waves * 2 * ceil_div(width, kLane) * kLane * 4;
  // ids and positions, once more where chunks are merged, and the partial sums
  p.total = p.id_bytes * (p.chunks > 1 ? 4 : 2) + p.partial_bytes;
  return p;
}

template <int TD, int OD>
const void* lookup_of(bool many, bool narrow) {
  return narrow ? (const void*)lookup_kernel<TD, OD, 1, true>
         : many ? (const void*)lookup_kernel<TD, OD, 4, false>
                : (const void*)lookup_kernel<TD, OD, 1, false>;
}
template <int DD, int GD>
const void* sum_of(bool narrow) {
  return narrow ? (const void*)sum_kernel<DD, GD, true> : (const void*)sum_kernel<DD, GD, false>;
}

template <int DD, int GD>
const void* few_of(bool narrow) {
  return narrow ? (const void*)few_kernel<DD, GD, true> : (const void*)few_kernel<DD, GD, false>;
}

int32_t check_ids(const void* ids, int32_t id_type, int64_t n) {
  if (id_type != RIP_INT32 && id_type != RIP_INT64)
    return fail(RIP_E_UNSUPPORTED, "unknown id type %d", id_type);
  if (n < 0) return fail(RIP_E_INVAL, "n_tokens %lld < 0", (long long)n);
  if (n > RIP_MAX_TOKENS)
    return fail(RIP_E_UNSUPPORTED, "n_tokens %lld > %d", (long long)n, RIP_MAX_TOKENS);
  if (n && !ids) return fail(RIP_E_INVAL, "ids is NULL");
  if (reinterpret_cast<uintptr_t>(ids) % (id_type == RIP_INT64 ? 8 : 4))
    return fail(RIP_E_ALIGN, "ids = %p is not aligned to its type", ids);
  return RIP_OK;
}

int32_t check_table(int64_t vocab, int64_t width) {
  if (vocab < 1 || width < 1)
    return fail(RIP_E_INVAL, "vocab %lld and width %lld must be >= 1", (long long)vocab,
                (long long)width);
  if (vocab > INT32_MAX - 1 || width > RIP_MAX_WIDTH)
    return fail(RIP_E_UNSUPPORTED, "vocab %lld or width %lld above the limit", (long long)vocab,
                (long long)width);
  return RIP_OK;
}

}  // namespace

int32_t check_matrix(const void* p, const char* what, int32_t dtype, int64_t rows, int64_t width,
                     int64_t ld) {
  if (!known_dtype(dtype)) return fail(RIP_E_UNSUPPORTED, "%s: unknown dtype %d", what, dtype);
  if (rows < 0 || width < 0 || ld < width)
    return fail(RIP_E_INVAL, "%s: %lld rows of %lld with row stride %lld", what, (long long)rows,
                (long long)width, (long long)ld);
  if (rows && width && !p) return fail(RIP_E_INVAL, "%s is NULL", what);
  if (reinterpret_cast<uintptr_t>(p) % elem_bytes(dtype))
    return fail(RIP_E_ALIGN, "%s = %p is not aligned to its type", what, p);
  return RIP_OK;
}

}  // namespace rip

using namespace rip;

extern "C" int32_t rip_embed_lookup(const void* table, int32_t table_dtype, int64_t vocab,
                                    int64_t width, int64_t ld_table, const void* ids,
                                    int32_t id_type, int64_t n_tokens, float scale, void* out,
                                    int32_t out_dtype, int64_t ld_out, void* stream) {
  clear_error();
  int32_t rc;
  if ((rc = check_ids(ids, id_type, n_tokens)) || (rc = check_table(vocab, width)) ||
      (rc = check_matrix(table, "table", table_dtype, vocab, width, ld_table)) ||
      (rc = check_matrix(out, "out", out_dtype, n_tokens, width, ld_out)))
    return rc;
  if (overlap(out, span(out_dtype, n_tokens, width, ld_out), table,
              span(table_dtype, vocab, width, ld_table)) ||
      overlap(out, span(out_dtype, n_tokens, width, ld_out), ids,
              n_tokens * (id_type == RIP_INT64 ? 8 : 4)))
    return fail(RIP_E_OVERLAP, "out overlaps table or ids");
  if (n_tokens == 0) return RIP_OK;
  const int64_t per_row = ceil_div(width, kLane);
  if (n_tokens * per_row >= (int64_t)1 << 31)
    return fail(RIP_E_UNSUPPORTED, "%lld tokens of width %lld are above the limit",
                (long long)n_tokens, (long long)width);
  // four rows to a thread where that leaves the card full
  const bool narrow = width < kLane, many = !narrow && n_tokens * per_row >= (int64_t)1 << 19;
  uint32_t units = (uint32_t)(ceil_div(n_tokens, many ? 4 : 1) * per_row);
  FastDiv div = FastDiv::make((uint32_t)per_row);
  int w = (int)width, wide = id_type == RIP_INT64;
  void* args[] = {&table, &vocab, &w,   &ld_table, &ids, &wide, &n_tokens,
                  &units, &div,   &scale, &out,    &ld_out};
  const void* fn = table_dtype == RIP_FP32
                       ? (out_dtype == RIP_FP32 ? lookup_of<RIP_FP32, RIP_FP32>(many, narrow)
                                                : lookup_of<RIP_FP32, RIP_BF16>(many, narrow))
                       : (out_dtype == RIP_FP32 ? lookup_of<RIP_BF16, RIP_FP32>(many, narrow)
                                                : lookup_of<RIP_BF16, RIP_BF16>(many, narrow));
  return launch(fn, dim3((uint32_t)ceil_div(units, kLookupBlock)), dim3(kLookupBlock), args, 0,
                stream, "rip_embed_lookup");
}

extern "C" int64_t rip_embed_grad_workspace(int64_t n_tokens, int64_t width) {
  if (n_tokens <= kFewTokens || n_tokens > RIP_MAX_TOKENS || width < 1 || width > RIP_MAX_WIDTH) return 0;
  return grad_plan(n_tokens, width).total;
}

extern "C" int32_t rip_embed_grad(const void* dout, int32_t dout_dtype, int64_t ld_dout,
                                  const void* ids, int32_t id_type, int64_t n_tokens, float scale,
                                  void* grad, int32_t grad_dtype, int64_t vocab, int64_t width,
                                  int64_t ld_grad, int32_t accumulate, void* workspace,
                                  int64_t workspace_bytes, void* stream) {
  clear_error();
  int32_t rc;
  if ((rc = check_ids(ids, id_type, n_tokens)) || (rc = check_table(vocab, width)) ||
      (rc = check_matrix(dout, "dout", dout_dtype, n_tokens, width, ld_dout)) ||
      (rc = check_matrix(grad, "grad", grad_dtype, vocab, width, ld_grad)))
    return rc;
  const int64_t grad_span = span(grad_dtype, vocab, width, ld_grad);
  const int64_t ids_span = n_tokens * (id_type == RIP_INT64 ? 8 : 4);
  if (overlap(grad, grad_span, dout, span(dout_dtype, n_tokens, width, ld_dout)) ||
      overlap(grad, grad_span, ids, ids_span))
    return fail(RIP_E_OVERLAP, "grad overlaps dout or ids");
  const int64_t need = rip_embed_grad_workspace(n_tokens, width);
  if (need > 0) {
    if (!workspace || workspace_bytes < need)
      return fail(RIP_E_INVAL, "workspace of %lld bytes, %lld needed", (long long)workspace_bytes,
                  (long long)need);
    if (reinterpret_cast<uintptr_t>(workspace) % 16)
      return fail(RIP_E_ALIGN, "workspace = %p is not 16-byte aligned", workspace);
    if (overlap(workspace, need, grad, grad_span) || overlap(workspace, need, ids, ids_span) ||
        overlap(workspace, need, dout, span(dout_dtype, n_tokens, width, ld_dout)))
      return fail(RIP_E_OVERLAP, "workspace overlaps another buffer");
  }
  if (n_tokens == 0 && accumulate) return RIP_OK;

  int w = (int)width, wide = id_type == RIP_INT64;
  const bool narrow = width < kLane;
  // Zeros that the memory-side cache holds stay there until the sums come (a table
  // of 206 MB: 64 us against 72 past it); more go past it (537 MB: 281 against 290).
  const bool stream_zeros = vocab * width * elem_bytes(grad_dtype) > kCacheBytes;
  Fill fill{grad, vocab, ld_grad, w, (int)(kFillBytes / (width * elem_bytes(grad_dtype))),
            stream_zeros, 0};
  if (fill.rows < 1) fill.rows = 1;
  if (fill.rows < vocab >> 20) fill.rows = (int)((vocab >> 20) + 1);  // within a launch's grid
  if (n_tokens <= kFewTokens) {
    int n = (int)n_tokens;
    const int64_t spread = ceil_div(vocab, 1024);  // rows of a workgroup that leave the card full
    if (fill.rows > spread) fill.rows = (int)spread;
    void* args[] = {&dout, &ld_dout, &ids, &wide, &n, &scale, &accumulate, &fill};
    const void* fn = dout_dtype == RIP_FP32
                         ? (grad_dtype == RIP_FP32 ? few_of<RIP_FP32, RIP_FP32>(narrow)
                                                   : few_of<RIP_FP32, RIP_BF16>(narrow))
                         : (grad_dtype == RIP_FP32 ? few_of<RIP_BF16, RIP_FP32>(narrow)
                                                   : few_of<RIP_BF16, RIP_BF16>(narrow));
    return launch(fn, dim3((uint32_t)ceil_div(vocab, fill.rows)), dim3(kFewThreads), args, 0,
                  stream, "rip_embed_grad: few");
  }

  GradPlan p = grad_plan(n_tokens, width);
  char* ws = static_cast<char*>(workspace);
  uint32_t* id_a = (uint32_t*)ws;
  uint32_t* pos_a = (uint32_t*)(ws + p.id_bytes);
  uint32_t* const id_merged = (uint32_t*)(ws + 2 * p.id_bytes);
  uint32_t* const pos_merged = (uint32_t*)(ws + 3 * p.id_bytes);
  uint32_t *id_b = p.chunks > 1 ? id_merged : id_a, *pos_b = p.chunks > 1 ? pos_merged : pos_a;
  float* partial = (float*)(ws + p.id_bytes * (p.chunks > 1 ? 4 : 2));

  // Keys run to `vocab` itself (ids outside the vocabulary).
  int key_bits = 1;
  while (((int64_t)1 << key_bits) <= vocab) ++key_bits;
  int passes = (key_bits + kMaxDigit - 1) / kMaxDigit;
  int bits = (key_bits + passes - 1) / passes;
  uint32_t v32 = (uint32_t)vocab;
  // Runs of rows to zero, all beside the sort, or a third of them beside the merge.
  const int64_t runs = accumulate ? 0 : ceil_div(vocab, fill.rows);
  const int64_t later = p.chunks > 1 ? runs / 3 : 0;
  {
    void* args[] = {&ids,      &wide,    &n_tokens, &v32,   &passes, &bits,
                    &p.chunks, &p.chunk, &id_a,     &pos_a, &fill};
    const void* fn = grad_dtype == RIP_FP32 ? (const void*)sort_kernel<RIP_FP32>
                                            : (const void*)sort_kernel<RIP_BF16>;
    if ((rc = launch(fn, dim3((uint32_t)(p.chunks + runs - later)), dim3(kSortThreads), args, 0,
                     stream, "rip_embed_grad: sort")))
      return rc;
  }
  if (p.chunks > 1) {
    int merges = (int)ceil_div(n_tokens, kMergeThreads);
    fill.first = runs - later;
    void* args[] = {&id_a, &pos_a, &n_tokens, &id_b, &pos_b, &merges, &fill};
    const void* fn = grad_dtype == RIP_FP32 ? (const void*)merge_kernel<RIP_FP32>
                                            : (const void*)merge_kernel<RIP_BF16>;
    if ((rc = launch(fn, dim3((uint32_t)(merges + later)), dim3(kMergeThreads), args, 0, stream,
                     "rip_embed_grad: merge")))
      return rc;
    for (int64_t run = (int64_t)kWays * kPart; run < n_tokens; run *= kWays) {
      uint32_t *id_in = id_b, *pos_in = pos_b;
      id_b = id_b == id_a ? id_merged : id_a;
      pos_b = pos_b == pos_a ? pos_merged : pos_a;
      int run32 = (int)run;
      void* more[] = {&id_in, &pos_in, &n_tokens, &run32, &id_b, &pos_b};
      if ((rc = launch((const void*)merge_runs_kernel, dim3((uint32_t)merges), dim3(kMergeThreads),
                       more, 0, stream, "rip_embed_grad: merge of runs")))
        return rc;
    }
  }
  const uint32_t columns = (uint32_t)ceil_div(width, kColumns);
  {
    void* args[] = {&dout,  &ld_dout, &id_b, &pos_b,   &n_tokens,   &v32,    &p.per,
                    &scale, &grad,    &w,    &ld_grad, &accumulate, &partial};
    const void* fn =
        dout_dtype == RIP_FP32
            ? (grad_dtype == RIP_FP32 ? sum_of<RIP_FP32, RIP_FP32>(narrow)
                                      : sum_of<RIP_FP32, RIP_BF16>(narrow))
            : (grad_dtype == RIP_FP32 ? sum_of<RIP_BF16, RIP_FP32>(narrow)
                                      : sum_of<RIP_BF16, RIP_BF16>(narrow));
    const uint32_t side = columns < kSumWaves ? columns : kSumWaves;
    if ((rc = launch(fn, dim3((uint32_t)p.waves, (columns + side - 1) / side), dim3(kWave * side),
                     args, 0, stream, "rip_embed_grad: sum")))
      return rc;
  }
  if (p.waves < 2) return RIP_OK;
  void* args[] = {&id_b, &n_tokens, &v32, &p.per,   &p.waves,   &partial,
                  &scale, &grad,    &w,   &ld_grad, &accumulate};
  const void* fn = grad_dtype == RIP_FP32 ? (narrow ? (const void*)join_kernel<RIP_FP32, true>
                                                    : (const void*)join_kernel<RIP_FP32, false>)
                                          : (narrow ? (const void*)join_kernel<RIP_BF16, true>
                                                    : (const void*)join_kernel<RIP_BF16, false>);
  return launch(fn, dim3((uint32_t)ceil_div(p.waves, kJoinWaves), columns), dim3(kWave * kJoinWaves),
                args, 0, stream, "rip_embed_grad: join");
}
