// Sequences of a cache or of linear states forked, reordered, compacted, freed.
//
// A copy, bound by the bytes that move: every source read once, every destination written once.
//
// Into another cache a CTA copies a part of one unit, eight 16-byte pieces of a thread in flight; the destinations of one source are
// neighbours in the grid, so that it is read from HBM once.  Nine of thirteen sequences x 24 units x 1001 slots, fp32, d 64: 38 us,
// 6.0 TB/s (by columns, as below, 48 us).
//
// In place the work is cut by columns, 16 bytes at one place of a unit, which a thread handles for all sequences: it fetches the
// column of every distinct source into its own part of shared memory (asynchronous 16-byte copies), then writes it to every
// destination, zeros of freed states among them.  So any map is right (cycles, forks, chains, freed sources): a column is written
// only after all of it has been read, and nobody else touches it.  Threads share nothing but the map, so nobody waits for anybody.
// Eight beams x 1024 units x 1024 slots: 6.1 GB in 979 us, 6.2 TB/s.  Small calls are bound by the CTAs' set-up, which finds out the
// sources behind two dependent loads and three barriers before a byte moves: a prompt forked into seven more samples in one layer,
// 138 MB, takes 28 us (4.9 TB/s) in 2048 CTAs of two columns a thread; ten sequences x 32 units x 2622 slots from one, fp32, 873 MB,
// 146 (6.0 TB/s).
#include "decoding.cuh"

namespace roco {
namespace {

constexpr int kMost = ROCO_REORDER_MAX_S;  // sequences of an in-place call

// A column that moves: number of the unit, its 16-byte chunks that move, the slot of a thread's room that they are kept in.
struct Place {
  long long unit;
  int end, slot;
};
constexpr int kListBytes = 2 * sizeof(Place) + 5 * sizeof(int);

__device__ __forceinline__ void fetch16(uint32_t dst, const void *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void fetch4(uint32_t dst, const void *src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void fetched() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// The source of destination b.
__device__ __forceinline__ int source_of(const ReorderParams &p, int b, bool report) {
  const int a = p.map[b];
  if (a >= 0 ? a < p.S_src : a == ROCO_REORDER_KEEP || a == ROCO_REORDER_FREE) return a == b && p.in_place ? ROCO_REORDER_KEEP : a;
  if (report) atomicOr(p.status, ROCO_DEV_BAD_MAP);
  return ROCO_REORDER_KEEP;
}

constexpr int kCopyThreads = 256, kCopyFlight = 8;

// Part of one unit into another cache, or other states.
__global__ void __launch_bounds__(kCopyThreads) reorder_copy_kernel(const ReorderParams p) {
  const int b = blockIdx.x % p.S_dst, rest = blockIdx.x / p.S_dst, g = rest / p.parts, part = rest - g * p.parts;
  const bool cache = p.arrays == 2;
  const int a = source_of(p, b, rest == 0);
  if (a == ROCO_REORDER_KEEP) return;
  const long long to = (long long)b * p.G + g, from = (long long)a * p.G + g;
  int live = 0;
  if (cache && a >= 0) {
    live = p.src_live[from];
    if (live < 0 || live > p.B_src) {
      if (part == 0 && threadIdx.x == 0) atomicOr(p.status, ROCO_DEV_BAD_LIVE);
      return;
    }
  }
  const int chunks = a < 0 && cache ? 0 : cache ? live << p.row_shift : (int)(p.src_unit / 16);
  constexpr int kTile = kCopyThreads * kCopyFlight;
  const int tiles = (chunks + kTile - 1) / kTile;
  for (int t = part; t < p.arrays * tiles; t += p.parts) {
    const int array = t >= tiles, c0 = (t - array * tiles) * kTile + threadIdx.x;
    const uint4 *src = reinterpret_cast<const uint4 *>(p.src[array] + from * p.src_unit);
    uint4 *dst = reinterpret_cast<uint4 *>(p.dst[array] + to * p.dst_unit);
    uint4 x[kCopyFlight];
#pragma unroll
    for (int u = 0; u < kCopyFlight; ++u) {
      const int c = c0 + u * kCopyThreads;
      x[u] = make_uint4(0, 0, 0, 0);   // (what a freed sequence's states become)
      if (a >= 0 && c < chunks) x[u] = __ldg(src + c);
    }
#pragma unroll
    for (int u = 0; u < kCopyFlight; ++u) {
      const int c = c0 + u * kCopyThreads;
      if (c < chunks) dst[c] = x[u];
    }
  }
  if (!cache) return;
  for (int k = part * kCopyThreads + threadIdx.x; k < p.B_dst; k += p.parts * kCopyThreads) {
    const long long i = from * p.B_src + k, o = to * p.B_dst + k;
    if (k < live) {
      const float s = p.src_s[i], q = p.src_q[i];
      const int n = p.src_n[i], pos = p.src_pos[i];
      p.dst_s[o] = s; p.dst_q[o] = q; p.dst_n[o] = n; p.dst_pos[o] = pos;
    } else {
      p.dst_pos[o] = -1;
    }
  }
  if (part == 0 && threadIdx.x == 0) {
    p.dst_live[to] = live;
    p.dst_t_next[to] = a < 0 ? 0 : p.src_t_next[from];
  }
}

__global__ void reorder_kernel(const ReorderParams p) {
  extern __shared__ uint4 room[];
  __shared__ int n_slots_, n_copies_, n_empty_, max_live;
  const int tid = threadIdx.x, threads = blockDim.x;
  const int g = blockIdx.x / p.parts, part = blockIdx.x - g * p.parts, S = p.S_dst;
  const bool cache = p.arrays == 2;
  // behind the threads' room (kListBytes for every sequence)
  Place *const from = reinterpret_cast<Place *>(room + threads * p.room), *const to = from + S;  // of every slot; of every copy
  int *const map = reinterpret_cast<int *>(to + S);   // a destination's source, KEEP or FREE
  int *const occupied = map + S;                      // occupied slots of every sequence in this unit
  int *const slot_of = occupied + S;                  // source sequence -> its slot, -1: none yet
  int *const live_of = slot_of + S;                   // slot -> its occupied slots in this unit; -1: not copied
  int *const empty = live_of + S;                     // destinations that are freed

  // which sources there are, and who gets them (up to kMost / threads sequences a thread)
  for (int i = tid; i < S; i += threads) {
    slot_of[i] = -1;
    occupied[i] = cache ? p.src_live[(long long)i * p.G + g] : 0;
    map[i] = source_of(p, i, blockIdx.x == 0);
  }
  if (tid == 0) n_slots_ = n_copies_ = n_empty_ = max_live = 0;
  __syncthreads();
  for (int i = tid; i < S; i += threads) {
    const int a = map[i];
    if (a == ROCO_REORDER_FREE) empty[atomicAdd(&n_empty_, 1)] = i;
    if (a < 0) continue;
    if (atomicCAS(&slot_of[a], -1, kMost) == -1) {   // the first to ask for it
      const int slot = atomicAdd(&n_slots_, 1);
      int live = occupied[a];
      if (cache && (live < 0 || live > p.B_src)) {
        if (part == 0) atomicOr(p.status, ROCO_DEV_BAD_LIVE);
        live = -1;
      }
      atomicMax(&max_live, live);
      live_of[slot] = live;
      from[slot] = {(long long)a * p.G + g, cache ? max(live, 0) << p.row_shift : (int)(p.src_unit / 16), slot};
      slot_of[a] = slot;
    }
  }
  __syncthreads();
  for (int i = tid; i < S; i += threads) {
    const int a = map[i];
    if (a < 0) continue;
    const int slot = slot_of[a];
    if (cache && live_of[slot] < 0) continue;
    to[atomicAdd(&n_copies_, 1)] = {(long long)i * p.G + g, from[slot].end, slot};
  }
  __syncthreads();
  launch_dependents();
  const int n_slots = n_slots_, n_copies = n_copies_, n_empty = n_empty_;
  const uint32_t mine = smem_u32(room + tid);
  const uint32_t step = threads * 16;  // from one of a thread's 16-byte places to its next

  // K and V, or the states: columns of 16 bytes
  const int chunks = cache ? max_live << p.row_shift : (int)(p.src_unit / 16);
  // columns of a thread at a time: as many as there is room for, but no more than leave work for every CTA of the unit
  const int lanes = p.parts * threads, share = (chunks * p.arrays + lanes - 1) / lanes;
  const int U = n_slots ? max(1, min(p.room / n_slots, share)) : 1;
  const int per = threads * U, tiles = (chunks + per - 1) / per, stat_tiles = cache ? (p.B_dst + threads - 1) / threads : 0;
  for (int t = part; t < stat_tiles + p.arrays * tiles; t += p.parts) {
    if (t < stat_tiles) {
      // statistics and positions: the four numbers of a slot are a column
      const int k = t * threads + tid;
      if (k >= p.B_dst) continue;
      for (int j = 0; j < n_slots; ++j) {
        if (k >= live_of[j]) continue;
        const long long at = from[j].unit * p.B_src + k;
        const uint32_t to = mine + (uint32_t)j * step;
        fetch4(to, p.src_s + at);
        fetch4(to + 4, p.src_q + at);
        fetch4(to + 8, p.src_n + at);
        fetch4(to + 12, p.src_pos + at);
      }
      fetched();
      for (int i = 0; i < n_copies; ++i) {
        const int j = to[i].slot;
        const long long at = to[i].unit * p.B_dst + k;
        if (k < live_of[j]) {
          const uint4 x = room[j * threads + tid];
          p.dst_s[at] = __uint_as_float(x.x);
          p.dst_q[at] = __uint_as_float(x.y);
          p.dst_n[at] = (int)x.z;
          p.dst_pos[at] = (int)x.w;
        } else {
          p.dst_pos[at] = -1;
        }
      }
      for (int i = 0; i < n_empty; ++i) p.dst_pos[((long long)empty[i] * p.G + g) * p.B_dst + k] = -1;
      continue;
    }
    const int array = t - stat_tiles >= tiles;
    const int c0 = (t - stat_tiles - array * tiles) * per + tid;
    const char *src = p.src[array] + c0 * 16LL;
    char *dst = p.dst[array] + c0 * 16LL;
    for (int u = 0; u < U; ++u) {
      const int c = c0 + u * threads;
#pragma unroll 4
      for (int j = 0; j < n_slots; ++j) {
        const Place f = from[j];
        if (c < f.end) fetch16(mine + (uint32_t)(j * U + u) * step, src + f.unit * p.src_unit + u * step);
      }
    }
    fetched();
    for (int u = 0; u < U; ++u) {
      const int c = c0 + u * threads;
#pragma unroll 4
      for (int i = 0; i < n_copies; ++i) {
        const Place t = to[i];
        if (c < t.end) *reinterpret_cast<uint4 *>(dst + t.unit * p.dst_unit + u * step) = room[(t.slot * U + u) * threads + tid];
      }
      // a freed sequence's states become zero here too: it may be the source of others, whose column this thread has fetched
      if (!cache && c < chunks)
        for (int i = 0; i < n_empty; ++i)
          *reinterpret_cast<uint4 *>(dst + ((long long)empty[i] * p.G + g) * p.dst_unit + u * step) = make_uint4(0, 0, 0, 0);
    }
  }
}

// live and t_next of every unit in place, where every CTA of the kernel above reads them: they change behind it.
__global__ void reorder_live_kernel(const ReorderParams p) {
  const int g = blockIdx.x, b = threadIdx.x;
  const int a = b < p.S_dst ? source_of(p, b, false) : ROCO_REORDER_KEEP;
  wait_for_launch_before();
  int live = 0, t_next = 0;
  if (a >= 0) {
    live = p.src_live[(long long)a * p.G + g];
    t_next = p.src_t_next[(long long)a * p.G + g];
  }
  __syncthreads();
  if (a == ROCO_REORDER_KEEP || live < 0 || live > p.B_src) return;
  p.dst_live[(long long)b * p.G + g] = live;
  p.dst_t_next[(long long)b * p.G + g] = t_next;
}

}  // namespace

roco_status launch_reorder(ReorderParams p, int sms, cudaStream_t stream) {
  const long long chunks = p.arrays * (p.src_unit / 16);
  if (!p.in_place) {
    constexpr int kTile = kCopyThreads * kCopyFlight;
    p.parts = (int)((chunks + kTile - 1) / kTile);
    const long long ctas = (long long)p.S_dst * p.G * p.parts;
    if (ctas > 0x7fffffffLL) return ROCO_ERR_UNSUPPORTED;
    reorder_copy_kernel<<<(unsigned)ctas, kCopyThreads, 0, stream>>>(p);
    return cudaGetLastError() == cudaSuccess ? ROCO_OK : ROCO_ERR_CUDA;
  }
  // Threads so that a CTA's places take 48 KB at most (four CTAs per SM) down to one warp; at least eight places each, for the
  // columns of few sources that are in flight together (16 beams x 512 states 37 us, with 64 KB 39; 54 sequences forked from one x 40 units x 1016
  // 199 and 215, 52 beams x 10 units x 3223, d 64, 128 and 120).  CTAs with two columns a thread, up to 64 per SM (16 beams x 512 states with
  // one and four columns 42 and 47 us where this took 40; eight beams x 1024 units with at most 16 and 32 CTAs per SM 1027 and 1008
  // us, with 64 972).
  int threads = 256;
  while (threads > 32 && threads * p.S_dst * 16 > 49152) threads /= 2;
  p.room = p.S_dst < 8 ? 8 : p.S_dst;
  const int smem = threads * p.room * 16 + p.S_dst * kListBytes;
  long long parts = (chunks + 2LL * threads - 1) / (2LL * threads), most = (64LL * sms + p.G - 1) / p.G;
  if (parts > most) parts = most;
  p.parts = parts < 1 ? 1 : (int)parts;
  if ((long long)p.G * p.parts > 0x7fffffffLL) return ROCO_ERR_UNSUPPORTED;
  static SmemLimit limit;
  if (!limit((const void *)reorder_kernel, 32 * kMost * 16 + kMost * kListBytes)) return ROCO_ERR_CUDA;
  reorder_kernel<<<(unsigned)(p.G * p.parts), threads, smem, stream>>>(p);
  if (cudaGetLastError() != cudaSuccess) return ROCO_ERR_CUDA;
  if (p.arrays == 1) return ROCO_OK;
  return launch_overlapped(reorder_live_kernel, (unsigned)p.G, kMost, 0, stream, p) ? ROCO_OK : ROCO_ERR_CUDA;
}

}  // namespace roco
