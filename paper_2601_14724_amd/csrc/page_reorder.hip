// Pages of beams after a choice of continuations, for gfx950 (see hermes_page_reorder).
//
// page_reorder   a group (the beams of one sequence in one layer) a workgroup, or several
//                workgroups: each finds the group's new tables, the first writes
//                them, and all share the copies of partly filled pages
//
// A group's room is a range of pages, so that which of them the new tables hold is a bitmap
// in LDS, and a free page a clear bit: no lists or counts are kept between calls, and
// what no beam goes on with is free without being told so.  One launch: the groups need
// nothing of each other.  Few bytes move (tables, and a page's live rows for every beam
// whose parent has another child), so it is bound by its chain: parents, lengths, tables,
// barrier, free pages, barrier, copies.
#include "tokens_internal.h"

namespace hermes {
namespace {

constexpr int kThreads = 512;

struct ReorderShared {
  uint32_t held[kRoomPages / 32];   // pages of the room that a new table holds
  int32_t parent[kMaxBeams], len[kMaxBeams];
  int32_t full[kMaxBeams];          // shared pages
  int32_t last[kMaxBeams];          // the parent's partly filled page (-1: none)
  int32_t kept[kMaxBeams];          // 1: the beam goes on in it
  int32_t total[kMaxBeams];         // entries of the new table
  int32_t first[kMaxBeams + 1];     // pages given to the beams before, and to all
  int32_t target[kMaxBeams];        // page that `last` is copied to (-1: none)
  int32_t room, pages;              // the group's room
  int32_t given;                    // of the pages asked for
};

__global__ __launch_bounds__(kThreads) void page_reorder(PageReorderArgs a) {
  __shared__ ReorderShared s;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int g = blockIdx.x / a.shares, share = blockIdx.x % a.shares, B = a.n_beams, rows = 1 << a.pool.log_rows;
  const int64_t row0 = (int64_t)g * B;
  if (tid == 0) {
    int room = a.room[2 * g], pages = a.room[2 * g + 1];
    if (room < 0 || pages < 0 || pages > kRoomPages || (int64_t)room + pages > a.pool.n_pages) {
      room = pages = 0;
      page_note(a.pool, HERMES_PAGE_BAD_ID);
    }
    s.room = room;
    s.pages = pages;
  }
  if (tid < B) {
    int p = a.parent[(int64_t)(g % a.n_seqs) * B + tid], n = 0;
    if (p < -1 || p >= B) {
      p = -1;
      page_note(a.pool, HERMES_PAGE_BAD_PARENT);
    }
    if (p >= 0) {
      n = a.kv_len[row0 + p];
      if (n < 0 || n > (int64_t)a.max_pages << a.pool.log_rows) {
        n = 0;
        page_note(a.pool, HERMES_PAGE_BAD_LENGTH);
      }
    }
    const int full = n >> a.pool.log_rows;
    const int want = p < 0 ? 0 : (int)(((int64_t)n + a.grow + rows - 1) >> a.pool.log_rows);
    s.parent[tid] = p;
    s.len[tid] = n;
    s.full[tid] = full;
    s.last[tid] = n & (rows - 1) ? a.tables[(row0 + p) * a.max_pages + full] : -1;
    s.total[tid] = min(want, a.max_pages);
    s.kept[tid] = 0;
    s.target[tid] = -1;
    if (want > a.max_pages) page_note(a.pool, HERMES_PAGE_NO_ROOM);
    if (share == 0) a.kv_len_out[row0 + tid] = n;
  }
  __syncthreads();
  const int room = s.room, pages = s.pages;
  for (int i = tid; i < (pages + 31) / 32; i += kThreads) s.held[i] = 0;
  __syncthreads();
  for (int b = wave; b < B; b += kThreads / 64) {
    const int32_t *from = a.tables + (row0 + max(s.parent[b], 0)) * a.max_pages;
    int32_t *to = a.tables_out + (row0 + b) * a.max_pages;
    const int full = s.full[b], end = share == 0 ? a.max_pages : full;
    for (int e = lane; e < end; e += 64) {
      const int id = e < full ? from[e] : -1;
      const unsigned at = (unsigned)id - (unsigned)room;
      if (e < full && at < (unsigned)pages) atomicOr(&s.held[at / 32], 1u << (at % 32));
      // (entries that get a page of their own are written below)
      if (share == 0 && (e < full || e >= s.total[b])) to[e] = id;
    }
  }
  __syncthreads();
  bool keep = false;
  if (tid < B) {
    const int id = s.last[tid];
    const unsigned at = (unsigned)id - (unsigned)room;
    keep = (s.len[tid] & (rows - 1)) != 0 && at < (unsigned)pages && (s.held[at / 32] >> (at % 32) & 1) == 0;
    for (int b = 0; keep && b < tid; ++b) keep = !((s.len[b] & (rows - 1)) != 0 && s.last[b] == id);
    s.kept[tid] = keep;
  }
  __syncthreads();
  if (keep) {
    const unsigned at = (unsigned)s.last[tid] - (unsigned)room;
    atomicOr(&s.held[at / 32], 1u << (at % 32));
    if (share == 0) a.tables_out[(row0 + tid) * a.max_pages + s.full[tid]] = s.last[tid];
  }
  __syncthreads();
  // The first wave gives out pages: entry full + kept + i of beam b gets the (first[b] + i)-th
  // free page.
  if (wave == 0) {
    int need = 0;
    if (lane < B) need = s.total[lane] - s.full[lane] - s.kept[lane];
    int end = need;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int x = __shfl_up(end, d);
      if (lane >= d) end += x;
    }
    if (lane < B) s.first[lane] = end - need;
    if (lane == B - 1) s.first[B] = end;
    const int all = __builtin_amdgcn_readlane(end, B - 1);
    int given = 0;
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    for (int w0 = 0; w0 * 32 < pages && given < all; w0 += 64) {
      const int w = w0 + lane, left = pages - 32 * w;
      uint32_t clear = left <= 0 ? 0u : ~s.held[w];
      if (left > 0 && left < 32) clear &= (1u << left) - 1u;
      const int n = __builtin_popcount(clear);
      int upto = n;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int x = __shfl_up(upto, d);
        if (lane >= d) upto += x;
      }
      int rank = given + upto - n;
      for (; clear != 0 && rank < all; clear &= clear - 1, ++rank) {
        const int id = room + 32 * w + __builtin_ctz(clear);
        int b = 0;
        while (s.first[b + 1] <= rank) ++b;
        const int e = s.full[b] + s.kept[b] + rank - s.first[b];
        if (share == 0) a.tables_out[(row0 + b) * a.max_pages + e] = id;
        if (e == s.full[b] && (s.len[b] & (rows - 1)) != 0) s.target[b] = id;
      }
      given += __builtin_amdgcn_readlane(upto, 63);
    }
    given = min(given, all);
    if (given < all && lane < B) {
      const int e0 = s.full[lane] + s.kept[lane];
      for (int i = max(given - s.first[lane], 0); i < need; ++i)
        if (share == 0) a.tables_out[(row0 + lane) * a.max_pages + e0 + i] = -1;
      if (lane == 0) page_note(a.pool, HERMES_PAGE_NO_ROOM);
    }
  }
  __syncthreads();
  // Copies: of every KV head's block the starts of its four parts (see PageBlock).
  const int64_t step = (int64_t)kThreads * a.shares;
  for (int b = 0; b < B; ++b) {
    const int source = s.last[b], target = s.target[b];
    if (target < 0) continue;
    if (source < 0 || source >= a.pool.n_pages) {
      if (tid == 0) page_note(a.pool, HERMES_PAGE_BAD_ID);
      continue;
    }
    const int n = ((s.len[b] & (rows - 1)) + 3) & ~3;
    const int wide = n * a.row_bytes / 16, fine = n * a.scale_bytes / 8;   // pieces of a part
    const int block = 2 * (wide + fine), all = block * a.pool.Hkv;
    const uint8_t *from = a.pool.pages + source * a.pool.page_bytes;
    uint8_t *to = a.pool.pages + target * a.pool.page_bytes;
    for (int64_t i = (int64_t)share * kThreads + tid; i < all; i += step) {
      const int h = (int)i / block, x = (int)i % block;
      const int64_t head = (int64_t)h * a.pool.block_bytes;
      if (x < 2 * wide) {
        const int part = x >= wide;
        const int64_t at = head + (int64_t)part * rows * a.row_bytes + 16 * (x - part * wide);
        *reinterpret_cast<uint4 *>(to + at) = *reinterpret_cast<const uint4 *>(from + at);
      } else {
        const int y = x - 2 * wide, part = y >= fine;
        const int64_t at = head + (int64_t)rows * (2 * a.row_bytes + part * a.scale_bytes) + 8 * (y - part * fine);
        *reinterpret_cast<uint2 *>(to + at) = *reinterpret_cast<const uint2 *>(from + at);
      }
    }
  }
}

}  // namespace

hipError_t launch_page_reorder(const PageReorderArgs &a, hipStream_t s) {
  hipLaunchKernelGGL((page_reorder), dim3(a.n_groups * a.shares), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace hermes
