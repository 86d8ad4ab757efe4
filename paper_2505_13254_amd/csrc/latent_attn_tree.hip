// Absorbed attention over latents on the matrix cores (see latent_attn_tree.h).
//
// A work item is a group of up to 128 rows of one sequence and one split of its pages; the last split also takes the tree's own rows. The
// host chooses how many pages a split has at most (lat_tree_plan); everything else of an item is found on the device, from the offsets and
// lengths.  Items are numbered by sequence, split and group, and each XCD has a run of neighbouring ones: the groups of a (sequence, split) find its pages in one L2.
// Splits hand over sums (records of R + 4 floats: O, reference, denominator), which a second launch merges.
#include <algorithm>

#include "latent_attn_tree.h"

namespace hs {

constexpr int LT_XCD = 8;
constexpr int LT_REC = LT_R + ATTN_REC_PAD;
constexpr int LT_OUT_PITCH = 1024 + 16;  // bytes of a row on its way out

struct LtArgs {
  LatTreeArgs a;
  float c2;    // scale in octaves
  int per;     // pages of a split at most
  int sp_max;  // splits of a sequence at most; 1: results are written directly
  int group;   // rows of an item at most: 128, 64 or 32
  float* part;
  int one_rows, one_len;  // B == 1: the tree's rows and the stored tokens
  int records;            // that part holds: n_sp of every row of a sequence with several splits, sequence by sequence
  int first[LT_XCD + 1];  // the first item of each XCD
};

// Splits of a sequence, and the first page of one.  The last split has the tree's own rows besides, and the page that ends inside: they count as LT_EXTRA pages.
constexpr int LT_EXTRA = 2;
__host__ __device__ __forceinline__ int lt_splits(int64_t pages, int per) { return pages <= per ? 1 : (int)((pages + LT_EXTRA + per - 1) / per); }
__host__ __device__ __forceinline__ int lt_first_page(int sp, int n_sp, int pages) {
  const int p = (int)((int64_t)sp * (pages + LT_EXTRA) / n_sp);
  return sp == n_sp || p > pages ? pages : p;
}

struct LtItem {
  int s, n0, M, sp, n_sp, rg;
  int rec0;  // the sequence's first record
  int64_t L;
};

struct LtLds {
  char ring[4 * LT_TILE];
  int parent[LT_MAX_TREE];
  float stat[4][2][32];
  int64_t out_at[4][32];  // where a wave's rows go
  unsigned odd[2];
  int again;  // some row's reference was too low
  int found[8];
  int sums[4][2];
};
static_assert(sizeof(LtLds) <= 160 * 1024, "LDS of a compute unit");

// Inclusive prefix sums of two numbers over the workgroup, and the totals.
__device__ __forceinline__ void lt_scan(int& x, int& y, int* all_x, int* all_y, LtLds& mem) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  x = wave_prefix_sum(x);
  y = wave_prefix_sum(y);
  if (lane == 63) mem.sums[wave][0] = x, mem.sums[wave][1] = y;
  __syncthreads();
  *all_x = *all_y = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w == wave) x += *all_x, y += *all_y;
    *all_x += mem.sums[w][0];
    *all_y += mem.sums[w][1];
  }
}

// What the device's arrays say of sequence s, within what the host's copies said.
__device__ __forceinline__ void lt_sequence(const LtArgs& g, int s, int* n0, int* M, int64_t* L, int* n_sp) {
  const LatTreeArgs& a = g.a;
  const int from = a.node_offsets[s], to = a.node_offsets[s + 1];
  const int64_t len = a.prefix_lens[s], most = std::min((int64_t)a.max_blocks * 64, (int64_t)HS_MX_MAX_TOKENS);
  *n0 = from;
  *L = len < 0 ? 0 : (len > most ? most : len);
  const int rows = from < 0 ? 0 : std::min(std::min(to - from, LT_MAX_TREE), a.NN - from);
  *M = rows < 0 ? 0 : rows;
  *n_sp = rows > 0 ? std::min(lt_splits((*L + 63) >> 6, g.per), g.sp_max) : 0;
}
__device__ __forceinline__ int lt_records(int M, int Hq, int n_sp) { return n_sp > 1 ? M * Hq * n_sp : 0; }

// The item of a workgroup: the j-th of XCD x's.
__device__ __forceinline__ bool lt_find(const LtArgs& g, LtItem& it, LtLds& mem) {
  const LatTreeArgs& a = g.a;
  const int x = (int)(blockIdx.x & (LT_XCD - 1)), j = (int)(blockIdx.x / LT_XCD), tid = threadIdx.x;
  const int item = g.first[x] + j;
  if (item >= g.first[x + 1]) return false;
  if (a.B == 1) {  // (no trip to memory)
    it.s = it.n0 = it.rec0 = 0;
    it.M = g.one_rows;
    it.L = g.one_len;
    it.n_sp = lt_splits((it.L + 63) >> 6, g.per);
    const int groups = (it.M * a.Hq + g.group - 1) / g.group;
    it.sp = item / groups;
    it.rg = item - it.sp * groups;
    return true;
  }
  if (tid == 0) mem.found[0] = -1;
  int items = 0, records = 0;
  for (int base = 0; base < a.B && items <= item; base += LT_THREADS) {
    const int s = base + tid;
    int n0 = 0, M = 0, n_sp = 0;
    int64_t L = 0;
    if (s < a.B) lt_sequence(g, s, &n0, &M, &L, &n_sp);
    const int groups = (M * a.Hq + g.group - 1) / g.group, mine = n_sp * groups, recs = lt_records(M, a.Hq, n_sp);
    int to = mine, rec_to = recs, all, all_recs;
    lt_scan(to, rec_to, &all, &all_recs, mem);
    const int at = item - (items + to - mine);
    if (at >= 0 && at < mine) {
      const int sp = at / groups;
      mem.found[0] = s;
      mem.found[1] = n0;
      mem.found[2] = M;
      mem.found[3] = sp;
      mem.found[4] = n_sp;
      mem.found[5] = at - sp * groups;
      mem.found[6] = (int)L;
      mem.found[7] = records + rec_to - recs;
    }
    items += all;
    records += all_recs;
    __syncthreads();
  }
  auto get = [&](int k) { return __builtin_amdgcn_readfirstlane(mem.found[k]); };
  it.s = get(0);
  if (it.s < 0) return false;
  it.n0 = get(1);
  it.M = get(2);
  it.sp = get(3);
  it.n_sp = get(4);
  it.rg = get(5);
  it.L = get(6);
  it.rec0 = get(7);
  return it.n_sp == 1 || it.rec0 + lt_records(it.M, a.Hq, it.n_sp) <= g.records;  // (always, where the arrays are as the host's copies)
}

// Rows from `first` on of a page in the ring become zero (what lies behind a sequence's last token may be anything, and 0 x NaN is NaN).
__device__ __forceinline__ void lt_blank(char* page, int first) {
  for (int x = (int)threadIdx.x; x < LT_PAGE / 16; x += LT_THREADS) {
    unsigned row, chunk;
    lt_what(x, &row, &chunk);
    if ((int)row >= first) *reinterpret_cast<uint4*>(page + 16 * x) = make_uint4(0u, 0u, 0u, 0u);
  }
}

template <int RB>
__device__ __forceinline__ void lt_run(const LtArgs& g, const LtItem& it, LtLds& mem) {
  constexpr int NB = RB == 1 ? 8 : 16;
  const LatTreeArgs& a = g.a;
  char* const lds = mem.ring;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int rb = RB == 4 ? wave : RB == 2 ? wave & 1 : 0, kh = RB == 4 ? 0 : wave >> 1, first_block = RB == 1 ? 8 * (wave & 1) : 0;
  const int rows = it.M * a.Hq, row_base = it.rg * g.group + 32 * rb;
  const int row = row_base + col < rows ? row_base + col : rows - 1;  // (rows behind the last repeat it)
  const int i = row / a.Hq, h = row - i * a.Hq;
  const bool last = it.sp == it.n_sp - 1;
  const int all_pages = (int)((it.L + 63) >> 6);
  const int p_lo = lt_first_page(it.sp, it.n_sp, all_pages), n_pages = lt_first_page(it.sp + 1, it.n_sp, all_pages) - p_lo;
  const int rest = n_pages > 0 && p_lo + n_pages == all_pages ? (int)(it.L & 63) : 0;  // tokens of the last page, where it ends inside
  const int n_full = n_pages - (rest > 0 ? 1 : 0);
  const int32_t* const table = a.table + (int64_t)it.s * a.max_blocks + p_lo;
  const char* const pool = static_cast<const char*>(a.pool);
  const bool once = rows <= g.group;  // nobody else reads the pages
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)lds;

  // ---- requests: the numbers of the pages, Q, the tree's last 64 rows that the group sees and the parents, the first page
  int page_base = 0, page_of = 0;  // pages, 64 of them at a time in the lanes
  auto look_up = [&](int t) {      // from the split's page t on
    const int p = t + lane < n_pages ? table[t + lane] : 0;
    page_of = p < 0 || p >= a.n_pages ? 0 : p;  // (an entry that is no page would be a caller's error)
    page_base = t;
  };
  look_up(0);
  // 64 tree rows (from 64 t on; rows behind the last repeat it) straight into the ring's first half, each piece to the place that it has in a page.
  constexpr int PIECES = LT_PAGE / 16 / LT_THREADS;  // 16-byte pieces to a thread
  auto tree_rows = [&](int t) {
    const int left = std::min(64, it.M - 64 * t);
    int id0 = tid;
    asm volatile("" : "+v"(id0));  // (no address of these is kept in registers through the pages)
    const int pieces = left > 32 ? PIECES : PIECES / 2;  // (of 32 rows or fewer nobody looks at the second tile)
#pragma unroll 1
    for (int x = 0; x < pieces; ++x) {
      unsigned r, c;
      lt_what(x * LT_THREADS + id0, &r, &c);
      const int64_t from = it.n0 + 64 * t + ((int)r < left ? (int)r : left - 1);
      lt_fetch_one(c < 64 ? static_cast<const bf16_t*>(a.c_tree) + from * a.c_stride + 8 * c : static_cast<const bf16_t*>(a.r_tree) + from * a.r_stride + 8 * (c - 64),
                   lds0 + (x * LT_THREADS + wave * 64) * 16);
    }
  };
  // What a thread fetched, once it is there: rows with a NaN or an infinity are noted, and those elements made zero: 0 x NaN must not reach rows that do not
  // see them.
  auto mend_tree = [&](int t) {
    int id0 = tid;
    asm volatile("" : "+v"(id0));
    const int pieces = it.M - 64 * t > 32 ? PIECES : PIECES / 2;
#pragma unroll 3
    for (int x = 0; x < pieces; ++x) {
      const unsigned id = x * LT_THREADS + id0;
      uint4 w = *reinterpret_cast<const uint4*>(lds + 16 * id);
      lt_ushort2 most = {0, 0};
      unsigned* const e = &w.x;
#pragma unroll
      for (int y = 0; y < 4; ++y) most = __builtin_elementwise_max(most, __builtin_bit_cast(lt_ushort2, e[y] & 0x7fff7fffu));
      if (most[0] >= 0x7f80 || most[1] >= 0x7f80) {
        unsigned r, c;
        lt_what(id, &r, &c);
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          if ((e[y] & 0x7f80u) == 0x7f80u) e[y] &= 0xffff0000u;
          if ((e[y] & 0x7f800000u) == 0x7f800000u) e[y] &= 0xffffu;
        }
        *reinterpret_cast<uint4*>(lds + 16 * id) = w;
        atomicOr(&mem.odd[r >> 5], 1u << (r & 31));
      }
    }
  };
  const int top_tree = (std::min(rows, (it.rg + 1) * g.group) - 1) / a.Hq / 64;
  const unsigned off = LT_ROW * wave + 16 * (lane ^ lt_key(wave)), rot = lt_rot_off(lane, wave);
  // 32-key tile n of the split: page n / 2, in slot (n + 2) % 4 of the ring
  auto request = [&](int n) {
    if (n < 2 * n_pages) {
      const char* const from = pool + (int64_t)__builtin_amdgcn_readlane(page_of, (n >> 1) - page_base) * LT_PAGE + (n & 1) * LT_TILE;
      const unsigned to = lds0 + ((n + 2) & 3) * LT_TILE + wave * 1024;
      lt_fetch(from, off, rot, to, to + LT_ROT, once);
    }
  };
  // Q by way of LDS, laid out like keys: the tile of each row block in the slot of its number, its 36 KB shared out among the waves that have the block.  (A lane
  // reading its own row from memory takes 16 bytes of a line at a time: 144 such loads a workgroup took 4 us.)
  LtState<NB> st;
  st.start(lane, first_block);
  {
    constexpr int MINE = 9 * RB;  // KB to a wave
    const int first_kb = MINE * (RB == 4 ? 0 : RB == 2 ? wave >> 1 : wave);
    const bf16_t* const q = static_cast<const bf16_t*>(a.q.p) + (it.n0 + i) * a.q.row + h * a.q.head;
    const bf16_t* const r = static_cast<const bf16_t*>(a.q_rope.p) + (it.n0 + i) * a.q_rope.row + h * a.q_rope.head;
    const unsigned to = lds0 + rb * LT_TILE;
#pragma unroll 3
    for (int x = first_kb; x < first_kb + MINE; ++x) {
      if (x < 32) {
        const uint64_t from = (uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(uintptr_t)q, x) |
                              (uint64_t)(unsigned)__builtin_amdgcn_readlane((int)((uintptr_t)q >> 32), x) << 32;
        lt_fetch_row(reinterpret_cast<const char*>(from), 16 * (lane ^ (int)lt_key(x)), to + 1024 * x);
      } else {
        const int row8 = 8 * (x - 32) + (lane >> 3);
        const int64_t from = __shfl((int64_t)(uintptr_t)r, row8);
        lt_fetch_one(reinterpret_cast<const char*>(from) + 16 * ((lane & 7) ^ ((row8 >> 1) & 7)), to + 1024 * x);
      }
    }
  }
  if constexpr (RB == 4) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  } else {
    request(0);
    request(1);
    if (n_pages > 0) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(2 * LT_LOADS) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
  }
  {
    auto key = st.keys(lds, rb * LT_TILE);
#pragma unroll
    for (int n = 0; n < LT_NK; ++n) st.q[st.step(n)] = key(n);
  }
  lt_meet();  // (the ring is free, or its first half)
  int up[LT_MAX_TREE / LT_THREADS];
  auto tree_there = [&]() {
    if (tid < 2) mem.odd[tid] = 0u;
#pragma unroll
    for (int x = 0; x < LT_MAX_TREE / LT_THREADS; ++x) mem.parent[x * LT_THREADS + tid] = up[x];
    lt_meet();
    mend_tree(top_tree);  // (the parents were requested behind the tree's rows, and are there)
  };
  if (last) {
    tree_rows(top_tree);
#pragma unroll
    for (int x = 0; x < LT_MAX_TREE / LT_THREADS; ++x) up[x] = a.parent[it.n0 + std::min(x * LT_THREADS + tid, it.M - 1)];
    if constexpr (RB < 4) tree_there();  // (in one branch with the loads: to the compiler they are on their way behind any other, and it waits for all in the page loop)
  }
  if constexpr (RB == 4) {
    request(0);
    request(1);
    if (last) tree_there();
  }
  const float c2 = g.c2;
  float reference = LT_FLOOR;
#pragma unroll 1
  for (bool first = true;; first = false) {
  st.clear(reference);

  // ---- the tree's own rows, from the last 64 that a row of the group sees down to the first, in the ring's first half
  if (last) {
    int cursor = i;  // the next row of the lane's root path
#pragma unroll 1
    for (int t = top_tree; t >= 0; --t) {
      if (!first || t < top_tree) {
        lt_meet();  // (the buffer's last readers are done)
        if (tid < 2) mem.odd[tid] = 0u;
        lt_meet();
        tree_rows(t);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        mend_tree(t);
      }
      lt_meet();
#pragma unroll 1
      for (int b = 1; b >= 0; --b) {
        unsigned word = 0u;  // the rows of these 32 that the lane's row sees
        const int base = 64 * t + 32 * b;
        while (cursor >= base) {
          word |= 1u << (cursor & 31);
          const int to = mem.parent[cursor];
          cursor = to < cursor ? to : -1;  // (a malformed tree cannot keep the walk from ending)
        }
        if (RB != 4 && b != kh) continue;
        if (__ballot(word != 0u) == 0ull) continue;
        const unsigned odd = mem.odd[b];
        lt_floatx16 S = st.scores(lds, b * LT_TILE);
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int k = 8 * (v >> 2) + 4 * half + (v & 3);
          S[v] = (word >> k) & 1u ? ((odd >> k) & 1u ? __builtin_nanf("") : S[v]) : -HS_INF;
        }
        st.take(lds, b * LT_TILE, S, c2);
      }
    }
    lt_meet();  // (the ring's first half is free)
  }
  // ---- full pages
  unsigned here = 2 * LT_TILE;  // where the page is in the ring
  if constexpr (RB == 4) {
    // three tiles are in the ring or on their way besides the one whose values are multiplied
    request(2);
    if (n_full > 0) {
      if (n_pages > 1) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(2 * LT_LOADS) : "memory");
      else asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(LT_LOADS) : "memory");
      lt_floatx16 S = st.scores(lds, here), N;
      uint4 P0, P1;
      // (two tiles a trip: the scores of one and of the next change places without a copy)
      for (int p = 0; p + 1 < n_full; ++p) {
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(LT_LOADS) : "memory");  // tile 2 p + 1 is there, 2 p + 2 on its way
        request(2 * p + 3);
        st.ahead(lds, here + LT_TILE, S, N, c2, P0, P1);
        st.product(lds, here, P0, P1);
        if (p + 2 - page_base >= 64) look_up(p + 2);
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(LT_LOADS) : "memory");
        request(2 * p + 4);
        st.ahead(lds, 2 * LT_TILE - here, N, S, c2, P0, P1);
        st.product(lds, here + LT_TILE, P0, P1);
        here = 2 * LT_TILE - here;
      }
      if (rest > 0) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(LT_LOADS) : "memory");
      else asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
      request(2 * n_full + 1);
      st.ahead(lds, here + LT_TILE, S, N, c2, P0, P1);
      st.product(lds, here, P0, P1);
      st.take(lds, here + LT_TILE, N, c2);
      here = 2 * LT_TILE - here;
    }
  } else {
    // each wave has one 32-key half of a page
    request(2);
    request(3);
    for (int n = 0; n < n_full; ++n) {
      if (n + 1 < n_pages) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(2 * LT_LOADS) : "memory");
      else asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
      const unsigned tile = here + kh * LT_TILE;
      const lt_floatx16 S = st.scores(lds, tile);
      st.take(lds, tile, S, c2);
      if (n + 2 - page_base >= 64) look_up(n + 2);
      lt_meet();  // every wave is done with the page
      request(2 * n + 4);
      request(2 * n + 5);
      here = 2 * LT_TILE - here;
    }
  }
  // ---- the page that ends inside
  if (rest > 0) {
    asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    lt_blank(lds + here, rest);
    lt_meet();
#pragma unroll 1
    for (int b = 0; b < 2; ++b) {
      if (RB != 4 && b != kh) continue;
      if (32 * b >= rest) continue;
      lt_floatx16 S = st.scores(lds, here + b * LT_TILE);
#pragma unroll
      for (int v = 0; v < 16; ++v) S[v] = 32 * b + 8 * (v >> 2) + 4 * half + (v & 3) < rest ? S[v] : -HS_INF;
      st.take(lds, here + b * LT_TILE, S, c2);
    }
  }
  // ---- a row whose scores rose too far above its reference?
  if (tid == 0) mem.again = 0;
  lt_meet();
  if (__ballot(st.rose(c2)) != 0ull && lane == 0) mem.again = 1;
  lt_meet();
  if (mem.again == 0) break;
  reference = st.seen;
  look_up(0);
  request(0);
  request(1);
  }

  // ---- out: the halves of the keys meet, then rows leave by way of LDS
  lt_meet();
  float total = lt_half_sum(st.l), top = st.m;
  constexpr int KEEP = RB == 4 ? NB : NB / 2;  // blocks that the wave writes
  int out_block = first_block;
  if constexpr (RB != 4) {
    const int other = wave ^ 2;
    if (half == 0) {
      mem.stat[wave][0][col] = top;
      mem.stat[wave][1][col] = total;
    }
    lt_meet();
    const float m2 = mem.stat[other][0][col], l2 = mem.stat[other][1][col];
    const float own = top;
    top = fmaxf(own, m2);
    const float mine = exp2_fast((own - top) * c2), theirs = exp2_fast((m2 - top) * c2);
    total = total * mine + l2 * theirs;
    float4* const to = reinterpret_cast<float4*>(lds) + wave * (KEEP * 4 * 64) + lane;
    const float4* const from = reinterpret_cast<const float4*>(lds) + other * (KEEP * 4 * 64) + lane;
#pragma unroll
    for (int t = 0; t < KEEP; ++t)
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const lt_floatx16 &lo = st.acc[t], &hi = st.acc[KEEP + t];
        to[(t * 4 + b) * 64] = kh == 0 ? make_float4(hi[4 * b] * mine, hi[4 * b + 1] * mine, hi[4 * b + 2] * mine, hi[4 * b + 3] * mine)
                                       : make_float4(lo[4 * b] * mine, lo[4 * b + 1] * mine, lo[4 * b + 2] * mine, lo[4 * b + 3] * mine);
      }
    lt_meet();
#pragma unroll
    for (int t = 0; t < KEEP; ++t)
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const float4 f = from[(t * 4 + b) * 64];
        const float add[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) st.acc[t][4 * b + e] = (kh == 0 ? st.acc[t][4 * b + e] : st.acc[KEEP + t][4 * b + e]) * mine + add[e];
      }
    out_block += kh * KEEP;
    lt_meet();
  }
  const int mine_rows = std::min(32, rows - row_base);
  if (mine_rows <= 0) return;
  const bool writes_stat = half == 0 && col < mine_rows && out_block == 0;
  char* const stage = lds + wave * 32 * LT_OUT_PITCH;
  const int64_t row0 = (int64_t)it.n0 * a.Hq + row_base, rec0 = it.rec0 + (int64_t)row_base * it.n_sp + it.sp;  // (records: row, then split)
  if (it.n_sp == 1) {
    const float inv = 1.f / total;
    if (writes_stat && a.lse != nullptr) a.lse[row0 + col] = top * a.scale + __log2f(total) * LT_LN2;
#pragma unroll
    for (int t = 0; t < KEEP; ++t)
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const lt_floatx2 x = {st.acc[t][4 * b] * inv, st.acc[t][4 * b + 1] * inv}, y = {st.acc[t][4 * b + 2] * inv, st.acc[t][4 * b + 3] * inv};
        *reinterpret_cast<uint2*>(stage + col * LT_OUT_PITCH + 64 * t + 16 * b + 8 * half) =
            make_uint2(__builtin_bit_cast(unsigned, __builtin_convertvector(x, lt_bf16x2)), __builtin_bit_cast(unsigned, __builtin_convertvector(y, lt_bf16x2)));
      }
    if (half == 0) mem.out_at[wave][col] = (it.n0 + i) * a.o_row + h * a.o_head;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    constexpr int PER_ROW = KEEP * 4;  // 16-byte pieces
#pragma unroll 4
    for (int x = lane; x < mine_rows * PER_ROW; x += 64) {
      const int r = x / PER_ROW, c = x % PER_ROW;
      *reinterpret_cast<uint4*>(static_cast<bf16_t*>(a.o) + mem.out_at[wave][r] + 32 * out_block + 8 * c) =
          *reinterpret_cast<const uint4*>(stage + r * LT_OUT_PITCH + 16 * c);
    }
  } else {
    if (writes_stat) {
      float* const rec = g.part + (rec0 + col * it.n_sp) * LT_REC;
      rec[LT_R] = top;
      rec[LT_R + 1] = total;
    }
    constexpr int PASS = KEEP < 8 ? KEEP : 8;  // blocks that a row on its way out has room for
#pragma unroll
    for (int x0 = 0; x0 < KEEP; x0 += PASS) {
#pragma unroll
      for (int t = 0; t < PASS; ++t)
#pragma unroll
        for (int b = 0; b < 4; ++b)
          *reinterpret_cast<float4*>(stage + col * LT_OUT_PITCH + 128 * t + 32 * b + 16 * half) =
              make_float4(st.acc[x0 + t][4 * b], st.acc[x0 + t][4 * b + 1], st.acc[x0 + t][4 * b + 2], st.acc[x0 + t][4 * b + 3]);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      constexpr int PER_ROW = PASS * 8;
#pragma unroll 4
      for (int x = lane; x < mine_rows * PER_ROW; x += 64) {
        const int r = x / PER_ROW, c = x % PER_ROW;
        *reinterpret_cast<float4*>(g.part + (rec0 + r * it.n_sp) * LT_REC + 32 * (out_block + x0) + 4 * c) =
            *reinterpret_cast<const float4*>(stage + r * LT_OUT_PITCH + 16 * c);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  }
}

// MOST: row blocks of an item at most.  (A kernel of its own for each: of groups of 32 rows a third of the code is fetched, and there is no scratch memory to set
// up: one token of 16 heads on 2048 18.5 -> 17.3 us, 64 sequences 66.6 -> 64.9 us.)
template <int MOST>
__global__ __launch_bounds__(LT_THREADS, 1) void k_lat_tree(LtArgs g) {
  __shared__ LtLds mem;
  LtItem it;
  if (!lt_find(g, it, mem)) return;
  const int left = std::min(g.group, it.M * g.a.Hq - it.rg * g.group);
  if constexpr (MOST == 4) {
    if (left > 64) return lt_run<4>(g, it, mem);
  }
  if constexpr (MOST >= 2) {
    if (left > 32) return lt_run<2>(g, it, mem);
  }
  lt_run<1>(g, it, mem);
}

// The merge of the splits: SHARE waves to a row, which take its records in turn, four at a time each.
constexpr int LTM_THREADS = 256;
template <int SHARE>
__global__ __launch_bounds__(LTM_THREADS) void k_lat_tree_merge(LtArgs g) {
  __shared__ float sums[SHARE > 1 ? SHARE : 1][64][10];
  const LatTreeArgs& a = g.a;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), way = wave % SHARE;
  const int64_t row = (int64_t)blockIdx.x * (LTM_THREADS / 64 / SHARE) + wave / SHARE;
  if (row >= (int64_t)a.NN * a.Hq) return;  // (SHARE > 1: the same for the workgroup)
  const int n = (int)((unsigned)row / (unsigned)a.Hq), h = (int)row - n * a.Hq;
  // the row's sequence, and its first record
  int M = 0, n_sp = 0, n0 = 0, rec0 = 0;
  if (a.B == 1) M = g.one_rows, n_sp = lt_splits((g.one_len + 63) >> 6, g.per);
  for (int base = 0; base < a.B && a.B > 1; base += 64) {
    int own_n0 = 0, own_M = 0, own_sp = 0;
    int64_t L;
    const bool there = base + lane < a.B;
    if (there) lt_sequence(g, base + lane, &own_n0, &own_M, &L, &own_sp);
    const unsigned long long mine = __ballot(there && own_n0 <= n && n < own_n0 + own_M);
    const int recs = lt_records(own_M, a.Hq, own_sp), upto = wave_prefix_sum(recs);
    if (mine != 0ull) {
      const int who = __builtin_ctzll(mine);
      M = __builtin_amdgcn_readlane(own_M, who);
      n_sp = __builtin_amdgcn_readlane(own_sp, who);
      n0 = __builtin_amdgcn_readlane(own_n0, who);
      rec0 += __builtin_amdgcn_readlane(upto - recs, who);
      break;
    }
    rec0 += __builtin_amdgcn_readlane(upto, 63);
  }
  if (n_sp <= 1 || rec0 + lt_records(M, a.Hq, n_sp) > g.records) return;
  const float* const rec = g.part + (rec0 + ((int64_t)(n - n0) * a.Hq + h) * n_sp) * LT_REC;
  float m = LT_FLOOR, total = 0.f;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int x0 = way; x0 < n_sp; x0 += 4 * SHARE) {
    float rm[4], rl[4];
    float4 v[4][2];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float* const r = rec + (int64_t)std::min(x0 + x * SHARE, n_sp - 1) * LT_REC;
      rm[x] = r[LT_R];
      rl[x] = r[LT_R + 1];
      v[x][0] = *reinterpret_cast<const float4*>(r + 8 * lane);
      v[x][1] = *reinterpret_cast<const float4*>(r + 8 * lane + 4);
    }
    const float up = fmaxf(fmaxf(m, fmaxf(rm[0], rm[1])), fmaxf(rm[2], rm[3])), old = exp2_fast((m - up) * g.c2);  // (records that stand for no split repeat the last)
    total *= old;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] *= old;
    m = up;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      if (x0 + x * SHARE >= n_sp) break;
      const float w = exp2_fast((rm[x] - m) * g.c2);
      const float f[8] = {v[x][0].x, v[x][0].y, v[x][0].z, v[x][0].w, v[x][1].x, v[x][1].y, v[x][1].z, v[x][1].w};
      total = __builtin_fmaf(w, rl[x], total);
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = __builtin_fmaf(w, f[e], acc[e]);
    }
  }
  if constexpr (SHARE > 1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[way][lane][e] = acc[e];
    sums[way][lane][8] = m;
    sums[way][lane][9] = total;
    __syncthreads();
    if (way != 0) return;
    float up = m;
#pragma unroll
    for (int w = 1; w < SHARE; ++w) up = fmaxf(up, sums[w][lane][8]);
    const float own = exp2_fast((m - up) * g.c2);
    total *= own;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] *= own;
#pragma unroll
    for (int w = 1; w < SHARE; ++w) {
      const float f = exp2_fast((sums[w][lane][8] - up) * g.c2);
      total = __builtin_fmaf(f, sums[w][lane][9], total);
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = __builtin_fmaf(f, sums[w][lane][e], acc[e]);
    }
    m = up;
  }
  const float inv = 1.f / total;
  unsigned w[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) w[x] = __builtin_bit_cast(unsigned, __builtin_convertvector((lt_floatx2{acc[2 * x] * inv, acc[2 * x + 1] * inv}), lt_bf16x2));
  *reinterpret_cast<uint4*>(static_cast<bf16_t*>(a.o) + n * a.o_row + h * a.o_head + 8 * lane) = make_uint4(w[0], w[1], w[2], w[3]);
  if (lane == 0 && a.lse != nullptr) a.lse[row] = m * a.scale + __log2f(total) * LT_LN2;
}

// ------------------------------------------------------------------------------------------------ the host's part
bool lat_tree_matrix(const LatTreeArgs& a, hs_dtype dt) {
  auto fits = [](const void* p, int64_t s, int64_t t) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && s % 8 == 0 && t % 8 == 0; };
  return dt == HS_BF16 && a.R == LT_R && a.Dr == LT_DR && fits(a.q.p, a.q.row, a.q.head) && fits(a.q_rope.p, a.q_rope.row, a.q_rope.head) &&
         fits(a.pool, 0, 0) && fits(a.c_tree, a.c_stride, 0) && fits(a.r_tree, a.r_stride, 0) && fits(a.o, a.o_row, a.o_head);
}

// Pages of a split, by estimated times.  (Constants fitted to calls with the group size forced: 100 rows of 16 heads on 8414 tokens 128 rows 56 to 58 us, 64 rows 69, 32 rows 129; 50 rows
// of 20 heads on 102 tokens 24, 21 and 18.)
LatPlan lat_tree_plan(const int32_t* no, const int64_t* pl, int32_t B, int32_t Hq) {
  int64_t longest = 1, widest = 0;
  for (int s = 0; s < B; ++s)
    if (no[s + 1] > no[s]) longest = std::max(longest, (pl[s] + 63) >> 6), widest = std::max(widest, (int64_t)(no[s + 1] - no[s]) * Hq);
  constexpr double CU = 256.0, REC = 0.0006, SPLIT = 0.1;  // compute units; us a row's record (all together), and a split in the merge
  // us of an item without pages, and of a page: by what the waves do with one, or by its share of what is read at a time (pages that several groups share come from
  // the second-level cache, no faster: 250 items' pages on their way are more than it holds)
  auto block = [](int64_t rows, int group) { return std::min<int64_t>(rows, group) > 64 ? 2 : std::min<int64_t>(rows, group) > 32 ? 1 : 0; };
  constexpr double FIXED[3] = {10.0, 11.0, 15.0}, PAGE[3] = {1.3, 2.0, 3.0}, ONCE = 0.0094, SHARED = 0.0129;
  auto item_us = [&](int64_t rows, int group, double pages, double busy) {
    const int k = block(rows, group);
    return FIXED[k] + pages * std::max(PAGE[k], busy * (rows <= group ? ONCE : SHARED));
  };
  LatPlan best = {};
  best.sp_max = 1;
  double best_us = 0.0, best_busy = CU;
  auto consider = [&](int64_t per, int group) {
    int64_t items = 0, sp_max = 1, records = 0;
    for (int s = 0; s < B; ++s) {
      const int64_t rows = (int64_t)(no[s + 1] - no[s]) * Hq, n_sp = lt_splits((pl[s] + 63) >> 6, (int)per);
      if (rows == 0) continue;
      items += n_sp * ((rows + group - 1) / group);
      sp_max = std::max(sp_max, n_sp);
      if (n_sp > 1) records += rows * n_sp;
    }
    const double busy = std::min(CU, (double)items);
    double sum = 0.0, most = 0.0;
    for (int s = 0; s < B; ++s) {
      const int64_t rows = (int64_t)(no[s + 1] - no[s]) * Hq, pages = (pl[s] + 63) >> 6, n_sp = lt_splits(pages, (int)per);
      if (rows == 0) continue;
      const double item = item_us(rows, group, (double)pages / (double)n_sp, busy);
      sum += item * (double)(n_sp * ((rows + group - 1) / group));
      most = std::max(most, item);
    }
    double us = (double)items <= CU ? most : std::max(most, sum / CU + 0.5 * most);
    if (sp_max > 1) us += 4.0 + REC * (double)records + SPLIT * (double)sp_max;
    if (best.per == 0 || (us < best_us && records <= LAT_MAX_RECORDS))
      best_us = us, best_busy = busy, best.per = (int)per, best.sp_max = (int)sp_max, best.group = group, best.records = records;
    return items;
  };
  for (int group : {LT_GROUP, LT_GROUP / 2, LT_GROUP / 4}) {
    if (group > LT_GROUP / 4 && widest <= group / 2) continue;  // (no group has so many rows)
    const int64_t whole = consider(longest, group);
    const bool few = whole <= 128;
    // the finest cuts whose items fill the compute units once, one and a half times, ..., and those of the longest sequences among very many
    for (int64_t target : {(int64_t)32, (int64_t)64, (int64_t)128, (int64_t)192, (int64_t)256, (int64_t)512, (int64_t)1024, whole + 256}) {
      if (target <= whole) continue;
      int64_t lo = 1, hi = longest;  // items(hi) <= target, or hi is the coarsest
      while (lo < hi) {
        const int64_t mid = (lo + hi) / 2;
        if (consider(mid, group) <= target) hi = mid;
        else lo = mid + 1;
      }
      if (lo == 1) break;
    }
    if (!few) break;  // smaller groups are for calls of few items
  }
  // runs of items for the XCDs: equal numbers while each has a compute unit, equal times otherwise
  auto items_of = [&](int s, double* cost) {
    const int64_t rows = (int64_t)(no[s + 1] - no[s]) * Hq;
    if (rows == 0) return (int64_t)0;
    const int64_t pages = (pl[s] + 63) >> 6, n_sp = lt_splits(pages, best.per);
    *cost = item_us(rows, best.group, (double)pages / (double)n_sp, best_busy);
    return n_sp * ((rows + best.group - 1) / best.group);
  };
  int64_t items = 0;
  double sum = 0.0, cost = 0.0;
  for (int s = 0; s < B; ++s) {
    const int64_t n = items_of(s, &cost);
    items += n;
    sum += cost * (double)n;
  }
  for (int x = 0; x <= LT_XCD; ++x) best.first[x] = items * x / LT_XCD;
  if (items > (int64_t)CU) {
    int64_t before = 0;
    double spent = 0.0;
    int x = 1;
    for (int s = 0; s < B; ++s) {
      const int64_t n = items_of(s, &cost);
      for (; x < LT_XCD && n > 0 && spent + cost * (double)n >= sum * x / LT_XCD; ++x)
        best.first[x] = before + std::min(n, (int64_t)((sum * x / LT_XCD - spent) / cost + 0.5));
      before += n;
      spent += cost * (double)n;
    }
    for (; x < LT_XCD; ++x) best.first[x] = items;
  }
  int64_t most = 0;
  for (int x = 0; x < LT_XCD; ++x) most = std::max(most, best.first[x + 1] - best.first[x]);
  best.grid = LT_XCD * most;
  return best;
}

size_t lat_tree_bytes(const LatPlan& p) { return align_up((size_t)p.records * LT_REC * 4, 256); }

hs_status lat_tree_launch(const LatTreeArgs& a, const LatPlan& p, int one_len, void* workspace, hipStream_t stream) {
  LtArgs g = {a, a.scale * LT_LOG2E, p.per, p.sp_max, p.group, static_cast<float*>(workspace), a.NN, one_len, (int)p.records, {}};
  for (int x = 0; x <= LT_XCD; ++x) g.first[x] = (int)p.first[x];
  if (p.group > 64) hipLaunchKernelGGL(k_lat_tree<4>, dim3((unsigned)p.grid), dim3(LT_THREADS), 0, stream, g);
  else if (p.group > 32) hipLaunchKernelGGL(k_lat_tree<2>, dim3((unsigned)p.grid), dim3(LT_THREADS), 0, stream, g);
  else hipLaunchKernelGGL(k_lat_tree<1>, dim3((unsigned)p.grid), dim3(LT_THREADS), 0, stream, g);
  const hs_status st = launch_status("latent attention");
  if (st != HS_OK || p.sp_max == 1) return st;
  const int64_t rows = (int64_t)a.NN * a.Hq;
  if (p.sp_max > 4) hipLaunchKernelGGL(k_lat_tree_merge<4>, dim3((unsigned)rows), dim3(LTM_THREADS), 0, stream, g);
  else hipLaunchKernelGGL(k_lat_tree_merge<1>, dim3((unsigned)((rows + 3) / 4)), dim3(LTM_THREADS), 0, stream, g);
  return launch_status("latent attention, merge");
}

}  // namespace hs
