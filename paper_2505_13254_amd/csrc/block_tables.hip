// hs_block_tables, hs_slot_map: which pages a sequence has, and where in the pool its rows go.
//
// A few bytes a sequence, a page's number an entry that changes hands and 8 bytes a row: bound by the launch and by chains of
// trips to memory, not by bandwidth, up to some 10^5 entries: tables 3.4 us for 16 sequences, 4.5 for 512; slots 4 us for 1000 rows, 12 for 1.5 million.
//
// hs_block_tables.  Free pages are a stack.  With F pages on it, R pages going back in this call and, in the order of
// sequences, released page t at place F + t, the k-th page taken is entry F + R - 1 - k of that row of pages.  Entries below F are
// read from the stack, those above it straight from the table rows of the sequences that give them back (which the call does
// not write), and what stays on the stack is written at places F .. only.  So no entry that one thread reads is written by
// another, and one launch does without any order between its workgroups.
// Every workgroup sums the sequences' releases and requests up by itself: a thread takes a run of neighbouring sequences, the
// runs' prefix sums stand in LDS, and any entry finds its sequence by a binary search over the runs and a walk through one of them (one
// sequence, up to 1024 of them).  Handing the sums from a first launch to a second would cost the second launch's 4 us.
#include "attn_common.h"

namespace hs {

constexpr int BT_THREADS = 1024;
constexpr int BT_ENTRIES = 4;  // table entries to a thread that the grid is sized for
constexpr int BT_GRID = 256;   // workgroups at most: each reads all sequences' lengths

struct BtArgs {
  const int64_t* want;
  int page_tokens, max_blocks, n_pages, B, per;  // per: sequences to a thread
  int32_t* table;
  const int32_t* held;
  int32_t* new_held;
  int32_t* free_pages;
  const int32_t* free_count;
  int32_t* new_free_count;
  int32_t* refused;
};

// Pages that sequence s has (within the table), and those that it is to have; `beyond`: more than a row of the table holds.
__device__ __forceinline__ void bt_of(const BtArgs& a, int s, int* held, int* need, bool* beyond) {
  const int h = a.held[s];
  const int64_t w = a.want[s];
  *held = h < 0 ? 0 : (h > a.max_blocks ? a.max_blocks : h);
  const int64_t n = w <= 0 ? 0 : (w - 1) / a.page_tokens + 1;
  *beyond = n > a.max_blocks;
  *need = *beyond ? *held : (int)n;
}

// Inclusive prefix sums of two numbers a thread over the workgroup.
__device__ __forceinline__ void bt_scan(int& x, int& y, int (*waves)[2]) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  x = wave_prefix_sum(x);
  y = wave_prefix_sum(y);
  if (lane == 63) waves[wave][0] = x, waves[wave][1] = y;
  __syncthreads();
  int u = lane < wave ? waves[lane][0] : 0, v = lane < wave ? waves[lane][1] : 0;  // (sixteen waves at most)
  u = wave_prefix_sum(u);
  v = wave_prefix_sum(v);
  x += __builtin_amdgcn_readlane(u, 63);
  y += __builtin_amdgcn_readlane(v, 63);
}

// The last place of sums [0, n) (rising, sums[0] = 0) that does not exceed t.
__device__ __forceinline__ int bt_find(const int* sums, int n, int t) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (sums[mid] <= t) lo = mid;
    else hi = mid;
  }
  return lo;
}

__global__ __launch_bounds__(BT_THREADS) void k_block_tables(BtArgs a) {
  __shared__ int ask_to[BT_THREADS], back_to[BT_THREADS], waves[BT_THREADS / 64][2], all[2];
  const int tid = threadIdx.x;
  int F = a.free_count[0];
  F = F < 0 ? 0 : (F > a.n_pages ? a.n_pages : F);
  int ask = 0, back = 0;
  const int first = tid * a.per, end = first + a.per < a.B ? first + a.per : a.B;
  for (int s = first; s < end; ++s) {
    int held, need;
    bool beyond;
    bt_of(a, s, &held, &need, &beyond);
    if (need > held) ask += need - held;
    else back += held - need;
  }
  const int mine_ask = ask, mine_back = back;
  bt_scan(ask, back, waves);
  ask_to[tid] = ask - mine_ask;
  back_to[tid] = back - mine_back;
  if (tid == BT_THREADS - 1) all[0] = ask, all[1] = back;
  __syncthreads();
  const int asked = all[0], R = all[1], total = F + R;
  // pages given: the requests in front of the first that does not fit
  int given = asked;
  if (asked > total) {
    const int run = bt_find(ask_to, BT_THREADS, total);
    given = ask_to[run];
    for (int s = run * a.per; s < a.B && s < (run + 1) * a.per; ++s) {
      int held, need;
      bool beyond;
      bt_of(a, s, &held, &need, &beyond);
      const int more = need > held ? need - held : 0;
      if (given + more > total) break;
      given += more;
    }
  }
  // the released page t: of which sequence, and at which place in its row
  auto released = [&](int t) {
    const int run = bt_find(back_to, BT_THREADS, t);
    int before = back_to[run];
    for (int s = run * a.per; s < a.B && s < (run + 1) * a.per; ++s) {
      int held, need;
      bool beyond;
      bt_of(a, s, &held, &need, &beyond);
      const int n = held > need ? held - need : 0;
      if (t < before + n) return a.table[(int64_t)s * a.max_blocks + need + (t - before)];
      before += n;
    }
    return -1;
  };
  const int stride = (int)gridDim.x * BT_THREADS, id = (int)blockIdx.x * BT_THREADS + tid;
  for (int64_t k = id; k < given; k += stride) {  // pages that come
    const int run = bt_find(ask_to, BT_THREADS, (int)k);
    int before = ask_to[run];
    for (int s = run * a.per; s < a.B && s < (run + 1) * a.per; ++s) {
      int held, need;
      bool beyond;
      bt_of(a, s, &held, &need, &beyond);
      const int n = need > held ? need - held : 0;
      if (k < before + n) {
        const int from = total - 1 - (int)k;
        a.table[(int64_t)s * a.max_blocks + held + ((int)k - before)] = from < F ? a.free_pages[from] : released(from - F);
        break;
      }
      before += n;
    }
  }
  for (int64_t t = id; t < total - given - F && F + t < a.n_pages; t += stride)  // pages that go and are not taken again
    a.free_pages[F + t] = released((int)t);
  for (int64_t s64 = id; s64 < a.B; s64 += stride) {
    const int s = (int)s64, run = s / a.per;
    int upto = ask_to[run], held = 0, need = 0;
    bool beyond = false;
    for (int x = run * a.per; x <= s; ++x) {
      bt_of(a, x, &held, &need, &beyond);
      upto += need > held ? need - held : 0;
    }
    const bool short_of = need > held && upto > total;
    a.new_held[s] = short_of ? held : need;
    if (a.refused != nullptr) a.refused[s] = beyond ? 2 : (short_of ? 1 : 0);
  }
  if (id == 0) a.new_free_count[0] = total - given;
}

// ------------------------------------------------------------------------------------------------ slots of rows
// A thread takes four neighbouring rows (of accepted paths one, which is scanned), finds the sequence of the first by a binary search and walks on from there; first rows, lengths and page counts of the
// sequences stand in LDS where they fit, so that a row waits for two trips to memory, these and its page's number (and the path of an accepted row).  (A
// search a row: 1.5 million rows of 512 sequences 14.8 us.)
constexpr int SM_THREADS = 256, SM_LDS = 1024;
constexpr int SM_GRID = 1024;  // workgroups at most: beyond that each takes several runs of rows, and reads the sequences once

struct SmArgs {
  const int32_t* node_offsets;
  int NN;
  const int32_t* accept_path;  // NULL: every row
  const int32_t* accept_len;
  int max_depth;
  const int32_t* table;
  int max_blocks, page_tokens, n_pages, B;
  const int32_t* held;
  const int64_t* cache_lens;
  int64_t* slots;
  int64_t* new_lens;
};
struct SmLds {
  int off[SM_LDS + 1], held[SM_LDS], accepted[SM_LDS];
  int64_t len[SM_LDS];
};

__device__ __forceinline__ int sm_accepted(const SmArgs& a, int n) { return n < 0 ? 0 : (n < a.max_depth ? n : a.max_depth); }
__device__ __forceinline__ int64_t sm_room(const SmArgs& a, int held) {  // tokens that a sequence's pages hold
  return (int64_t)(held < 0 ? 0 : (held > a.max_blocks ? a.max_blocks : held)) * a.page_tokens;
}

template <bool PATH>
constexpr int SM_ROWS = PATH ? 1 : 4;
template <bool PATH>
__global__ __launch_bounds__(SM_THREADS) void k_slot_map(SmArgs a) {
  constexpr int ROWS = SM_ROWS<PATH>;
  __shared__ SmLds mem;
  const int tid = threadIdx.x;
  const bool small = a.B <= SM_LDS;
  if (small) {
    for (int s = tid; s <= a.B; s += SM_THREADS) {
      mem.off[s] = a.node_offsets[s];
      if (s < a.B) {
        mem.len[s] = a.cache_lens[s];
        mem.held[s] = a.held != nullptr ? a.held[s] : a.max_blocks;
        if (PATH) mem.accepted[s] = a.accept_len[s];
      }
    }
    __syncthreads();
  }
  auto off = [&](int s) { return small ? mem.off[s] : a.node_offsets[s]; };
  auto len = [&](int s) { return small ? mem.len[s] : a.cache_lens[s]; };
  auto room = [&](int s) { return sm_room(a, small ? mem.held[s] : a.held != nullptr ? a.held[s] : a.max_blocks); };
  auto accepted = [&](int s) { return sm_accepted(a, small ? mem.accepted[s] : a.accept_len[s]); };
  const int last = off(a.B);
  const bool wide = reinterpret_cast<uintptr_t>(a.slots) % 16 == 0;
  for (int64_t first = ((int64_t)blockIdx.x * SM_THREADS + tid) * ROWS; first < a.NN; first += (int64_t)gridDim.x * SM_THREADS * ROWS) {
    int64_t slot[ROWS];
    int s = 0, end = 0;
    if (first < last) {
      int hi = a.B;  // the last sequence that begins at or before the row
      while (hi - s > 1) {
        const int mid = (s + hi) >> 1;
        if (off(mid) <= first) s = mid;
        else hi = mid;
      }
      end = off(s + 1);
    }
#pragma unroll
    for (int x = 0; x < ROWS; ++x) {
      const int64_t row = first + x;
      slot[x] = -1;
      if (row >= last || row >= a.NN) continue;
      while (row >= end && s + 1 < a.B) end = off(++s + 1);
      const int local = (int)row - off(s);
      int at = local;
      if (PATH && local > 0) {  // the row's place in the accepted path
        const int n = accepted(s);
        const int32_t* const path = a.accept_path + (int64_t)s * a.max_depth;
        at = -1;
        for (int j0 = 0; j0 < n && at < 0; j0 += 8) {
          int p[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) p[j] = path[j0 + j < n ? j0 + j : n - 1];
#pragma unroll
          for (int j = 7; j >= 0; --j) at = j0 + j < n && p[j] == local ? j0 + j + 1 : at;  // (the first place that names the row)
        }
      }
      const int64_t token = len(s) + at;
      if (at < 0 || token < 0 || token >= room(s)) continue;
      const int64_t block = token >> 32 == 0 ? (int64_t)((unsigned)token / (unsigned)a.page_tokens) : token / a.page_tokens;
      const int page = a.table[(int64_t)s * a.max_blocks + block];
      if (page >= 0 && page < a.n_pages) slot[x] = (int64_t)page * a.page_tokens + (token - block * a.page_tokens);
    }
    if (ROWS == 4 && wide && first + 3 < a.NN) {
      reinterpret_cast<longlong2*>(a.slots + first)[0] = make_longlong2(slot[0], slot[1 % ROWS]);
      reinterpret_cast<longlong2*>(a.slots + first)[1] = make_longlong2(slot[2 % ROWS], slot[3 % ROWS]);
      continue;
    }
#pragma unroll
    for (int x = 0; x < ROWS; ++x)
      if (first + x < a.NN) a.slots[first + x] = slot[x];
  }
  if (a.new_lens == nullptr) return;
  for (int64_t i = (int64_t)blockIdx.x * SM_THREADS + tid; i < a.B; i += (int64_t)gridDim.x * SM_THREADS) {
    const int q = (int)i;
    int64_t n = off(q + 1) - off(q);
    if (PATH && n > 0) n = 1 + accepted(q);
    const int64_t l = len(q), most = room(q);
    a.new_lens[q] = l + n <= most ? l + n : (l > most ? l : most);
  }
}

static bool bt_known(const void* p) {  // an address that kernels can use
  hipPointerAttribute_t at = {};
  if (hipPointerGetAttributes(&at, p) != hipSuccess) {
    (void)hipGetLastError();  // (the next launch would report it)
    return false;
  }
  return at.type != hipMemoryTypeUnregistered && at.devicePointer != nullptr;
}

}  // namespace hs

using namespace hs;

extern "C" hs_status hs_block_tables(const int64_t* want, int32_t page_tokens, int32_t* block_table, int32_t max_blocks, const int32_t* held,
                                     int32_t* new_held, int32_t* free_pages, int32_t n_pages, const int32_t* free_count, int32_t* new_free_count,
                                     int32_t* refused, int32_t B, hs_stream stream) {
  clear_error();
  HS_REQUIRE(B >= 0 && page_tokens >= 1 && max_blocks >= 0 && n_pages >= 0, HS_ERR_SHAPE, "hs_block_tables: B=%d page_tokens=%d max_blocks=%d n_pages=%d", B,
             page_tokens, max_blocks, n_pages);
  HS_REQUIRE((int64_t)B * (max_blocks > 0 ? max_blocks : 1) < (int64_t)1 << 30 && n_pages < 1 << 30 && B <= 1 << 20, HS_ERR_UNSUPPORTED,
             "hs_block_tables: B * max_blocks and n_pages must be below 2^30, B at most 2^20");
  HS_REQUIRE(free_count && new_free_count, HS_ERR_NULL, "hs_block_tables: NULL count");
  HS_REQUIRE(B == 0 || (want && held && new_held && (block_table || max_blocks == 0) && (free_pages || n_pages == 0)), HS_ERR_NULL,
             "hs_block_tables: NULL argument");
  auto apart = [&](const void* p, size_t n, const void* q, size_t m) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(p), y = reinterpret_cast<uintptr_t>(q);
    return x + n <= y || y + m <= x;
  };
  HS_REQUIRE(apart(held, 4 * (size_t)B, new_held, 4 * (size_t)B) && apart(free_count, 4, new_free_count, 4), HS_ERR_SHAPE,
             "hs_block_tables: new_held and new_free_count must not overlap held and free_count");
  // Without sequences the count is still handed on.  (Such a call has always succeeded without a GPU and with any addresses, as every call of the library that has
  // nothing to do: counts that the runtime knows nothing of are left alone.)
  if (B == 0 && !(bt_known(free_count) && bt_known(new_free_count))) return HS_OK;
  BtArgs a = {want, page_tokens, max_blocks, n_pages, B, (B + BT_THREADS - 1) / BT_THREADS, block_table, held, new_held, free_pages, free_count, new_free_count, refused};
  int64_t grid = ((int64_t)B * max_blocks + BT_THREADS * BT_ENTRIES - 1) / (BT_THREADS * BT_ENTRIES);
  grid = grid < 1 ? 1 : (grid > BT_GRID ? BT_GRID : grid);
  hipLaunchKernelGGL(k_block_tables, dim3((unsigned)grid), dim3(BT_THREADS), 0, static_cast<hipStream_t>(stream), a);
  return launch_status("block tables");
}

extern "C" hs_status hs_slot_map(const int32_t* node_offsets, int32_t NN, const int32_t* accept_path, const int32_t* accept_len, int32_t max_depth,
                                 const int32_t* block_table, int32_t max_blocks, int32_t page_tokens, int32_t n_pages, const int32_t* held,
                                 const int64_t* cache_lens, int64_t* slots, int64_t* new_lens, int32_t B, hs_stream stream) {
  clear_error();
  HS_REQUIRE(B >= 0 && NN >= 0 && page_tokens >= 1 && max_blocks >= 0 && n_pages >= 0, HS_ERR_SHAPE,
             "hs_slot_map: B=%d NN=%d page_tokens=%d max_blocks=%d n_pages=%d", B, NN, page_tokens, max_blocks, n_pages);
  HS_REQUIRE((accept_path == nullptr) == (accept_len == nullptr) && (accept_path == nullptr || max_depth >= 1), HS_ERR_SHAPE,
             "hs_slot_map: accept_path and accept_len go together, with max_depth >= 1");
  HS_REQUIRE(B > 0 || NN == 0, HS_ERR_SHAPE, "hs_slot_map: rows without sequences");
  if (B == 0) return HS_OK;
  HS_REQUIRE(node_offsets && cache_lens && (slots || NN == 0) && (block_table || max_blocks == 0), HS_ERR_NULL, "hs_slot_map: NULL argument");
  if (new_lens != nullptr) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(cache_lens), y = reinterpret_cast<uintptr_t>(new_lens);
    HS_REQUIRE(x + 8 * (uintptr_t)B <= y || y + 8 * (uintptr_t)B <= x, HS_ERR_SHAPE, "hs_slot_map: new_lens must not overlap cache_lens");
  }
  SmArgs a = {node_offsets, NN, accept_path, accept_len, max_depth, block_table, max_blocks, page_tokens, n_pages, B, held, cache_lens, slots, new_lens};
  const int run = SM_THREADS * (accept_path != nullptr ? SM_ROWS<true> : SM_ROWS<false>);
  const int64_t runs = ((int64_t)NN + run - 1) / run, grid = runs < 1 ? 1 : (runs > SM_GRID ? SM_GRID : runs);
  if (accept_path != nullptr) hipLaunchKernelGGL(k_slot_map<true>, dim3((unsigned)grid), dim3(SM_THREADS), 0, static_cast<hipStream_t>(stream), a);
  else hipLaunchKernelGGL(k_slot_map<false>, dim3((unsigned)grid), dim3(SM_THREADS), 0, static_cast<hipStream_t>(stream), a);
  return launch_status("slot map");
}
