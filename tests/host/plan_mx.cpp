// Host-only driver for the planner of hs_tree_attention_mx (tests/test_attention_mx_plan.py compiles it, which includes the
// planner's source, with AddressSanitizer and UndefinedBehaviorSanitizer on the host side).  Nothing touches a GPU.
//
//   plan_mx fuzz N SEED   plans N random batches and checks what the kernels rely on; "ok ITEMS"
//   plan_mx args N SEED   makes the real call of N random batches on addresses that nothing looks at and checks what its launches are
//                         given: every sequence of the host arrays, and no address of the device's; "ok LAUNCHES"
//   plan_mx form          reads "FMT Hq Hkv D B rows... lens..." lines and prints, for every sequence with rows,
//                         "form blocks groups splits pages" (form: 0, 1 private, 2, 3 shared), a line to a batch
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "tree_attention_mx.hip"

extern "C" hipError_t hipGetLastError() { return hipSuccess; }  // (the launches are stubs)

static std::vector<std::pair<hs::MxAttnArgs, unsigned>> launched;
namespace hs {
void attn_mx_launch_e4m3(const MxAttnArgs& a, unsigned items, hipStream_t) { launched.emplace_back(a, items); }
void attn_mx_launch_e2m1(const MxAttnArgs& a, unsigned items, hipStream_t) { launched.emplace_back(a, items); }
}  // namespace hs

static unsigned long long state = 88172645463325252ull;
static unsigned rnd() {
  state ^= state << 13, state ^= state >> 7, state ^= state << 17;
  return (unsigned)(state >> 11);
}
#define CHECK(x)                                                    \
  do {                                                              \
    if (!(x)) {                                                     \
      std::printf("line %d: %s (batch %ld)\n", __LINE__, #x, batch); \
      std::exit(1);                                                 \
    }                                                               \
  } while (0)
static long batch = 0;

// x / d as the device computes it, by a reciprocal that may be off by `ulps` units in the last place.
static int div_by_product(int x, int d, int ulps) {
  float r = 1.0f / (float)d;
  for (int i = 0; i < std::abs(ulps); ++i) r = std::nextafter(r, ulps > 0 ? 2.0f : 0.0f);
  int q = (int)((float)x * r);
  const int rest = x - q * d;
  q += rest < 0 ? -1 : rest >= d ? 1 : 0;
  return q;
}

struct Batch {
  std::vector<int32_t> no;
  std::vector<int64_t> lens;
  int Hq, Hkv, D, fmt;
};

// The cut of one sequence: every row block and every page in exactly one item, no split without keys, as many splits as the merge takes.
static void check_cut(const hs::MxCut& c, int M, int G, int L) {
  CHECK(c.n_blk == (G * M + 31) / 32 && c.n_rg >= 1 && c.n_rg <= c.n_blk && c.n_blk < (1 << 16) && c.n_rg < (1 << 16));
  const int each = c.n_blk / c.n_rg, more = c.n_blk - each * c.n_rg, largest = each + (more > 0 ? 1 : 0);
  CHECK(largest <= 8 && each >= 1);
  CHECK(c.form == (largest > 4 ? hs::MX_SHARED_8 : largest > 2 ? hs::MX_SHARED_4 : largest > 1 ? hs::MX_PRIVATE_2 : hs::MX_PRIVATE_1));
  int next = 0;
  for (int rg = 0; rg < c.n_rg; ++rg) {  // (as mx_place deals them)
    CHECK(rg * each + (rg < more ? rg : more) == next);
    next += each + (rg < more ? 1 : 0);
  }
  CHECK(next == c.n_blk);
  const int64_t pages = ((int64_t)L + 63) / 64, tiles = (M + 63) / 64;
  CHECK(c.n_sp >= 1 && c.n_sp <= hs::MXA_SPLITS && c.pages >= 1);
  CHECK((int64_t)c.n_sp * c.pages >= pages);  // (the last split takes what is left, and the tree's rows)
  if (c.n_sp > 1) {
    // every split but the last holds a page; where the last one's pages leave no room, the tree's rows are a split of their own
    CHECK((int64_t)(c.n_sp - 2) * c.pages < pages);
    CHECK((int64_t)(c.n_sp - 1) * c.pages >= pages || pages + tiles <= (int64_t)c.n_sp * c.pages);
  }
}

static void check_batch(const Batch& b) {
  const int B = (int)b.lens.size(), G = b.Hq / b.Hkv;
  if (mx_attn_host_check(b.no.data(), b.lens.data(), B, b.Hq, b.Hkv, b.D) != HS_OK) {
    CHECK(hs_tree_attention_mx_workspace(b.no.data(), b.lens.data(), B, b.Hq, b.Hkv, b.D) == 0);
    return;
  }
  const size_t room = hs_tree_attention_mx_workspace(b.no.data(), b.lens.data(), B, b.Hq, b.Hkv, b.D);
  static hs::MxPlan p;
  for (int fmt = 0; fmt < 2; ++fmt) {
    std::memset(static_cast<void*>(&p), 0xa5, sizeof(p));  // (nothing of an earlier plan is taken for this one's)
    hs::mx_plan(b.no.data(), b.lens.data(), B, b.Hq, b.Hkv, b.D, fmt, p);
    CHECK(mx_bytes(p, b.D) <= room && p.records <= hs::MXA_RECORDS);
    int64_t items = 0, records = 0;
    std::vector<int> seen(B, 0);
    auto count = [&](const hs::MxCut& c, int s) {
      const int M = b.no[s + 1] - b.no[s];
      check_cut(c, M, G, (int)b.lens[s]);
      ++seen[s];
      items += (int64_t)c.n_sp * c.n_rg * b.Hkv;
      records += c.n_sp > 1 ? (int64_t)M * b.Hq * c.n_sp : 0;
    };
    if (B <= hs::MXA_ENTRIES) {
      CHECK(p.n_seq <= hs::MXA_ENTRIES);
      for (int i = 0; i < p.n_seq; ++i) {
        CHECK(p.seq[i].s >= 0 && p.seq[i].s < B);
        count(p.seq[i].cut, p.seq[i].s);
      }
    } else {
      for (int s = 0; s < B; ++s) {
        const int M = b.no[s + 1] - b.no[s];
        if (M == 0) continue;
        const hs::MxCut c = hs::mx_cut(M, G, (int)b.lens[s], p.cuts);
        count(c, s);
        // the workgroups repeat this cut with divisions by a float product
        const int pages = ((int)b.lens[s] + 63) / 64, all = pages + (M + 63) / 64, per = p.cuts.pages[c.form];
        for (int ulps = -1; ulps <= 1; ++ulps) {
          const int least = div_by_product(all + hs::MXA_SPLITS - 2, hs::MXA_SPLITS - 1, ulps);
          CHECK(least == (all + hs::MXA_SPLITS - 2) / (hs::MXA_SPLITS - 1));
          const int n = per < least ? least : per < 1 ? 1 : per, even = div_by_product(all + n - 1, n, ulps);
          CHECK(even == (all + n - 1) / n && div_by_product(all + even - 1, even, ulps) == (all + even - 1) / even);
          CHECK(div_by_product(pages + c.pages - 1, c.pages, ulps) == (pages + c.pages - 1) / c.pages);
        }
      }
    }
    for (int s = 0; s < B; ++s) CHECK(seen[s] == (b.no[s + 1] > b.no[s] ? 1 : 0));
    CHECK(items == p.items && records == p.records);
  }
}

static Batch random_batch(int it) {
  static const int heads[][2] = {{32, 8}, {8, 8}, {64, 8}, {4, 1}, {12, 4}, {6, 3}, {1024, 1}, {40, 40}, {7, 1}, {4096, 4096}};
  Batch b;
  const int* h = heads[rnd() % (it % 10 == 0 ? 10 : 8)];
  const int B = it % 40 == 0 ? 1 + rnd() % 700 : it % 8 == 0 ? 60 + rnd() % 10 : 1 + rnd() % 20;
  b.Hq = h[0], b.Hkv = h[1], b.D = rnd() % 3 ? 128 : 64, b.fmt = 0;
  b.no.assign(1, 0);
  const int kind = rnd() % 5, most_rows = kind == 0 ? 1 : kind == 1 ? 130 : 1024;
  const int64_t most_len = kind == 4 ? HS_MX_MAX_TOKENS : kind == 3 ? 100000 : 5000;
  for (int s = 0; s < B; ++s) {
    const unsigned r = rnd();
    const int M = r % 9 == 0 ? 0 : r % 9 == 1 ? 1 : r % 9 == 2 ? most_rows : (int)(rnd() % (most_rows + 1));
    const unsigned l = rnd();
    const int64_t edge = (int64_t)(rnd() % 40) * 64 + (int)(rnd() % 3) - 1;
    b.lens.push_back(l % 9 == 0 ? 0 : l % 9 == 1 ? most_len : l % 9 < 4 ? (edge < 0 ? 0 : edge) : (int64_t)(rnd() % (most_len + 1)));
    b.no.push_back(b.no.back() + M);
  }
  return b;
}

// A launch's arguments name sequences of the batch, as the host arrays have them, and as many items as its grid.
static void check_arguments(const hs::MxAttnArgs& a, unsigned grid, const Batch& b, std::vector<int>& seen) {
  const int B = (int)b.lens.size();
  int64_t items = 0;
  auto one = [&](int s, int n0, int M, int64_t L, const hs::MxCut& c) {
    CHECK(s >= 0 && s < B && n0 == b.no[s] && M == b.no[s + 1] - n0 && L == b.lens[s]);
    ++seen[s];
    items += (int64_t)c.n_sp * c.n_rg * b.Hkv;
  };
  CHECK((a.n_entries > 0) == (B <= hs::MXA_ENTRIES) && a.n_entries <= hs::MXA_ENTRIES);
  for (int i = 0; i < a.n_entries; ++i) {
    const hs::MxEntry& e = a.entries[i];
    hs::MxCut c = {};
    c.n_sp = e.n_sp_form & 255, c.n_rg = (int)((unsigned)e.groups >> 16);
    CHECK(e.first == items);
    one(e.n_sp_form >> 16, e.n0, e.M, e.L, c);
  }
  if (a.n_entries == 0) {
    CHECK(a.n_seqs >= 1 && a.n_seqs <= hs::MXA_SEQS && a.seq0 >= 0 && a.seq0 + a.n_seqs <= B);
    for (int i = 0; i < a.n_seqs; ++i) {
      const int M = a.seqs[i + 1].n0 - a.seqs[i].n0;
      if (M > 0) one(a.seq0 + i, a.seqs[i].n0, M, a.seqs[i].L, hs::mx_cut(M, a.G, a.seqs[i].L, a.cuts));
    }
  }
  CHECK(items == (int64_t)grid);
}

// Addresses of device arrays that a launch must not depend on: a captured one keeps the lengths that it was planned with.
static int check_launches(const Batch& b) {
  const int B = (int)b.lens.size();
  if (mx_attn_host_check(b.no.data(), b.lens.data(), B, b.Hq, b.Hkv, b.D) != HS_OK || b.no.back() == 0) return 0;
  const int64_t lens_at = 0x5a5a5a5a00ll, offsets_at = 0x6b6b6b6b00ll, other = 0x7c7c7c7c00ll;
  auto at = [](int64_t x) { return reinterpret_cast<void*>(x); };
  launched.clear();
  const hs_status st = hs_tree_attention_mx(at(other), (int64_t)b.Hq * b.D, at(other), at(other), at(other), at(other), HS_MX_E4M3, at(other), (int64_t)b.Hkv * b.D, at(other),
                                            (int64_t)b.Hkv * b.D, (const int32_t*)at(other), (const int32_t*)at(offsets_at), b.no.data(), (const int32_t*)at(other), 4, 1000,
                                            (const int64_t*)at(lens_at), b.lens.data(), B, b.Hq, b.Hkv, b.D, HS_BF16, 0.1f, at(other), nullptr, at(other), 1ll << 40, nullptr);
  CHECK(!launched.empty());
  std::vector<int> seen(B, 0);
  for (const auto& l : launched) {
    for (size_t i = 0; i + 8 <= sizeof(l.first); i += 8) {
      int64_t word;
      std::memcpy(&word, reinterpret_cast<const char*>(&l.first) + i, 8);
      CHECK(word != lens_at && word != offsets_at);
    }
    check_arguments(l.first, l.second, b, seen);
  }
  for (int s = 0; s < B; ++s) CHECK(seen[s] == (b.no[s + 1] > b.no[s] ? 1 : 0));
  CHECK(st == HS_OK);
  return (int)launched.size();
}

int main(int argc, char** argv) {
  if (argc >= 2 && std::strcmp(argv[1], "fuzz") == 0) {
    const int n = std::atoi(argv[2]);
    state ^= (unsigned long long)std::atoll(argv[3]) * 0x9e3779b97f4a7c15ull;
    long rows = 0;
    for (int it = 0; it < n; ++it, ++batch) {
      const Batch b = random_batch(it);
      rows += b.no.back();
      check_batch(b);
    }
    // a row of a KV head to its tree row, as the kernel divides (mx_own): every group size, the rows around each multiple
    for (int G = 1; G <= 1024; ++G) {
      const float inv = 1.f / (float)G;
      for (int q = 0; q <= 1024; ++q)
        for (int d = -1; d <= 1; ++d) {
          const int r = q * G + d;
          if (r >= 0 && r < G * 1024) CHECK((int)(((float)r + 0.5f) * inv) == r / G);
        }
    }
    // items, splits and row groups of mx_place: 23 bits by any divisor
    for (int i = 0; i < 2000000; ++i) {
      const int d = 1 + rnd() % (1u << (1 + rnd() % 17)), q = rnd() % ((1 << 23) / d);
      for (int x = q * d - 1; x <= q * d + 1; ++x)
        if (x >= 0 && x < 1 << 23)
          for (int ulps = -1; ulps <= 1; ++ulps) CHECK(div_by_product(x, d, d == 1 ? 0 : ulps) == x / d);  // (1 / 1 is exact)
    }
    std::printf("ok %ld\n", rows);
    return 0;
  }
  if (argc >= 2 && std::strcmp(argv[1], "args") == 0) {
    state ^= (unsigned long long)std::atoll(argv[3]) * 0x9e3779b97f4a7c15ull;
    long launches = 0;
    for (int it = 0; it < std::atoi(argv[2]); ++it, ++batch) {
      Batch b = random_batch(it % 2 ? 40 : it);
      for (auto& l : b.lens) l %= 200;  // (no splits: the merge's launch is not a stub)
      launches += check_launches(b);
    }
    std::printf("ok %ld\n", launches);
    return 0;
  }
  if (argc >= 2 && std::strcmp(argv[1], "form") == 0) {
    Batch b;
    int B;
    static hs::MxPlan p;
    while (std::scanf("%d %d %d %d %d", &b.fmt, &b.Hq, &b.Hkv, &b.D, &B) == 5) {
      b.no.assign(1, 0), b.lens.assign(B, 0);
      for (int s = 0, m; s < B; ++s) {
        if (std::scanf("%d", &m) != 1) return 1;
        b.no.push_back(b.no.back() + m);
      }
      for (int s = 0; s < B; ++s) {
        long long l;
        if (std::scanf("%lld", &l) != 1) return 1;
        b.lens[s] = l;
      }
      hs::mx_plan(b.no.data(), b.lens.data(), B, b.Hq, b.Hkv, b.D, b.fmt, p);
      for (int s = 0; s < B; ++s) {
        const int M = b.no[s + 1] - b.no[s];
        if (M == 0) continue;
        hs::MxCut c = {};
        if (B <= hs::MXA_ENTRIES) {
          for (int i = 0; i < p.n_seq; ++i)
            if (p.seq[i].s == s) c = p.seq[i].cut;
        } else {
          c = hs::mx_cut(M, b.Hq / b.Hkv, (int)b.lens[s], p.cuts);
        }
        std::printf("%d %d %d %d %d;", c.form, c.n_blk, c.n_rg, c.n_sp, c.pages);
      }
      std::printf("\n");
    }
    return 0;
  }
  return 2;
}
