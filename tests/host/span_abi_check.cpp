// Host build of the C ABI layer of attention over spans and of decode over shared
// prefixes (basp_api_span.cpp, basp_api_shared.cpp) with every kernel launch replaced by
// a recorder, meant to run under AddressSanitizer and UndefinedBehaviorSanitizer:
// misuses and extreme sizes return their status and launch nothing, valid calls on
// fake aligned addresses launch what their arguments say, and the cuts of both
// operators keep their promises over many sizes.  Prints "span abi ok <cases>"; exits
// 1 at the first failure.
#include "../../paper_2609_03151_amd/csrc/basp_api_shared.cpp"
#include "../../paper_2609_03151_amd/csrc/basp_api_span.cpp"

#include <limits.h>
#include <stdio.h>

#include <algorithm>
#include <random>
#include <vector>

namespace basp {
static int g_launches = 0;
static SpanArgs g_span;
static SharedArgs g_shared;
static bool g_bf16;
hipError_t launch_span_fwd(const SpanArgs &a, uint16_t *, float *, hipStream_t) {
  ++g_launches;
  g_span = a;
  return hipSuccess;
}
hipError_t launch_span_bwd(const SpanArgs &a, const uint16_t *, const float *, const uint16_t *, void *,
                           void *, void *, bool bf16, void *, hipStream_t) {
  ++g_launches;
  g_span = a;
  g_bf16 = bf16;
  return hipSuccess;
}
hipError_t launch_attn_decode_shared(const SharedArgs &a, hipStream_t) {
  ++g_launches;
  g_shared = a;
  return hipSuccess;
}
}  // namespace basp

extern "C" hipError_t hipGetLastError(void) { return hipSuccess; }

static int g_cases = 0;
#define CHECK(cond)                                          \
  do {                                                       \
    ++g_cases;                                               \
    if (!(cond)) {                                           \
      printf("FAIL line %d: %s\n", __LINE__, #cond);         \
      return 1;                                              \
    }                                                        \
  } while (0)

static void *at(uintptr_t x) { return reinterpret_cast<void *>(x); }

using namespace basp;

// The cut of attn_span_bwd's key pass: regions of the workspace in order, every (key tile,
// row chunk) pair once, lists and launches within their bounds.
static int span_cuts() {
  for (int d : {64, 80, 96, 128})
    for (int n_k : {1, 2, 8})
      for (int rep : {1, 3, 8})
        for (int b : {1, 3, 40, 65535})
          for (long long S : {1ll, 2ll, 63ll, 64ll, 65ll, 127ll, 129ll, 1000ll, 2049ll, 8191ll, 16384ll,
                              65537ll, 131072ll, 1000003ll, 1048577ll, 2097152ll, 4194303ll,
                              (1ll << 30) / ((long long)d * n_k * rep) - 257}) {
            if (S < 1 || check_shape(b, (int)S, n_k * rep, n_k, d) != BASP_OK) continue;
            SpanArgs s{};
            const int spans = 0;
            s.spans = &spans;
            s.b = b, s.S = (int)S, s.Hl = n_k * rep, s.Hkl = n_k, s.d = d;
            s.scale = 1.f;
            const SpanCut c = span_cut(s);
            CHECK(c.chunk_rows >= kKvKeys && c.chunk_rows % kKvKeys == 0 && c.nchunks >= 1);
            CHECK((long long)c.nchunks * c.chunk_rows >= S && (c.nchunks - 1ll) * c.chunk_rows < S);
            CHECK(c.nsplits >= 1 && c.nsplits <= rep && c.ktiles == (S + 127) / 128);
            CHECK(c.chunk_rows / kSpanStep <= span_max_steps(d) && span_max_steps(d) <= 65536);
            const size_t Sp = (S + 63) / 64 * 64, slots = (size_t)c.nchunks * c.nsplits;
            CHECK((size_t)c.Sp == Sp && c.rows % 256 == 0 && c.hulls % 256 == 0 &&
                  c.touched % 256 == 0 && c.parts % 256 == 0);
            CHECK(c.rows >= (size_t)b * s.Hl * Sp * 8 && c.hulls >= c.rows + (size_t)b * Sp * 8);
            CHECK(c.touched >= c.hulls + (size_t)b * (Sp / 32) * 16);
            CHECK(c.parts >= c.touched + slots * b * n_k * c.ktiles * 4);
            CHECK(c.bytes == c.parts + (slots > 1 ? 2 * slots * b * S * n_k * d * 4 : 0));
            CHECK(span_bwd_workspace_bytes(s) == c.bytes);
            if (!span_bwd_fits(s)) continue;
            const int T = c.chunk_rows / kKvKeys, causal = kv_units(c.nchunks, T);
            const long long blocks = span_key_blocks(s, c);
            CHECK(blocks == ((long long)causal + (long long)c.nchunks * c.ktiles) * c.nsplits * b * n_k);
            CHECK((blocks + span_dq_blocks(s)) * kSpanThreads <= 0xFFFFFFFFll);
            if ((size_t)c.nchunks * c.ktiles > 100000) continue;
            std::vector<int> seen((size_t)c.nchunks * c.ktiles);
            for (int pair = 0; pair < causal + c.nchunks * c.ktiles; ++pair) {  // as the kernel has it
              int kt, ch;
              if (pair < causal) {
                kv_unit(pair, c.nchunks, T, kt, ch);
                if (kt >= c.ktiles) continue;
              } else {
                kt = (pair - causal) % c.ktiles, ch = (pair - causal) / c.ktiles;
                if (kt < (ch + 1) * T) continue;
              }
              ++seen[(size_t)ch * c.ktiles + kt];
            }
            for (size_t i = 0; i < seen.size(); ++i)
              if (seen[i] != 1) {
                // causal units leave out chunks that end before the keys only
                printf("FAIL pair %zu seen %d: S=%lld d=%d n_k=%d rep=%d b=%d\n", i, seen[i], S, d, n_k,
                       rep, b);
                return 1;
              }
            ++g_cases;
          }
  return 0;
}

// The cut of attn_decode_shared: regions in order, and room for the chunks and members of any
// groups.
static int shared_cuts() {
  std::mt19937 rng(1);
  for (int b : {1, 2, 3, 5, 64, 129, 512, 513, 4096, 100003})
    for (int n_k : {1, 2, 8})
      for (int rep : {1, 4, 7, 16, 17, 32, 40})
        for (int n_groups : {0, 1, 2, 7, 128, 129, 5000})
          for (int len : {1, 64, 128, 129, 4096, 131072, 1 << 30}) {
            const int n_q = n_k * rep, d = 80;
            if (check_decode(b, n_q, n_k, d, len) != BASP_OK) {
              CHECK(basp_attn_decode_shared_workspace_bytes(b, n_q, n_k, d, len, n_groups) == 0);
              continue;
            }
            const SharedCut c = shared_cut(b, n_q, n_k, d, len, n_groups);
            CHECK(c.local == (b <= kLocalSeqs && n_groups <= kLocalGroups));
            CHECK(c.rows == 64 || c.rows == 128);
            const int sharing = std::min(n_groups, b / 2);
            CHECK((c.chunks == 0) == (sharing == 0) && (c.splits == 0) == (sharing == 0));
            CHECK((long long)c.chunks * n_k * c.splits == c.prefix_blocks);
            CHECK(c.own.groups >= 1 && c.own.groups <= (sharing ? 256 : 512));
            CHECK(((long long)c.prefix_blocks + c.own.groups) * 256 <= 0xFFFFFFFFll);
            CHECK(c.vheads == n_k * c.own.row_groups);
            CHECK(c.splits <= std::max(1, (len + 127) / 128));
            const size_t row = (size_t)d * 4;
            CHECK(c.records >= c.ints + (4 * (size_t)b + 2 + 3 * (size_t)n_groups) * 4);
            CHECK(c.records % 16 == 0 && c.open % 16 == 0 && c.own_ml % 16 == 0 && c.own_o % 16 == 0 &&
                  c.row_ml % 16 == 0 && c.row_o % 16 == 0 && c.part_ml % 16 == 0 && c.part_o % 16 == 0);
            CHECK(c.open >= c.records + (size_t)c.chunks * 16);
            CHECK(c.own_ml >= c.open + (size_t)b * c.vheads * sizeof(DecodeOpen));
            CHECK(c.own_o >= c.own_ml + (size_t)c.own.groups * 2 * c.own.rows * 8);
            CHECK(c.row_ml >= c.own_o + (size_t)c.own.groups * 2 * c.own.rows * row);
            CHECK(c.row_o >= c.row_ml + (sharing ? (size_t)b * n_q * 8 : 0));
            CHECK(c.part_ml >= c.row_o + (sharing ? (size_t)b * n_q * row : 0));
            CHECK(c.part_o >= c.part_ml + (size_t)c.prefix_blocks * c.rows * 8);
            CHECK(c.bytes == c.part_o + (size_t)c.prefix_blocks * c.rows * row);
            CHECK(basp_attn_decode_shared_workspace_bytes(b, n_q, n_k, d, len, n_groups) == c.bytes);
            // units of all sequences and what they are dealt out by, in 32 bits
            const long long units = (long long)b * c.vheads * ((len + 127ll) / 128 + 1);
            CHECK(units + c.own.groups <= INT_MAX);
            for (int turn = 0; turn < 3; ++turn) {  // equal, random and one large group
              long long chunks = 0, left = b;
              for (int g = 0; g < n_groups && left > 0; ++g) {
                long long n = turn == 0 ? b / n_groups
                              : turn == 1 ? 1 + (long long)(rng() % (unsigned)std::max(1, 2 * b / n_groups))
                                          : (g == 0 ? b - 2ll * (sharing - 1) : 2);
                n = std::min(n, left);
                left -= n;
                if (n >= 2) chunks += (n * rep + c.rows - 1) / c.rows;
              }
              CHECK(chunks <= c.chunks);
            }
          }
  return 0;
}

int main() {
  void *p[12];
  for (int i = 0; i < 12; ++i) p[i] = at(0x100000u * (i + 1));
  float *f[12];
  for (int i = 0; i < 12; ++i) f[i] = static_cast<float *>(p[i]);
  const int *ints = static_cast<int *>(p[9]);
  const int big[] = {INT_MIN, INT_MIN + 1, -1, 0, 1, 7, 128, 65536, INT_MAX - 1, INT_MAX};
  const long long strides[] = {LLONG_MIN, -1, 0, 64, 1ll << 31, 1ll << 40, LLONG_MAX};

  // Extreme sizes in every place: a status, no overflow, and a launch only when OK.
  for (int x : big)
    for (int y : big)
      for (int z : big) {
        for (long long row : strides) {
          int before = g_launches;
          int rc = basp_attn_span_fwd(p[0], p[1], p[2], ints, f[3], p[4], f[5], x, y, z, 1, 64, row, 64,
                                      64, 0.1f, 0.f, nullptr);
          CHECK((rc == BASP_OK && x != 0 && y != 0) == (g_launches == before + 1));
          before = g_launches;
          rc = basp_attn_span_bwd(p[0], p[1], p[2], ints, f[3], p[4], f[5], p[6], p[7], p[8], p[10],
                                  p[11], (size_t)-1, x, y, z, z, 64, 1ll << 20, row, 64, 0.1f, 30.f,
                                  BASP_F32, nullptr);
          CHECK((rc == BASP_OK && x != 0 && y != 0) == (g_launches == before + 1));
          before = g_launches;
          rc = basp_attn_decode_shared(p[0], p[1], p[2], nullptr, nullptr, ints, ints, ints, ints, f[3],
                                       p[4], f[5], p[6], (size_t)-1, x, y, 1, 64, 16, 100, 4, z > 0 ? z : 1,
                                       z, row, 0.1f, 5.f, BASP_BF16, nullptr);
          CHECK((rc == BASP_OK && x != 0) == (g_launches == before + 1));
        }
        basp_attn_span_bwd_workspace_bytes(x, y, z, z, 64);
        basp_attn_span_bwd_workspace_bytes(x, y, z, 1, 128);
        basp_attn_decode_shared_workspace_bytes(x, y, z, 64, 1000, 3);
        basp_attn_decode_shared_workspace_bytes(x, y, 1, 64, z, x);
      }

  // What a valid call launches.
  CHECK(basp_attn_span_fwd(p[0], p[1], p[2], ints, f[3], p[4], f[5], 3, 1000, 14, 2, 96, 18 * 96,
                           2 * 96, 4 * 96, 0.125f, 30.f, nullptr) == BASP_OK);
  CHECK(g_span.q.p == p[0] && g_span.k.row_elems == 192 && g_span.v.row_elems == 384 &&
        g_span.spans == ints && g_span.slopes == f[3] && g_span.Hl == 14 && g_span.Hkl == 2 &&
        g_span.cap == 30.f && g_span.scale == 0.125f);
  const size_t need = basp_attn_span_bwd_workspace_bytes(3, 1000, 14, 2, 96);
  for (size_t have : {need, need - 1})
    CHECK(basp_attn_span_bwd(p[0], p[1], p[2], nullptr, nullptr, p[4], f[5], p[6], p[7], p[8], p[10],
                             p[11], have, 3, 1000, 14, 2, 96, 14 * 96, 192, 192, 0.125f, 0.f, BASP_BF16,
                             nullptr) == (have == need ? BASP_OK : BASP_ERR_WORKSPACE));
  CHECK(g_bf16 && g_span.spans == nullptr && g_span.cap == 0.f);
  unsigned char *sc = static_cast<unsigned char *>(p[7]);
  const size_t room = basp_attn_decode_shared_workspace_bytes(5, 14, 2, 80, 5000, 2);
  for (size_t have : {room, room - 1})
    CHECK(basp_attn_decode_shared(p[0], p[1], p[2], sc, sc, ints, ints, ints, ints, f[3], p[4], f[5], p[6],
                                  have, 5, 14, 2, 80, 16, 9, 400, 5000, 2, 28 * 80, 0.5f, 20.f, BASP_E4M3,
                                  nullptr) == (have == room ? BASP_OK : BASP_ERR_WORKSPACE));
  CHECK(g_shared.d.n_q == 14 && g_shared.n_groups == 2 && g_shared.cap == 20.f &&
        g_shared.d.s.page_log2 == 4 && g_shared.d.workspace == p[6] && g_shared.d.q_row == 2240);
  if (span_cuts() || shared_cuts()) return 1;
  printf("span abi ok %d\n", g_cases);
  return 0;
}
