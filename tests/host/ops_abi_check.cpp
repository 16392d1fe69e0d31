// Host build of the C ABI layer of the operators around attention
// (basp_api_ops.cpp) with every kernel launch replaced by a recorder, meant to run
// under AddressSanitizer and UndefinedBehaviorSanitizer: misuses and extreme sizes
// return their status and launch nothing, valid calls on fake aligned addresses
// launch what their arguments say, and the cut of an attention call keeps its
// promises over many sizes.  Prints "ops abi ok <cases>"; exits 1 at the first
// failure.
#include "../../paper_2609_03151_amd/csrc/basp_api_ops.cpp"

#include <limits.h>
#include <stdio.h>

namespace basp {
static int g_launches = 0;
static NormArgs g_norm;
static CacheArgs g_cache;
static DecodeArgs g_decode;
hipError_t launch_norm_rope(NormArgs a, int, bool, bool, hipStream_t) {
  ++g_launches;
  g_norm = a;
  return hipSuccess;
}
int norm_bwd_blocks(uint32_t rows, int) { return rows < 1024 ? (int)rows : 1024; }
hipError_t launch_norm_rope_bwd(const NormArgs &a, float *, int, bool, bool, bool, hipStream_t) {
  ++g_launches;
  g_norm = a;
  return hipSuccess;
}
hipError_t launch_kv_write(const CacheArgs &a, hipStream_t) {
  ++g_launches;
  g_cache = a;
  return hipSuccess;
}
hipError_t launch_kv_read(const CacheArgs &a, hipStream_t) {
  ++g_launches;
  g_cache = a;
  return hipSuccess;
}
hipError_t launch_attn_decode(const DecodeArgs &a, hipStream_t) {
  ++g_launches;
  g_decode = a;
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

int main() {
  using namespace basp;
  void *p[12];
  for (int i = 0; i < 12; ++i) p[i] = at(0x100000u * (i + 1));
  float *f[12];
  for (int i = 0; i < 12; ++i) f[i] = static_cast<float *>(p[i]);
  const int *table = static_cast<int *>(p[8]), *ints = static_cast<int *>(p[9]);
  const int big[] = {INT_MIN, INT_MIN + 1, -1, 0, 1, 7, 128, 65536, INT_MAX - 1, INT_MAX};

  // Extreme sizes in every place: a status, no overflow, and a launch only when OK.
  for (int x : big)
    for (int y : big)
      for (int z : big) {
        int before = g_launches;
        int rc = basp_qk_norm_rope(p[0], p[1], p[2], p[3], f[4], f[5], f[6], f[7], nullptr, x, y, z,
                                   1, 128, 64, INT_MAX, 1ll << 40, 128, 1ll << 40, 128, 1e-6f, 0, 0,
                                   BASP_BF16, nullptr);
        CHECK((rc == BASP_OK && (x == 0 || y == 0)) == (rc == BASP_OK && g_launches == before));
        before = g_launches;
        rc = basp_qk_norm_rope_bwd(p[0], p[1], p[2], p[3], p[2], p[3], f[4], f[5], f[4], f[5], f[6],
                                   f[7], ints, p[10], (size_t)-1, x, y, 1, z, 64, 64, 1, 64,
                                   1ll << 40, 1e-6f, INT_MAX, 1, BASP_F32, BASP_F32, nullptr);
        CHECK((rc == BASP_OK && (x == 0 || y == 0)) == (rc == BASP_OK && g_launches == before));
        basp_qk_norm_rope_bwd_workspace_bytes(x, y, z, z, 64);
        before = g_launches;
        rc = basp_kv_write(p[0], p[1], p[2], p[3], nullptr, nullptr, table, ints, nullptr, x, y, z, 64,
                           64, 1000, 1000, 1ll << 40, 1ll << 40, BASP_BF16, nullptr);
        CHECK((rc == BASP_OK && (x == 0 || y == 0)) == (rc == BASP_OK && g_launches == before));
        rc = basp_kv_read(p[2], p[3], nullptr, nullptr, table, nullptr, nullptr, p[0], p[1], 1, 1, 1,
                          64, 16, x, y, BASP_BF16, nullptr);
        CHECK((rc == BASP_OK) == (x >= 1 && y >= 1));  // x pages of one head: below 2^31
        before = g_launches;
        rc = basp_attn_decode(p[0], p[2], p[3], nullptr, nullptr, table, ints, p[4], nullptr, p[10],
                              (size_t)-1, x, y, 1, 64, 16, 100, z > 0 ? z : 1, z, 1ll << 40, 0.1f,
                              BASP_BF16, nullptr);
        CHECK((rc == BASP_OK && x == 0) == (rc == BASP_OK && g_launches == before));
        basp_attn_decode_workspace_bytes(x, y, z, 64, 1000);
        basp_attn_decode_workspace_bytes(x, y, 1, 64, z);
      }

  // What a valid call launches.
  CHECK(basp_qk_norm_rope(p[0], p[1], p[2], p[3], f[4], f[5], f[6], f[7], ints, 3, 1000, 28, 4, 96, 48,
                          70000, 36 * 96, 36 * 96, 28 * 96, 4 * 96, 1e-5f, 0, 1, BASP_BF16,
                          nullptr) == BASP_OK);
  CHECK(g_norm.side[0].rows == 84000 && g_norm.side[1].rows == 12000 && g_norm.rot == 48);
  CHECK(g_norm.side[0].x == p[0] && g_norm.side[1].y == p[3] && g_norm.side[1].y_row == 384);
  CHECK(g_norm.by_S.div(2999) == 2 && g_norm.side[1].by_n.div(11) == 2);
  // Without rotation no table bounds pos0, and pos0 + t in 32 bits must not come out
  // negative, the mark of padding.
  CHECK(basp_qk_norm_rope(p[0], p[1], p[2], p[3], f[4], f[5], nullptr, nullptr, nullptr, 4, 3000, 7, 1,
                          96, 0, 0, 1024, 96, 672, 96, 1e-6f, INT_MAX, 0, BASP_BF16,
                          nullptr) == BASP_OK);
  CHECK((long long)g_norm.pos0 + 3000 <= INT_MAX);
  unsigned char *sc[2] = {static_cast<unsigned char *>(p[4]), static_cast<unsigned char *>(p[5])};
  CHECK(basp_kv_write(p[0], p[1], p[2], p[3], sc[0], sc[1], table, ints, ints, 5, 33, 2, 128, 256, 77,
                      9, 1024, 512, BASP_E4M3, nullptr) == BASP_OK);
  CHECK(g_cache.rows == 330 && g_cache.s.page_log2 == 8 && g_cache.s.e4m3 && g_cache.x_row[0] == 1024);
  CHECK(basp_attn_decode(p[0], p[2], p[3], sc[0], sc[1], table, ints, p[6], f[7], p[10],
                         basp_attn_decode_workspace_bytes(5, 14, 2, 80, 5000), 5, 14, 2, 80, 16, 9, 400,
                         5000, 28 * 80, 0.5f, BASP_E4M3, nullptr) == BASP_OK);
  CHECK(g_decode.n_q == 14 && g_decode.workspace == p[10] && g_decode.max_len == 5000);
  CHECK(basp_attn_decode(p[0], p[2], p[3], nullptr, nullptr, table, ints, p[6], nullptr, nullptr, 0, 5,
                         14, 2, 80, 16, 9, 400, 128, 28 * 80, 0.5f, BASP_BF16, nullptr) == BASP_OK);
  CHECK(g_decode.workspace == nullptr);  // one unit each: nothing to join

  // The cut: at least one workgroup and never more than three per CU; every
  // descriptor and partial result inside the workspace; none where no head has two
  // units.
  for (int b : {1, 2, 3, 64, 767, 768, 769, 5000, 1 << 20})
    for (int n_k : {1, 2, 8})
      for (int rep : {1, 4, 7, 16, 17, 32, 33, 100})
        for (int len : {1, 127, 128, 129, 256, 4096, 131072, 1 << 30}) {
          const DecodeCut c = decode_cut(b, n_k * rep, n_k, 80, len);
          CHECK(c.rows == (rep > 16 ? 32 : 16) && c.row_groups * c.rows >= rep &&
                (c.row_groups - 1) * c.rows < rep);
          CHECK(c.groups >= 1 && c.groups <= 768 && c.opens >= 1 && c.opens <= c.groups);
          const long long heads = (long long)b * n_k * c.row_groups;
          CHECK(c.opens == heads || c.opens == c.groups);
          CHECK((c.bytes == 0) == (len <= kDecodeUnit));
          if (c.bytes)
            CHECK(c.bytes == (size_t)c.opens * 16 + (size_t)c.groups * 2 * c.rows * 82 * 4);
        }
  printf("ops abi ok %d\n", g_cases);
  return 0;
}
