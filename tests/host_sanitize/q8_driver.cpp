// The host side of the 8-bit operators' entry points (csrc/q8_api.hip) with the kernel launchers stubbed out, for a build with
// -fsanitize=address,undefined.  Pointers are fake addresses: nothing dereferences them on the host.
#include <cstdint>
#include <cstdio>

#include "../../paper_2511_19797_amd/csrc/q8.h"
#include "../../include/tvmattn.h"

static int launches = 0, fails = 0;
namespace tvm {
hipError_t launch_rowquant(const RowsQ8Args&, int, hipStream_t) { return ++launches, hipSuccess; }
hipError_t launch_gelu_q8(const RowsQ8Args&, int, hipStream_t) { return ++launches, hipSuccess; }
hipError_t launch_gate_adaln_q8(const GateAdalnQ8Args&, int, hipStream_t) { return ++launches, hipSuccess; }
hipError_t launch_linear_q8(const LinearQ8Args&, int, hipStream_t) { return ++launches, hipSuccess; }
}  // namespace tvm
#define EXPECT(cond) \
  do { \
    if (!(cond)) ++fails, std::printf("FAILED %d: %s\n", __LINE__, #cond); \
  } while (0)

static void* P(uint64_t a) { return reinterpret_cast<void*>(a); }
static float* F(uint64_t a) { return reinterpret_cast<float*>(a); }

int main() {
  const uint64_t G = 1ull << 50;
  const int dims[] = {-1, 0, 1, 7, 8, 16, 4096, 1 << 20, INT32_MAX};
  const long long pitches[] = {-1, 0, 8, 1ll << 20, 1ll << 40, INT64_MAX};
  // extreme sizes: nothing may overflow on the way to the verdict, and what is refused is not launched
  for (int R : dims)
    for (int C : dims)
      for (long long ld : pitches)
        for (int dtype : {0, 1, 5}) {
          const int before = launches;
          const int a = tvmattn_rowquant_fwd(R, C, dtype, P(G), P(2 * G), ld, P(3 * G), F(4 * G), P(5 * G), F(6 * G), nullptr);
          const int b = tvmattn_gelu_jvp_fwd_q8(R, C, dtype, P(G), nullptr, ld, P(3 * G), F(4 * G), nullptr, nullptr, nullptr);
          EXPECT(launches - before == (a == 0) + (b == 0) && a == b);
          for (int K : {16, 1 << 16, INT32_MAX}) {
            const int was = launches;
            const int c = tvmattn_linear_jvp_fwd_q8(R, K, C, dtype, P(G), F(2 * G), P(3 * G), F(4 * G), ld, P(5 * G), F(6 * G), P(7 * G),
                                                    P(8 * G), P(9 * G), ld, nullptr);
            EXPECT(launches - was == (c == 0));
          }
        }
  for (int B : dims)
    for (int T : dims)
      for (int C : dims)
        for (float eps : {0.f, 1e-6f, -1.f, 1.f / 0.f, 0.f / 0.f}) {
          const int before = launches;
          const int a = tvmattn_gate_adaln_jvp_fwd_q8(B, T, C, TVMATTN_BF16, P(G), P(2 * G), P(3 * G), P(4 * G), F(5 * G), F(6 * G), F(7 * G),
                                                      F(8 * G), F(9 * G), F(10 * G), eps, P(11 * G), P(12 * G), P(13 * G), F(14 * G),
                                                      P(15 * G), F(16 * G), nullptr);
          EXPECT(launches - before == (a == 0));
        }
  EXPECT(launches > 20);
  std::puts(fails ? "host checks failed" : "host checks ok");
  return fails != 0;
}
