// What csrc/fp8_gemm.cu needs of the library's other sources, and a product at made-up addresses.
#include "../../paper_2507_19131_b200/csrc/kernels.h"

extern "C" int fake_sms();
namespace mixaq {
thread_local int g_launches;
int sm_count() { return fake_sms(); }
}

extern "C" int ask_matmul(long m, long n, long k, int w_block_rows, long offset) {
  char* const at = reinterpret_cast<char*>(0x7000'0000'0000 + offset);
  mixaq::Fp8MatmulArgs g = {};
  g.a = {reinterpret_cast<uint8_t*>(at), m, (k + 15) / 16 * 16, 1, reinterpret_cast<float*>(at), 1, m};
  g.w = {reinterpret_cast<uint8_t*>(at), n, (k + 15) / 16 * 16, w_block_rows, reinterpret_cast<float*>(at), 1, n};
  g.K = k; g.y = at; g.y_stride = n;
  return mixaq::launch_fp8_matmul(g, nullptr);
}
