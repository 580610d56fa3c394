// Calls the layers and losses with addresses that nothing is read from and prints what each call launches; one call a line of standard
// input:
//   forward|backward  ROWS IN OUT IN_TYPE OUT_TYPE ACT OFF   (OFF: bytes that x, W and grad_y lie off 16)
//   distill           TYPE ROWS V K WHAT                     (WHAT: 0 the loss, 1 the gradient, 2 both)
//   preference        B PAIRS
// -> the call's status, workspace bytes, then kernel, workgroups, threads of a workgroup, bytes of LDS of each launch
#include <cstdio>
#include <cstring>
#include <string>

#include "../../include/spcfg.h"
#include "record_launches.h"

static std::string g_out;
void record_launch(const char* kernel, dim3 grid, dim3 block, size_t lds) {
  std::string k(kernel);
  const size_t a = k.find('k'), e = k.find('<');
  k = k.substr(a, (e == std::string::npos ? k.size() : e) - a);
  char s[160];
  snprintf(s, sizeof(s), " %s %lld %u %zu", k.c_str(), (long long)grid.x * grid.y * grid.z, block.x * block.y * block.z, lds);
  g_out += s;
}
namespace spcfg { int launch_status() { return SPCFG_OK; } }

int main() {
  char what[16];
  char* const base = reinterpret_cast<char*>((size_t)1 << 44);
  const auto at = [&](int i, long long off = 0) { return (void*)(base + ((size_t)i << 40) + off); };
  while (scanf("%15s", what) == 1) {
    g_out.clear();
    size_t bytes = 0;
    int rc;
    if (strcmp(what, "forward") == 0 || strcmp(what, "backward") == 0) {
      spcfg_dense_config c{};
      c.struct_size = sizeof(c);
      int off;
      if (scanf("%d %d %d %d %d %d %d", &c.rows, &c.in, &c.out, &c.in_type, &c.out_type, &c.activation, &off) != 7) return 1;
      rc = spcfg_dense_workspace_bytes(&c, &bytes);
      if (rc == 0 && what[0] == 'f')
        rc = spcfg_dense_forward(&c, at(1, off), at(2, off), at(3), nullptr, at(4), at(5), at(6), bytes, nullptr);
      else if (rc == 0)
        rc = spcfg_dense_backward(&c, at(1, off), at(2, off), c.activation ? at(3) : nullptr, at(4, off), nullptr, at(5), at(6), at(7),
                                  at(8), bytes, nullptr);
    } else if (strcmp(what, "distill") == 0) {
      int type, rows, V, k, way;
      if (scanf("%d %d %d %d %d", &type, &rows, &V, &k, &way) != 5) return 1;
      rc = spcfg_distill_workspace_bytes(rows, V, &bytes);
      float *loss = (float*)at(4), *lse = (float*)at(5);
      const int32_t* ids = (const int32_t*)at(3);
      if (rc == 0)
        rc = way == 0 ? spcfg_distill_forward(type, rows, V, k, at(1), at(2), ids, 1.0f, loss, lse, at(6), bytes, nullptr)
             : way == 1 ? spcfg_distill_backward(type, rows, V, k, at(1), at(2), ids, 1.0f, lse, nullptr, at(7), nullptr)
                        : spcfg_distill_forward_backward(type, rows, V, k, at(1), at(2), ids, 1.0f, nullptr, loss, lse, at(7), at(6),
                                                         bytes, nullptr);
    } else {
      int B, n;
      if (scanf("%d %d", &B, &n) != 2) return 1;
      rc = spcfg_preference_forward_backward(B, n, (float*)at(1), nullptr, (int32_t*)at(2), (int32_t*)at(3), 1.0f, 0.0f, nullptr,
                                             (float*)at(4), (float*)at(5), (float*)at(6), nullptr);
    }
    printf("%d %zu%s\n", rc, bytes, g_out.c_str());
  }
  return 0;
}
