"""The C entry points whose kernels wait hand them the word that a wait which gives up is reported in: kv_api.cu built with stand-ins
for the launches, no device needed."""
import os
import subprocess

from paper_2511_04063_b200 import build

PROGRAM = r"""
#include <cstdio>
#include "kv_common.cuh"
namespace dq {
namespace { int word; int* seen[2]; }
namespace mx { dq_status current_device(Device& d) { d.sms = 148; d.d_status = &word; return DQ_OK; } }
namespace kv {
int64_t attention_workspace(int) { return 1; }
dq_status rope(cudaStream_t, const mx::Device&, int, const RopeArgs&) { return DQ_OK; }
dq_status append(cudaStream_t, const mx::Device&, int, int, const AppendArgs&) { return DQ_OK; }
dq_status dequantize(cudaStream_t, const mx::Device&, int, int, const AppendArgs&) { return DQ_OK; }
dq_status evict(cudaStream_t, const mx::Device&, int, const EvictArgs&) { return DQ_OK; }
dq_status attention(cudaStream_t, const mx::Device&, int, int, const AttentionArgs& a) { seen[0] = a.d_status; return DQ_OK; }
dq_status attention_weights(cudaStream_t, const mx::Device&, int, int, const AttentionArgs& a) { seen[1] = a.d_status; return DQ_OK; }
}  // namespace kv
}  // namespace dq
int main() {
  void* at = (void*)4096;                                       // (an address that nothing follows)
  dq_heads_t q = {at, 128, 128, 1};
  dq_kv_cache_t c = {at, 1, (const int32_t*)at, (const int32_t*)at, 1, 1, 1, 128, 16};
  if (dq_kv_attention(&q, DQ_BF16, 1, &c, nullptr, 1.f, &q, nullptr, at, nullptr) != DQ_OK) return 1;
  if (dq_kv_attention_weights(&q, DQ_BF16, 1, (const float*)at, &c, nullptr, 1.f, nullptr, (float*)at, 16, nullptr) != DQ_OK) return 2;
  return dq::seen[0] != &dq::word ? 3 : dq::seen[1] != &dq::word ? 4 : 0;
}
"""


def test_waiting_kernels_are_given_the_status_word(tmp_path):
    source, binary = tmp_path / "status.cu", tmp_path / "status"
    source.write_text(PROGRAM)
    built = subprocess.run([build._nvcc(), *build.NVCC_FLAGS, str(source), os.path.join(build.CSRC, "kv_api.cu"), "-o", str(binary)],
                           capture_output=True, text=True, timeout=600)
    assert built.returncode == 0, built.stderr
    assert subprocess.run([str(binary)], timeout=60).returncode == 0
