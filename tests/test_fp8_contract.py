"""What can be seen without a GPU of the 8-bit operands' kernels and entry points."""
import os
import re
import subprocess

import pytest

from paper_1905_10759_b200 import build

build.build_lib()


def source(name):
    with open(os.path.join(build.CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


@pytest.mark.parametrize("name,published", [("fp8_gemm.cu", "sfull"), ("fp8_weight_grad.cu", "bfull")])
def test_what_crosses_a_pair_of_ctas_is_released_and_acquired_at_cluster_scope(name, published):
    """The arrival that releases nothing beyond its CTA frees what was read (barriers called ...empty) and announces nothing that was
    written; the barrier that does is completed by st_async_u32 from the other CTA and waited for with an acquire of that scope."""
    code = source(name)
    freed = re.findall(r"mbar_arrive_cluster_read\((.*)\);", code)
    assert freed and all("empty" in a for a in freed), freed
    assert re.search(r"st_async_u32\([^;]*%s" % published, code)
    waits = re.findall(r"\bwait(\.cluster)?\((?:smem_u32\(&%s\[|%s_a)" % (published, published), code)
    assert waits and all(waits), waits


# A barrier of one arrival and a byte count, as the copies of a pair complete on; a wait that could not end by itself exits.
MODEL = r"""
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#define __device__
#define __forceinline__ inline
constexpr uint32_t kDrainPolls = 1;
constexpr int S = 5;
constexpr uint32_t BYTES = 100;
static int64_t lead_n, other_n;
struct Bar { int pending = 1; int64_t tx = 0; uint32_t phase = 0; int64_t coming = 0; };      // coming: bytes in flight
static Bar bars[S];
static void turn(Bar& b) { if (b.pending == 0 && b.tx == 0) { b.phase++; b.pending = 1; } }
static Bar& of(uint64_t* p);
static uint64_t mem[S];
static Bar& of(uint64_t* p) { return bars[p - mem]; }
static void mbar_arrive_expect_tx(uint64_t* p, uint32_t n) { Bar& b = of(p); b.tx += n; b.pending--; turn(b); }
static void mbar_complete_tx(uint64_t* p, uint32_t n) { Bar& b = of(p); b.tx -= n; turn(b); }
static bool mbar_wait_quiet(uint64_t* p, uint32_t parity, uint32_t) {
  Bar& b = of(p);
  b.tx -= b.coming; b.coming = 0; turn(b);                       // what is in flight lands
  if ((b.phase & 1) == parity) { printf("%lld %lld: a wait that does not end\n", (long long)lead_n, (long long)other_n); exit(1); }
  return true;
}
FUNCTION
int main() {
  for (lead_n = 0; lead_n <= 4 * S; lead_n++)
    for (other_n = lead_n < S ? 0 : lead_n - S; other_n <= lead_n + S; other_n++) {
      for (Bar& b : bars) b = Bar();
      const int64_t last = lead_n > other_n ? lead_n : other_n;
      // a stage comes round only once both CTAs' copies of its last turn have landed
      for (int64_t i = 0; i < last; i++) {
        Bar& b = bars[i % S];
        b.tx -= b.coming; b.coming = 0; turn(b);
        if (i < lead_n) { b.tx += 2 * BYTES; b.pending--; b.coming += BYTES; }
        if (i < other_n) b.coming += BYTES;
      }
      if (last - lead_n > S || last - other_n > S) continue;
      drain_pair_copies<S>(mem, lead_n, other_n, BYTES);
      for (const Bar& b : bars)
        if (b.coming != 0) { printf("%lld %lld: a copy that nobody waited for\n", (long long)lead_n, (long long)other_n); return 1; }
    }
  return 0;
}
"""


def test_a_kernel_that_gives_up_waits_for_its_pair_s_copies(tmp_path):
    """However far each CTA of a pair came before a wait gave up, the first one waits until every copy of both has landed, and none
    of its waits is for bytes that never come: the function that does it, compiled for the host with a model of the barriers."""
    body = re.search(r"template <int STAGES>\n__device__ __forceinline__ void drain_pair_copies.*?\n}\n", source("fp8_tile.cuh"), re.S)
    (tmp_path / "model.cpp").write_text(MODEL.replace("FUNCTION", body.group(0)))
    subprocess.run(["g++", "-std=c++17", "-o", str(tmp_path / "model"), str(tmp_path / "model.cpp")], check=True)
    run = subprocess.run([str(tmp_path / "model")], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout


@pytest.mark.parametrize("name", ["fp8_gemm.cu", "fp8_weight_grad.cu"])
def test_no_kernel_leaves_by_the_clock(name):
    code = source(name)
    assert "nanosleep" not in code and "leave_cluster(" in code and "drain_pair_copies<STAGES>(" in code


def test_rows_too_far_apart_are_refused_by_every_argument():
    """Fake addresses, never dereferenced."""
    import ctypes
    from paper_1905_10759_b200 import hbmm
    lib, by, P = hbmm._lib, ctypes.byref, ctypes.c_void_p
    x = hbmm.hbmm_fp8_operand(8, 256, 0x1000, 256, 0x2000, 4, 1, 0)
    for ld in (1 << 62, 1 << 60, 1 << 39):                 # fp32: 2^64, 2^62, 2^41 bytes
        for dtype in (0, 1):
            assert lib.hbmm_fp8_quantize(P(0x4000), dtype, 8, 256, ld, by(x), None) == hbmm.ERR_UNSUPPORTED
            assert lib.hbmm_fp8_binarize_backward(by(x), P(0x4000), dtype, ld, 32, P(0x8000), 256, None) == hbmm.ERR_UNSUPPORTED
            assert lib.hbmm_fp8_binarize_backward(by(x), P(0x4000), dtype, 256, 32, P(0x8000), ld, None) == hbmm.ERR_UNSUPPORTED


@pytest.mark.parametrize("family", [0, 100, 200, 309, 600, -400])
def test_families_without_a_wait_to_expire_are_refused(family):
    from paper_1905_10759_b200 import hbmm
    assert hbmm._lib.hbmm_debug_expire_wait_of(family, None) == hbmm.ERR_INVALID_ARG
