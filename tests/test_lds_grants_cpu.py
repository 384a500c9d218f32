"""csrc/lds_grant.h on the CPU: a kernel's dynamic LDS is granted on every device
that launches it, once for each larger size, and a grant that fails is not kept."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_14782_amd", "csrc")

MAIN = r"""
#include <cstdio>
#include <thread>
#include <vector>
#include "lds_grant.h"
using namespace bacon;

#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)

int main() {
  LdsGrants g;
  std::vector<size_t> asked;
  int status = 0;
  auto ask = [&](size_t b) { asked.push_back(b); return status; };
  CHECK(g.grant(0, 64 * 1024, ask) == 0 && asked.empty());
  CHECK(g.grant(0, 100000, ask) == 0 && asked.size() == 1);
  CHECK(g.grant(0, 100000, ask) == 0 && g.grant(0, 90000, ask) == 0 && asked.size() == 1);
  CHECK(g.grant(1, 90000, ask) == 0 && asked.size() == 2 && asked.back() == 90000);     // another device
  CHECK(g.grant(0, 120000, ask) == 0 && asked.size() == 3);
  CHECK(g.grant(1, 100000, ask) == 0 && asked.size() == 4);
  status = 7;                                                                            // a refusal is returned,
  CHECK(g.grant(2, 90000, ask) == 7 && g.grant(2, 90000, ask) == 7 && asked.size() == 6); // and asked again
  status = 0;
  CHECK(g.grant(2, 90000, ask) == 0 && g.grant(2, 90000, ask) == 0 && asked.size() == 7);
  for (int device : {-1, 64, 100000}) {                                                  // none of the table's
    const size_t n = asked.size();
    CHECK(g.grant(device, 90000, ask) == 0 && g.grant(device, 90000, ask) == 0 && asked.size() == n + 2);
  }
  // threads that ask for different sizes: the last grant is the largest
  LdsGrants h;
  size_t last = 0;
  std::vector<std::thread> ts;
  for (size_t i = 0; i < 8; ++i)
    ts.emplace_back([&, i] { h.grant(3, 70000 + 1000 * i, [&](size_t b) { last = b; return 0; }); });
  for (auto &t : ts) t.join();
  CHECK(last == 77000);
  return 0;
}
"""


def test_grants_are_by_device(tmp_path):
    src, exe = tmp_path / "grants.cpp", str(tmp_path / "grants")
    src.write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-pthread", "-I", CSRC, "-o", exe, str(src)], check=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert res.returncode == 0, res.stdout


def test_kernels_are_granted_by_no_other_way():
    """Every launch of the library takes its grant from there, and looks at its status."""
    for name in os.listdir(CSRC):
        with open(os.path.join(CSRC, name)) as f:
            text = f.read()
        if name != "allow_lds.h":
            assert "hipFuncSetAttribute" not in text, name
        for line in text.splitlines():
            if "allow_lds<" in line:
                assert "hipError_t e = allow_lds<" in line, (name, line)
