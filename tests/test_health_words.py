"""What rg_device_status makes of the kernels' health words: compiled from its header for the host, no GPU needed."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, TIMEOUT, PAGE = 0, 8, 9

PROGRAM = """
#include <stdio.h>
#include <stdlib.h>
#include "rg_health.h"
int main(int argc, char** argv) {
  uint32_t w[6], code = 77;
  for (int i = 0; i < 6; ++i) w[i] = (uint32_t)strtoul(argv[1 + i], nullptr, 0);
  const int status = rg::health_of(w, 4, w + 4, 2, &code);
  printf("%d %u %d", status, code, rg::health_of(w, 4, w + 4, 2, nullptr));
}
"""


@pytest.fixture(scope="module")
def health(tmp_path_factory):
    d = tmp_path_factory.mktemp("health")
    (d / "main.cpp").write_text(PROGRAM)
    paths = [os.path.join(ROOT, "paper_2609_11356_b200", "csrc")]
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", *(f"-I{p}" for p in paths), "-o", str(d / "main"), str(d / "main.cpp")], check=True)

    def run(waits, pages):
        out = subprocess.run([str(d / "main"), *map(str, [*waits, *pages])], check=True, capture_output=True, text=True).stdout.split()
        assert out[0] == out[2]
        return int(out[0]), int(out[1])

    return run


@pytest.mark.parametrize("waits,pages,status,code", [
    ((0, 0, 0, 0), (0, 0), OK, 0), ((0, 0, 0, 0), (0x2B00, 0), PAGE, 0x2B00), ((0, 0, 0, 0), (0, 0x2A00), PAGE, 0x2A00), ((0, 0, 0, 0), (0x2B00, 0x2A00), PAGE, 0x2B00),
    ((0xE00, 0, 0, 0), (0, 0), TIMEOUT, 0xE00), ((0, 0x11, 0x1200, 0), (0, 0), TIMEOUT, 0x11), ((0, 0, 0, 0x2500), (0, 0), TIMEOUT, 0x2500),
    ((0, 0, 0, 0x2500), (0x2B00, 0), TIMEOUT, 0x2500), ((0, 0, 0, 0x3740), (0x2B00, 0x2A00), TIMEOUT, 0x3740), ((0, 0, 0x1200, 0), (0, 0x2A00), TIMEOUT, 0x1200),
])
def test_a_wait_that_gave_up_goes_before_a_bad_page(health, waits, pages, status, code):
    assert health(waits, pages) == (status, code)


def test_no_word_takes_both_kinds_of_code():
    """The kernels keep the first code of a word: a page's in the word of the waits would hide a wait that gives up later."""
    import re
    csrc = os.path.join(ROOT, "paper_2609_11356_b200", "csrc")
    kinds = {}
    for name in sorted(os.listdir(csrc)):
        for word, code in re.findall(r"atomicCAS\(&?(\w+), 0u, ([^;]*)\);", open(os.path.join(csrc, name)).read()):
            kinds.setdefault((name, word), set()).add("page" if "RG_PAGE_CODE" in code else "wait")
    assert kinds[("rg_paged_attention.cu", "g_paged_attn_status_word")] == {"wait"}
    assert kinds[("rg_paged_attention.cu", "g_paged_attn_page_word")] == {"page"}
    assert all(len(k) == 1 for k in kinds.values()), kinds
