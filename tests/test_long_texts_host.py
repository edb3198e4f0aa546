"""Searches and strides over the places of long texts, at sizes where a sum of two places passes 32 bits: the kernels' own header on the host."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2104_11981_b200", "csrc")


def _run(tmp_path, body):
    source, program = str(tmp_path / "places.cpp"), str(tmp_path / "places")
    with open(source, "w") as f:
        f.write('#include <cstdio>\n#include <initializer_list>\n#include "dlm_places.h"\n' + body)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wno-unknown-pragmas", "-fsanitize=signed-integer-overflow",
                    "-fno-sanitize-recover=all", "-I", CSRC, source, "-o", program], check=True)
    done = subprocess.run([program], capture_output=True, text=True)
    assert done.returncode == 0, done.stderr
    return [int(v) for v in done.stdout.split()]


SEARCH = """
struct Keys {  // keys[i] = i / 3, of which none exists outside [0, count)
    int count;
    mutable int wrong = 0;
    uint32_t operator[](uint32_t i) const {
        wrong += i >= (uint32_t)count;
        return (uint32_t)i / 3;
    }
};
int main() {
    for (int count : {0, 1, 1000, (1 << 30) + 1000, 2147483647}) {
        const Keys keys{count};
        for (uint32_t v : {0u, 1u, 333u, 357913941u, 715827882u, 0xffffffffu})
            std::printf("%d ", dlm::lower_bound(keys, count, v));
        std::printf("%d ", keys.wrong);
    }
}
"""


def test_searches_among_more_than_2_to_the_30_keys(tmp_path):
    want = []
    for count in (0, 1, 1000, (1 << 30) + 1000, 2 ** 31 - 1):
        want += [min(count, 3 * v) for v in (0, 1, 333, 357913941, 715827882, 0xffffffff)] + [0]
    assert _run(tmp_path, SEARCH) == want


STRIDE = """
int main() {
    for (uint32_t first : {0u, 2147483647u - 700u, 2147483647u - 1u, 2147483647u, 2147483647u + 200u}) {
        const uint32_t end = first ? 2147483647u : 1000u;
        uint32_t count = 0, wrong = 0, next = first;
        dlm::each_place<256, 4>(first, end, [&](uint32_t k) {
            wrong += k != next || k >= end || ++count > 4;
            next = k + 256;
        });
        std::printf("%u %u ", count, wrong);
    }
}
"""


def test_strides_that_end_at_2_to_the_31_places(tmp_path):
    assert _run(tmp_path, STRIDE) == [4, 0, 3, 0, 1, 0, 0, 0, 0, 0]
