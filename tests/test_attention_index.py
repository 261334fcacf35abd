"""Index arithmetic of the attention kernels, compiled for the host and tried at its edges."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_19677_gb300", "csrc")


def run(tmp_path, body):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text('#include <limits.h>\n#include <stdio.h>\n#include <stdint.h>\n#include "cr_attn_index.cuh"\n'
                   "int main()\n{\n" + body + "\nreturn 0;\n}\n")
    subprocess.run(["g++", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", CSRC, str(src), "-o",
                    str(exe)], check=True)
    return subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()


def test_marks_that_nobody_set_stay_within_the_ctas(tmp_path):
    """What memory may hold where a CTA gave up before it set its marks."""
    run(tmp_path, r"""
    const int some[] = {INT_MIN, INT_MIN + 1, -1000000, -2, -1, 0, 1, 2, 150, 151, 152, 303, 304, 511, 1 << 20, INT_MAX - 1,
                        INT_MAX};
    const int ctas[] = {1, 2, 152, 304, 511};
    for (int n : ctas)
        for (int a : some)
            for (int b : some) {
                const cr_cta_span s = cr_marked_ctas(a, b, n);
                if (s.first < 0 || s.n < 1 || s.n > (unsigned)n || s.first + (long long)s.n > n) return 1;
                if (0 <= a && a <= b && b < n && (s.first != a || s.n != (unsigned)(b - a + 1))) return 2;
            }
    """)


def test_the_join_takes_no_mark_as_it_finds_it():
    """Every use of the marks goes through the function above."""
    text = open(os.path.join(CSRC, "cr_attn.cu")).read()
    uses = [line for line in text.splitlines() if "first_cta[" in line or "last_cta[" in line]
    reads = [line for line in uses if "] = (int)blockIdx.x" not in line]
    assert len(reads) == 2 and all("cr_marked_ctas(" in line for line in reads)


def test_no_load_takes_the_path_for_data_that_nothing_writes():
    """Kernels of these files are resident while the one before them may still write what they read: only ordinary loads
    are ordered by their wait for it."""
    for name in ("cr_attn.cu", "cr_pages.cu", "cr_tensor.cuh"):
        text = open(os.path.join(CSRC, name)).read()
        assert not [w for w in ("__ldg(", "ld.global.nc", "__restrict__") if w in text], name


def test_tiles_and_masks_of_the_longest_sequences(tmp_path):
    """Against 64-bit arithmetic, up to the 2^31 - 8 tokens that a row can have; no signed sum passes 32 bits."""
    run(tmp_path, r"""
    const long long top = (1ll << 31) - 8;
    const long long at[] = {0, 1, 2, 63, 64, 65, 127, 128, 129, 1000, 1 << 30, top - 129, top - 128, top - 65, top - 64,
                            top - 17, top - 16, top - 9, top - 8, top - 1, top};
    for (long long n : at) {
        if (cr_key_tiles((int)n, 128) != (n + 127) / 128) return 1;
        for (long long lo : at) {
            const long long t = (n + 63) / 64 - lo / 64;
            if (cr_few_tiles((int)lo, (int)n, 64) != (t > 1 ? t : 1)) return 2;
            for (long long base : at)
                for (int d = -32; d <= 32; d += 16) {
                    const long long key = base / 16 * 16 + d;
                    if (key < 0 || key > (1ll << 31) - 16) continue;
                    const cr_keys16 s = cr_seen16((int)key, (int)lo, (int)n);
                    int seen = 0;
                    for (int j = 0; j < 16; ++j) {
                        const bool want = key + j >= lo && key + j < n;
                        if (s.sees(j) != want) return 3;
                        seen += want;
                    }
                    if (s.all() != (seen == 16)) return 4;
                    if (seen && !s.any()) return 5;
                }
        }
    }
    """)


def test_no_kernel_returns_before_it_has_waited_for_the_one_before():
    """A kernel's end stands for the end of all before it: whoever waits for it counts on that."""
    for name in ("cr_attn.cu", "cr_pages.cu"):
        text = open(os.path.join(CSRC, name)).read()
        kernels = text.split("__global__ ")[1:]
        assert len(kernels) >= 5
        for k in kernels:
            head, body = k.split("{", 1)
            before = body.split("cr_wait_previous();", 1)
            assert len(before) == 2 and "return" not in before[0], head
