"""A request's rows from two starts that may hold anything, on the host: what the serving kernels count lies in the
call's rows, in numbers that no product with the heads of a group wraps."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

INT_MAX, INT_MIN = 2 ** 31 - 1, -2 ** 31


def test_request_rows_are_cut_off_before_they_are_counted(tmp_path):
    ends = [INT_MIN, INT_MIN + 1, -5, -2, -1, 0, 1, 2, 4, 5, 6, 7, 8, 100, 1 << 20, (1 << 20) + 1, 1 << 30, INT_MAX - 1, INT_MAX]
    src = tmp_path / "request_rows.hip"
    src.write_text('''#include <stdio.h>
#include "kv8.h"
int main() {
    const int32_t ends[] = {%s};
    for (int32_t rows : {0, 1, 7, 1 << 20})
        for (int32_t a : ends)
            for (int32_t b : ends) {
                const pipo::RequestRows r = pipo::request_rows(a, b, rows);
                printf("%%d %%d %%d %%d %%d\\n", rows, a, b, r.first, r.n);
            }
    return 0;
}''' % ", ".join("INT32_MIN" if e == INT_MIN else str(e) for e in ends))
    exe = tmp_path / "request_rows"
    subprocess.run([HIPCC, "--offload-host-only", "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2605_27255_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    got = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines()
    assert len(got) == 4 * len(ends) ** 2
    for line in got:
        rows, a, b, first, n = map(int, line.split())
        want = range(rows)[max(a, 0):max(b, 0)]         # (a slice of the rows: empty where they end before they begin)
        assert n == len(want) and 0 <= first <= rows and first + n <= rows and (n == 0 or first == want[0]), line
        assert n * 16 < 2 ** 31 and first * 16 < 2 ** 31
