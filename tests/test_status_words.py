"""The device status is kept in a word per file of kernels: a read or a clear that fails loses no timeout.  A small program
compiled against the header, with words that fail on demand (no GPU)."""
import shutil
import subprocess

import pytest

from paper_2509_26092_gb300 import build_lib

PROGRAM = r"""
#include <cstdio>
#include "dbl_status.cuh"

static int word[3], fail_read = -1, fail_clear = -1;
template <int I> int read(int* v) { *v = word[I]; return fail_read == I ? DBL_ERR_CUDA : DBL_OK; }
template <int I> int clear() { if (fail_clear == I) return DBL_ERR_CUDA; word[I] = DBL_OK; return DBL_OK; }

int main()
{
    const dbl::StatusWord words[] = {{read<0>, clear<0>}, {read<1>, clear<1>}, {read<2>, clear<2>}};
    int bad = 0, n = 0;
    for (int set = 0; set < 8; ++set)
        for (int r = -1; r < 3; ++r)
            for (int c = -1; c < 3; ++c, ++n) {
                for (int i = 0; i < 3; ++i) word[i] = set >> i & 1 ? DBL_ERR_TIMEOUT : DBL_OK;
                fail_read = r, fail_clear = c;
                int status = 12345;
                const int rc = dbl::take_status_words(words, 3, &status);
                const int want = set ? DBL_ERR_TIMEOUT : DBL_OK;
                if (rc == DBL_OK && status != want) bad = 1, std::printf("%d %d %d: status %d\n", set, r, c, status);
                if ((rc == DBL_OK) != (r < 0 && !(c >= 0 && set >> c & 1))) bad = 1, std::printf("%d %d %d: rc %d\n", set, r, c, rc);
                fail_read = fail_clear = -1;
                int again = 12345;
                if (dbl::take_status_words(words, 3, &again) != DBL_OK) bad = 1;
                // what a failed call did not report the next one does; what was reported is gone
                if (again != (rc == DBL_OK ? DBL_OK : want)) bad = 1, std::printf("%d %d %d: then %d\n", set, r, c, again);
            }
    return bad || n != 128;
}
"""


def test_a_failed_call_loses_no_timeout(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    src, exe = tmp_path / "words.cpp", tmp_path / "words"
    src.write_text(PROGRAM)
    r = subprocess.run([cxx, "-std=c++17", "-Wall", "-I", build_lib.CSRC, "-I", build_lib.INCLUDE, str(src), "-o", str(exe)],
                       capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout
