"""Which row arguments share memory, against a comparison byte by byte."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "strided_rows.h"
using micro::RowSpan;
int main() {
    std::srand(5);
    char* base = reinterpret_cast<char*>(1 << 20);
    long shared = 0, apart = 0;
    for (int n = 0; n < 400000; ++n) {
        RowSpan s[2];
        const int64_t stride = 1 + std::rand() % 12;
        for (RowSpan& r : s) {
            r.rows = std::rand() % 5;
            r.stride = stride;
            r.width = std::rand() % 4 == 0 ? stride : std::rand() % (stride + 1);
            if (r.rows < 2 && std::rand() % 2) r.stride = r.width = std::rand() % 40;  // one run of any length
            r.at = base + std::rand() % 40;
        }
        bool meet = false;
        std::vector<char> taken(1000, 0);
        for (int64_t i = 0; i < s[0].rows; ++i)
            for (int64_t k = 0; k < s[0].width; ++k) taken[(const char*)s[0].at - base + i * s[0].stride + k] = 1;
        for (int64_t i = 0; i < s[1].rows; ++i)
            for (int64_t k = 0; k < s[1].width; ++k) meet = meet || taken[(const char*)s[1].at - base + i * s[1].stride + k];
        if (micro::rows_share_bytes(s[0], s[1]) != meet || micro::rows_share_bytes(s[1], s[0]) != meet) {
            std::printf("wrong: %d\n", n);
            return 1;
        }
        ++(meet ? shared : apart);
    }
    // different strides: never taken for apart where they are not
    for (int n = 0; n < 400000; ++n) {
        RowSpan s[2];
        for (RowSpan& r : s) r = {base + std::rand() % 60, std::rand() % 5, 1 + std::rand() % 12, 0};
        for (RowSpan& r : s) r.width = std::rand() % (r.stride + 1);
        bool meet = false;
        std::vector<char> taken(1000, 0);
        for (int64_t i = 0; i < s[0].rows; ++i)
            for (int64_t k = 0; k < s[0].width; ++k) taken[(const char*)s[0].at - base + i * s[0].stride + k] = 1;
        for (int64_t i = 0; i < s[1].rows; ++i)
            for (int64_t k = 0; k < s[1].width; ++k) meet = meet || taken[(const char*)s[1].at - base + i * s[1].stride + k];
        if (meet && !micro::rows_share_bytes(s[0], s[1])) {
            std::printf("missed: %d\n", n);
            return 1;
        }
    }
    std::printf("%d\n", shared > 1000 && apart > 1000);
}
"""


def test_against_every_byte(tmp_path):
    src, exe = tmp_path / "rows.cpp", tmp_path / "rows"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-I",
                    os.path.join(ROOT, "paper_2310_00967_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.strip() == "1"
