"""The tokens of the balance kernels' workgroups, on the host: the chunks of every group cover its tokens once, and no token's number
leaves 64 bits' range where tokens near 2^31 are stepped over, in chunks of none at the end of a short last group among them."""
import os
import shutil
import subprocess

import pytest

from paper_2512_10236_amd import _build

SOURCE = r"""
#include "ficco_token_run.h"
#include <cstdio>
#include <initializer_list>
#include <type_traits>
using namespace ficco;
// what the kernels do with a run: a thread's first token, and its next
static_assert(std::is_same<decltype(TokenRun{}.begin + 255), int64_t>::value && std::is_same<decltype(TokenRun{}.end), int64_t>::value, "64 bits");
int main()
{
    const int64_t all[] = {1, 2, 63, 1000, 65536, (1ll << 31) - 257, (1ll << 31) - 256, (1ll << 31) - 1};
    const int64_t sizes[] = {1, 7, 100, 4096, 1ll << 20, 3ll << 29, 1ll << 30, (1ll << 31) - 1};
    const int64_t parts[] = {1, 2, 3, 40, 1024};
    int64_t runs = 0;
    for (int64_t tokens : all)
        for (int64_t size : sizes)
            for (int64_t part : parts) {
                const int64_t group = size < tokens ? size : tokens, groups = (tokens + group - 1) / group;
                if (groups > 1 << 20) continue;
                const int64_t per_group = part < group ? part : group, each = (group + per_group - 1) / per_group;
                if (groups * per_group > 1 << 21) continue;
                int64_t next = 0;
                for (int64_t c = 0; c < groups * per_group; ++c, ++runs) {
                    const TokenRun r = token_run((int32_t)c, (int32_t)per_group, (int32_t)each, (int32_t)group, (int32_t)tokens);
                    const int64_t end = r.group + 1 < groups ? (r.group + 1) * group : tokens;
                    bool ok = r.group == c / per_group && r.begin == next && r.end >= r.begin && r.end <= end && r.end - r.begin <= each;
                    for (int thread : {0, 3, 255})               // past the end, never below zero
                        for (int64_t t = r.begin + thread, turn = 0; turn < 2; t += 256, ++turn) ok = ok && t >= 0;
                    if (c % per_group == per_group - 1) ok = ok && r.end == end;
                    if (!ok) { printf("tokens %ld group %ld per_group %ld chunk %ld: %ld..%ld\n", (long)tokens, (long)group, (long)per_group, (long)c, (long)r.begin, (long)r.end); return 1; }
                    next = r.end;
                }
                if (next != tokens) return 2;
            }
    printf("%ld runs\n", (long)runs);
    return 0;
}
"""


def test_runs_cover_all_tokens(tmp_path):
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("no g++")
    src, exe = tmp_path / "runs.cpp", str(tmp_path / "runs")
    src.write_text(SOURCE)
    r = subprocess.run([cxx, "-std=c++17", "-O1", "-I", _build.CSRC, str(src), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout
    assert int(r.stdout.split()[0]) > 1000


def test_the_kernels_take_their_tokens_from_it():
    """Every token of ficco_balance.hip comes from a run: no other loop bound or start has tokens in 32 bits."""
    with open(os.path.join(_build.CSRC, "ficco_balance.hip")) as f:
        text = f.read()
    kernels = text[:text.index("int checked(")]
    assert kernels.count("= chunk_run(a, blockIdx.x)") == 2
    assert "int t = " not in kernels and "int begin" not in kernels and "int64_t first = run.begin + sub" in kernels
