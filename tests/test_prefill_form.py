"""The rule for prompt attention's row tiles (CPU: the host function itself)."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_24270_amd", "csrc")


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    """rule(name, arguments, ...) -> the values of a host function of prefill_form.h."""
    def run(name, *cases):
        d = tmp_path_factory.mktemp("form")
        src = d / "f.cpp"
        src.write_text('#include <cstdio>\n#include "prefill_form.h"\nint main() {\n' + "".join(
            f'std::printf("%d\\n", (int)asym::{name}({", ".join(map(str, c))}));\n' for c in cases) + "}\n")
        r = subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(d / "f")],
                           capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        return [int(x) for x in subprocess.run([str(d / "f")], capture_output=True, text=True).stdout.split()]
    return run


@pytest.fixture(scope="module")
def wide(rule):
    """wide((B, query heads a key/value head, key/value heads, T_q), ...) -> whether each takes 256-row tiles."""
    return lambda *cases: rule("prefill_wide", *cases)


def test_rows_that_fill_two_wide_tiles_a_cu(wide):
    assert wide((1, 4, 8, 16384), (1, 4, 8, 4096), (1, 4, 8, 4095), (8, 4, 8, 8191), (2, 1, 16, 8192), (1, 32, 1, 4096),
                (1, 128, 8, 2 ** 31 - 1), (0, 1, 1, 0)) == [1, 1, 0, 1, 1, 1, 1, 0]


def test_sequences_that_one_narrow_tile_holds(wide):
    # a verification step of 8 tokens, prompts of 16 and of 32 (128 rows), of 33; one token each; a long prompt among them
    assert wide((512, 4, 8, 512 * 8), (512, 4, 8, 512 * 16), (512, 4, 8, 512 * 32), (512, 4, 8, 512 * 33), (4200, 4, 8, 4200),
                (65, 1, 32, 65 * 128), (65, 1, 32, 65 * 129), (512, 4, 8, 511 * 8 + 16384)) == [0, 0, 0, 1, 0, 0, 1, 1]


def test_launches_that_32_bits_count(rule):
    assert rule("prefill_fits", ((1 << 23) - 1, "true"), (1 << 23, "true"), ((1 << 24) - 1, "false"), (1 << 24, "false")) == [
        1, 0, 1, 0]
    # what fits in wide tiles fits in narrow ones, of which there are twice as many at most: 128 rows and less a sequence
    B, heads = 690_000, 8
    rows = 128 * B
    assert rule("prefill_fits", ((rows // 256 + B) * heads, "true"), ((rows // 128 + B) * heads, "false")) == [1, 1]
