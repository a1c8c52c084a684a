"""The rule by which a product takes its form, compiled from the library's source for the host, against the tests' own copy."""
import ctypes
import pathlib
import subprocess

import numpy as np
import pytest

import fp8_forms as forms

CSRC = pathlib.Path(__file__).resolve().parents[1] / "paper_2609_03844_amd" / "csrc"
FORMS = ("rows", "64", "128", "256")


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    source = (CSRC / "sbw_fp8.hip").read_text()
    part = source[source.index("enum class Form"):source.index("int64_t part_pitch")]
    code = f"""#include <algorithm>
#include <cstdint>
constexpr int kBlock = 128;
inline int64_t blocks_of(int64_t n) {{ return (n + kBlock - 1) / kBlock; }}
{part}
extern "C" int64_t rule(int64_t M, int64_t N, int64_t K, int inside, int direct) {{
  const Plan p = plan_of(M, N, K, inside != 0, direct != 0);
  return p.parts * 4 + static_cast<int>(p.form);
}}
"""
    at = tmp_path_factory.mktemp("rule")
    (at / "rule.cpp").write_text(code)
    subprocess.run(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", str(at / "rule.cpp"), "-o", str(at / "rule.so")], check=True)
    call = ctypes.CDLL(str(at / "rule.so")).rule
    call.restype, call.argtypes = ctypes.c_int64, [ctypes.c_int64] * 3 + [ctypes.c_int] * 2
    return call


def test_forms_are_the_librarys(rule):
    rng = np.random.default_rng(0)
    sizes = np.exp2(rng.uniform(0, [12, 17, 15], (20000, 3))).astype(np.int64)
    for M, N, K in [*sizes.tolist(), *(s[:3] for s in forms.WIDE_SIZES)]:
        for inside in (False, True):
            for direct in (False, True):
                got = rule(M, N, K, inside, direct)
                assert (FORMS[got % 4], got // 4) == forms.plan_of(M, N, K, inside, direct), (M, N, K, inside, direct)


def test_the_wide_sizes_reach_what_they_are_for():
    """Every path of the 256 x 256 forms: scales as words of memory or as bytes, turned starts, parts of K and ends of K."""
    reached = set()
    for M, N, K, inside, *_ in forms.WIDE_SIZES:
        form, parts = forms.plan_of(M, N, K, inside, True)
        assert form == "256", (M, N, K)
        each, parts = forms.parts_taken(parts, K)
        blocks = forms.blocks_of(K)
        # product_tiles_kernel's own conditions
        in_tiles = inside and K % 16 == 0
        reached.add((in_tiles, parts > 1, K % 16 != 0, blocks % 4 == 0, in_tiles and each % 4 == 0 and each >= 32))
    for wanted in ((True, False, False, True, True),        # one part, words, turned starts: a head's logits
                   (True, False, False, False, False),      # one part, bytes
                   (True, True, False, True, True),         # parts of K, words
                   (True, True, False, False, True),        # parts of K, bytes: a head's gradient of the hidden states
                   (False, False, True, False, False),      # columns that end inside 16
                   (False, False, False, True, False)):
        assert wanted in reached, wanted
