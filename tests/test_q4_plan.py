"""Launch shapes of the 4-bit cache's operators (csrc/q4_plan.hpp, host arithmetic only),
compiled for the CPU."""
import ctypes as C
import os
import random
import subprocess

import pytest

from paper_2606_10944_amd import build as hip_build

CSRC = os.path.join(hip_build.HERE, "csrc")

SHIM = r"""
#include "q4_plan.hpp"
extern "C" {
void shape(int64_t B, int64_t H, int64_t G, int64_t T, int list, int64_t keys, int bf16,
           int64_t d, int64_t* out) {
  const thin::Q4AttnShape s = thin::q4_attention_shape(B, H, G, T, list != 0, keys, d, bf16 != 0);
  out[0] = s.waves;
  out[1] = s.splits;
  out[2] = s.least;
  out[3] = thin::q4_row_tiles(G, T, list != 0);
  out[4] = (int64_t)thin::q4_attention_bytes(B, H, out[3], s.splits, 128);
}
int64_t select_tokens(int64_t slices, int64_t blocks, int64_t T) {
  return thin::q4_select_tokens(slices, blocks, T);
}
int fused(int64_t slices, int64_t blocks, int64_t T) {
  return thin::q4_select_fused(slices, blocks, T);
}
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "shim.cpp").write_text(SHIM)
    so = d / "shim.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC,
                    str(d / "shim.cpp"), "-o", str(so)], check=True)
    lib = C.CDLL(str(so))
    lib.select_tokens.restype = C.c_int64
    return lib


def shape(plan, *a, d=128):
    out = (C.c_int64 * 5)()
    B, H, G, T, lst, keys, bf16 = a
    plan.shape(*[C.c_int64(x) for x in (B, H, G, T)], C.c_int(lst), C.c_int64(keys), C.c_int(bf16),
               C.c_int64(d), out)
    return list(out)


def test_attention_shapes_hold_what_the_kernels_assume(plan):
    rng = random.Random(0)
    kinds = set()
    for _ in range(20000):
        B = int(2 ** rng.uniform(0, 16))
        H = max(1, min(65535 // B, int(2 ** rng.uniform(0, 7))))
        G = int(2 ** rng.uniform(0, 10))
        T = 1 if rng.random() < 0.4 else int(2 ** rng.uniform(0, 20))
        lst, bf16 = rng.random() < 0.4, rng.random() < 0.5
        keys = 64 * rng.randint(1, 32768) if lst else int(2 ** rng.uniform(0, 21))
        waves, splits, least, tiles, ws = shape(plan, B, H, G, T, lst, keys, bf16,
                                                  d=rng.choice((32, 64, 128)))
        kinds.add((waves, splits > 1, lst))
        assert waves in (0, 4, 8) and 1 <= splits <= 512 and least >= 1
        assert waves or not lst  # lists have no kernel for many rows
        if splits > 1:
            # a sequence's shares fit the join, the table the launch's entries
            steps = -(-keys // 32)
            if waves and not lst:
                assert -(-steps // least) <= 512 and B <= 256 and B * splits > B
            assert B * H * tiles * splits < 2 ** 31
            slot = (16 * 128 + 32) * 4
            assert ws == B * H * tiles * splits * slot + tiles * B * 8
        else:
            assert ws == 0
    assert kinds == {(0, False, False), (0, True, False), (4, False, False), (4, True, False),
                     (8, False, False), (4, False, True), (4, True, True), (8, False, True)}


@pytest.mark.parametrize("a,want", [
    ((8, 8, 4, 1, 0, 65536, 1), (4, 8)),       # a step over long caches: 512 workgroups
    ((2, 4, 4, 1, 0, 1000, 0), (8, 1)),        # short caches: one launch
    ((256, 4, 4, 1, 0, 65536, 1), (4, 2)),     # many slices: in two, for unequal lengths
    ((32, 8, 4, 1, 0, 4096, 1), (8, 1)),       # a workgroup for every compute unit
    ((16, 8, 4, 1, 0, 4096, 1), (4, 4)),       # for half of them
    ((1, 8, 4, 4096, 0, 16384, 1), (0, 1)),    # a prompt
    ((1, 8, 4, 256, 0, 16384, 1), (0, 8)),     # a chunk: 64 workgroups share out 16384 rows
    ((1, 8, 4, 4096, 1, 2048, 1), (4, 1)),     # lists for every token of a prompt
])
def test_attention_shapes_of_ordinary_calls(plan, a, want):
    assert tuple(shape(plan, *a)[:2]) == want


def test_waves_follow_the_workgroups_a_compute_unit_holds(plan):
    for lst in (0, 1):
        for n, d, waves in ((256, 128, 8), (257, 128, 4), (257, 64, 8), (511, 32, 8), (512, 64, 4)):
            assert shape(plan, n, 1, 4, 1, lst, 1024, 1, d=d)[0] == waves


def test_selection_holds_bounded_scores(plan):
    rng = random.Random(1)
    for _ in range(5000):
        slices, blocks = int(2 ** rng.uniform(0, 16)), int(2 ** rng.uniform(0, 15))
        T = int(2 ** rng.uniform(0, 20))
        n = plan.select_tokens(C.c_int64(slices), C.c_int64(blocks), C.c_int64(T))
        assert 1 <= n <= T
        assert n == 1 or n * slices * blocks * 8 <= 64 << 20
        if plan.fused(C.c_int64(slices), C.c_int64(blocks), C.c_int64(T)):
            # 16 tokens' scores and the queries' parts (d = 128) in LDS
            assert 16 * ((blocks + 15) // 16 * 16 + 4) * 4 + 16384 + 1024 <= 160 * 1024
