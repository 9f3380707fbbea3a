"""The rules on sizes for products of 4-bit weights and for segments of the gated delta rule (csrc/q8_route.h, here as plain C): the sizes of the GPU
tests reach every kernel that the rules choose."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import test_gpu_delta_segments as segments
import test_gpu_w4_ranges as ranges
import test_gpu_w4_tiles as tiles

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FORMS = ["stream", "32x32, four groups of waves", "64x32, four", "64x32, two", "128x32", "128x64", "128x96", "256x64"]


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("route") / "q8_route_host.so")
    subprocess.run(["gcc", "-O2", "-std=c11", "-Wall", "-Werror", "-shared", "-fPIC", "-I" + os.path.join(ROOT, "paper_1804_05038_amd", "csrc"),
                    os.path.join(ROOT, "tests", "support", "q8_route_host.c"), "-o", so, "-lm"], check=True)
    return ctypes.CDLL(so)


def test_every_form_of_the_products_has_sizes(lib):
    assert list(tiles.TILES) == FORMS and all(len(v) >= 2 for v in tiles.TILES.values())


@pytest.mark.parametrize("form,rows,cols,n", tiles.CASES)
def test_sizes_take_their_form(lib, form, rows, cols, n):
    for group in (32, 64, 128):
        got = FORMS[lib.q8x_w4_route(rows, cols, n, group, 1)]
        assert got == (form if form != "256x64" or group > 32 else "128x64")        # (the finest groups' numbers do not fit into the registers there)


def test_scales_of_any_size_are_tested_in_every_form(lib):
    assert {FORMS[lib.q8x_w4_route(*size, group, 1)] for size in ranges.FORMS for group in (32, 64, 128)} == set(FORMS)


def test_results_over_the_vectors_go_in_two_launches(lib):
    for rows, cols, n in tiles.TILES["stream"]:
        assert FORMS[lib.q8x_w4_route(rows, cols, n, 64, 0)] != "stream"


def test_forms_of_drawn_sizes_are_the_known_ones(lib):
    rng = np.random.default_rng(0)
    seen = set()
    for _ in range(20000):
        rows, cols, n = (int(np.exp(rng.uniform(np.log(a), np.log(b)))) for a, b in ((1, 1 << 24), (1, 16385), (1, 1 << 20)))
        seen.add(lib.q8x_w4_route(rows, cols, n, int(rng.choice([32, 64, 128])), 1))
    assert seen <= set(range(len(FORMS))) and len(seen) >= 7


@pytest.mark.parametrize("lengths,hk,hv,dk,dv,edges,off16", segments.SEGMENTED)
def test_long_sequences_go_in_segments(lib, lengths, hk, hv, dk, dv, edges, off16):
    assert lib.q8x_delta_segment(5 + sum(lengths) + 3, len(lengths), hv, dk, dv) >= 4
    assert lib.q8x_delta_segment(sum(lengths), len(lengths), hv, dk, dv) >= 4


def test_every_width_goes_in_segments(lib):
    """Keys up to 64, 128 and 256 numbers, each in whole pieces and not; values in one slice of the first pass and in more."""
    kinds = {((dk > 64) + (dk > 128), dk % 4 == 0 and dv % 4 == 0 and not off16) for _, _, _, dk, dv, _, off16 in segments.SEGMENTED}
    assert kinds == {(w, v) for w in range(3) for v in (False, True)}
    assert {(dv + 63) // 64 for _, _, _, _, dv, _, _ in segments.SEGMENTED} >= {1, 2, 3}


def test_the_other_tests_that_speak_of_segments(lib):
    """test_gpu_delta_finite and test_gpu_delta_ranges."""
    assert lib.q8x_delta_segment(2048, 1, 2, 32, 40) >= 4
    assert lib.q8x_delta_segment(1200, 1, 2, 48, 36) >= 4 and lib.q8x_delta_segment(1200, 1, 2, 64, 32) >= 4


def test_segments_end_before_the_sequence_does(lib):
    """Any sizes: none, or at least four chunks, and at least two segments for each sequence."""
    rng = np.random.default_rng(1)
    for _ in range(20000):
        L, S, hv, dk, dv = (int(np.exp(rng.uniform(0, np.log(b)))) for b in (1 << 24, 65537, 1025, 257, 257))
        seg = lib.q8x_delta_segment(L, S, hv, dk, dv)
        assert seg == 0 or (seg >= 4 and 2 * seg * S <= L // 32)
