"""How the gated delta rule cuts its sequences into pieces (csrc/la_delta_cut.h), without a GPU."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def cuts(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("cut") / "delta_cut_probe")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", os.path.join(ROOT, "tests", "delta_cut_probe.cpp"), "-o", exe], check=True)

    def run(sizes, element):
        """[(heads, D, M, chunks)], bytes of an element -> [(pieces, chunks a piece)]"""
        lines = subprocess.run([exe], input="\n".join(" ".join(map(str, (*s, element))) for s in sizes), capture_output=True, text=True, check=True).stdout.split("\n")
        return [tuple(map(int, line.split())) for line in lines if line]

    return run


def sizes():
    rng = random.Random(5)
    out = [(int(2 ** rng.uniform(0, 14)), rng.choice((32, 64, 128)), 16 * rng.randint(1, 32), int(2 ** rng.uniform(0, 15))) for _ in range(3000)]
    return out + [(h, D, 64, n) for h in (1, 2, 16) for D in (32, 64, 128) for n in (*range(1, 200), 1 << 14, 1 << 25)]


@pytest.mark.parametrize("element", [2, 4])
def test_pieces_cover_every_chunk_once_and_none_is_empty(cuts, element):
    for size, (pieces, length) in zip(sizes(), cuts(sizes(), element)):
        chunks = size[3]
        assert 1 <= pieces <= 64 and (pieces - 1) * length < chunks <= pieces * length, (size, pieces, length)


@pytest.mark.parametrize("element", [2, 4])
def test_few_long_sequences_are_cut_and_many_are_not(cuts, element):
    for D in (32, 64, 128):
        for chunks in (32, 128, 1024):
            assert cuts([(1, D, 64, chunks)], element)[0][0] >= 4
            assert cuts([(1024, D, 64, chunks), (512, D, 128, chunks)], element) == [(1, chunks)] * 2
        assert cuts([(1, D, 64, 1), (1, D, 64, 2)], element) == [(1, 1), (1, 2)]


def test_the_workspaces_have_room_for_the_pieces(cuts):
    from paper_2006_16236_amd import binding
    lib = binding.raw()
    up = lambda n: -(-n // 256) * 256
    rng = random.Random(6)
    for code, C, tri in ((0, 32, 32 * 32), (1, 64, 96 * 32)):
        some = [(rng.randint(1, 5), rng.randint(1, 9), rng.choice((32, 64, 128)), 16 * rng.randint(1, 12), int(2 ** rng.uniform(0, 15))) for _ in range(300)]
        for (B, H, D, M, N), (pieces, _) in zip(some, cuts([(B * H, D, M, -(-N // C)) for B, H, D, M, N in some], 2 if code else 4)):
            units, cut = B * H * -(-N // C), B * H * pieces if pieces > 1 else 0
            fwd = up(units * 2 * tri * 4) + up(units * 4 * C * 4) + up(cut * D * M * 4) + up(cut * D * D * 4)
            kept, back = up(units * C * M * 4) + up(units * D * M * 4), up(units * C * M * 4) + up(units * D * M * 4) + up(cut * D * M * 4)
            assert lib.la_delta_fwd_workspace(B, N, H, 1, D, M, code, 0) == fwd
            assert lib.la_delta_fwd_workspace(B, N, H, 1, D, M, code, 1) == fwd + kept
            assert lib.la_delta_bwd_workspace(B, N, H, 1, D, M, code, 1) == back
            assert lib.la_delta_bwd_workspace(B, N, H, 1, D, M, code, 0) == back + fwd + kept
