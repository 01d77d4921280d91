"""How the selective scan cuts its sequences into pieces (csrc/la_scan_cut.h), forwards and backwards, without a GPU."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def cuts(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("cut") / "scan_cut_probe")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", os.path.join(ROOT, "tests", "scan_cut_probe.cpp"), "-o", exe], check=True)

    def run(sizes):
        """[(B, N, E, G, S)] -> [((tiles, pieces, piece_tiles) forwards, backwards)]"""
        text = "\n".join(" ".join(map(str, s)) for s in sizes)
        lines = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.split("\n")
        numbers = [tuple(map(int, line.split())) for line in lines if line]
        assert len(numbers) == len(sizes)
        return [(n[:3], n[3:]) for n in numbers]

    return run


def sizes():
    rng, out = random.Random(4), []
    for _ in range(4000):
        G = rng.choice((1, 1, 2, 4))
        out.append((int(2 ** rng.uniform(0, 9)), int(2 ** rng.uniform(0, 17)), G * int(2 ** rng.uniform(0, 11)), G, rng.choice((8, 16, 32))))
    out += [(1, n, 64, 1, S) for n in (*range(1, 300), 1 << 20, 1 << 30) for S in (8, 16, 32)]
    return out


def test_pieces_cover_every_tile_once_and_none_is_empty(cuts):
    for size, both in zip(sizes(), cuts(sizes())):
        for tiles, pieces, piece_tiles in both:
            assert tiles == -(-size[1] // 16), size
            assert 1 <= pieces and (pieces - 1) * piece_tiles < tiles <= pieces * piece_tiles, (size, tiles, pieces, piece_tiles)
            assert piece_tiles >= 4 or pieces == 1, (size, tiles, pieces, piece_tiles)


def test_few_long_sequences_are_cut_and_many_are_not(cuts):
    for S in (8, 16, 32):
        for N in (1000, 4096, 32768, 1 << 20):
            for _, pieces, _ in cuts([(1, N, 64, 1, S)])[0]:
                assert pieces >= N // 16 // 8 or pieces >= 32, (S, N, pieces)
        for (_, forward, _), (_, backward, _) in cuts([(256, 4096, 192, 1, S), (1, 4096, 64 * 768, 1, S), (1, 100, 64, 1, S), (8, 16, 64, 1, S)]):
            assert forward == backward == 1


def test_the_workspaces_have_room_for_the_pieces(cuts):
    from paper_2006_16236_amd import binding
    lib = binding.raw()
    up = lambda n: -(-n // 256) * 256
    some = [s for s in sizes() if s[0] * s[1] * s[2] < 1 << 36][:600]
    for (B, N, E, G, S), ((_, fwd, _), (_, bwd, _)) in zip(some, cuts(some)):
        room = lambda p: 0 if p < 2 else up(B * E * S * 4 * p) + up(B * p * E * 4)
        blocks, keep = G * -(-(E // G) // 64), up(B * E * S * 4 * -(-N // 16))
        sums = up(blocks * B * N * 2 * S * 4) + up(B * bwd * E * (S + 2) * 4)
        assert lib.la_scan_fwd_workspace(B, N, E, G, S, 0, 1) == room(fwd)
        assert lib.la_scan_fwd_workspace(B, N, E, G, S, 0, 3) == room(fwd) + keep
        assert lib.la_scan_bwd_workspace(B, N, E, G, S, 0, 3) == room(bwd) + sums
        assert lib.la_scan_bwd_workspace(B, N, E, G, S, 0, 1) == keep + max(room(fwd), room(bwd)) + sums
