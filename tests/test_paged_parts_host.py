"""Which part of a paged attention launch every workgroup finds, on the host: the kernels' own search, its lanes run in turn."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

from paper_2512_24086_amd import build as b
from paper_2512_24086_amd import rf2

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def parts(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("parts") / "parts.so")
    rocm = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(b.hipcc()))), "include")
    subprocess.run(["g++", "-std=c++17", "-O2", "-U_FORTIFY_SOURCE", "-w", "-shared", "-fPIC", "-I", rocm, "-I", os.path.join(b.ROOT, "include"),
                    "-I", b.CSRC, os.path.join(HERE, "paged_parts_host.cpp"), "-o", lib], check=True)
    fn = C.CDLL(lib).paged_parts

    def of(heads, kv, new, ctx, pad=0, d=64, page=64, row=None):
        """(rows of a tile, [workgroups, 9], joints listed, joints and places there are) of a launch."""
        lens = np.array(new, dtype=np.int32) + np.array(ctx, dtype=np.int32)
        cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        n_tokens = int(cu[-1]) + pad
        row = row or max(1, -(-int(lens.max()) // page))
        cfg = rf2.rf2_paged_config(heads, kv, d, page, 1, len(new), row, n_tokens, 0, 1, 0.0)
        about, room = np.zeros(4, dtype=np.int32), 1 << 20
        found = np.zeros((room, 9), dtype=np.int32)
        grid = fn(C.byref(cfg), len(new), n_tokens, *(x.ctypes.data_as(C.c_void_p) for x in (lens, cu, found)), C.c_int64(room),
                  about.ctypes.data_as(C.c_void_p))
        assert grid > 0
        return int(about[0]), found[:grid], int(about[1]), int(about[2]), int(about[3])
    return of


def check(heads, kv, new, ctx, rows, found, listed, most_joints, places):
    """Every tile of every K/V head is taken once, in parts that cover its keys; places and joints are a part's and a tile's own."""
    group, of_joint = heads // kv, 2 if rows < 128 else 8
    mine = found[found[:, 0] == 1]
    seq, head, tile, chunk, tiles, units, place, joint = mine[:, 1:].T
    assert (head >= 0).all() and (head < kv).all() and (tile >= 0).all() and (tile < tiles).all() and (chunk >= 0).all()
    spots, lists = [], []
    for s, (n, x) in enumerate(zip(new, ctx)):
        here = seq == s
        if n == 0:
            assert not here.any(), s
            continue
        its_tiles, all_units = -(-n * group // rows), max(1, -(-(n + x) // 32))
        assert here.any() and (tiles[here] == its_tiles).all() and len(set(units[here])) == 1, s
        chunks = int(chunk[here].max()) + 1
        assert (chunks - 1) * units[here][0] < all_units <= chunks * units[here][0], s
        number = (head[here].astype(np.int64) * its_tiles + tile[here]) * chunks + chunk[here]
        assert np.array_equal(np.sort(number), np.arange(kv * its_tiles * chunks)), (s, len(number), kv * its_tiles * chunks)
        if chunks == 1:
            assert (place[here] == -1).all(), s
            continue
        spots.append(place[here])
        # a tile's parts stand `tiles` places apart, and list their rows at one joint
        order = np.lexsort((chunk[here], tile[here], head[here]))
        by_tile, joints = place[here][order].reshape(-1, chunks), joint[here][order].reshape(-1, chunks)
        assert (np.diff(by_tile, axis=1) == its_tiles).all() and (joints == joints[:, :1]).all(), s
        for t in range(its_tiles):
            of_tile = -(-min(rows, n * group - t * rows) // of_joint)
            for h in range(kv):
                lists.append(np.arange(of_tile) + joints[h * its_tiles + t, 0])
    spots, lists = np.concatenate(spots or [[]]), np.concatenate(lists or [[]])
    assert len(set(spots)) == len(spots) and (not len(spots) or 0 <= spots.min() and spots.max() < places)
    assert np.array_equal(np.sort(lists), np.arange(listed)) and listed <= most_joints


CASES = {
    "one": dict(heads=2, kv=1, new=[1], ctx=[0]),
    "one_long": dict(heads=8, kv=2, new=[1], ctx=[20011]),
    "steps": dict(heads=32, kv=8, new=[1] * 64, ctx=[(i * 977) % 9000 for i in range(64)]),
    "short_chunks": dict(heads=32, kv=8, new=[6] * 20, ctx=[(i * 977) % 9000 for i in range(20)]),
    "prompts": dict(heads=8, kv=2, new=[200, 1, 77, 640, 33], ctx=[0, 500, 31, 129, 2000], pad=9),
    "mixed": dict(heads=16, kv=4, new=[1] * 12 + [700, 0, 1, 1], ctx=[(i * 431) % 6000 for i in range(16)]),
    "frames": dict(heads=5, kv=5, new=[4680], ctx=[28080], d=128),
    "hundred": dict(heads=4, kv=1, new=[(i % 7 == 3) * 40 + i % 3 for i in range(100)], ctx=[(91 * i) % 500 for i in range(100)], d=128),
    "three_hundred": dict(heads=8, kv=8, new=[1] * 300, ctx=[(977 * i) % 60 + 9000 * (i % 150 == 7) for i in range(300)]),
    # more than 1,024 tiles that are not cut: of one sequence, behind one that is cut, of few rows
    "long_prompt": dict(heads=32, kv=8, new=[40000], ctx=[0]),
    "long_prompt_by_a_tile": dict(heads=32, kv=1, new=[4097], ctx=[0]),
    "long_prompt_40_heads": dict(heads=40, kv=40, new=[129000], ctx=[0], d=128),
    "cut_before_long": dict(heads=32, kv=8, new=[3200, 7360], ctx=[100000, 0], d=128),
    "long_before_many": dict(heads=32, kv=1, new=[5000] + [1] * 64, ctx=[0] * 65),
    "long_few_rows": dict(heads=16, kv=1, new=[2200] + [0, 1] * 900 + [0] * 2295, ctx=[0] * 4096),
    "long_32_rows": dict(heads=32, kv=1, new=[1100] + [0, 1] * 1400 + [0] * 1295, ctx=[0] * 4096),
    "thousand_chunks": dict(heads=3, kv=3, new=[20 + i % 9 for i in range(1000)], ctx=[(i * 131) % 300 for i in range(1000)]),
}


@pytest.mark.parametrize("name", list(CASES))
def test_every_tile_is_taken_once(name, parts):
    case = dict(CASES[name])
    check(case["heads"], case["kv"], case["new"], case["ctx"], *parts(**case))


@pytest.mark.parametrize("new", [[5000] + [1] * 64, [5000] + [1] * 63 + [2] * 66, [6000, 0, 3] + [0] * 100, [5000] + [1] * 255, [1100] + [0, 1] * 2047 + [0]],
                         ids=lambda new: f"{len(new)}_sequences")
def test_what_a_workgroup_finds_is_a_part(new, parts):
    """A prompt of more than 1,024 tiles before other sequences: no workgroup finds a head, a tile or a part that there is not, workgroup 0
    among them, which looks through all sequences."""
    rows, found, listed, most_joints, places = parts(32, 1, new, [0] * len(new))
    seq, head, tile, chunk, tiles, units, place, joint = found[found[:, 0] == 1][:, 1:].T
    held = np.array([-(-n * 32 // rows) for n in new])
    assert (held[seq] > 0).all() and (tiles == held[seq]).all()
    assert (head == 0).all() and (tile >= 0).all() and (tile < tiles).all() and (chunk >= 0).all()
    keys = np.maximum(-(-np.array(new) // 32), 1)
    assert (chunk * units < keys[seq]).all()
    assert (place < places).all() and ((place < 0) | (joint + rows // (2 if rows < 128 else 8) <= most_joints)).all()


@pytest.mark.parametrize("seed", range(8))
def test_batches_at_random(seed, parts):
    rng = np.random.default_rng(seed)
    for _ in range(4):
        kv, group, n = int(rng.choice([1, 2, 3, 5, 8, 16, 40])), int(rng.choice([1, 2, 4, 7, 12])), int(rng.choice([1, 2, 8, 40, 64, 65, 130, 257, 400]))
        longest, most = int(np.exp(rng.uniform(2, 11))), int(rng.choice([1, 4, 30, 200])) if n > 8 else int(rng.choice([1, 30, 2000]))
        new = np.where(rng.random(n) < 0.3, 0, rng.integers(1, most + 1, n))
        new[rng.integers(n)] = 1 if rng.random() < 0.6 else 20000 // (group * kv)
        case = dict(heads=kv * group, kv=kv, new=new.tolist(), ctx=rng.integers(0, longest, n).tolist(), pad=int(rng.choice([0, 0, 77])),
                    d=int(rng.choice([64, 128])), page=int(rng.choice([32, 256])))
        check(case["heads"], case["kv"], case["new"], case["ctx"], *parts(**case))
