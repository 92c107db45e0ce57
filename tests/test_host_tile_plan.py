"""CPU-only tests of the rule that chooses workgroups for the attention of prompts and of drafted trees (csrc/tile_plan.h)."""

import random
import re
import shutil
import subprocess

import numpy as np
import pytest

import tile_plan
from paper_2508_15806_amd import binding as B
from tile_cases import PROMPTS, TREES

ALL = {(dtype, d, waves) for dtype in range(5) for d in (64, 128) for i, waves in enumerate(tile_plan.shapes()) if tile_plan.has_shape(dtype, d, i)}


def draws(seed, count):
    rng = random.Random(seed)
    for _ in range(count):
        Hkv, G, d = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 8, 16, 32]), rng.choice([64, 128])
        seqs = int(2 ** rng.uniform(0, 5))
        n = [int(2 ** rng.uniform(0, 12)) for _ in range(seqs)]
        h = rng.choice([0, 0, 1])
        m = [x + int(h * 2 ** rng.uniform(0, 15)) for x in n]
        yield rng, Hkv, G, d, seqs, n, m


def cu(x):
    return np.concatenate([[0], np.cumsum(x)])


def test_every_program_of_the_library_is_reached():
    """The kernels that are built, the shapes that the rule knows, and those that some call takes are the same."""
    nm = shutil.which("nm") or "/opt/rocm/llvm/bin/llvm-nm"
    names = subprocess.run([nm, "-DC", B.LIB_PATH], check=True, capture_output=True, text=True).stdout
    for table, dtypes in (("PromptTab", range(4)), ("PromptTabOne", range(1, 4)), ("TreeTab<64>", range(5)), ("TreeTab<600>", range(5))):
        for kernel in ("attend_tiles_kernel", "join_tiles_kernel")[:1 if table == "PromptTabOne" else 2]:
            built = {(int(k), int(d), (int(q), int(w))) for k, d, q, w in re.findall(r" slkv::%s<(\d+), (\d+), (\d+), (\d+), slkv::%s ?>" % (kernel, re.escape(table)), names)}
            assert built == {x for x in ALL if x[0] in dtypes}, (kernel, table)
    prompts, trees = set(), set()
    for rng, Hkv, G, d, seqs, n, m in draws(1, 6000):
        dtype = rng.randrange(4)
        prompts.add((dtype, d, tile_plan.prompt(B.PromptBatch(dtype, seqs, G * Hkv, Hkv, d, cu(n), cu(m))).waves))
        dtype, T, room = rng.randrange(5), int(2 ** rng.uniform(0, 6.01)), int(2 ** rng.uniform(3, 14))
        trees.add((dtype, d, tile_plan.tree(B.CacheLayout(dtype, seqs, G * Hkv, Hkv, d, np.arange(seqs * Hkv + 1) * room), T).waves))
    assert prompts == {x for x in ALL if x[0] < 4} and trees == ALL


def test_the_plan_is_the_librarys():
    for rng, Hkv, G, d, seqs, n, m in draws(2, 200):
        batch = B.PromptBatch(rng.randrange(4), seqs, G * Hkv, Hkv, d, cu(n), cu(m))
        assert tile_plan.prompt(batch).workspace == B.slkv_prompt_workspace_bytes(batch)
        lay, T = B.CacheLayout(rng.randrange(5), seqs, G * Hkv, Hkv, d, cu(np.repeat(m, Hkv))), rng.randint(1, 64)
        assert tile_plan.tree(lay, T).workspace == B.slkv_tree_workspace_bytes(lay, T)


@pytest.mark.parametrize("n,m,in_order", [([2000] * 8, None, True), ([110, 900], None, True), ([110, 4000, 3000, 900, 2500], None, False), ([3000] * 5, [3000] * 4 + [3100], False)])
def test_order_of_tiles(n, m, in_order):
    plan = tile_plan.prompt(B.PromptBatch(B.SLKV_BF16, len(n), 32, 8, 128, cu(n), None if m is None else cu(m)))
    assert plan.in_order == in_order and not plan.split


CODES = {"f32": B.SLKV_F32, "bf16": B.SLKV_BF16, "f16": B.SLKV_F16, "bf16_kv8": B.SLKV_BF16_KV_FP8, "bf16_kv4": B.SLKV_BF16_KV_MXFP4}


@pytest.mark.parametrize("dtype,d,waves,kind,Hq,Hkv,n,m", PROMPTS)
def test_programs_of_the_prompt_cases(dtype, d, waves, kind, Hq, Hkv, n, m):
    plan = tile_plan.prompt(B.PromptBatch(CODES[dtype], len(n), Hq, Hkv, d, cu(n), None if m is None else cu(m)))
    assert plan.waves == waves and plan.split == (kind == "split") and plan.in_order == (kind != "by keys")
    assert plan.blocks > 256 or plan.split or waves[0] * waves[1] == 4


@pytest.mark.parametrize("dtype,d,waves,kind,Hq,Hkv,seqs,T,room", TREES)
def test_programs_of_the_tree_cases(dtype, d, waves, kind, Hq, Hkv, seqs, T, room):
    plan = tile_plan.tree(B.CacheLayout(CODES[dtype], seqs, Hq, Hkv, d, np.arange(seqs * Hkv + 1) * room), T)
    assert plan.waves == waves and plan.split == (kind == "split")
    assert plan.blocks > 256 or plan.split or waves[0] * waves[1] == 4


def test_the_cases_are_all_programs():
    kinds = {(c[0], c[1], c[2], c[3]) for c in PROMPTS}
    for dtype in ("f32", "bf16", "f16", "bf16_kv8"):
        for d in (64, 128):
            for i, waves in enumerate(tile_plan.shapes()):
                if tile_plan.has_shape(CODES[dtype], d, i):
                    # (few queries of E4M3 rows: no call has so many tiles of them, of unequal sequences)
                    assert {k for k in ("split", "in order", "by keys") if (dtype, d, waves, k) in kinds} >= ({"split", "in order"} if (dtype, waves) == ("bf16_kv8", (1, 4)) else {"split", "in order", "by keys"})
    assert {(CODES[c[0]], c[1], c[2], c[3]) for c in TREES} == {x + (k,) for x in ALL for k in ("split", "whole")}
