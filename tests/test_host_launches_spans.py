"""What the host side launches for windows with sinks, trees, rows at positions and kept rows, with the launches recorded instead of
made, and the ranges and work that its workgroups compute for themselves.  No GPU."""
import ctypes
import itertools
import os
import random
import subprocess

import numpy as np
import pytest

from paper_2501_05408_amd import tempo as T
from spans_cases import WIDE
from spans_reference import sees_chain, sees_tree

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
AT = 1 << 20                              # pointers that are checked for NULL and alignment, never read
STORES = [T.TEMPO_BF16, T.TEMPO_E4M3, T.TEMPO_F32]


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    path = str(tmp_path_factory.mktemp("host") / "host_launches_spans.so")
    subprocess.check_call(
        ["g++", "-std=c++17", "-O1", "-w", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-D__HIP_PLATFORM_AMD__", "-x", "c++",
         "-fsanitize=signed-integer-overflow", "-fsanitize-undefined-trap-on-error",
         os.path.join(ROOT, "tests", "host_launches_spans.cpp"), "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"),
         "-I", os.path.join(ROOT, "paper_2501_05408_amd", "csrc"), "-o", path])
    lib = ctypes.CDLL(path)
    for name, (res, args) in T.SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    lib.host_launches_take.restype = ctypes.c_char_p
    return lib


def taken(lib):
    out = []
    for line in lib.host_launches_take().decode().splitlines():
        name, *fields = line.split()
        out.append((name, {k: int(v) for k, v in (f.split("=") for f in fields)}))
    return out


def store(Hkv, D, Z, columns, dtype):
    return T.make_kv(AT, AT << 1, AT, 1 << 20, columns, Z, Hkv, D, dtype, 0)


def tile_range(lib, *args):
    out = (ctypes.c_int32 * 4)()
    lib.span_range_of(*args, out)
    return tuple(out)


# ---- ranges ----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("tree", [False, True])
def test_groups_of_a_tile_hold_every_key_that_its_rows_see_once(lib, tree):
    r = random.Random(3)
    for _ in range(2500):
        t, rows, G = r.randrange(0, 400), r.randrange(1, 60), r.choice([1, 2, 3, 5, 8, 20, 100])
        window = r.choice([0, 1, 2, 31, 32, 33, r.randrange(1, 300)]) if tree else r.choice([1, 2, 31, 32, 33, r.randrange(1, 300)])
        sinks = r.choice([0, 1, 31, 32, 33, r.randrange(0, 300)]) if window else 0
        columns = r.choice([16, 32, 128])
        parents = [r.randrange(-1, i) if i else -1 for i in range(rows)]
        seen = sees_tree(t, parents, window, sinks) if tree else sees_chain(t, rows, window, sinks)
        for tile in range((rows * G + columns - 1) // columns):
            first, last = tile * columns // G, min(((tile + 1) * columns - 1) // G, rows - 1)
            lo, sink_groups, g_lo, groups = tile_range(lib, t, tile, columns, G, rows, window, sinks, int(tree))
            numbers = [i if i < sink_groups else i - sink_groups + g_lo for i in range(groups)]
            assert numbers == [lib.span_group_of(t, 0 if tree else first, last, window, sinks, i) for i in range(groups)]
            assert len(set(numbers)) == groups and numbers == sorted(numbers) and numbers[-1] == (t + last) // 32
            wanted = {int(j) // 32 for j in np.nonzero(seen[first:last + 1].any(0))[0]}
            assert wanted <= set(numbers)
            # and little else: a tree's windows begin where its shallowest node's does
            if not tree:
                assert set(numbers) <= wanted | {n for n in numbers if n * 32 <= lo < n * 32 + 32 or n * 32 < sinks}
                assert lo == max(0, t + first - window + 1) if window else lo == 0


def test_ranges_far_out(lib):
    far = 2 ** 31 - 2000
    assert tile_range(lib, far, 0, 16, 1, 1, 2 ** 31 - 1, 2 ** 31 - 1, 0) == (0, 0, 0, far // 32 + 1)
    lo, sink_groups, g_lo, groups = tile_range(lib, far, 0, 16, 1, 16, 1000, 2 ** 31 - 1, 0)
    assert lo == far - 999 and sink_groups == g_lo == lo // 32 and groups == (far + 15) // 32 + 1
    assert tile_range(lib, far, 3, 128, 1, 512, 1, 4, 0) == (far + 384, 1, (far + 384) // 32, 1 + (far + 511) // 32 - (far + 384) // 32 + 1)


@pytest.mark.parametrize("Hkv", [1, 3, 8])
def test_all_wide_work_is_taken_once(lib, Hkv):
    out = (ctypes.c_int32 * 4)()
    for blocks, B, splits in itertools.product((1, 2, 8, 9, 13, 30), (1, 2, 5), (1, 2, 3)):
        for fewer in sorted({0, 1, blocks // 3, blocks - 1, blocks}):
            seen, dies = set(), {}
            for z, y, x in itertools.product(range(splits), range(B), range(Hkv * blocks)):
                lib.wide_work_of(x, y, z, Hkv * blocks, B, splits, Hkv, fewer, out)
                hkv, block, b, split = got = tuple(out)
                assert 0 <= hkv < Hkv and 0 <= block < blocks and 0 <= b < B and 0 <= split < splits
                seen.add(got)
                dies.setdefault((x + Hkv * blocks * (y + B * z)) % 8, []).append((b, hkv, split, -block))
            assert len(seen) == Hkv * blocks * B * splits
            if blocks > 8:                    # a die's blocks follow each other, those with fewer keys last, from the longest on
                units = Hkv * B * splits
                for run in dies.values():
                    most = [w for w in run if -w[3] >= fewer]
                    assert run[:len(most)] == most == sorted(most)
                    rest = run[len(most):]
                    if units % 8 == 0:
                        assert rest == sorted(rest, key=lambda w: (w[3], w[:3])) and len({w[:3] for w in rest}) <= units // 8


def test_blocks_with_fewer_keys(lib):
    r = random.Random(9)
    for _ in range(3000):
        t, window, G, tile, blocks = r.randrange(0, 300), r.randrange(1, 400), r.choice([1, 3, 8, 20, 128]), r.choice([32, 64, 96, 128]), r.randrange(9, 60)
        fewer = lib.fewer_keys_of(t, window, G, tile, blocks)
        assert fewer == sum(t + n * tile // G < window and t + n * tile / G < window for n in range(blocks))
    assert lib.fewer_keys_of(0, 0, 3, 128, 40) == 0 and lib.fewer_keys_of(2 ** 31 - 200, 2 ** 31 - 1, 128, 32, 2 ** 20) == 796
    assert lib.fewer_keys_of(0, 2 ** 31 - 1, 128, 32, 1000) == 1000


# ---- launches --------------------------------------------------------------------------------------------

def shapes(r):
    Hkv, G, D, Z = r.choice([1, 2, 8]), r.choice([1, 3, 4, 8, 16, 17, 32, 33, 64, 128]), r.choice([64, 128]), r.choice([32, 64, 256])
    return Hkv, G, D, Z, r.choice(STORES), r.choice([1, 2, 16, 100]), int(2 ** r.uniform(0, 20)) - 1


def check(lib, f, batch, Hq, G, D, rows, t, window, sinks, tree, nbytes, ragged):
    tiles = (rows * G + f["tile"] - 1) // f["tile"]
    assert f["tile"] in (16, 32, 64, 96, 128) and f["waves"] in (1, 2, 4, 8) and f["direct"] == (f["splits"] == 1)
    assert f["direct"] or f["end"] <= AT + nbytes  # partials lie in the workspace
    for at in ({t, 0, t // 2, max(0, t - 1), max(0, t - 31)} if ragged else {t}):
        for tile in {0, tiles // 2, tiles - 1}:
            groups = tile_range(lib, at, tile, f["tile"], G, rows, window, sinks, int(tree))[3]
            assert (groups + f["split_groups"] - 1) // f["split_groups"] <= f["splits"]


def test_trees_are_launched_whole_and_in_their_workspace(lib):
    r = random.Random(5)
    for _ in range(3000):
        Hkv, G, D, Z, dtype, batch, t = shapes(r)
        nodes, window = r.choice([1, 2, 8, r.randrange(1, 257), 256]), r.choice([0, 0, 1, int(2 ** r.uniform(0, 14))])
        sinks, ragged = r.choice([0, 4, r.randrange(0, 500)]) if window else 0, r.random() < 0.4
        kv = store(Hkv, D, Z, (t + nodes) // Z + 1, dtype)
        nbytes = lib.tempo_attn_tree_workspace_bytes(ctypes.byref(kv), batch, G * Hkv, nodes, t + r.choice([0, 0, 1000]), window, sinks)
        lib.host_launches_take()
        assert lib.tempo_attn_tree(ctypes.byref(kv), AT, AT, AT, AT if ragged else None, batch, G * Hkv, nodes, t, AT if ragged else None, window,
                                   sinks, 0.1, AT, nbytes, None) == T.TEMPO_OK
        (name, f), *rest = taken(lib)
        assert name == ("spans_f32" if dtype == T.TEMPO_F32 else "spans_wide" if f["tile"] > 32 else "spans") and f["tree"] == 1 and f["k"] == 0
        assert [n for n, _ in rest] == ([] if f["splits"] == 1 else ["combine_spans"])
        check(lib, f, batch, G * Hkv, G, D, nodes, t, window, sinks, True, nbytes, ragged)


def test_steps_with_sinks_write_their_row_once(lib):
    r = random.Random(6)
    for _ in range(3000):
        Hkv, G, D, Z, dtype, batch, t = shapes(r)
        window, sinks, ragged = int(2 ** r.uniform(0, 14)), r.choice([0, 4, r.randrange(0, 500)]), r.random() < 0.4
        kv = store(Hkv, D, Z, t // Z + 1, dtype)
        nbytes = lib.tempo_attn_sinks_workspace_bytes(ctypes.byref(kv), batch, G * Hkv, 1, t, window, sinks)
        lib.host_launches_take()
        assert lib.tempo_decode_step_sinks(ctypes.byref(kv), AT, 3 * AT, AT, AT, batch, G * Hkv, t, AT if ragged else None, window, sinks, 0.1, AT,
                                           nbytes, None) == T.TEMPO_OK
        names = taken(lib)
        fused = G <= 32 and dtype != T.TEMPO_F32
        if not fused:
            (name, f), *names = names
            assert name == "append" and f["t"] == t and f["count"] == 1 and f["k"] == 3 * AT
        (name, f), *rest = names
        assert name in (("spans_f32",) if dtype == T.TEMPO_F32 else ("spans", "spans_wide")) and f["k"] == (3 * AT if fused else 0) and f["tree"] == 0
        assert G > 32 or name != "spans_wide"
        assert [n for n, _ in rest] == ([] if f["splits"] == 1 else ["combine_spans"])
        check(lib, f, batch, G * Hkv, G, D, 1, t, window, sinks, False, nbytes, ragged)


def test_prompts_with_sinks_are_written_then_answered(lib):
    r = random.Random(7)
    for _ in range(2000):
        Hkv, G, D, Z, dtype, batch, t = shapes(r)
        count, window, sinks = int(2 ** r.uniform(0, 13)), int(2 ** r.uniform(0, 13)), r.choice([0, 4, r.randrange(0, 500)])
        if batch * count * Hkv * D >= 2 ** 31 or batch * count > 200000:
            continue
        kv = store(Hkv, D, Z, (t + count) // Z + 1, dtype)
        nbytes = lib.tempo_prefill_sinks_workspace_bytes(ctypes.byref(kv), batch, G * Hkv, t + count - 1 + r.choice([0, 0, 5000]))
        lib.host_launches_take()
        assert lib.tempo_prefill_sinks(ctypes.byref(kv), AT, AT, AT, AT, batch, G * Hkv, t, count, None, window, sinks, 0.1, AT, nbytes, None) == T.TEMPO_OK
        names = taken(lib)
        fused = count == 1 and G <= 32 and dtype != T.TEMPO_F32
        if not fused:
            (name, f), *names = names
            assert name == "append" and f["t"] == t and f["count"] == count
        (name, f), *rest = names
        assert [n for n, _ in rest] == ([] if f["splits"] == 1 else ["combine_spans"])
        check(lib, f, batch, G * Hkv, G, D, count, t, window, sinks, False, nbytes, False)


def test_calls_far_out_do_not_overflow(lib):
    for dtype, rows, window, sinks in itertools.product(STORES, (1, 5, 200), (1, 1000, 2 ** 31 - 1), (0, 4, 2 ** 31 - 1)):
        t = 2 ** 31 - 129 - rows
        kv = store(2, 128, 256, 1 << 24, dtype)
        for heads in (2, 8, 256):
            nbytes = lib.tempo_attn_sinks_workspace_bytes(ctypes.byref(kv), 3, heads, rows, t, window, sinks)
            assert nbytes > 0
            lib.host_launches_take()
            args = (ctypes.byref(kv), AT, AT, 3, heads, rows, t, AT, window, sinks, 0.1, AT)
            assert lib.tempo_attn_sinks(*args, nbytes, None) == T.TEMPO_OK
            (_, f), *_ = taken(lib)
            check(lib, f, 3, heads, heads // 2, 128, rows, t, window, sinks, False, nbytes, True)
        tree = lib.tempo_attn_tree_workspace_bytes(ctypes.byref(kv), 3, 8, rows, t, 0, 0)
        assert lib.tempo_attn_tree(ctypes.byref(kv), AT, AT, AT, None, 3, 8, rows, t, None, 0, 0, 0.1, AT, tree, None) == T.TEMPO_OK
        taken(lib)


def test_a_workspace_too_small_launches_nothing(lib):
    kv = store(8, 128, 64, 1000, T.TEMPO_BF16)
    nbytes = lib.tempo_attn_tree_workspace_bytes(ctypes.byref(kv), 1, 24, 8, 9000, 0, 0)
    lib.host_launches_take()
    for given in (0, 255, 256, nbytes // 200):
        assert lib.tempo_attn_tree(ctypes.byref(kv), AT, AT, AT, None, 1, 24, 8, 9000, None, 0, 0, 0.1, AT, given, None) == T.TEMPO_ERR_WORKSPACE
        assert lib.tempo_decode_step_sinks(ctypes.byref(kv), AT, AT, AT, AT, 1, 24, 3000, None, 2000, 4, 0.1, AT, given, None) == T.TEMPO_ERR_WORKSPACE
        assert lib.tempo_prefill_sinks(ctypes.byref(kv), AT, AT, AT, AT, 1, 24, 3000, 20, None, 2000, 4, 0.1, AT, given, None) == T.TEMPO_ERR_WORKSPACE
    assert taken(lib) == []


def test_rows_at_positions_and_kept_rows(lib):
    rope = T.tempo_rope(AT, AT, 500, 128)
    kv = store(8, 128, 64, 1000, T.TEMPO_BF16)
    axes = T.make_rope_axes([i % 3 for i in range(64)])
    assert lib.tempo_rope_kv_append_at(ctypes.byref(kv), ctypes.byref(rope), ctypes.byref(axes), AT, AT, AT, AT, AT, 2, 24, 7, None, 5, None, None) == T.TEMPO_OK
    assert lib.tempo_rope_kv_append_at(ctypes.byref(kv), ctypes.byref(rope), None, AT, AT, AT, None, None, 2, 0, 7, AT, 5, AT, None) == T.TEMPO_OK
    assert lib.tempo_rope_rotate_at(ctypes.byref(rope), None, AT, AT, AT, T.TEMPO_F32, 2, 5, 24, None) == T.TEMPO_OK
    (_, a), (_, b), (_, c) = taken(lib)
    bits = [sum((i % 3) << (2 * (i - at)) for i in range(at, at + 32)) for at in (0, 32)]
    assert (a["Hq"], a["Hrows"], a["axes"], a["rows"], a["low"], a["high"]) == (24, 8, 3, 500, bits[0], bits[1])
    assert (b["Hq"], b["Hrows"], b["axes"], b["low"], b["high"]) == (0, 8, 1, 0, 0) and (c["Hq"], c["Hrows"], c["k"]) == (24, 0, 0)
    layers = T.make_kv_layers([T.make_kv(AT * (2 * i + 3), AT * (2 * i + 4), AT, 100, 50, 64, 8, 128, T.TEMPO_BF16) for i in range(130)])
    assert lib.tempo_kv_keep(layers, 130, 4, 90, AT, 20, AT, 6, None) == T.TEMPO_OK
    got = taken(lib)
    assert [f["layers"] for _, f in got] == [64, 64, 2]
    assert [f["first"] for _, f in got] == [3 * AT, 131 * AT, 259 * AT] and [f["last"] for _, f in got] == [130 * AT, 258 * AT, 262 * AT]


def test_a_pool_twice_among_the_layers_is_refused(lib):
    one = T.make_kv(AT, 2 * AT, AT, 100, 50, 64, 8, 128, T.TEMPO_BF16)
    for k, v in ((AT, 3 * AT), (3 * AT, 2 * AT), (2 * AT, 3 * AT), (3 * AT, AT), (3 * AT, 3 * AT)):
        layers = T.make_kv_layers([one, T.make_kv(k, v, AT, 100, 50, 64, 8, 128, T.TEMPO_BF16)])
        assert lib.tempo_kv_keep(layers, 2, 4, 90, None, 20, AT, 6, None) == T.TEMPO_ERR_SHAPE
    assert taken(lib) == []


@pytest.mark.parametrize("dtype", STORES)
def test_calls_up_to_their_documented_limit_are_launched(lib, dtype):
    """Steps, heads and batches at the limits of one call and one beyond: launched, in a grid that fits, or refused with a size of 0."""
    most = 1 << (26 if dtype == T.TEMPO_F32 else 29)

    def call(batch, Hkv, G, D, rows, window, sinks, t=0):
        kv = store(Hkv, D, 256, 1 << 24, dtype)
        nbytes = lib.tempo_attn_sinks_workspace_bytes(ctypes.byref(kv), batch, Hkv * G, rows, t, window, sinks)
        lib.host_launches_take()
        status = lib.tempo_attn_sinks(ctypes.byref(kv), AT, AT, batch, Hkv * G, rows, t, None, window, sinks, 0.1, AT, nbytes, None)
        got = taken(lib)
        assert (status == T.TEMPO_OK) == bool(got) == (nbytes > 0) and status in (T.TEMPO_OK, T.TEMPO_ERR_SHAPE)
        for name, f in got[:1]:
            tiles = Hkv * ((rows * G + f["tile"] - 1) // f["tile"])
            assert tiles * 64 * f["waves"] < 2 ** 31 and tiles * batch * f["splits"] < 2 ** 31 and f["splits"] < 65536
        return status

    heads = [(1, 1), (8, 1), (1, 128), (8, 16), (500, 128), (65535, 1), (1000, 3)]
    for (Hkv, G), D, (window, sinks) in itertools.product(heads, (64, 128), ((1, 0), (1, 4), (300, 4), (5000, 33))):
        rows = most // (Hkv * G)
        if rows <= 1 << 24:
            assert call(1, Hkv, G, D, rows, window, sinks) == T.TEMPO_OK
            assert call(1, Hkv, G, D, rows + 1, window, sinks) == T.TEMPO_ERR_SHAPE
        else:
            assert call(1, Hkv, G, D, 1 << 24, window, sinks) == T.TEMPO_OK
            assert call(1, Hkv, G, D, (1 << 24) + 1, window, sinks) == T.TEMPO_ERR_SHAPE
    # workgroups of a batch
    for batch, Hkv, G, rows in ((65535, 32767, 1, 1), (65535, 8, 1, 65536), (60000, 8, 16, 4400)):
        fits = batch * Hkv * ((rows * G + 15) // 16) < 2 ** 31
        assert call(batch, Hkv, G, 64, rows, 300, 4) == (T.TEMPO_OK if fits else T.TEMPO_ERR_SHAPE)
    assert call(65535, 8, 1, 64, 65520, 300, 4) == T.TEMPO_OK and call(65535, 8, 1, 64, 65537, 300, 4) == T.TEMPO_ERR_SHAPE


def test_the_calls_whose_wide_answers_are_tested_go_wide(lib):
    """The cases of test_gpu_spans_wide.py, and that they take in what that kernel has: tiles of 64 to 128 columns, one range and many, steps and
    trees, both stores and head lengths, a window and a range more than 64 tiles long."""
    seen = set()
    for dtype, what, Hq, Hkv, D, Z, B, t, rows, window, sinks, ragged, counts in WIDE:
        kv = store(Hkv, D, Z, (t + rows) // Z + 1, dtype)
        lib.host_launches_take()
        at, n, ref, size = AT if ragged else None, AT if counts else None, ctypes.byref(kv), 1 << 40
        if what == "tree":
            assert lib.tempo_attn_tree(ref, AT, AT, AT, n, B, Hq, rows, t, at, window, sinks, 0.1, AT, size, None) == T.TEMPO_OK
        elif what == "block":
            assert lib.tempo_attn_sinks(ref, AT, AT, B, Hq, rows, t, at, window, sinks, 0.1, AT, size, None) == T.TEMPO_OK
        else:
            assert lib.tempo_prefill_sinks(ref, AT, AT, AT, AT, B, Hq, t, rows, n, window, sinks, 0.1, AT, size, None) == T.TEMPO_OK
        launches = dict(taken(lib))
        f = launches["spans_wide"]
        split, one_range = f["splits"] > 1, f["split_groups"] // (Z // 32)
        seen |= {(dtype, D, what, split), (dtype, D, f["tile"]), (dtype, what, rows > 64, window > 0)}
        if sinks and (t - window) // Z > 64:
            seen.add((dtype, D, "far"))
        if not split and one_range > 64:
            seen.add((dtype, D, "long"))
    for dtype, D in itertools.product((T.TEMPO_BF16, T.TEMPO_E4M3), (64, 128)):
        assert {(dtype, D, "far"), (dtype, D, "long"), (dtype, D, 128)} <= seen
        assert {(dtype, D, "prompt", False), (dtype, D, "prompt", True), (dtype, D, "tree", False)} <= seen
    assert {(T.TEMPO_BF16, 128, 64), (T.TEMPO_BF16, 128, 96), (T.TEMPO_E4M3, 128, 96), (T.TEMPO_E4M3, 64, 96)} <= seen
    for dtype in (T.TEMPO_BF16, T.TEMPO_E4M3):
        assert {(dtype, 128, "tree", True), (dtype, "tree", True, False), (dtype, "tree", True, True), (dtype, "tree", False, False)} <= seen
