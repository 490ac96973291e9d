"""What the host side launches for 8-bit stores and lists of blocks, with the launches recorded instead of made."""
import ctypes
import os
import random
import subprocess

import pytest

from paper_2501_05408_amd import tempo as T

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
AT = 1 << 20                              # pointers that are checked for NULL and alignment, never read
E4M3 = T.TEMPO_E4M3


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    path = str(tmp_path_factory.mktemp("host") / "host_launches_e4m3.so")
    subprocess.check_call(
        ["g++", "-std=c++17", "-O1", "-w", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-D__HIP_PLATFORM_AMD__", "-x", "c++",
         "-fsanitize=signed-integer-overflow", "-fsanitize-undefined-trap-on-error",
         os.path.join(ROOT, "tests", "host_launches_e4m3.cpp"), "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"),
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


def store(Hkv, D, Z, columns, ring=0, dtype=E4M3):
    return T.make_kv(AT, AT, AT, 1 << 20, columns, Z, Hkv, D, dtype, ring)


def assert_keys_launched(f, G, t, window, queries, tile):
    """The launched splits reach from the first key of the first step to the last step."""
    first = max(0, t - window + 1) if window else 0
    assert (t + queries - 1 >> f["tps_log2"]) - (first >> f["tps_log2"]) + 1 <= f["grid_splits"] <= f["num_splits"]


def test_every_visible_key_of_a_step_is_launched(lib):
    r = random.Random(1)
    for _ in range(3000):
        Hkv, G, D, Z = r.choice([1, 2, 8]), r.choice([1, 3, 4, 16, 17, 64, 128]), r.choice([64, 128]), r.choice([32, 64, 256])
        C = r.randrange(1, 128 // G + 1)
        batch, t = r.choice([1, 2, 16, 300]), int(2 ** r.uniform(0, 22)) - 1
        window, ragged = r.choice([0, 0, 1, int(2 ** r.uniform(0, 14))]), r.random() < 0.4
        kv = store(Hkv, D, Z, (t + C) // Z + 1)
        nbytes = lib.tempo_attn_block_workspace_bytes(ctypes.byref(kv), batch, G * Hkv, C, t)
        args = (ctypes.byref(kv), AT, AT, batch, G * Hkv, C, t, AT if ragged else None)
        lib.host_launches_take()
        rc = (lib.tempo_attn_block_window(*args, window, 0.1, AT, nbytes, None) if window
              else lib.tempo_attn_block_causal(*args, 0.1, AT, nbytes, None))
        if rc == T.TEMPO_ERR_SHAPE:      # batch * queries * heads beyond what the block entry points take
            continue
        assert rc == T.TEMPO_OK
        (name, f), *rest = taken(lib)
        assert name == "partial_e4m3" and f["waves"] in (1, 2, 4, 8) and f["waves"] * 32 <= 1 << f["tps_log2"]
        assert [n for n, _ in rest] == ([] if f["num_splits"] == 1 else ["combine"]) and f["direct"] == (f["num_splits"] == 1)
        assert f["num_splits"] * batch * C * G * Hkv * (D + 2) * 4 <= nbytes + 512
        assert_keys_launched(f, G, t, window, C, Z)
        if ragged:                       # any earlier step too
            for at in (0, t // 3, t // 2, max(0, t - 1)):
                first = max(0, at - window + 1) if window else 0
                assert (at + C - 1 >> f["tps_log2"]) - (first >> f["tps_log2"]) + 1 <= f["grid_splits"]


def prefill(lib, kv, batch, Hq, t, count, window=0, counts=None, nbytes=0, rows=AT, out=1 << 44, workspace=AT):
    lib.host_launches_take()
    args = (ctypes.byref(kv), AT, rows, rows, out, batch, Hq, t, count, counts)
    rc = (lib.tempo_prefill_window(*args, window, 0.1, workspace, nbytes, None) if window
          else lib.tempo_prefill_causal(*args, 0.1, workspace, nbytes, None))
    return rc, taken(lib)


def test_prompts_are_written_and_answered_once_within_the_promised_workspace(lib):
    r = random.Random(2)
    for _ in range(1500):
        Hkv, G, D, Z = r.choice([1, 2, 8]), r.choice([1, 3, 4, 17, 100]), r.choice([64, 128]), r.choice([32, 64, 256])
        batch, count, t = r.choice([1, 2, 16]), int(2 ** r.uniform(0, 12)), r.choice([0, 0, int(2 ** r.uniform(0, 14))])
        window, block, Hq = r.choice([0, 0, int(2 ** r.uniform(0, 12))]), 128 // G, G * Hkv
        ring = 0
        if window and r.random() < 0.5:
            ring = T.tempo_ring_blocks(window, Z, min(block, count))
        counts = AT if not ring and r.random() < 0.3 else None
        last = t + count - 1
        kv = store(Hkv, D, Z, ring or last // Z + 1, ring)
        nbytes = lib.tempo_prefill_workspace_bytes(ctypes.byref(kv), batch, Hq, ring * Z + 128 if ring else last)
        rc, launches = prefill(lib, kv, batch, Hq, t, count, window, counts, nbytes)
        assert rc == T.TEMPO_OK, (Hkv, G, D, Z, batch, count, t, window, ring)
        written = step = t
        copy = None
        for name, f in launches:
            if name == "append":
                assert f["t"] == written and f["steps"] == count and f["k"] == AT + (written - t) * Hkv * D * 2
                written += f["count"]
            elif name == "unpack":
                copy = f
                assert f["end"] <= AT + nbytes and f["table"] >= AT and f["k"] >= f["table"] + 4 * batch * f["tiles"]
            elif name in ("partial_e4m3", "prompt", "short_prompt"):
                C = f["queries"]
                assert f["t"] == step and written >= step + C and f["window"] == window and f["steps"] == count
                if ring:                 # no row the answers need has been written over
                    assert max(0, step - window + 1) // Z + ring > (written - 1) // Z
                if name == "partial_e4m3":
                    assert C * G <= 128
                else:                    # everything the steps see has been turned, into places of its own
                    lo = max(0, step - window + 1) if window else 0
                    assert copy["first"] == lo >> 5 and copy["first"] + copy["groups"] == (step + C - 1 >> 5) + 1
                    assert (step + C - 1) // Z - lo // Z + 1 <= copy["tiles"] if copy["mask"] != 2 ** 31 - 1 else (step + C - 1) // Z < copy["tiles"]
                    assert f["num_splits"] * batch * C * Hq * (D + 2) * 4 <= copy["table"] - AT + 512 or f["direct"]
                    copy = None
                step += C
        assert written == step == t + count
        if counts or count * G > 128:
            small = lib.tempo_attn_block_workspace_bytes(ctypes.byref(kv), batch, Hq, block, last) if not ring else 0
            if small and any(n == "unpack" for n, _ in launches):
                rc, launches = prefill(lib, kv, batch, Hq, t, count, window, counts, 4096)
                assert rc == T.TEMPO_ERR_WORKSPACE and not launches      # refused before anything is written
        else:
            assert not any(n == "unpack" for n, _ in launches) or ring


def test_two_blocks_behind_a_long_history_are_answered_over_the_codes(lib):
    for t, count, window, ways in ((100, 42, 0, ["partial_e4m3"]), (3000, 64, 0, ["partial_e4m3"] * 2), (1500, 64, 0, ["prompt"]), (3000, 64, 700, ["prompt"]),
                                   (3000, 43, 300, ["partial_e4m3"] * 2), (30000, 84, 0, ["partial_e4m3"] * 2), (30000, 85, 0, ["prompt"])):
        kv = store(8, 128, 64, (t + count) // 64 + 1)
        rc, launches = prefill(lib, kv, 2, 24, t, count, window, nbytes=1 << 40)
        assert rc == T.TEMPO_OK and [n for n, _ in launches if n in ("partial_e4m3", "prompt", "short_prompt")] == ways, (t, count, window)
        assert len(launches) <= lib.tempo_prefill_launches(ctypes.byref(kv), 2, 24, count)
        if len(ways) == 2:               # one after the other, in the call's own rows
            a, z = [f for n, f in launches if n == "partial_e4m3"]
            assert (a["t"], a["queries"], z["t"], z["queries"]) == (t, 42, t + 42, count - 42) and a["steps"] == z["steps"] == count
            assert z["out"] - a["out"] == 42 * 24 * 128 * 2


def test_prompts_keep_to_the_smallest_workspace_that_is_taken(lib):
    r = random.Random(4)
    up = lambda n: (n + 255) // 256 * 256  # noqa: E731
    for _ in range(250):
        Hkv, G, D, Z = r.choice([1, 2, 8]), r.choice([1, 3, 4, 17, 100]), r.choice([64, 128]), r.choice([32, 64, 256])
        batch, count, t = r.choice([1, 2, 16]), int(2 ** r.uniform(0, 11)), r.choice([0, 0, int(2 ** r.uniform(0, 14))])
        window, block, Hq = r.choice([0, int(2 ** r.uniform(0, 12))]), 128 // G, G * Hkv
        ring = T.tempo_ring_blocks(window, Z, min(block, count)) * r.choice([1, 2]) if window and r.random() < 0.7 else 0
        counts = AT if not ring and r.random() < 0.3 else None
        kv = store(Hkv, D, Z, ring or (t + count - 1) // Z + 1, ring)
        low, high = 0, lib.tempo_prefill_workspace_bytes(ctypes.byref(kv), batch, Hq, ring * Z + 128 if ring else t + count - 1)
        while low < high:                # (enough)
            middle = (low + high) // 2
            taken_at = prefill(lib, kv, batch, Hq, t, count, window, counts, middle)[0] == T.TEMPO_OK
            low, high = (low, middle) if taken_at else (middle + 1, high)
        for nbytes in (low, low + 1, low + 300):
            rc, launches = prefill(lib, kv, batch, Hq, t, count, window, counts, nbytes)
            assert rc == T.TEMPO_OK
            room = nbytes
            for name, f in launches:
                if name == "unpack":
                    assert f["end"] <= AT + nbytes
                    room = f["table"] - AT
                elif name in ("partial_e4m3", "prompt", "short_prompt"):
                    rows = batch * f["queries"] * Hq * f["num_splits"]
                    assert f["direct"] or up(rows * 8) + up(rows * D * 4) <= room
                    room = nbytes


def test_prompts_beyond_one_launchs_index_range_are_written_whole_before_answers(lib):
    Hkv, G, D, Z, batch, count = 8, 3, 128, 256, 64, 70000
    kv = store(Hkv, D, Z, count // Z + 1)
    rc, launches = prefill(lib, kv, batch, G * Hkv, 0, count, nbytes=1 << 45)
    assert rc == T.TEMPO_OK
    names = [n for n, _ in launches]
    chunks = names.count("append")
    assert chunks > 1 and names[:chunks] == ["append"] * chunks
    assert all(batch * f["count"] * Hkv * D <= 2 ** 31 - 1 for n, f in launches if n == "append")


def test_ring_prompts_whose_answers_lie_over_their_rows(lib):
    """Several chunks: the rows are copied first, or the call is refused; clear of the rows neither happens."""
    Hkv, G, D, Z, window, count, batch = 2, 3, 128, 64, 100, 1000, 2
    ring = T.tempo_ring_blocks(window, Z, 42)
    kv = store(Hkv, D, Z, ring, ring)
    need = lib.tempo_prefill_workspace_bytes(ctypes.byref(kv), batch, G * Hkv, ring * Z + 128)
    rows = 1 << 44
    bytes_of_rows = batch * count * Hkv * D * 2
    rc, launches = prefill(lib, kv, batch, G * Hkv, 0, count, window, nbytes=need + 2 * bytes_of_rows + 512, rows=rows, out=rows)
    assert rc == T.TEMPO_OK and [n for n, _ in launches][:2] == ["stream_copy"] * 2
    assert all(f["k"] != rows for n, f in launches if n == "append")
    seen = set()
    for nbytes in range(0, need + 1, need // 64):    # whatever the workspace holds: a copy is read, or nothing is launched
        rc, launches = prefill(lib, kv, batch, G * Hkv, 0, count, window, nbytes=nbytes, rows=rows, out=rows)
        apart, plain = prefill(lib, kv, batch, G * Hkv, 0, count, window, nbytes=nbytes, rows=rows, out=1 << 45)
        assert "stream_copy" not in [n for n, _ in plain] and (rc != T.TEMPO_OK or apart == T.TEMPO_OK)
        if rc == T.TEMPO_OK:
            assert [n for n, _ in launches][:2] == ["stream_copy"] * 2
        else:
            assert rc == T.TEMPO_ERR_WORKSPACE and not launches
        seen.add((rc, apart))
    assert seen == {(T.TEMPO_ERR_WORKSPACE, T.TEMPO_ERR_WORKSPACE), (T.TEMPO_ERR_WORKSPACE, T.TEMPO_OK), (T.TEMPO_OK, T.TEMPO_OK)}
    rc, launches = prefill(lib, kv, batch, G * Hkv, 0, count, window, nbytes=need, rows=rows, out=1 << 45)
    assert rc == T.TEMPO_OK and "stream_copy" not in [n for n, _ in launches]


@pytest.mark.parametrize("ragged", [False, True])
def test_no_alloc_steps_take_a_plan_that_fits_the_array(lib, ragged):
    for G, Hkv, D, batch, t in ((3, 8, 128, 64, 8191), (8, 8, 128, 64, 30000), (16, 1, 64, 500, 65535), (100, 4, 128, 20, 20000), (3, 8, 128, 1, 100)):
        kv = store(Hkv, D, 64, t // 64 + 1)
        lib.host_launches_take()
        rc = lib.tempo_decode_step_causal_noalloc(ctypes.byref(kv), AT, AT, AT, AT, batch, G * Hkv, t, AT if ragged else None, 0.1, None)
        launches = taken(lib)
        if rc == T.TEMPO_ERR_WORKSPACE:   # one split each already exceeds it
            assert batch * G * Hkv * (D + 2) * 4 > 8 << 20 or ragged
            continue
        assert rc == T.TEMPO_OK
        name, f = launches[0]
        assert name == "partial_e4m3" and f["num_splits"] * batch * G * Hkv * (D + 2) * 4 <= (8 << 20) and f["grid_splits"] >= (t >> f["tps_log2"]) + 1


@pytest.mark.parametrize("dtype", [T.TEMPO_BF16, E4M3])
def test_lists_are_launched_whole_within_the_promised_workspace(lib, dtype):
    r = random.Random(3)
    for _ in range(1500):
        Hkv, G, D, Z = r.choice([1, 2, 8]), r.choice([1, 3, 16, 17, 128]), r.choice([64, 128]), r.choice([32, 64, 256])
        batch, t, count = r.choice([1, 5, 64]), int(2 ** r.uniform(0, 20)), int(2 ** r.uniform(0, 13))
        kv = store(Hkv, D, Z, t // Z + 1, dtype=dtype)
        nbytes = lib.tempo_attn_selected_workspace_bytes(ctypes.byref(kv), batch, G * Hkv, count)
        lib.host_launches_take()
        rc = lib.tempo_attn_selected(ctypes.byref(kv), AT, AT, AT, count, batch, G * Hkv, t, None, 0.1, AT, nbytes, None)
        assert rc == T.TEMPO_OK
        (name, f), *rest = taken(lib)
        assert name == "selected" and f["num_splits"] == f["grid_splits"] == (count * Z - 1 >> f["tps_log2"]) + 1 <= 1024
        assert f["num_splits"] * batch * G * Hkv * (D + 2) * 4 <= nbytes + 512
        assert [n for n, _ in rest] == ([] if f["direct"] else ["combine_selected"])
        if rest:
            assert rest[0][1]["t"] == count * Z - 1


def test_launches_of_a_sparse_step(lib):
    kv = store(8, 128, 64, 1024)
    nbytes = lib.tempo_step_selected_workspace_bytes(ctypes.byref(kv), 2, 24, 65535, 32)
    for t in (5, 65471, 65535):
        lib.host_launches_take()
        assert lib.tempo_decode_step_selected(ctypes.byref(kv), AT, AT, AT, AT, AT, AT, 32, 1, 2, 2, 24, t, None, 0.1, AT, nbytes, None) == T.TEMPO_OK
        names = [n for n, _ in taken(lib)]
        assert names[:2] == ["select", "selected"] and len(names) <= 3
    for t, count, launched in ((0, 63, False), (0, 64, True), (63, 1, True), (64, 63, False), (100, 28, True), (100, 27, False)):
        lib.host_launches_take()
        assert lib.tempo_block_bounds(ctypes.byref(kv), AT, 2, t, None, count, None, None) == T.TEMPO_OK
        assert bool(taken(lib)) == launched
    # nothing is launched by a step that is refused
    assert lib.tempo_decode_step_selected(ctypes.byref(kv), AT, AT, AT, AT, AT, AT, 32, 1, 2, 2, 24, 65535, None, 0.1, AT, nbytes - 1, None) == T.TEMPO_ERR_WORKSPACE
    assert not taken(lib)


def assert_within_the_launches_promised(lib, kv, batch, Hq, t, count, window, out, counts=None):
    rows = 1 << 44
    rc, launches = prefill(lib, kv, batch, Hq, t, count, window, counts, nbytes=1 << 46, rows=rows, out=out)
    assert rc == T.TEMPO_OK
    bound = lib.tempo_prefill_launches(ctypes.byref(kv), batch, Hq, count)
    assert len(launches) <= bound, (kv.dtype, kv.ring_blocks, batch, Hq, t, count, window, [n for n, _ in launches], bound)
    return [n for n, _ in launches]


def test_prompts_keep_to_the_number_of_launches_promised(lib):
    # chunks of 64 and 20 steps deep in the sequence, two blocks over the codes and one; answers over the rows
    kv = store(8, 128, 32, 64, ring=64)
    names = assert_within_the_launches_promised(lib, kv, 1, 24, 32 * 10000, 84, 1950, 1 << 44)
    assert names.count("stream_copy") == 2 and names.count("partial_e4m3") == 3
    r = random.Random(5)
    for _ in range(3000):
        Hkv, G, D, Z = r.choice([1, 2, 8]), r.choice([1, 3, 4, 17, 100]), r.choice([64, 128]), r.choice([32, 64, 256])
        dtype = r.choice([E4M3, E4M3, T.TEMPO_BF16, T.TEMPO_F32])
        batch, count, t = r.choice([1, 2, 16]), int(2 ** r.uniform(0, 9)), r.choice([0, 0, int(2 ** r.uniform(0, 16))])
        window, block = r.choice([0, int(2 ** r.uniform(0, 12)), int(2 ** r.uniform(0, 12))]), 128 // G
        ring = T.tempo_ring_blocks(window, Z, min(block, count)) * r.choice([1, 2]) if window and r.random() < 0.8 else 0
        kv = store(Hkv, D, Z, ring or (t + count - 1) // Z + 1, ring, dtype)
        counts = AT if not ring and dtype != T.TEMPO_F32 and r.random() < 0.3 else None
        assert_within_the_launches_promised(lib, kv, batch, G * Hkv, t, count, window, r.choice([1 << 44, (1 << 44) + 64, 1 << 45]), counts)
    # beyond the index range of one launch: chunks of little more than a block
    for count in (129, 240, 2000):
        kv = store(64, 64, 256, 100)
        assert_within_the_launches_promised(lib, kv, 4000, 64, 0, count, 0, 1 << 45)
