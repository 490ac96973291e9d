"""Host side of windows with sinks, trees, rows at positions of their own and kept rows: sizes, and bad arguments refused before any
launch.  No test here computes anything on a GPU."""
import ctypes

import numpy as np
import pytest

from paper_2501_05408_amd import tempo as T
from spans_reference import sees_chain

FAKE = 1 << 20      # checked for NULL and alignment, never read
BIG = 1 << 40


def kv_desc(dtype=T.TEMPO_BF16, D=128, Z=64, Hkv=2, num_blocks=3, max_blocks=4, pools=(FAKE, 4 * FAKE, FAKE), ring=0):
    return T.make_kv(*pools, num_blocks, max_blocks, Z, Hkv, D, dtype, ring)


@pytest.mark.parametrize("window,sinks,Z,queries", [(1, 0, 32, 1), (1, 1, 32, 1), (2, 33, 32, 1), (32, 32, 32, 1), (33, 4, 32, 5), (1000, 4, 64, 7), (64, 0, 1, 3)])
def test_blocks_of_windows_with_sinks(window, sinks, Z, queries):
    first, turn = T.tempo_sink_blocks(window, sinks, Z, queries)
    assert first == len({j // Z for j in range(sinks)})
    most = 0
    for t in range(window + 2 * Z, window + 4 * Z):
        tiles = {j // Z for i in range(queries) for j in range(t + i - window + 1, t + i + 1)}
        most = max(most, len(tiles))
    assert turn == most
    # no two tiles that a call sees share a block
    for t in range(0, window + sinks + 5 * Z, max(1, Z // 7)):
        tiles = sorted({int(j) // Z for j in np.nonzero(sees_chain(t, queries, window, sinks).any(0))[0]})
        blocks = [n if n < first else first + (n - first) % turn for n in tiles]
        assert len(set(blocks)) == len(blocks)


def test_blocks_of_windows_with_sinks_refused():
    lib, a, b = T.load(), ctypes.c_int32(), ctypes.c_int32()
    for bad in ((0, 1, 32, 1), (1, -1, 32, 1), (1, 1, 0, 1), (1, 1, 32, 0)):
        assert lib.tempo_sink_blocks(*bad, ctypes.byref(a), ctypes.byref(b)) == T.TEMPO_ERR_RANGE
    assert lib.tempo_sink_blocks(1, 1, 32, 1, None, ctypes.byref(b)) == T.TEMPO_ERR_NULL
    assert lib.tempo_sink_blocks(1, 1, 32, 1, ctypes.byref(a), None) == T.TEMPO_ERR_NULL
    assert T.tempo_sink_blocks(2 ** 31 - 1, 2 ** 31 - 1, 1, 1) == (2 ** 31 - 1, 2 ** 31 - 1)
    # more tiles than an int32 counts
    for window, queries in ((2 ** 31 - 1, 2), (2 ** 31 - 1, 2 ** 31 - 1), (2, 2 ** 31 - 1)):
        assert lib.tempo_sink_blocks(window, 0, 1, queries, ctypes.byref(a), ctypes.byref(b)) == T.TEMPO_ERR_RANGE
    assert T.tempo_sink_blocks(2 ** 31 - 1, 0, 4, 2 ** 31 - 1) == (0, 2 ** 30)


GOOD = dict(kv=None, q=FAKE, k=FAKE, v=FAKE, out=FAKE, parents=FAKE, nodes=None, batch=2, Hq=6, rows=5, t=100, steps=None, window=20, sinks=4,
            scale=0.1, ws=FAKE, nbytes=BIG)


def call(which, **more):
    a = dict(GOOD, kv=kv_desc())
    a.update(more)
    lib, kv = T.load(), None if a["kv"] is None else ctypes.byref(a["kv"])
    rope = T.tempo_rope(FAKE, FAKE, a.get("positions", 1000), a.get("rope_dim", 128))
    tail = (a["window"], a["sinks"], a["scale"], a["ws"], a["nbytes"], None)
    if which == "tree":
        return lib.tempo_attn_tree(kv, a["q"], a["out"], a["parents"], a["nodes"], a["batch"], a["Hq"], a["rows"], a["t"], a["steps"], *tail)
    if which == "sinks":
        return lib.tempo_attn_sinks(kv, a["q"], a["out"], a["batch"], a["Hq"], a["rows"], a["t"], a["steps"], *tail)
    if which == "step":
        return lib.tempo_decode_step_sinks(kv, a["q"], a["k"], a["v"], a["out"], a["batch"], a["Hq"], a["t"], a["steps"], *tail)
    if which == "rope_step":
        return lib.tempo_rope_decode_step_sinks(kv, ctypes.byref(rope), a["q"], a["k"], a["v"], a["out"], a["batch"], a["Hq"], a["t"], a["steps"], *tail)
    if which == "prompt":
        return lib.tempo_prefill_sinks(kv, a["q"], a["k"], a["v"], a["out"], a["batch"], a["Hq"], a["t"], a["rows"], a["nodes"], *tail)
    return lib.tempo_rope_prefill_sinks(kv, ctypes.byref(rope), a["q"], a["k"], a["v"], a["out"], a["batch"], a["Hq"], a["t"], a["rows"], a["nodes"], *tail)


CALLS = ["tree", "sinks", "step", "rope_step", "prompt", "rope_prompt"]


@pytest.mark.parametrize("which", CALLS)
def test_attention_over_spans_is_refused(which):
    null, shape, reach, space, kind = T.TEMPO_ERR_NULL, T.TEMPO_ERR_SHAPE, T.TEMPO_ERR_RANGE, T.TEMPO_ERR_WORKSPACE, T.TEMPO_ERR_DTYPE
    assert call(which, kv=None) == null
    for name in ["q", "out"] + (["parents"] if which == "tree" else ["k", "v"] if which not in ("tree", "sinks") else []):
        assert call(which, **{name: None}) == null
    for i in range(3):
        pools = [FAKE] * 3
        pools[i] = None
        assert call(which, kv=kv_desc(pools=pools)) == null
    assert call(which, kv=kv_desc(7)) == kind
    if which == "rope_prompt":
        assert call(which, kv=kv_desc(T.TEMPO_F32)) == kind
    assert call(which, kv=kv_desc(ring=2)) == shape
    assert call(which, kv=kv_desc(D=96)) == shape and call(which, kv=kv_desc(Z=16)) == shape
    for batch in (0, -1, 65536):
        assert call(which, batch=batch) == shape
    for heads in (0, 5, 2 * 129, 65538):
        assert call(which, Hq=heads) == shape
    assert call(which, t=-1) == reach and call(which, t=256) == reach and call(which, t=2 ** 31 - 3) == reach
    assert call(which, window=-1) == reach and call(which, sinks=-1) == reach
    assert call(which, window=0, sinks=1) == reach
    if which != "tree":
        assert call(which, window=0, sinks=0) == reach
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert call(which, scale=scale) == reach
    assert call(which, ws=None) == space and call(which, ws=FAKE + 16) == space and call(which, nbytes=0) == space
    if which in ("tree", "sinks", "prompt", "rope_prompt"):
        assert call(which, rows=0) == shape and call(which, rows=-3) == shape
        assert call(which, t=252) == reach                     # the last row behind the table
    if which == "tree":
        assert call(which, rows=257, kv=kv_desc(max_blocks=100)) == shape
    if which == "prompt":
        assert call(which, rows=(1 << 24) + 1, kv=kv_desc(max_blocks=1 << 20)) == shape
        assert call(which, batch=65535, rows=60000, kv=kv_desc(max_blocks=1 << 20)) == shape
    if which.startswith("rope"):
        assert call(which, positions=100) == reach and call(which, rope_dim=64) == shape


def test_workspaces_of_spans():
    for dtype in (T.TEMPO_BF16, T.TEMPO_E4M3, T.TEMPO_F32):
        kv = kv_desc(dtype, max_blocks=1 << 20, num_blocks=100)
        for batch, Hq in ((1, 6), (16, 24), (3, 2)):
            if Hq % kv.num_kv_heads:
                continue
            last = 0
            for t in (0, 1, 31, 32, 500, 5000, 100000, 2000000):
                tree = T.tempo_attn_tree_workspace_bytes(kv, batch, Hq, 33, t)
                assert tree >= last > -1 and tree % 256 == 0
                last = tree
                # a window bounds it
                bound = T.tempo_attn_sinks_workspace_bytes(kv, batch, Hq, 1, t, 300, 4)
                assert 0 < bound <= T.tempo_attn_sinks_workspace_bytes(kv, batch, Hq, 1, 2000000, 300, 4)
        assert T.tempo_attn_sinks_workspace_bytes(kv, 16, 24, 1, 1000, 300, 4) == T.tempo_attn_sinks_workspace_bytes(kv, 16, 24, 1, 2000000, 300, 4)
    good = kv_desc()
    for bad in (kv_desc(7), kv_desc(ring=2), kv_desc(D=32)):
        assert T.tempo_attn_tree_workspace_bytes(bad, 2, 6, 5, 100) == 0
        assert T.tempo_attn_sinks_workspace_bytes(bad, 2, 6, 5, 100, 10, 1) == 0
        assert T.tempo_prefill_sinks_workspace_bytes(bad, 2, 6, 100) == 0
    assert T.tempo_attn_tree_workspace_bytes(good, 2, 6, 257, 100) == 0 and T.tempo_attn_tree_workspace_bytes(good, 2, 5, 5, 100) == 0
    assert T.tempo_attn_tree_workspace_bytes(good, 2, 6, 5, -1) == 0 and T.tempo_attn_tree_workspace_bytes(good, 2, 6, 5, 100, -1) == 0
    assert T.tempo_attn_sinks_workspace_bytes(good, 2, 6, 5, 100, 0, 0) == 0 and T.tempo_attn_sinks_workspace_bytes(good, 2, 6, 0, 100, 5, 0) == 0
    assert T.tempo_prefill_sinks_workspace_bytes(good, 0, 6, 100) == 0


def place(**more):
    a = dict(kv=kv_desc(), rope=T.tempo_rope(FAKE, FAKE, 1000, 128), axes=None, positions=FAKE, k=FAKE, v=FAKE, q=FAKE, q_out=FAKE, batch=2, Hq=6,
             t=100, steps=None, count=5, counts=None)
    a.update(more)
    ref = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731
    return T.load().tempo_rope_kv_append_at(ref(a["kv"]), ref(a["rope"]), ref(a["axes"]), a["positions"], a["k"], a["v"], a["q"], a["q_out"], a["batch"],
                                            a["Hq"], a["t"], a["steps"], a["count"], a["counts"], None)


def test_rows_at_positions_are_refused():
    null, shape, reach = T.TEMPO_ERR_NULL, T.TEMPO_ERR_SHAPE, T.TEMPO_ERR_RANGE
    for name in ("kv", "rope", "positions", "k", "v", "q", "q_out"):
        assert place(**{name: None}) == null
    assert place(kv=kv_desc(pools=(FAKE, None, FAKE))) == null
    assert place(rope=T.tempo_rope(None, FAKE, 1000, 128)) == null and place(rope=T.tempo_rope(FAKE + 4, FAKE, 1000, 128)) == shape
    assert place(rope=T.tempo_rope(FAKE, FAKE, 1000, 64)) == shape and place(rope=T.tempo_rope(FAKE, FAKE, 0, 128)) == reach
    assert place(batch=0) == shape and place(batch=65536) == shape and place(count=0) == shape and place(Hq=5) == shape
    assert place(t=-1) == reach and place(t=252) == reach and place(t=2 ** 31 - 4) == reach
    assert place(kv=kv_desc(ring=2), count=129) == reach
    assert place(kv=kv_desc(max_blocks=1 << 20), batch=4000, count=60000) == shape
    five = T.make_rope_axes([0, 4])
    assert place(axes=five) == shape
    wrong = T.make_rope_axes([0, 2])
    wrong.axes = 2
    assert place(axes=wrong) == reach
    none = T.make_rope_axes([0])
    none.axes = 0
    assert place(axes=none) == shape
    with pytest.raises(T.TempoError):
        T.make_rope_axes([])
    with pytest.raises(T.TempoError):
        T.make_rope_axes([0] * 65)


def test_rotation_at_positions_is_refused():
    lib, null, shape = T.load(), T.TEMPO_ERR_NULL, T.TEMPO_ERR_SHAPE
    rope = T.tempo_rope(FAKE, FAKE, 1000, 128)

    def rotate(rope=rope, axes=None, positions=FAKE, x=FAKE, y=FAKE, dtype=T.TEMPO_BF16, batch=2, count=5, heads=6):
        return lib.tempo_rope_rotate_at(None if rope is None else ctypes.byref(rope), None if axes is None else ctypes.byref(axes), positions, x, y,
                                        dtype, batch, count, heads, None)
    assert rotate(rope=None) == null and rotate(positions=None) == null and rotate(x=None) == null and rotate(y=None) == null
    assert rotate(dtype=T.TEMPO_E4M3) == T.TEMPO_ERR_DTYPE and rotate(dtype=9) == T.TEMPO_ERR_DTYPE
    assert rotate(rope=T.tempo_rope(FAKE, FAKE, 1000, 96)) == shape and rotate(rope=T.tempo_rope(FAKE, None, 1000, 64)) == null
    assert rotate(batch=0) == shape and rotate(count=0) == shape and rotate(heads=0) == shape and rotate(batch=65535, count=60000, heads=60) == shape
    assert rotate(axes=T.make_rope_axes([5])) == shape


def test_positions_and_kept_rows_are_refused():
    lib, null, shape, reach = T.load(), T.TEMPO_ERR_NULL, T.TEMPO_ERR_SHAPE, T.TEMPO_ERR_RANGE
    assert lib.tempo_tree_positions(None, FAKE, 1, 5, 0, None, None) == null and lib.tempo_tree_positions(FAKE, None, 1, 5, 0, None, None) == null
    for bad in ((0, 5, 0), (65536, 5, 0), (1, 0, 0), (1, 257, 0)):
        assert lib.tempo_tree_positions(FAKE, FAKE, *bad, None, None) == shape
    assert lib.tempo_tree_positions(FAKE, FAKE, 1, 5, -1, None, None) == reach
    assert lib.tempo_tree_positions(FAKE, FAKE, 1, 5, 2 ** 31 - 3, None, None) == reach

    def keep(layers=None, n=None, batch=2, t=100, nodes=20, kept=FAKE, count=5):
        layers = [kv_desc(), kv_desc(pools=(2 * FAKE, 3 * FAKE, FAKE))] if layers is None else layers
        kvs = T.make_kv_layers(layers) if layers else None
        return lib.tempo_kv_keep(kvs, len(layers) if n is None else n, batch, t, None, nodes, kept, count, None)
    assert keep([], 1) == null and keep(kept=None) == null and keep([kv_desc(), kv_desc(pools=(FAKE, None, FAKE))]) == null
    assert keep(n=0) == shape and keep(batch=0) == shape and keep(batch=65536) == shape and keep(count=0) == shape and keep(count=129) == shape
    assert keep(nodes=0) == shape
    for other in (kv_desc(Z=32), kv_desc(D=64), kv_desc(Hkv=1), kv_desc(T.TEMPO_E4M3), kv_desc(num_blocks=4), kv_desc(max_blocks=5), kv_desc(ring=2),
                  kv_desc(pools=(FAKE, FAKE, 2 * FAKE))):
        assert keep([kv_desc(), other]) == shape
    assert keep(t=-1) == reach and keep(t=250) == reach and keep(t=2 ** 31 - 10) == reach and keep(t=250, nodes=1, count=7) == reach
    assert keep([kv_desc(ring=2)], nodes=129) == reach


def test_axes_made_for_another_head_dim_are_refused():
    """A list of 32 axes with tables of 64 pairs, and of 64 with tables of 32: by the binding, and a list that is too short by the library too."""
    few, many = T.make_rope_axes([0] * 10 + [1] * 22), T.make_rope_axes([i % 3 for i in range(64)])
    wide, narrow = T.tempo_rope(FAKE, FAKE, 1000, 128), T.tempo_rope(FAKE, FAKE, 1000, 64)
    for axes, rope in ((few, wide), (many, narrow), (T.make_rope_axes([0]), wide)):
        with pytest.raises(T.TempoError) as e:
            T.tempo_rope_rotate_at(rope, axes, FAKE, FAKE, FAKE, T.TEMPO_BF16, 2, 5, 6, stream=FAKE)
        assert e.value.status == T.TEMPO_ERR_SHAPE
        with pytest.raises(T.TempoError) as e:
            T.tempo_rope_kv_append_at(kv_desc(D=rope.head_dim), rope, axes, FAKE, FAKE, FAKE, None, None, 2, 0, 100, None, 5, stream=FAKE)
        assert e.value.status == T.TEMPO_ERR_SHAPE
    assert place(axes=few) == T.TEMPO_ERR_RANGE
    assert T.load().tempo_rope_rotate_at(ctypes.byref(wide), ctypes.byref(few), FAKE, FAKE, FAKE, T.TEMPO_BF16, 2, 5, 6, None) == T.TEMPO_ERR_RANGE


def test_steps_that_meet_in_a_block_are_refused(monkeypatch):
    """Of a table that names blocks in turn: calls whose steps, windows and sinks have a slot each go through, others are refused before a launch."""
    import random
    import torch
    from paper_2501_05408_amd.store import BlockStore
    launched = []
    for name in ("tempo_attn_sinks", "tempo_decode_step_sinks", "tempo_prefill_sinks", "tempo_attn_tree", "tempo_kv_keep", "tempo_rope_kv_append_at"):
        monkeypatch.setattr(T, name, lambda *a, name=name, **k: launched.append(name))
    r = random.Random(12)
    refused = 0
    for turn in range(400):
        Z, window, sinks, queries = r.choice([32, 64]), r.randrange(1, 200), r.choice([0, 1, 5, 32, 33, 70]), r.choice([1, 1, 3, 50])
        table, blocks = BlockStore.sinks_table(2, 1200, Z, window, sinks, queries)
        st = BlockStore(2, 4, 2, 64, Z, 1200, T.TEMPO_BF16, device="cpu", num_blocks=blocks, block_table=table)
        st.rope = T.tempo_rope(FAKE, FAKE, 2000, 64)
        def meets(t, rows, window, sinks):
            keys = sorted(set(range(0, min(sinks, t + rows))) | set(range(max(0, t - window + 1) if window else 0, t + rows)))
            slots = [(int(table[0, j // Z]), j % Z) for j in keys]
            # ... and sinks that a later step has been written over
            over = any(int(table[0, n]) in table[0, -(-sinks // Z):(t + rows - 1) // Z + 1].tolist() for n in range(-(-sinks // Z))) if sinks else False
            return len(set(slots)) < len(slots) or (over and t + rows > sinks)
        # what the table is made for
        t, rows = r.randrange(0, 1200 - queries), r.randrange(1, queries + 1)
        ids = torch.zeros((2, rows), dtype=torch.int32)
        per = torch.zeros(2, dtype=torch.int32) if r.random() < 0.5 else None
        launched.clear()
        st.attend_sinks(None, None, t, rows, window, sinks, per)
        st.step_sinks(None, None, None, None, t, window, sinks, per)
        st.prefill_sinks(None, None, None, None, t, rows, window, sinks)
        st.attend_tree(None, None, ids, t, window=window, sinks=sinks, t_per_seq=per)
        st.keep(ids, t, rows)
        st.rope_append_at(None, torch.zeros((2, rows, 2, 64)), None, t)
        assert len(launched) == 6 and not meets(t, rows, window, sinks)
        # anything else
        rows, w, s = r.randrange(1, 400), r.choice([window, r.randrange(1, 400)]), r.choice([sinks, 0, r.randrange(0, 150)])
        t = r.randrange(0, 1200 - rows)
        ids = torch.zeros((2, rows), dtype=torch.int32)
        k = torch.zeros((2, rows, 2, 64))
        for bad, call in ((meets(t, rows, w, s), lambda: st.attend_sinks(None, None, t, rows, w, s)),
                          (meets(t, rows, w, s), lambda: st.prefill_sinks(None, None, None, None, t, rows, w, s)),
                          (meets(t, 1, w, s), lambda: st.step_sinks(None, None, None, None, t, w, s)),
                          (meets(t, min(rows, 256), w, s), lambda: st.attend_tree(None, None, ids[:, :256], t, window=w, sinks=s)),
                          (meets(t, min(rows, 256), 0, 0), lambda: st.attend_tree(None, None, ids[:, :256], t)),
                          (meets(t, rows, 1, 0), lambda: st.rope_append_at(None, k, None, t)),
                          (meets(t, min(rows, 100), 1, 0), lambda: st.keep(ids[:, :min(rows, 100)], t, 1))):
            launched.clear()
            if bad:
                with pytest.raises(T.TempoError) as e:
                    call()
                assert e.value.status == T.TEMPO_ERR_RANGE and launched == []
                refused += 1
            else:
                call()
                assert len(launched) == 1
    assert 200 < refused < 2500
    # sequences that share a block with each other, or have one each, are nothing to refuse
    st = BlockStore(2, 4, 2, 64, 32, 127, T.TEMPO_BF16, device="cpu", num_blocks=7, block_table=torch.tensor([[0, 1, 2, 3], [0, 4, 5, 6]]))
    st.attend_tree(None, None, torch.zeros((2, 9), dtype=torch.int32), 100)


def test_workspaces_of_spans_do_not_grow_beyond_a_prompts(monkeypatch):
    import torch
    from paper_2501_05408_amd.store import BlockStore
    given = []
    for name in ("tempo_attn_sinks", "tempo_prefill_sinks", "tempo_attn_tree"):
        monkeypatch.setattr(T, name, lambda *a, **k: given.append(a[-1]))
    for B, Hq, Hkv, D, max_t in ((1, 8, 2, 64, 3000), (4, 24, 8, 128, 2000), (2, 4, 4, 64, 100)):
        st = BlockStore(B, Hq, Hkv, D, 64, max_t, T.TEMPO_BF16, device="cpu")
        most = T.tempo_prefill_sinks_workspace_bytes(st.kv, B, Hq, st.max_t)
        given.clear()
        for rows in (1, 2, 5, 9, 20, 50, 90):
            st.attend_sinks(None, None, 0, rows, 2000, 4)
            st.attend_tree(None, None, torch.zeros((B, rows), dtype=torch.int32), 0)
            assert max(given) <= most
        st.prefill_sinks(None, None, None, None, 0, 100, 50, 4)
        assert given[-1] == most and len(st._span_ws) <= 20
