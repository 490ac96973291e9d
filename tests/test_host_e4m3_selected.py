"""Host side of the 8-bit block store and of the attention over selected blocks: layout, sizes, and bad arguments
refused before any launch.  No test here computes anything on a GPU."""
import ctypes

import numpy as np
import pytest

from paper_2501_05408_amd import tempo as T

FAKE = 1 << 20      # checked for NULL and alignment, never read
BIG = 1 << 40


def kv_desc(dtype=T.TEMPO_E4M3, D=128, Z=64, Hkv=2, num_blocks=3, max_blocks=4, pools=(FAKE, FAKE, FAKE), ring=0):
    return T.make_kv(*pools, num_blocks, max_blocks, Z, Hkv, D, dtype, ring)


# ---- the 8-bit store -----------------------------------------------------------------------------------

@pytest.mark.parametrize("D,Z,Hkv,blocks", [(64, 32, 1, 2), (128, 64, 3, 2), (128, 256, 1, 1)])
def test_codes_and_scale_bytes_fill_the_pool_once(D, Z, Hkv, blocks):
    kv = kv_desc(D=D, Z=Z, Hkv=Hkv, num_blocks=blocks)
    total = T.tempo_kv_pool_bytes(kv)
    assert total == blocks * Hkv * Z * (D + 1)
    for which in (0, 1):
        seen = np.zeros(total, dtype=int)
        for block in range(blocks):
            for head in range(Hkv):
                for slot in range(Z):
                    seen[T.tempo_kv_scale_offset(kv, which, block, head, slot)] += 1
                    for d in range(D):
                        at = T.tempo_kv_element_offset(kv, which, block, head, slot, d)
                        tile = (block * Hkv + head) * Z * D
                        assert tile <= at < tile + Z * D
                        # keys: a row's 8 consecutive dims lie side by side; values: a dim's 4 consecutive slots
                        if which == 0 and d % 8 == 0:
                            assert at % 8 == 0
                        if which == 1 and slot % 4 == 0:
                            assert at % 4 == 0
                        seen[at] += 1
        assert (seen == 1).all()


def test_offsets_outside_the_store_and_of_other_stores():
    kv = kv_desc()
    good = (0, 2, 1, 63)
    assert T.tempo_kv_scale_offset(kv, *good) > 0
    for bad in ((2, 2, 1, 63), (-1, 2, 1, 63), (0, 3, 1, 63), (0, -1, 1, 63), (0, 2, 2, 63), (0, 2, 1, 64), (0, 2, 1, -1)):
        assert T.tempo_kv_scale_offset(kv, *bad) == -1
    for dtype in (T.TEMPO_BF16, T.TEMPO_F32, 3, -1):
        assert T.tempo_kv_scale_offset(kv_desc(dtype), *good) == -1
    assert T.tempo_kv_scale_offset(kv_desc(Z=16), *good) == -1 and T.tempo_kv_pool_bytes(kv_desc(Z=16)) == 0


def test_an_8_bit_store_is_refused_where_it_has_no_kernel():
    lib, kv, rope = T.load(), kv_desc(), T.tempo_rope(FAKE, FAKE, 1000, 128)
    ref, r = ctypes.byref(kv), ctypes.byref(rope)
    assert lib.tempo_attn_decode_padded_causal(ref, FAKE, FAKE, 2, 6, 10, None, 20, 0.1, FAKE, BIG, None) == T.TEMPO_ERR_DTYPE
    assert lib.tempo_attn_worklist_bytes(ref, 2, 6, 100, 0) == 0
    assert lib.tempo_attn_worklist_build(ref, 2, 6, 100, FAKE, 0, FAKE, BIG, None) == T.TEMPO_ERR_DTYPE
    assert lib.tempo_decode_step_ragged(ref, FAKE, FAKE, FAKE, FAKE, 2, 6, 100, FAKE, 0, 0.1, FAKE, FAKE, BIG, None) == T.TEMPO_ERR_DTYPE
    assert lib.tempo_rope_rotate(r, FAKE, FAKE, T.TEMPO_E4M3, 2, 6, 5, None, None) == T.TEMPO_ERR_DTYPE


def test_bad_arguments_of_an_8_bit_store():
    lib = T.load()

    def append(kv, batch=2, t=5, k=FAKE, count=1):
        return lib.tempo_kv_append_block(ctypes.byref(kv), k, FAKE, batch, t, None, count, None)

    def attend(kv, batch=2, Hq=6, t=5, scale=0.1, ws=FAKE, nbytes=BIG, window=0):
        if window:
            return lib.tempo_attn_decode_window(ctypes.byref(kv), FAKE, FAKE, batch, Hq, t, None, window, scale, ws, nbytes, None)
        return lib.tempo_attn_decode_causal(ctypes.byref(kv), FAKE, FAKE, batch, Hq, t, None, scale, ws, nbytes, None)

    for kv in (kv_desc(Z=16), kv_desc(Z=48), kv_desc(D=96), kv_desc(Hkv=0), kv_desc(num_blocks=0), kv_desc(ring=3), kv_desc(ring=8)):
        assert append(kv) == T.TEMPO_ERR_SHAPE and attend(kv) == T.TEMPO_ERR_SHAPE
    for kv in (kv_desc(pools=(None, 1, 1)), kv_desc(pools=(1, None, 1)), kv_desc(pools=(1, 1, None))):
        assert append(kv) == T.TEMPO_ERR_NULL and attend(kv) == T.TEMPO_ERR_NULL
    good = kv_desc()
    assert append(good, k=None) == T.TEMPO_ERR_NULL and append(good, batch=0) == T.TEMPO_ERR_SHAPE and append(good, t=256) == T.TEMPO_ERR_RANGE
    assert append(good, t=200, count=57) == T.TEMPO_ERR_RANGE and append(good, count=0) == T.TEMPO_ERR_SHAPE
    assert append(kv_desc(ring=2), count=129) == T.TEMPO_ERR_RANGE
    assert attend(good, Hq=5) == T.TEMPO_ERR_SHAPE and attend(good, Hq=258) == T.TEMPO_ERR_SHAPE and attend(good, t=256) == T.TEMPO_ERR_RANGE
    assert attend(good, scale=0.0) == T.TEMPO_ERR_RANGE and attend(good, scale=float("nan")) == T.TEMPO_ERR_RANGE
    assert attend(good, ws=None) == T.TEMPO_ERR_WORKSPACE and attend(good, ws=FAKE + 8) == T.TEMPO_ERR_WORKSPACE
    assert attend(good, nbytes=16) == T.TEMPO_ERR_WORKSPACE
    assert attend(kv_desc(ring=2), t=128) == T.TEMPO_ERR_RANGE and attend(kv_desc(ring=2), t=500, window=66) == T.TEMPO_ERR_RANGE


# ---- selected blocks -------------------------------------------------------------------------------------

STORES = [T.TEMPO_BF16, T.TEMPO_E4M3]


def bounds(kv, to=FAKE, batch=2, t=5, count=1):
    return T.load().tempo_block_bounds(ctypes.byref(kv), to, batch, t, None, count, None, None)


def select(kv, at=FAKE, q=FAKE, out=FAKE, count=3, first=1, last=1, batch=2, Hq=6, t=250, ws=FAKE, nbytes=BIG):
    return T.load().tempo_select_blocks(ctypes.byref(kv), at, q, out, count, first, last, batch, Hq, t, None, ws, nbytes, None)


def attend(kv, q=FAKE, out=FAKE, selected=FAKE, count=3, batch=2, Hq=6, t=250, scale=0.1, ws=FAKE, nbytes=BIG):
    return T.load().tempo_attn_selected(ctypes.byref(kv), q, out, selected, count, batch, Hq, t, None, scale, ws, nbytes, None)


def step(kv, at=FAKE, q=FAKE, k=FAKE, v=FAKE, out=FAKE, selected=FAKE, count=3, first=1, last=1, batch=2, Hq=6, t=250, scale=0.1, ws=FAKE, nbytes=BIG):
    return T.load().tempo_decode_step_selected(ctypes.byref(kv), at, q, k, v, out, selected, count, first, last, batch, Hq, t, None, scale, ws,
                                               nbytes, None)


@pytest.mark.parametrize("call", [bounds, select, attend, step])
def test_stores_that_have_no_selected_attention(call):
    assert call(kv_desc(T.TEMPO_F32)) == T.TEMPO_ERR_DTYPE and call(kv_desc(7)) == T.TEMPO_ERR_DTYPE
    for dtype in STORES:
        assert call(kv_desc(dtype, ring=2)) == T.TEMPO_ERR_SHAPE and call(kv_desc(dtype, D=96)) == T.TEMPO_ERR_SHAPE
        assert call(kv_desc(dtype, pools=(None, 1, 1))) == T.TEMPO_ERR_NULL and call(kv_desc(dtype, pools=(1, 1, None))) == T.TEMPO_ERR_NULL
        for batch in (0, -1, 65536):
            assert call(kv_desc(dtype), batch=batch) == T.TEMPO_ERR_SHAPE


@pytest.mark.parametrize("dtype", STORES)
def test_bad_arguments_of_the_selected_calls(dtype):
    kv = kv_desc(dtype)
    for call, names in ((bounds, ["to"]), (select, ["at", "q", "out"]), (attend, ["q", "out", "selected"]),
                        (step, ["at", "q", "k", "v", "out", "selected"])):
        for name in names:
            assert call(kv, **{name: None}) == T.TEMPO_ERR_NULL
        assert call(kv, t=-1) == T.TEMPO_ERR_RANGE and call(kv, t=256) == T.TEMPO_ERR_RANGE and call(kv, t=2 ** 31 - 1) == T.TEMPO_ERR_RANGE
    for call in (select, attend, step):
        assert call(kv, Hq=5) == T.TEMPO_ERR_SHAPE and call(kv, Hq=2 * 129) == T.TEMPO_ERR_SHAPE and call(kv, Hq=0) == T.TEMPO_ERR_SHAPE
        assert call(kv, count=0) == T.TEMPO_ERR_SHAPE and call(kv, count=(1 << 30) // 64 + 1) == T.TEMPO_ERR_SHAPE
        assert call(kv, ws=None) == T.TEMPO_ERR_WORKSPACE and call(kv, ws=FAKE + 16) == T.TEMPO_ERR_WORKSPACE
        assert call(kv, nbytes=100) == T.TEMPO_ERR_WORKSPACE
    for call in (select, step):
        for first, last in ((1, 0), (-1, 1), (2, 2), (0, 4), (2 ** 31 - 1, 2 ** 31 - 1)):
            assert call(kv, first=first, last=last) == T.TEMPO_ERR_RANGE
        assert call(kv, at=FAKE + 8) == T.TEMPO_ERR_SHAPE
    assert bounds(kv, to=FAKE + 8) == T.TEMPO_ERR_SHAPE
    assert bounds(kv, count=0) == T.TEMPO_ERR_SHAPE and bounds(kv, t=0, count=257) == T.TEMPO_ERR_RANGE
    for call in (attend, step):
        for scale in (0.0, -1.0, float("inf"), float("nan")):
            assert call(kv, scale=scale) == T.TEMPO_ERR_RANGE
    assert bounds(kv, t=5, count=58) == T.TEMPO_OK           # completes no block: nothing to launch


def test_workspaces():
    kv = kv_desc(num_blocks=5000, max_blocks=5000)
    assert T.tempo_block_bounds_bytes(kv) == 5000 * 2 * 2 * 128 * 2
    assert T.tempo_select_workspace_bytes(kv, 3, 6, 64 * 100 - 1) == 19 * 256   # 3 * 2 * 100 scores of 8 bytes, in whole 256 bytes
    for count in (1, 2, 7, 100, 4000):
        partials = T.tempo_attn_selected_workspace_bytes(kv, 3, 6, count)
        assert 0 < partials <= T.tempo_attn_workspace_bytes(kv, 3, 6, count * 64 - 1)
        assert T.tempo_step_selected_workspace_bytes(kv, 3, 6, 6399, count) == partials + 19 * 256
    for bad in (kv_desc(T.TEMPO_F32), kv_desc(ring=2), kv_desc(D=32)):
        assert T.tempo_block_bounds_bytes(bad) == 0 and T.tempo_select_workspace_bytes(bad, 1, 6, 10) == 0
        assert T.tempo_attn_selected_workspace_bytes(bad, 1, 6, 1) == 0 and T.tempo_step_selected_workspace_bytes(bad, 1, 6, 10, 1) == 0
    assert T.tempo_select_workspace_bytes(kv, 1, 5, 10) == 0 and T.tempo_select_workspace_bytes(kv, 1, 6, -1) == 0
    assert T.tempo_attn_selected_workspace_bytes(kv, 1, 6, 0) == 0 and T.tempo_attn_selected_workspace_bytes(kv, 0, 6, 1) == 0
