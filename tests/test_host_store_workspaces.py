"""The workspaces that a BlockStore keeps: how many a loop of calls allocates, and that none is given back which a captured
graph may still write to.  The library's calls are recorded instead of made; no GPU."""
import gc
import weakref

import pytest
import torch

from paper_2501_05408_amd import tempo as T
from paper_2501_05408_amd.store import BlockStore

Z = 32


@pytest.fixture
def calls(monkeypatch):
    """(workspace, bytes) of every call, the workspace as a weak reference."""
    seen = []

    def record(*args):
        seen.append((weakref.ref(args[-2]), args[-1]))

    for name in ("tempo_select_blocks", "tempo_attn_selected", "tempo_decode_step_selected", "tempo_attn_block_causal"):
        monkeypatch.setattr(T, name, record)
    return seen


def make_store(max_t, batch=2, ring=0):
    return BlockStore(batch, 6, 2, 64, Z, max_t, T.TEMPO_BF16, device="cpu", ring_blocks=ring)


def held(calls):
    gc.collect()
    alive = {id(w()): w().numel() for w, _ in calls if w() is not None}
    assert all(w() is not None and w().numel() >= nbytes for w, nbytes in calls)
    return list(alive.values())


@pytest.mark.parametrize("call", ["step", "choose and attend"])
def test_a_sparse_decode_loop_allocates_once(calls, call):
    st = make_store(200 * Z - 1)
    for t in range(0, 200 * Z, Z // 2):
        if call == "step":
            st.step_selected(None, None, None, None, None, t, 8)
        else:
            lists = st.select_blocks(None, None, t, 8)
            st.attend_selected(None, None, lists, t)
    need = T.tempo_step_selected_workspace_bytes(st.kv, 2, 6, 200 * Z - 1, 8)
    if call == "step":
        assert held(calls) == [need]
    else:
        assert len(held(calls)) <= 2 and sum(held(calls)) <= 2 * need


def test_lists_that_grow_with_the_sequence_keep_less_than_four_times_the_largest_need(calls):
    st = make_store(400 * Z - 1)
    for t in range(0, 400 * Z, Z):
        st.step_selected(None, None, None, None, None, t, t // Z // 4 + 2)
    need = T.tempo_step_selected_workspace_bytes(st.kv, 2, 6, 400 * Z - 1, 101)
    assert sum(held(calls)) < 4 * need and len(held(calls)) < 10


def test_the_workspace_is_what_the_call_promises_at_every_step(calls):
    st = make_store(50 * Z - 1)
    for t in (50 * Z - 1, 0, 31, 700):
        st.step_selected(None, None, None, None, None, t, 5)
        assert calls[-1][1] >= T.tempo_step_selected_workspace_bytes(st.kv, 2, 6, t, 5)
        st.select_blocks(None, None, t, 5)
        assert calls[-1][1] >= T.tempo_select_workspace_bytes(st.kv, 2, 6, t)


def test_rings_are_refused(calls):
    st = make_store(1000, ring=4)
    for call in (lambda: st.select_blocks(None, None, 5, 2), lambda: st.step_selected(None, None, None, None, None, 5, 2),
                 lambda: st.attend_selected(None, None, torch.zeros((2, 2, 2), dtype=torch.int32), 5)):
        with pytest.raises(T.TempoError):
            call()
    assert not calls


def test_a_wider_block_leaves_the_workspace_of_a_narrower_one(calls):
    st = make_store(1000)
    for queries in (1, 2, 1, 7, 42, 3):
        st.attend_block(None, None, 5, queries)
    need = T.tempo_attn_block_workspace_bytes(st.kv, 2, 6, 42, 1000)
    assert sum(held(calls)) < 4 * need
