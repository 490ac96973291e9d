"""Attention over 8-bit stores and lists of blocks whose columns take several workgroups, in launches whose units of work
(sequence, kv head, split) are no multiple of the 8 dies: every workgroup's own columns, keys and rows, against the oracle."""
import numpy as np
import pytest
import torch

import test_gpu_e4m3 as e4m3
import test_gpu_selected as selected
from paper_2501_05408_amd import tempo as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,D,B,t,window,ragged,queries", [
    (9, 3, 64, 5, 700, 0, False, 30), (40, 5, 128, 3, 290, 70, True, 9), (24, 6, 128, 2, 1000, 0, False, 32), (96, 1, 64, 11, 150, 0, True, 1),
    (64, 1, 128, 1, 3000, 0, False, 2), (100, 2, 128, 9, 64, 33, False, 1)])
def test_blocks(Hq, Hkv, D, B, t, window, ragged, queries):
    e4m3.test_attention(Hq, Hkv, D, 64, B, t, window, ragged, queries)


@pytest.mark.parametrize("Hq,Hkv,D,B,t,ragged,window", [(120, 3, 64, 3, 200, True, 0), (64, 1, 128, 9, 333, False, 0), (210, 5, 128, 2, 95, False, 50)])
def test_fused_steps(Hq, Hkv, D, B, t, ragged, window):
    e4m3.test_fused_steps_are_the_write_and_the_attention(Hq, Hkv, D, B, t, ragged, window)


@pytest.mark.parametrize("plan", [T.tempo_plan(64, 13, 2), T.tempo_plan(256, 4, 8)])
def test_splits(plan):
    """As many units as the plan has splits, for each of three heads."""
    Hq, Hkv, D, Z, B, t, queries = 15, 3, 64, 32, 1, 800, 20
    st, q, K, V, first, _ = e4m3.filled(51, Hq, Hkv, D, Z, B, t, 0, False, queries)
    nbytes = T.tempo_attn_plan_workspace_bytes(st.kv, B * queries, Hq, plan)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=e4m3.DEV)
    out = torch.empty((B, queries, Hq, D), dtype=torch.bfloat16, device=e4m3.DEV)
    T.tempo_attn_block_with_plan(st.kv, e4m3.bf16(q), out, B, Hq, queries, t, None, 0, st.scale, plan, ws, nbytes)
    for c in range(queries):
        e4m3.assert_attention(out[:, c], q[:, c], K, V, first + c, 0, st.scale, f"step {c}")


@pytest.mark.parametrize("dtype", selected.STORES)
@pytest.mark.parametrize("Hq,Hkv,D,B,t,count,ragged", [(60, 3, 64, 5, 900, 6, True), (128, 1, 128, 9, 2000, 20, False), (250, 5, 128, 1, 500, 3, False),
                                                     (36, 2, 64, 7, 3000, 40, True)])
def test_lists(dtype, Hq, Hkv, D, B, t, count, ragged):
    selected.test_attention_over_lists(dtype, Hq, Hkv, D, 64, B, t, count, ragged, True)


def test_lists_of_one_sequence_leave_the_rows_behind_it():
    st, q, K, V = selected.filled(52, T.TEMPO_E4M3, 1, 48, 1, 64, 32, 300)
    out = torch.full((3, 48, 64), 7.0, dtype=torch.bfloat16, device=selected.DEV)
    lists = np.array([[[0, 4, 9, -1]]])
    st.attend_selected(selected.bf16(q), out[1:2], selected.ints(lists), 300)
    selected.assert_attend(out[1:2], q, K, V, lists, 32, np.full(1, 300), st.scale, "one sequence")
    assert (out[0] == 7).all() and (out[2] == 7).all()
