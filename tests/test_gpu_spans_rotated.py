"""Rotary steps with sinks, and trees of placed rows, from the keys that the store holds and the queries that the library turns: what is left
is the attention's own error (spans_reference.within).  And the calls that write their rows, captured."""
import numpy as np
import pytest
import torch

from paper_2501_05408_amd import synth
from paper_2501_05408_amd import tempo as T
from paper_2501_05408_amd.store import BlockStore
from spans_reference import attention, sees_chain, sees_tree, within, within_fp32

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
STORES = [T.TEMPO_BF16, T.TEMPO_E4M3, T.TEMPO_F32]


def np64(x):
    return x.detach().float().cpu().numpy().astype(np.float64)


def normal(seed, shape, dtype):
    x = torch.from_numpy(synth.normal_as(seed, 1, shape, "f32")).to(DEV)
    return x if dtype == T.TEMPO_F32 else x.to(torch.bfloat16)


def ints(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)


def near(dtype, got, q, K, V, seen):
    out, size = attention(q, K, V, seen)
    within_fp32(got, out, size, q, K) if dtype == T.TEMPO_F32 else within(got, out, size)


def tables(st, rows):
    a = torch.arange(rows, dtype=torch.float64, device=DEV)[:, None] * 10000.0 ** (-torch.arange(st.D // 2, dtype=torch.float64, device=DEV) * 2 / st.D)
    st.set_rope(a.cos().float(), a.sin().float())


@pytest.mark.parametrize("dtype", STORES)
@pytest.mark.parametrize("Hq,Hkv,D,Z,B,window,sinks,ragged", [(6, 2, 128, 32, 2, 50, 5, False), (4, 4, 64, 64, 3, 40, 33, True), (40, 2, 128, 32, 2, 9, 1, True),
                                                              (64, 2, 64, 32, 1, 20, 0, False), (24, 8, 128, 32, 2, 100, 4, True)])
def test_rotary_steps_from_the_keys_they_wrote(dtype, Hq, Hkv, D, Z, B, window, sinks, ragged):
    steps, lag = 230, np.array([0, 7, 70])[:B] if ragged else np.zeros(B, dtype=int)
    st = BlockStore(B, Hq, Hkv, D, Z, steps, dtype, device=DEV, fill="nan")
    tables(st, steps)
    q, k, v = normal(1, (steps, B, Hq, D), dtype), normal(2, (steps, B, Hkv, D), dtype), normal(3, (steps, B, Hkv, D), dtype)
    out, turned = torch.zeros_like(q[0]), torch.zeros_like(q[0])
    for i in range(steps):
        at = np.maximum(i - lag, 0)
        per = ints(at) if ragged else None
        st.step_sinks(q[i], k[i], v[i], out, i, window, sinks, per, rope=True)
        if i in (0, 1, 31, 32, 33, 63, 64, 101, 128, 200, 229):
            st.rope_rotate(q[i], turned, i, per)
            K, V = (np64(x) for x in st.gather(0, i + 1))
            for b in range(B):
                end = int(at[b]) + 1
                near(dtype, np64(out)[b][None], np64(turned)[b][None], K[b, :end], V[b, :end], sees_chain(int(at[b]), 1, window, sinks))


@pytest.mark.parametrize("dtype", STORES)
@pytest.mark.parametrize("Hq,Hkv,D,Z,B,t,nodes,window,sinks", [(6, 2, 128, 32, 3, 45, 14, 0, 0), (24, 8, 64, 64, 2, 200, 40, 30, 4), (4, 1, 128, 32, 2, 0, 70, 0, 0)])
def test_trees_of_placed_rows_from_the_keys_they_wrote(dtype, Hq, Hkv, D, Z, B, t, nodes, window, sinks):
    rng = np.random.default_rng(nodes)
    st = BlockStore(B, Hq, Hkv, D, Z, t + nodes - 1, dtype, device=DEV, fill="nan")
    tables(st, t + nodes)
    if t:
        st.rope_append_at(ints(np.tile(np.arange(t)[:, None], (B, 1, 1))), normal(4, (B, t, Hkv, D), dtype), normal(5, (B, t, Hkv, D), dtype), 0)
    steps = np.array([t, t // 2, t // 3])[:B]
    parents = np.stack([[int(rng.integers(-1, i)) if i else -1 for i in range(nodes)] for _ in range(B)])
    positions = st.tree_positions(ints(parents), t, ints(steps))
    q, k, v = normal(6, (B, nodes, Hq, D), dtype), normal(7, (B, nodes, Hkv, D), dtype), normal(8, (B, nodes, Hkv, D), dtype)
    out = torch.zeros_like(q)
    st.rope_append_at(positions[..., None].contiguous(), k, v, t, q, q, ints(steps))
    st.attend_tree(q, out, ints(parents), t, None, window, sinks, ints(steps))
    K, V = (np64(x) for x in st.gather(0, t + nodes))
    for b in range(B):
        end = int(steps[b]) + nodes
        near(dtype, np64(out)[b], np64(q)[b], K[b, :end], V[b, :end], sees_tree(int(steps[b]), parents[b], window, sinks))


@pytest.mark.parametrize("dtype", STORES)
def test_calls_that_write_their_rows_captured(dtype):
    """A step, a prompt and a tree, with their rows, in one graph; replayed with other inputs, steps, positions and counts, on a store that goes on."""
    B, Hq, Hkv, D, Z, t, rows, nodes, window, sinks = 2, 6, 2, 128, 32, 150, 21, 18, 60, 5
    def fresh():
        st = BlockStore(B, Hq, Hkv, D, Z, t + rows + nodes, dtype, device=DEV)
        tables(st, t + rows + nodes + 1)
        st.append_block(normal(9, (B, t, Hkv, D), dtype), normal(10, (B, t, Hkv, D), dtype), 0, t)
        return st
    shapes = [(B, Hq, D), (B, Hkv, D), (B, Hkv, D), (B, rows, Hq, D), (B, rows, Hkv, D), (B, rows, Hkv, D), (B, nodes, Hq, D), (B, nodes, Hkv, D), (B, nodes, Hkv, D)]
    ins = [normal(11, s, dtype) for s in shapes]
    steps, counts, parents = ints([t, t]), ints([rows, rows]), ints(np.full((B, nodes), -1))
    outs = [torch.zeros_like(ins[i]) for i in (0, 3, 6)]
    turned = torch.zeros_like(ins[6])

    def run(st, outs, turned):
        q, k, v, pq, pk, pv, tq, tk, tv = ins
        st.step_sinks(q, k, v, outs[0], t, window, sinks, steps, rope=True)
        st.prefill_sinks(pq, pk, pv, outs[1], t + 1, rows, window, sinks, counts, rope=dtype != T.TEMPO_F32)
        positions = torch.empty_like(parents)
        T.tempo_tree_positions(parents, positions, B, nodes, t, steps)
        st.rope_append_at(positions[..., None], tk, tv, t, tq, turned, steps)
        st.attend_tree(turned, outs[2], parents, t, None, window, sinks, steps)

    st, other = fresh(), fresh()
    run(st, outs, turned)
    run(other, [torch.zeros_like(o) for o in outs], torch.zeros_like(turned))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(st, outs, turned)
    rng = np.random.default_rng(3)
    for turn in range(4):
        for i, x in enumerate(ins):
            x.copy_(normal(30 + 10 * turn + i, x.shape, dtype))
        steps.copy_(ints([t - turn, 40 + 9 * turn])), counts.copy_(ints([rows - turn, max(0, rows - 8 * turn)]))
        parents.copy_(ints(np.stack([[int(rng.integers(-1, i)) if i else -1 for i in range(nodes)] for _ in range(B)])))
        for o in outs:
            o.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        eager, eager_turned = [torch.full_like(o, 5.0) for o in outs], torch.zeros_like(turned)
        run(other, eager, eager_turned)
        torch.cuda.synchronize()
        for a, b in zip(outs + [turned, st.k_pool.view(torch.uint8), st.v_pool.view(torch.uint8)],
                        eager + [eager_turned, other.k_pool.view(torch.uint8), other.v_pool.view(torch.uint8)]):
            assert torch.equal(a, b)
        K, V = (np64(x) for x in st.gather(0, t + rows))
        for b in range(B):
            at = int(steps[b])
            near(dtype, np64(outs[2])[b], np64(turned)[b], K[b, :at + nodes], V[b, :at + nodes], sees_tree(at, parents[b].cpu().numpy(), window, sinks))
