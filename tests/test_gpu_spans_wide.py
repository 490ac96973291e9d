"""The kernel for many (row, head) columns of windows with sinks and of trees, on the GPU, against the definitions in 64 bits (tolerance:
spans_reference.within).  test_host_launches_spans.py checks that the calls go to that kernel."""
import math

import numpy as np
import pytest
import torch

from paper_2501_05408_amd import synth
from paper_2501_05408_amd import tempo as T
from paper_2501_05408_amd.store import BlockStore
from spans_cases import WIDE
from spans_reference import sees_chain, sees_tree

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
UNTOUCHED = 7.0


def normal(seed, shape):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(0.0, 1.0, generator=g)


def ints(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)


def make_store(seed, dtype, B, Hq, Hkv, D, Z, max_t):
    """Blocks in a random order, NaN wherever nothing is written."""
    columns = max_t // Z + 1
    n = B * columns + 3
    table = torch.from_numpy(synth.permutation(seed, 77, n)[:B * columns].reshape(B, columns).copy())
    return BlockStore(B, Hq, Hkv, D, Z, max_t, dtype, device=DEV, num_blocks=n, block_table=table, fill="nan")


def write(st, b, k, v):
    """Steps 0 .. of one sequence."""
    if not k.shape[0]:
        return
    row = st.block_table[b:b + 1].contiguous()
    kv = T.make_kv(st.k_pool, st.v_pool, row, st.num_blocks, st.max_blocks_per_seq, st.Z, st.Hkv, st.D, st.dtype)
    T.tempo_kv_append_block(kv, k[None].contiguous(), v[None].contiguous(), 1, 0, None, k.shape[0])
    torch.cuda.synchronize()


def tree_of(n, rng):
    return np.array([max(-1, i - 1 - int(rng.integers(0, 4))) if i % 3 else int(rng.integers(-1, i)) if i else -1 for i in range(n)])


def check(got, q, K, V, seen):
    """got, q [n][Hq][D], K, V [T][Hkv][D] as the store holds them, seen [n][T].  The bound of spans_reference.within()."""
    n, Hq, D = q.shape
    Hkv, G = K.shape[1], Hq // K.shape[1]
    some = torch.from_numpy(seen.any(0)).to(DEV)
    seen = torch.from_numpy(seen).to(DEV)[:, some].repeat_interleave(G, 0)
    worst = 0.0
    for h in range(Hkv):
        k, v = K[some, h].double(), V[some, h].double()
        x = q[:, h * G:(h + 1) * G].reshape(n * G, D).double() @ k.t().contiguous() / math.sqrt(D)
        w = torch.softmax(x.masked_fill(~seen, -math.inf), -1)
        out, size = w @ v, w @ v.abs()
        bound = 1.03 * 2.0 ** -8 * (size + 2 * out.abs()) + 1e-30
        off = (got[:, h * G:(h + 1) * G].reshape(n * G, D).double() - out).abs() / bound
        assert not torch.isnan(off).any()
        worst = max(worst, float(off.max()))
    assert worst <= 1.0, f"{worst:.3f} of the bound"


def framed(like):
    """A tensor like `like` between two frames, filled with UNTOUCHED, and a check that the frames are as they were."""
    whole = torch.full((like.numel() + 8192,), UNTOUCHED, dtype=like.dtype, device=DEV)

    def intact():
        assert bool((whole[:4096] == UNTOUCHED).all()) and bool((whole[-4096:] == UNTOUCHED).all())
    return whole[4096:4096 + like.numel()].view(like.shape), intact


@pytest.mark.parametrize("dtype,what,Hq,Hkv,D,Z,B,t,rows,window,sinks,ragged,counts", WIDE)
def test_answers_of_many_columns(dtype, what, Hq, Hkv, D, Z, B, t, rows, window, sinks, ragged, counts):
    rng = np.random.default_rng(t + rows)
    steps = np.array([t] + [int(rng.integers(0, t + 1)) for _ in range(B - 1)]) if ragged else np.full(B, t)
    n = np.resize([rows, max(1, rows // 3), 0, rows - 1], B) if counts else np.full(B, rows)
    parents = np.stack([tree_of(rows, rng) for _ in range(B)])
    seen = [sees_tree(int(steps[b]), parents[b, :n[b]], window, sinks) if what == "tree" else sees_chain(int(steps[b]), int(n[b]), window, sinks) for b in range(B)]
    q, k, v = normal(1, (B, rows, Hq, D)), normal(2, (B, t + rows, Hkv, D)), normal(3, (B, t + rows, Hkv, D))
    for b in range(B):  # what no row of a sequence sees
        dead = torch.from_numpy(~seen[b].any(0)).to(DEV)
        k[b, :len(dead)][dead], v[b, :len(dead)][dead] = math.nan, math.inf
    st = make_store(t, dtype, B, Hq, Hkv, D, Z, t + rows - 1)
    for b in range(B):
        write(st, b, *(x[b, :t if what == "prompt" else steps[b] + n[b]] for x in (k, v)))
    out, intact = framed(q)
    some = ints(n) if counts else None
    if what == "tree":
        st.attend_tree(q, out, ints(parents), t, some, window, sinks, ints(steps) if ragged else None)
    elif what == "block":
        st.attend_sinks(q, out, t, rows, window, sinks, ints(steps) if ragged else None)
    else:
        st.prefill_sinks(q, k[:, t:].contiguous(), v[:, t:].contiguous(), out, t, rows, window, sinks, some)
    intact()
    k_held, v_held = st.gather(0, t + rows)
    for b in range(B):
        assert bool((out[b, n[b]:] == UNTOUCHED).all())
        if n[b]:
            end = steps[b] + n[b]
            check(out[b, :n[b]], q[b, :n[b]], k_held[b, :end], v_held[b, :end], seen[b])


@pytest.mark.parametrize("dtype", [T.TEMPO_BF16, T.TEMPO_E4M3])
@pytest.mark.parametrize("Hq,Hkv,D,Z,B,t,rows,window,sinks,counts", [
    (24, 8, 64, 32, 4, 371, 1000, 349, 40, True), (32, 8, 128, 32, 16, 103, 266, 40, 100, False), (64, 4, 128, 64, 1, 7336, 185, 2924, 100, False)])
def test_a_rotated_prompt_of_many_columns(dtype, Hq, Hkv, D, Z, B, t, rows, window, sinks, counts):
    """The bits of the rotated rows' prompt, whose answers are within the bound."""
    q, k, v = normal(4, (B, rows, Hq, D)), normal(5, (B, t + rows, Hkv, D)), normal(6, (B, t + rows, Hkv, D))
    angle = torch.arange(t + rows, dtype=torch.float64, device=DEV)[:, None] * 10000.0 ** (-torch.arange(D // 2, dtype=torch.float64, device=DEV) * 2 / D)
    n = np.resize([rows, max(1, rows // 3), 0, rows - 1], B) if counts else np.full(B, rows)
    got = []
    for fused in (True, False):
        st = make_store(t, dtype, B, Hq, Hkv, D, Z, t + rows - 1)
        st.set_rope(angle.cos().float(), angle.sin().float())
        st.rope_append_block(k[:, :t].contiguous(), v[:, :t].contiguous(), 0, t)
        new_k, new_v, out = k[:, t:].contiguous(), v[:, t:].contiguous(), torch.full_like(q, UNTOUCHED)
        turned_q = q.clone()
        if fused:
            st.prefill_sinks(q, new_k, new_v, out, t, rows, window, sinks, ints(n) if counts else None, rope=True)
        else:
            positions = ints(np.tile(t + np.arange(rows), (B, 1)))
            for x, heads in ((turned_q, Hq), (new_k, Hkv)):
                T.tempo_rope_rotate_at(st.rope, None, positions, x, x, T.TEMPO_BF16, B, rows, heads)
            st.prefill_sinks(turned_q, new_k, new_v, out, t, rows, window, sinks, ints(n) if counts else None)
        got.append([out] + [torch.nan_to_num(x.float(), nan=99.0) for x in st.gather(0, t + rows)])
    for a, b in zip(*got):
        assert torch.equal(a, b)
    for b in range(0, B, 3):
        if n[b]:
            end = t + n[b]
            check(got[0][0][b, :n[b]], turned_q[b, :n[b]], got[0][1][b, :end], got[0][2][b, :end], sees_chain(t, int(n[b]), window, sinks))


@pytest.mark.parametrize("dtype", [T.TEMPO_BF16, T.TEMPO_E4M3])
def test_many_columns_captured(dtype):
    """A prompt that writes its rows and a wide tree in one graph, replayed with other inputs, counts and steps; eager work between the replays."""
    Hq, Hkv, D, Z, B, t, rows, nodes, window, sinks = 64, 4, 128, 32, 4, 900, 300, 250, 333, 40
    st = make_store(9, dtype, B, Hq, Hkv, D, Z, t + rows - 1)
    st.append_block(normal(7, (B, t, Hkv, D)), normal(8, (B, t, Hkv, D)), 0, t)
    q, k, v = normal(9, (B, rows, Hq, D)), normal(10, (B, rows, Hkv, D)), normal(11, (B, rows, Hkv, D))
    n, steps, parents = ints(np.full(B, rows)), ints(np.full(B, t)), ints(np.full((B, nodes), -1))
    out, tree = torch.zeros_like(q), torch.zeros_like(q[:, :nodes])

    def both(a, z):
        st.prefill_sinks(q, k, v, a, t, rows, window, sinks, n)
        st.attend_tree(q[:, :nodes].contiguous(), z, parents, t, None, window, sinks, steps)

    both(out, tree)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(out, tree)
    rng = np.random.default_rng(5)
    for turn in range(4):
        for i, x in enumerate((q, k, v)):
            x.copy_(normal(20 + 3 * turn + i, x.shape))
        # (the tree's steps lie behind what the prompt of this turn wrote, or before it)
        n.copy_(ints([rows, rows - turn, rows, rows])), steps.copy_(ints([t, t - 40 - turn, 10 * turn, t - 300]))
        parents.copy_(ints(np.stack([tree_of(nodes, rng) for _ in range(B)])))
        out.fill_(UNTOUCHED), tree.fill_(UNTOUCHED)
        graph.replay()
        torch.cuda.synchronize()
        eager, eager_tree = torch.full_like(out, UNTOUCHED), torch.full_like(tree, UNTOUCHED)
        both(eager, eager_tree)
        assert torch.equal(out, eager) and torch.equal(tree, eager_tree)
        k_held, v_held = st.gather(0, t + rows)
        for b in range(B):
            count, at = int(n[b]), int(steps[b])
            check(out[b, :count], q[b, :count], k_held[b, :t + count], v_held[b, :t + count], sees_chain(t, count, window, sinks))
            check(tree[b], q[b, :nodes], k_held[b, :at + nodes], v_held[b, :at + nodes], sees_tree(at, parents[b].cpu().numpy(), window, sinks))
