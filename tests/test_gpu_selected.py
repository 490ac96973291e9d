"""Sparse decode attention on the GPU: bounds of blocks (exact), the choice of blocks against the formula in 64 bits
(equal), attention over lists of blocks against the fp64 oracle, and whole steps.

Tolerance of answers as in test_gpu_e4m3.py: 2^-8 (A + 2 |o|), A = sum p_j |v_j| / sum p_j, and 3% of it for fp32."""
import numpy as np
import pytest
import torch

from e4m3_reference import held
from oracle import tempo_oracle as oracle
from paper_2501_05408_amd import synth
from paper_2501_05408_amd import tempo as T
from paper_2501_05408_amd.store import BlockStore

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
STORES = [T.TEMPO_BF16, T.TEMPO_E4M3]


def np64(x):
    return x.detach().float().cpu().numpy().astype(np.float64)


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(DEV).to(torch.bfloat16)


def ints(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)


def normal(seed, which, shape):
    return synth.normal_as(seed, which, shape, "bf16").astype(np.float64)


def make_store(seed, dtype, B, Hq, Hkv, D, Z, max_t):
    columns = max_t // Z + 1
    n = B * columns + 3
    table = torch.from_numpy(synth.permutation(seed, 77, n)[:B * columns].reshape(B, columns).copy())
    return BlockStore(B, Hq, Hkv, D, Z, max_t, dtype, device=DEV, num_blocks=n, block_table=table, fill="nan")


def kept(dtype, x):
    return held(x) if dtype == T.TEMPO_E4M3 else x


def filled(seed, dtype, B, Hq, Hkv, D, Z, t):
    q, K, V = normal(seed, 1, (B, Hq, D)), normal(seed, 2, (B, t + 1, Hkv, D)), normal(seed, 3, (B, t + 1, Hkv, D))
    st = make_store(seed, dtype, B, Hq, Hkv, D, Z, t)
    st.append_block(bf16(K), bf16(V), 0, t + 1)
    return st, q, kept(dtype, K), kept(dtype, V)


# ---- bounds -----------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", STORES)
@pytest.mark.parametrize("D,Z,t,count,ragged", [(128, 64, 0, 64, False), (64, 32, 0, 200, False), (128, 32, 31, 1, False), (64, 64, 40, 150, False),
                                                (128, 256, 100, 500, False), (128, 32, 70, 65, True), (64, 64, 190, 2, True), (128, 64, 10, 20, False)])
def test_bounds_of_the_completed_blocks(dtype, D, Z, t, count, ragged):
    B, Hkv = 3, 2
    last = t + count - 1
    st, _, K, _ = filled(21, dtype, B, 2 * Hkv, Hkv, D, Z, last)
    first = np.array([t, 0, t // 2]) if ragged else np.full(B, t)
    rows = np.array([count, count // 2, 0])
    for counts in (None, rows):
        bounds = st.new_bounds().fill_(7.0)
        st.update_bounds(bounds, t, count, ints(first) if ragged else None, None if counts is None else ints(counts))
        got, table = np64(bounds), st.block_table.cpu().numpy()
        ref = np.full_like(got, 7.0)
        for b in range(B):
            n = count if counts is None else counts[b]
            for block in range(first[b] // Z, (first[b] + n) // Z):
                keys = K[b, block * Z:(block + 1) * Z]                      # [Z][Hkv][D]
                ref[table[b, block], :, 0], ref[table[b, block], :, 1] = keys.min(0), keys.max(0)
        np.testing.assert_array_equal(got, ref)


@pytest.mark.parametrize("dtype", STORES)
def test_bounds_of_a_block_with_nan_are_nan(dtype):
    B, Hkv, D, Z, t = 1, 2, 128, 32, 63
    st = make_store(22, dtype, B, 4, Hkv, D, Z, t)
    K = normal(22, 1, (B, t + 1, Hkv, D))
    K[0, 40, 1, 77] = np.nan
    K[0, 3, 0, 5] = np.inf                                                   # an 8-bit store holds NaN for it
    st.append_block(bf16(K), bf16(K), 0, t + 1)
    bounds = st.new_bounds()
    st.update_bounds(bounds, 0, t + 1)
    got, table = np64(bounds)[st.block_table.cpu().numpy()[0]], None
    nan = np.isnan(got)
    assert nan[1, 1, :, 77].all()
    if dtype == T.TEMPO_E4M3:
        assert nan[0, 0, :, 5].all() and nan.sum() == 4
    else:
        assert got[0, 0, 1, 5] == np.inf and nan.sum() == 2


# ---- choice -----------------------------------------------------------------------------------------

def choose(q, lo, hi, newest, pick, first, last):
    """q [G][D], lo, hi [blocks][D] in 64 bits: the ascending list, padded with -1."""
    if newest < pick:
        took = list(range(newest + 1))
    else:
        score = np.maximum(q[:, None] * lo[None], q[:, None] * hi[None]).sum(-1).max(0)
        score = np.where(np.isnan(np.maximum(q[:, None] * lo[None], q[:, None] * hi[None]).sum(-1)).any(0), np.inf, score)
        rest = [n for n in range(first, newest - last + 1)]
        nan = [np.isnan(lo[n]).any() or np.isnan(hi[n]).any() for n in range(newest + 1)]
        rest.sort(key=lambda n: (not nan[n], -score[n], n))
        took = sorted(list(range(first)) + rest[:pick - first - last] + list(range(newest - last + 1, newest + 1)))
    return np.array(took + [-1] * (pick - len(took)))


def assert_choice(st, bounds, q, t, steps, pick, first, last):
    B, Hkv, G = st.batch, st.Hkv, st.Hq // st.Hkv
    got = st.select_blocks(bounds, bf16(q), t, pick, first, last, None if steps is None else ints(steps)).cpu().numpy()
    edges, table = np64(bounds), st.block_table.cpu().numpy()
    for b in range(B):
        newest = (t if steps is None else min(max(int(steps[b]), 0), t)) // st.Z
        for h in range(Hkv):
            e = edges[table[b, :newest + 1], h]
            np.testing.assert_array_equal(got[b, h], choose(q[b, h * G:(h + 1) * G], e[:, 0], e[:, 1], newest, pick, first, last), f"sequence {b}, head {h}")
    return got


def random_bounds(st, seed, levels=0):
    """Bounds without keys; with `levels`, of a few whole values only, so that scores are equal often."""
    shape = (st.num_blocks, st.Hkv, st.D)
    a, b = normal(seed, 5, shape), normal(seed, 6, shape)
    if levels:
        a, b = np.round(a * levels) * 1.0, np.round(b * levels) * 1.0
    return bf16(np.stack([np.minimum(a, b), np.maximum(a, b)], axis=2))


@pytest.mark.parametrize("Hq,Hkv,D,Z,B,t,pick,first,last,ragged",
                         [(6, 2, 128, 32, 2, 1000, 8, 1, 2, False), (8, 8, 64, 32, 3, 999, 5, 0, 1, False), (24, 8, 128, 64, 3, 5000, 16, 1, 2, True),
                          (32, 1, 64, 32, 1, 2047, 32, 3, 3, False), (100, 1, 128, 32, 2, 500, 4, 1, 1, False), (4, 2, 64, 32, 2, 40000, 300, 2, 5, True),
                          (2, 1, 128, 256, 1, 20000, 3, 1, 2, False), (2, 2, 64, 32, 2, 300, 10, 1, 1, False), (2, 2, 64, 32, 2, 300, 40, 1, 1, False),
                          (6, 2, 128, 32, 5, 31, 1, 0, 1, False), (6, 2, 128, 32, 2, 640, 21, 1, 20, True), (2, 1, 64, 32, 1, 300000, 17, 1, 1, False)])
def test_choice(Hq, Hkv, D, Z, B, t, pick, first, last, ragged):
    st = make_store(23, T.TEMPO_BF16, B, Hq, Hkv, D, Z, t)
    steps = synth.integers(23, 9, B, 0, t) if ragged else None
    q = normal(23, 7, (B, Hq, D))
    assert_choice(st, random_bounds(st, 23), q, t, steps, pick, first, last)
    few = np.round(q)
    few[np.abs(q) < 1.2] = 0                                                  # few terms, whole ones: many equal scores
    assert_choice(st, random_bounds(st, 24, 1), few, t, steps, pick, first, last)
    assert_choice(st, random_bounds(st, 24), np.zeros_like(q), t, steps, pick, first, last)  # all equal


def test_choice_between_scores_that_fp32_does_not_tell_apart():
    """Scores 2^24 + n: their order is lost in 24 bits."""
    D, Z, blocks = 64, 32, 200
    st = make_store(25, T.TEMPO_BF16, 1, 1, 1, D, Z, blocks * Z - 1)
    order = synth.permutation(25, 1, blocks)
    edge = np.zeros((st.num_blocks, 1, 2, D))
    table = st.block_table.cpu().numpy()[0]
    edge[table, 0, :, 0], edge[table, 0, :, 1] = 2.0 ** 24, order[:, None]
    got = assert_choice(st, bf16(edge), np.concatenate([[1.0, 1.0], np.zeros(D - 2)]).reshape(1, 1, D), blocks * Z - 1, None, 20, 0, 1)
    best = sorted(sorted(range(blocks - 1), key=lambda n: -order[n])[:19] + [blocks - 1])
    assert got[0, 0].tolist() == best


@pytest.mark.parametrize("close", [5, 40, 63, 64, 65, 150])
def test_choice_among_blocks_that_are_closer_than_fp32_sums_tell(close):
    """`close` blocks with scores of 2^12 + k 2^-8 in random order around the border, the others clearly above or below."""
    D, Z, blocks, pick = 128, 32, 400, 100
    st = make_store(34, T.TEMPO_BF16, 2, 4, 2, D, Z, blocks * Z - 1)
    rng = np.random.default_rng(close)
    edge = np.zeros((st.num_blocks, 2, 2, D))
    table = st.block_table.cpu().numpy()
    above = pick - 2 - close // 2
    for b in range(2):
        for h in range(2):
            order = rng.permutation(np.arange(1, blocks - 1))
            place = edge[table[b], h]
            place[order, 1, 5] = 3000.0
            place[order[:above], 1, 5] = 6000.0
            near = order[above:above + close]
            place[near, 1, 5], place[near, 1, 77] = 4096.0, rng.permutation(close) / 256.0
            edge[table[b], h] = place
    q = np.zeros((2, 4, D))
    q[:, :, 5] = q[:, :, 77] = 1.0
    q[:, 1::2] *= 0.5
    assert_choice(st, bf16(edge), q, blocks * Z - 1, None, pick, 1, 1)


def test_choice_of_nan_infinite_and_extreme_bounds():
    D, Z, blocks, B = 64, 32, 100, 2
    st = make_store(26, T.TEMPO_BF16, B, 2, 1, D, Z, blocks * Z - 1)
    bounds = random_bounds(st, 26)
    table = st.block_table.cpu().numpy()
    for b in range(B):
        for n, value in ((10, np.nan), (50, np.inf), (70, -np.inf), (80, 3.3e38), (81, -3.3e38), (90, np.nan)):
            bounds[table[b, n], 0, 0 if value == -np.inf else 1, 3 * b] = value
    q = normal(26, 7, (B, 2, D))
    got = st.select_blocks(bounds, bf16(q), blocks * Z - 1, 6, 1, 1).cpu().numpy()
    for b in range(B):
        assert {0, 10, 90, blocks - 1} <= set(got[b, 0].tolist()) and (np.diff(got[b, 0]) > 0).all()


@pytest.mark.parametrize("D,Hq,blocks,Z", [(64, 2, 100, 32), (128, 20, 300, 32), (128, 6, 5000, 32)])
def test_zero_times_an_infinite_bound_is_nan_on_either_side(D, Hq, blocks, Z):
    """max(q lo, q hi) with q = 0, or with an infinite q and a bound of 0: a NaN product is taken, whichever it is."""
    st = make_store(37, T.TEMPO_BF16, 2, Hq, 1, D, Z, blocks * Z - 1)
    bounds = random_bounds(st, 37)
    table = st.block_table.cpu().numpy()
    q = normal(37, 7, (2, Hq, D))
    q[0, 1, 3], q[1, 0, D - 1] = 0.0, -0.0
    for b, d in ((0, 3), (1, D - 1)):
        bounds[table[b, 11], 0, 0, d] = -np.inf                              # the smaller bound: the larger product is 0, the other NaN
        bounds[table[b, 40], 0, 1, d] = np.inf
        bounds[table[b, 77], 0, 0, d], bounds[table[b, 77], 0, 1, d] = -np.inf, np.inf
    got = assert_choice(st, bounds, q, blocks * Z - 1, None, 6, 1, 1)
    assert all({11, 40, 77} <= set(got[b, 0].tolist()) for b in range(2))
    clean = random_bounds(st, 38)
    q[0, 0, 5] = np.inf
    clean[table[0], 0, 0, 5], clean[table[0], 0, 1, 5] = 1.0, 2.0            # scores of +inf but where a bound is 0
    clean[table[0, 23], 0, 0, 5] = 0.0
    got = st.select_blocks(clean, bf16(q), blocks * Z - 1, 3, 1, 1).cpu().numpy()
    assert got[0, 0].tolist() == [0, 23, blocks - 1]


@pytest.mark.parametrize("bound,query", [(2.0 ** -130, 1.0), (2.0 ** -130, 2.0 ** 100), (2.0 ** -70, 2.0 ** -75), (2.0 ** 60, 2.0 ** 60), (1.0, 2.0 ** -20)])
def test_choice_at_the_ends_of_the_range(bound, query):
    """Bounds that bf16 holds as subnormals, products that fp32 does, and large ones."""
    st = make_store(35, T.TEMPO_BF16, 2, 6, 2, 64, 32, 32 * 300 - 1)
    spread = normal(35, 7, (2, 6, 64))
    bounds = (random_bounds(st, 35).double() * 4).round().clamp(-16, 16) * bound     # whole multiples: exact
    assert_choice(st, bounds.to(torch.bfloat16), np64(bf16(spread)) * query, 32 * 300 - 1, None, 20, 1, 2)


# ---- attention over lists ------------------------------------------------------------------------------

def assert_attend(got, q, K, V, lists, Z, steps, scale, what):
    """q [B][Hq][D]; K, V [B][T][Hkv][D]; lists [B][Hkv][count]."""
    B, Hq, D = q.shape
    Hkv = K.shape[2]
    G = Hq // Hkv
    for b in range(B):
        for h in range(Hkv):
            rows = [j for n in lists[b, h] if 0 <= n <= steps[b] // Z for j in range(n * Z, min(n * Z + Z, steps[b] + 1))]
            mine = np64(got)[b, h * G:(h + 1) * G]
            if not rows:
                assert (mine == 0).all(), f"{what}: no key, {mine}"
                continue
            k, v, x = K[b:b + 1, rows, h:h + 1], V[b:b + 1, rows, h:h + 1], q[b:b + 1, h * G:(h + 1) * G]
            ref, size = (oracle.attend(x, k, y, len(rows) - 1, 0, scale)[0] for y in (v, np.abs(v)))
            err, tol = np.abs(mine - ref), 1.03 * 2.0 ** -8 * (size + 2 * np.abs(ref))
            assert np.isfinite(err).all() and (err <= tol).all(), f"{what}, sequence {b}, head {h}: {(err / tol).max():.3f} of the tolerance"


def random_lists(seed, B, Hkv, blocks, count, holes):
    rng = np.random.default_rng(seed)
    lists = np.full((B, Hkv, count), -1)
    for b in range(B):
        for h in range(Hkv):
            got = rng.permutation(blocks)[:count]
            lists[b, h, :len(got)] = got
            if holes:
                lists[b, h, rng.random(count) < 0.3] = rng.choice([-1, -5, blocks + 3, 2 ** 31 - 1, -2 ** 31])
    return lists


@pytest.mark.parametrize("dtype", STORES)
@pytest.mark.parametrize("Hq,Hkv,D,Z,B,t,count,ragged,holes",
                         [(6, 2, 128, 32, 2, 500, 4, False, False), (8, 2, 64, 64, 3, 1000, 7, True, True), (24, 8, 128, 64, 2, 3000, 33, False, False),
                          (32, 4, 128, 256, 2, 1500, 3, True, False), (16, 16, 64, 32, 2, 300, 10, False, True), (40, 2, 64, 64, 1, 700, 5, False, False),
                          (128, 1, 128, 32, 1, 400, 9, False, True), (2, 2, 128, 32, 1, 0, 1, False, False), (3, 1, 64, 32, 4, 100, 200, True, True),
                          (8, 1, 128, 32, 1, 9000, 250, False, False)])
def test_attention_over_lists(dtype, Hq, Hkv, D, Z, B, t, count, ragged, holes):
    st, q, K, V = filled(27, dtype, B, Hq, Hkv, D, Z, t)
    steps = synth.integers(27, 9, B, 0, t) if ragged else np.full(B, t)
    lists = random_lists(28, B, Hkv, t // Z + 1, count, holes)
    out = st.attend_selected(bf16(q), st.new_out(), ints(lists), t, ints(steps) if ragged else None)
    assert_attend(out, q, K, V, lists, Z, steps, st.scale, "list")


@pytest.mark.parametrize("dtype", STORES)
def test_lists_without_keys_and_with_repeats(dtype):
    Hq, Hkv, D, Z, B, t = 6, 2, 128, 32, 3, 400
    st, q, K, V = filled(29, dtype, B, Hq, Hkv, D, Z, t)
    for count in (1, 5, 300):                                               # one split, several, more than eight
        lists = np.full((B, Hkv, count), -1)
        lists[1, 0, 0] = 12                                                 # the newest block, incomplete
        lists[2, :, -1] = 3
        if count > 1:
            lists[2, 0, :3] = 3                                             # counts as often as it is listed
        out = st.attend_selected(bf16(q), st.new_out().fill_(5.0), ints(lists), t)
        assert_attend(out, q, K, V, lists, Z, np.full(B, t), st.scale, f"{count} entries")


@pytest.mark.parametrize("dtype", STORES)
def test_blocks_that_are_not_listed_are_not_read_and_nan_shows(dtype):
    Hq, Hkv, D, Z, B, t = 4, 2, 64, 32, 1, 319
    st = make_store(30, dtype, B, Hq, Hkv, D, Z, t)
    q, K, V = normal(30, 1, (B, Hq, D)), normal(30, 2, (B, t + 1, Hkv, D)), normal(30, 3, (B, t + 1, Hkv, D))
    K[0, 2 * Z:3 * Z, 0, :] = np.nan                                          # block 2: nothing but NaN
    st.append_block(bf16(K), bf16(V), 0, t + 1)
    lists = np.array([[[0, 5, 9, -1], [1, 2, 3, 4]]])
    K0 = np.where(np.isnan(K), 0.0, K)
    out = st.attend_selected(bf16(q), st.new_out(), ints(lists), t)
    assert_attend(out, q, kept(dtype, K0), kept(dtype, V), lists, Z, np.full(B, t), st.scale, "NaN elsewhere")
    for entries in ([2], [2, -1, 0, -1], [2] * 40):
        out = st.attend_selected(bf16(q), st.new_out(), ints(np.array([[entries, entries]])), t)
        assert np.isnan(np64(out)[0, :2]).all() and np.isfinite(np64(out)[0, 2:]).all()


@pytest.mark.parametrize("dtype", STORES)
def test_all_blocks_are_the_dense_attention(dtype):
    Hq, Hkv, D, Z, B, t = 24, 8, 128, 64, 2, 777
    st, q, K, V = filled(31, dtype, B, Hq, Hkv, D, Z, t)
    lists = np.broadcast_to(np.arange(t // Z + 1), (B, Hkv, t // Z + 1))
    out = st.attend_selected(bf16(q), st.new_out(), ints(lists), t)
    assert_attend(out, q, K, V, lists, Z, np.full(B, t), st.scale, "all blocks")
    dense = np64(st.attend_causal(bf16(q), st.new_out(), t))
    size = oracle.attend(q, K, np.abs(V), t, 0, st.scale)
    assert (np.abs(np64(out) - dense) <= 2 * 1.03 * 2.0 ** -8 * (size + 2 * np.abs(dense))).all()


def test_offsets_beyond_32_bits():
    """The last blocks of a pool of more than 2^32 elements: bounds, choice, attention over a list, a whole step."""
    Hq, Hkv, D, Z, B, t = 6, 2, 128, 256, 1, 2047
    blocks = (1 << 32) // (Hkv * Z * D) + 40
    pools = [torch.empty((blocks, Hkv, Z * D), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    table = torch.arange(blocks - 1, blocks - 1 - (t // Z + 1), -1, dtype=torch.int32).reshape(1, -1)
    st = BlockStore(B, Hq, Hkv, D, Z, t, T.TEMPO_BF16, device=DEV, num_blocks=blocks, block_table=table, pools=pools)
    q, K, V = normal(36, 1, (B, Hq, D)), normal(36, 2, (B, t + 1, Hkv, D)), normal(36, 3, (B, t + 1, Hkv, D))
    st.append_block(bf16(K[:, :t]), bf16(V[:, :t]), 0, t)
    bounds = st.new_bounds()
    st.update_bounds(bounds, 0, t)
    selected = torch.empty((B, Hkv, 5), dtype=torch.int32, device=DEV)
    out = st.step_selected(bounds, bf16(q), bf16(K[:, t]), bf16(V[:, t]), st.new_out(), t, 5, selected=selected)
    lists = selected.cpu().numpy()
    for h in range(Hkv):
        keys = K[0, :, h].reshape(-1, Z, D)
        np.testing.assert_array_equal(lists[0, h], choose(q[0, 3 * h:3 * h + 3], keys.min(1), keys.max(1), t // Z, 5, 1, 1))
    assert_attend(out, q, K, V, lists, Z, np.full(B, t), st.scale, "far blocks")


# ---- together ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", STORES)
@pytest.mark.parametrize("Hq,Hkv,D,Z,B,prompt,steps,count,first,last", [(6, 2, 128, 32, 2, 150, 70, 4, 1, 2), (8, 2, 64, 32, 3, 100, 40, 6, 0, 1),
                                                                       (20, 1, 64, 64, 1, 0, 200, 2, 1, 1)])
def test_a_prompt_and_steps(dtype, Hq, Hkv, D, Z, B, prompt, steps, count, first, last):
    """Prompts of different lengths written and bounded, then steps of every sequence at its own position."""
    n, G = prompt + steps, Hq // Hkv
    K, V, q = normal(32, 2, (B, n, Hkv, D)), normal(32, 3, (B, n, Hkv, D)), normal(32, 1, (steps, B, Hq, D))
    st = make_store(32, dtype, B, Hq, Hkv, D, Z, n - 1)
    bounds = st.new_bounds().fill_(float("nan"))
    lengths = np.array([max(0, prompt - 37 * b) for b in range(B)])
    if prompt:
        st.append_block(bf16(K[:, :prompt]), bf16(V[:, :prompt]), 0, prompt)
        st.update_bounds(bounds, 0, prompt, count_per_seq=ints(lengths))
    Kh, Vh, table = kept(dtype, K), kept(dtype, V), st.block_table.cpu().numpy()
    rows = np.arange(B)
    for i in range(steps):
        at = lengths + i
        selected = torch.empty((B, Hkv, count), dtype=torch.int32, device=DEV)
        out = st.step_selected(bounds, bf16(q[i]), bf16(K[rows, at]), bf16(V[rows, at]), st.new_out(), int(at.max()), count, first, last,
                               ints(at), selected=selected)
        if i % 7 and i + 3 < steps:
            continue
        lists, edges = selected.cpu().numpy(), np64(bounds)
        for b in range(B):
            newest = at[b] // Z
            for h in range(Hkv):
                whole = [Kh[b, m * Z:(m + 1) * Z, h] for m in range((at[b] + 1) // Z)]
                lo, hi = (np.array([f(w, 0) for w in whole] + [np.zeros(D)] * (newest + 1 - len(whole))) for f in (np.min, np.max))
                for m in range(len(whole)):
                    np.testing.assert_array_equal(edges[table[b, m], h], np.stack([lo[m], hi[m]]))
                np.testing.assert_array_equal(lists[b, h], choose(q[i, b, h * G:(h + 1) * G], lo, hi, newest, count, first, last))
        assert_attend(out, q[i], Kh, Vh, lists, Z, at, st.scale, f"step {i}")


@pytest.mark.parametrize("dtype", STORES)
@pytest.mark.parametrize("Hq,Hkv,D,Z,B,t,count,first,last,ragged",
                         [(6, 2, 128, 32, 2, 32 * 192 - 1, 9, 1, 2, False), (6, 2, 128, 32, 2, 32 * 193 - 1, 9, 1, 2, False), (8, 2, 64, 32, 3, 7000, 40, 1, 2, True),
                          (20, 1, 64, 32, 2, 32 * 96 - 1, 7, 1, 1, False), (20, 1, 64, 32, 2, 32 * 97 - 1, 7, 1, 1, False), (16, 8, 64, 32, 32, 200, 3, 1, 2, True),
                          (16, 8, 64, 32, 33, 200, 3, 1, 2, True), (2, 2, 128, 64, 2, 63, 1, 0, 1, False), (6, 2, 128, 32, 1, 319, 5, 2, 3, False),
                          (128, 1, 128, 32, 2, 1999, 6, 0, 1, False)])
def test_a_step_is_its_parts(dtype, Hq, Hkv, D, Z, B, t, count, first, last, ragged):
    """The bits of the calls one by one: rows, bounds, choice and answers."""
    one, q, K, V = filled(35, dtype, B, Hq, Hkv, D, Z, t)
    two, *_ = filled(35, dtype, B, Hq, Hkv, D, Z, t)
    steps = ints(np.where(np.arange(B) % 3 == 1, (synth.integers(35, 9, B, 0, t) + 1) // Z * Z + Z - 1, synth.integers(35, 9, B, 0, t))) if ragged else None
    k, v = bf16(normal(35, 7, (B, Hkv, D))), bf16(normal(35, 8, (B, Hkv, D)))
    a, b = random_bounds(one, 35), random_bounds(two, 35)
    lists = torch.empty((B, Hkv, count), dtype=torch.int32, device=DEV)
    out = one.step_selected(a, bf16(q), k, v, one.new_out(), t, count, first, last, steps, selected=lists)
    two.append(k, v, t, steps)
    two.update_bounds(b, t, 1, steps)
    chosen = two.select_blocks(b, bf16(q), t, count, first, last, steps)
    assert torch.equal(lists, chosen) and torch.equal(out, two.attend_selected(bf16(q), two.new_out(), chosen, t, steps))
    for x, y in ((one.k_pool, two.k_pool), (one.v_pool, two.v_pool), (a, b)):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    assert (np.sort(lists.cpu().numpy(), axis=-1) == lists.cpu().numpy()).all() or t // Z < count or ragged


@pytest.mark.parametrize("dtype", STORES)
def test_captured_and_replayed_and_two_streams(dtype):
    Hq, Hkv, D, Z, B, t, count = 24, 8, 128, 64, 2, 4095, 8
    st, q, K, V = filled(33, dtype, B, Hq, Hkv, D, Z, t)
    bounds = st.new_bounds()
    st.update_bounds(bounds, 0, t)
    k, v, qd = bf16(K[:, t]), bf16(V[:, t]), bf16(q)
    selected = torch.empty((B, Hkv, count), dtype=torch.int32, device=DEV)
    eager = st.step_selected(bounds, qd, k, v, st.new_out(), t, count, selected=selected).clone()
    side, other = torch.cuda.Stream(), st.new_out()
    ws = torch.empty(T.tempo_attn_selected_workspace_bytes(st.kv, B, Hq, count), dtype=torch.uint8, device=DEV)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        T.tempo_attn_selected(st.kv, qd, other, selected, count, B, Hq, t, None, st.scale, ws, ws.numel())
    again = st.attend_selected(qd, st.new_out(), selected, t)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(eager, other) and torch.equal(eager, again)
    out, chosen, graph = st.new_out(), torch.empty_like(selected), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        st.step_selected(bounds, qd, k, v, out, t, count, selected=chosen)
    for i in range(4):
        qd.copy_(bf16(normal(40 + i, 1, (B, Hq, D))))
        eager = st.step_selected(bounds, qd, k, v, st.new_out(), t, count, selected=selected).clone()
        out.zero_()
        chosen.fill_(-9)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(chosen, selected)


@pytest.mark.parametrize("dtype", STORES)
@pytest.mark.parametrize("t0", [32 * 192 - 4, 90])
def test_a_captured_step_at_every_sequences_own_position(dtype, t0):
    """One capture for many steps: the positions are read from the device; blocks are completed on the way, and the number of blocks
    that the launch is made for lies on either side of what one workgroup scores itself."""
    Hq, Hkv, D, Z, B, steps, count = 6, 2, 64, 32, 3, 8, 4
    most = t0 + steps
    K, V, q = normal(36, 2, (B, most, Hkv, D)), normal(36, 3, (B, most, Hkv, D)), normal(36, 1, (steps, B, Hq, D))
    st, other = make_store(36, dtype, B, Hq, Hkv, D, Z, most + 40), make_store(36, dtype, B, Hq, Hkv, D, Z, most + 40)
    a, b = st.new_bounds(), other.new_bounds()
    lengths = np.array([t0, t0 // 2, 3])
    for s, bounds in ((st, a), (other, b)):
        s.append_block(bf16(K[:, :t0]), bf16(V[:, :t0]), 0, t0)
        s.update_bounds(bounds, 0, t0, count_per_seq=ints(lengths))
    at, qd = ints(lengths), bf16(q[0])
    k, v = torch.empty((B, Hkv, D), dtype=torch.bfloat16, device=DEV), torch.empty((B, Hkv, D), dtype=torch.bfloat16, device=DEV)
    out, chosen, selected = st.new_out(), torch.empty((B, Hkv, count), dtype=torch.int32, device=DEV), torch.empty((B, Hkv, count), dtype=torch.int32, device=DEV)
    need = T.tempo_step_selected_workspace_bytes(st.kv, B, Hq, most + 40, count)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        T.tempo_decode_step_selected(st.kv, a, qd, k, v, out, chosen, count, 1, 1, B, Hq, most + 40, at, st.scale, ws, need)
    for i in range(steps):
        now = lengths + i
        at.copy_(ints(now)), qd.copy_(bf16(q[i]))
        k.copy_(bf16(K[np.arange(B), now])), v.copy_(bf16(V[np.arange(B), now]))
        graph.replay()
        eager = other.step_selected(b, qd, k, v, other.new_out(), int(now.max()), count, 1, 1, ints(now), selected=selected)
        torch.cuda.synchronize()
        assert torch.equal(chosen, selected)
        err = np.abs(np64(out) - np64(eager))  # (another plan: another order of fp32 sums, and weights rounded under other references)
        assert (err <= 2 * 1.03 * 2.0 ** -8 * (np.abs(np64(eager)) * 2 + 4)).all()
    for x, y in ((st.k_pool, other.k_pool), (st.v_pool, other.v_pool)):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@pytest.mark.parametrize("dtype", STORES)
@pytest.mark.parametrize("Hq,Hkv,t0,count", [(6, 2, 32 * 192 - 4, 4), (6, 2, 90, 4), (40, 2, 700, 3), (6, 2, 4000, 60)])
def test_answers_of_a_captured_step_are_the_definitions(dtype, Hq, Hkv, t0, count):
    """Replays at every sequence's own position, each against the 64-bit answer over the chosen blocks: a key left out, taken
    twice or taken from another position shows."""
    D, Z, B, steps, G = 64, 32, 3, 8, Hq // Hkv
    most = t0 + steps
    K, V, q = normal(39, 2, (B, most, Hkv, D)), normal(39, 3, (B, most, Hkv, D)), normal(39, 1, (steps, B, Hq, D))
    Kh, Vh = kept(dtype, K), kept(dtype, V)
    st = make_store(39, dtype, B, Hq, Hkv, D, Z, most + 40)
    bounds, lengths = st.new_bounds(), np.array([t0, t0 // 2, 3])
    st.append_block(bf16(K[:, :t0]), bf16(V[:, :t0]), 0, t0)
    st.update_bounds(bounds, 0, t0, count_per_seq=ints(lengths))
    at, qd, k, v = ints(lengths), bf16(q[0]), bf16(K[:, 0]), bf16(V[:, 0])
    out, chosen, graph = st.new_out(), torch.empty((B, Hkv, count), dtype=torch.int32, device=DEV), torch.cuda.CUDAGraph()
    need = T.tempo_step_selected_workspace_bytes(st.kv, B, Hq, most + 40, count)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        T.tempo_decode_step_selected(st.kv, bounds, qd, k, v, out, chosen, count, 1, 1, B, Hq, most + 40, at, st.scale, ws, need)
    for i in range(steps):
        now = lengths + i
        at.copy_(ints(now)), qd.copy_(bf16(q[i]))
        k.copy_(bf16(K[np.arange(B), now])), v.copy_(bf16(V[np.arange(B), now]))
        graph.replay()
        torch.cuda.synchronize()
        lists = chosen.cpu().numpy()
        for b in range(B):
            whole = Kh[b, :(now[b] + 1) // Z * Z].reshape(-1, Z, Hkv, D)
            for h in range(Hkv):
                edges = np.zeros((2, now[b] // Z + 1, D))
                edges[0, :len(whole)], edges[1, :len(whole)] = whole[:, :, h].min(1), whole[:, :, h].max(1)
                np.testing.assert_array_equal(lists[b, h], choose(q[i, b, h * G:(h + 1) * G], *edges, now[b] // Z, count, 1, 1))
        assert_attend(out, q[i], Kh, Vh, lists, Z, now, st.scale, f"replay {i}")
