"""kv_plan on the GPU against a loop over requests."""
import random

import pytest
import torch

from kv_testutil import plan as plan_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2606_04238_amd as qm
    qm.library()
    return qm


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def run(q, lens, new, table, free, n_free, page, tokens, plan=None):
    T, F = i32(table).view(len(lens), -1), i32(free)
    p = q.kv_plan(plan or q.KVPlan(len(lens), tokens), i32(lens), i32(new), T, F, i32([n_free]), page)
    torch.cuda.synchronize()
    return dict(slots=p.slots.tolist(), positions=p.positions.tolist(), starts=p.starts.tolist(), lens=p.lens.tolist(),
                n_free=p.n_free.tolist(), short=p.short.tolist(), table=T.tolist(), free=F.tolist())


def state(rng, B, W, page, spare, ended, most_new):
    lens = [rng.choice([0, 1, page - 1, page, page + 1, rng.randint(0, W * page)]) for _ in range(B)]
    lens = [min(x, W * page) for x in lens]
    used = [-(-x // page) for x in lens]
    ids = list(range(sum(used) + spare))
    rng.shuffle(ids)
    table, at = [[-7] * W for _ in range(B)], 0
    for b in range(B):
        table[b][:used[b]] = ids[at:at + used[b]]
        at += used[b]
    free = ids[at:] + [-9] * at
    new = [-1 if rng.random() < ended else rng.choice([0, 1, 1, 1, rng.randint(0, most_new)]) for _ in range(B)]
    return lens, new, table, free, spare


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("B,W,page,spare,ended,most", [
    (1, 1, 16, 0, 0.0, 3), (3, 5, 16, 2, 0.3, 40), (8, 9, 64, 20, 0.0, 1), (37, 12, 32, 9, 0.2, 60), (256, 7, 16, 60, 0.1, 30),
    (257, 5, 128, 300, 0.05, 200), (1025, 3, 16, 400, 0.3, 20), (2048, 3, 16, 1500, 0.2, 6), (70, 64, 256, 1000, 0.5, 3000)])
def test_against_a_loop(q, B, W, page, spare, ended, most, seed):
    rng = random.Random(1000 * B + seed)
    lens, new, table, free, n = state(rng, B, W, page, spare, ended, most)
    total = sum(max(x, 0) for x in new)
    tokens = rng.choice([total, total + 5, max(0, total - 3), 0 if seed == 3 else total])
    print("\n[case]", B, W, page, spare, "tokens", total, tokens, flush=True)
    got, want = run(q, lens, new, table, free, n, page, tokens), plan_ref(lens, new, table, free, n, page, tokens)
    for name in want:
        assert got[name] == want[name], name


def test_numbers_outside_their_range(q):
    """lens past the table, below zero and n_free past the stack are taken as the nearest inside."""
    lens, new, table, free = [-5, 1 << 30, 20, 33], [1, 1, -4, 0], [[-1, -1, -1], [0, 1, 2], [3, 4, 9], [5, 6, 7]], [8, 9, 10]
    for n in (-3, 0, 2, 3, 99):
        got, want = run(q, lens, new, table, free, n, 16, 9), plan_ref(lens, new, table, free, n, 16, 9)
        assert got == want, n


def test_sums_past_32_bits(q):
    """New tokens whose sum passes 2^31: starts stop there, nobody past `tokens` is served."""
    got = run(q, [0, 3, 5], [1, 2 ** 31 - 1, 2 ** 31 - 1], [[0, 0], [1, 1], [2, 2]], [3, 4], 2, 16, 4)
    assert got["starts"] == [0, 1, 2 ** 31 - 1, 2 ** 31 - 1] and got["lens"] == [1, 3, 5] and got["short"] == [2]
    assert got["slots"] == [64, -1, -1, -1] and got["positions"] == [0, 3, 4, 5] and got["n_free"] == [1]


def test_a_chain_in_place_and_a_graph(q):
    """lens and n_free advance in place, eagerly and in a replayed graph, pages end and are used again."""
    B, W, page = 5, 6, 16
    for graph in (False, True):
        lens, nf = i32([0] * B), i32([20])
        table, free, new = i32([[-1] * W] * B), i32(list(range(20))), i32([1] * B)
        p = q.KVPlan(B, 40, lens=lens, n_free=nf)
        step = lambda: q.kv_plan(p, lens, new, table, free, nf, page)
        if graph:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                step()
            torch.cuda.synchronize()
            lens.zero_(), nf.fill_(20), table.fill_(-1), free.copy_(torch.arange(20, dtype=torch.int32))
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                step()
            step = g.replay
        rng = random.Random(7)
        R = dict(lens=[0] * B, n_free=[20], table=[[-1] * W for _ in range(B)], free=list(range(20)))
        for i in range(60):
            add = [rng.choice([-1, 0, 1, 1, 7, 17]) for _ in range(B)]
            new.copy_(i32(add))
            step()
            torch.cuda.synchronize()
            R = plan_ref(R["lens"], add, R["table"], R["free"], R["n_free"][0], page, 40)
            assert lens.tolist() == R["lens"] and nf.tolist() == R["n_free"] and p.slots.tolist() == R["slots"], i
            assert table.tolist() == R["table"] and free.tolist() == R["free"] and p.short.tolist() == R["short"], i


def test_pages_past_the_last_slot(q):
    """A page number whose slots would pass 2^31 (or below 0) has none: slot -1, as for a refused request."""
    for page, last in ((16, 2 ** 27 - 1), (64, 2 ** 25 - 1), (256, 2 ** 23 - 1)):
        table = [[last, 0], [last + 1, 0], [2 * last + 2, 0], [-3, 0], [2 ** 31 - 1, 0], [7, 0]]
        got = run(q, [5] * 6, [2] * 6, table, [0], 0, page, 12)
        assert got["slots"] == [last * page + 5, last * page + 6, -1, -1, -1, -1, -1, -1, -1, -1, 7 * page + 5, 7 * page + 6], page
        assert got["lens"] == [7] * 6 and got["short"] == [0]
