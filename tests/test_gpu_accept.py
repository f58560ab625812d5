"""dsk_accept_draft against Python loops: whole numbers and copied rows, so equal or wrong."""
import numpy as np
import pytest
import torch

from step_testutil import D, accept_reference, i32, random_parents, starts

pytestmark = pytest.mark.gpu


def _dsk():
    import paper_2602_03184_amd as dsk
    return dsk


def _drafts(rng, n_new, spread=4, hit=0.85, vocab=1000):
    parents = [random_parents(rng, n, spread) for n in n_new]
    draft = [rng.integers(0, vocab, n).tolist() for n in n_new]
    target = []
    for up, tok in zip(parents, draft):
        t = rng.integers(0, vocab, len(up)).tolist()
        for i in range(len(up)):
            kids = [j for j in range(len(up)) if up[j] == i]
            if kids and rng.random() < hit:
                t[i] = tok[kids[int(rng.integers(0, len(kids)))]]
        target.append(t)
    return parents, draft, target


def _flat(x):
    return i32([v for y in x for v in y] or [0])


def _check(n_new, parents, draft, target, *, layers=2, Hkv=2, packed, max_nodes, max_path=None, room=None, lens=None, nhd=False):
    dsk = _dsk()
    B = len(n_new)
    lens = [3 + 5 * s for s in range(B)] if lens is None else lens
    row0 = starts([a + max(b, 1) + 2 for a, b in zip(lens, n_new)])
    rows = row0[-1] if room is None else room
    g = torch.Generator(device="cuda")
    g.manual_seed(1)

    def cache(n):
        if nhd:
            return torch.randn(layers, n, Hkv, D + 8, generator=g, device="cuda").bfloat16()[..., :D].transpose(1, 2)
        return torch.randn(layers, Hkv, n, D, generator=g, device="cuda").bfloat16()
    K, V = cache(rows), cache(rows)
    N, cu = sum(n_new), starts(n_new)
    Kd, Vd = (cache(max(N, 1)), cache(max(N, 1))) if packed else (None, None)
    K0, V0, ids = K.clone(), V.clone(), torch.full((rows,), -5, dtype=torch.int32, device="cuda")
    max_path = max_nodes if max_path is None else max_path
    acc = dsk.make_acceptor(K, V, seq_row0=i32(row0[:-1]), seq_len=i32(lens), cu_new=i32(cu), parent=_flat(parents),
                            draft_ids=_flat(draft), target_ids=_flat(target), max_nodes=max_nodes, max_path=max_path,
                            Kd=Kd, Vd=Vd, token_ids=ids)
    acc.step()
    torch.cuda.synchronize()
    want_ids, wantK, wantV = ids.clone().fill_(-5), K0.clone(), V0.clone()
    paths = []
    for s in range(B):
        left = max(0, rows - row0[s] - lens[s])
        n = n_new[s] if packed else min(n_new[s], left)
        path, nxt = accept_reference(parents[s][:n], draft[s], target[s], min(max_path, left))
        paths.append(path)
        assert acc.path[s].tolist() == path + [-1] * (max_path - len(path))
        assert int(acc.n_accepted[s]) == len(path) and int(acc.len_new[s]) == lens[s] + len(path) and int(acc.next_id[s]) == nxt
        for i, node in enumerate(path):
            at = row0[s] + lens[s] + i
            want_ids[at] = draft[s][node]
            for x, old, own in ((wantK, K0, Kd), (wantV, V0, Vd)):
                x[:, :, at] = own[:, :, cu[s] + node] if packed else old[:, :, row0[s] + lens[s] + node]
    assert torch.equal(ids, want_ids)
    assert torch.equal(K, wantK) and torch.equal(V, wantV)
    return acc, paths


@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("max_nodes", [1, 2, 33, 64, 65, 200, 256])
def test_trees(packed, max_nodes):
    rng = np.random.default_rng(max_nodes)
    n_new = [max_nodes, 0, 1, max_nodes // 2, max_nodes, max(1, max_nodes - 1), max_nodes]
    _check(n_new, *_drafts(rng, n_new, spread=2 if max_nodes > 64 else 4, hit=0.97), packed=packed, max_nodes=max_nodes,
           nhd=max_nodes == 64)


@pytest.mark.parametrize("packed", [True, False])
def test_a_chain_that_is_accepted_whole_and_one_that_is_not_at_all(packed):
    chain = [list(range(-1, 39))] * 2                            # many more rows than are on their way at once
    draft = [list(range(100, 140))] * 2
    target = [list(range(101, 141)), [7] * 40]
    acc, _ = _check([40, 40], chain, draft, target, packed=packed, max_nodes=40)
    assert acc.n_accepted.tolist() == [40, 1] and acc.next_id.tolist() == [140, 7]


def test_the_lowest_of_equal_children_is_taken_and_only_later_nodes_count():
    #        0 <- 1, 2, 3 (all the right token); 3 <- 4; a "parent" behind its child never ends a walk
    _check([5], [[-1, 0, 0, 0, 3]], [[9, 5, 5, 5, 6]], [[5, 6, 6, 6, 1]], packed=True, max_nodes=5)
    _check([4], [[1, 0, 3, 2]], [[9, 5, 5, 5]], [[5, 5, 5, 5]], packed=True, max_nodes=4)
    _check([2], [[0, 0]], [[5, 5]], [[5, 5]], packed=True, max_nodes=2)


@pytest.mark.parametrize("layers, Hkv", [(1, 1), (3, 5), (32, 8)])
def test_layers_and_heads(layers, Hkv):
    rng = np.random.default_rng(3)
    _check([20, 6], *_drafts(rng, [20, 6], hit=1.0), packed=False, max_nodes=20, layers=layers, Hkv=Hkv)


@pytest.mark.parametrize("packed", [True, False])
def test_paths_end_with_their_room(packed):
    dsk = _dsk()
    chain, draft, target = [list(range(-1, 9))], [list(range(10))], [list(range(1, 11))]
    acc, paths = _check([10], chain, draft, target, packed=packed, max_nodes=10, max_path=4)
    assert len(paths[0]) == 4 and int(acc.dev_status.item()) == dsk.DSK_ERR_CAPACITY
    acc, paths = _check([10], chain, draft, target, packed=packed, max_nodes=10, lens=[20], room=26)
    assert len(paths[0]) == 6 and int(acc.dev_status.item()) == dsk.DSK_ERR_CAPACITY
    acc, paths = _check([10], chain, draft, target, packed=packed, max_nodes=10, lens=[20], room=20)
    assert paths[0] == []


def test_the_walk_alone_and_a_table_that_does_not_fit():
    dsk = _dsk()
    common = dict(seq_row0=i32([0, 50]), seq_len=i32([5, 6]), parent=i32([-1, 0, 1, -1, 0]), draft_ids=i32([1, 2, 3, 4, 5]),
                  target_ids=i32([2, 3, 9, 5, 8]), max_nodes=3, total_rows=100)
    acc = dsk.make_acceptor(None, None, cu_new=i32([0, 3, 5]), **common)
    acc.step()
    torch.cuda.synchronize()
    assert acc.path.tolist() == [[0, 1, 2], [0, 1, -1]] and acc.next_id.tolist() == [9, 8]
    assert acc.len_new.tolist() == [8, 8] and int(acc.dev_status.item()) == 0
    for cu, path in (([0, 3, 9], [[0, 1, 2], [0, 1, -1]]), ([0, 4, 5], [[0, 1, 2], [0, -1, -1]]),
                     ([-1, 3, 2], [[-1, -1, -1], [-1, -1, -1]])):
        acc = dsk.make_acceptor(None, None, cu_new=i32(cu), **common)
        acc.step()
        torch.cuda.synchronize()
        assert acc.path.tolist() == path and int(acc.dev_status.item()) == dsk.DSK_ERR_SHAPE


def test_rows_and_layers_beyond_32_bits():
    """Layers 2^30 channels apart, and rows of 10240 channels of which the last lie beyond 2^31."""
    dsk = _dsk()
    step, chain = 1 << 30, [list(range(-1, 11))]
    draft, target = [list(range(100, 112))], [list(range(101, 113))]
    common = dict(cu_new=i32([0, 12]), parent=_flat(chain), draft_ids=_flat(draft), target_ids=_flat(target), max_nodes=12)
    own = torch.randn(4, 3, 2, 12, D, device="cuda").bfloat16()  # of K and V; layers, heads, nodes
    base = torch.empty(2 * step + 400 * D, dtype=torch.bfloat16, device="cuda")
    K, V = (base.as_strided((3, 2, 50, D), (step, 100 * D, D, 1), o) for o in (0, 200 * D))
    acc = dsk.make_acceptor(K, V, seq_row0=i32([5]), seq_len=i32([30]), Kd=own[0], Vd=own[1], **common)
    acc.step()
    torch.cuda.synchronize()
    assert acc.path.tolist() == [list(range(12))]
    assert torch.equal(K[:, :, 35:47], own[0]) and torch.equal(V[:, :, 35:47], own[1])
    del base, K, V
    cache = torch.empty(225_000, 80, D, dtype=torch.bfloat16, device="cuda")
    K, V = cache[:, 2:4].transpose(0, 1), cache[:, 78:80].transpose(0, 1)
    skip = [[-1, 0, 0, 2, 2, 4, 4, 6, 6, 8, 8, 10]]              # 0 and its even descendants
    draft = [[1, 90, 2, 90, 3, 90, 4, 90, 5, 90, 6, 90]]
    target = [[2, 0, 3, 0, 4, 0, 5, 0, 6, 0, 7, 0]]
    at = 100_000 + 120_000
    K[:, at:at + 12], V[:, at:at + 12] = own[2, 0], own[3, 0]
    common.update(parent=_flat(skip), draft_ids=_flat(draft), target_ids=_flat(target))
    acc = dsk.make_acceptor(K, V, seq_row0=i32([100_000]), seq_len=i32([120_000]), **common)
    acc.step()
    torch.cuda.synchronize()
    assert acc.path[0, :6].tolist() == [0, 2, 4, 6, 8, 10] and int(acc.next_id) == 7
    for X, old in ((K, own[2, 0]), (V, own[3, 0])):
        assert torch.equal(X[:, at:at + 6], old[:, ::2]) and torch.equal(X[:, at + 6:at + 12], old[:, 6:])
    del cache, K, V
    torch.cuda.empty_cache()


def test_no_token_at_all():
    dsk = _dsk()
    K, V = (torch.full((1, 2, 9, D), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    none = i32([])
    acc = dsk.make_acceptor(K, V, seq_row0=i32([0, 5]), seq_len=i32([3, 2]), cu_new=i32([0, 0, 0]), parent=none, draft_ids=none,
                            target_ids=none, max_nodes=4)
    acc.step()
    torch.cuda.synchronize()
    assert acc.n_accepted.tolist() == [0, 0] and acc.len_new.tolist() == [3, 2] and acc.next_id.tolist() == [-1, -1]
    assert bool((acc.path == -1).all()) and bool((K == 5.0).all()) and bool((V == 5.0).all())


@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("room, end", [(6, 3), (4, 4), (4, 5), (1, 1), (1, 2), (0, 0), (0, 1)])
def test_only_a_path_that_is_cut_reports_its_end(packed, room, end):
    """A chain of 10 nodes of which `end` are right, in a cache with rows for `room` of them: the status says whether a further
    node would have been accepted, not whether there are nodes without a row."""
    dsk = _dsk()
    chain, draft = [list(range(-1, 9))] if end else [[]], [list(range(10))] if end else [[]]
    target = [[t + 1 if t + 1 < end else 99 for t in range(10)]] if end else [[]]
    acc, paths = _check([10 if end else 0], chain, draft, target, packed=packed, max_nodes=10, lens=[20], room=20 + room)
    assert len(paths[0]) == min(room, end)
    assert int(acc.dev_status.item()) == (dsk.DSK_ERR_CAPACITY if end > room else 0)
