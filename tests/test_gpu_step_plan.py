"""dsk_step_plan against Python loops: whole numbers, so equal or wrong."""
import numpy as np
import pytest
import torch

from step_testutil import ancestors, i32, pack_mask, random_parents, starts

pytestmark = pytest.mark.gpu


def _dsk():
    import paper_2602_03184_amd as dsk
    return dsk


def _run(n_new, lens, row0, total_rows, max_tokens, parents=None, max_nodes=0, want_mask=None):
    dsk = _dsk()
    flat = None
    if parents is not None:
        flat = i32(([p for up in parents for p in up] + [7] * max_tokens)[:max_tokens])   # rubbish behind the last
    p = dsk.make_step_plan(seq_row0=i32(row0), seq_len=i32(lens), n_new=i32(n_new), max_tokens=max_tokens,
                           total_rows=total_rows, parent=flat, max_nodes=max_nodes, want_mask=want_mask)
    for t in (p.tok_seq, p.tok_pos, p.tok_row) + ((p.mask,) if p.mask is not None else ()):
        t.fill_(77)
    p.step()
    torch.cuda.synchronize()
    return p


def _expect(p, n_new, lens, row0, max_tokens, depth, status=0):
    cu = np.minimum(starts(n_new), max_tokens)
    assert p.cu_new.tolist() == cu.tolist()
    seq, pos, row = [-1] * max_tokens, [0] * max_tokens, [-1] * max_tokens
    for s in range(len(n_new)):
        for i, t in enumerate(range(cu[s], cu[s + 1])):
            seq[t], pos[t], row[t] = s, lens[s] + depth[s][i], row0[s] + lens[s] + i
    assert p.tok_seq.tolist() == seq and p.tok_pos.tolist() == pos and p.tok_row.tolist() == row
    assert int(p.dev_status.item()) == status


@pytest.mark.parametrize("n_new", [[1], [0], [0, 0, 5], [3, 0, 0, 1], [1024], [1023, 1, 1025], [5000, 1, 0, 777],
                                   [1] * 255, [2] * 256, [1] * 257, list(range(300)), [0] * 1000 + [1, 0, 2]])
@pytest.mark.parametrize("spare", [0, 9])
def test_prompts(n_new, spare):
    """Tokens that follow each other: counts around the tile of a workgroup, empty sequences, more sequences than threads."""
    rng = np.random.default_rng(len(n_new))
    lens = rng.integers(0, 5000, len(n_new)).tolist()
    row0 = starts([a + b for a, b in zip(lens, n_new)])
    most = max(sum(n_new) + spare, 1)
    p = _run(n_new, lens, row0[:-1], row0[-1], most)
    _expect(p, n_new, lens, row0, most, [list(range(n)) for n in n_new])
    assert p.mask is None


@pytest.mark.parametrize("max_nodes", [1, 31, 32, 33, 64, 65, 200, 256])
def test_trees(max_nodes):
    rng = np.random.default_rng(max_nodes)
    n_new = [max_nodes, 0, 1, max_nodes // 2, max_nodes, max(1, max_nodes - 1)] + [max_nodes] * 3
    parents = [random_parents(rng, n, spread=1 if s == 0 else 6, forest=s == 3) for s, n in enumerate(n_new)]
    lens = rng.integers(0, 70000, len(n_new)).tolist()
    row0 = starts([a + b for a, b in zip(lens, n_new)])
    p = _run(n_new, lens, row0[:-1], row0[-1], sum(n_new) + 5, parents, max_nodes)
    seen = [ancestors(up) for up in parents]
    _expect(p, n_new, lens, row0, sum(n_new) + 5, [d for _, d in seen])
    want = pack_mask([m for m, _ in seen] + [np.zeros((5, 1), dtype=bool)], (max_nodes + 31) // 32)
    assert torch.equal(p.mask.cpu(), want)


def test_mask_of_a_chain_and_positions_without_masks():
    n_new, lens, row0 = [40, 3], [10, 0], [0, 60]
    p = _run(n_new, lens, row0, 100, 43, None, 40, want_mask=True)
    _expect(p, n_new, lens, row0, 43, [list(range(n)) for n in n_new])
    assert torch.equal(p.mask.cpu(), pack_mask([np.tril(np.ones((n, n), dtype=bool)) for n in n_new], 2))
    rng = np.random.default_rng(1)
    parents = [random_parents(rng, n) for n in n_new]
    p = _run(n_new, lens, row0, 100, 43, parents, 40, want_mask=False)
    _expect(p, n_new, lens, row0, 43, [ancestors(up)[1] for up in parents])


def test_what_does_not_fit_is_reported_and_cut():
    dsk = _dsk()
    p = _run([4, 5], [0, 0], [0, 10], 100, 7)                    # more tokens than the arrays hold
    _expect(p, [4, 5], [0, 0], [0, 10], 7, [range(4), range(5)], dsk.DSK_ERR_CAPACITY)
    p = _run([2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1], [0, 0, 0], [0, 0, 0], 100, 3)   # sums beyond 32 bits
    assert p.cu_new.tolist() == [0, 3, 3, 3] and int(p.dev_status.item()) == dsk.DSK_ERR_CAPACITY
    p = _run([3, -2, 1], [0, 0, 0], [0, 10, 20], 100, 4)
    _expect(p, [3, 0, 1], [0, 0, 0], [0, 10, 20], 4, [range(3), [], range(1)], dsk.DSK_ERR_SHAPE)
    p = _run([3], [98], [0], 100, 3)                             # rows behind the cache's end
    assert p.tok_row.tolist() == [98, 99, -1] and p.tok_pos.tolist() == [98, 99, 100]
    assert int(p.dev_status.item()) == dsk.DSK_ERR_CAPACITY
    p = _run([1, 1, 1], [2 ** 31 - 1, -1, 0], [5, 5, -1], 100, 3)
    assert p.tok_row.tolist() == [-1, -1, -1] and int(p.dev_status.item()) == dsk.DSK_ERR_CAPACITY
    p = _run([9, 2], [0, 0], [0, 10], 100, 11, [[-1, 0, 1, 2, 3, 4, 5, 6, 7], [-1, 0]], 4)   # a larger tree than announced
    assert p.cu_new.tolist() == [0, 4, 6] and int(p.dev_status.item()) == dsk.DSK_ERR_SHAPE


@pytest.mark.parametrize("parent", [[-1, 1, 0], [-1, 5, 0], [-1, -7, 0], [0, 0, 0]])
def test_parents_that_are_none(parent):
    """A node that follows itself, a later node or nothing that exists is taken as a root, and the walk ends."""
    dsk = _dsk()
    p = _run([3], [10], [0], 100, 3, [parent], 32)
    kept = [u if -1 <= u < j else -1 for j, u in enumerate(parent)]
    seen, depth = ancestors(kept)
    _expect(p, [3], [10], [0], 3, [depth], dsk.DSK_ERR_ORDER)
    assert torch.equal(p.mask.cpu(), pack_mask([seen], 1))


def test_many_sequences():
    n_new = [(7 * s) % 5 for s in range(65535)]
    row0 = starts([n + 2 for n in n_new])
    lens = [2] * len(n_new)
    most = sum(n_new) + 100
    p = _run(n_new, lens, row0[:-1], row0[-1], most)
    _expect(p, n_new, lens, row0, most, [range(n) for n in n_new])


def test_masks_beyond_32_bits():
    """2^28 tokens and more with mask rows of eight words."""
    dsk = _dsk()
    n = (1 << 28) + 5
    p = dsk.make_step_plan(seq_row0=i32([0, 1000]), seq_len=i32([10, 20]), n_new=i32([256, 200]), max_tokens=n, total_rows=2000,
                           max_nodes=256, want_mask=True)
    p.step()
    torch.cuda.synchronize()
    assert p.cu_new.tolist() == [0, 256, 456] and int(p.dev_status) == 0
    for t in (p.tok_seq[456:], p.tok_row[456:]):
        assert int(t.min()) == int(t.max()) == -1
    assert int(p.mask[456:].abs().max()) == 0
    assert p.mask[255].tolist() == [-1] * 8 and p.mask[455].tolist() == [-1] * 6 + [(1 << 8) - 1, 0]
    del p, t
    torch.cuda.empty_cache()


def test_counts_that_pass_32_bits_when_added():
    dsk = _dsk()
    most = 2 ** 31 - 1
    for B in (5, 300):                                           # a sequence a thread, and several
        p = dsk.make_step_plan(seq_row0=i32([0] * B), seq_len=i32([3] * B), n_new=i32([2] + [most] * (B - 1)), max_tokens=most,
                               total_rows=100)
        p.step()
        torch.cuda.synchronize()
        assert p.cu_new.tolist() == [0, 2] + [most] * (B - 1) and int(p.dev_status) == dsk.DSK_ERR_CAPACITY
        assert p.tok_seq[:4].tolist() == [0, 0, 1, 1] and p.tok_row[:4].tolist() == [3, 4, 3, 4]
        assert p.tok_seq[-2:].tolist() == [1, 1] and p.tok_row[-1:].tolist() == [-1] and p.tok_pos[-1:].tolist() == [most - 1 - 2 + 3]
        del p
        torch.cuda.empty_cache()
