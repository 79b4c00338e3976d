"""Token streams at the end of their room: the last rows' trees, prompts that do not fit, sequences that are full."""
import pytest
import torch

from test_gpu_speculative import Speaker, near, whole

pytestmark = pytest.mark.gpu
BF16, I32 = torch.bfloat16, torch.int32

# 25 nodes: node 20 is the third of a branch (0, 8, 20), which twenty other nodes separate from the root
TREE = [-1] + [0] * 8 + [1 + i % 8 for i in range(8)] + [8] * 8


def branch(up, j):
    return (branch(up, up[j]) if up[j] >= 0 else []) + [j]


def rows(gen, n):
    return torch.randn(n, 256, generator=gen).to(BF16).cuda()


def check_nodes(lib, sp, st, seqs, up):
    """Every node's hidden row is that of its branch behind the sequence alone."""
    emb = st.embeds.view(len(seqs), len(up), 256)
    got = st.hidden.float().cpu().view(len(seqs), len(up), 256)
    for i, s in enumerate(seqs):
        want = whole(lib, sp.ctx, sp.bb, [torch.cat([s, emb[i, branch(up, j)]]) for j in range(len(up))])
        near([got[i, j: j + 1] for j in range(len(up))], [w[-1:] for w in want])


def test_a_trees_rows_have_places_up_to_the_last_run(lib):
    """45 rows of 64 and a tree of 25: its nodes end at place 69, a kept one of them moves, and the next tree sees it."""
    from paper_2607_16074_amd import step
    sp, gen = Speaker(lib), torch.Generator().manual_seed(1)
    st = step.SpeculativeStep(sp.model, [0], [1], 64, 25, TREE, 16)
    seq = rows(gen, 45)
    st.prefill(seq, [45])
    for path in ([0, 8, 20], [0, 8, 24], [0, 3, 11]):
        st.embeds.copy_(rows(gen, 25))
        st.extend()
        torch.cuda.synchronize()
        check_nodes(lib, sp, st, [seq], TREE)
        st.path[0, :3] = torch.tensor(path, dtype=I32)
        st.n_path.fill_(3)
        st.keep()
        seq = torch.cat([seq, st.embeds[path]])
    assert st.past.tolist() == [54]


@pytest.mark.parametrize("parents", [None, [-1, 0, 0, 1, 1, 2]])
@pytest.mark.parametrize("captured", [False, True])
def test_a_full_sequence_stands_still_beside_others(lib, parents, captured):
    """Runs go on while a sequence has fewer rows than its room; then it keeps its rows, and says so, and others go on."""
    from paper_2607_16074_amd import step
    sp, gen = Speaker(lib), torch.Generator().manual_seed(2)
    nodes = len(parents) if parents else 4
    up = parents or list(range(-1, nodes - 1))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        st = step.SpeculativeStep(sp.model, [0, 1], [1, 2], 37, nodes, parents, 16, lib.Context(side))
        seqs = [rows(gen, n) for n in (31, 37, 3)]
        st.prefill(torch.cat(seqs), [31, 37, 3])
        graph = None
        if captured:
            past = st.past.clone()
            st.run()  # (everything is loaded before a capture)
            st.past.copy_(past)
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                st.run()
        for turn in range(9):
            st.embeds.copy_(rows(gen, 3 * nodes))
            st.tokens.copy_(torch.randint(0, 33, (3 * nodes,), generator=gen))
            before = st.past.tolist()
            graph.replay() if graph else st.run()
            side.synchronize()
            after, count, nxt, path = (t.tolist() for t in (st.past, st.n_path, st.next, st.path))
            emb = st.embeds.view(3, nodes, 256)
            going = [i for i in range(3) if before[i] < 37]
            for i in range(3):
                if i not in going:
                    assert (after[i], count[i], nxt[i], path[i]) == (before[i], 0, -1, [-1] * nodes)
                    continue
                assert after[i] == before[i] + count[i] and count[i] >= 1 and 0 <= nxt[i] < (40, 33, 33)[i]
                want = whole(lib, sp.ctx, sp.bb, [torch.cat([seqs[i], emb[i, branch(up, j)]]) for j in range(nodes)])
                got = st.hidden.float().cpu().view(3, nodes, 256)[i]
                near([got[j: j + 1] for j in range(nodes)], [w[-1:] for w in want])
                seqs[i] = torch.cat([seqs[i], emb[i, path[i][: count[i]]]])
        assert before[0] >= 37 and before[1] == 37 and before[2] < 37


def test_a_full_sequence_samples_nothing(lib):
    """The same of a step against the caller's probabilities."""
    from paper_2607_16074_amd import step
    sp, gen = Speaker(lib), torch.Generator().manual_seed(3)
    st = step.SpeculativeStep(sp.model, [0], [2], 16, 2, None, 16)
    st.prefill(rows(gen, 20), [16, 4])
    st.embeds.copy_(rows(gen, 4))
    st.tokens.fill_(5)
    p = torch.zeros(4, 40, device="cuda")
    p[:, 5] = 1.0
    st.extend()
    st.sample([p], torch.full((4,), 0.5, device="cuda"), torch.full((2,), 0.5, device="cuda"))
    st.keep()
    assert (st.n_path.tolist(), st.next.tolist(), st.past.tolist()) == ([0, 2], [-1, 5], [16, 6])
    assert st.path.tolist() == [[-1, -1], [0, 1]]


@pytest.mark.parametrize("side", [False, True])
def test_prompts_beyond_the_room_are_refused(lib, side):
    """Whatever call they come in, and before anything is written; what fits exactly is taken."""
    from paper_2607_16074_amd import step
    sp, gen = Speaker(lib), torch.Generator().manual_seed(4)
    ctx = lib.Context(torch.cuda.Stream()) if side else None
    st = step.SpeculativeStep(sp.model, [0], [2], 48, 1, page_size=16, ctx=ctx)
    x, y = rows(gen, 48), rows(gen, 3)
    st.prefill(torch.cat([x[:40], y]), [40, 3])
    torch.cuda.synchronize()
    k, v = st.cache.k.clone(), st.cache.v.clone()
    for lens in ([40, 0], [9, 1]):
        with pytest.raises(ValueError, match="room"):
            st.prefill(rows(gen, sum(lens)), lens)
    torch.cuda.synchronize()
    assert st.past.tolist() == [40, 3] and torch.equal(st.cache.k, k) and torch.equal(st.cache.v, v)
    got = st.prefill(x[40:], [8, 0])
    torch.cuda.synchronize()
    near([got.float().cpu()], [whole(lib, sp.ctx, sp.bb, [x])[0][40:]])
    assert st.past.tolist() == [48, 3]
    st.prefill(x[:0], [0, 0])
    with pytest.raises(ValueError, match="room"):
        st.prefill(rows(gen, 1), [1, 0])
    st.prefill(rows(gen, 1), [0, 1])  # (a full sequence does not keep others from theirs)
    torch.cuda.synchronize()
    assert st.past.tolist() == [48, 4]
