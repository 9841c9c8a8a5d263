"""Model.verify: a decoder stack over drafted trees, against the same stack run
token by token along every branch."""

import numpy as np
import pytest
import torch

from oracle import tree as ref
from paper_2606_09061_amd import model as M

pytestmark = pytest.mark.gpu

CFG = M.ModelConfig(hidden=256, layers=3, hq=4, hkv=2, head_dim=64, inter=512, vocab=1024)
# Both runs of the stack round to bf16 at the same places but attend in other
# orders.  A value is rounded some 8 times per layer, half a step of 2^-8 at
# most and about 2^-9.8 in the mean square each time: sqrt(2 * 3 * 8) 2^-9.8 =
# 0.8 % between the runs if every rounding fell apart, five times that allowed.
REL = 0.04


def _model(slots):
    return M.Model(CFG, max_seqs=slots, max_seq_len=256, max_tokens=2048, seed=11)


def _feed(m, rows, tokens):
    """One forward over given tokens; (greedy tokens of the rows, hidden states)."""
    tokens = torch.as_tensor(np.concatenate(tokens), device=m.dev, dtype=torch.int64)
    m.tokens[:len(tokens)] = tokens
    out = m.forward(np.array(rows, np.int32))
    return out.tolist(), m.x[:len(tokens)].clone()


def _close(a, b, what):
    a, b = a.double(), b.double()
    rel = ((a - b).norm(dim=-1) / b.norm(dim=-1)).max().item()
    print(f"  {what}: relative {rel:.2e}", flush=True)
    assert rel <= REL, what


def _logits(m, x):
    x = x.double()
    h = x / (x.pow(2).mean(-1, keepdim=True) + CFG.eps).sqrt() * m.final_norm.double()
    return h, h @ m.lm_head.double().t()


def _greedy(prompt, n):
    """The model's own continuation of a prompt."""
    m, out = _model(1), []
    token = _feed(m, [(0, 0, len(prompt), len(prompt))], [prompt])[0]
    for i in range(n):
        out.append(token[0])
        at = len(prompt) + i
        token = _feed(m, [(0, at, 1, at + 1)], [token])[0]
    return out


def test_verify_agrees_with_every_branch_run_alone():
    rng = np.random.default_rng(3)
    prompts = [rng.integers(0, CFG.vocab, 37), rng.integers(0, CFG.vocab, 20)]
    # trees: the model's own next tokens among wrong ones
    trees = []
    for prompt in prompts:
        g = _greedy(prompt, 5)
        #          0     1      2     3      4      5     6      7     8
        tokens = [g[0], 5,     g[1], g[1],  17,    g[2], 900,   g[3], 3]
        parents = [-1,  0,     0,    1,     2,     2,    5,     5,    7]
        trees.append((tokens, parents))
    rows = [(r, len(p), 9, len(p) + 9) for r, p in enumerate(prompts)]
    m = _model(3)
    _feed(m, [(r, 0, len(p), len(p)) for r, p in enumerate(prompts)], prompts)
    tokens = np.concatenate([t for t, _ in trees]).astype(np.int32)
    parents = np.concatenate([p for _, p in trees]).astype(np.int32)
    got = m.verify(rows, torch.from_numpy(tokens).to(m.dev), torch.from_numpy(parents).to(m.dev),
                   max_path=6)
    target, path, count, after = (t.cpu().numpy() for t in got)
    x = m.x[:18].clone()

    # the path follows from the targets, and holds the model's own tokens
    fake = np.zeros((18, CFG.vocab))
    fake[np.arange(18), target] = 1
    want = ref.verify(fake, tokens, parents, rows, 6)
    for a, b in zip((target, path, count, after), want):
        assert np.array_equal(a, b)
    assert count.min() >= 3, count

    # every node's chain on a slot of its own
    alone = _model(18)
    chains, begin = [], []
    for r, prompt in enumerate(prompts):
        for j in range(9):
            chains.append([trees[r][0][k] for k in reversed(ref.ancestors(parents[9 * r:9 * r + 9], j))])
            begin.append(prompt)
    _feed(alone, [(i, 0, len(p), len(p)) for i, p in enumerate(begin)], begin)
    rows2 = [(i, len(p), len(c), len(p) + len(c)) for i, (p, c) in enumerate(zip(begin, chains))]
    _, xs = _feed(alone, rows2, chains)
    last = np.cumsum([len(c) for c in chains]) - 1
    _close(x, xs[last], "hidden states of the nodes")
    h, logits = _logits(m, xs[last])
    slack = 2 * REL * h.norm(dim=-1) * m.lm_head.double().norm(dim=-1).max()
    chosen = logits[torch.arange(18), torch.from_numpy(target).long().to(m.dev)]
    assert (chosen >= logits.amax(-1) - slack).all()

    # what was kept: the next token decodes as behind the same chain alone
    nxt = [(r, len(p) + int(count[r]), 1, len(p) + int(count[r]) + 1) for r, p in enumerate(prompts)]
    _, y = _feed(m, nxt, [[after[0]], [after[1]]])
    ends = [9 * r + int(path[r, count[r] - 1]) for r in range(2)]
    _, z = _feed(alone, [(e, rows2[e][3], 1, rows2[e][3] + 1) for e in ends],
                 [[after[0]], [after[1]]])
    _close(y, z, "the token behind the accepted path")


def test_verify_of_single_nodes_is_a_decode_step():
    rng = np.random.default_rng(4)
    prompts = [rng.integers(0, CFG.vocab, n) for n in (12, 33, 5)]
    a, b = _model(3), _model(3)
    rows = [(r, 0, len(p), len(p)) for r, p in enumerate(prompts)]
    first = _feed(a, rows, prompts)[0]
    assert _feed(b, rows, prompts)[0] == first
    rows = [(r, len(p), 1, len(p) + 1) for r, p in enumerate(prompts)]
    _, x = _feed(a, rows, [[t] for t in first])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = b.verify(rows, torch.tensor(first, dtype=torch.int32, device=b.dev),
                   torch.full((3,), -1, dtype=torch.int32, device=b.dev), max_path=1, stream=s)
    s.synchronize()
    _close(b.x[:3], x, "single nodes")
    assert got[2].tolist() == [1, 1, 1] and got[1].tolist() == [[0], [0], [0]]
    assert torch.equal(got[0], got[3])


def test_verify_of_empty_batches_and_its_refusals():
    m = _model(2)
    none = torch.empty(0, dtype=torch.int32, device=m.dev)
    target, path, count, after = m.verify([(0, 5, 0, 5)], none, none, max_path=2)
    assert len(target) == 0 and count.tolist() == [0] and after.tolist() == [-1]
    assert path.tolist() == [[-1, -1]]
    for rows, most in (([(0, 0, 257, 257)], 2), ([(0, 0, 1, 1)], 0), ([(0, 0, 1, 1)], 257),
                       ([(0, 0, 2049, 2049)], 2)):
        with pytest.raises(ValueError):
            m.verify(rows, none, none, max_path=most)
    with pytest.raises(M.cp.CpError):
        m.verify([(0, 0, 2, 2)], none, none)
    bare = M.Model(CFG, max_seqs=1, max_seq_len=64, max_tokens=64, seed=1, lm_head=False)
    with pytest.raises(ValueError):
        bare.verify([(0, 0, 1, 1)], none, none)


def test_verify_refuses_other_tokens():
    """Before anything runs: the model's buffers and cache stay as they were."""
    m = _model(1)
    t = torch.zeros(3, dtype=torch.int32, device=m.dev)
    par = torch.tensor([-1, 0, 0], dtype=torch.int32, device=m.dev)
    m.pos.fill_(-7)
    m.x.fill_(2)
    before, kc = m.x.data_ptr(), [k.view(torch.int16).clone() for k in m.kc]
    for tok, parents in ((t[:2], par), (t.repeat(2), par), (t.long(), par), (t.cpu(), par),
                         (t[None], par), (t, par[:2]), (t, par.long()), (t, par.cpu())):
        with pytest.raises(M.cp.CpError):
            m.verify([(0, 0, 3, 3)], tok, parents)
    torch.cuda.synchronize()
    assert m.x.data_ptr() == before and m.x.shape[0] == 2048
    assert (m.x == 2).all() and (m.pos == -7).all()
    assert all(torch.equal(k.view(torch.int16), w) for k, w in zip(m.kc, kc))


def _drafted(m, seed=5):
    """A prompt of 30 tokens, then a star-shaped tree whose last node is the one
    that agrees: it moves over the others' slots."""
    rng = np.random.default_rng(seed)
    prompt = rng.integers(0, CFG.vocab, 30)
    after = _feed(m, [(0, 0, 30, 30)], [prompt])[0][0]
    m.verify([(0, 30, 1, 31)], torch.tensor([after], dtype=torch.int32, device=m.dev),
             torch.tensor([-1], dtype=torch.int32, device=m.dev))
    return after


def _star(m, root, right):
    tokens = torch.tensor([root, (right + 1) % CFG.vocab, (right + 2) % CFG.vocab, right],
                          dtype=torch.int32, device=m.dev)
    parents = torch.tensor([-1, 0, 0, 0], dtype=torch.int32, device=m.dev)
    return m.verify([(0, 30, 4, 34)], tokens, parents)


def test_verify_compacts_the_pools_that_the_layers_used():
    """A layer's pools replaced between two iterations: the next one appends to,
    attends over and compacts the new ones."""
    a, b = _model(1), _model(1)
    root = _drafted(a)
    assert _drafted(b) == root
    b.kc[1], b.vc[1] = b.kc[1].clone(), b.vc[1].clone()
    right = int(_star(a, root, 0)[0][0])        # what the root is followed by
    _star(b, root, 0)
    got, want = _star(b, root, right), _star(a, root, right)
    for x, y in zip(got, want):
        assert torch.equal(x, y)
    assert want[1][0, :3].tolist() == [0, 3, -1]
    # every layer's K and V of the committed tokens
    for x, y in zip(b.kc + b.vc, a.kc + a.vc):
        for p in (30, 31):
            at, slot = int(a.bt[0, p // CFG.block_size]), p % CFG.block_size
            is_k = x.shape[3] == CFG.head_dim
            u, w = (t[at, :, slot] if is_k else t[at, :, :, slot] for t in (x, y))
            assert torch.equal(u.view(torch.int16), w.view(torch.int16))


@pytest.mark.parametrize("which", ["tokens", "parents", "table"])
def test_verify_refuses_before_anything_runs(which):
    """Tokens or parents that are not dense, and rows outside the table."""
    m = _model(1)
    tokens = torch.zeros(6, dtype=torch.int32, device=m.dev)[::2]
    parents = torch.tensor([-1, -1, 0, 0, 0, 0], dtype=torch.int32, device=m.dev)[::2]
    if which != "tokens":
        tokens = tokens.contiguous()
    if which != "parents":
        parents = parents.contiguous()
    rows = [(1, 0, 3, 3)] if which == "table" else [(0, 0, 3, 3)]
    m.pos.fill_(-7)
    m.x.fill_(2)
    for x in m.kc + m.vc:
        x.fill_(3)
    with pytest.raises(M.cp.CpError):
        m.verify(rows, tokens, parents)
    torch.cuda.synchronize()
    assert (m.x == 2).all() and (m.pos == -7).all()
    assert all((x == 3).all() for x in m.kc + m.vc)


@pytest.mark.parametrize("change", ["shared", "shape", "missing"])
def test_verify_refuses_other_pools_before_anything_runs(change):
    m = _model(1)
    m.x.fill_(2)
    for x in m.kc + m.vc:
        x.fill_(3)
    pools = m.kc + m.vc
    if change == "shared":
        m.kc[2] = m.kc[1]
    elif change == "shape":
        m.vc[2] = m.vc[2][:-1]
    else:
        m.kc = m.kc[:2]
    t = torch.zeros(3, dtype=torch.int32, device=m.dev)
    with pytest.raises(M.cp.CpError):
        m.verify([(0, 0, 3, 3)], t, torch.tensor([-1, 0, 0], dtype=torch.int32, device=m.dev))
    torch.cuda.synchronize()
    assert (m.x == 2).all() and all((x == 3).all() for x in pools)
