"""Steps as a server runs them: drafted trees verified and compacted, beams forked and reordered.

A token's QKV row depends on the token alone (a table per layer), so that what the cache has to hold for a request follows from its tokens and
positions; outputs are held against the 64-bit definitions over exactly those tokens."""
import threading

import numpy as np
import pytest
import torch

from branching_inputs import TreeCase, random_parents
from oracle import branching, serving
from serving_inputs import BF16_HALF

pytestmark = pytest.mark.gpu

L, HQ, HK, D, PAGE, VOCAB = 2, 8, 2, 64, 16, 300


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2604_12782_b200 import binding
    return binding


def dev(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def zeros(*shape):
    return torch.zeros(*shape, dtype=torch.int32, device="cuda")


class Server:
    """Caches of L layers, page tables of R rows, and the pool of free pages on the host."""

    def __init__(self, B, R, n_pages=120, cols=24, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.B, self.R, self.cols, self.n_pages = B, R, cols, n_pages
        self.tables = [(torch.randn(VOCAB, (HQ + 2 * HK) * D, generator=g) * 1.5).to(torch.bfloat16) for _ in range(L)]
        nan = float("nan")
        self.k = torch.full((L, n_pages, PAGE, HK, D), nan, dtype=torch.bfloat16, device="cuda")
        self.v = torch.full((L, n_pages, PAGE, HK, D), nan, dtype=torch.bfloat16, device="cuda")
        self.caches = [B.KvCache(k, v) for k, v in zip(self.k, self.v)]
        self.layers = B.KvLayers(self.caches)
        self.table, self.len = torch.full((R, cols), -1, dtype=torch.int32, device="cuda"), zeros(R)
        self.refs = zeros(n_pages)
        self.free = list(np.random.default_rng(seed).permutation(n_pages))
        self.inv = (1e-4 ** (np.arange(D // 2) / (D // 2))).astype(np.float32)
        self.rope = B.Rope(torch.from_numpy(self.inv).cuda())
        self.gq, self.gk = (torch.rand(D, generator=g).to(torch.bfloat16) + 0.5 for _ in range(2))
        self.scale = D ** -0.5

    def step(self, tokens, new, parents=None):
        """New tokens of every row (a tree's where there are parents, else in order).  Returns the layers' attention outputs [T, HQ, D]."""
        B, T = self.B, len(tokens)
        row, kv, slots, pos, taken = zeros(self.R + 1), zeros(self.R), zeros(T), zeros(T), zeros(1)
        B.osc_kv_slots(self.len, dev(new), None, PAGE, dev(self.free), self.table, row, kv, slots, pos, taken)
        mask = zeros(T, 2) if parents is not None else None
        if parents is not None:
            B.osc_tree_mask(dev(parents), row, self.len, mask, pos)
        ws = torch.empty(B.osc_paged_attention_workspace_bytes(T, HQ, D, self.R), dtype=torch.uint8, device="cuda")
        out = []
        for layer in range(L):
            q, o = (torch.empty(T, HQ * D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            B.osc_qk_norm_rope(self.tables[layer][torch.as_tensor(np.asarray(tokens))].cuda(), HQ, self.caches[layer], q, pos, self.rope, gamma_q=self.gq.cuda(),
                               gamma_k=self.gk.cuda(), slots=slots)
            if parents is None:
                B.osc_paged_attention(q, self.caches[layer], row, kv, self.table, o, ws, self.scale, max_new=max(new))
            else:
                B.osc_tree_attention(q, self.caches[layer], row, kv, self.table, mask, o, ws, self.scale, max_new=max(new))
            out.append(o.view(T, HQ, D))
        n = taken.item()
        for p in self.free[:n]:
            self.refs[int(p)] += 1
        self.free = self.free[n:]
        self.row, self.kv, self.pos = row, kv, pos
        return out

    def heads(self, layer, tokens, positions):
        """(queries, keys, values) of tokens at positions, in 64 bits, before any rounding but the table's."""
        x = self.tables[layer][torch.as_tensor(np.asarray(tokens))].double().numpy().reshape(len(tokens), HQ + 2 * HK, D)
        p = np.asarray(positions)[None]
        q, _ = serving.qk_norm_rope(x[:, :HQ], self.gq.double().numpy(), 1e-6, self.inv, None, p, False)
        k, _ = serving.qk_norm_rope(x[:, HQ:HQ + HK], self.gk.double().numpy(), 1e-6, self.inv, None, p, False)
        return q, k, x[:, HQ + HK:]

    def check(self, out, t, history, token):
        """Row t of a step's outputs: `token` behind `history`."""
        for layer in range(L):
            n = len(history)
            q, k, v = self.heads(layer, list(history) + [token], range(n + 1))
            o, _, av, sm = serving.attention(q[-1:].reshape(1, HK, HQ // HK, D), k, v, np.array([n + 1]), self.scale)
            # Queries and keys are rounded to bf16 in the kernels (half a step each), which moves a score by at most 2 * 2^-8 (and a second order) of
            # the sum of magnitudes sm, and a weight by e^(+-2 d) against the others; weights in bf16 and the output's rounding: half a step each.
            d = 2.02 * BF16_HALF * sm[0][..., None]
            err = (np.expm1(2 * d) + BF16_HALF + 2.0 ** -16) * av[0]
            tol = err + BF16_HALF * (np.abs(o[0]) + err)
            got = out[layer][t].double().cpu().numpy().reshape(HK, HQ // HK, D)
            assert (np.abs(got - o[0]) <= tol).all(), (layer, t, np.max(np.abs(got - o[0]) / tol))

    def give_back(self, to):
        freed, n = torch.full((self.n_pages,), -1, dtype=torch.int32, device="cuda"), zeros(1)
        self.B.osc_kv_trim(self.len, to, PAGE, self.table, self.refs, freed, n)
        self.free = self.free + freed[:n.item()].tolist()


def test_trees_verified_step_by_step(B):
    R = 3
    s, rng = Server(B, R), np.random.default_rng(1)
    history = [list(rng.integers(0, VOCAB, n)) for n in (40, 5, 17)]
    out = s.step(sum(history, []), [len(h) for h in history])
    for r in range(R):
        t = sum(len(h) for h in history[:r + 1]) - 1
        s.check(out, t, history[r][:-1], history[r][-1])
    s.len.copy_(s.kv)
    for step in range(4):
        new = [int(rng.integers(1, 50)) for _ in range(R)]
        parents = [random_parents(rng, n) for n in new]
        tokens = [rng.integers(0, VOCAB, n) for n in new]
        out = s.step(np.concatenate(tokens), new, np.concatenate(parents))
        # the target's choice at every node, from logits of the last layer's output: a child that holds the chosen token is accepted, and so on
        T = sum(new)
        head = torch.randn(HQ * D, VOCAB, generator=torch.Generator().manual_seed(step)).cuda()
        logits = (out[-1].reshape(T, -1).float() @ head).to(torch.bfloat16)
        lse, top, top_lp = torch.zeros(T, device="cuda"), zeros(T, 4), torch.zeros(T, 4, device="cuda")
        drafted, lp = dev(np.concatenate(tokens))[:, None].contiguous(), torch.zeros(T, 1, device="cuda")
        B.osc_token_logprobs(logits, drafted, lp, lse=lse, top_ids=top, top_logprobs=top_lp)
        ref = branching.token_logprobs(logits.double().cpu().numpy(), drafted.cpu().numpy(), 1.0, 4)
        # (fp32 next to logits of a few hundred at most: 2^-24 a rounding of |y|, a dozen of them)
        assert np.array_equal(top.cpu().numpy(), ref[3]) and np.abs(lp.cpu().numpy() - ref[0]).max() < 12 * 2.0 ** -24 * (logits.float().abs().max().item() + 10)
        keep, at = [], 0
        for r in range(R):
            path, kids = [], [i for i in range(new[r]) if parents[r][i] == -1]
            while kids:                                  # the child that the (random) target finds most likely, for a few steps
                best = max(kids, key=lambda i: lp[at + i].item())
                if path and rng.random() < 0.2:
                    break
                path.append(best)
                kids = [i for i in range(new[r]) if parents[r][i] == path[-1]]
            # every node's row sees the request's history and its own ancestors
            for i in (0, new[r] - 1, path[-1]):
                line, j = [], parents[r][i]
                while j >= 0:
                    line.append(tokens[r][j])
                    j = parents[r][j]
                s.check(out, at + i, history[r] + line[::-1], tokens[r][i])
            keep.append(path)
            history[r] += [int(tokens[r][i]) for i in path]
            at += new[r]
        cols = max(len(p) for p in keep)
        B.osc_kv_compact(s.layers, s.row, s.kv, s.table, dev([p + [-1] * (cols - len(p)) for p in keep]), dev([len(p) for p in keep]), s.len)
        assert s.len.tolist() == [len(h) for h in history]
        # what lies behind the accepted tokens goes back to the pool
        after = s.len.clone()
        s.len.copy_(s.kv)
        s.give_back(after)
        s.len.copy_(after)
        held = s.table[s.table >= 0].tolist()
        assert sorted(held + [int(p) for p in s.free]) == list(range(s.n_pages)) and len(held) == sum(-(-len(h) // PAGE) for h in history)
    # and single tokens after that
    tokens = rng.integers(0, VOCAB, R)
    out = s.step(tokens, [1] * R)
    for r in range(R):
        s.check(out, r, history[r], int(tokens[r]))


def test_beams_forked_and_reordered(B):
    """Two requests with four beams each, over pages that fill up and are forked."""
    beams, R = 4, 8
    s, rng = Server(B, R, n_pages=200, seed=3), np.random.default_rng(4)
    prompts = [list(rng.integers(0, VOCAB, n)) for n in (30, 15)]
    new = [0] * R
    for q in range(2):
        new[q * beams] = len(prompts[q])
    s.step(sum(prompts, []), new)
    s.len.copy_(s.kv)
    history = [None] * R
    for q in range(2):
        history[q * beams] = list(prompts[q])
    pairs = [(q * beams, q * beams + j) for q in range(2) for j in range(1, beams)]
    for step in range(12):
        # forks, with the pages that are not full copied
        if pairs:
            src, dst = dev([a for a, _ in pairs]), dev([b for _, b in pairs])
            c, taken = [zeros(len(pairs)) for _ in range(3)], zeros(1)
            B.osc_kv_fork(src, dst, s.len, PAGE, dev(s.free), s.table, s.refs, *c, taken)
            B.osc_kv_copy_pages(s.layers, *c)
            s.free = s.free[taken.item():]
            for a, b in pairs:
                history[b] = list(history[a])
        assert s.len.tolist() == [len(h) for h in history]
        tokens = rng.integers(0, VOCAB, R)
        out = s.step(tokens, [1] * R)
        for r in range(R):
            s.check(out, r, history[r], int(tokens[r]))
            history[r].append(int(tokens[r]))
        s.len.copy_(s.kv)
        # no page is held by more rows than it counts, none is held and free at once
        held = s.table[s.table >= 0].cpu().numpy()
        assert np.array_equal(np.bincount(held, minlength=s.n_pages), s.refs.cpu().numpy()) and not set(held.tolist()) & {int(p) for p in s.free}
        # some beams end: their pages go back, their rows are taken by forks of others
        dead = [int(q * beams + j) for q in range(2) for j in rng.permutation(beams)[:rng.integers(0, beams)]]
        to = s.len.clone()
        to[torch.tensor(dead, dtype=torch.long, device="cuda")] = 0
        s.give_back(to)
        live = [[r for r in range(q * beams, (q + 1) * beams) if r not in dead] for q in range(2)]
        pairs = [(int(rng.choice(live[d // beams])), d) for d in dead]
    assert s.refs.sum().item() == sum(-(-len(h) // PAGE) for r, h in enumerate(history) if r not in dead)


def test_calls_at_once_from_several_threads(B):
    """Trees, scores and moves on streams of their own, workspaces of their own."""
    cases = [TreeCase(100 + i, 4, 4, 128, 16, [9 + i, 30], [80, 400 + 50 * i]) for i in range(4)]
    want = [c.reference() for c in cases]
    errors = []

    def work(i):
        try:
            st = torch.cuda.Stream()
            with torch.cuda.stream(st):
                x = torch.randn(7, 5000 + i, device="cuda", generator=torch.Generator(device="cuda").manual_seed(i))
                lse, top, tlp = torch.zeros(7, device="cuda"), zeros(7, 3), torch.zeros(7, 3, device="cuda")
                for _ in range(20):
                    o, l2 = cases[i].run(B, stream=st)
                    B.osc_token_logprobs(x, lse=lse, top_ids=top, top_logprobs=tlp, stream=st)
                st.synchronize()
                n = int(cases[i].rows[-1])
                go = o[:n].double().cpu().numpy().reshape(want[i][0].shape)
                assert (np.abs(go - want[i][0]) <= want[i][2]).all()
                assert torch.allclose(lse, torch.logsumexp(x, 1), atol=1e-4) and torch.equal(top, torch.topk(x, 3, dim=1).indices.int())
        except Exception as e:      # noqa: BLE001
            errors.append((i, repr(e)))
    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    torch.cuda.synchronize()
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
