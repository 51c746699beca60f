"""A step of a beam search captured once and replayed: pages given back, rows forked, pages copied, new tokens placed, with the pool of free pages and the
counts of the pages that osc_kv_slots takes (which it does not keep) on the device, by the caller."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

L, HK, D, PAGE = 2, 2, 64, 16


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2604_12782_b200 import binding
    return binding


def zeros(*shape):
    return torch.zeros(*shape, dtype=torch.int32, device="cuda")


class Beams:
    """R rows of a table; a pool of n_pages + 1 places: the free pages in order, then -1."""

    def __init__(self, B, R, n_pages, cols):
        self.B, self.R, self.n_pages = B, R, n_pages
        self.k, self.v = (torch.full((L, n_pages, PAGE, HK, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.layers = B.KvLayers([B.KvCache(a, b) for a, b in zip(self.k, self.v)])
        self.table, self.len, self.to = torch.full((R, cols), -1, dtype=torch.int32, device="cuda"), zeros(R), zeros(R)
        self.refs = zeros(n_pages + 1)                 # (the last one takes what counts for nothing)
        self.pool = torch.cat([torch.randperm(n_pages, generator=torch.Generator().manual_seed(1)).int().cuda(), torch.full((1,), -1, dtype=torch.int32, device="cuda")])
        self.n_pool = torch.full((1,), n_pages, dtype=torch.int64, device="cuda")
        self.at = torch.arange(n_pages + 1, device="cuda")
        self.freed, self.n_freed, self.taken = zeros(n_pages), zeros(1), zeros(1)
        self.copies = [zeros(R) for _ in range(3)]
        # what a step is given: which rows go on, the forks (-1: none), a token for every row
        self.alive, self.src, self.dst, self.token = torch.ones(R, dtype=torch.int32, device="cuda"), zeros(R) - 1, zeros(R) - 1, torch.zeros(R, dtype=torch.bfloat16, device="cuda")
        self.fresh, self.row, self.kv, self.slots, self.pos = torch.ones(R, dtype=torch.int32, device="cuda"), zeros(R + 1), zeros(R), zeros(R), zeros(R)

    def drop(self, taken):
        """The pool without its first `taken` pages."""
        self.pool.copy_(self.pool[torch.clamp(self.at + taken, max=self.n_pages)])
        self.n_pool -= taken

    def step(self):
        B = self.B
        torch.mul(self.len, self.alive, out=self.to)
        B.osc_kv_trim(self.len, self.to, PAGE, self.table, self.refs, self.freed, self.n_freed, n_pages=self.n_pages)
        self.len.copy_(self.to)
        place = torch.where(self.at[:-1] < self.n_freed, self.n_pool + self.at[:-1], self.n_pages)
        self.pool.scatter_(0, place, self.freed)
        self.pool[-1:] = -1
        self.n_pool += self.n_freed
        B.osc_kv_fork(self.src, self.dst, self.len, PAGE, self.pool, self.table, self.refs, *self.copies, self.taken, n_pages=self.n_pages)
        B.osc_kv_copy_pages(self.layers, *self.copies)
        self.drop(self.taken)
        B.osc_kv_slots(self.len, self.fresh, None, PAGE, self.pool, self.table, self.row, self.kv, self.slots, self.pos, self.taken)
        # osc_kv_slots keeps no counts: its pages have one holder each from here on
        self.refs.index_add_(0, torch.where(self.at < self.taken, self.pool, self.n_pages), torch.ones_like(self.pool))
        self.drop(self.taken)
        for x in (self.k, self.v):
            x.view(L, -1, HK * D)[:, self.slots.long()] = self.token[None, :, None].expand(L, self.R, HK * D)
        self.len.copy_(self.kv)


@pytest.mark.parametrize("seed", [0, 1])
def test_a_captured_step_of_a_beam_search(B, seed):
    R, rng = 8, np.random.default_rng(seed)
    s = Beams(B, R, 200, 12)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    history = [[] for _ in range(R)]

    def give(alive, pairs, tokens):
        s.alive.copy_(torch.tensor(alive, dtype=torch.int32))
        p = np.full((2, R), -1)
        for i, (a, b) in enumerate(pairs):
            p[:, i] = a, b
        s.src.copy_(torch.from_numpy(p[0]))
        s.dst.copy_(torch.from_numpy(p[1]))
        s.token.copy_(torch.tensor(tokens, dtype=torch.float32))

    def check():
        table, refs, n = s.table.cpu().numpy(), s.refs.cpu().numpy(), int(s.n_pool.item())
        held = table[table >= 0]
        assert np.array_equal(np.bincount(held, minlength=s.n_pages), refs[:s.n_pages]), "counts"
        pool = s.pool.cpu().numpy()
        assert (pool[n:] == -1).all() and sorted(set(held.tolist()) | set(pool[:n].tolist())) == list(range(s.n_pages)) and len(set(held.tolist())) + n == s.n_pages, "pool"
        k = s.k.float().cpu().numpy()
        for r in range(R):
            assert s.len[r].item() == len(history[r])
            for layer in range(L):
                got = [k[layer, table[r, i // PAGE], i % PAGE] for i in range(len(history[r]))]
                assert all((x == t).all() for x, t in zip(got, history[r])), (r, layer)
        assert torch.equal(s.k[:, s.table[0, 0].long()].view(torch.int16), s.v[:, s.table[0, 0].long()].view(torch.int16))

    with torch.cuda.stream(st):
        tokens = rng.integers(1, 200, R)
        give([1] * R, [], tokens)
        s.step()                                    # also warms up what the capture needs
        for r in range(R):
            history[r].append(int(tokens[r]))
    st.synchronize()
    check()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        s.step()
    for _ in range(70):
        dead = sorted(int(x) for x in rng.permutation(R)[:rng.integers(0, R - 1)])
        live = [r for r in range(R) if r not in dead]
        pairs = [(int(rng.choice(live)), d) for d in dead]
        tokens = rng.integers(1, 200, R)
        with torch.cuda.stream(st):
            give([0 if r in dead else 1 for r in range(R)], pairs, tokens)
            g.replay()
        st.synchronize()
        for a, b in pairs:
            history[b] = list(history[a])
        for r in range(R):
            history[r].append(int(tokens[r]))
        check()
