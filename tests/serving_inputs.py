"""Inputs and tolerances of the tests around the paged key/value cache."""
import numpy as np
import torch

from oracle import serving

BF16_HALF = torch.finfo(torch.bfloat16).eps / 2       # 2^-8: a rounding to bf16, relative to the value


class AttnCase:
    """A step of R requests over a paged cache.  Everything that no row may use holds NaN: the rest of a last page, pages
    no table names, and query rows behind the last request.  Table columns behind a request's pages hold page
    numbers outside the cache."""

    def __init__(self, seed, Hk, G, D, page, new, kv, prefix=(), groups=None, layout="nhd", tail_rows=0, q_mul=2.0, device="cuda"):
        rng = np.random.default_rng(seed)
        self.Hk, self.G, self.D, self.page = Hk, G, D, page
        self.new, self.kv, self.prefix = list(new), list(kv), list(prefix)
        R, P, Hq = len(new), len(self.prefix), Hk * G
        self.groups = list(groups) if groups is not None else ([R * g // P for g in range(P + 1)] if P else [0])
        self.rows = np.concatenate([[0], np.cumsum(self.new)]).astype(int)
        self.T = int(self.rows[-1]) + tail_rows
        g = torch.Generator().manual_seed(seed)
        own_pages = [-(-n // page) for n in self.kv]
        pre_pages = [-(-n // page) for n in self.prefix]
        n_pages = sum(own_pages) + sum(pre_pages) + 2
        order = list(rng.permutation(n_pages))
        shape = (n_pages, page, Hk, D)

        def store():
            nan = float("nan")
            if layout == "nhd":
                return torch.full(shape, nan, dtype=torch.bfloat16, device=device), torch.full(shape, nan, dtype=torch.bfloat16, device=device)
            if layout == "hnd":      # [page][head][token][channel]
                return tuple(torch.full((n_pages, Hk, page, D), nan, dtype=torch.bfloat16, device=device).permute(0, 2, 1, 3) for _ in range(2))
            both = torch.full((n_pages, 2, page, Hk, D + 8), nan, dtype=torch.bfloat16, device=device)   # K and V of a page side by side
            return both[:, 0, :, :, :D], both[:, 1, :, :, :D]
        self.k, self.v = store()

        def place(lens, counts):
            cols = max(counts + [0]) + 1
            tab = np.full((max(len(lens), 1), cols), n_pages + 7, np.int32)
            tab[:, ::2] = -3
            out = []
            for i, (n, c) in enumerate(zip(lens, counts)):
                pages = [int(order.pop()) for _ in range(c)]
                tab[i, :c] = pages
                K, V = (torch.randn(n, Hk, D, generator=g).to(torch.bfloat16) for _ in range(2))
                for j, p in enumerate(pages):
                    m = min(page, n - j * page)
                    self.k[p, :m] = K[j * page:j * page + m].to(device)
                    self.v[p, :m] = V[j * page:j * page + m].to(device)
                out.append((K.double().numpy(), V.double().numpy()))
            return torch.from_numpy(tab).to(device), out
        self.table, self.own = place(self.kv, own_pages)
        self.ptable, self.pre = place(self.prefix, pre_pages)
        q = torch.randn(self.T, Hq * D, generator=g) * q_mul
        q[int(self.rows[-1]):] = float("nan")
        self.q_host = q.to(torch.bfloat16)
        self.q = self.q_host.to(device)
        dev = lambda x: torch.tensor(list(x), dtype=torch.int32, device=device)      # noqa: E731
        self.row_off, self.kv_len = dev(self.rows), dev(self.kv)
        self.group_off, self.prefix_len = (dev(self.groups), dev(self.prefix)) if P else (None, None)
        self.scale = 1.0 / np.sqrt(D)

    def group_of(self, r):
        for g in range(len(self.prefix)):
            if self.groups[g] <= r < self.groups[g + 1]:
                return g
        return -1

    def reference(self):
        """(o, lse, tolerance of o, tolerance of lse) for the rows of all requests.

        Scores: D products of bf16 numbers (exact) summed in fp32, each of the D additions off by at most 2^-23 of the sum of
        magnitudes (a tensor core may truncate), then scaled with three roundings: d = (D + 3) 2^-23 scale sum|q k|, which moves a weight
        by a factor e^(+-d) against its sum's e^(+-d).  Weights are rounded to bf16 (2^-8) in the products, not in the sum; exp2 and the
        joins are off by a few 2^-22 each (2^-18 covers sixteen).  Sums over N keys in fp32: N 2^-23.  Last, o is rounded to bf16."""
        n_rows, Hq = int(self.rows[-1]), self.Hk * self.G
        o, lse = np.zeros((n_rows, Hq, self.D)), np.full((n_rows, Hq), -np.inf)
        to, tl = np.zeros_like(o), np.zeros_like(lse)
        q = self.q_host.double().numpy().reshape(self.T, self.Hk, self.G, self.D)
        for r, (n, kv) in enumerate(zip(self.new, self.kv)):
            a = self.rows[r]
            gi = self.group_of(r)
            K, V = self.own[r]
            shared = self.prefix[gi] if gi >= 0 else 0
            if gi >= 0:
                K, V = np.concatenate([self.pre[gi][0], K]), np.concatenate([self.pre[gi][1], V])
            own_seen = np.maximum(kv - n + np.arange(n) + 1, 0)
            oo, ll, av, sm = serving.attention(q[a:a + n], K, V, shared + own_seen, self.scale)
            N = shared + kv
            d = (self.D + 3) * 2.0 ** -23 * sm.reshape(n, Hq)
            rel = np.expm1(2 * d) + N * 2.0 ** -23 + 2.0 ** -18
            oo, av, ll = oo.reshape(n, Hq, self.D), av.reshape(n, Hq, self.D), ll.reshape(n, Hq)
            o[a:a + n], lse[a:a + n] = oo, ll
            err = (BF16_HALF + rel)[..., None] * av
            to[a:a + n] = err + BF16_HALF * (np.abs(oo) + err) + 1e-38
            with np.errstate(invalid="ignore"):
                tl[a:a + n] = d + rel + 2.0 ** -21 * (np.abs(np.where(np.isinf(ll), 0, ll)) + np.log(max(N, 1)) + 1)
        return o, lse, to, tl

    def run(self, B, max_new=0, pad=0, stream=None, with_lse=True):
        """The library's call on buffers filled with 7; pad widens the rows of Q and O.  Returns (o, lse) tensors."""
        Hq, D, T = self.Hk * self.G, self.D, self.T
        qbig = torch.full((T, Hq * D + pad), float("nan"), dtype=torch.bfloat16, device="cuda")
        qbig[:, :Hq * D] = self.q
        self.obig = torch.full((T, Hq * D + pad), 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((T, Hq), 7.0, dtype=torch.float32, device="cuda") if with_lse else None
        P = len(self.prefix)
        ws = torch.full((B.osc_paged_attention_workspace_bytes(T, Hq, D, len(self.new), P),), 0xFF, dtype=torch.uint8, device="cuda")
        B.osc_paged_attention(qbig[:, :Hq * D], B.KvCache(self.k, self.v), self.row_off, self.kv_len, self.table, self.obig[:, :Hq * D], ws,
                              self.scale, lse=lse, group_off=self.group_off, prefix_len=self.prefix_len,
                              prefix_table=self.ptable if P else None, max_new=max_new, stream=stream)
        return self.obig[:, :Hq * D], lse

    def check(self, o, lse, what=""):
        n_rows, Hq = int(self.rows[-1]), self.Hk * self.G
        ro, rl, to, tl = self.reference()
        go = o[:n_rows].float().cpu().numpy().astype(np.float64).reshape(n_rows, Hq, self.D)
        bad = ~(np.abs(go - ro) <= to)
        assert not bad.any(), (f"{what}: {bad.sum()} of {bad.size} outputs off; rows {np.unique(np.nonzero(bad)[0])[:8]} heads "
                               f"{np.unique(np.nonzero(bad)[1])[:8]}; worst {np.nanmax(np.abs(go - ro) / to)} of the tolerance")
        assert (o[n_rows:].float() == 7.0).all(), f"{what}: rows behind the last request were written"
        if lse is not None:
            gl = lse[:n_rows].cpu().numpy().astype(np.float64)
            empty = np.isinf(rl)
            assert (gl[empty] == -np.inf).all() and np.isfinite(gl[~empty]).all(), f"{what}: lse of empty rows"
            assert (np.abs(gl[~empty] - rl[~empty]) <= tl[~empty]).all(), f"{what}: lse off by {np.abs(gl[~empty] - rl[~empty]).max()}"
            assert (lse[n_rows:] == 7.0).all(), f"{what}: lse behind the last request was written"
