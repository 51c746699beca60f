"""Inputs and tolerances of the tests for requests with more than one continuation."""
import numpy as np
import torch

from oracle import branching
from serving_inputs import BF16_HALF, AttnCase


def random_parents(rng, n):
    """Parents of a drafted tree's tokens: chains, branches and several roots."""
    p = np.empty(n, np.int64)
    for i in range(n):
        x = rng.random()
        p[i] = i - 1 if i == 0 or x < 0.4 else -1 if x < 0.5 else rng.integers(max(0, i - 10), i)
    return p


class TreeCase(AttnCase):
    """A step of R requests whose new tokens see one another by a mask: trees, or any bits (style "any"), or none at all ("none")."""

    def __init__(self, seed, Hk, G, D, page, new, kv, words=None, style="tree", ld_pad=0, **kw):
        super().__init__(seed, Hk, G, D, page, new, kv, **kw)
        rng = np.random.default_rng(seed + 1)
        self.words = words or max(1, -(-max(self.new) // 32))
        self.bits = np.zeros((self.T, 32 * self.words), bool)
        n_rows = int(self.rows[-1])
        if style == "tree":
            par = np.concatenate([random_parents(rng, n) for n in self.new] + [np.full(self.T - n_rows, -1)])
            self.bits[:], _ = branching.tree_mask(par, self.rows, None, self.words)
        elif style == "any":
            self.bits[:] = rng.random(self.bits.shape) < 0.3
        self.bits[n_rows:] = True
        big = np.full((self.T, self.words + ld_pad), -1, np.int32)
        big[:, :self.words] = branching.packed(self.bits)
        self.mask = torch.from_numpy(big).to(self.q.device)[:, :self.words]

    def sees(self, r):
        """bool [n][shared + kv]"""
        n, kv, g = self.new[r], self.kv[r], self.group_of(r)
        shared = self.prefix[g] if g >= 0 else 0
        out = np.zeros((n, shared + kv), bool)
        out[:, :max(shared + kv - n, shared if kv < n else 0)] = True
        if kv < n:
            out[:, :shared] = True
        for m in range(min(n, 32 * self.words)):
            at = kv - n + m
            if at >= 0:
                out[:, shared + at] = self.bits[self.rows[r]:self.rows[r] + n, m]
        for m in range(32 * self.words, n):
            if kv - n + m >= 0:
                out[:, shared + kv - n + m] = False
        return out

    def reference(self):
        """As AttnCase's, with every row's own set of keys: N, smax and the sums are over the keys that it sees."""
        n_rows, Hq = int(self.rows[-1]), self.Hk * self.G
        o, lse = np.zeros((n_rows, Hq, self.D)), np.full((n_rows, Hq), -np.inf)
        to, tl = np.zeros_like(o), np.zeros_like(lse)
        q = self.q_host.double().numpy().reshape(self.T, self.Hk, self.G, self.D)
        for r, n in enumerate(self.new):
            a, g = self.rows[r], self.group_of(r)
            K, V = self.own[r]
            if g >= 0:
                K, V = np.concatenate([self.pre[g][0], K]), np.concatenate([self.pre[g][1], V])
            oo, ll, av, sm = branching.attention(q[a:a + n], K, V, self.sees(r), self.scale)
            d = (self.D + 3) * 2.0 ** -23 * sm.reshape(n, Hq)
            rel = np.expm1(2 * d) + len(K) * 2.0 ** -23 + 2.0 ** -18
            oo, av, ll = oo.reshape(n, Hq, self.D), av.reshape(n, Hq, self.D), ll.reshape(n, Hq)
            o[a:a + n], lse[a:a + n] = oo, ll
            err = (BF16_HALF + rel)[..., None] * av
            to[a:a + n] = err + BF16_HALF * (np.abs(oo) + err) + 1e-38
            tl[a:a + n] = d + rel + 2.0 ** -21 * (np.abs(np.where(np.isinf(ll), 0, ll)) + np.log(max(len(K), 1)) + 1)
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
        B.osc_tree_attention(qbig[:, :Hq * D], B.KvCache(self.k, self.v), self.row_off, self.kv_len, self.table, self.mask, self.obig[:, :Hq * D], ws,
                             self.scale, lse=lse, group_off=self.group_off, prefix_len=self.prefix_len,
                             prefix_table=self.ptable if P else None, max_new=max_new, stream=stream)
        return self.obig[:, :Hq * D], lse

    def spoil(self, r, m, channels, value):
        """Values of new token m of request r, in the given channels of every head: `value`, in the cache and in the definition."""
        at = self.kv[r] - self.new[r] + m
        assert at >= 0
        page = int(self.table[r, at // self.page])
        self.v[page, at % self.page][:, channels] = value
        self.own[r][1][at][:, channels] = float(value)

    def check_odd(self, o, lse, what=""):
        """As check, where values may be Inf or NaN: those reach the rows that see them, in their channels, and no others."""
        n_rows, Hq = int(self.rows[-1]), self.Hk * self.G
        with np.errstate(invalid="ignore"):
            ro, rl, to, tl = self.reference()
        go = o[:n_rows].float().cpu().numpy().astype(np.float64).reshape(n_rows, Hq, self.D)
        gl = lse[:n_rows].cpu().numpy().astype(np.float64)
        assert np.array_equal(np.isnan(ro), np.isnan(go)), f"{what}: NaN where there should be none, or none where there should be"
        inf = np.isinf(ro)
        assert np.array_equal(inf, np.isinf(go)) and (ro[inf] == go[inf]).all(), f"{what}: Inf"
        fine = np.isfinite(ro)
        assert (np.abs(go[fine] - ro[fine]) <= to[fine]).all(), f"{what}: outputs off"
        seen = np.isfinite(rl)
        assert (gl[~seen] == -np.inf).all() and (np.abs(gl[seen] - rl[seen]) <= tl[seen]).all(), f"{what}: lse"
