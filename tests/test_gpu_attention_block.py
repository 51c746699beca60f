"""The attention block as a server runs it: RMSNorm with the QKV projection, slots, norm and rotation into the cache,
attention over the cache, o_proj.  A prefix and ragged prompts first, then decoding steps from one captured graph whose
lengths, pages and slots move on on the device.  Every stage is compared with its definition on what the stage
before it left on the device, and the cache at the end with everything that was written."""
import numpy as np
import pytest
import torch

from oracle import serving
from paper_2604_12782_b200 import synth
from serving_inputs import BF16_HALF, AttnCase

pytestmark = pytest.mark.gpu

from gpu_util import assert_within_tolerance, dev_bf16, host_bf16_bits, host_f64  # noqa: E402

HIDDEN, HQ, HK, D, PAGE, EPS = 512, 4, 2, 64, 16, 1e-6
WIDTH = (HQ + 2 * HK) * D


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2604_12782_b200 import binding
    return binding


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Block:
    def __init__(self, B, n_pages):
        rng = np.random.default_rng(0)
        qkv, o = synth.osc_linear_case(1, 1, HIDDEN, WIDTH, 1), synth.osc_linear_case(2, 1, HQ * D, HIDDEN, 1)
        self.B, self.qkv, self.o = B, qkv, o
        self.w_qkv, self.w_o = (B.osc_prepare_weights(dev_bf16(c["W"]), c["lut"]) for c in (qkv, o))
        self.gamma = synth.f32_to_bf16_bits(rng.uniform(0.5, 1.5, HIDDEN).astype(np.float32))
        self.gq, self.gk = (synth.f32_to_bf16_bits(rng.uniform(0.5, 1.5, D).astype(np.float32)) for _ in range(2))
        self.inv = (1e-4 ** (np.arange(D // 2) / (D // 2))).astype(np.float32)
        self.rope = B.Rope(torch.from_numpy(self.inv).cuda())
        nan = float("nan")
        self.k, self.v = (torch.full((n_pages, PAGE, HK, D), nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.cache = B.KvCache(self.k, self.v)
        self.dg, self.dgq, self.dgk = dev_bf16(self.gamma), dev_bf16(self.gq), dev_bf16(self.gk)
        self.free = i32(np.random.default_rng(3).permutation(n_pages))

    def buffers(self, T, R, P):
        B, bf16 = self.B, dict(dtype=torch.bfloat16, device="cuda")
        a, b = B.osc_act_sizes(self.w_qkv, T), B.osc_act_sizes(self.w_o, T)
        return dict(x=torch.zeros(T, HIDDEN, **bf16), qkv=torch.zeros(T, WIDTH, **bf16), q=torch.zeros(T, HQ * D, **bf16),
                    o=torch.zeros(T, HQ * D, **bf16), y=torch.zeros(T, HIDDEN, **bf16), lse=torch.zeros(T, HQ, device="cuda"),
                    row_off=i32([0] * (R + 1)), kv_len=i32([0] * R), slots=i32([0] * T), pos=i32([0] * T), taken=i32([0]),
                    ws=torch.empty(max(a.workspace_bytes, b.workspace_bytes), dtype=torch.uint8, device="cuda"),
                    wa=torch.empty(B.osc_paged_attention_workspace_bytes(T, HQ, D, R, P), dtype=torch.uint8, device="cuda"))

    def step(self, b, cached, fresh, base, table, group_off=None, prefix_len=None, prefix_table=None, max_new=0):
        B = self.B
        B.osc_kv_slots(cached, fresh, base, PAGE, self.free, table, b["row_off"], b["kv_len"], b["slots"], b["pos"], b["taken"])
        B.osc_rmsnorm_linear(self.w_qkv, b["x"], self.dg, EPS, b["qkv"], b["ws"])
        B.osc_qk_norm_rope(b["qkv"], HQ, self.cache, b["q"], b["pos"], self.rope, gamma_q=self.dgq, gamma_k=self.dgk, eps=EPS, slots=b["slots"])
        B.osc_paged_attention(b["q"], self.cache, b["row_off"], b["kv_len"], table, b["o"], b["wa"], D ** -0.5, lse=b["lse"], group_off=group_off,
                              prefix_len=prefix_len, prefix_table=prefix_table, max_new=max_new)
        B.osc_linear(self.w_o, b["o"], b["y"], b["ws"])
        # the next step: the lengths grow, the free list moves on by what was taken
        cached += fresh
        at = torch.arange(self.free.numel(), device="cuda") + b["taken"]
        self.free.copy_(self.free[at.clamp_max(self.free.numel() - 1)])

    def check(self, oracle, b, new, kv, prefix, table, ptable, base, what):
        """new, kv: of this step; the cache must hold all kv keys by now."""
        n = sum(new)
        ref, T, _, _ = oracle.linear(oracle.rmsnorm(host_bf16_bits(b["x"][:n]), self.gamma, EPS), self.qkv["W"], self.qkv["lut"])
        assert_within_tolerance(host_f64(b["qkv"][:n]), ref, T, f"{what}: QKV")
        pos = np.concatenate([np.arange(k - m, k) + s for m, k, s in zip(new, kv, base)]).astype(int)
        assert np.array_equal(b["pos"][:n].cpu().numpy(), pos)
        x = host_f64(b["qkv"][:n]).reshape(n, HQ + 2 * HK, D)

        def turned(heads, gamma, got, name):
            r, size = serving.qk_norm_rope(heads, synth.bf16_bits_to_f64(gamma), EPS, self.inv, None, pos[None], False)
            tol = BF16_HALF * np.abs(r) + (1 + BF16_HALF) * 2.0 ** -19 * size + 1e-38       # as in the call's own tests
            assert (np.abs(got - r) <= tol).all(), f"{what}: {name}"
        turned(x[:, :HQ], self.gq, host_f64(b["q"][:n]).reshape(n, HQ, D), "Q")
        kc, vc = host_f64(self.k), host_f64(self.v)

        def gather(row, m):
            pages = [int(p) for p in row[:-(-m // PAGE)]]
            return tuple(np.concatenate([c[p] for p in pages])[:m] if pages else np.zeros((0, HK, D)) for c in (kc, vc))
        tab = table.cpu().numpy()
        own = [gather(tab[r], m) for r, m in enumerate(kv)]
        fresh_k = np.concatenate([K[m - f:m] for (K, _), m, f in zip(own, kv, new)])
        fresh_v = np.concatenate([V[m - f:m] for (_, V), m, f in zip(own, kv, new)])
        turned(x[:, HQ:HQ + HK], self.gk, fresh_k, "K")
        assert np.array_equal(fresh_v, x[:, HQ + HK:]), f"{what}: V"
        c = object.__new__(AttnCase)
        c.Hk, c.G, c.D, c.new, c.kv, c.prefix, c.T, c.scale = HK, HQ // HK, D, new, kv, prefix, n, D ** -0.5
        c.groups, c.rows, c.q_host, c.own = [0, len(new)], np.concatenate([[0], np.cumsum(new)]).astype(int), b["q"][:n].cpu(), own
        c.pre = [gather(ptable.cpu().numpy()[0], prefix[0])] if prefix else []
        c.check(b["o"][:n], b["lse"][:n], f"{what}: attention")
        ref, T, _, _ = oracle.linear(host_bf16_bits(b["o"][:n]), self.o["W"], self.o["lut"])
        assert_within_tolerance(host_f64(b["y"][:n]), ref, T, f"{what}: o_proj")


def test_prefix_prompts_and_captured_decoding(B, oracle):
    L = Block(B, 40)
    g = torch.Generator().manual_seed(5)

    def tokens(b, n):
        b["x"].zero_()
        b["x"][:n] = torch.randn(n, HIDDEN, generator=g).to(torch.bfloat16).cuda()
    # the prefix, as a request of its own: its pages become the group's
    S = 40
    pre, pre_table, pre_cached = L.buffers(S, 1, 0), i32(np.full((1, 4), -1)), i32([0])
    tokens(pre, S)
    L.step(pre, pre_cached, i32([S]), None, pre_table)
    B.osc_sync_check()
    L.check(oracle, pre, [S], [S], [], pre_table, None, [0], "prefix")
    # ragged prompts behind it, one of them empty
    new = [20, 5, 70, 1, 0]
    R = len(new)
    table, cached, base, groups = i32(np.full((R, 6), -1)), i32([0] * R), i32([S] * R), i32([0, R])
    prompts = L.buffers(sum(new), R, 1)
    tokens(prompts, sum(new))
    L.step(prompts, cached, i32(new), base, table, groups, pre_cached, pre_table)
    B.osc_sync_check()
    L.check(oracle, prompts, new, new, [S], table, pre_table, [S] * R, "prompts")
    # decoding from one captured graph, rows for three more tokens than there are
    d, fresh = L.buffers(R + 3, R, 1), i32([1] * R)
    st, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=st):
        L.step(d, cached, fresh, base, table, groups, pre_cached, pre_table, max_new=1)
    d["o"].zero_()
    kv = list(new)
    for i in range(18):                                  # far enough that every request takes a new page
        tokens(d, R)
        graph.replay()
        kv = [m + 1 for m in kv]
        B.osc_sync_check()
        assert cached.tolist() == kv and d["slots"].tolist()[R:] == [-1] * 3
        if i in (0, 10, 17):
            L.check(oracle, d, [1] * R, kv, [S], table, pre_table, [S] * R, f"decoding step {i}")
            assert (d["o"][R:] == 0).all()
    used = -(-S // PAGE) + sum(-(-m // PAGE) for m in kv)
    held = torch.cat([pre_table[0, :3]] + [table[r, :-(-m // PAGE)] for r, m in enumerate(kv)]).tolist()
    assert len(held) == used and len(set(held)) == used and min(held) >= 0, "a page was handed out twice"
    # slots that no token took hold what they held before
    taken = torch.zeros(L.k.shape[0], PAGE, dtype=torch.bool)
    for pages, n in [(pre_table[0].tolist(), S)] + [(table[r].tolist(), m) for r, m in enumerate(kv)]:
        for j in range(n):
            taken[pages[j // PAGE], j % PAGE] = True
    for c in (L.k, L.v):
        nan = torch.isnan(c.float()).cpu()
        assert nan[~taken].all() and not nan[taken].any()


def test_a_prompt_in_pieces_is_the_prompt(B, oracle):
    """The same tokens at once, in pieces of odd sizes, and one by one: each run agrees with the definition on its own
    cache, and the values in the caches are the same within the projection's bound."""
    n, caches = 61, []
    g = torch.Generator().manual_seed(6)
    x = torch.randn(n, HIDDEN, generator=g).to(torch.bfloat16).cuda()
    for pieces in ([n], [17, 1, 30, 13], [1] * n):
        L = Block(B, 6)
        table, cached, at = i32(np.full((1, 4), -1)), i32([0]), 0
        for m in pieces:
            b = L.buffers(m, 1, 0)
            b["x"].copy_(x[at:at + m])
            L.step(b, cached, i32([m]), None, table)
            at += m
            B.osc_sync_check()
            if m > 1 or at % 20 == 0:
                L.check(oracle, b, [m], [at], [], table, None, [0], f"pieces {len(pieces)}, to {at}")
        caches.append(L.v[table[0].long()].view(-1, HK, D)[:n].clone())
    for v in caches[1:]:
        # the projection may sum in another order for another number of rows; the bound of its own test, doubled for two runs
        ref, T, _, _ = oracle.linear(oracle.rmsnorm(host_bf16_bits(x), L.gamma, EPS), L.qkv["W"], L.qkv["lut"])
        bound = 2 * (2.0 ** -7 * np.abs(ref) + 1e-3 * T).reshape(n, -1, D)[:, HQ + HK:]
        assert (np.abs(host_f64(v) - host_f64(caches[0])) <= bound).all()
