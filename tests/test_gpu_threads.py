"""Host threads: distinct handles on distinct streams, called from several threads at once.

ctypes releases the interpreter lock for the duration of a foreign call, so the calls below do run inside the
library at the same time (validation, kernel selection, tensor-map encoding, launches).  Every thread must get,
bit for bit, what the same call gives when it runs alone.
"""
import threading

import numpy as np
import pytest
import torch

from paper_2604_12782_b200 import synth

pytestmark = pytest.mark.gpu

from gpu_util import assert_within_tolerance, dev_bf16, host_bf16_bits, host_f64, poison  # noqa: E402


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2604_12782_b200 import binding
    return binding


SHAPES = [(16, 512, 256, "osc"), (200, 1024, 320, "osc"), (700, 512, 512, "fp8"), (1300, 768, 448, "osc"),
          (64, 2048, 128, "mxfp8"), (3000, 256, 192, "fp8")]


def make_job(B, seed, M, K, N, kind):
    if kind == "osc":
        c = synth.osc_linear_case(seed, M, K, N, 2)
        w = B.osc_prepare_weights(dev_bf16(c["W"]), c["lut"])
        ws = poison(B.osc_act_sizes(w, M).workspace_bytes)
        call = B.osc_linear
    elif kind == "fp8":
        c = synth.fp8_linear_case(seed, M, K, N)
        w = B.osc_fp8_prepare_weights(dev_bf16(c["W"]))
        ws = poison(B.osc_fp8_act_sizes(w, M).workspace_bytes)
        call = B.osc_fp8_linear
    else:
        c = synth.fp8_linear_case(seed, M, K, N)
        w = B.osc_mxfp8_prepare_weights(dev_bf16(c["W"]))
        ws = poison(B.osc_mxfp8_act_sizes(w, M).workspace_bytes)
        call = B.osc_mxfp8_linear
    return {"c": c, "w": w, "ws": ws, "call": call, "X": dev_bf16(c["X"]), "kind": kind, "M": M, "N": N}


def test_concurrent_calls_from_host_threads(B, oracle):
    jobs = [make_job(B, 40 + i, *s) for i, s in enumerate(SHAPES)]
    alone = []
    for j in jobs:                       # each call on its own, default stream
        Y = torch.full((j["M"], j["N"]), float("nan"), dtype=torch.bfloat16, device="cuda")
        j["call"](j["w"], j["X"], Y, j["ws"])
        B.osc_sync_check()
        alone.append(host_bf16_bits(Y))
    # the first one also against the oracle, so that "alone" is not only compared with itself
    c = jobs[0]["c"]
    Yref, T, *_ = oracle.linear(c["X"], c["W"], c["lut"])
    assert_within_tolerance(host_f64(dev_bf16(alone[0])), Yref, T, "single call")

    torch.cuda.synchronize()
    rounds = 25
    errors, outs = [], [None] * len(jobs)
    start = threading.Barrier(len(jobs))

    def worker(i):
        try:
            j = jobs[i]
            st = torch.cuda.Stream()
            Ys = [torch.full((j["M"], j["N"]), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(rounds)]
            torch.cuda.synchronize()
            start.wait()
            with torch.cuda.stream(st):
                for Y in Ys:
                    j["call"](j["w"], j["X"], Y, j["ws"], stream=st)
            st.synchronize()
            outs[i] = [host_bf16_bits(Y) for Y in Ys]
        except Exception as e:           # reported by the main thread
            errors.append((i, repr(e)))

    threads = [threading.Thread(target=worker, args=(i,)) for i in range(len(jobs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    B.osc_sync_check()
    for i, ys in enumerate(outs):
        for r, y in enumerate(ys):
            assert np.array_equal(y, alone[i]), f"job {i} ({SHAPES[i]}), round {r}: differs from the call made alone"


class CacheStep:
    """One step over a paged cache: slots of its tokens, norm and rotation into the cache, attention; everything its own."""

    def __init__(self, B, seed, new, old, Hq, Hk, D, page, prefix, max_new):
        g = torch.Generator().manual_seed(seed)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")      # noqa: E731
        R, T = len(new), sum(new)
        own, pre = [-(-(o + n) // page) for o, n in zip(old, new)], -(-prefix // page)
        n_pages, cols = sum(own) + pre, max(own)
        pages = torch.randperm(n_pages, generator=g).tolist()
        self.k, self.v = (torch.randn(n_pages, page, Hk, D, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
        self.cache, self.rope = B.KvCache(self.k, self.v), B.Rope((1e-4 ** (torch.arange(D // 2) / (D // 2))).cuda())
        self.prefix, self.ptable = i32([prefix]), i32([[pages.pop() for _ in range(pre)]])
        table = torch.full((R, cols), -1, dtype=torch.int32)
        for r, o in enumerate(old):
            for j in range(-(-o // page)):
                table[r, j] = pages.pop()
        self.table, self.free = table.cuda(), i32(pages)
        self.old, self.new, self.base, self.groups = i32(old), i32(new), i32([prefix] * R), i32([0, R])
        self.qkv = torch.randn(T, (Hq + 2 * Hk) * D, generator=g).to(torch.bfloat16).cuda()
        self.gamma = torch.ones(D, dtype=torch.bfloat16, device="cuda")
        self.Hq, self.D, self.page, self.max_new, self.B = Hq, D, page, max_new, B
        self.ints = [torch.zeros(n, dtype=torch.int32, device="cuda") for n in (R + 1, R, T, T, 1)]
        self.q = torch.zeros(T, Hq * D, dtype=torch.bfloat16, device="cuda")
        self.ws = torch.empty(B.osc_paged_attention_workspace_bytes(T, Hq, D, R, 1), dtype=torch.uint8, device="cuda")

    def outputs(self):
        T = self.q.shape[0]
        return torch.full((T, self.Hq * self.D), float("nan"), dtype=torch.bfloat16, device="cuda"), torch.full((T, self.Hq), float("nan"), device="cuda")

    def __call__(self, o, lse, stream=None):
        B, (row_off, kv_len, slots, pos, taken) = self.B, self.ints
        B.osc_kv_slots(self.old, self.new, self.base, self.page, self.free, self.table, row_off, kv_len, slots, pos, taken, stream=stream)
        B.osc_qk_norm_rope(self.qkv, self.Hq, self.cache, self.q, pos, self.rope, gamma_q=self.gamma, gamma_k=self.gamma, slots=slots, stream=stream)
        B.osc_paged_attention(self.q, self.cache, row_off, kv_len, self.table, o, self.ws, self.D ** -0.5, lse=lse, group_off=self.groups,
                              prefix_len=self.prefix, prefix_table=self.ptable, max_new=self.max_new, stream=stream)


STEPS = [([1] * 6, [300, 5, 90, 64, 0, 33], 8, 2, 128, 16, 150, 1), ([40, 1, 70], [0, 500, 20], 8, 2, 64, 32, 70, 0),
         ([200], [100], 4, 4, 128, 64, 1000, 0), ([1], [700], 32, 8, 128, 16, 1, 1), ([5] * 20, [60] * 20, 12, 3, 64, 16, 333, 0)]


def test_cache_steps_from_host_threads(B):
    steps, alone = [CacheStep(B, 70 + i, *s) for i, s in enumerate(STEPS)], []
    for s in steps:
        o, lse = s.outputs()
        s(o, lse)
        B.osc_sync_check()
        assert not torch.isnan(o.float()).any() and not torch.isnan(lse).any()
        alone.append([t.clone() for t in (o, lse, s.q, s.k, s.v, s.table, *s.ints)])
    torch.cuda.synchronize()
    rounds, errors, outs = 20, [], [None] * len(steps)
    start = threading.Barrier(len(steps))

    def worker(i):
        try:
            s, st = steps[i], torch.cuda.Stream()
            bufs = [s.outputs() for _ in range(rounds)]
            torch.cuda.synchronize()
            start.wait()
            with torch.cuda.stream(st):
                for o, lse in bufs:
                    s(o, lse, stream=st)
            st.synchronize()
            outs[i] = bufs
        except Exception as e:           # reported by the main thread
            errors.append((i, repr(e)))

    threads = [threading.Thread(target=worker, args=(i,)) for i in range(len(steps))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    B.osc_sync_check()
    for i, (s, want) in enumerate(zip(steps, alone)):
        for r, (o, lse) in enumerate(outs[i]):
            assert torch.equal(o, want[0]) and torch.equal(lse, want[1]), f"step {i}, round {r}: differs from the step made alone"
        assert all(torch.equal(a, b) for a, b in zip((s.q, s.k, s.v, s.table, *s.ints), want[2:])), f"step {i}"


def test_cache_steps_allocate_nothing(B):
    """The first call of every kernel may load it; after that the device's free memory stays where it is."""
    steps = [CacheStep(B, 80 + i, *s) for i, s in enumerate(STEPS)]
    bufs = [s.outputs() for s in steps]
    for s, b in zip(steps, bufs):
        s(*b)
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    for _ in range(10):
        for s, b in zip(steps, bufs):
            s(*b)
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == free
