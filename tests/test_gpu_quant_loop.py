"""The 8-bit cache in a decode loop, as it would be used: blocks are assigned, prompts are stored, tokens are appended and
attended to, the cache is loaded for a compression step on per-head ranges, stored again shorter, its blocks are given
back, and decoding goes on; also captured into a graph."""
import math

import numpy as np
import pytest
import torch

from paper_2512_07993_amd import binding as B

from quant_helpers import D, U_OUT, attend_reference, check_close, VALUES

pytestmark = pytest.mark.gpu

L, H, G, BS, BATCH = 2, 2, 4, 16, 3
ROOM, ROOM_SENT = 512, 64
PROMPTS, BUDGET, ALPHA, WINDOW = [200, 333, 97], 96, 8, 32


class Loop:
    def __init__(self, seed):
        dev = "cuda"
        self.gen = torch.Generator(device=dev)
        self.gen.manual_seed(seed)
        blocks = BATCH * ROOM // BS
        z = lambda *s: torch.zeros(s, dtype=torch.int32, device=dev)
        self.pages = B.Pages(z(BATCH, ROOM // BS), z(BATCH), torch.randperm(blocks, generator=self.gen, device=dev).to(torch.int32),
                             torch.tensor([blocks], dtype=torch.int32, device=dev), BS)
        pool = lambda: torch.full((L, blocks, BS, H, D), 0x7F, dtype=torch.uint8, device=dev)
        byte = lambda: torch.zeros((L, H, blocks), dtype=torch.uint8, device=dev)
        self.qc = B.QuantCache(pool(), pool(), byte(), byte(), self.pages.block_table)
        self.len = z(L, H, BATCH)
        self.status = z(1)
        self.page_ws = torch.empty(B.skipkv_pages_workspace_bytes(self.pages) + 256, dtype=torch.uint8, device=dev)
        self.dense = [[[torch.zeros((0, D), dtype=torch.float64, device=dev) for _ in range(BATCH)] for _ in range(H)] for _ in range(2 * L)]

    def randn(self, *shape):
        return torch.randn(shape, generator=self.gen, device="cuda").bfloat16()

    def grow(self, counts):
        off = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
        slots = torch.full((L * H, int(sum(counts))), -7, dtype=torch.int32, device="cuda")
        B.skipkv_pages_update(self.pages, self.len, off, int(sum(counts)), slots, self.page_ws, self.status)
        return off, slots

    def store(self, counts):
        """One call per layer, as a model's layers come by."""
        off, slots = self.grow(counts)
        n = int(sum(counts))
        for l in range(L):
            k, v = self.randn(1, H, n, D), self.randn(1, H, n, D) * 2
            rows = B.Cache(k, v, H * G, off, None, None, n, 0)
            B.skipkv_quant_store(self.qc, rows, l, self.len[l:l + 1], None, self.status)
        self.len += (off[1:] - off[:-1])[None, None, :]
        return slots

    def values(self, l, h, b):
        """What the cache holds, decoded on the host side of things."""
        n = int(self.len[l, h, b])
        t = torch.arange(n, device="cuda")
        p = self.pages.block_table[b, t // BS].long()
        table = torch.from_numpy(VALUES).cuda()
        return [(table[x[l, p, t % BS, h].long()] * torch.exp2(e[l, h, p].double() - 127)[:, None]).cpu().numpy()
                for x, e in ((self.qc.k, self.qc.k_exp), (self.qc.v, self.qc.v_exp))]

    def attend(self, l, ms):
        q = self.randn(sum(ms), H * G, D)
        out, lse = torch.empty_like(q), torch.empty((sum(ms), H * G), device="cuda")
        off = torch.tensor(np.concatenate([[0], np.cumsum(ms)]), dtype=torch.int32, device="cuda")
        qs = B.Queries(q, out, off, max_q=max(ms), max_len=ROOM, scale=1 / math.sqrt(D), lse=lse)
        ws = torch.empty(B.skipkv_quant_attend_workspace_bytes(self.qc, qs) + 256, dtype=torch.uint8, device="cuda")
        B.skipkv_quant_attend(self.qc, l, qs, self.len[l], ws, self.status)
        return q, out

    def check_attend(self, ms):
        for l in range(L):
            q, out = self.attend(l, ms)
            at = 0
            for b, m in enumerate(ms):
                for h in range(H):
                    k, v = self.values(l, h, b)
                    ref, _, tol, _ = attend_reference(q[at:at + m, h * G:(h + 1) * G].double().cpu().numpy(), k, v, m, 1 / math.sqrt(D), 2.0 ** -8)
                    check_close(out[at:at + m, h * G:(h + 1) * G].double().cpu().numpy(), ref, tol + U_OUT[torch.bfloat16] * (np.abs(ref) + tol),
                                "layer %d head %d sequence %d" % (l, h, b))
                at += m


def test_decode_loop_with_a_compression_step():
    s = Loop(1)
    slots = s.store(PROMPTS)
    assert int((slots < 0).sum()) == 0
    s.check_attend([200, 60, 97])
    for _ in range(20):
        slots = s.store([1, 1, 1])
    # the slot map names the slots that hold the last tokens: theirs are the values that the load returns there
    for l in range(L):
        for h in range(H):
            for b in range(BATCH):
                slot = int(slots[l * H + h, b])
                n = int(s.len[l, h, b])
                assert slot // BS == int(s.pages.block_table[b, (n - 1) // BS]) and slot % BS == (n - 1) % BS
    s.check_attend([1, 1, 1])
    # ---- the step: the cache in bf16, packed by room; sentences of ten tokens
    seq_off = torch.tensor([0, ROOM, 2 * ROOM, 3 * ROOM], dtype=torch.int32, device="cuda")
    sent_ptr = torch.tensor([b * (ROOM_SENT + 1) for b in range(BATCH + 1)], dtype=torch.int32, device="cuda")
    T, S = BATCH * ROOM, BATCH * ROOM_SENT
    k, v = (torch.zeros((L, H, T, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache = B.Cache(k, v, H * G, seq_off, sent_ptr, sent_ptr, T, S)
    B.skipkv_quant_load(s.qc, cache, 0, None, s.len, s.status)
    for b in range(BATCH):
        kk, vv = s.values(1, 1, b)
        n = len(kk)
        np.testing.assert_array_equal(k[1, 1, b * ROOM:b * ROOM + n].double().cpu().numpy(), kk)
        np.testing.assert_array_equal(v[1, 1, b * ROOM:b * ROOM + n].double().cpu().numpy(), vv)
    cnt = torch.zeros((L, H, BATCH), dtype=torch.int32, device="cuda")
    offs = torch.zeros((L, H, S + BATCH), dtype=torch.int32, device="cuda")
    for b in range(BATCH):
        n = int(s.len[0, 0, b])
        cut = list(range(0, n, 10)) + [n]
        cnt[:, :, b] = len(cut) - 1
        offs[:, :, b * (ROOM_SENT + 1):b * (ROOM_SENT + 1) + len(cut)] = torch.tensor(cut, dtype=torch.int32, device="cuda")
    params = B.Params(ALPHA, WINDOW, BUDGET, dev_status=s.status)
    ws = torch.empty(B.skipkv_ranges_workspace_bytes(cache, params) + 256, dtype=torch.uint8, device="cuda")
    f = lambda *sh: torch.zeros(sh, dtype=torch.float32, device="cuda")
    i = lambda *sh: torch.zeros(sh, dtype=torch.int32, device="cuda")
    new_len, new_off, new_cnt, kept = i(L, H, BATCH), i(L, H, S + BATCH), i(L, H, BATCH), i(L, H, BATCH, BUDGET)
    before = [[[s.values(l, h, b) for b in range(BATCH)] for h in range(H)] for l in range(L)]
    B.skipkv_step_ranges(cache, B.Ranges(s.len, cnt, offs), params, s.randn(L, BATCH, H * G, ALPHA, D), None, f(L, H, S), f(L, H, S), None, None,
                         kept, new_len, new_off, new_cnt, BUDGET, ws)
    assert bool((new_len <= BUDGET).all()) and int(s.status.item()) == 0
    held = s.pages.n_held.clone()
    s.len = new_len.clone()
    B.skipkv_quant_store(s.qc, cache, 0, None, s.len, s.status)
    s.grow([0, 0, 0])                                                  # the blocks beyond the new lengths are given back
    need = (s.len.amax((0, 1)) + BS - 1) // BS
    assert torch.equal(s.pages.n_held, need) and bool((need < held).all())
    assert int(s.pages.n_free.item()) + int(need.sum()) == BATCH * ROOM // BS
    for l in range(L):
        for h in range(H):
            for b in range(BATCH):
                idx = kept[l, h, b, :int(s.len[l, h, b])].cpu().numpy()
                for got, was in zip(s.values(l, h, b), before[l][h][b]):
                    # a kept row is the same row but where it falls among a larger scale's subnormals: 2^-10 of a scale of at
                    # most 16 (values below 7168)
                    assert np.abs(got - was[idx]).max() <= 16 * 2.0 ** -10
    # ---- decoding goes on
    for _ in range(5):
        s.store([1, 1, 1])
    s.check_attend([1, 1, 1])
    s.store([0, 30, 2])
    s.check_attend([1, 30, 2])
    assert int(s.status.item()) == 0


def test_a_decode_step_captured_into_a_graph():
    # tables, stores and attention of one token each, replayed with eager work in between; every replay equals an eager twin
    a, b = Loop(2), Loop(2)
    for s in (a, b):
        s.store(PROMPTS)
    n = BATCH
    off = torch.arange(BATCH + 1, dtype=torch.int32, device="cuda")

    def buffers(s):
        x = dict(k=s.randn(L, H, n, D), v=s.randn(L, H, n, D), q=s.randn(n, H * G, D))
        x["out"] = [torch.zeros_like(x["q"]) for _ in range(L)]
        x["slots"] = torch.zeros((L * H, n), dtype=torch.int32, device="cuda")
        qs = B.Queries(x["q"], x["out"][0], off, max_q=1, max_len=ROOM, scale=0.09)
        x["ws"] = torch.empty(B.skipkv_quant_attend_workspace_bytes(s.qc, qs) + 256, dtype=torch.uint8, device="cuda")
        return x

    def step(s, x):
        B.skipkv_pages_update(s.pages, s.len, off, n, x["slots"], s.page_ws, s.status)
        rows = B.Cache(x["k"], x["v"], H * G, off, None, None, n, 0)
        B.skipkv_quant_store(s.qc, rows, 0, s.len, None, s.status)
        s.len += 1
        for l in range(L):
            qs = B.Queries(x["q"], x["out"][l], off, max_q=1, max_len=ROOM, scale=0.09)
            B.skipkv_quant_attend(s.qc, l, qs, s.len[l], x["ws"], s.status)

    xa, xb = buffers(a), buffers(b)
    keep = a.len.clone(), [t.clone() for t in (a.pages.block_table, a.pages.n_held, a.pages.free_list, a.pages.n_free, a.qc.k, a.qc.v, a.qc.k_exp, a.qc.v_exp)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(a, xa)                                                    # once before the capture
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    a.len.copy_(keep[0])
    for t, was in zip((a.pages.block_table, a.pages.n_held, a.pages.free_list, a.pages.n_free, a.qc.k, a.qc.v, a.qc.k_exp, a.qc.v_exp), keep[1]):
        t.copy_(was)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, xa)
    for i in range(40):
        for x in ("k", "v", "q"):
            fresh = a.randn(*xa[x].shape) * (1 + i % 5)
            xa[x].copy_(fresh)
            xb[x].copy_(fresh)
        graph.replay()
        step(b, xb)
        for l in range(L):
            assert torch.equal(xa["out"][l], xb["out"][l]), (i, l)
        assert torch.equal(xa["slots"], xb["slots"]) and torch.equal(a.pages.n_held, b.pages.n_held) and torch.equal(a.len, b.len)
        assert torch.equal(a.pages.block_table, b.pages.block_table)
        if i % 7 == 0:
            torch.cuda.synchronize()
    assert torch.equal(a.qc.k, b.qc.k) and torch.equal(a.qc.v_exp, b.qc.v_exp) and int(a.status.item()) == int(b.status.item()) == 0
    assert int(a.len[0, 0, 0]) == PROMPTS[0] + 40
