"""The operators of a decode step together, the way a serving loop uses them: prompts in chunks, then steps of one token per
sequence captured in a CUDA graph (tables, then per layer norm + rotation + cache write and attention), sequences that end
and others that take their pages."""
import numpy as np
import pytest
import torch

from paper_2606_29986_b200 import hma
from records import Paged, records, write
from test_gpu_append import assert_rows, norm_rope_oracle
from test_gpu_step import step_oracle

HQ, HKV, B, MAX_PAGES, PAGES, LAYERS, N = 6, 2, 5, 14, 40, 2, 160
WINDOW, SINKS = 20, 3                                     # of the second layer; the first one sees everything


class Loop:
    def __init__(self, fmt, seed=0):
        self.desc = hma.make_desc(LAYERS, HQ, HKV, PAGES, fmt)
        self.cache = hma.KVCache(self.desc, fill=0xEE)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.table, self.ctx = torch.full((B, MAX_PAGES), -1, **i32), torch.zeros(B, **i32)
        self.free, self.count = torch.randperm(PAGES, generator=torch.Generator().manual_seed(seed)).int().cuda(), torch.tensor([PAGES], **i32)
        self.new, self.starts = torch.zeros(B, **i32), torch.zeros(B + 1, **i32)
        self.pos, self.slots = torch.zeros(N, **i32), torch.zeros(N, dtype=torch.int64, device="cuda")
        self.rope = hma.hma_rope_table(1e4 ** (-np.arange(32) / 32), MAX_PAGES * 16)
        g = torch.Generator().manual_seed(seed + 1)
        self.w = [[torch.randn(128, generator=g).bfloat16().cuda() for _ in (0, 1)] for _ in range(LAYERS)]
        self.qkv = torch.zeros((LAYERS, N, (HQ + 2 * HKV) * 128), dtype=torch.bfloat16, device="cuda")
        self.q, self.k = torch.zeros((LAYERS, N, HQ, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((LAYERS, N, HKV, 128), dtype=torch.bfloat16, device="cuda")
        self.out = torch.zeros((LAYERS, B, HQ, 128), device="cuda")
        self.ws = hma.new_workspace(self.desc, B)
        # the same in numpy
        self.np_table, self.np_free, self.np_count, self.np_ctx = np.full((B, MAX_PAGES), -1, np.int32), self.free.cpu().numpy(), PAGES, np.zeros(B, np.int64)
        self.layers = [np.full(hma.hma_cache_layer_bytes(self.desc), 0xEE, np.uint8) for _ in range(LAYERS)]
        self.scale = 1 / np.sqrt(128.0)

    def launch(self, attend):
        hma.hma_step_tables(self.cache, self.ctx, self.new, self.table, self.free, self.count, self.ctx, self.starts, self.pos, self.slots)
        for l in range(LAYERS):
            hma.hma_qk_norm_rope(self.cache, l, self.qkv[l], *self.w[l], 1e-5, self.rope, self.pos, self.q[l], k_out=self.k[l], slots=self.slots)
            if attend and l == 0:
                hma.hma_decode_attention(self.cache, l, self.q[l][:B], self.out[l], self.table, self.ctx, self.scale, self.ws)
            elif attend:
                hma.hma_decode_attention_window(self.cache, l, self.q[l][:B], self.out[l], self.table, self.ctx, WINDOW, SINKS, self.scale, self.ws)

    def step(self, new, seed, attend, run):
        x = torch.randn(self.qkv.shape, generator=torch.Generator().manual_seed(seed)).bfloat16()
        self.qkv.copy_(x)
        self.new.copy_(torch.tensor(new, dtype=torch.int32))
        run()
        torch.cuda.synchronize()
        want, flag = step_oracle(self.np_ctx, new, self.np_table, self.np_free, self.np_count, N, PAGES)
        assert flag == 0 and hma.hma_error_flags(self.cache) == 0
        self.np_table, self.np_count, self.np_ctx = want["table"], want["left"], want["context"]
        assert np.array_equal(self.table.cpu().numpy(), want["table"]) and np.array_equal(self.slots.cpu().numpy(), want["slots"])
        x = x.float().numpy().reshape(LAYERS, N, HQ + 2 * HKV, 128)
        for l in range(LAYERS):
            ws = [w.float().cpu().numpy() for w in self.w[l]]
            assert_rows(self.q[l].double().cpu().numpy(), *norm_rope_oracle(x[l][:, :HQ], ws[0], 1e-5, self.rope.cpu().numpy(), want["positions"], False))
            assert_rows(self.k[l].double().cpu().numpy(), *norm_rope_oracle(x[l][:, HQ:HQ + HKV], ws[1], 1e-5, self.rope.cpu().numpy(), want["positions"], False))
            assert write(self.layers[l], self.desc, want["slots"], self.k[l].float().cpu().numpy(), x[l][:, HQ + HKV:]) == 0
            assert np.array_equal(self.cache.layers[l].cpu().numpy(), self.layers[l])
            if attend:
                p = Paged.__new__(Paged)               # its reference, over this loop's cache
                p.lens, p.hq, p.hkv, p.fmt, p.desc, p.table, p.clean, p.scale, p.q = self.np_ctx, HQ, HKV, self.desc.format, self.desc, self.np_table, self.layers, self.scale, self.q[l][:B]
                ref, tol = p.reference(layer=l, window=WINDOW if l else None, sinks=SINKS if l else 0)
                assert (np.abs(self.out[l].double().cpu().numpy() - ref[:, 0]) <= tol[:, 0]).all()

    def release(self, done):
        hma.hma_release_pages(self.cache, torch.tensor(done, dtype=torch.int32, device="cuda"), self.ctx, self.table, self.free, self.count)
        assert hma.hma_error_flags(self.cache) == 0
        for b in range(B):
            if done[b]:
                n = (int(self.np_ctx[b]) + 15) // 16
                self.np_free[self.np_count:self.np_count + n] = self.np_table[b, :n]
                self.np_count += n
                self.np_table[b, :n] = -1
                self.np_ctx[b] = 0
        assert int(self.count) == self.np_count and np.array_equal(self.free[:self.np_count].cpu().numpy(), self.np_free[:self.np_count])


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", [hma.HMA_KV_BFP8, hma.HMA_KV_BFP4, hma.HMA_KV_BF16])
def test_serving_loop(fmt):
    lp = Loop(fmt)
    lp.step([50, 16, 0, 33, 7], 1, False, lambda: lp.launch(False))              # prompts, in two chunks where they are long
    lp.step([30, 0, 95, 0, 1], 2, False, lambda: lp.launch(False))
    lp.step([1] * B, 3, True, lambda: lp.launch(True))                             # (also the first calls on this device)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        lp.launch(True)
    for i in range(18):                                                           # across page ends of every sequence
        lp.step([1] * B, 10 + i, True, g.replay)
    lp.release([0, 1, 0, 0, 1])
    lp.step([0, 40, 0, 0, 64], 50, False, lambda: lp.launch(False))              # their places and pages go to new requests
    for i in range(3):
        lp.step([1] * B, 60 + i, True, g.replay)


@pytest.mark.gpu
def test_tensors_of_another_device_are_refused(monkeypatch):
    """Every tensor has to be on the current device (here the binding is told that another one is current, so nothing is launched)."""
    cache, i32 = hma.KVCache(hma.make_desc(1, 8, 8, 4)), dict(dtype=torch.int32, device="cuda")
    z = lambda *s: torch.zeros(s, **i32)
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
    slots, ws = torch.full((1,), -1, dtype=torch.int64, device="cuda"), hma.new_workspace(cache.desc, 1)
    calls = [lambda: hma.hma_step_tables(cache, z(1), z(1), z(1, 2), z(4), z(1), z(1), z(2), z(1), slots),
             lambda: hma.hma_release_pages(cache, z(1), z(1), z(1, 2), z(4), z(1)),
             lambda: hma.hma_rope_table([1.0] * 8, 4),
             lambda: hma.hma_kv_append(cache, 0, bf(1, 8, 128), bf(1, 8, 128), slots),
             lambda: hma.hma_qk_norm_rope(cache, 0, bf(1, 24 * 128), None, None, 1e-6, None, None, bf(1, 8, 128), slots=slots),
             lambda: hma.hma_decode_attention_window(cache, 0, bf(1, 8, 128), bf(1, 8, 128), z(1, 2), z(1), 4, 0, 1.0, ws)]
    for call in calls:
        call()
    torch.cuda.synchronize()
    assert hma.hma_error_flags(cache) == 0
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    for call in calls:
        with pytest.raises(hma.HmaError):
            call()
