"""GPU test of a layer's steps over pages as a program runs them: norms and rotation of the projections' rows, keys and values
written, a prompt taken in chunks over the pages, then decode steps, with a sliding window and without; captured decode
steps replay.  Each step is compared with 64 bits on what it was given."""
import math

import numpy as np
import pytest
import torch

import kv_ref as R
import window_ref as W
from test_gpu_rotate import EPS, check, dev, frequencies, reference as rotated

pytestmark = pytest.mark.gpu
H, G, C = 2, 3, 16


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g
    g.build()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


class Layer:
    """Pages, and beside them, in 64 bits, the keys and values that went into them."""

    def __init__(self, D, requests, room, dtype, window, sinks):
        from paper_2609_38706_gb300 import service
        self.D, self.window, self.sinks, self.dtype = D, window, sinks, dtype
        stride = -(-room // C)
        self.kv = service.KVPages(requests * stride + 2, C, H, D)
        g = torch.Generator(device="cuda").manual_seed(3)
        self.pages = torch.randperm(requests * stride, generator=g, device="cuda").to(torch.int32).view(requests, stride)
        self.rotary = service.Rotary(D, D // 2, factor=4.0, context=64, amplitude=1.0 + 0.1 * math.log(4.0))
        self.w = [(1 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(dtype) for _ in (0, 1)]
        self.held = [[np.zeros((0, H, D))] * 2 for _ in range(requests)]
        self.len = torch.zeros(requests, dtype=torch.int32, device="cuda")
        self.g = g

    def rows(self, n):
        return torch.randn((n, H * G + 2 * H, self.D), generator=self.g, device="cuda").to(self.dtype)

    def step(self, new, decode=False):
        """`new` tokens a request through the layer, each stage compared with 64 bits."""
        name = {torch.bfloat16: "bf16", torch.float16: "fp16"}[self.dtype]
        qkv = self.rows(sum(new))
        q, k, v = qkv[:, : H * G], qkv[:, H * G: H * G + H], qkv[:, H * G + H:]
        before = [x.double().cpu().numpy() for x in (q, k)]
        off = dev(np.concatenate(([0], np.cumsum(new))).astype(np.int64))
        start = self.len.clone()
        self.kv.rotate(q, k, off, start, self.rotary, *self.w, eps=EPS, out=(q, k))
        at = np.concatenate([np.arange(s, s + n, dtype=np.float64) for s, n in zip(start.tolist(), new)])
        f = frequencies(self.D // 2, factor=4.0, context=64.0)
        for x, y, w in zip(before, (q, k), self.w):
            check(y, *rotated(x, w.double().cpu().numpy(), at, f, False, 1.0 + 0.1 * math.log(4.0), name))
        self.kv.write(k, v, off, start, self.pages)
        self.len += dev(np.array(new, np.int32))
        limits = dict(window=self.window, sinks=self.sinks)
        if decode:
            out, lse = self.kv.attend(q.view(len(new), new[0], H * G, self.D), self.len, self.pages, **limits)
            out, lse = out.flatten(0, 1), lse.flatten(0, 1)
        else:
            out, lse = self.kv.attend_chunk(q, off, self.len, self.pages, **limits)
        self.kv.check()
        a = 0
        for r, n in enumerate(new):
            rows = slice(a, a + n)
            if n == 0:
                continue
            paged = [R.dequantise(*R.quantise(x[rows].float().cpu().numpy(), 1.0), 1.0) for x in (k, v)]
            self.held[r] = [np.concatenate(p) for p in zip(self.held[r], paged)]
            kk, vv = self.held[r]
            m = len(kk)
            ok = W.seen(m - n, n, m, self.window, self.sinks)
            for h in range(H * G):
                x = q[rows, h].double().cpu().numpy()
                o, l, _, mag = W.attend(x, kk[:, h // G], vv[:, h // G], ok, self.D ** -0.5)
                err = R.score_error(x, kk[:, h // G], self.D ** -0.5)
                assert np.all(np.abs(out[rows, h].double().cpu().numpy() - o) <= R.out_bound(o, mag, R.U["fp16"], R.U[name], err, m))
                assert np.all(np.abs(lse[rows, h].double().cpu().numpy() - l) <= R.lse_bound(l, err, m))
            a += n


@pytest.mark.parametrize("window,sinks", [(None, 0), (90, 3)])
@pytest.mark.parametrize("D,dtype", [(64, torch.float16), (128, torch.bfloat16)])
def test_chunks_then_decode(D, dtype, window, sinks):
    layer = Layer(D, 3, 400, dtype, window, sinks)
    for new in ([100, 7, 33], [130, 0, 1], [20, 150, 64]):
        layer.step(new)
    for _ in range(2):
        layer.step([1, 1, 1], decode=True)
    layer.step([3, 3, 3], decode=True)
    layer.step([5, 1, 9])


def test_captured_step():
    """A decode step of four calls, replayed with other rows and growing lengths."""
    layer = Layer(128, 2, 300, torch.bfloat16, 50, 2)
    layer.step([40, 90])
    qkv = layer.rows(2)
    q, k, v = qkv[:, : H * G], qkv[:, H * G: H * G + H], qkv[:, H * G + H:]
    off, weight = dev(np.arange(3)), torch.zeros(layer.pages.shape, device="cuda")

    def step():
        qr, kr = layer.kv.rotate(q, k, off, layer.len, layer.rotary, *layer.w)
        layer.kv.write(kr, v, off, layer.len, layer.pages)
        layer.len.add_(1)
        return layer.kv.attend(qr.unsqueeze(1), layer.len, layer.pages, weight=weight, window=50, sinks=2)

    saved = layer.len.clone(), layer.kv.pool.clone()
    step()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, lse = step()
    want = []
    inputs = [layer.rows(2) for _ in range(3)]
    for captured in (False, True):
        layer.len.copy_(saved[0]), layer.kv.pool.copy_(saved[1]), weight.zero_()
        for i, x in enumerate(inputs):
            qkv.copy_(x)
            if captured:
                g.replay()
                assert torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1]) and torch.equal(weight, want[i][2])
            else:
                o, l = step()
                want.append((o.clone(), l.clone(), weight.clone()))
    layer.kv.check()


def test_the_readmes_lines_run():
    import os
    import re
    from paper_2609_38706_gb300.service import KVPages
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    block = next(b for b in re.findall(r"```python\n(.*?)```", text, re.S) if "kv.rotate(" in b)
    x = lambda n, h: torch.randn((n, h, 128), device="cuda").to(torch.bfloat16)  # noqa: E731
    off, w = dev(np.array([0, 40, 60])), torch.ones(128, dtype=torch.bfloat16, device="cuda")
    env = dict(kv=KVPages(8, 16, 2, 128), q=x(60, 4), k=x(60, 2), v=x(60, 2), tok_off=off, q_off=off, q_weight=w, k_weight=w,
               start=dev(np.zeros(2, np.int32)), pages=dev(np.arange(6, dtype=np.int32).reshape(2, 3)),
               kv_len=dev(np.array([40, 20], np.int32)))
    for line in block.strip().split("\n"):
        if "kv.attend(" in line:
            env["q"] = env["q"][:2].unsqueeze(1)
        exec(line, env)
    assert env["out"].shape == (2, 1, 4, 128) and bool(env["out"].isfinite().all())
