"""GPU test of the serving example's numbers end to end against 64 bits: keys, pages written and hit, prefix read back, prompt
attention, decode steps over the pages.  A page table in another order, or of other pages, does not pass."""
import os
import sys

import numpy as np
import pytest
import torch

import kv_ref as R

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g
    g.build()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def paged(x):
    """bfloat16 rows as 64-bit values, behind the 4-bit page."""
    x = x.float().cpu().numpy()
    return R.dequantise(*R.quantise(x, 1.0), 1.0) if x.size else x.astype(np.float64)


def plain(x):
    return x.double().cpu().numpy()


def expected(q, k, v, last, wo, scale, u_p):
    """Logits of a query [heads, D] over k, v [n, kv_heads, D], and a bound on what the kernels and the projection may be off."""
    H, G = k.shape[1], q.shape[0] // k.shape[1]
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    for h in range(q.shape[0]):
        kk, vv = k[: last + 1, h // G], v[: last + 1, h // G]
        o, _, _, mag = R.attend(q[None, h], kk, vv, np.array([last]), scale)
        err = R.score_error(q[None, h], kk, scale)
        out[h], tol[h] = o[0], R.out_bound(o, mag, u_p, R.U["bf16"], err, last + 1)[0]
    o, t, w = out.reshape(-1), tol.reshape(-1), np.abs(wo)
    logits = o @ wo
    # the projection: the outputs' error through it, 32-bit sums of products of 16-bit values, its own rounding
    bound = t @ w + (len(o) + 8) * 2.0 ** -23 * (np.abs(o) @ w)
    return logits, bound * (1 + R.U["bf16"]) + R.U["bf16"] * np.abs(logits) + 2.0 ** -20


class Recorder:
    """A layer whose projections are kept."""

    def __init__(self, layer):
        self.layer, self.calls = layer, []

    def project(self, tokens):
        q, k, v = self.layer.project(tokens)
        self.calls.append((q, k, v))
        return q, k, v

    def logits(self, attended):
        return self.layer.logits(attended)


@pytest.mark.parametrize("n,extra", [(140, 0), (100, 30), (128, 0), (37, 5)])
def test_answers_from_hits_and_decode_steps(n, extra):
    import serve_from_pages as ex
    C, D, scale = ex.CHUNK, ex.D, ex.D ** -0.5
    rng = np.random.default_rng(n)
    layer = Recorder(ex.Layer(2))
    server = ex.Server(layer, 64)
    wo = plain(layer.layer.wo)
    prompt = rng.integers(0, ex.VOCAB, n).tolist()

    # cold: every key is the projection's own
    logits, _, _, hit = server.prefill([prompt], room=8)
    q, k, v = layer.calls[-1]
    assert hit == [0] and k.shape[0] == n
    cold_k, cold_v = k, v
    want, bound = expected(plain(q[-1]), plain(k), plain(v), n - 1, wo, scale, R.U["bf16"])
    assert np.all(np.abs(plain(logits[0]) - want) <= bound)

    # the same prompt, longer by `extra`, served from what the first one left
    tail = rng.integers(0, ex.VOCAB, extra).tolist()
    logits, table, kv_len, hit = server.prefill([prompt + tail], room=8)
    chunks = n // C
    assert hit == [chunks]
    q, k, v = layer.calls[-1]
    total, start = n + extra, min(chunks * C, n + extra - 1)
    assert k.shape[0] == total - start
    old_k, old_v = paged(cold_k[: chunks * C]), paged(cold_v[: chunks * C])  # what the pages hold
    read = [torch.from_numpy(x[:start]).to(torch.bfloat16).double().numpy() for x in (old_k, old_v)]  # rounded by the read
    want, bound = expected(plain(q[-1]), np.concatenate((read[0], plain(k))), np.concatenate((read[1], plain(v))), total - 1, wo,
                           scale, R.U["bf16"])
    assert np.all(np.abs(plain(logits[0]) - want) <= bound)

    # decode steps over pages alone
    fresh = slice(chunks * C - start, None)  # a prompt that is hit whole keeps its last token's page
    all_k, all_v = (np.concatenate((a, paged(b[fresh]))) for a, b in ((old_k, k), (old_v, v)))
    weight = torch.zeros(table.shape, dtype=torch.float32, device="cuda")
    for step in range(3):
        token = logits.argmax(-1).to(torch.int32)
        logits, kv_len = server.decode(token, table, kv_len, weight)
        q, k, v = layer.calls[-1]
        all_k, all_v = np.concatenate((all_k, paged(k))), np.concatenate((all_v, paged(v)))
        want, bound = expected(plain(q[0]), all_k, all_v, total + step, wo, scale, R.U["fp16"])
        assert np.all(np.abs(plain(logits[0]) - want) <= bound)
    server.kv.check()

    # other pages, or the same ones in another order: the bound notices
    q = layer.calls[-1][0]
    for other in (table.roll(1, 1), table.clone()):
        if torch.equal(other, table):
            other[0, 0] = server.free[0]
        out, _ = server.kv.attend(q.unsqueeze(1), kv_len, other.clamp(min=0))
        assert not np.all(np.abs(plain(layer.logits(out)[0]) - want) <= bound)
    server.kt.close()
