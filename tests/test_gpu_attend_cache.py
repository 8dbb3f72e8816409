"""GPU tests of attention over the 4-bit page cache against a plain 64-bit implementation, with the pages' accumulated
weights."""
import numpy as np
import pytest
import torch

import kv_ref as R

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g
    g.build()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def random_pool(slots, C, H, D, rng):
    """Quantised gaussians in every page."""
    pool = np.zeros((slots, H, C // 16, 16 * (D + D // 8)), np.uint8)
    for j in (0, 1):
        code, s = R.quantise(rng.standard_normal((slots, H, C // 16, 16, D)).astype(np.float32), 1.0)
        pool[..., 8 * D * j: 8 * D * (j + 1)] = (code[..., 0::2] | (code[..., 1::2] << 4)).reshape(*code.shape[:3], -1)
        pool[..., 16 * D + D * j: 16 * D + D * (j + 1)] = s.reshape(*s.shape[:3], -1)
    return pool.reshape(slots, -1)


def make(lens, C, H, D, seed, stride=None, spare=1):
    rng = np.random.default_rng(seed)
    stride = stride or max(1, max(-(-n // C) for n in lens))
    slots = len(lens) * stride + spare
    pages = rng.permutation(slots)[: len(lens) * stride].reshape(len(lens), stride).astype(np.int32)
    return random_pool(slots, C, H, D, rng), pages, rng


def cache(pool, C, H, D, k_scale=1.0, v_scale=1.0):
    from paper_2609_38706_gb300.service import KVPages
    return KVPages(pool.shape[0], C, H, D, k_scale, v_scale, pool=dev(pool))


def reference(pool, pages, lens, q, C, H, D, scale, k_scale=1.0, v_scale=1.0):
    """out, lse, per-page weights, mag and the scores' error bound."""
    n_q, G = q.shape[1], q.shape[2] // H
    out, mag = np.zeros(q.shape), np.zeros(q.shape)
    lse, weight, err = np.zeros(q.shape[:3]), np.zeros(pages.shape), 0.0
    for r, n in enumerate(lens):
        if n:
            k, v = R.get_tokens(pool, pages[r, : -(-n // C)], n, C, H, D)
            k, v = k * float(np.float32(k_scale)), v * float(np.float32(v_scale))
        else:
            k = v = np.zeros((0, H, D))
        for h in range(H * G):
            last = n - n_q + np.arange(n_q)
            o, l, p, m = R.attend(q[r, :, h], k[:, h // G], v[:, h // G], last, scale)
            out[r, :, h], lse[r, :, h], mag[r, :, h] = o, l, m
            if n:
                err = max(err, R.score_error(q[r, :, h], k[:, h // G], scale))
                full = np.zeros(-(-n // C) * C)
                full[:n] = p.sum(0)
                weight[r, : -(-n // C)] += full.reshape(-1, C).sum(1)
    return out, lse, weight, mag, err


CASES = [
    # lens, n_q, C, H, G, D, dtype, k_scale, v_scale
    ([1], 1, 16, 1, 1, 64, "bf16", 1.0, 1.0),
    ([0, 1, 15, 16, 17], 1, 16, 2, 4, 128, "bf16", 1.0, 1.0),
    ([300, 47, 48, 49], 1, 48, 2, 3, 64, "fp16", 0.0173, 0.25),
    ([1000, 129], 2, 256, 1, 8, 128, "fp16", 1.0, 1.0),
    ([5, 3, 70], 4, 32, 2, 3, 64, "bf16", 1.0, 1.0),       # 12 rows; queries before position 0
    ([2500, 700], 1, 16, 1, 16, 128, "bf16", 1.0, 2.0),    # two column tiles, several splits
    ([333], 5, 16, 1, 7, 128, "fp16", 1.0, 1.0),           # 35 rows: row tiles
    ([4100], 1, 64, 3, 5, 64, "fp16", 1.0, 1.0),
    ([20000], 1, 256, 1, 2, 128, "bf16", 1.0, 1.0),
]


@pytest.mark.parametrize("weigh", [False, True])
@pytest.mark.parametrize("lens,n_q,C,H,G,D,dtype,k_scale,v_scale", CASES)
def test_matches_reference(lens, n_q, C, H, G, D, dtype, k_scale, v_scale, weigh):
    pool, pages, rng = make(lens, C, H, D, 21)
    kv = cache(pool, C, H, D, k_scale, v_scale)
    q = torch.from_numpy(rng.standard_normal((len(lens), n_q, H * G, D)) * (2 / k_scale)).to(DT[dtype])
    scale = D ** -0.5
    w0 = rng.uniform(0, 2, pages.shape).astype(np.float32)
    weight = dev(w0) if weigh else None
    out, lse = kv.attend(q.cuda(), dev(np.array(lens, np.int32)), dev(pages), scale, weight)
    kv.check()
    ref, rl, rw, mag, err = reference(pool, pages, lens, q.double().numpy(), C, H, D, scale, k_scale, v_scale)
    n = max(lens)
    # the weights are rounded to halves for the product with V, whatever the type of q
    assert np.all(np.abs(out.double().cpu().numpy() - ref) <= R.out_bound(ref, mag, R.U["fp16"], R.U[dtype], err, n))
    gl = lse.double().cpu().numpy()
    none = np.isneginf(rl)
    assert np.array_equal(none, np.isneginf(gl))
    assert np.all(np.abs(gl[~none] - rl[~none]) <= R.lse_bound(rl, err, n)[~none])
    if weigh:
        got = weight.double().cpu().numpy()
        used = np.arange(pages.shape[1]) < np.array([-(-x // C) for x in lens])[:, None]
        assert np.array_equal(got[~used], w0.astype(np.float64)[~used])
        bound = (2 * np.expm1(err) + (n + 128) * 2.0 ** -24) * rw + 2.0 ** -23 * (w0 + rw)
        assert np.all(np.abs(got - w0 - rw) <= bound + 1e-9)


@pytest.mark.parametrize("weigh", [False, True])
def test_more_requests_than_places_longest_first(weigh):
    """Long and short requests, equal and empty ones, in more blocks than the GPU holds: each gets its own answer."""
    rng = np.random.default_rng(31)
    lens = [int(x) for x in rng.integers(1, 200, 90)]
    lens[3], lens[17], lens[40], lens[41], lens[89] = 1100, 0, 1039, 1040, 700
    lens[50:60] = [64] * 10
    C, H, G, D = 16, 8, 2, 64
    pages = np.zeros((90, 69), np.int32)
    slots = 0
    for r, n in enumerate(lens):
        k = -(-n // C)
        pages[r, :k] = slots + np.arange(k)
        slots += k
    pool = random_pool(slots, C, H, D, rng)
    kv = cache(pool, C, H, D)
    q = torch.from_numpy(rng.standard_normal((90, 1, H * G, D))).to(torch.bfloat16)
    weight = torch.zeros(pages.shape, dtype=torch.float32, device="cuda") if weigh else None
    out, lse = kv.attend(q.cuda(), dev(np.array(lens, np.int32)), dev(pages), 0.125, weight)
    kv.check()
    ref, rl, rw, mag, err = reference(pool, pages, lens, q.double().numpy(), C, H, D, 0.125)
    assert np.all(np.abs(out.double().cpu().numpy() - ref) <= R.out_bound(ref, mag, R.U["fp16"], R.U["bf16"], err, 1100))
    gl, none = lse.double().cpu().numpy(), np.isneginf(rl)
    assert np.array_equal(none, np.isneginf(gl))
    assert np.all(np.abs(gl[~none] - rl[~none]) <= R.lse_bound(rl, err, 1100)[~none])
    if weigh:
        got = weight.double().cpu().numpy()
        assert np.all(np.abs(got - rw) <= (2 * np.expm1(err) + 1300 * 2.0 ** -24) * rw + 2.0 ** -23 * rw + 1e-9)


def test_wide_range_of_scores_moves_the_reference():
    """Scores that grow by hundreds along the tokens, and queries far outside a half's range."""
    lens, C, H, G, D = [900], 16, 1, 4, 128
    pool, pages, rng = make(lens, C, H, D, 22)
    kv = cache(pool, C, H, D)
    for amp in (1e-30, 3e4, 1e20):
        q = torch.from_numpy(rng.standard_normal((1, 1, 4, D)) * amp).to(torch.bfloat16)
        scale = 8.0 / amp
        out, lse = kv.attend(q.cuda(), dev(np.array(lens, np.int32)), dev(pages), scale)
        ref, rl, _, mag, err = reference(pool, pages, lens, q.double().numpy(), C, H, D, float(np.float32(scale)))
        assert np.all(np.abs(out.double().cpu().numpy() - ref) <= R.out_bound(ref, mag, R.U["fp16"], R.U["bf16"], err, 900))
        assert np.all(np.abs(lse.double().cpu().numpy() - rl) <= R.lse_bound(rl, err, 900))
    kv.check()


@pytest.mark.parametrize("D,G,n_q", [(64, 3, 1), (128, 8, 2)])
def test_scores_beyond_a_weights_exponents(D, G, n_q):
    """Scores 2^24 and more apart: keys and queries with one nonzero value of few bits each, so that 32 bits hold the
    scores exactly: the heaviest keys, several alike, share the weight."""
    C, H, lens = 16, 2, [700, 33]
    rng = np.random.default_rng(5)
    n_pages = [-(-n // C) for n in lens]
    pages = np.arange(2 * max(n_pages), dtype=np.int32).reshape(2, -1)
    pool = random_pool(pages.size, C, H, D, rng).reshape(pages.size, H, -1)
    pool[..., : 8 * D] = 0
    pool[..., 0: 8 * D: D // 2] = rng.choice((2, 4, 7, 10, 15), pool[..., 0: 8 * D: D // 2].shape)  # 1, 2, 6, -1, -6
    pool[..., 16 * D: 17 * D] = 0x38  # 1.0
    pool = pool.reshape(pages.size, -1)
    kv = cache(pool, C, H, D)
    q = np.zeros((2, n_q, H * G, D), np.float32)
    q[..., 0] = 2.0 ** rng.choice((3, 20, 30, 45, 90), q.shape[:3])
    scale = 0.37
    qt = torch.from_numpy(q).to(torch.bfloat16)
    weight = torch.zeros(pages.shape, dtype=torch.float32, device="cuda")
    out, lse = kv.attend(qt.cuda(), dev(np.array(lens, np.int32)), dev(pages), scale, weight)
    kv.check()
    got_w = weight.double().cpu().numpy()
    for r, n in enumerate(lens):
        k, v = R.get_tokens(pool, pages[r, : n_pages[r]], n, C, H, D)
        total = 0.0
        for h in range(H * G):
            for i in range(n_q):
                m = n - n_q + i + 1
                s = float(q[r, i, h, 0]) * k[:m, h // G, 0]
                w = np.exp(scale * (s - s.max()))
                ref = w @ v[:m, h // G] / w.sum()
                err = (np.minimum(scale * (s.max() - s), 40.0) * 2.0 ** -21).max()
                rel = 2 * np.expm1(err) + 2.0 ** -8 + m * 2.0 ** -24
                got = out[r, i, h].double().cpu().numpy()
                assert np.all(np.abs(got - ref) <= rel * (np.abs(v[:m, h // G]).max() + np.abs(ref)))
                want = scale * s.max() + np.log(w.sum())
                assert abs(float(lse[r, i, h]) - want) <= 2.0 ** -21 * abs(want) + 2.0 ** -18
                total += 1.0
        # every query's weights add up to 1 over the pages
        assert abs(got_w[r].sum() - total) <= total * (n * 2.0 ** -22 + 2.0 ** -18)


def poison(pool, slot, tok, head, C, D, what):
    """Marks one scale byte of a token NaN: block 1 of its K or V."""
    gb = 16 * (D + D // 8)
    base = (head * (C // 16) + tok // 16) * gb + (16 * D if what == "k" else 17 * D)
    pool[slot, base + (tok % 16) * (D // 16) + 1] = 0x7F


@pytest.mark.parametrize("D", [64, 128])
def test_stale_and_non_finite_bytes(D):
    """Bytes past kv_len are never used; a NaN token reaches only the queries that see it."""
    lens, n_q, C, H, G = [40, 27], 4, 16, 2, 2
    pool, pages, rng = make(lens, C, H, D, 23)
    q = torch.from_numpy(rng.standard_normal((2, n_q, H * G, D))).to(torch.float16).cuda()
    args = q, dev(np.array(lens, np.int32)), dev(pages)
    want, wl = cache(pool, C, H, D).attend(*args)
    dirty = pool.copy()
    for r, n in enumerate(lens):
        for pos in range(n, pages.shape[1] * C):
            for h in range(H):
                R.put_token(dirty, pages[r, pos // C], pos % C, h, C, H, D, *(np.full(D, 15, np.uint8), np.full(D // 16, 0x7F, np.uint8)) * 2)
    got, gl = cache(dirty, C, H, D).attend(*args)
    assert torch.equal(got, want) and torch.equal(gl, wl)
    # request 0: V of token 38 of head 0 (seen by queries 2, 3); request 1: K of token 25 of head 1 (queries 2, 3)
    bad = pool.copy()
    poison(bad, pages[0, 38 // C], 38 % C, 0, C, D, "v")
    poison(bad, pages[1, 25 // C], 25 % C, 1, C, D, "k")
    got, gl = cache(bad, C, H, D).attend(*args)
    assert torch.equal(got[0, :, G:], want[0, :, G:]) and torch.equal(got[1, :, :G], want[1, :, :G])
    assert torch.equal(got[0, :2], want[0, :2]) and torch.equal(got[1, :2], want[1, :2])
    assert torch.isnan(got[0, 2:, :G, 16:32]).all() and torch.equal(got[0, 2:, :G, :16], want[0, 2:, :G, :16])
    assert torch.isnan(got[1, 2:, G:]).all()


def test_repeats_bit_for_bit_and_shared_pages():
    """Two requests on the same slots get the same answers; a second call the same bits, weights included."""
    C, H, G, D = 16, 2, 4, 128
    pool, pages, rng = make([700], C, H, D, 24)
    pages = np.concatenate((pages, pages))
    kv = cache(pool, C, H, D)
    q = torch.from_numpy(rng.standard_normal((1, 1, H * G, D))).to(torch.bfloat16).cuda().expand(2, -1, -1, -1)
    res = []
    for _ in range(2):
        w = torch.zeros(pages.shape, dtype=torch.float32, device="cuda")
        res.append((*kv.attend(q, dev(np.array([700, 700], np.int32)), dev(pages), weight=w), w))
    for a, b in zip(*res):
        assert torch.equal(a, b) and torch.equal(a[0], a[1])
    kv.check()


@pytest.mark.parametrize("what", ["slot", "long", "negative"])
def test_device_errors(what):
    from paper_2609_38706_gb300 import pk
    lens, C, H, D = [40, 40], 16, 1, 64
    pool, pages, rng = make(lens, C, H, D, 25)
    n = np.array(lens, np.int32)
    if what == "slot":
        pages[1, 1] = 0x7FFFFFFF
    else:
        n[1] = 49 if what == "long" else -1
    kv = cache(pool, C, H, D)
    q = torch.from_numpy(rng.standard_normal((2, 1, 2, D))).to(torch.bfloat16).cuda()
    kv.attend(q, dev(n), dev(pages), weight=torch.zeros(pages.shape, device="cuda"))
    assert kv.take_status() == pk.PK_ERR_ARG
    pages = np.clip(pages, 0, pool.shape[0] - 1)
    kv.attend(q, dev(np.array(lens, np.int32)), dev(pages))
    kv.check()


def test_refusals():
    from paper_2609_38706_gb300 import pk
    pool, pages, rng = make([40], 16, 2, 64, 26)
    kv = cache(pool, 16, 2, 64)
    q = torch.zeros((1, 1, 4, 64), dtype=torch.bfloat16, device="cuda")
    n, p = dev(np.array([40], np.int32)), dev(pages)
    bad = [(q[0], n, p), (q.float(), n, p), (q[:, :, :3], n, p), (q[..., :32], n, p), (q, n.long(), p), (q, n, p.long()),
           (q, n, p[0])]
    for a in bad:
        with pytest.raises(pk.PKError):
            kv.attend(*a)
    with pytest.raises(pk.PKError):
        kv.attend(q, n, p, float("inf"))
    with pytest.raises(pk.PKError):
        kv.attend(q, n, p, weight=torch.zeros((1, 2), device="cuda"))
