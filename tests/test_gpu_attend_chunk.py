"""GPU tests of attention of chunks of new tokens over the 4-bit page cache, with and without a sliding window, against a plain
64-bit implementation."""
import numpy as np
import pytest
import torch

import kv_ref as R
import window_ref as W
from test_gpu_attend_cache import DT, cache, dev, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g
    g.build()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def offsets(lens):
    return dev(np.concatenate(([0], np.cumsum(lens))).astype(np.int64))


def reference(pool, pages, new, lens, q, C, H, D, scale, window=None, sinks=0, k_scale=1.0, v_scale=1.0):
    """out, lse, mag, the scores' error bound, and which pages are seen."""
    G = q.shape[1] // H
    out, mag = np.zeros(q.shape), np.zeros(q.shape)
    lse, err = np.zeros(q.shape[:2]), 0.0
    used, at = np.zeros(pages.shape, bool), 0
    for r, (m, n) in enumerate(zip(new, lens)):
        ok = W.seen(n - m, m, n, window, sinks)
        full = np.zeros((m, pages.shape[1] * C), bool)
        full[:, :n] = ok
        used[r] = full.reshape(m, pages.shape[1], C).any((0, 2))
        k = v = np.zeros((0, H, D))
        if n:
            k, v = R.get_tokens(pool, np.where(used[r], pages[r], 0)[: -(-n // C)], n, C, H, D)
            k, v = k * float(np.float32(k_scale)), v * float(np.float32(v_scale))
        for h in range(H * G):
            x = q[at: at + m, h]
            o, l, _, a = W.attend(x, k[:, h // G], v[:, h // G], ok, scale)
            out[at: at + m, h], lse[at: at + m, h], mag[at: at + m, h] = o, l, a
            if n and m:
                err = max(err, R.score_error(x, k[:, h // G], scale))
        at += m
    return out, lse, mag, err, used


def check(out, lse, ref, rl, mag, err, dtype, n):
    # the weights are rounded to halves for the product with V, whatever the type of q
    assert np.all(np.abs(out.double().cpu().numpy() - ref) <= R.out_bound(ref, mag, R.U["fp16"], R.U[dtype], err, n))
    gl = lse.double().cpu().numpy()
    none = np.isneginf(rl)
    assert np.array_equal(none, np.isneginf(gl))
    assert np.all(np.abs(gl[~none] - rl[~none]) <= R.lse_bound(rl, err, n)[~none])


CASES = [
    # new, lens, C, H, G, D, dtype, window, sinks, k_scale, v_scale
    ([1], [1], 16, 1, 1, 64, "bf16", None, 0, 1.0, 1.0),
    ([1, 0, 3], [5, 9, 3], 16, 2, 4, 128, "bf16", None, 0, 1.0, 1.0),
    ([40, 5, 0, 7], [40, 3, 0, 300], 48, 2, 3, 64, "fp16", None, 0, 0.0173, 0.25),   # 3 tokens for 5 queries
    ([130, 257], [130, 300], 16, 1, 1, 128, "fp16", None, 0, 1.0, 1.0),
    ([33, 64, 65], [500, 64, 1000], 256, 2, 4, 128, "bf16", None, 0, 1.0, 2.0),
    ([100], [1000], 32, 1, 7, 64, "bf16", None, 0, 1.0, 1.0),
    ([10], [9000], 64, 2, 5, 128, "fp16", None, 0, 1.0, 1.0),        # cut into pieces
    ([3, 20], [6000, 40], 16, 1, 16, 64, "bf16", None, 0, 1.0, 1.0),  # pieces, and a request too short for more than one
    ([2], [700], 16, 1, 130, 64, "fp16", None, 0, 1.0, 1.0),         # more heads in a group than a tile's rows
    ([2, 9] * 20, [30, 9] * 20, 16, 1, 2, 64, "bf16", None, 0, 1.0, 1.0),  # more requests than a warp has lanes
    ([1], [1], 16, 1, 1, 64, "bf16", 1, 0, 1.0, 1.0),
    ([40, 5, 0, 7], [40, 3, 0, 300], 48, 2, 3, 64, "fp16", 1, 1, 1.0, 1.0),
    ([130, 257], [130, 600], 16, 1, 1, 128, "fp16", 64, 4, 1.0, 1.0),
    ([33, 64, 65], [500, 64, 1000], 256, 2, 4, 128, "bf16", 17, 0, 1.0, 2.0),
    ([100, 300], [1000, 300], 32, 1, 7, 64, "bf16", 129, 33, 1.0, 1.0),
    ([10], [9000], 64, 2, 5, 128, "fp16", 4000, 200, 1.0, 1.0),       # pieces
    ([10], [5000], 64, 1, 2, 128, "bf16", 4990, 3, 1.0, 1.0),         # the gap is a few tokens
    ([2], [700], 16, 1, 130, 64, "fp16", 100, 10, 1.0, 1.0),
    ([2, 9] * 20, [30, 9] * 20, 16, 1, 2, 64, "bf16", 5, 2, 1.0, 1.0),
    ([300], [400], 16, 1, 2, 64, "bf16", 10, 100000, 1.0, 1.0),       # everything is a first token
    ([300], [400], 16, 1, 2, 64, "bf16", 100000, 0, 1.0, 1.0),
]


@pytest.mark.parametrize("new,lens,C,H,G,D,dtype,window,sinks,k_scale,v_scale", CASES)
def test_matches_reference(new, lens, C, H, G, D, dtype, window, sinks, k_scale, v_scale):
    pool, pages, rng = make(lens, C, H, D, 21, spare=3)
    q = torch.from_numpy(rng.standard_normal((sum(new), H * G, D)) * (2 / k_scale)).to(DT[dtype])
    scale = D ** -0.5
    ref, rl, mag, err, used = reference(pool, pages, new, lens, q.double().numpy(), C, H, D, scale, window, sinks, k_scale, v_scale)
    kv = cache(pool, C, H, D, k_scale, v_scale)
    pages = np.where(used, pages, -1)  # what nobody sees may have been given back
    out, lse = kv.attend_chunk(q.cuda(), offsets(new), dev(np.array(lens, np.int32)), dev(pages), scale, window=window, sinks=sinks)
    kv.check()
    check(out, lse, ref, rl, mag, err, dtype, max(lens))


@pytest.mark.parametrize("window,sinks", [(None, 0), (300, 4)])
@pytest.mark.parametrize("D", [64, 128])
def test_what_lies_behind_a_request_is_never_used(D, window, sinks):
    """Pages whose places behind the request's end, and slots of nobody, hold NaN marks: the same bits."""
    new, lens, C, H, G = [30, 1, 200], [500, 17, 250], 16, 2, 2
    pool, pages, rng = make(lens, C, H, D, 9, spare=5)
    q = torch.from_numpy(rng.standard_normal((sum(new), H * G, D))).to(torch.bfloat16).cuda()
    args = (offsets(new), dev(np.array(lens, np.int32)), dev(pages))
    want = cache(pool, C, H, D).attend_chunk(q, *args, window=window, sinks=sinks)
    dirty = np.full_like(pool, 0x7F).reshape(pool.shape[0], H, C // 16, 16, -1)
    gb = 16 * (D + D // 8)
    clean = pool.reshape(pool.shape[0], H, C // 16, gb)
    dirty = dirty.reshape(pool.shape[0], H, C // 16, gb)
    for r, n in enumerate(lens):
        for p in range(-(-n // C)):
            slot, tokens = pages[r, p], min(C, n - p * C)
            for t in range(tokens):
                g, i = divmod(t, 16)
                for off, width in ((0, D // 2), (8 * D, D // 2), (16 * D, D // 16), (17 * D, D // 16)):
                    at = slice(off + i * width, off + (i + 1) * width)
                    dirty[slot, :, g, at] = clean[slot, :, g, at]
    got = cache(dirty.reshape(pool.shape), C, H, D).attend_chunk(q, *args, window=window, sinks=sinks)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("D,window,sinks", [(64, None, 0), (128, None, 0), (64, 20, 5), (128, 150, 5)])
def test_marked_blocks_reach_only_queries_that_see_them(D, window, sinks):
    """NaN blocks in V and K, in tiles that all queries see, at the causal edge and at the window's ends."""
    m, n, C, H, G = 40, 400, 16, 1, 2
    pool, pages, rng = make([n], C, H, D, 8)
    q = torch.from_numpy(rng.standard_normal((m, G, D))).to(torch.float16).cuda()
    args = (q, offsets([m]), dev(np.array([n], np.int32)), dev(pages))
    clean, clean_lse = cache(pool, C, H, D).attend_chunk(*args, window=window, sinks=sinks)
    for which in (0, 1):  # K, V
        for j in (2, 5, 120, 210, 341, 350, 361, 380, 383, 384, 399):
            marked = pool.copy()
            marked.reshape(-1, C // 16, 16 * (D + D // 8))[pages[0, j // C], 0, 16 * D + which * D + j % C * (D // 16) + 1] = 0x7F
            out, lse = cache(marked, C, H, D).attend_chunk(*args, window=window, sinks=sinks)
            sees = torch.from_numpy(W.seen(n - m, m, n, window, sinks)[:, j]).cuda()
            assert torch.equal(out[~sees], clean[~sees]) and torch.equal(lse[~sees], clean_lse[~sees]), (which, j)
            if which:
                hit = torch.zeros(D, dtype=torch.bool, device="cuda")
                hit[16:32] = True
                assert bool(out[sees][..., hit].isnan().all()) and torch.equal(out[sees][..., ~hit], clean[sees][..., ~hit]), j
                assert torch.equal(lse, clean_lse)
            else:
                assert bool(out[sees].isnan().all()) and bool(lse[sees].isnan().all()), j


def test_marked_blocks_in_pieces():
    """The same where the keys are cut."""
    m, n, C, H, G, D = 3, 5000, 16, 1, 2, 64
    pool, pages, rng = make([n], C, H, D, 8)
    q = torch.from_numpy(rng.standard_normal((m, G, D))).to(torch.bfloat16).cuda()
    args = (q, offsets([m]), dev(np.array([n], np.int32)), dev(pages))
    clean, clean_lse = cache(pool, C, H, D).attend_chunk(*args)
    for j in (700, n - 2):
        marked = pool.copy()
        marked.reshape(-1, C // 16, 16 * (D + D // 8))[pages[0, j // C], 0, 17 * D + j % C * (D // 16) + 3] = 0xFF
        out, lse = cache(marked, C, H, D).attend_chunk(*args)
        sees = torch.arange(n - m, n, device="cuda") >= j
        assert torch.equal(out[~sees], clean[~sees]) and torch.equal(lse, clean_lse)
        assert bool(out[sees][..., 48:].isnan().all()) and torch.equal(out[sees][..., :48], clean[sees][..., :48])


@pytest.mark.parametrize("new,lens", [([20, 30], [100, 400]), ([4, 3], [6000, 100])])
def test_errors_reported(new, lens):
    from paper_2609_38706_gb300 import pk
    C, H, G, D = 16, 1, 2, 64
    pool, pages, rng = make(lens, C, H, D, 3)
    kv = cache(pool, C, H, D)
    q = torch.from_numpy(rng.standard_normal((sum(new), H * G, D))).to(torch.bfloat16).cuda()
    off, n, a = offsets(new), dev(np.array(lens, np.int32)), new[0]
    want = kv.attend_chunk(q, off, n, dev(pages))
    kv.check()
    # a slot out of range: the queries that see it
    bad = pages.copy()
    bad[0, lens[0] // C - 1] = 1 << 20
    out, lse = kv.attend_chunk(q, off, n, dev(bad))
    assert kv.take_status() == pk.PK_ERR_ARG
    assert bool(out[:a].isnan().all()) and bool(lse[:a].isnan().all())
    assert torch.equal(out[a:], want[0][a:]) and torch.equal(lse[a:], want[1][a:])
    # a length out of range counts as 0
    for length in (-1, pages.shape[1] * C + 1, -2 ** 31, 2 ** 31 - 1):
        out, lse = kv.attend_chunk(q, off, dev(np.array([length, lens[1]], np.int32)), dev(pages))
        assert kv.take_status() == pk.PK_ERR_ARG
        assert bool((out[:a] == 0).all()) and bool(torch.isneginf(lse[:a]).all())
        err = (out[a:].double() - want[0][a:].double()).abs()  # (keys may be cut elsewhere)
        assert bool((err <= 0.02 * want[0][a:].double().abs().max()).all())
    # offsets out of order or range: nothing is written
    for o in ([0, a, sum(new) + 1], [0, a, a - 1], [-1, a, sum(new)], [5, 2, sum(new)], [0, 2 ** 62, sum(new)]):
        out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
        scratch = torch.zeros(pk.pk_attend_chunk_scratch_bytes(kv.kv, q.dtype, q.shape[0], 2, H * G, pages.shape[1], 0, 0), dtype=torch.uint8, device="cuda")
        pk.pk_attend_chunk(kv.kv, q, out, lse, dev(np.array(o)), n, dev(pages), 1.0, 0, 0, scratch, kv.status)
        assert kv.take_status() == pk.PK_ERR_ARG, o
        assert bool((out == 7).all()) and bool((lse == 7).all()), o


@pytest.mark.parametrize("R_", [2, 40])
def test_errors_of_many_requests(R_):
    """Bad offsets of one of few or of many requests: nothing is written."""
    from paper_2609_38706_gb300 import pk
    C, H, D = 16, 1, 64
    lens = [20] * R_
    pool, pages, rng = make(lens, C, H, D, 3)
    kv = cache(pool, C, H, D)
    q = torch.from_numpy(rng.standard_normal((2 * R_, 2, D))).to(torch.bfloat16).cuda()
    off = np.arange(0, 2 * R_ + 1, 2)
    off[R_ - 1] = -5
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    scratch = torch.zeros(pk.pk_attend_chunk_scratch_bytes(kv.kv, q.dtype, q.shape[0], R_, 2, pages.shape[1], 0, 0), dtype=torch.uint8, device="cuda")
    pk.pk_attend_chunk(kv.kv, q, out, lse, dev(off), dev(np.array(lens, np.int32)), dev(pages), 1.0, 0, 0, scratch, kv.status)
    assert kv.take_status() == pk.PK_ERR_ARG and bool((out == 7).all()) and bool((lse == 7).all())


def test_strides_and_rows_of_no_request():
    """q and out as parts of wider rows; rows before the first and behind the last request stay as they are; no lse asked for."""
    from paper_2609_38706_gb300 import pk
    new, lens, C, H, G, D = [5, 20], [60, 33], 16, 2, 3, 128
    pool, pages, rng = make(lens, C, H, D, 3)
    kv = cache(pool, C, H, D)
    qkv = torch.from_numpy(rng.standard_normal((30, H * G + 2 * H, D))).to(torch.float16).cuda()
    q, off, n = qkv[:, : H * G], dev(np.array([2, 7, 27])), dev(np.array(lens, np.int32))
    want, _ = kv.attend_chunk(q[2:27].contiguous(), offsets(new), n, dev(pages))
    wide = torch.full((30, H * G + 1, D), 7.0, dtype=torch.float16, device="cuda")
    out = wide[:, : H * G]
    scratch = torch.zeros(pk.pk_attend_chunk_scratch_bytes(kv.kv, q.dtype, 30, 2, H * G, pages.shape[1], 0, 0), dtype=torch.uint8, device="cuda")
    pk.pk_attend_chunk(kv.kv, q, out, None, off, n, dev(pages), D ** -0.5, 0, 0, scratch, kv.status)
    kv.check()
    assert torch.equal(out[2:27], want)
    assert bool((wide[:2] == 7).all()) and bool((wide[27:] == 7).all()) and bool((wide[:, H * G] == 7).all())


@pytest.mark.parametrize("m,n", [(20, 300), (2, 6000)])
def test_far_scores_keep_their_order(m, n):
    """Scores of 2^24 and more, whose rounding is wider than a weight's exponents: the heaviest key wins, its value comes out."""
    C, H, G, D = 16, 1, 1, 64
    pool, pages, rng = make([n], C, H, D, 3)
    q = torch.from_numpy(rng.standard_normal((m, G, D)) * 2.0 ** 28).to(torch.bfloat16)
    kv = cache(pool, C, H, D)
    for sign in (1.0, -1.0):
        out, lse = kv.attend_chunk(q.cuda(), offsets([m]), dev(np.array([n], np.int32)), dev(pages), sign)
        kv.check()
        k, v = R.get_tokens(pool, pages[0], n, C, H, D)
        for i in range(m):
            s = sign * (k[: n - m + i + 1, 0] @ q[i, 0].double().numpy())
            top = np.sort(s)[-2:]
            # 64 products summed in 32 bits
            room = 72 * 2.0 ** -23 * float(np.abs(q[i].double().numpy()).sum() * np.abs(k).max())
            assert abs(float(lse[i, 0]) - top[1]) <= room
            if top[1] - top[0] > 2 * room + 100:  # no other key weighs anything
                got = out[i, 0].double().cpu().numpy()
                assert np.all(np.abs(got - v[s.argmax(), 0]) <= 2.0 ** -8 * np.abs(v[s.argmax(), 0]))


def roomy(pages, D=64):
    """The same pages with room in the table for so many more that queries are worth making halves of."""
    return np.concatenate([pages, np.full((pages.shape[0], 2 ** 20 // D * 8), -1, pages.dtype)], 1)


@pytest.mark.parametrize("room", [False, True])
@pytest.mark.parametrize("far,D,window", [(2.0 ** 27, 64, None), (2.0 ** 30, 128, 300), (2.0 ** 45, 64, 300), (2.0 ** 60, 128, None)])
def test_wide_queries(far, D, window, room):
    """Rows with one large value, behind which K holds nothing, beside ordinary ones: these keep their bits, also where halves
    cannot hold both."""
    m, n, C, H, G = 20, 700, 16, 1, 2
    pool, pages, rng = make([n], C, H, D, 5)
    pool.reshape(-1, C // 16, 16 * (D + D // 8))[:, :, 0: 8 * D: D // 2] &= 0xF0  # K: dimension 0 holds nothing
    q = torch.from_numpy(rng.standard_normal((m, G, D))).to(torch.bfloat16)
    q[3:, :, 0] = far
    kv = cache(pool, C, H, D)
    out, lse = kv.attend_chunk(q.cuda(), offsets([m]), dev(np.array([n], np.int32)), dev(roomy(pages) if room else pages),
                               window=window, sinks=2)
    kv.check()
    small = np.where(np.arange(D) == 0, 0, q.double().numpy())
    small[:3] = q[:3].double().numpy()
    ref, rl, mag, err, _ = reference(pool, pages, [m], [n], small, C, H, D, D ** -0.5, window, 2)
    check(out, lse, ref, rl, mag, err, "bf16", n)


@pytest.mark.parametrize("room", [False, True])
@pytest.mark.parametrize("small", [2.0 ** -100, 2.0 ** -130, 0.0])
def test_tiny_and_infinite_queries(small, room):
    """Rows of tiny values weigh all keys alike; an infinity or NaN reaches its own row only."""
    m, n, C, H, G, D = 6, 300, 16, 1, 1, 64
    pool, pages, rng = make([n], C, H, D, 5)
    q = torch.from_numpy(rng.standard_normal((m, G, D))).to(torch.bfloat16)
    q[1] *= small
    kv = cache(pool, C, H, D)
    args = (offsets([m]), dev(np.array([n], np.int32)), dev(roomy(pages) if room else pages))
    out, lse = kv.attend_chunk(q.cuda(), *args)
    ref, rl, mag, err, _ = reference(pool, pages, [m], [n], q.double().numpy(), C, H, D, D ** -0.5)
    check(out, lse, ref, rl, mag, err, "bf16", n)
    for bad in (float("inf"), float("nan")):
        odd = q.clone()
        odd[4, 0, 9] = bad
        got, glse = kv.attend_chunk(odd.cuda(), *args)
        kv.check()
        keep = [0, 1, 2, 3, 5]
        check(got[keep], glse[keep], ref[keep], rl[keep], mag[keep], err, "bf16", n)
        assert bool(got[4].isnan().any())


@pytest.mark.parametrize("new,lens,C,H,G,D,window", [([40, 5, 0, 7], [40, 3, 0, 300], 48, 2, 3, 64, None), ([130, 257], [130, 300], 16, 1, 1, 128, None),
                                                     ([2, 9] * 20, [30, 9] * 20, 16, 1, 2, 64, None), ([700], [700], 16, 1, 130, 64, None),
                                                     ([33, 64, 65], [500, 64, 1000], 256, 2, 4, 128, 17)])
def test_queries_as_halves_or_not_are_the_same(new, lens, C, H, G, D, window):
    """A table with room for long requests has the call make halves of its queries, which are as exact: the same products,
    in sums that may be cut at other keys only.  Rows of no request, here NaN, have no say."""
    from paper_2609_38706_gb300 import pk
    pool, pages, rng = make(lens, C, H, D, 8, spare=2)
    n_q, dt = sum(new), torch.bfloat16
    q = torch.full((n_q + 70, H * G, D), float("nan"), dtype=dt, device="cuda")
    q[3: 3 + n_q] = torch.from_numpy(rng.standard_normal((n_q, H * G, D)) * 10.0 ** rng.uniform(-3, 1, (n_q, H * G, 1))).to(dt).cuda()
    off, n, kv, got = offsets(new) + 3, dev(np.array(lens, np.int32)), cache(pool, C, H, D), []
    for table in (pages, roomy(pages)):
        table = dev(table)
        out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
        nbytes = pk.pk_attend_chunk_scratch_bytes(kv.kv, dt, q.shape[0], len(new), H * G, table.shape[1], window or 0, 2)
        pk.pk_attend_chunk(kv.kv, q, out, lse, off, n, table, D ** -0.5, window or 0, 2,
                           torch.zeros(nbytes, dtype=torch.uint8, device="cuda"), kv.status)
        kv.check()
        assert bool((out[:3] == 7).all()) and bool((out[3 + n_q:] == 7).all()) and bool((lse[3 + n_q:] == 7).all())
        got.append((nbytes, out[3: 3 + n_q].clone(), lse[3: 3 + n_q].clone()))
    assert window or got[1][0] - got[0][0] >= q.numel() * 2  # a window bounds the keys whatever the table holds
    ref, rl, mag, err, _ = reference(pool, pages, new, lens, q[3: 3 + n_q].double().cpu().numpy(), C, H, D, D ** -0.5, window, 2)
    for _, out, lse in got:
        check(out, lse, ref, rl, mag, err, "bf16", max(lens))


def test_one_token_chunks_are_decode_steps():
    """Chunks of one token against the decode call: the same numbers to both calls' error."""
    lens, C, H, G, D = [1, 50, 700], 16, 2, 4, 128
    pool, pages, rng = make(lens, C, H, D, 3)
    kv = cache(pool, C, H, D)
    q = torch.from_numpy(rng.standard_normal((3, H * G, D)) * 2).to(torch.bfloat16)
    n, p = dev(np.array(lens, np.int32)), dev(pages)
    for window, sinks in ((None, 0), (33, 2)):
        a, la = kv.attend_chunk(q.cuda(), offsets([1, 1, 1]), n, p, window=window, sinks=sinks)
        b, lb = kv.attend(q.cuda().unsqueeze(1), n, p, window=window, sinks=sinks)
        kv.check()
        ref, rl, mag, err, _ = reference(pool, pages, [1, 1, 1], lens, q.double().numpy(), C, H, D, D ** -0.5, window, sinks)
        bound = R.out_bound(ref, mag, R.U["fp16"], R.U["bf16"], err, max(lens))
        assert np.all(np.abs((a.double() - b.squeeze(1).double()).cpu().numpy()) <= 2 * bound)
        assert np.all(np.abs((la - lb.squeeze(1)).double().cpu().numpy()) <= 2 * R.lse_bound(rl, err, max(lens)))


@pytest.mark.parametrize("window", [None, 100])
def test_captured_with_other_lengths(window):
    """Replayed with other lengths, offsets and values than it was captured with; two calls' scratch is their own."""
    C, H, G, D = 16, 2, 2, 64
    pool, pages, rng = make([6000, 500], C, H, D, 4)
    kv = cache(pool, C, H, D)
    q = torch.from_numpy(rng.standard_normal((24, H * G, D))).to(torch.float16).cuda()
    off, n, p = dev(np.array([0, 12, 24])), dev(np.array([6000, 20], np.int32)), dev(pages)
    kv.attend_chunk(q, off, n, p, window=window)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a = kv.attend_chunk(q, off, n, p, window=window, sinks=3)
        b = kv.attend_chunk(q, off, n, p)
    for o, lens in (([0, 1, 24], [5000, 500]), ([0, 24, 24], [30, 0]), ([4, 8, 20], [6000, 400])):
        off.copy_(dev(np.array(o))), n.copy_(dev(np.array(lens, np.int32)))
        q.copy_(torch.from_numpy(rng.standard_normal(q.shape)))
        g.replay()
        for got, want in ((a, kv.attend_chunk(q, off, n, p, window=window, sinks=3)), (b, kv.attend_chunk(q, off, n, p))):
            assert torch.equal(got[0][o[0]: o[2]], want[0][o[0]: o[2]]) and torch.equal(got[1][o[0]: o[2]], want[1][o[0]: o[2]])
    kv.check()


def test_on_a_pool_with_a_stream():
    from paper_2609_38706_gb300.service import KVPages
    new, lens, C, H, D = [40, 3], [300, 4000], 16, 2, 64
    pool, pages, rng = make(lens, C, H, D, 4)
    q = torch.from_numpy(rng.standard_normal((43, 4, D))).to(torch.float16).cuda()
    off, n, p = offsets(new), dev(np.array(lens, np.int32)), dev(pages)
    want = cache(pool, C, H, D).attend_chunk(q, off, n, p)
    side = torch.cuda.Stream()
    kv = KVPages(pool.shape[0], C, H, D, stream=side, pool=dev(pool))
    side.wait_stream(torch.cuda.current_stream())
    got = [kv.attend_chunk(q, off, n, p) for _ in range(3)]
    kv.check()
    assert all(torch.equal(x[0], want[0]) and torch.equal(x[1], want[1]) for x in got)


def test_nothing_to_do():
    pool, pages, rng = make([40], 16, 1, 64, 4)
    kv = cache(pool, 16, 1, 64)
    empty = torch.zeros((0, 2, 64), dtype=torch.float16, device="cuda")
    kv.attend_chunk(empty, dev(np.array([0, 0])), dev(np.array([40], np.int32)), dev(pages))
    q = torch.zeros((3, 2, 64), dtype=torch.float16, device="cuda")
    kv.attend_chunk(q, dev(np.array([0])), dev(np.zeros(0, np.int32)), dev(np.zeros((0, 3), np.int32)))
    out, lse = kv.attend_chunk(q, dev(np.array([0, 3])), dev(np.zeros(1, np.int32)), dev(np.zeros((1, 0), np.int32)))
    kv.check()
    assert bool((out == 0).all()) and bool(torch.isneginf(lse).all())


def test_refusals():
    from paper_2609_38706_gb300 import pk
    pool, pages, rng = make([40], 16, 2, 64, 4)
    kv = cache(pool, 16, 2, 64)
    q = torch.zeros((4, 4, 64), dtype=torch.float16, device="cuda")
    ok = dict(q=q, q_off=dev(np.array([0, 4])), kv_len=dev(np.array([40], np.int32)), pages=dev(pages))
    kv.attend_chunk(**ok)
    for change in (dict(q=q.float()), dict(q=q[:, :3]), dict(q=q[..., :32]), dict(q=q.unsqueeze(0)), dict(q=q.cpu()),
                   dict(q=q.clone().requires_grad_()), dict(q_off=ok["q_off"].int()), dict(q_off=ok["q_off"][:1]),
                   dict(kv_len=ok["kv_len"].long()), dict(pages=ok["pages"].long()), dict(pages=ok["pages"][0]),
                   dict(window=0), dict(window=-3), dict(window=1 << 31), dict(window=5, sinks=-1), dict(window=5, sinks=1 << 31),
                   dict(scale=float("nan")), dict(scale=3e38), dict(pages=ok["pages"].cpu())):
        with pytest.raises(pk.PKError):
            kv.attend_chunk(**{**ok, **change})
    with pytest.raises(pk.PKError):  # scratch of another call
        pk.pk_attend_chunk(kv.kv, q, torch.empty_like(q), None, ok["q_off"], ok["kv_len"], ok["pages"], 1.0, 0, 0,
                           torch.zeros(8, dtype=torch.uint8, device="cuda"), kv.status)


def test_pool_past_32_bits():
    """Pages whose bytes lie behind 4 GiB answer as the same pages in a small pool, in chunks and in windowed steps."""
    from paper_2609_38706_gb300.service import KVPages
    new, lens, C, H, D = [30, 2], [300, 90], 256, 8, 128
    pool, pages, rng = make(lens, C, H, D, 4)
    q = torch.from_numpy(rng.standard_normal((32, 16, D))).to(torch.bfloat16).cuda()
    small = cache(pool, C, H, D)
    n_slots = (1 << 32) // pool.shape[1] + 40
    big = KVPages(n_slots, C, H, D)
    base = n_slots - pool.shape[0]
    big.pool[base:] = dev(pool)
    off, n = offsets(new), dev(np.array(lens, np.int32))
    for window, sinks in ((None, 0), (60, 2)):
        a = small.attend_chunk(q, off, n, dev(pages), window=window, sinks=sinks)
        b = big.attend_chunk(q, off, n, dev(pages + base), window=window, sinks=sinks)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    one = q[:2].view(2, 1, 16, D)
    a = small.attend(one, n, dev(pages), window=60, sinks=2)
    b = big.attend(one, n, dev(pages + base), window=60, sinks=2)
    big.check()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("new,lens,window", [([700] * 6, [900] * 6, None), ([64] * 50, [400] * 50, 100), ([2000], [2000], None),
                                             ([1] * 300, [33] * 300, None), ([9] * 3, [20000, 150, 9000], 15000)])
def test_many_shapes_against_small_calls(new, lens, window):
    """Calls whose work is cut in many ways: each request alone, in a call of its own, is cut elsewhere; both are within the
    bounds that the small cases hold to, so they differ by two of them at most."""
    C, H, G, D = 16, 2, 2, 64
    pool, pages, rng = make(lens, C, H, D, 6)
    kv = cache(pool, C, H, D)
    q = torch.from_numpy(rng.standard_normal((sum(new), H * G, D))).to(torch.float16).cuda()
    n, p = dev(np.array(lens, np.int32)), dev(pages)
    out, lse = kv.attend_chunk(q, offsets(new), n, p, window=window, sinks=4)
    a = 0
    for r, m in enumerate(new):
        if r % max(1, len(new) // 5) == 0:
            o, l = kv.attend_chunk(q[a: a + m].contiguous(), offsets([m]), n[r: r + 1].clone(), p[r: r + 1].clone(), window=window, sinks=4)
            k, v = R.get_tokens(pool, pages[r], lens[r], C, H, D)
            err = R.score_error(q[a: a + m].double().cpu().numpy(), k, D ** -0.5)
            # mag, a mean of magnitudes, is at most the largest
            bound = 2 * R.out_bound(o.double().cpu().numpy(), np.abs(v).max(), R.U["fp16"], R.U["fp16"], err, lens[r])
            assert np.all(np.abs((out[a: a + m].double() - o.double()).cpu().numpy()) <= bound)
            assert np.all(np.abs((lse[a: a + m] - l).double().cpu().numpy()) <= 2 * R.lse_bound(l.double().cpu().numpy(), err, lens[r]))
        a += m
    kv.check()
