"""GPU tests of the norms of queries and keys with their rotation against a plain 64-bit implementation."""
import math

import numpy as np
import pytest
import torch

import kv_ref as R

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
EPS = 1e-6


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g
    g.build()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def frequencies(rot, base=10000.0, factor=1.0, context=0.0, low=1.0, high=32.0):
    f = base ** (np.arange(rot // 2) * (-2.0 / rot))
    stays = np.clip((context * f / (2 * math.pi) - low) / (high - low), 0, 1) if context else 0.0
    return stays * f + (1 - stays) * f / factor


def reference(x, w, pos, f, interleaved, amp, dtype):
    """float64 rows [n, heads, D] -> (result, bound on its error)."""
    D, rot = x.shape[-1], 2 * len(f)
    y, part = x.copy(), 2.0 ** -30
    if w is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + np.float32(EPS)) * w
        # D squares summed in 32 bits, the mean, eps, the root (2 units), and two products
        part = (D / 2 + 8) * 2.0 ** -24
    t = pos[:, None, None] * f
    c, s = np.cos(t) * amp, np.sin(t) * amp
    at = np.arange(rot // 2)
    i, j = (2 * at, 2 * at + 1) if interleaved else (at, at + rot // 2)
    out, size = y.copy(), np.abs(y)
    a, b = y[..., i], y[..., j]
    out[..., i], out[..., j] = a * c - b * s, a * s + b * c
    mag = amp * (np.abs(a) + np.abs(b))
    # the angle: its table's entry in 64 bits, 2^-32 of a turn, 24 bits of half a turn; sine and cosine to 2 units; their
    # product with amp, two products and a sum of 32 bits
    slack = part + (np.abs(t) * 2.0 ** -48 + 2.0 ** -29 + math.pi * 2.0 ** -24) + 2.0 ** -22 + 3 * 2.0 ** -24
    bound = part * size
    bound[..., i] = mag * slack
    bound[..., j] = mag * slack
    return out, bound * (1 + R.U[dtype]) + R.U[dtype] * np.abs(out) + 2.0 ** -24 * (dtype == "fp16")


def check(got, want, bound):
    assert np.all(np.abs(got.double().cpu().numpy() - want) <= bound)


CASES = [
    # lens, starts, q heads, kv heads, D, rotary, interleaved, norms, dtype, scaling
    ([1], [0], 1, 1, 64, 64, False, "", "bf16", {}),
    ([1, 0, 3, 2], [5, 7, 0, 131071], 4, 2, 128, 128, False, "qk", "bf16", {}),
    ([7, 1], [1000, 2 ** 31 - 1], 3, 1, 128, 128, True, "qk", "fp16", dict(base=500000.0, factor=8.0, context=8192.0)),
    ([33], [12345], 5, 5, 64, 32, True, "k", "fp16", dict(factor=4.0)),
    ([40, 41], [0, 99], 7, 1, 64, 48, False, "q", "bf16", {}),
    ([12], [2 ** 30], 32, 8, 128, 16, False, "qk", "fp16", dict(factor=40.0, context=4096.0, high=8.0)),
    ([300, 5, 0, 260], [0, 31, 2, 77777], 32, 8, 128, 96, True, "", "bf16", {}),
    ([20], [100], 0, 3, 64, 64, False, "k", "bf16", {}),
    ([20], [100], 9, 0, 128, 112, False, "q", "fp16", {}),
]


@pytest.mark.parametrize("lens,starts,qh,kh,D,rot,interleaved,norms,dtype,scaling", CASES)
def test_matches_reference(lens, starts, qh, kh, D, rot, interleaved, norms, dtype, scaling):
    from paper_2609_38706_gb300 import service
    rng = np.random.default_rng(5)
    n, amp = sum(lens), 1.0 + 0.1 * math.log(scaling.get("factor", 1.0))
    qkv = torch.from_numpy(rng.standard_normal((n, qh + 2 * kh, D)) * np.exp(rng.standard_normal((n, 1, 1)))).to(DT[dtype]).cuda()
    q, k = qkv[:, :qh], qkv[:, qh: qh + kh]
    w = [torch.from_numpy(rng.uniform(0.5, 1.5, D)).to(DT[dtype]).cuda() if x in norms else None for x in "qk"]
    off = dev(np.concatenate(([0], np.cumsum(lens))).astype(np.int64))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    rotary = service.Rotary(D, rot, interleaved=interleaved, amplitude=amp, **scaling)
    qo, ko = service.rotate(q, k, off, dev(np.array(starts, np.int32)), rotary, *w, eps=EPS, status=status)
    assert status.item() == 0 and qo.is_contiguous() and ko.is_contiguous()
    pos = np.concatenate([np.arange(s, s + m, dtype=np.float64) for s, m in zip(starts, lens)])
    f = frequencies(rot, **scaling)
    for x, y, z in ((q, qo, w[0]), (k, ko, w[1])):
        check(y, *reference(x.double().cpu().numpy(), None if z is None else z.double().cpu().numpy(), pos, f, interleaved, amp, dtype))
    # in place, through the pool's method: the same bits, and the values between them stay
    kv = service.KVPages(2, 16, 1, D)
    before = qkv.clone()
    a, b = kv.rotate(q, k, off, dev(np.array(starts, np.int32)), rotary, *w, eps=EPS, out=(q, k))
    kv.check()
    assert a is q and b is k and torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(qkv[:, qh + kh:], before[:, qh + kh:])


def simple(n, heads=(4, 2), D=64, dtype=torch.bfloat16, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn((n, h, D), generator=g, device="cuda").to(dtype) for h in heads]


def test_rows_of_no_request_and_bad_offsets():
    from paper_2609_38706_gb300 import pk, service
    q, k = simple(20)
    rotary = service.Rotary(64)
    good = service.rotate(q, k, dev(np.array([0, 20])), dev(np.array([3], np.int32)), rotary)
    # rows before the first and behind the last request are left as they were
    out = [torch.full_like(x, 7.0) for x in (q, k)]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    service.rotate(q, k, dev(np.array([4, 9, 15])), dev(np.array([7, 12], np.int32)), rotary, out=out, status=status)
    assert status.item() == 0
    for x, y in zip(out, good):
        assert torch.equal(x[4:15], y[4:15]) and bool((x[:4] == 7).all()) and bool((x[15:] == 7).all())
    # each is reported, and its tokens are not written
    for off, start in (([0, 5, 21], [3, 8]), ([0, 5, 3], [3, 8]), ([-1, 5, 20], [2, 8]), ([0, 5, 20], [3, -1]),
                       ([0, 5, 20], [3, 2 ** 31 - 15]), ([2 ** 62, 5, 20], [3, 8])):
        out = [torch.full_like(x, 7.0) for x in (q, k)]
        status.zero_()
        bad = start[1] < 0 or start[1] > 2 ** 30
        service.rotate(q, k, dev(np.array(off)), dev(np.array(start, np.int32)), rotary, out=out, status=status)
        assert status.item() == (pk.PK_OK if start[1] == 2 ** 31 - 15 else pk.PK_ERR_ARG), (off, start)
        if bad and start[1] < 0:
            for x, y in zip(out, good):
                assert torch.equal(x[:5], y[:5]) and bool((x[5:] == 7).all())
    status.zero_()
    out = [torch.full_like(x, 7.0) for x in (q, k)]
    service.rotate(q, k, dev(np.array([0, 20])), dev(np.array([2 ** 31 - 10], np.int32)), rotary, out=out, status=status)
    assert status.item() == pk.PK_ERR_ARG and bool((out[0][10:] == 7).all()) and not bool((out[0][:10] == 7).any())


def test_nothing_to_do():
    from paper_2609_38706_gb300 import service
    rotary = service.Rotary(64)
    q, k = simple(0)
    service.rotate(q, k, dev(np.array([0, 0])), dev(np.zeros(1, np.int32)), rotary)
    q, k = simple(3)
    service.rotate(q, k, dev(np.zeros(1, np.int64)), dev(np.zeros(0, np.int32)), rotary)


def test_large_and_odd_values_stay_in_their_row():
    """A row past the top of 32 bits when squared is still normed; infinities and NaN reach their own row only."""
    from paper_2609_38706_gb300 import service
    q, k = simple(4)
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    rotary, off, start = service.Rotary(64), dev(np.array([0, 4])), dev(np.array([9], np.int32))
    clean = service.rotate(q, k, off, start, rotary, w, w)
    q[1, 2] *= 2.0 ** 100
    k[0, 1] = 0.0
    k[3, 0, 5] = float("nan")
    q[2, 0, 40] = float("inf")
    qo, ko = service.rotate(q, k, off, start, rotary, w, w)
    assert torch.equal(ko[0, 1], torch.zeros_like(ko[0, 1])) and bool(ko[3, 0].isnan().all())
    assert not bool(qo[2, 0].isfinite().all())
    # eps is nothing beside the mean of squares, here or there: the same row times 2^100 is the same row, to eps' share
    # (its mean of squares is above 0.3), half a unit of the result, and what the sum's rounding differs by
    assert bool(((qo[1, 2].double() - clean[0][1, 2].double()).abs() <= clean[0][1, 2].double().abs() * 2.0 ** -7 + 2.0 ** -16).all())
    for x, y, skip in ((qo, clean[0], [(1, 2), (2, 0)]), (ko, clean[1], [(0, 1), (3, 0)])):
        same = torch.ones(x.shape[:2], dtype=torch.bool)
        for s in skip:
            same[s] = False
        assert torch.equal(x[same.cuda()], y[same.cuda()])


@pytest.mark.parametrize("interleaved", [False, True])
def test_scores_depend_on_distance_alone(interleaved):
    """q at position p and k at p - 100: their product is the same wherever p lies, to the rounding of the rows."""
    from paper_2609_38706_gb300 import service
    q, k = simple(1, heads=(1, 1), D=128, dtype=torch.float16)
    rotary, off = service.Rotary(128, interleaved=interleaved), dev(np.array([0, 1]))
    at = lambda x, p: service.rotate(x, x, off, dev(np.array([p], np.int32)), rotary)[0].double()  # noqa: E731
    scores = [float((at(q, p) * at(k, p - 100)).sum()) for p in (100, 1000, 123456, 2 ** 31 - 1)]
    # each row is off by half a unit a value, in both factors, and the angle's bits
    room = 2 * float((q.double().abs().sum() * k.double().abs().max())) * (R.U["fp16"] + 2.0 ** -20)
    assert max(scores) - min(scores) <= 2 * room
    assert abs(scores[0] - float((q.double() * k.double()).sum())) > 0.1  # and it does depend on the distance


def test_captured_and_on_another_stream():
    from paper_2609_38706_gb300 import service
    q, k = simple(50, dtype=torch.float16)
    w = torch.ones(64, dtype=torch.float16, device="cuda")
    rotary, off, start = service.Rotary(64), dev(np.array([0, 20, 50])), dev(np.array([3, 1000], np.int32))
    out = [torch.empty_like(q), torch.empty_like(k)]
    service.rotate(q, k, off, start, rotary, w, w, out=out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        service.rotate(q, k, off, start, rotary, w, w, out=out)
    for seed in (1, 2):
        a, b = simple(50, dtype=torch.float16, seed=seed)
        q.copy_(a), k.copy_(b), start.fill_(17 * seed)
        g.replay()
        want = service.rotate(a, b, off, start, rotary, w, w)
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    side = torch.cuda.Stream()
    kv = service.KVPages(2, 16, 1, 64, stream=side)
    side.wait_stream(torch.cuda.current_stream())
    got = kv.rotate(q, k, off, start, rotary, w, w)
    kv.check()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_refusals():
    from paper_2609_38706_gb300 import pk, service
    q, k = simple(4)
    rotary, off, start = service.Rotary(64), dev(np.array([0, 4])), dev(np.array([9], np.int32))
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    ok = dict(q=q, k=k, tok_off=off, start=start, rotary=rotary)
    service.rotate(**ok)
    for change in (dict(q=q.float()), dict(k=k.half()), dict(k=k[:3]), dict(q=q.transpose(1, 2)), dict(q=q.cpu()),
                   dict(rotary=service.Rotary(128)), dict(q_weight=w.half()), dict(k_weight=w[:32]), dict(q_weight=w.cpu()),
                   dict(k_weight=w.clone().requires_grad_()), dict(q=q.clone().requires_grad_()), dict(eps=0.0),
                   dict(tok_off=off.int()), dict(start=start.long()), dict(out=(q, q)), dict(out=(q[:, :1].expand(4, 4, 64), k)),
                   dict(rotary=service.Rotary(64, device="cpu"))):
        with pytest.raises(pk.PKError):
            service.rotate(**{**ok, **change})
