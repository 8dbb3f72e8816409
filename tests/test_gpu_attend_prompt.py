"""GPU tests of attention over packed prompts against a plain 64-bit implementation."""
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


def offs(n):
    return np.concatenate(([0], np.cumsum(n))).astype(np.int64)


def inputs(lq, lk, H, G, D, dtype, seed, peak=1.0):
    rng = np.random.default_rng(seed)
    f = lambda n, h, a: torch.from_numpy((a * rng.standard_normal((n, h, D))).astype(np.float32)).to(DT[dtype])
    return f(sum(lq), H * G, peak), f(sum(lk), H, 1.0), f(sum(lk), H, 1.0)


def check(q, k, v, lq, lk, out, lse, dtype, scale, rows=None):
    """Every query of `rows` (None: all) of every request and head against the reference."""
    qo, ko = offs(lq), offs(lk)
    G = q.shape[1] // k.shape[1]
    q, k, v = (x.double().cpu().numpy() for x in (q, k, v))
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for r in range(len(lq)):
        i = np.arange(lq[r]) if rows is None else np.unique(np.clip(rows, 0, lq[r] - 1)) if lq[r] else np.arange(0)
        for h in range(q.shape[1]):
            kk, vv = k[ko[r]:ko[r + 1], h // G], v[ko[r]:ko[r + 1], h // G]
            qq = q[qo[r] + i, h]
            if not len(i):
                continue
            ref, rl, _, mag = R.attend(qq, kk, vv, i + lk[r] - lq[r], scale)
            err = R.score_error(qq, kk, scale) if lk[r] else 0.0
            got, gl = out[qo[r] + i, h], lse[qo[r] + i, h]
            assert np.all(np.abs(got - ref) <= R.out_bound(ref, mag, R.U[dtype], R.U[dtype], err, lk[r])), (r, h)
            none = np.isneginf(rl)
            assert np.array_equal(none, np.isneginf(gl))
            assert np.all(np.abs(gl[~none] - rl[~none]) <= R.lse_bound(rl, err, lk[r])[~none]), (r, h)


CASES = [
    ([1], [1], 1, 1, 64, "bf16"),
    ([1, 1, 1], [1, 77, 500], 2, 4, 128, "fp16"),
    ([5, 0, 63, 64, 65], [5, 3, 63, 64, 65], 2, 3, 64, "bf16"),
    ([127, 128, 129, 200], [127, 128, 129, 200], 1, 1, 128, "bf16"),
    ([33, 7], [300, 1000], 2, 7, 128, "bf16"),
    ([9, 4], [5, 0], 1, 2, 64, "fp16"),            # queries before the first key: empty rows
    ([257, 130], [400, 130], 1, 8, 64, "fp16"),
    ([40], [41], 1, 16, 128, "fp16"),
    ([3], [130], 1, 129, 64, "bf16"),              # a group larger than a tile's rows
    ([0], [0], 1, 1, 64, "bf16"),
    ([3, 2], [0, 0], 2, 2, 128, "fp16"),           # no key at all
    ([300] * 7, [300] * 7, 2, 2, 128, "bf16"),
    ([3, 0, 40] * 11, [5, 2, 90] * 11, 2, 3, 64, "fp16"),  # more requests than a warp has lanes
    ([2] * 32, [9] * 32, 1, 1, 128, "bf16"),
]


@pytest.mark.parametrize("lq,lk,H,G,D,dtype", CASES)
def test_matches_reference(lq, lk, H, G, D, dtype):
    from paper_2609_38706_gb300 import service
    q, k, v = inputs(lq, lk, H, G, D, dtype, 11)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = service.attend_prompt(q.cuda(), k.cuda(), v.cuda(), dev(offs(lq)), dev(offs(lk)), status=status)
    assert int(status.item()) == 0
    check(q, k, v, lq, lk, out, lse, dtype, D ** -0.5)


def test_long_prompt_sampled_rows():
    from paper_2609_38706_gb300 import service
    lq, lk = [2500], [4001]
    q, k, v = inputs(lq, lk, 1, 2, 128, "bf16", 12, peak=3.0)
    out, lse = service.attend_prompt(q.cuda(), k.cuda(), v.cuda(), dev(offs(lq)), dev(offs(lk)))
    check(q, k, v, lq, lk, out, lse, "bf16", 128 ** -0.5, rows=np.array([0, 1, 63, 64, 127, 128, 1000, 2431, 2498, 2499]))


@pytest.mark.parametrize("H,G,D,dtype", [(8, 4, 128, "bf16"), (4, 3, 64, "fp16")])
def test_many_more_blocks_than_the_gpu_holds(H, G, D, dtype):
    """Several rounds of blocks on every SM, calls back to back: the same bits each time, sampled rows against the
    reference."""
    from paper_2609_38706_gb300 import service
    lq = [512, 341, 470, 375, 256, 314, 374, 452]
    lk = [n + 300 * (i % 3) for i, n in enumerate(lq)]
    q, k, v = inputs(lq, lk, H, G, D, dtype, 19)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = q.cuda(), k.cuda(), v.cuda(), dev(offs(lq)), dev(offs(lk))
    res = [service.attend_prompt(*args, status=status) for _ in range(6)]
    assert int(status.item()) == 0
    for out, lse in res[1:]:
        assert torch.equal(out, res[0][0]) and torch.equal(lse, res[0][1])
    check(q, k, v, lq, lk, *res[0], dtype, D ** -0.5, rows=np.array([0, 31, 64, 200, 255, 256, 300, 511]))


@pytest.mark.parametrize("R,H,G,D,dtype", [(7, 8, 4, 128, "bf16"), (41, 4, 3, 64, "fp16"), (1, 4, 128, 64, "bf16")])
def test_blocks_take_items_as_they_come(R, H, G, D, dtype):
    """More items than SMs and many keys a request: a block's next item is the next that has not started.  Requests
    without queries or keys among them, calls back to back and on two streams: the same bits each time."""
    from paper_2609_38706_gb300 import service
    rng = np.random.default_rng(R)
    lq = [int(x) for x in rng.integers(60, 400 if R < 32 else 90, R)]
    lk = [n + int(x) for n, x in zip(lq, rng.integers(1300, 2400, R))]
    if R > 1:
        lq[3], lk[5] = 0, 0
    q, k, v = inputs(lq, lk, H, G, D, dtype, 23)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = q.cuda(), k.cuda(), v.cuda(), dev(offs(lq)), dev(offs(lk))
    res = [service.attend_prompt(*args, status=status) for _ in range(4)]
    torch.cuda.synchronize()
    for s in [torch.cuda.Stream() for _ in range(2)]:
        with torch.cuda.stream(s):
            res.append(service.attend_prompt(*args, status=status))
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    for out, lse in res[1:]:
        assert torch.equal(out, res[0][0]) and torch.equal(lse, res[0][1])
    check(q, k, v, lq, lk, *res[0], dtype, D ** -0.5, rows=np.array([0, 41, 84, 300]))


@pytest.mark.parametrize("R,n,prefix,H,G,D", [(8, 300, 1700, 8, 4, 128), (40, 100, 1400, 4, 3, 64), (8, 300, 0, 8, 4, 128)])
def test_captured_calls_replay_the_same(R, n, prefix, H, G, D):
    """Two calls behind each other in a CUDA graph, replayed: the bits of a plain call, either way of giving out items."""
    from paper_2609_38706_gb300 import service
    q, k, v = (x.cuda() for x in inputs([n] * R, [n + prefix] * R, H, G, D, "bf16", 29))
    qo, ko = dev(offs([n] * R)), dev(offs([n + prefix] * R))
    want = service.attend_prompt(q, k, v, qo, ko)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = [service.attend_prompt(q, k, v, qo, ko) for _ in range(2)]
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for out, lse in got:
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
def test_scales_and_peaked_rows(scale):
    """A scale of 0 weighs all keys alike; a large one is decided by the maximum, which moves as keys come."""
    from paper_2609_38706_gb300 import service
    lq, lk = [150], [333]
    q, k, v = inputs(lq, lk, 1, 2, 64, "fp16", 13)
    k[:] = k * torch.linspace(0.1, 3.0, lk[0]).view(-1, 1, 1).to(k.dtype)  # later keys larger
    out, lse = service.attend_prompt(q.cuda(), k.cuda(), v.cuda(), dev(offs(lq)), dev(offs(lk)), scale)
    check(q, k, v, lq, lk, out, lse, "fp16", scale)


def test_strided_tensors():
    from paper_2609_38706_gb300 import pk
    lq, H, G, D = [70, 20], 2, 2, 64
    q, k, v = inputs(lq, lq, H, G, D, "bf16", 14)
    t = sum(lq)
    fused = torch.zeros((t, H * G + 2 * H, D), dtype=q.dtype, device="cuda")
    fused[:, :H * G], fused[:, H * G:H * G + H], fused[:, H * G + H:] = q.cuda(), k.cuda(), v.cuda()
    whole = torch.full((H * G, t, 2 * D), 7.0, dtype=q.dtype, device="cuda")
    out = whole[:, :, :D].transpose(0, 1)  # head-major, every second half row left alone
    lse = torch.empty((t, H * G), dtype=torch.float32, device="cuda")
    off = dev(offs(lq))
    scratch = torch.empty(pk.pk_attend_prompt_scratch_bytes(2), dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    pk.pk_attend_prompt(fused[:, :H * G], fused[:, H * G:H * G + H], fused[:, H * G + H:], out, lse, off, off, 0.125,
                        scratch, status)
    check(q, k, v, lq, lq, out, lse, "bf16", 0.125)
    assert torch.all(whole[:, :, D:] == 7.0) and int(status.item()) == 0


def test_keys_broadcast_over_heads():
    """One head's keys and values for every KV head, as expanded tensors (stride 0)."""
    from paper_2609_38706_gb300 import service
    lq = [70, 33]
    q, k, v = (x.cuda() for x in inputs(lq, lq, 1, 6, 64, "bf16", 20))
    off = dev(offs(lq))
    one, _ = service.attend_prompt(q, k, v, off, off)
    three, _ = service.attend_prompt(q, k.expand(-1, 3, -1), v.expand(-1, 3, -1), off, off)
    assert torch.equal(one, three)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("D,G", [(64, 1), (128, 4)])
def test_masked_places_do_not_leak(value, D, G):
    """Non-finite keys and values reach only the queries that attend them, never another request."""
    from paper_2609_38706_gb300 import service
    lq = [90, 140]
    q, k, v = inputs(lq, lq, 1, G, D, "bf16", 15)
    off = dev(offs(lq))
    clean, _ = service.attend_prompt(q.cuda(), k.cuda(), v.cuda(), off, off)
    k2, v2 = k.clone(), v.clone()
    v2[60, 0, 5] = value                # request 0, dimension 5 of token 60
    k2[75, 0, 3] = float("nan")         # request 0, scores of token 75
    v2[90 + 130, 0, :] = value          # request 1, token 130
    out, lse = service.attend_prompt(q.cuda(), k2.cuda(), v2.cuda(), off, off)
    assert torch.equal(out[:60], clean[:60])
    keep = [d for d in range(D) if d != 5]
    assert torch.equal(out[60:75][..., keep], clean[60:75][..., keep])
    assert not torch.isfinite(out[60:75, :, 5]).any()
    assert torch.isnan(out[75:90]).all() and torch.isfinite(lse[:75]).all()
    assert torch.equal(out[90:220], clean[90:220])
    assert not torch.isfinite(out[220:]).any()


def test_outputs_repeat_and_other_rows_stay():
    from paper_2609_38706_gb300 import pk
    lq, lk = [100, 64], [100, 90]
    q, k, v = (x.cuda() for x in inputs(lq, lk, 2, 2, 128, "bf16", 16))
    qo = offs(lq) + 0
    qo[2] -= 10  # the last ten rows belong to no request
    outs = []
    for _ in range(2):
        out = torch.full_like(q, 3.0)
        lse = torch.full(q.shape[:2], 3.0, device="cuda")
        scratch = torch.empty(pk.pk_attend_prompt_scratch_bytes(2), dtype=torch.uint8, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        pk.pk_attend_prompt(q, k, v, out, lse, dev(qo), dev(offs(lk)), 0.1, scratch, status)
        assert int(status.item()) == 0
        outs.append((out, lse))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    assert torch.all(outs[0][0][154:] == 3.0) and torch.all(outs[0][1][154:] == 3.0)


@pytest.mark.parametrize("many_requests", [0, 50])
@pytest.mark.parametrize("what", ["q order", "k range", "k negative"])
def test_bad_offsets_write_nothing(what, many_requests):
    from paper_2609_38706_gb300 import pk, service
    lq = [30, 30]
    q, k, v = (x.cuda() for x in inputs(lq, lq, 1, 1, 64, "fp16", 17))
    many = np.full(many_requests, 60, np.int64)  # empty requests behind the two
    qo, ko = np.concatenate((offs(lq), many)), np.concatenate((offs(lq), many))
    if what == "q order":
        qo[1] = 70
    elif what == "k range":
        ko[2:] = 61
    else:
        ko[0] = -1
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 5.0)
    scratch = torch.empty(pk.pk_attend_prompt_scratch_bytes(len(qo) - 1), dtype=torch.uint8, device="cuda")
    pk.pk_attend_prompt(q, k, v, out, None, dev(qo), dev(ko), 1.0, scratch, status)
    assert int(status.item()) == pk.PK_ERR_ARG and torch.all(out == 5.0)


def test_refusals():
    from paper_2609_38706_gb300 import pk, service
    q, k, v = (x.cuda() for x in inputs([8], [8], 2, 2, 64, "bf16", 18))
    off = dev(offs([8]))
    for a in ((q.float(), k, v), (q, k, v.half()), (q[:, :3], k, v), (q, k, v[:4]), (q[..., :32], k[..., :32], v[..., :32]),
              (q, k[:, :, ::2], v[:, :, ::2])):
        with pytest.raises(pk.PKError):
            service.attend_prompt(*a, off, off)
    with pytest.raises(pk.PKError):
        service.attend_prompt(q, k, v, off.cpu(), off)
    with pytest.raises(pk.PKError):
        service.attend_prompt(q, k.cpu(), v, off, off)
    with pytest.raises(pk.PKError):
        service.attend_prompt(q, k, v, off, off, float("nan"))
    with pytest.raises(pk.PKError):
        service.attend_prompt(q, k, v, off.int(), off)
    with pytest.raises(pk.PKError):
        service.attend_prompt(q, k, v, off, dev(offs([4, 4])))


@pytest.mark.parametrize("D,G", [(64, 3), (128, 1), (128, 7)])
def test_scores_beyond_a_weights_exponents(D, G):
    """Scores 2^24 and more apart from each other, up to near the top of their type: 32 bits hold them exactly here
    (one nonzero value a key, powers of two), so the softmax is exact: the heaviest keys share the weight."""
    from paper_2609_38706_gb300 import service
    H, lq, lk = 2, [70, 5], [200, 133]
    rng = np.random.default_rng(2)
    q = np.zeros((sum(lq), H * G, D), np.float32)
    q[..., 0] = 2.0 ** rng.choice((0, 20, 30, 45, 60), q.shape[:2])
    k = np.zeros((sum(lk), H, D), np.float32)
    k[..., 0] = rng.choice((-1, 1, 1.0078125, 2.0 ** 20, 2.0 ** 40, -2.0 ** 40), k.shape[:2])
    v = rng.standard_normal(k.shape).astype(np.float32)
    q, k, v = (torch.from_numpy(x).to(torch.bfloat16) for x in (q, k, v))
    out, lse = service.attend_prompt(q.cuda(), k.cuda(), v.cuda(), dev(offs(lq)), dev(offs(lk)), 0.37)
    qd, kd, vd = (x.double().numpy() for x in (q, k, v))
    qo, ko = offs(lq), offs(lk)
    for r in range(2):
        for h in range(H * G):
            kk, vv = kd[ko[r]:ko[r + 1], h // G, 0], vd[ko[r]:ko[r + 1], h // G]
            for i in range(lq[r]):
                n = i + lk[r] - lq[r] + 1
                s = qd[qo[r] + i, h, 0] * kk[:n]
                w = np.exp(0.37 * (s - s.max()))
                ref = w @ vv[:n] / w.sum()
                # the scale's log2 e rounds to 32 bits, and the scores' distances with it
                err = np.minimum(0.37 * (s.max() - s), 40.0) * 2.0 ** -22
                rel = 2 * np.expm1(err.max()) + 2.0 ** -8 + n * 2.0 ** -24
                assert np.all(np.abs(out[qo[r] + i, h].double().cpu().numpy() - ref) <= rel * (np.abs(vv[:n]).max() + np.abs(ref)))
                assert abs(float(lse[qo[r] + i, h]) - (0.37 * s.max() + np.log(w.sum()))) <= 2.0 ** -21 * abs(0.37 * s.max()) + 2.0 ** -18


def test_unused_rows_of_a_tile_may_hold_anything():
    """Groups of 3 and 7 leave rows of a 128-row tile without a query: what shared memory holds there (here the values
    of an earlier call, up to the type's top) does not matter, and keeps no warp."""
    from paper_2609_38706_gb300 import service
    big = torch.full((300, 8, 64), 3e38, dtype=torch.bfloat16, device="cuda")
    service.attend_prompt(big, big[:, :2].contiguous(), big[:, :2].contiguous(), dev(offs([300])), dev(offs([300])))
    for G in (3, 7):
        lq, lk = [300, 40], [300, 90]
        q, k, v = inputs(lq, lk, 2, G, 64, "bf16", G)
        out, lse = service.attend_prompt(q.cuda(), k.cuda(), v.cuda(), dev(offs(lq)), dev(offs(lk)), 0.125)
        check(q, k, v, lq, lk, out, lse, "bf16", 0.125)
