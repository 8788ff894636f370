"""GPU parity of the position ids with axes (exact) and of the embedding by them against the fp64 oracle.

The embedding: sine and cosine of an angle reduced to half turns with 24 bits, 2^-22 at most, products and sum in fp32 and half a
step of bf16 (2^-8 of the value): |error| <= 2^-8 |x'| + 2^-21 (|a| + |b|)."""
import numpy as np
import pytest
import torch

from oracle import axes as A
from paper_2602_24082_b200 import workloads as W

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, np.int32))).cuda()


def _spans(rows, seed, most, side, in_responses=True):
    """Random spans inside segments, some that fill one, some next to each other."""
    rng = np.random.default_rng(seed)
    starts, grids = [], []
    for a, n, _, _, seg in W.Workload("s", rows, 1, 1, 64, seed=0).segments():
        if seg and not in_responses:
            continue
        at, end = a + int(rng.integers(0, 4)), a + n
        for _ in range(most):
            f, h, w = (int(rng.integers(1, side + 1)) for _ in range(3))
            if at + f * h * w > end:
                continue
            starts.append(at)
            grids.append((f, h, w))
            at += f * h * w + int(rng.choice([0, 1, 7]))
    return starts, np.asarray(grids, np.int32).reshape(-1, 3)


STRUCTURES = {
    "pair": [[(64, (32, 48))]],
    "ragged": [[(257, (5, 128, 31))], [(1, (1, 300))]],
    "ones": [[(1, (1,) * 37)] for _ in range(9)],
    "one_token": [[(1, (1,))]],
    "long": [[(5000, (900, 1300))], [(3001, (1, 2000, 7))]],
    "groups": [[(40, (9, 30)), (7, (12,))]] * 60,
}


@pytest.mark.parametrize("rows", list(STRUCTURES.values()), ids=list(STRUCTURES))
@pytest.mark.parametrize("most,side", [(0, 1), (2, 3), (40, 1), (3000, 1), (9, 9)])
def test_position_ids(rows, most, side):
    from paper_2602_24082_b200 import binding as B
    starts, grids = _spans(rows, most + side, most, side)
    plan = B.plan_for(W.Workload("axes", rows, 2, 1, 64, seed=0), desc_on_device=side == 1)
    pos, status = B.pp_position_ids_axes(plan, _i32(starts), _i32(grids))
    assert plan.status() == (0, 0) and status.tolist() == [0, 0]
    assert np.array_equal(pos.cpu().numpy(), A.position_ids(rows, starts, grids))
    if not most:
        assert torch.equal(pos, B.pp_position_ids(plan).expand(3, -1))


def test_more_spans_in_a_group_than_a_block_holds_at_a_time():
    from paper_2602_24082_b200 import binding as B
    rows = [[(50, (4,)), (9000, (5000, 7))], [(30, (4,))]]
    starts = list(range(54, 9054, 3)) + list(range(9056, 14050, 5)) + [14055]     # 1024 at a time
    grids = [[(1, 1, 3), (1, 1, 1), (2, 1, 1), (1, 3, 1)][i % 4] for i in range(len(starts))]
    plan = B.plan_for(W.Workload("axes", rows, 2, 1, 64, seed=0))
    pos, status = B.pp_position_ids_axes(plan, _i32(starts), _i32(grids))
    assert status.tolist() == [0, 0]
    assert np.array_equal(pos.cpu().numpy(), A.position_ids(rows, starts, grids))


def test_more_segments_and_spans_than_a_block_holds():
    from paper_2602_24082_b200 import binding as B
    rows = [[(3, (2, 1)), (5, (7,))]] * 800
    starts = [a + 1 for a, n, _, _, seg in W.Workload("s", rows, 1, 1, 64, seed=0).segments() if n in (3, 5, 7)]
    grids = [[(1, 1, 2), (2, 1, 1), (1, 2, 1)][i % 3] for i in range(len(starts))]
    assert len(starts) == 2400
    plan = B.plan_for(W.Workload("axes", rows, 2, 1, 64, seed=0))
    pos, status = B.pp_position_ids_axes(plan, _i32(starts), _i32(grids))
    assert status.tolist() == [0, 0]
    assert np.array_equal(pos.cpu().numpy(), A.position_ids(rows, starts, grids))


@pytest.mark.parametrize("starts,grids,first", [
    ([2, 20], [(1, 2, 2), (1, 0, 3)], 1),                      # an empty side
    ([2, 20], [(1, -2, 2), (1, 1, 3)], 0),
    ([60], [(1, 5, 1)], 0),                                    # beyond the prompt's end
    ([62, 63], [(1, 1, 2), (1, 1, 1)], 1),                     # overlap
    ([20, 2], [(1, 1, 2), (1, 1, 1)], 1),                      # not ascending
    ([-1], [(1, 1, 2)], 0),
    ([143], [(1, 1, 2)], 0),                                   # beyond the last token
    ([7000], [(1, 1, 2)], 0),
    ([3], [(2147483647, 2147483647, 2147483647)], 0),
    ([2147483647], [(1, 1, 2147483647)], 0),
    ([-2147483648], [(1, 1, 2147483647)], 0),
], ids=str)
def test_spans_that_break_the_rules_are_reported(starts, grids, first):
    from paper_2602_24082_b200 import binding as B
    plan = B.plan_for(W.Workload("axes", STRUCTURES["pair"], 2, 1, 64, seed=0))
    out = torch.full((4, 144), -7, dtype=torch.int32, device="cuda")
    _, status = B.pp_position_ids_axes(plan, _i32(starts), _i32(grids), out=out[:3])
    assert status.tolist() == [1, first] and (out[3] == -7).all() and plan.status() == (0, 0)


ROWS = [[(33, (5, 28, 31))], [(1, (1, 30))]]
T = 129


def _rope_case(Hq, Hkv, D, seed):
    g = torch.Generator().manual_seed(seed)
    q, k = (torch.randn(T, h, D, generator=g).bfloat16().cuda() for h in (Hq, Hkv))
    from paper_2602_24082_b200 import binding as B
    return B.plan_for(W.Workload("axes", ROWS, Hq, Hkv, D, seed=0)), q, k


def _check(got, x, pos, axis, base, inverse):
    x64 = x.double().cpu().numpy()
    want = A.rope(x64, pos, axis, base, inverse)
    half = x64.shape[-1] // 2
    size = np.abs(x64[..., :half]) + np.abs(x64[..., half:])
    tol = 2.0 ** -8 * np.abs(want) * (1 + 2.0 ** -7) + 2.0 ** -21 * np.concatenate([size, size], -1)
    err = np.abs(got.double().cpu().numpy() - want)
    assert (err <= tol).all(), (err / tol).max()


SECTIONS = {64: [(8, 12, 12), (32,), (1, 30, 1), (8, 8, 8, 8)], 96: [(12, 18, 18), (48,), (0, 24, 24)],
            128: [(16, 24, 24), (64,), (20, 4, 40), (16, 16, 16, 16)]}


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (7, 1), (32, 8), (14, 2), (64, 8), (140, 20)])
@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("inverse", [False, True])
def test_rope_parity(Hq, Hkv, D, inverse):
    from paper_2602_24082_b200 import binding as B
    plan, q, k = _rope_case(Hq, Hkv, D, Hq + D)
    q0, k0 = q.clone(), k.clone()
    rng = np.random.default_rng(D)
    for i, sections in enumerate(SECTIONS[D]):
        pos = rng.integers(0, 131072, (len(sections), T))
        # text far behind, the largest and smallest numbers, and in front of the start
        pos[:, :6] = [0, 1, 2147483647, -2147483648, -5, 1 << 20]
        base, interleaved = [10000.0, 500000.0, 1000000.0][i % 3], bool(i % 2)
        axis = B.axis_of_frequency(sections, interleaved)
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        B.pp_rope_qk_axes(plan, q, k, _i32(pos), sections, base, interleaved, inverse, q_out=qo, k_out=ko)
        assert torch.equal(q, q0) and torch.equal(k, k0)
        _check(qo, q, pos, axis, base, inverse)
        _check(ko, k, pos, axis, base, inverse)
        # in place
        a, b = q.clone(), k.clone()
        r = B.pp_rope_qk_axes(plan, a, b, _i32(pos), sections, base, interleaved, inverse)
        assert r[0].data_ptr() == a.data_ptr() and torch.equal(a, qo) and torch.equal(b, ko)
        # out of and into the buffer of a fused projection, whose other parts stay as they are
        fused = torch.full((T, Hq + 2 * Hkv, D), 3.0, dtype=torch.bfloat16, device="cuda")
        fq, fk = fused[:, :Hq], fused[:, Hq:Hq + Hkv]
        fq.copy_(q)
        fk.copy_(k)
        a.zero_(), b.zero_()
        B.pp_rope_qk_axes(plan, fq, fk, _i32(pos), sections, base, interleaved, inverse, q_out=a, k_out=b)
        assert torch.equal(a, qo) and torch.equal(b, ko) and torch.equal(fq, q) and torch.equal(fk, k)
        B.pp_rope_qk_axes(plan, q, k, _i32(pos), sections, base, interleaved, inverse, q_out=fq, k_out=fk)
        assert torch.equal(fq, qo) and torch.equal(fk, ko) and (fused[:, Hq + Hkv:] == 3).all()
        B.pp_rope_qk_axes(plan, fq.copy_(q), fk.copy_(k), _i32(pos), sections, base, interleaved, inverse)
        assert torch.equal(fq, qo) and torch.equal(fk, ko) and (fused[:, Hq + Hkv:] == 3).all()
    assert plan.status() == (0, 0)


def test_the_inverse_is_the_transpose():
    """<rotate(x), y> = <x, inverse(y)>: both products of bf16-rounded vectors, 2^-8 of a norm each."""
    from paper_2602_24082_b200 import binding as B
    plan, q, k = _rope_case(4, 2, 128, 5)
    y, z = torch.randn_like(q), torch.randn_like(k)
    pos = _i32(np.random.default_rng(1).integers(0, 9000, (3, T)))
    new = lambda a, b: dict(q_out=torch.empty_like(a), k_out=torch.empty_like(b))
    rq, rk = B.pp_rope_qk_axes(plan, q, k, pos, (16, 24, 24), **new(q, k))
    iy, iz = B.pp_rope_qk_axes(plan, y, z, pos, (16, 24, 24), inverse=True, **new(y, z))
    dot = lambda a, b: float((a.double() * b.double()).sum())
    for x, rx, g, ig in ((q, rq, y, iy), (k, rk, z, iz)):
        assert abs(dot(rx, g) - dot(x, ig)) <= 2 * 2.0 ** -8 * float(x.double().norm() * g.double().norm())


def test_offsets_beyond_32_bits():
    """Tokens whose elements lie beyond 2^31 and 2^32 in the fused buffer."""
    from paper_2602_24082_b200 import binding as B
    rows, Hq, Hkv, D = [[(50000, (20000, 4000))]], 32, 8, 128
    n = 74000
    plan = B.plan_for(W.Workload("axes", rows, Hq, Hkv, D, seed=0))
    fused = torch.empty(n, 460 * D, dtype=torch.bfloat16, device="cuda")     # 4.36 G elements
    heads = fused.view(n, 460, D)
    q, k = heads[:, :Hq], heads[:, Hq:Hq + Hkv]
    q.normal_(), k.normal_()
    pos = torch.arange(n, dtype=torch.int32, device="cuda").expand(3, n).contiguous()
    tail = slice(n - 50, n)
    q0, k0 = q[tail].clone(), k[tail].clone()
    B.pp_rope_qk_axes(plan, q, k, pos, (16, 24, 24))
    for got, x in ((q[tail], q0), (k[tail], k0)):
        _check(got, x, np.tile(np.arange(n - 50, n), (3, 1)), B.axis_of_frequency((16, 24, 24)), 10000.0, False)


def test_streams_and_graphs():
    from paper_2602_24082_b200 import binding as B
    plan, q, k = _rope_case(8, 2, 128, 9)
    starts, grids = _spans(ROWS, 3, 3, 2)
    starts, grids = _i32(starts), _i32(grids)

    def step():
        pos, _ = B.pp_position_ids_axes(plan, starts, grids)
        return (pos,) + tuple(B.pp_rope_qk_axes(plan, q, k, pos, (16, 24, 24), q_out=torch.empty_like(q), k_out=torch.empty_like(k)))

    want = step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        there = step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            held = step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(there, want))
    q.copy_(q.flip(0))
    grids.fill_(1)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(held, step()))
    assert not torch.equal(held[0], want[0]) and not torch.equal(held[1], want[1])


def test_refusals():
    from paper_2602_24082_b200 import binding as B
    plan, q, k = _rope_case(4, 2, 64, 1)
    pos = torch.zeros(3, T, dtype=torch.int32, device="cuda")
    s = (8, 12, 12)
    for args in ((q[:-1], k, pos), (q.float(), k, pos), (q, k.cpu(), pos), (q, q, pos), (q, k, pos[:2]),
                 (q, k, pos.long()), (q, k, pos[0]), (q.transpose(0, 1), k, pos), (q[:, :, ::2], k, pos)):
        with pytest.raises(ValueError):
            B.pp_rope_qk_axes(plan, *args, s)
    for sections in ((8, 12), (8, 12, 13), (), (8, 8, 8, 4, 4), (40, -8, 0)):
        with pytest.raises(ValueError):
            B.pp_rope_qk_axes(plan, q, k, pos[:len(sections)], sections)
    for base in (1.0, 0.0, -3.0, float("nan"), 1e13):
        with pytest.raises(B.PPError):
            B.pp_rope_qk_axes(plan, q, k, pos, s, base)
    odd = torch.zeros(T, 4 * 64 + 4, dtype=torch.bfloat16, device="cuda")[:, :256].unflatten(1, (4, 64))
    with pytest.raises(B.PPError) as e:        # tokens that do not start at 16 bytes
        B.pp_rope_qk_axes(plan, odd, k, pos, s)
    assert e.value.code == -4
    for start, grid in ((pos[0, :2], pos[:, :2]), (pos[0, :2].float(), pos[:2, :3].contiguous()), (pos[0, :2].cpu(), pos[:2, :3].contiguous())):
        with pytest.raises(ValueError):
            B.pp_position_ids_axes(plan, start, grid)
    with pytest.raises(ValueError):
        B.pp_position_ids_axes(plan, pos[0, :0], pos[:0, :3].contiguous(), out=pos[:2])
