"""GPU: the rotary embedding with several axes (squat_rope_apply) against float64.

Tolerance.  The angle's rest is exact to 2^-32 turns and rounded to a float (24 bits) of half turns: at most pi 2^-25 radians.  The sine
and cosine are good to one unit in the last place (2^-24 at most, below 1).  So either is off by less than 3 * 2^-24, the two
products and the sum round once each (2^-24), and a result by less than 6 * 2^-24 (|a| + |b|); bf16 rounds it by 2^-8 of itself."""
import pytest
import torch

import paper_2503_24358_b200 as sq
from paged import D, gen, normal

pytestmark = pytest.mark.gpu


def reference(x, positions, sections, base, inverse):
    n = sum(sections)
    axis = [a for a, m in enumerate(sections) for _ in range(m)]
    y = x.double().clone()
    for i in range(n):
        angle = positions[axis[i]].double() * base ** (-i / n) * (-1 if inverse else 1)
        c, s = torch.cos(angle).unsqueeze(1), torch.sin(angle).unsqueeze(1)
        a, b = x[..., i].double(), x[..., n + i].double()
        y[..., i], y[..., n + i] = a * c - b * s, b * c + a * s
    mag = x.double().abs()
    mag = torch.cat((mag[..., :n] + mag[..., n:2 * n],) * 2 + (0 * mag[..., 2 * n:],), -1)
    return y, mag


def check(y, x, positions, sections, base=10000.0, inverse=False):
    ref, mag = reference(x, positions, sections, base, inverse)
    tol = 6 * 2.0 ** -24 * mag + (2.0 ** -8 * ref.abs() if y.dtype == torch.bfloat16 else 0) + 1e-30
    assert ((y.double() - ref).abs() <= tol).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sections", [(64,), (16, 24, 24), (32, 32), (8, 12, 12), (8, 0, 0, 16), (8,)])
@pytest.mark.parametrize("tokens, heads", [(1, (8, 8)), (33, (32, 8)), (1003, (3, 1))])
def test_queries_and_keys(dtype, sections, tokens, heads):
    g = gen(tokens)
    plan = sq.RopePlan(sections)
    q, k = (normal(g, tokens, h, D).to(dtype) for h in heads)
    pos = torch.randint(0, 1 << 20, (len(sections), tokens), generator=g, device="cuda", dtype=torch.int32)
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    sq.squat_rope_apply(plan, pos, q, k, q_out, k_out)
    check(q_out, q, pos, sections)
    check(k_out, k, pos, sections)
    assert torch.equal(q_out[..., 2 * sum(sections):], q[..., 2 * sum(sections):])
    # the inverse is the gradient: it turns the result back
    sq.squat_rope_apply(plan, pos.long(), q, k, q_out, k_out, inverse=True)
    check(q_out, q, pos, sections, inverse=True)
    check(k_out, k, pos, sections, inverse=True)


def test_in_place_strided_one_side_and_int64():
    g = gen(5)
    plan = sq.RopePlan((16, 24, 24), base=1e6)
    qkv = normal(g, 77, 32 + 16, D).to(torch.bfloat16)
    q, k, rest = qkv[:, :32], qkv[:, 32:40], qkv[:, 40:].clone()
    q0, k0 = q.clone(), k.clone()
    wide = torch.randint(-5000, 1 << 30, (6, 100), generator=g, device="cuda")
    pos = wide[::2, 10:87]
    sq.squat_rope_apply(plan, pos, q, k)
    check(q, q0, pos, (16, 24, 24), 1e6)
    check(k, k0, pos, (16, 24, 24), 1e6)
    assert torch.equal(qkv[:, 40:], rest)
    k1 = k.clone()
    sq.squat_rope_apply(plan, pos, k=k, inverse=True)
    check(k, k1, pos, (16, 24, 24), 1e6, True)
    assert ((k.double() - k0.double()).abs() <= 2.0 ** -8 * 3 * (k0.double().abs() + k0.double().roll(64, -1).abs())).all()
    by_head = torch.empty((9, 77, D), device="cuda").transpose(0, 1)          # [tokens, heads, d] of a [heads, tokens, d] buffer
    x = normal(g, 77, 9, D)
    sq.squat_rope_apply(plan, pos, x, q_out=by_head)
    check(by_head, x, pos, (16, 24, 24), 1e6)


def test_far_positions_keep_their_angle():
    """Positions up to 2^62: the rest of the angle is what integer arithmetic on the plan's own fractions says."""
    plan = sq.RopePlan((64,))
    pos = torch.tensor([0, 1, -1, 2 ** 31 + 5, 2 ** 40 + 123, 2 ** 62 - 7], dtype=torch.int64, device="cuda")
    x = torch.zeros(6, 1, D, device="cuda")
    x[..., :64] = 1.0
    y = torch.empty_like(x)
    sq.squat_rope_apply(plan, pos, x, q_out=y)
    for i in (0, 1, 17, 63):
        turns = [((p * plan._plan.turn[i] + 2 ** 63) % 2 ** 64 - 2 ** 63) / 2 ** 64 for p in pos.tolist()]
        a = torch.tensor(turns, dtype=torch.float64, device="cuda") * (2 * torch.pi)
        assert ((y[:, 0, i].double() - a.cos()).abs() <= 6 * 2.0 ** -24).all() and ((y[:, 0, 64 + i].double() - a.sin()).abs() <= 6 * 2.0 ** -24).all()


def test_plan_angles_are_the_tables():
    """One axis of 64 pairs is the embedding of the reader for keys stored before it."""
    import math
    plan = sq.RopePlan((64,))
    t = sq.squat_rope_table(64)
    for i in range(64):
        a = plan._plan.turn[i] / 2 ** 64 * 2 * math.pi
        assert abs(float(t[((2 + 5) * 64 + i) * 2]) - math.cos(5 * a)) < 1e-7 and abs(float(t[((2 + 5) * 64 + i) * 2 + 1]) - math.sin(5 * a)) < 1e-7


def test_graph_replay_reads_new_positions():
    g = gen(8)
    plan = sq.RopePlan((32, 32))
    q, pos = normal(g, 40, 4, D), torch.zeros((2, 40), dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        sq.squat_rope_apply(plan, pos, q, q_out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sq.squat_rope_apply(plan, pos, q, q_out=out)
    pos.copy_(torch.randint(0, 9999, (2, 40), generator=g, device="cuda"))
    graph.replay()
    check(out, q, pos, (32, 32))
