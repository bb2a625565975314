"""GPU: groups quantized into pages and read back, bit by bit against the definition; keys with error feedback against the
quantizer of contiguous caches, whose bytes they are, and what is read back against its dequantizer."""
import math

import pytest
import torch

import paper_2503_24358_b200 as sq
from paged import D, META, deq_pool, gen, normal, unpack

pytestmark = pytest.mark.gpu


def contiguous(s, k, v, bits, G, meta):
    """Cache of one sequence as the existing entry points write it: [1, H, T, ...] each."""
    T, H, _ = k.shape
    e = lambda *shape, dtype=META[meta]: torch.empty((1, H, *shape), dtype=dtype, device="cuda")  # noqa: E731
    row = D * bits // 8
    out = [e(T, row, dtype=torch.uint8), e(T // G, D), e(T // G, D), e(T, row, dtype=torch.uint8), e(T, D // G), e(T, D // G)]
    sq.squat_quantize_keys(s, k.transpose(0, 1).unsqueeze(0), bits, G, *out[:3])
    sq.squat_quantize_values(v.transpose(0, 1).unsqueeze(0), bits, G, *out[3:])
    return out


def at_slots(tensors, slots, P, G):
    """The pool's tensors at the slots, as [1, H, T, ...]."""
    page, off = slots.long() // P, slots.long() % P
    tok = off.unsqueeze(1) + torch.arange(G, device="cuda")
    rows = lambda t: t[page.unsqueeze(1), :, tok].flatten(0, 1).transpose(0, 1).unsqueeze(0)  # noqa: E731
    grids = lambda t: t[page, :, off // G].transpose(0, 1).unsqueeze(0)  # noqa: E731
    kc, ks, kz, vc, vs, vz = tensors
    return [rows(kc), grids(ks), grids(kz), rows(vc), rows(vs), rows(vz)]


def inputs(seed, T, H, dtype, kind="normal"):
    g = gen(seed)
    k, v = normal(g, T, H, D), normal(g, T, H, D)
    if kind == "ties":                                        # values on a coarse grid: many lie on a border exactly
        k, v = (torch.randint(-6, 7, (T, H, D), generator=g, device="cuda").float() / 2 for _ in range(2))
    if kind == "wide":
        k, v = k * torch.exp(8 * normal(g, T, H, D)), v * torch.exp(8 * normal(g, T, H, D))
    return k.to(dtype), v.to(dtype), g


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("meta", ["f32", "f16"])
@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("G, pages_of, groups, H", [(32, 1, 1, 1), (32, 3, 29, 8), (64, 2, 9, 3), (128, 1, 7, 8)])
@pytest.mark.parametrize("kind", ["normal", "ties", "wide"])
def test_write_and_read_back(dtype, meta, bits, G, pages_of, groups, H, kind):
    if kind == "wide" and meta == "f16":
        kind = "normal"                                       # ranges beyond binary16 have a test of their own
    P, T = G * pages_of, G * groups
    k, v, g = inputs(T + bits, T, H, dtype, kind)
    n_pages = -(-groups // pages_of) + 2
    slots = (torch.randperm(n_pages * pages_of, generator=g, device="cuda")[:groups] * G).to(torch.int32)
    pool = sq.PagePool.empty(n_pages, P, H, bits, G, meta_dtype=META[meta])
    before = [t.random_(0, 100).clone() if t.dtype == torch.uint8 else t.normal_().clone() for t in pool.tensors]
    sq.squat_get_device_status()
    sq.squat_pages_write(pool, slots, k, v)
    got = at_slots(pool.tensors, slots, P, G)
    # grids: the definition in float32, and within a bit of what the quantizers of contiguous caches store
    L, stored = 2 ** bits - 1, META[meta]
    want = contiguous(sq.Subspace(H), k, v, bits, G, meta)
    for x, dim, scale, zero, other in ((k.float().unflatten(0, (-1, G)), 1, got[1], got[2], want[1:3]), (v.float().unflatten(2, (-1, G)), 3, got[4], got[5], want[4:])):
        lo, hi = x.amin(dim), x.amax(dim)
        mine = ((hi - lo) * torch.tensor(1.0 / L, dtype=torch.float32, device="cuda")).to(stored)
        assert torch.equal(scale[0].transpose(0, 1), mine) and torch.equal(zero[0].transpose(0, 1), lo.to(stored))
        assert torch.equal(zero, other[1]) and bool(((scale - other[0]).abs() <= torch.finfo(stored).eps * other[0]).all())
    want = [t.contiguous() for t in got]
    # nothing else was written
    untouched = torch.ones(n_pages * pages_of, dtype=torch.bool, device="cuda")
    untouched[slots.long() // G] = False
    for t, b in zip(pool.tensors, before):
        per = t.shape[2] // pages_of
        a, b = (x.unflatten(2, (pages_of, per)).transpose(1, 2).flatten(0, 1)[untouched] for x in (t, b))
        assert torch.equal(a, b)
    for out_dtype in (torch.float32, torch.bfloat16):
        k_out, v_out = (torch.empty((T, H, D), dtype=out_dtype, device="cuda") for _ in range(2))
        sq.squat_pages_read(pool, slots, k_out, v_out)
        for kind_code, out, part in ((sq.SQUAT_KEYS, k_out, want[:3]), (sq.SQUAT_VALUES, v_out, want[3:])):
            ref = torch.empty((1, H, T, D), dtype=out_dtype, device="cuda")
            sq.squat_dequantize(kind_code, *part, 1, H, T, D, bits, G, ref)
            assert torch.equal(out, ref[0].transpose(0, 1))
    # codes: values to the last operation in float32, keys as real arithmetic on the stored grid
    dk, dv = deq_pool(pool.tensors, bits, G)
    page, tok = slots.long() // P, (slots.long() % P).unsqueeze(1) + torch.arange(G, device="cuda")
    for x, d, exact in ((k, dk, True), (v, dv, False)):
        code, scale, zero = (d[n][page.unsqueeze(1), :, tok].flatten(0, 1) for n in ("code", "scale", "zero"))
        t = (x.double() - zero) / scale if exact else ((x.float() - zero.float()) / scale.float()).double()
        assert torch.equal(code, torch.where(scale > 0, torch.round(t).clamp(0, L), 0.0))
    assert sq.squat_get_device_status() & ~sq.FLAG_ZERO_RANGE == 0


@pytest.mark.parametrize("build", ["rank 8", "dense", "block 32"])
@pytest.mark.parametrize("meta", ["f32", "f16"])
def test_keys_with_error_feedback(build, meta):
    H, G, bits, groups = 4, 32, 2, 21
    k, v, g = inputs(3, G * groups, H, torch.bfloat16)
    s = sq.Subspace(H)
    q = (normal(g, 2 * H, 300, 16) @ normal(g, 2 * H, 16, D)).to(torch.bfloat16)
    sq.squat_build_subspace(s, q, 8 if build == "rank 8" else 32, 1e-3, 32 if build == "block 32" else 1)
    pool = sq.PagePool.empty(13, 64, H, bits, G, meta_dtype=META[meta])
    slots = (torch.randperm(26, generator=g, device="cuda")[:groups] * G).to(torch.int32)
    ws = torch.empty(sq.squat_pages_write_workspace_bytes(pool, G * groups), dtype=torch.uint8, device="cuda")
    sq.squat_pages_write(pool, slots, k, v, s, ws)
    want = contiguous(s, k, v, bits, G, meta)
    got = at_slots(pool.tensors, slots, 64, G)
    for i in (0, 1, 2, 5):                                    # keys, and the values' zero-points
        assert torch.equal(got[i], want[i])
    plain = sq.PagePool.empty(13, 64, H, bits, G, meta_dtype=META[meta])
    sq.squat_pages_write(plain, slots, v=v)
    assert all(torch.equal(a, b) for a, b in zip(pool.tensors[3:], plain.tensors[3:]))


def test_padding_places_outside_the_pool_and_one_side_only():
    H, G, bits = 2, 32, 2
    k, v, g = inputs(1, 5 * G, H, torch.float32)
    pool = sq.PagePool.empty(3, 64, H, bits, G)
    good = torch.tensor([64, 128, 0], dtype=torch.int32, device="cuda")
    bad = torch.tensor([64, -1, 128, 192, 0], dtype=torch.int32, device="cuda")      # 192 is behind the last page
    sq.squat_get_device_status()
    rows = torch.cat([torch.arange(a * G, a * G + G) for a in (0, 2, 4)]).cuda()
    sq.squat_pages_write(pool, good, k[rows], v[rows])
    want = [t.clone() for t in pool.tensors]
    assert sq.squat_get_device_status() == 0
    for t in pool.tensors:
        t.zero_()
    sq.squat_pages_write(pool, bad, k, v)
    assert sq.squat_get_device_status() == sq.FLAG_PAGES
    assert all(torch.equal(a, b) for a, b in zip(pool.tensors, want))
    out = torch.full((5 * G, H, D), 7.0, device="cuda")
    ref = torch.empty((3 * G, H, D), device="cuda")
    sq.squat_pages_read(pool, bad, v_out=out)
    sq.squat_pages_read(pool, good, v_out=ref)
    assert sq.squat_get_device_status() == sq.FLAG_PAGES
    assert torch.equal(out[rows], ref) and bool((out[G:2 * G] == 7).all()) and bool((out[3 * G:4 * G] == 7).all())
    # an offset inside a group, and only one side
    sq.squat_pages_write(pool, torch.tensor([33], dtype=torch.int32, device="cuda"), k[:G])
    assert sq.squat_get_device_status() == sq.FLAG_PAGES and all(torch.equal(a, b) for a, b in zip(pool.tensors, want))
    sq.squat_pages_write(pool, good[:1], k=2 * k[:G])
    assert not torch.equal(pool.k_scales, want[1]) and all(torch.equal(a, b) for a, b in zip(pool.tensors[3:], want[3:]))
    sq.squat_pages_write(pool, good[:0], k[:0], v[:0])


@pytest.mark.parametrize("meta", ["f32", "f16"])
def test_constant_and_not_finite_groups(meta):
    H, G, bits = 1, 32, 2
    k, v, _ = inputs(2, G, H, torch.float32)
    k[:, 0, 3] = 1.5
    v[4, 0, :32] = -2.0
    pool = sq.PagePool.empty(1, 32, H, bits, G, meta_dtype=META[meta])
    slot = torch.zeros(1, dtype=torch.int32, device="cuda")
    sq.squat_get_device_status()
    sq.squat_pages_write(pool, slot, k, v)
    assert sq.squat_get_device_status() == sq.FLAG_ZERO_RANGE
    out = torch.empty_like(k), torch.empty_like(v)
    sq.squat_pages_read(pool, slot, *out)
    assert bool((out[0][:, 0, 3] == 1.5).all()) and bool((out[1][4, 0, :32] == -2).all())
    k[7, 0, 3], v[4, 0, 9] = float("nan"), float("inf")
    sq.squat_pages_write(pool, slot, k, v)
    assert sq.squat_get_device_status() & sq.FLAG_NONFINITE
    again = torch.empty_like(k), torch.empty_like(v)
    sq.squat_pages_read(pool, slot, *again)
    keep = torch.arange(D, device="cuda") != 3
    assert torch.equal(again[0][..., keep], out[0][..., keep])                       # the trouble stays in its group
    assert torch.equal(again[1][:4], out[1][:4]) and torch.equal(again[1][4, 0, 32:], out[1][4, 0, 32:])


def test_strided_pages_far_offsets_and_strided_rows():
    """Pages of two layers side by side, and token indexes whose bytes pass 32 bits; keys and values out of a fused projection."""
    H, G, bits, P = 2, 128, 2, 128
    g = gen(4)
    qkv = normal(g, 2 * G, 8 + 2 * H, D).to(torch.bfloat16)
    k, v = qkv[:, 8:8 + H], qkv[:, 8 + H:]
    far = (1 << 27) + 2 * H * P                                # tokens between pages: 4 GB of codes
    shapes = ((P, D * bits // 8, torch.uint8), (1, D, torch.float16), (1, D, torch.float16))
    t = []
    for rows, row, dtype in (*shapes, (P, D * bits // 8, torch.uint8), (P, 1, torch.float16), (P, 1, torch.float16)):
        per = rows * row // P if rows == P else row / G
        flat = torch.empty(int((far + 2 * H * P) * per), dtype=dtype, device="cuda")
        t.append([torch.as_strided(flat, (2, H, rows, row), (int(far * per), int(P * per), row, 1), int(layer * H * P * per)) for layer in (0, 1)])
    pool = sq.PagePool(*(x[1] for x in t))
    dense = sq.PagePool.empty(2, P, H, bits, G, meta_dtype=torch.float16)
    slots = torch.tensor([P, 0], dtype=torch.int32, device="cuda")
    for x in t:
        x[0].zero_()
    sq.squat_pages_write(pool, slots, k, v)
    sq.squat_pages_write(dense, slots, k.contiguous(), v.contiguous())
    for a, b, other in zip(pool.tensors, dense.tensors, (x[0] for x in t)):
        assert torch.equal(a, b) and not other.any()
    out = torch.zeros((2 * G, 8 + 2 * H, D), dtype=torch.bfloat16, device="cuda")
    ref = torch.empty((2, 2 * G, H, D), dtype=torch.bfloat16, device="cuda")
    sq.squat_pages_read(pool, slots, out[:, 8:8 + H], out[:, 8 + H:])
    sq.squat_pages_read(dense, slots, ref[0], ref[1])
    assert torch.equal(out[:, 8:8 + H], ref[0]) and torch.equal(out[:, 8 + H:], ref[1]) and not out[:, :8].any()


def test_graph_replay_with_other_places():
    H, G = 2, 32
    k, v, _ = inputs(6, 2 * G, H, torch.bfloat16)
    pool = sq.PagePool.empty(4, 64, H, 4, G)
    slots = torch.tensor([0, 32], dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        sq.squat_pages_write(pool, slots, k, v)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    out = torch.empty_like(k), torch.empty_like(v)
    with torch.cuda.graph(graph):
        sq.squat_pages_write(pool, slots, k, v)
        sq.squat_pages_read(pool, slots, *out)
    first = [t.clone() for t in pool.tensors]
    slots.copy_(torch.tensor([192, 64], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    for t, f in zip(at_slots(pool.tensors, slots, 64, G), at_slots(first, torch.tensor([0, 32], device="cuda"), 64, G)):
        assert torch.equal(t, f)
    ref = torch.empty_like(k), torch.empty_like(v)
    sq.squat_pages_read(pool, torch.tensor([0, 32], dtype=torch.int32, device="cuda"), *ref)
    assert torch.equal(out[0], ref[0]) and torch.equal(out[1], ref[1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_error_feedback_from_a_shared_projection_in_a_graph(dtype):
    H, G, bits, groups = 2, 32, 2, 6
    g = gen(11)
    projection = normal(g, groups * G, 4 * H, D).to(dtype)     # queries of two heads each, keys, values
    k, v = projection[:, 2 * H:3 * H], projection[:, 3 * H:]
    s = sq.Subspace(H)
    sq.squat_build_subspace(s, normal(g, 2 * H, 300, D).to(torch.bfloat16), 8, 1e-3, 1)
    pool = sq.PagePool.empty(5, 64, H, bits, G)
    blank = [t.zero_() for t in pool.tensors]
    slots = torch.tensor([64, -1, 0, 288, 128, 32], dtype=torch.int32, device="cuda")
    ws = torch.empty(sq.squat_pages_write_workspace_bytes(pool, groups * G), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sq.squat_pages_write(pool, slots, k, v, s, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sq.squat_pages_write(pool, slots, k, v, s, ws)
    for t in blank:
        t.zero_()
    projection.copy_(normal(g, groups * G, 4 * H, D).to(dtype))
    slots.copy_(torch.tensor([256, 32, -1, 96, 160, 0], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    written = [0, 1, 3, 4, 5]
    got = at_slots(pool.tensors, slots[written], 64, G)
    rows = torch.tensor(written, device="cuda").repeat_interleave(G) * G + torch.arange(G, device="cuda").repeat(len(written))
    want = contiguous(s, k[rows].contiguous(), v[rows].contiguous(), bits, G, "f32")
    for i in (0, 1, 2, 5):                                    # keys, and the values' zero-points
        assert torch.equal(got[i], want[i])
    free = torch.ones(5, 2, dtype=torch.bool, device="cuda")
    free[slots[written].long() // 64, slots[written].long() % 64 // G] = False
    assert not any(pool.tensors[i].unflatten(2, (2, -1)).transpose(1, 2)[free].any() for i in (0, 3))


def odd_group(x, kind):
    """A group [n] whose grid is no ordinary one."""
    y = x.clone()
    if kind == "constant":
        y[:] = 1.5
    elif kind == "zero":
        y[:] = 0.0
    elif kind in ("nan", "inf", "-inf"):
        y[len(y) // 3] = float(kind)
    elif kind == "infinite range":
        y[0], y[1] = 3e38, -3e38
    else:
        y *= {"subnormal scale": 3e-39, "tiny scale": 1e-32, "huge scale": 1e33}[kind]
    return y


KINDS = ["constant", "zero", "nan", "inf", "-inf", "infinite range", "subnormal scale", "tiny scale", "huge scale"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("meta", ["f32", "f16"])
@pytest.mark.parametrize("bits, G", [(2, 32), (4, 32), (2, 64), (4, 128)])
def test_odd_groups_leave_their_neighbours_alone(kind, dtype, meta, bits, G):
    """Codes, grids and flags of groups with a constant or not finite channel (token), or one whose scale is far from 1: every
    code by the definition, in float64 (values in float32) on the stored grid, of the odd groups and of those beside them."""
    H, L = 2, 2 ** bits - 1
    k, v, _ = inputs(bits + G, G, H, torch.float32)
    for j in range(8):                                        # one at every place of an octet, then two, then all eight
        k[:, 0, 8 * j + j] = odd_group(k[:, 0, 8 * j + j], kind)
        for c in (8 * (8 + j) + j, 8 * (8 + j) + (j + 3) % 8):
            k[:, 0, c] = odd_group(k[:, 0, c], kind)
    for c in range(40, 48):
        k[:, 1, c] = odd_group(k[:, 1, c], kind)
    for t in range(0, G, 3):
        a = t // 3 % (D // G) * G
        v[t, t % H, a:a + G] = odd_group(v[t, t % H, a:a + G], kind)
    k, v = k.to(dtype), v.to(dtype)
    pool = sq.PagePool.empty(1, G, H, bits, G, meta_dtype=META[meta])
    sq.squat_get_device_status()
    sq.squat_pages_write(pool, torch.zeros(1, dtype=torch.int32, device="cuda"), k, v)
    flags = sq.squat_get_device_status()
    dk, dv = deq_pool(pool.tensors, bits, G)
    for x, d, dim, exact in ((k, dk, 0, True), (v, dv, 2, False)):
        code, scale, zero = (d[n][0].transpose(0, 1) for n in ("code", "scale", "zero"))                    # [G, H, D]
        groups = x.float().unflatten(dim, (-1, G)) if dim else x.float().unsqueeze(0)
        over = 3 if dim == 2 else 1
        lo, hi = groups.amin(over, keepdim=True), groups.amax(over, keepdim=True)
        for stored, grid in ((scale, (hi - lo) * torch.tensor(1.0 / L, dtype=torch.float32, device="cuda")), (zero, lo)):
            grid = grid.to(META[meta]).expand_as(groups)
            torch.testing.assert_close(stored, (grid.flatten(2, 3) if dim == 2 else grid[0]).double(), rtol=0, atol=0, equal_nan=True)
        t = (x.double() - zero) / scale if exact else ((x.float() - zero.float()) / scale.float()).double()
        ok = (scale > 0) & (scale < math.inf)
        assert torch.equal(code, torch.where(ok, torch.round(t).clamp(0, L), 0.0))
    want_flags = {"constant": sq.FLAG_ZERO_RANGE, "zero": sq.FLAG_ZERO_RANGE, "nan": sq.FLAG_NONFINITE, "inf": sq.FLAG_NONFINITE, "-inf": sq.FLAG_NONFINITE, "infinite range": sq.FLAG_NONFINITE}
    if meta == "f32":
        assert flags == want_flags.get(kind, 0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_keys_and_values_read_into_one_tensor(dtype):
    """k_out and v_out may lie between each other's rows, but share none: refused exactly where two rows meet, else read in full."""
    H, G = 3, 32
    k, v, _ = inputs(8, G, H, torch.float32)
    pool = sq.PagePool.empty(1, G, H, 2, G)
    slots = torch.zeros(1, dtype=torch.int32, device="cuda")
    sq.squat_pages_write(pool, slots, k, v)
    ref = torch.empty((2, G, H, D), dtype=dtype, device="cuda")
    sq.squat_pages_read(pool, slots, *ref)
    found = {True: 0, False: 0}
    for kt, kh in ((H * D, D), (2 * H * D, D), (2 * H * D, 2 * D), (D, G * D), (2 * D, 2 * G * D), (D + 8, G * (D + 8))):
        span = (G - 1) * kt + (H - 1) * kh + D
        rows = torch.tensor([t * kt + h * kh for t in range(G) for h in range(H)])
        for at in [x * D for x in range(-2 * H * G, 2 * H * G + 1, 5)] + [D, -D, H * D, 8, -8, D - 8, D + 8, -D - 8, span, -span, span - 8, 8 - span]:
            flat = torch.zeros(2 * span + abs(at), dtype=dtype, device="cuda")
            a, b = (torch.as_strided(flat, (G, H, D), (kt, kh, 1), max(0, x)) for x in (-at, at))
            meet = bool(((rows.unsqueeze(1) - rows - at).abs() < D).any())
            found[meet] += 1
            if meet:
                with pytest.raises(sq.SquatError):
                    sq.squat_pages_read(pool, slots, a, b)
                assert not flat.any()
            else:
                sq.squat_pages_read(pool, slots, a, b)
                assert torch.equal(a, ref[0]) and torch.equal(b, ref[1])
    assert min(found.values()) > 100, found


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bits, G", [(2, 32), (4, 64), (4, 128)])
@pytest.mark.parametrize("kind", ["normal", "ties", "wide"])
def test_codes_beside_those_of_a_contiguous_cache(dtype, bits, G, kind):
    """Scales that differ in the last bit (2^-23 of themselves) move a border by at most L 2^-23 steps, and the float32 difference and
    quotient of values round by 2^-24 of L steps each: codes differ by one, and only next to a border, where either level is as near."""
    H, L, T = 3, 2 ** bits - 1, 5 * G
    k, v, _ = inputs(T + bits, T, H, dtype, kind)
    pool = sq.PagePool.empty(5, G, H, bits, G)
    sq.squat_pages_write(pool, G * torch.arange(5, dtype=torch.int32, device="cuda"), k, v)
    other = contiguous(sq.Subspace(H), k, v, bits, G, "f32")
    dk, dv = deq_pool(pool.tensors, bits, G)
    for x, d, codes in ((k, dk, other[0]), (v, dv, other[3])):
        code, scale, zero = (d[n].transpose(1, 2).flatten(0, 1) for n in ("code", "scale", "zero"))
        theirs = unpack(codes[0].transpose(0, 1), bits)
        apart = (code - theirs).abs()
        border = (torch.maximum(code, theirs) - 0.5 - (x.double() - zero) / scale).abs()
        assert bool(((apart == 0) | ((apart == 1) & (border <= L * 2.0 ** -22))).all())
        print(kind, "codes that differ:", int((apart != 0).sum()), "of", apart.numel())
