"""CPU-only: what the entry points of the paged cache, its attention and the rotary embedding refuse.  Every call ends at the
library's own argument checks, before anything touches a GPU; addresses are checked, never read."""
import ctypes
import math

import pytest
import torch

import paper_2503_24358_b200 as sq
from paper_2503_24358_b200 import build as sq_build

A, MISALIGNED = 4096, 4100
OK, INVALID, SHAPE, UNSUPPORTED = 0, 1, 2, 3


@pytest.fixture(scope="module", autouse=True)
def lib():
    sq_build.build()
    return sq.binding._load()


def pool(**kw):
    p = dict(k_codes=A, k_scales=A, k_zeros=A, v_codes=A, v_scales=A, v_zeros=A, page_stride=8 * 64, head_stride=64, n_pages=4, page_tokens=64,
             n_kv_heads=8, head_dim=128, bits=2, group_size=32, meta16=0)
    p.update(kw)
    return sq.PagePool._Struct(*[p[n] for n, _ in sq.PagePool._Struct._fields_])


BAD_POOLS = [(dict(n_pages=-1), INVALID), (dict(page_tokens=0), INVALID), (dict(n_kv_heads=0), INVALID), (dict(meta16=2), INVALID), (dict(page_stride=-64), INVALID),
             (dict(head_dim=64), UNSUPPORTED), (dict(bits=3), UNSUPPORTED), (dict(bits=8), UNSUPPORTED), (dict(group_size=48), UNSUPPORTED), (dict(page_tokens=48), SHAPE),
             (dict(page_tokens=96, group_size=64), SHAPE), (dict(head_stride=72), SHAPE), (dict(page_stride=8 * 64 + 8), SHAPE), (dict(head_stride=32), INVALID),
             (dict(page_stride=32), INVALID), (dict(n_pages=1 << 26, page_tokens=64), UNSUPPORTED), (dict(k_codes=None), INVALID), (dict(v_zeros=None), INVALID),
             (dict(k_scales=MISALIGNED), INVALID), (dict(v_codes=MISALIGNED), INVALID), (dict(n_kv_heads=70000), UNSUPPORTED)]


def write(lib, p=None, s=None, slots=A, T=64, dtype=1, k=A, kt=1024, kh=128, v=A, vt=1024, vh=128, ws=None, ws_bytes=0):
    p = pool() if p is None else p
    return lib.squat_pages_write(s, ctypes.addressof(p), slots, T, dtype, k, kt, kh, v, vt, vh, ws, ws_bytes, None)


def read(lib, p=None, slots=A, T=64, dtype=1, k=A, kt=1024, kh=128, v=A, vt=1024, vh=128):
    p = pool() if p is None else p
    return lib.squat_pages_read(ctypes.addressof(p), slots, T, dtype, k, kt, kh, v, vt, vh, None)


def attend(lib, p=None, q=A, n_q=4, hq=32, qt=4096, qh=128, seqs=2, q_start=A, cached=A, table=A, width=3, kn=A, vn=A, n_new=5, knt=1024, knh=128, vnt=1024, vnh=128,
           starts=A, lens=A, max_q=2, causal=1, scale=0.0, out=A, ot=4096, oh=128, lse=None, ws=A, ws_bytes=1 << 40):
    p = pool() if p is None else p
    return lib.squat_chunk_attention(q, n_q, hq, qt, qh, ctypes.addressof(p), seqs, q_start, cached, table, width, kn, vn, n_new, knt, knh, vnt, vnh, starts, lens, max_q,
                                     causal, scale, out, ot, oh, lse, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [write, read, attend])
@pytest.mark.parametrize("kw, status", BAD_POOLS)
def test_pools(lib, call, kw, status):
    assert call(lib, pool(**kw)) == status


def test_no_pool(lib):
    assert lib.squat_pages_read(None, A, 64, 1, A, 1024, 128, A, 1024, 128, None) == INVALID
    assert lib.squat_pages_write_workspace_bytes(None, 64) == 0
    p = pool(bits=5)
    assert lib.squat_pages_write_workspace_bytes(ctypes.addressof(p), 64) == 0
    p = pool()
    assert lib.squat_pages_write_workspace_bytes(ctypes.addressof(p), 64) == 64 * 8 * 32 + 2 * 2 * 8 * 128 * 4


@pytest.mark.parametrize("call", [write, read])
@pytest.mark.parametrize("kw, status", [
    (dict(T=48), SHAPE), (dict(T=-32), INVALID), (dict(dtype=2), INVALID), (dict(slots=None), INVALID), (dict(slots=A + 2), INVALID), (dict(k=MISALIGNED), INVALID),
    (dict(v=MISALIGNED), INVALID), (dict(kt=1025), INVALID), (dict(vh=-128), INVALID), (dict(dtype=0, kt=1026), INVALID), (dict(T=0), OK), (dict(k=None, v=None), OK)])
def test_rows(lib, call, kw, status):
    assert call(lib, **kw) == status


def test_rows_that_are_written_lie_apart(lib):
    assert read(lib, kt=0) == INVALID and read(lib, vh=64) == INVALID


@pytest.mark.parametrize("kw, status", [
    (dict(n_q=-1), INVALID), (dict(hq=0), INVALID), (dict(hq=12), SHAPE), (dict(seqs=-1), INVALID), (dict(width=-1), INVALID), (dict(n_new=-1), INVALID),
    (dict(max_q=-1), INVALID), (dict(causal=2), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=math.inf), INVALID), (dict(scale=math.nan), INVALID),
    (dict(q=None), INVALID), (dict(q=MISALIGNED), INVALID), (dict(qt=4100), INVALID), (dict(out=None), INVALID), (dict(out=MISALIGNED), INVALID), (dict(ot=64), INVALID),
    (dict(oh=0), INVALID), (dict(q_start=None), INVALID), (dict(q_start=A + 1), INVALID), (dict(cached=None), INVALID), (dict(table=None), INVALID), (dict(table=A + 2), INVALID),
    (dict(kn=None), INVALID), (dict(vn=None), INVALID), (dict(starts=None), INVALID), (dict(lens=None), INVALID), (dict(lens=A + 3), INVALID), (dict(knt=1028), INVALID),
    (dict(vnh=-8), INVALID), (dict(kn=MISALIGNED), INVALID), (dict(lse=A + 2), INVALID), (dict(ws=None), INVALID), (dict(ws=A + 16), INVALID), (dict(ws_bytes=1024), INVALID),
    (dict(n_q=1 << 27), UNSUPPORTED), (dict(n_q=0), OK), (dict(seqs=0), OK)])
def test_attention(lib, kw, status):
    assert attend(lib, **kw) == status


def test_workspace_sizes(lib):
    f = sq.squat_chunk_attention_workspace_bytes
    assert f(4, 32, 8, 2) > 0 and f(4, 32, 8, 2) % 256 == 0
    assert f(-1, 32, 8, 2) == f(4, 0, 8, 2) == f(4, 32, 0, 2) == f(4, 30, 8, 2) == f(4, 32, 8, -1) == 0


def test_rope_plans():
    for sections in ((64,), (16, 24, 24), (8, 0, 8), (8, 8, 8, 8)):
        p = sq.RopePlan(sections)
        assert p._plan.n_pairs == sum(sections) and p._plan.n_axes == len(sections)
        n = sum(sections)
        for i in range(n):
            assert abs(p._plan.turn[i] / 2 ** 64 * 2 * math.pi - 10000.0 ** (-i / n)) <= 2.0 ** -50
            assert p._plan.axis[i] == next(a for a in range(len(sections)) if i < sum(sections[:a + 1]))
    for sections, status in (((63,), SHAPE), ((72,), SHAPE), ((0,), SHAPE), ((4,), SHAPE), ((-8, 16), INVALID), ((), INVALID), ((8,) * 5, INVALID)):
        with pytest.raises(sq.SquatError) as e:
            sq.RopePlan(sections)
        assert e.value.status == status
    for kw, status in ((dict(base=1.0), INVALID), (dict(base=math.inf), INVALID), (dict(base=math.nan), INVALID), (dict(head_dim=64), UNSUPPORTED)):
        with pytest.raises(sq.SquatError) as e:
            sq.RopePlan((32,), **kw)
        assert e.value.status == status


def rope(lib, plan=None, positions=A, p64=0, axis_stride=7, T=7, d=128, dtype=1, inverse=0, q=A, hq=4, qs=(512, 128), qo=2 * A, qos=(512, 128), k=A, hk=2, ks=(256, 128), ko=2 * A, kos=(256, 128)):
    plan = sq.RopePlan() if plan is None else plan
    return lib.squat_rope_apply(plan.address if plan else None, positions, p64, axis_stride, T, d, dtype, inverse, q, hq, *qs, qo, *qos, k, hk, *ks, ko, *kos, None)


@pytest.mark.parametrize("kw, status", [
    (dict(plan=False), INVALID), (dict(p64=2), INVALID), (dict(T=-1), INVALID), (dict(d=64), UNSUPPORTED), (dict(dtype=5), INVALID), (dict(inverse=3), INVALID), (dict(positions=None), INVALID),
    (dict(positions=A + 2), INVALID), (dict(positions=A + 4, p64=1), INVALID), (dict(axis_stride=-1), INVALID), (dict(q=None), INVALID), (dict(ko=None), INVALID), (dict(q=MISALIGNED), INVALID),
    (dict(qs=(516, 128)), INVALID), (dict(ks=(-256, 128)), INVALID), (dict(qos=(64, 128)), INVALID), (dict(kos=(256, 64)), INVALID), (dict(qo=A, qos=(1024, 128)), INVALID),
    (dict(T=0), OK), (dict(hq=0, hk=0), OK)])
def test_rope(lib, kw, status):
    assert rope(lib, **kw) == status


def test_rope_with_a_broken_plan(lib):
    p = sq.RopePlan((32, 32))
    p._plan.axis[40] = 2
    assert rope(lib, p) == INVALID
    p = sq.RopePlan((32,))
    p._plan.n_pairs = 65
    assert rope(lib, p) == INVALID


def _tensors(n=3, H=2, P=64, G=32, bits=2, meta=torch.float32):
    z = lambda *shape, dtype=meta: torch.zeros((n, H, *shape), dtype=dtype)  # noqa: E731
    row = 16 * bits
    return [z(P, row, dtype=torch.uint8), z(P // G, 128), z(P // G, 128), z(P, row, dtype=torch.uint8), z(P, 128 // G), z(P, 128 // G)]


def test_tensors_that_are_no_pool():
    """The binding checks shapes, types and strides before the library sees an address."""
    with pytest.raises(ValueError, match="CUDA"):
        sq.PagePool(*_tensors())
    for i, t in ((0, torch.int8), (3, torch.int32), (1, torch.float16), (4, torch.float64), (5, torch.float16)):
        x = _tensors()
        x[i] = x[i].to(t)
        with pytest.raises(ValueError):
            sq.PagePool(*x)
    for i in range(6):
        x = _tensors()
        x[i] = x[i][:, :, :-1]
        with pytest.raises(ValueError):
            sq.PagePool(*x)
        x = _tensors()
        x[i] = x[i].transpose(0, 1).contiguous().transpose(0, 1)           # strides of its own
        with pytest.raises(ValueError):
            sq.PagePool(*x)
        x = _tensors()
        x[i] = x[i].transpose(2, 3).contiguous().transpose(2, 3)
        with pytest.raises(ValueError):
            sq.PagePool(*x)
        x = _tensors()
        x[i] = x[i][0]
        with pytest.raises(ValueError):
            sq.PagePool(*x)


def test_binding_refuses_other_types_and_shapes():
    plan = sq.RopePlan()
    x = torch.zeros(4, 2, 128)
    with pytest.raises(TypeError):
        sq.squat_rope_apply(plan, torch.zeros(4), x)
    with pytest.raises(ValueError):
        sq.squat_rope_apply(plan, torch.zeros(2, 4, dtype=torch.int32), x)
    with pytest.raises(ValueError):
        sq.squat_rope_apply(plan, torch.zeros(4, dtype=torch.int32), x, x.bfloat16())
    with pytest.raises(ValueError):
        sq.squat_rope_apply(plan, torch.zeros(4, dtype=torch.int32), x, q_out=x[:3])
    with pytest.raises(ValueError):
        sq.squat_rope_apply(plan, torch.zeros(4, dtype=torch.int32), x.transpose(1, 2))


def test_places_that_overlap_across_dimensions(lib):
    # every stride holds a row (a page), but head 1 of token 0 (page 0) is head 0 of token 1
    assert read(lib, T=64, kt=128, kh=128) == INVALID
    assert attend(lib, n_q=4, ot=128, oh=128) == INVALID
    assert rope(lib, qos=(128, 128)) == INVALID
    p = pool(page_stride=64, head_stride=64)
    assert lib.squat_pages_write_workspace_bytes(ctypes.addressof(p), 64) == 0
    # either dimension may be the inner one
    assert lib.squat_pages_write_workspace_bytes(ctypes.addressof(pool(page_stride=64, head_stride=64 * pool().n_pages)), 64) > 0


def test_more_tokens_than_32_bits_count(lib):
    assert attend(lib, width=(1 << 31) // pool().page_tokens) == UNSUPPORTED
    assert attend(lib, n_new=(1 << 31) - 1) == UNSUPPORTED
    assert rope(lib, hq=(1 << 31) - 1) == UNSUPPORTED


class OnDevice(torch.Tensor):
    """Host memory that says it is on a CUDA device (device 0 unless `at` is set)."""
    at = 0
    is_cuda = property(lambda self: True)

    def get_device(self):
        return self.at


def _fake(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnDevice)


def _fake_calls():
    """The four calls and the tensors that each takes, all on device 0."""
    i32 = lambda *shape: _fake(*shape, dtype=torch.int32)  # noqa: E731
    pool = lambda: [t.as_subclass(OnDevice) for t in _tensors()]  # noqa: E731
    plan = sq.RopePlan()

    def rope(**t):
        sq.squat_rope_apply(plan, **t)

    def on_pool(call, **t):
        call(sq.PagePool(*(t.pop(f"pool{i}") for i in range(6))), **t)

    def attention(**t):
        p = sq.PagePool(*(t.pop(f"pool{i}") for i in range(6)))
        sq.squat_chunk_attention(pool=p, max_q=1, **t)

    pages = {f"pool{i}": t for i, t in enumerate(pool())}
    rows = {n: _fake(64, 2, 128) for n in ("k", "v")}
    yield rope, dict(positions=i32(1, 4), q=_fake(4, 2, 128), k=_fake(4, 2, 128), q_out=_fake(4, 2, 128), k_out=_fake(4, 2, 128))
    yield lambda **t: on_pool(sq.squat_pages_write, **t), dict(pages, slots=i32(2), workspace=_fake(4096, dtype=torch.uint8), **rows)
    yield lambda **t: on_pool(sq.squat_pages_read, **t), dict(pages, slots=i32(2), k_out=rows["k"], v_out=rows["v"])
    yield attention, dict(pages, q=_fake(3, 4, 128), q_start=i32(3), cached_len=i32(2), page_table=i32(2, 1), out=_fake(3, 4, 128), workspace=_fake(4096, dtype=torch.uint8),
                          k_new=_fake(5, 2, 128), v_new=_fake(5, 2, 128), new_start=i32(2), new_len=i32(2), lse=_fake(3, 4, dtype=torch.float32))


def test_tensors_of_another_device(monkeypatch):
    """Each of a call's tensors on another device than the current one, or on the host, is refused before the library sees an address."""
    seen = []

    class Calls:
        def __getattr__(self, name):
            return lambda *args: seen.append(name) or 0

    monkeypatch.setattr(sq.binding, "_direct", Calls)
    monkeypatch.setattr(sq.binding, "_stream", lambda stream: None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for i, (call, tensors) in enumerate(_fake_calls()):
        call(**tensors)
        assert len(seen) == i + 1
        for name, x in tensors.items():
            if name.startswith("pool") and name != "pool0":
                continue                                      # (the six have one device, which PagePool checks)
            for at in (1, -1):
                x.at = at
                with pytest.raises(ValueError, match="cuda:1" if at == 1 else "CUDA"):
                    call(**tensors)
            del x.at
        assert len(seen) == i + 1
    # an empty pool is nowhere
    call(**dict(tensors, **{f"pool{i}": t for i, t in enumerate(_tensors(n=0))}))
    assert len(seen) == i + 2


def test_keys_and_values_that_are_read_into_one_place(lib):
    row = 256                                                 # bytes of a bf16 row
    assert read(lib, k=A, v=A) == INVALID                     # the same rows
    assert read(lib, k=A, v=A + 7 * row) == INVALID           # one head on
    assert read(lib, k=A + 63 * 1024 * 2, v=A) == INVALID     # the last token on the first, from either side
    assert read(lib, k=A, v=A + 16) == INVALID                # a part of a row
    assert read(lib, k=A, kt=2048, v=A + 2048, vt=1024) == INVALID      # between each other's, with other strides
    assert read(lib, k=A, kt=2048, v=A + 2048 - 16, vt=2048) == INVALID


def test_workspaces_with_holes(monkeypatch):
    """What the kernels may write is the workspace's bytes in a row: views that have fewer, or others in between, are refused."""
    class Calls:
        def __getattr__(self, name):
            return lambda *args: pytest.fail("called")

    monkeypatch.setattr(sq.binding, "_direct", Calls)
    monkeypatch.setattr(sq.binding, "_stream", lambda stream: None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for call, tensors in _fake_calls():
        for bad in (_fake(1, dtype=torch.uint8).expand(4096), _fake(8192, dtype=torch.uint8)[::2]):
            if "workspace" in tensors:
                with pytest.raises(ValueError, match="contiguous"):
                    call(**dict(tensors, workspace=bad))
