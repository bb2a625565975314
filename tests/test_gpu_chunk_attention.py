"""GPU: attention of new tokens over pages (squat_chunk_attention) against float64.

Tolerances.  Element by element, paged.attention's bound: what binary16 operands may change (2^-11 of scale x code, of the zero-point and of
their sum, for keys through the scores' exponentials), the weights' own rounding, and 2^-8 of the result for its rounding to bf16;
where magnitudes send the kernel to bf16 operands, eight times the operands' part.  Over all elements the roundings are independent: a result's
last rounding has a root mean square of at most 2^-8 / sqrt(3) of it, operands add a fraction of that, so the relative
2-norm of the error stays below 2^-8."""
import math

import pytest
import torch

import paper_2503_24358_b200 as sq
from paged import D, META, Batch, gen, normal

pytestmark = pytest.mark.gpu


def call(b, lse=True, max_q=None, **kw):
    out = torch.full(b.q.shape, 9.0, dtype=torch.bfloat16, device="cuda")
    l = torch.full(b.q.shape[:2], 9.0, device="cuda") if lse else None
    mq = b.max_q if max_q is None else max_q
    ws = torch.empty(sq.squat_chunk_attention_workspace_bytes(b.q.shape[0], b.Hq, b.H, mq), dtype=torch.uint8, device="cuda")
    ws.fill_(255)                                              # NaN: nothing may be read that the call has not written
    sq.squat_chunk_attention(b.q, sq.PagePool(*b.tensors), b.q_start, b.cached, b.page_table, out, ws, mq, b.k_new, b.v_new, b.new_start,
                             b.new_len, causal=b.causal, softmax_scale=b.scale, lse=l, **kw)
    return out, l


def check(b, out, lse, wider=1.0):
    ref, ref_lse, bound = b.expected()
    n = b.n_q
    o, ref, bound = out[:n].double(), ref[:n], bound[:n]
    assert bool(torch.isfinite(o).all())
    worst = ((o - ref).abs() / (wider * bound + 2.0 ** -8 * ref.abs() + 1e-12)).max().item() if n else 0.0
    rms = ((o - ref).norm() / ref.norm().clamp(min=1e-30)).item() if n else 0.0
    assert worst <= 1.0, (worst, rms)
    assert rms <= 2.0 ** -8 * wider ** 0.5, rms
    assert bool((out[n:] == 9).all())
    if lse is not None:
        empty = torch.isinf(ref_lse[:n])
        assert torch.equal(torch.isinf(lse[:n]), empty) and bool((out[:n][empty] == 0).all())
        err = (lse[:n].double() - ref_lse[:n])[~empty].abs()
        # scores off by their bound (eps below 1/2 of it and the weights' rounding): the denominator's logarithm by no more
        assert err.numel() == 0 or err.max().item() <= 0.02 * wider
    return worst, rms


SEQS = {
    "one token": [(1, 64, 1)],
    "first token": [(1, 0, 1)],
    "decode": [(1, 4096, 17), (1, 0, 3), (1, 640, 1), (1, 2944, 31), (1, 128, 127)],
    "drafts": [(5, 1280, 5), (1, 256, 9), (7, 0, 7), (3, 8064, 40)],
    "chunk": [(40, 384, 40), (1, 128, 2), (129, 512, 140)],
    "holes": [(0, 128, 0), (2, 256, 2), (0, 0, 0), (3, 0, 1), (1, 384, 0), (4, 128, 0), (0, 512, 7)],
}


@pytest.mark.parametrize("name", list(SEQS))
@pytest.mark.parametrize("bits, G, meta, pages_of", [(2, 32, "f32", 4), (2, 32, "f16", 2), (2, 64, "f32", 1), (2, 64, "f16", 2), (2, 128, "f32", 3), (2, 128, "f16", 1),
                                                     (4, 32, "f32", 2), (4, 32, "f16", 1), (4, 64, "f32", 2), (4, 64, "f16", 1), (4, 128, "f32", 1), (4, 128, "f16", 2)])
@pytest.mark.parametrize("heads", [(8, 8), (8, 2)])
def test_sequences(name, bits, G, meta, pages_of, heads):
    seqs = [(nq, c // G * G, r) for nq, c, r in SEQS[name]]
    b = Batch(len(name) + bits + G, seqs, *heads, bits, G, meta, pages_of, spare_q=3)
    sq.squat_get_device_status()
    print(check(b, *call(b)))
    assert sq.squat_get_device_status() == 0


@pytest.mark.parametrize("heads", [(3, 1), (12, 4), (32, 1), (64, 2)])
def test_head_layouts(heads):
    b = Batch(sum(heads), [(1, 320, 5), (4, 96, 4), (2, 0, 3)], *heads, 2, 32)
    check(b, *call(b))


@pytest.mark.parametrize("scale", [0.25, 0.01])
@pytest.mark.parametrize("causal", [True, False])
def test_scale_and_no_mask(causal, scale):
    b = Batch(2, [(9, 256, 9), (1, 512, 130), (3, 128, 1), (2, 0, 0)], 8, 4, 4, 64, causal=causal, scale=scale)
    check(b, *call(b))


def test_many_sequences():
    """More sequences than a CTA has threads, most of them short, one long."""
    seqs = [(i % 3, 32 * (i % 5), i % 4 + 1) for i in range(300)]
    seqs[170] = (1, 6400, 5)
    b = Batch(7, seqs, 4, 2, 2, 32)
    check(b, *call(b))


def test_max_q_is_only_a_hint():
    b = Batch(9, [(3, 640, 3), (40, 128, 40), (1, 1024, 1)], 8, 2, 2, 32)
    for mq in (0, 1, 40, 4000):
        check(b, *call(b, max_q=mq))


def test_result_is_one_token_where_the_query_says_so():
    """Every cached token and row gets a query of its own that is far nearer to its key than to any other: out is its value, so a
    token in the wrong place, a lost or a doubled one is seen."""
    G, c, r = 32, 416, 19
    b = Batch(11, [(c + r, c, r)], 2, 1, 4, G, causal=False)
    from paged import deq_pool
    k, v = deq_pool(b.tensors, 4, G)
    t = torch.arange(c, device="cuda")
    page, off = b.page_table[0, t // b.P].long(), t % b.P
    f = int(b.new_start[0])
    keys = torch.cat([(k["zero"] + k["scale"] * k["code"])[page, 0, off], b.k_new[f:f + r, 0].double()])
    vals = torch.cat([(v["zero"] + v["scale"] * v["code"])[page, 0, off], b.v_new[f:f + r, 0].double()])
    b.q = (3.0 * keys / keys.norm(dim=1, keepdim=True) * math.sqrt(D)).unsqueeze(1).expand(-1, 2, -1).to(torch.bfloat16).contiguous()
    out, lse = call(b)
    check(b, out, None)
    assert ((out[:, 0].double() - vals).norm(dim=1) / vals.norm(dim=1)).max().item() < 0.05


@pytest.mark.parametrize("q_size, k_size, v_size", [(3e4, 1e-5, 1.0), (1e-4, 5e4, 1.0), (1.0, 1.0, 3e5), (1.0, 1.0, 1e-6), (1e-20, 1e20, 1e-20)])
@pytest.mark.parametrize("bits, G", [(2, 32), (4, 128)])
def test_magnitudes_beyond_binary16(q_size, k_size, v_size, bits, G):
    b = Batch(13, [(2, 5 * G, 9), (1, 0, 3), (40, 2 * G, 41)], 4, 2, bits, G, q_size=q_size, k_size=k_size, v_size=v_size)
    out, lse = call(b)
    check(b, out, None, wider=8.0)


def test_what_is_not_seen_does_not_matter():
    """NaN and infinities in rows that a query does not see: padding, later tokens, other sequences, and pages behind the length."""
    for nq, c, r in ((6, 96, 9), (70, 160, 71)):
        b = Batch(17, [(nq, c, r), (1, 32, 2)], 4, 2, 2, 32)
        clean, _ = call(b)
        f = int(b.new_start[0])
        b.k_new[f + r - 1, 0, 5], b.v_new[f + r - 1, 1, 7] = math.inf, math.nan
        b.v_new[f + r - 2, 0, 100] = -math.inf
        out, _ = call(b)
        # the last query's row: keys of head 0, values of head 1; the row before it: values of head 0, for two queries
        assert torch.equal(out[:nq - 2], clean[:nq - 2]) and torch.equal(out[nq:], clean[nq:])
        bad = torch.zeros_like(out[:nq], dtype=torch.bool)
        bad[nq - 1, 2:, 7] = True
        assert bool(torch.isnan(out[nq - 1, 2:, 7]).all())
        assert bool((out[nq - 2, :2, 100] == -math.inf).all())
        assert torch.equal(out[nq - 2, 2:], clean[nq - 2, 2:])
        keep = torch.arange(D, device="cuda") != 7
        assert torch.equal(out[nq - 1, 2:, keep], clean[nq - 1, 2:, keep])


def test_strides_streams_and_a_shared_projection():
    g = gen(21)
    b = Batch(21, [(4, 128, 4), (1, 256, 1), (11, 64, 11)], 8, 2, 2, 32)
    n = b.n_q
    wide = torch.empty((n, 8 + 4, D), dtype=torch.bfloat16, device="cuda")
    wide[:, :8] = b.q
    b.new_start = b.q_start[:-1].contiguous()
    wide[:, 8:] = normal(g, n, 4, D).to(torch.bfloat16)
    b.q, b.k_new, b.v_new = wide[:, :8], wide[:, 8:10], wide[:, 10:]
    ref, _ = call(b)
    check(b, ref, None)
    out = torch.empty((8, n, D), dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    ws = torch.empty(sq.squat_chunk_attention_workspace_bytes(n, 8, 2, b.max_q), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    sq.squat_chunk_attention(b.q, sq.PagePool(*b.tensors), b.q_start, b.cached, b.page_table, out, ws, b.max_q, b.k_new, b.v_new, b.new_start, b.new_len, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(out, ref)


def test_lengths_and_pages_outside_their_limits():
    """Flagged, cut to the limits, and the other sequences come out right (to their bounds: where a sum is cut into parts depends on
    all lengths)."""
    seqs = [(1, 128, 3), (1, 256, 2), (2, 64, 4)]
    b = Batch(23, seqs, 4, 2, 2, 32)
    clean, _ = call(b)
    ref, _, bound = b.expected()
    right = lambda out, rows: bool(((out.double() - ref)[rows].abs() <= (bound + 2.0 ** -8 * ref.abs())[rows]).all())  # noqa: E731
    sq.squat_get_device_status()
    for field, i, value in (("cached", 0, 10 ** 9), ("cached", 0, -5), ("cached", 0, 37), ("new_len", 0, 10 ** 6), ("new_start", 0, -9), ("new_len", 0, -1),
                            ("page_table", 0, 10 ** 6), ("page_table", 0, -3)):
        t = getattr(b, field)
        old = t.clone()
        (t[0] if field == "page_table" else t)[i] = value
        out, _ = call(b)
        assert sq.squat_get_device_status() == sq.FLAG_PAGES
        assert right(out, slice(1, None))
        t.copy_(old)
    old = b.q_start.clone()
    b.q_start.copy_(torch.tensor([0, 1, 2, 10 ** 6], dtype=torch.int32))
    out, _ = call(b)
    assert sq.squat_get_device_status() == sq.FLAG_PAGES and right(out, slice(0, 2))
    b.q_start.copy_(old)
    out, _ = call(b)
    assert sq.squat_get_device_status() == 0 and torch.equal(out, clean)


def test_graph_replay_with_other_lengths():
    """A captured step runs again with more cached tokens, other rows and other pages, and two graphs share a workspace in turn."""
    b = Batch(27, [(1, 320, 2), (1, 64, 5), (3, 640, 3)], 8, 4, 2, 32)
    pool = sq.PagePool(*b.tensors)
    out = torch.empty_like(b.q)
    ws = torch.empty(sq.squat_chunk_attention_workspace_bytes(b.n_q, 8, 4, 3), dtype=torch.uint8, device="cuda")
    run = lambda: sq.squat_chunk_attention(b.q, pool, b.q_start, b.cached, b.page_table, out, ws, 3, b.k_new, b.v_new, b.new_start, b.new_len)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for gr in graphs:
        with torch.cuda.graph(gr):
            run()
    for seqs in (b.seqs, [(1, 0, 1), (1, 96, 4), (3, 512, 3)], [(2, 128, 2), (0, 0, 0), (3, 608, 0)]):
        b.seqs = seqs
        b.cached.copy_(torch.tensor([c for _, c, _ in seqs], dtype=torch.int32))
        b.new_len.copy_(torch.tensor([r for _, _, r in seqs], dtype=torch.int32))
        starts = [0, seqs[0][0], seqs[0][0] + seqs[1][0], sum(s[0] for s in seqs)]
        b.q_start.copy_(torch.tensor(starts, dtype=torch.int32))
        b.page_table.copy_(b.page_table.clamp(min=0))
        for gr in graphs:
            out.fill_(9)
            gr.replay()
            torch.cuda.synchronize()
            check(b, out, None)
        first = out.clone()
        graphs[0].replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first)


def test_far_pages():
    """Token indexes whose bytes pass 32 bits."""
    H, G, bits, P = 1, 128, 2, 128
    far = (1 << 27) + P
    b = Batch(29, [(1, 2 * P, 1), (3, P, 5)], 2, H, bits, G, "f16", pages_of=1)
    ref, _ = call(b)
    t = []
    for x in b.tensors:
        per = x[0, 0].numel() / P
        flat = torch.empty(int((far * 3 + P) * per), dtype=x.dtype, device="cuda")
        y = torch.as_strided(flat, x.shape, (int(far * per), int(P * per), x.shape[3], 1))
        y.copy_(x)
        t.append(y)
    b.tensors = t
    out, _ = call(b)
    assert torch.equal(out, ref)


def test_a_step_end_to_end():
    """Positions, write with error feedback, attention over pages and residual rows, read back: three steps of two sequences, against
    float64 on what was read back."""
    Hq, H, G, bits, P = 8, 2, 32, 2, 64
    g = gen(31)
    plan = sq.RopePlan((16, 24, 24))
    s = sq.Subspace(H)
    prompt = normal(g, Hq, 256, D).to(torch.bfloat16)
    sq.squat_build_subspace(s, prompt, 16, 1e-3)
    pool = sq.PagePool.empty(9, P, H, bits, G)
    table = torch.tensor([[4, 1, 7, 3], [0, 8, 2, 6]], dtype=torch.int32, device="cuda")
    lengths = (64, 96), (32, 0), (7, 5)                         # new tokens of either sequence and step; the last are not full groups
    cached, at = [0, 0], 0
    rows = [torch.empty((0, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(4)]        # k, v of each sequence in full precision
    for n0, n1 in lengths:
        T = n0 + n1
        qkv = normal(g, T, Hq + 2 * H, D).to(torch.bfloat16)
        pos = torch.randint(0, 500, (3, T), generator=g, device="cuda", dtype=torch.int32)
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
        sq.squat_rope_apply(plan, pos, q, k)
        i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        out = torch.empty((T, Hq, D), dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(sq.squat_chunk_attention_workspace_bytes(T, Hq, H, max(n0, n1)), dtype=torch.uint8, device="cuda")
        sq.squat_chunk_attention(q, pool, i32(0, n0, T), i32(*cached), table, out, ws, max(n0, n1), k, v, i32(0, n0), i32(n0, n1))
        a = 0
        for i, n in enumerate((n0, n1)):
            if n == 0:
                continue
            kk, vv = torch.empty((cached[i], H, D), device="cuda"), torch.empty((cached[i], H, D), device="cuda")
            slots = i32(*[int(table[i, t // P]) * P + t % P for t in range(0, cached[i], G)])
            sq.squat_pages_read(pool, slots, kk, vv)
            keys, vals = torch.cat((kk.double(), k[a:a + n].double())), torch.cat((vv.double(), v[a:a + n].double()))
            seen = torch.arange(keys.shape[0], device="cuda").unsqueeze(0) <= (torch.arange(n, device="cuda") + cached[i]).unsqueeze(1)
            for h in range(H):
                sc = torch.einsum("qhd,td->hqt", q[a:a + n, 4 * h:4 * h + 4].double(), keys[:, h]) / math.sqrt(D)
                w = torch.softmax(sc.masked_fill(~seen, -math.inf), 2)
                ref = torch.einsum("hqt,td->qhd", w, vals[:, h])
                o = out[a:a + n, 4 * h:4 * h + 4].double()
                assert ((o - ref).norm() / ref.norm()).item() <= 2.0 ** -8
            a += n
        full = [n // G * G for n in (n0, n1)]
        take = torch.cat([torch.arange(full[0]), n0 + torch.arange(full[1])]).cuda()
        slots = i32(*[int(table[i, (cached[i] + t) // P]) * P + (cached[i] + t) % P for i in (0, 1) for t in range(0, full[i], G)])
        if take.numel():
            wws = torch.empty(sq.squat_pages_write_workspace_bytes(pool, take.numel()), dtype=torch.uint8, device="cuda")
            sq.squat_pages_write(pool, slots, k[take], v[take], s, wws)
        cached = [c + f for c, f in zip(cached, full)]
    assert cached == [96, 96]


@pytest.mark.parametrize("heads, nq", [((8, 1), 1), ((9, 1), 1), ((8, 1), 2), ((17, 1), 1), ((8, 1), 3), ((5, 1), 5), ((24, 1), 1), ((25, 1), 1), ((8, 1), 16), ((43, 1), 3), ((16, 2), 32), ((1, 1), 257)])
def test_row_counts_around_the_kernels_borders(heads, nq):
    """8, 9, 16, 17, 24, 25, 128, 129, 256 and 257 rows per KV head, alone (sequences of one length) and with shorter sequences."""
    for seqs in ([(nq, 416, nq), (nq, 32, nq + 3)], [(nq, 416, nq), (max(1, nq // 3), 704, 2), (1, 96, 1)]):
        b = Batch(nq + heads[0], seqs, *heads, 2, 32, pages_of=3)
        check(b, *call(b))


def test_calls_at_the_same_time():
    """Two streams, each with its workspace: few rows on one, many on the other."""
    small = Batch(41, [(1, 1024, 9)] * 12, 8, 8, 2, 32)
    large = Batch(43, [(90, 640, 97), (1, 320, 1), (200, 0, 200)], 8, 2, 4, 64, "f16")
    want = [call(b, lse=False)[0] for b in (small, large)]
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [torch.zeros_like(b.q) for b in (small, large)]
    spaces = [torch.empty(sq.squat_chunk_attention_workspace_bytes(b.n_q, b.Hq, b.H, b.max_q), dtype=torch.uint8, device="cuda") for b in (small, large)]
    pools = [sq.PagePool(*b.tensors) for b in (small, large)]
    torch.cuda.synchronize()
    for _ in range(20):
        for b, st, out, ws, pool in zip((small, large), streams, outs, spaces, pools):
            sq.squat_chunk_attention(b.q, pool, b.q_start, b.cached, b.page_table, out, ws, b.max_q, b.k_new, b.v_new, b.new_start, b.new_len, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])


@pytest.mark.parametrize("bits, G, meta", [(2, 32, "f32"), (4, 64, "f16")])
@pytest.mark.parametrize("nq", [1, 5, 40])
def test_a_page_outside_the_pool_is_not_read(bits, G, meta, nq):
    """Page 0 is no sequence's and holds NaN: the result stays finite."""
    b = Batch(5 + nq, [(nq, 4 * G, nq + 2), (1, 3 * G, 2), (nq, 0, nq)], 4, 2, bits, G, meta, pages_of=1)
    ref, _, bound = b.expected()
    t = []
    for x in b.tensors:
        first = torch.zeros_like(x[:1])
        t.append(torch.cat((first.fill_(math.nan if x.is_floating_point() else 255), x)))
    b.tensors = t
    b.page_table = torch.where(b.page_table >= 0, b.page_table + 1, b.page_table)
    n = b.tensors[0].shape[0]
    sq.squat_get_device_status()
    for at in range(4):
        for bad in (-1, n, 2 ** 31 - 1, -2 ** 31):
            old = int(b.page_table[0, at])
            b.page_table[0, at] = bad
            out, lse = call(b)
            assert sq.squat_get_device_status() == sq.FLAG_PAGES
            assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
            assert bool(((out.double() - ref)[nq:].abs() <= (bound + 2.0 ** -8 * ref.abs())[nq:]).all())
            b.page_table[0, at] = old


@pytest.mark.parametrize("v_size", [1e-6, 1e-9, 1e-20])
@pytest.mark.parametrize("nq, rows", [(1, 0), (2, 0), (5, 0), (40, 0), (1, 40), (40, 70)])
@pytest.mark.parametrize("bits, G", [(2, 32), (4, 64)])
def test_values_below_binary16(v_size, nq, rows, bits, G):
    """Scales and zero-points that binary16 would round to zero (below 2^-25), in segments without and with rows in full precision:
    done in bf16, within the bounds of test_magnitudes_beyond_binary16."""
    b = Batch(3, [(nq, 6 * G, rows)], 4, 1, bits, G, v_size=v_size, causal=False)
    out, lse = call(b)
    ref, ref_lse, bound = b.expected()
    assert bool(((out.double() - ref).abs() <= 8 * bound + 2.0 ** -8 * ref.abs()).all())
    assert ((out.double() - ref).norm() / ref.norm()).item() <= 2.0 ** -8 * 8 ** 0.5
    assert (lse.double() - ref_lse).abs().max().item() <= 0.02 * 8


@pytest.mark.parametrize("q_size, k_size", [(600.0, 1e-4), (600.0, 1e-5), (600.0, 1e-7), (1.0, 1e-6), (1.0, 1e-9), (1e-3, 1e-3), (1e-6, 1.0), (1e-9, 1.0), (1e-9, 1e-9)])
@pytest.mark.parametrize("nq, rows", [(1, 0), (2, 0), (5, 0), (40, 0), (1, 40), (40, 70)])
@pytest.mark.parametrize("bits, G, meta", [(2, 32, "f32"), (4, 64, "f32"), (4, 64, "f16")])
def test_keys_and_queries_below_binary16(q_size, k_size, nq, rows, bits, G, meta):
    """Scores of ordinary size from keys or queries that binary16 would round to a few bits or to zero, with the softmax scale that
    goes with them: done in bf16, within the bounds of test_magnitudes_beyond_binary16."""
    if meta == "f16" and k_size < 1e-6:
        k_size = 1e-6                                          # what such metadata can hold
    b = Batch(3, [(nq, 6 * G, rows)], 4, 1, bits, G, meta, q_size=q_size, k_size=k_size, causal=False, scale=0.2 / (q_size * k_size))
    out, lse = call(b)
    ref, ref_lse, bound = b.expected()
    assert bool(((out.double() - ref).abs() <= 8 * bound + 2.0 ** -8 * ref.abs()).all())
    assert ((out.double() - ref).norm() / ref.norm()).item() <= 2.0 ** -8 * 8 ** 0.5
    assert (lse.double() - ref_lse).abs().max().item() <= 0.02 * 8


@pytest.mark.parametrize("bits, G, meta", [(2, 32, "f32"), (4, 32, "f32"), (2, 128, "f16"), (4, 64, "f16")])
@pytest.mark.parametrize("heads, nq", [((2, 2), 1), ((8, 1), 1), ((8, 1), 2), ((8, 1), 3), ((8, 1), 16), ((8, 1), 40)])
def test_scores_that_binary16_holds_exactly(bits, G, meta, heads, nq):
    """Queries 0, 1/2 or 1 with either sign, scales 1/8 to 3/8, zero-points in 32nds below 8: keys have 9 bits, and products with a
    scaled query and a code under its bias (up to 3/8 x 1039) are multiples of 2^-6 whose sums stay below 2^16, so binary16 and float32
    hold them exactly, in every kernel.  What is left of lse's error, in powers of two of the exponent: the rounded softmax scale, its
    product with a score and with the maximum, and their difference (below 32 each: 2^-19), one of 2^-21 for the exponential, 2^-24 for
    each term of the sum, and 2^-22 of lse for the logarithm.  bf16 would be off by up to 2^-6 in a key."""
    c, r = 7 * G, nq + 20
    b = Batch(51 + nq, [(nq, c, r), (1, 2 * G, 3)], *heads, bits, G, meta, scale=0.04)
    g = gen(bits + nq)
    multiples = lambda lo, hi, of, x: (torch.randint(lo, hi, x.shape, generator=g, device="cuda") / of).to(x.dtype)  # noqa: E731
    b.q = multiples(-2, 3, 2, b.q)
    b.k_new.copy_(multiples(-16, 17, 8, b.k_new))
    b.v_new.copy_(multiples(-16, 17, 8, b.v_new))
    b.tensors[1], b.tensors[2] = multiples(1, 4, 8, b.tensors[1]), multiples(-255, 256, 32, b.tensors[2])
    out, lse = call(b)
    ref, ref_lse, _ = b.expected()
    tol = (4 * 2.0 ** -19 + 2.0 ** -21 + (c + r) * 2.0 ** -24) * math.log(2) + 2.0 ** -22 * ref_lse.abs()
    assert float((ref_lse * 1.4427).abs().max()) < 32
    err = (lse.double() - ref_lse).abs()
    print("lse off by", err.max().item(), "allowed", tol.min().item())
    assert bool((err <= tol).all())
    check(b, out, None)
