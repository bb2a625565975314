"""Plain float64 forms of the paged cache's operators, and inputs for them, for the tests.  Nothing here calls the library."""
import math

import torch

D = 128
META = {"f32": torch.float32, "f16": torch.float16}


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def unpack(packed, bits):
    per = 8 // bits
    parts = [(packed.to(torch.int64) // 2 ** (bits * i)) % 2 ** bits for i in range(per)]
    return torch.stack(parts, -1).flatten(-2).double()


def random_pool(g, n_pages, page_tokens, H, bits, G, meta, k_size=1.0, v_size=1.0):
    """Six tensors of a pool with random codes; the values they stand for have about the given size."""
    L = 2 ** bits - 1
    codes = lambda: torch.randint(0, 256, (n_pages, H, page_tokens, D * bits // 8), generator=g, device="cuda", dtype=torch.uint8)  # noqa: E731

    def grids(size, *shape):
        scale = (0.5 + torch.rand(shape, generator=g, device="cuda")) * (3.0 * size / L)
        zero = -scale * L / 2 + 0.3 * size * torch.randn(shape, generator=g, device="cuda")
        return scale.to(META[meta]), zero.to(META[meta])

    ks, kz = grids(k_size, n_pages, H, page_tokens // G, D)
    vs, vz = grids(v_size, n_pages, H, page_tokens, D // G)
    return [codes(), ks, kz, codes(), vs, vz]


def deq_pool(tensors, bits, G):
    """Scales, zero-points and codes of every place in the pool as float64 [n_pages, H, page_tokens, D]: (k, v), each a dict."""
    kc, ks, kz, vc, vs, vz = tensors
    k = dict(code=unpack(kc, bits), scale=ks.double().repeat_interleave(G, 2), zero=kz.double().repeat_interleave(G, 2))
    v = dict(code=unpack(vc, bits), scale=vs.double().repeat_interleave(G, 3), zero=vz.double().repeat_interleave(G, 3))
    return k, v


def attention(q, k, v, scale, nq, nk_cached, causal, k_err=None, v_err=None):
    """One sequence and KV head in float64.  q [nq, per, D]; k, v [tokens, D], the first nk_cached of them seen by all; k_err, v_err:
    bounds of what enters the tensor cores in their place.  Returns out, lse and a bound of the error of `out` before its last
    rounding: weights off by a factor within 1 + eps move a weighted mean by at most 2 eps / (1 - eps) sum w |v|."""
    n = k.shape[0]
    rows = n - nk_cached
    if n == 0 or nq == 0:
        return torch.zeros_like(q), torch.full_like(q[..., 0], -math.inf), torch.zeros_like(q)
    seen = torch.ones(nq, n, dtype=torch.bool, device=q.device)
    if causal:
        limit = torch.arange(nq, device=q.device) + rows - nq + 1
        seen = (torch.arange(n, device=q.device) - nk_cached).unsqueeze(0) < limit.clamp(min=0).unsqueeze(1)
        seen |= (torch.arange(n, device=q.device) < nk_cached).unsqueeze(0)
    s = torch.einsum("jhd,td->jht", q, k) * scale
    s = s.masked_fill(~seen.unsqueeze(1), -math.inf)
    empty = ~seen.any(1)
    lse = torch.logsumexp(s, 2)
    w = torch.exp(s - torch.where(empty.unsqueeze(1), 0.0, lse).unsqueeze(2))
    vv = torch.where(seen.any(0).unsqueeze(1), v, 0.0)
    out = torch.einsum("jht,td->jhd", w, vv)
    if k_err is None:
        return out, lse, None
    ds = torch.einsum("jhd,td->jht", q.abs(), k_err) * scale
    eps = torch.expm1(torch.where(seen.unsqueeze(1), ds, 0.0).amax(2)) + 2.0 ** -8
    bound = 2 * eps / (1 - eps).clamp(min=0.5)
    bound = bound.unsqueeze(2) * torch.einsum("jht,td->jhd", w, vv.abs()) + torch.einsum("jht,td->jhd", w, v_err)
    return out, lse, bound


class Batch:
    """Sequences (queries, cached tokens, rows in full precision) over a random pool, and what the call takes."""

    def __init__(self, seed, seqs, Hq, H, bits, G, meta="f32", pages_of=2, causal=True, scale=0.0, q_size=1.0, k_size=1.0, v_size=1.0, spare_q=0):
        g = gen(seed)
        self.seqs, self.Hq, self.H, self.bits, self.G, self.causal, self.scale = seqs, Hq, H, bits, G, causal, scale
        self.P = P = G * pages_of
        need = [-(-c // P) for _, c, _ in seqs]
        n = sum(need) + 1
        self.tensors = random_pool(g, n, P, H, bits, G, meta, k_size, v_size)
        order = torch.randperm(n, generator=g, device="cuda").to(torch.int32).tolist()
        width = max(need + [1])
        table, a = [], 0
        for m in need:
            table.append(order[a:a + m] + [-1] * (width - m))
            a += m
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        self.page_table = ints(table).reshape(len(seqs), width)
        starts = [0]
        for nq, _, _ in seqs:
            starts.append(starts[-1] + nq)
        self.q_start, self.cached = ints(starts), ints([c for _, c, _ in seqs])
        self.n_q = starts[-1]
        # rows of the sequences with gaps between them, which hold NaN
        at, first = 3, []
        for _, _, r in seqs:
            first.append(at)
            at += r + 2
        self.new_start, self.new_len = ints(first), ints([r for _, _, r in seqs])
        self.q = (q_size * normal(g, self.n_q + spare_q, Hq, D)).to(torch.bfloat16)
        kv = torch.cat((k_size * normal(g, at, H, D), v_size * normal(g, at, H, D)), 1).to(torch.bfloat16)
        used = torch.zeros(at, dtype=torch.bool, device="cuda")
        for f, (_, _, r) in zip(first, seqs):
            used[f:f + r] = True
        kv[~used] = math.nan
        self.k_new, self.v_new = kv[:, :H], kv[:, H:]
        self.max_q = max([nq for nq, _, _ in seqs] + [0])

    def expected(self):
        """out, lse, bound over all rows, float64 (NaN where no sequence owns a row)."""
        k, v = deq_pool(self.tensors, self.bits, self.G)
        u = 2.0 ** -11                                                  # binary16's rounding; bf16's where values leave its range
        scale = self.scale or 1.0 / math.sqrt(D)
        out = torch.full((self.q.shape[0], self.Hq, D), math.nan, dtype=torch.float64, device="cuda")
        bound, lse = out.clone(), out[..., 0].clone()
        per = self.Hq // self.H
        a = 0
        for i, (nq, c, r) in enumerate(self.seqs):
            t = torch.arange(c, device="cuda")
            page, off = self.page_table[i, t // self.P].long(), t % self.P
            f = int(self.new_start[i])
            for h in range(self.H):
                parts, errs = [], []
                for x, new in ((k, self.k_new), (v, self.v_new)):
                    sc, z, code = (x[n][page, h, off] for n in ("scale", "zero", "code"))
                    val = z + sc * code
                    rows = new[f:f + r, h].double()
                    parts.append(torch.cat((val, rows)))
                    errs.append(torch.cat((u * (z.abs() + (sc * code).abs() + val.abs()), 0 * rows)))
                o, l, b = attention(self.q[a:a + nq, h * per:(h + 1) * per].double(), parts[0], parts[1], scale, nq, c, self.causal, errs[0], errs[1])
                out[a:a + nq, h * per:(h + 1) * per], lse[a:a + nq, h * per:(h + 1) * per], bound[a:a + nq, h * per:(h + 1) * per] = o, l, b
            a += nq
        return out, lse, bound
