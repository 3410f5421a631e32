"""The paged cache in plain form, in float64 where numbers are computed: caches with
random contents, garbage wherever no sequence has a row, and the reference of
every entry point."""
import math

import torch

import paper_2607_22586_gb300 as M

U32, UBF = 2.0 ** -24, 2.0 ** -8          # half a step of float32 and bfloat16, relative
DT = {"bf16": torch.bfloat16, "f32": torch.float32, "i8": torch.int8}


def quantise(x):
    """Codes and scales of rows, in float32 as the header writes them."""
    x = x.float()
    most = x.abs().amax(-1)
    fine = torch.isfinite(x).all(-1)
    full = torch.full_like(most, 127.0)               # torch divides by a number as a product with its reciprocal
    inv = torch.where(fine & (most >= 2.0 ** -110), full / most, torch.zeros_like(most))
    code = torch.round(torch.nan_to_num(x * inv[..., None], 0, 0, 0)).to(torch.int8)
    return code, torch.where(fine, most / full, torch.full_like(most, math.nan))


class Cache:
    """A pool with its page table in no order and `lens` [L, B, Hkv]; room for `room`
    rows more in every sequence. Whatever no row was written to holds garbage:
    NaN in scales and float pages."""

    def __init__(self, lens, d, kind, page, seed=0, room=0, spare=2, extra_entries=1, device="cuda"):
        gen = torch.Generator().manual_seed(seed)
        self.lens_host = torch.as_tensor(lens, dtype=torch.int32)
        if self.lens_host.dim() == 2:
            self.lens_host = self.lens_host[None]
        self.L, self.B, self.H = self.lens_host.shape
        self.d, self.kind, self.page = d, kind, page
        need = (self.lens_host + room + page - 1) // page
        total = int(need.sum())
        self.n_pages = total + spare
        most = int(need.max()) + extra_entries
        order = torch.randperm(self.n_pages, generator=gen)[:total].to(torch.int32)
        # entries that no row needs hold bad pages
        table = torch.randint(-5, 0, (self.L, self.B, self.H, most), generator=gen, dtype=torch.int32)
        table[..., 0::2] = self.n_pages + 7
        table[torch.arange(most) < need[..., None]] = order
        self.table, self.lens = table.to(device), self.lens_host.to(device)
        shape = (self.n_pages, page, d)
        if kind == "i8":
            self.kp, self.vp = (torch.randint(-127, 128, shape, generator=gen, dtype=torch.int8).to(device) for _ in range(2))
            self.ks, self.vs = (torch.full(shape[:2], math.nan, device=device) for _ in range(2))
        else:
            self.kp, self.vp = (torch.full(shape, math.nan, dtype=DT[kind], device=device) for _ in range(2))
            self.ks = self.vs = None

    def struct(self, layer=None):
        at = slice(None) if layer is None else slice(layer, layer + 1)
        return M.make_cache(self.kp, self.vp, self.table[at], self.lens[at], self.ks, self.vs)

    def slots(self, l, b, h, pos):
        pos = torch.as_tensor(pos, device=self.table.device).long()
        return self.table[l, b, h].long()[pos // self.page] * self.page + pos % self.page

    def put(self, l, b, h, pos, k, v):
        """Plain write of rows of any type at positions."""
        s = self.slots(l, b, h, pos)
        for x, pages, scales in ((k, self.kp, self.ks), (v, self.vp, self.vs)):
            if self.kind == "i8":
                code, scale = quantise(x)
                pages.view(-1, self.d)[s] = code
                scales.view(-1)[s] = scale
            else:
                pages.view(-1, self.d)[s] = x.to(pages.dtype)

    def get(self, l, b, h, pos):
        """Plain read of positions: K and V in float64."""
        s = self.slots(l, b, h, pos)
        out = []
        for pages, scales in ((self.kp, self.ks), (self.vp, self.vs)):
            x = pages.view(-1, self.d)[s].double()
            out.append(x * scales.view(-1)[s].double()[:, None] if self.kind == "i8" else x)
        return out

    def fill_random(self, seed=1, spread=1.0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for l in range(self.L):
            for b in range(self.B):
                for h in range(self.H):
                    n = int(self.lens_host[l, b, h])
                    if n:
                        k, v = (torch.randn((n, self.d), generator=gen, device="cuda") for _ in range(2))
                        self.put(l, b, h, torch.arange(n), k * spread, v)
        return self

    def tensors(self):
        return [x for x in (self.kp, self.vp, self.ks, self.vs, self.lens, self.table) if x is not None]

    def clone_tensors(self):
        return [x.clone() for x in self.tensors()]


def same(a, b):
    """Equal to the bit, NaN included."""
    view = {2: torch.int16, 4: torch.int32, 1: torch.int8}
    return a.shape == b.shape and torch.equal(a.view(view[a.element_size()]), b.view(view[b.element_size()]))


def cu_of(new):
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    return cu


def shape_of(cache, new, hq, dtype, layers=None, stride_kv=0):
    return M.make_shape(hq, cache.H, cache.d, 2, 0 if dtype == "bf16" else 1, cu_of(new), [1] * len(new),
                        n_layers=cache.L if layers is None else layers, layer_stride_kv=stride_kv)


def workspace(shape, struct):
    n = M.mmshift_cache_workspace_size(shape, struct)
    ws = torch.full((n,), 0xA5, dtype=torch.uint8, device="cuda")     # only the status word has to be zero
    ws[:256].zero_()
    return ws, n


def attend(cache, q, new, causal=True, scale=0.0, layer=0, stride=0, lse=True, out=None, status=0):
    """One call of mmshift_cache_attention on q [T, Hq, d]."""
    dtype = "bf16" if q.dtype == torch.bfloat16 else "f32"
    struct = cache.struct(layer)
    shape = shape_of(cache, new, q.shape[1], dtype, layers=1)
    ws, n = workspace(shape, struct)
    if out is None:
        out = torch.full(q.shape, math.nan, dtype=q.dtype, device="cuda")
    ls = torch.full(q.shape[:2], math.nan, device="cuda") if lse else None
    M.check(M.mmshift_cache_attention(shape, struct, q, stride, int(causal), scale, out, ls, ws, n), "attention")
    assert M.mmshift_poll_status(ws) == status
    return out, ls


def reference(cache, q, new, causal=True, scale=0.0, layer=0, gone=None):
    """out and lse in float64, and how far the kernel's may lie from them (element by element).

    z is a sum of d products accumulated in float32 and scaled (and, in base 2, turned): off by at
    most (d + 4) U32 times the sum of the products' magnitudes. A weight e^(z - m) is then off by 2 z's
    error and by 4 U32 (exponential), relatively, and for bfloat16 rows by UBF more: its rounding, an
    8-bit row's scale multiplied in before (U32). The sum over n keys adds n U32. out is a mean of v
    with these weights: its error is the weights' relative error times the mean of |v|, for
    numerator and denominator, and its own rounding to the row type."""
    B, H, d, r = cache.B, cache.H, cache.d, q.shape[1] // cache.H
    bf = q.dtype == torch.bfloat16
    scale = scale or 1.0 / math.sqrt(d)
    cu = cu_of(new)
    out, tol = torch.zeros(q.shape, dtype=torch.float64, device="cuda"), torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    ltol = torch.zeros_like(lse)
    for b, n in enumerate(new):
        for h in range(H):
            m = int(cache.lens_host[layer, b, h])
            for i in range(n):
                end = m - n + i + 1 if causal else m
                if end <= 0:
                    continue
                pos = torch.arange(end, device="cuda")
                if gone is not None:
                    pos = pos[~gone(layer, b, h, pos)]
                    if not len(pos):
                        continue
                k, v = cache.get(layer, b, h, pos)
                x = q[cu[b] + i, h * r:(h + 1) * r].double()
                z = x @ k.T * scale
                zerr = ((d + 4) * U32 * (x.abs() @ k.abs().T) * scale).amax(-1)
                p = torch.softmax(z, -1)
                top = torch.logsumexp(z, -1)
                lse[cu[b] + i, h * r:(h + 1) * r] = torch.where(top == math.inf, math.nan, top)   # by definition
                ltol[cu[b] + i, h * r:(h + 1) * r] = zerr + (8 + end) * U32 + 2 * U32 * (z.abs().amax(-1) + 1)
                o = p @ v
                rel = 4 * zerr + (16 + 2 * end) * U32 + (UBF + U32 if bf else 0)
                out[cu[b] + i, h * r:(h + 1) * r] = o
                tol[cu[b] + i, h * r:(h + 1) * r] = rel[:, None] * (p @ v.abs()) + (UBF if bf else U32) * o.abs() + 1e-37
    return out, lse, tol * 1.01, ltol * 1.01


def check_attention(got, want, what=""):
    (out, lse), (ro, rl, tol, ltol) = got, want
    for name, x, y, t in (("out", out.double(), ro, tol), ("lse", lse.double(), rl, ltol)):
        fine = torch.isfinite(y)
        assert torch.equal(torch.isnan(x), torch.isnan(y)), (what, name, "NaN")
        assert torch.equal(x[~fine & ~torch.isnan(y)], y[~fine & ~torch.isnan(y)]), (what, name, "infinite")
        over = ((x - y).abs() > t) & fine
        assert not over.any(), (what, name, int(over.sum()), float(((x - y).abs() / t.clamp(min=1e-300))[fine].max()),
                                over.nonzero()[:5].tolist())
