"""Batches over a paged cache for the GPU tests: plans, caches in several memory orders, and poison in every place that a call
may not read."""
import torch

import attention_reference as ref
from paper_2309_12307_amd import binding

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}


def in_memory(x, layout):
    """x (pages, page, Hkv, ...) on the GPU with its axes in another order in memory, or with room between them."""
    if layout == "head":
        return x.transpose(1, 2).contiguous().transpose(1, 2)
    if layout == "gaps":
        wide = torch.empty(x.shape[0], x.shape[1] + 1, x.shape[2] + 1, *x.shape[3:], dtype=x.dtype, device=x.device)
        wide.view(torch.uint8).fill_(255)
        view = wide[:, 1:, :-1]
        view.copy_(x) if x.dtype != TYPES["e4m3"] else view.view(torch.uint8).copy_(x.view(torch.uint8))
        return view
    return x.contiguous()


class Batch:
    """lens: (rows, cached tokens) of every sequence.  The pages lie in the cache in no order; those of no sequence, what lies
    behind a sequence's tokens and the rows before and behind the batch hold NaN."""

    def __init__(self, lens, H, Hkv, D, page, dtype="bf16", cache="bf16", layout="token", seed=0, before=0, behind=0, bad_pages=(), cols=None, size=1.0):
        gen = torch.Generator().manual_seed(seed)
        self.dt, self.cache_dt, self.page = TYPES[dtype], TYPES[cache], page
        self.lens, self.H, self.Hkv, self.D = lens, H, Hkv, D
        counts = [-(-max(kv, 0) // page) for _, kv in lens]
        self.cols = cols or max(1, max(counts)) + 1
        pages = sum(counts) + 3
        order = torch.randperm(pages, generator=gen).int()
        self.table = torch.full((len(lens), self.cols), -7, dtype=torch.int32)
        first = 0
        for b, n in enumerate(counts):
            n_in = min(n, self.cols)
            self.table[b, :n_in] = order[first:first + n_in]
            first += n
        for b, col, value in bad_pages:
            self.table[b, col] = value
        starts = [before]
        for n, _ in lens:
            starts.append(starts[-1] + n)
        self.T = starts[-1] + behind
        self.row_start = torch.tensor(starts, dtype=torch.int32)
        self.kv_len = torch.tensor([kv for _, kv in lens], dtype=torch.int32)
        self.own = torch.zeros(self.T, dtype=torch.bool)
        self.own[starts[0]:starts[-1]] = True
        live = torch.zeros(pages, page, dtype=torch.bool)     # places that hold a token
        for b, (_, kv) in enumerate(lens):
            for j in range(0, max(kv, 0), page):
                pg = int(self.table[b, j // page]) if j // page < self.cols else -1
                if 0 <= pg < pages:
                    live[pg, :min(page, kv - j)] = True
        self.live = live
        self.host = {}
        for name in ("k", "v"):
            x = torch.randn(pages, page, Hkv, D, generator=gen)
            if cache == "e4m3":
                y, e = ref.quantise(x * size)
                y = y.float().to(self.cache_dt)
                bits = y.view(torch.uint8)
                bits[~live] = 0x7F
                e[~live] = 255
                self.host[name], self.host[name + "_exp"] = bits.view(self.cache_dt), e
            else:
                x = x.to(self.cache_dt)
                x[~live] = float("nan")
                self.host[name], self.host[name + "_exp"] = x, None
        self.dev = {n: in_memory(x.cuda(), layout) if x is not None else None for n, x in self.host.items()}
        self.plan = dict(row_start=self.row_start.cuda(), kv_len=self.kv_len.cuda(), page_table=self.table.cuda())

        def rows(h):
            x = torch.randn(self.T, h, D, generator=gen).to(self.dt)
            x[~self.own] = float("nan")
            return x
        self.q, self.k, self.v = rows(H), rows(Hkv), rows(Hkv)

    def caches(self):
        return dict(k_cache=self.dev["k"], v_cache=self.dev["v"], k_exp=self.dev["k_exp"], v_exp=self.dev["v_exp"])

    def params(self, **kw):
        return binding.make_paged_params(**{**self.plan, **self.caches(), **kw})

    def reference(self, window=0, sinks=0, scale=None, host=None):
        h = host or self.host
        return ref.paged_reference(self.q, h["k"], h["v"], h["k_exp"], h["v_exp"], self.row_start, self.kv_len, self.table, window, sinks, scale)

    def attend(self, window=0, sinks=0, workspace="wanted", max_kv=0, scale=0.0, q=None):
        """o and lse, which start as 5 and 7."""
        q = self.q.cuda() if q is None else q
        o = torch.full((self.T, self.H, self.D), 5.0, dtype=self.dt, device="cuda")
        lse = torch.full((self.H, self.T), 7.0, device="cuda")
        kw = dict(q=q, o=o, lse=lse, window=window, sinks=sinks, max_kv=max_kv, scale=scale)
        n = binding.paged_workspace_bytes(self.params(**kw)) if workspace == "wanted" else workspace
        ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda") if n else None
        binding.s2attn_paged_fwd(self.params(workspace=ws, **kw))
        torch.cuda.synchronize()
        return o, lse

    def check(self, o, lse, want):
        own = self.own
        ref.hold("o", o, want, own)
        ref.hold("lse", lse, want, (slice(None), own))
        assert (o[~own.cuda()] == 5).all() and (lse[:, ~own.cuda()] == 7).all(), "rows of no sequence"
