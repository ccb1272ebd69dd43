"""Attention under a window and sinks in 64 bits, element by element with the bounds that the kernels' roundings allow.

Position p sees key j iff j <= p and (window == 0 or p - j < window or j < sinks).

Bounds (u: half a bf16 step relative to the value, 2^-8, or 0 for fp32; f = 2^-24, half an fp32 step):
  score        the D products of fp32 sums, the scale and the exponent's argument:  d = f ((D + 4) scale |q| |k| + 4 (|s| + |lse|) + 4)
  P            its relative error is at most rho = 3 d + (n + 8) f for n visible keys (d: the row's largest)
  o            (u + rho) P |v| + u |o|          P is rounded before P v, o when it is stored
  lse          d + (n + 8) f + 2 f |lse|
  delta        sum |do| bound(o) + D f sum |do o|
  dS           P ((D + 1) f |do| |v| + bound(delta) + rho |dP - delta|) (1 + u) + u |dS|
  dv           ((u + rho + m f) P)^T |do| + u |dv|, m terms a sum; dq, dk the same from dS, with scale
Sums of many roundings are far below their bound, so the root mean square of the errors is held too: roundings are independent
and uniform within half a step, a variance of bound^2 / 3 each at most, and what fp32 adds goes in with its bound."""
import torch

F = 2.0 ** -24
RMS_SLACK = 1.1   # of a mean over thousands of elements, against its expectation


def visible(pos, keys, window, sinks):
    """(rows, keys) bool for rows at positions pos (a tensor) and keys 0 .. keys - 1."""
    j = torch.arange(keys)[None]
    p = pos[:, None]
    m = j <= p
    return m & ((p - j < window) | (j < sinks)) if window > 0 else m


def half_step(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else 0.0


def head_forward(q, k, v, mask, scale, u):
    """One head: q (n, D), k, v (keys, D), mask (n, keys), all float64.  Rows without a visible key: o = 0, lse = -inf."""
    D = q.shape[1]
    s = scale * q @ k.T
    x = s.masked_fill(~mask, -torch.inf)
    lse = torch.logsumexp(x, 1)
    some = mask.any(1)
    P = torch.where(some[:, None], torch.exp(x - torch.where(some, lse, 0.0)[:, None]), 0.0)
    o = P @ v
    safe = torch.where(some, lse, 0.0).abs()
    d = torch.where(mask, (D + 4) * scale * (q.abs() @ k.abs().T) + 4 * s.abs(), 0.0).amax(1) if k.shape[0] else torch.zeros_like(safe)
    d = F * (d + 4 * safe + 4)
    n = mask.sum(1)
    rho = 3 * d + (n + 8) * F
    Pv = P @ v.abs()
    b_o = (u + rho[:, None]) * Pv + u * o.abs()
    var_o = (u * u / 3) * ((P * P) @ (v * v) + o * o) + (rho[:, None] * Pv) ** 2
    b_lse = d + (n + 8) * F + 2 * F * safe
    return dict(o=o, lse=lse, P=P, b_o=b_o, var_o=var_o, b_lse=b_lse, rho=rho)


def window_reference(q, k, v, do, window, sinks, scale=None, heads=None):
    """q, do (B, N, H, D), k, v (B, N, Hkv, D) on the CPU, of the type that the kernels get.  Returns o, lse (B, H, N), dq, dk, dv
    with bounds b_* and variances var_*.  `heads`: only these (their kv heads' gradients then lack the others)."""
    u = half_step(q.dtype)
    B, N, H, D = q.shape
    r = H // k.shape[2]
    scale = scale or D ** -0.5
    q, k, v = (x.double() for x in (q, k, v))
    do = do.double() if do is not None else None
    mask = visible(torch.arange(N), N, window, sinks)
    out = {}
    for n, like in (("o", q), ("dq", q), ("dk", k), ("dv", v)):
        for pre in ("", "b_", "var_"):
            out[pre + n] = torch.zeros_like(like)
    out["lse"], out["b_lse"] = torch.zeros(B, H, N, dtype=torch.float64), torch.zeros(B, H, N, dtype=torch.float64)
    for b in range(B):
        for h in heads if heads is not None else range(H):
            c = h // r
            Q, K, V = q[b, :, h], k[b, :, c], v[b, :, c]
            x = head_forward(Q, K, V, mask, scale, u)
            P, o, rho = x["P"], x["o"], x["rho"][:, None]
            out["o"][b, :, h], out["b_o"][b, :, h], out["var_o"][b, :, h] = o, x["b_o"], x["var_o"]
            out["lse"][b, h], out["b_lse"][b, h] = x["lse"], x["b_lse"]
            if do is None:
                continue
            DO = do[b, :, h]
            dP = DO @ V.T
            delta = (DO * o).sum(1, keepdim=True)
            # what is left of delta's error where rounding is independent, and where it is not
            fine = (DO.abs() * rho * (P @ V.abs())).sum(1, keepdim=True) + D * F * (DO * o).abs().sum(1, keepdim=True)
            b_delta = (DO.abs() * x["b_o"]).sum(1, keepdim=True) + D * F * (DO * o).abs().sum(1, keepdim=True)
            # P of the forward is rounded once for all D columns: its part of delta's error is sum_j u P_ij |dP_ij| at most
            var_delta = (u * u / 3) * (((DO * o) ** 2).sum(1, keepdim=True) + ((P * dP) ** 2).sum(1, keepdim=True))
            dS = P * (dP - delta)
            e32 = P * ((D + 1) * F * (DO.abs() @ V.abs().T) + rho * (dP - delta).abs())
            E = (e32 + P * b_delta) * (1 + u) + u * dS.abs()
            f32 = e32 + P * fine
            m = (N * r + 8) * F

            def add(name, value, bound, variance):
                out[name][b, :, c if name != "dq" else h] += value
                out["b_" + name][b, :, c if name != "dq" else h] += bound
                out["var_" + name][b, :, c if name != "dq" else h] += variance

            add("dq", scale * dS @ K, scale * (E @ K.abs() + m * dS.abs() @ K.abs()),
                scale ** 2 * (var_delta * (P @ K) ** 2 + (u * u / 3) * (dS * dS) @ (K * K) + (f32 @ K.abs() + m * dS.abs() @ K.abs()) ** 2))
            add("dk", scale * dS.T @ Q, scale * (E.T @ Q.abs() + m * dS.abs().T @ Q.abs()),
                scale ** 2 * ((P * P * var_delta).T @ (Q * Q) + (u * u / 3) * (dS * dS).T @ (Q * Q) + (f32.T @ Q.abs() + m * dS.abs().T @ Q.abs()) ** 2))
            add("dv", P.T @ DO, ((u + rho + m) * P).T @ DO.abs(),
                (u * u / 3) * (P * P).T @ (DO * DO) + (((rho + m) * P).T @ DO.abs()) ** 2)
    for n in ("dq", "dk", "dv"):
        out["b_" + n] += max(u, F) * out[n].abs()
        out["var_" + n] += (max(u, F) ** 2 / 3) * out[n] ** 2
    out["b_o"] += F * out["o"].abs()
    out["var_o"] += (F * out["o"]) ** 2
    return out


def hold(name, got, ref, at=None):
    """`got` within the reference's bounds, each element and the root mean square."""
    got = got.detach().double().cpu()
    want, bound = ref[name], ref["b_" + name]
    var = ref.get("var_" + name)
    if at is not None:
        got, want, bound = got[at], want[at], bound[at]
        var = var[at] if var is not None else None
    none = torch.isinf(want)
    assert torch.equal(got[none], want[none]), (name, "rows without a visible key")
    err = torch.where(none, 0.0, (got - want).abs())
    assert torch.isfinite(got[~none]).all(), (name, "not finite")
    bad = ~none & (err > bound)
    assert not bad.any(), (name, int(bad.sum()), float((err / bound)[bad].max()), [int(x[0]) for x in bad.nonzero(as_tuple=True)])
    if var is not None and err.numel() >= 4096:
        rms, most = err.square().mean().sqrt(), RMS_SLACK * var.mean().sqrt()
        assert rms <= most, (name, "rms", float(rms), float(most))


# ---- the paged cache -----------------------------------------------------------------------------------------------

def quantise(x):
    """Rows (.., D) -> (values as e4m3 holds them, in float64, exponent byte): the scale is the least power of two that brings
    the largest finite magnitude to 448 or less, between 2^-110 and 2^120; infinities and NaN become NaN."""
    x = x.double()
    fin = torch.isfinite(x)
    amax = torch.where(fin, x.abs(), 0.0).amax(-1)
    e = torch.ceil(torch.log2(torch.where(amax > 0, amax, 1e-300) / 448.0))
    e = torch.where(amax > 448.0 * 2.0 ** e, e + 1, e)             # log2 is rounded: the condition itself decides
    e = torch.where(amax <= 448.0 * 2.0 ** (e - 1), e - 1, e).clamp(-110, 120)
    y = x / 2.0 ** e[..., None]
    step = 2.0 ** (torch.floor(torch.log2(torch.where(y == 0, 1.0, y.abs()))).clamp(min=-6) - 3)
    y = torch.where(fin, torch.round(y / step) * step, torch.nan)   # torch.round: halves to even
    return y, (e + 127).to(torch.uint8)


def cached_rows(cache, exp, table_row, kv, page):
    """Cached tokens 0 .. kv - 1 of one sequence in float64 (kv, Hkv, D), and which of them exist."""
    pages = cache.shape[0]
    j = torch.arange(max(kv, 0))
    col = j // page
    inside = col < table_row.numel()
    pg = torch.where(inside, table_row[col.clamp(max=table_row.numel() - 1)].long(), -1)
    there = (pg >= 0) & (pg < pages)
    at = pg.clamp(0, pages - 1)
    x = cache[at, j % page].double() if kv > 0 else torch.zeros(0, *cache.shape[2:], dtype=torch.float64)
    if exp is not None and kv > 0:
        x = x * 2.0 ** (exp[at, j % page].double() - 127)[..., None]
    return torch.where(there[:, None, None], x, 0.0), there


def paged_reference(q, k_cache, v_cache, k_exp, v_exp, row_start, kv_len, table, window, sinks, scale=None):
    """q (T, H, D); everything on the CPU.  o, lse (H, T) and bounds; `own`: the rows that belong to a sequence."""
    T, H, D = q.shape
    page, Hkv = k_cache.shape[1], k_cache.shape[2]
    u = half_step(q.dtype)
    scale = scale or D ** -0.5
    out = {n: torch.zeros(T, H, D, dtype=torch.float64) for n in ("o", "b_o", "var_o")}
    out["lse"], out["b_lse"] = torch.full((H, T), -torch.inf, dtype=torch.float64), torch.zeros(H, T, dtype=torch.float64)
    own = torch.zeros(T, dtype=torch.bool)
    for b in range(kv_len.numel()):
        s0, s1, kv = int(row_start[b]), int(row_start[b + 1]), int(kv_len[b])
        if s1 <= s0:
            continue
        own[s0:s1] = True
        K, there = cached_rows(k_cache, k_exp, table[b], kv, page)
        V, _ = cached_rows(v_cache, v_exp, table[b], kv, page)
        pos = kv - (s1 - s0) + torch.arange(s1 - s0)
        mask = visible(pos, max(kv, 0), window, sinks) & there[None]
        K, V = (torch.where(there[:, None, None], x, 0.0) for x in (K, V))
        for h in range(H):
            c = h // (H // Hkv)
            x = head_forward(q[s0:s1, h].double(), K[:, c], V[:, c], mask, scale, u)
            out["o"][s0:s1, h], out["b_o"][s0:s1, h], out["var_o"][s0:s1, h] = x["o"], x["b_o"] + F * x["o"].abs(), x["var_o"] + (F * x["o"]) ** 2
            out["lse"][h, s0:s1], out["b_lse"][h, s0:s1] = x["lse"], x["b_lse"]
    out["own"] = own
    return out
