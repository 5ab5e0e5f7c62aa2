"""Inputs for the tests of pages in 8 bits and of attention with a window and sinks."""
import numpy as np

import oracle.attn_oracle as ao
from attn_cases import Problem, torch_type


def split8(desc, buffer, by_slot):
    """(codes, scales) of a K buffer (by_slot) or a V buffer in 8 bits, on the host."""
    n, kv, page, dim = desc.n_pages, desc.kv_heads, desc.page_size, desc.head_dim
    b = buffer.cpu().numpy()
    codes = b[:n * kv * page * dim].reshape((n, kv, page, dim) if by_slot else (n, kv, dim, page))
    return codes, b[n * kv * page * dim:].view(np.float32).reshape(n, kv, page // 16)


def join8(codes, scales, device="cuda:0"):
    import torch
    return torch.from_numpy(np.concatenate([codes.reshape(-1).view(np.uint8), scales.astype(np.float32).reshape(-1).view(np.uint8)])).to(device)


def into_8_bits(values, live, dtype, rng, by_slot):
    """Codes and scales of pages of float64 values; slots without a token (live [page][slot]) hold any code, blocks without one any scale, NaN
    and infinities among them."""
    x = values if by_slot else values.transpose(0, 1, 3, 2)
    n, kv, page, dim = x.shape
    scales = rng.choice([np.nan, np.inf, -np.inf, 0.0, 1e-38, 3e38, 7.0], (n, kv, page // 16)).astype(np.float32)
    codes = rng.integers(0, 256, x.shape, dtype=np.uint8)
    for p in range(n):
        for b in range(page // 16):
            at = slice(16 * b, 16 * b + 16)
            if live[p, at].any():
                for h in range(kv):
                    now = x[p, h, at][live[p, at]]
                    scales[p, h, b] = ao.scale_for(np.abs(now).max(), dtype)
                    codes[p, h, at][live[p, at]] = ao.nearest_code(now / scales[p, h, b])
    return (codes if by_slot else np.ascontiguousarray(codes.transpose(0, 1, 3, 2))), scales


class Windowed(Problem):
    """A problem whose rows see a window and sinks (window None: all up to their own), over pages in 16 or in 8 bits."""

    def __init__(self, *args, bits=16, window=None, sinks=0, give_back=False, **kw):
        import torch
        import paper_2402_15319_amd as vq
        super().__init__(*args, **kw)
        self.bits, self.window, self.sinks = bits, window, sinks
        rng = np.random.default_rng(kw.get("seed", 0) + 1)
        if bits == 8:
            f = lambda t: t.double().numpy()  # noqa: E731
            k, v = into_8_bits(f(self.k_host), self.live, self.dtype, rng, True), into_8_bits(f(self.v_host), self.live, self.dtype, rng, False)
            tt = torch_type(self.dtype)
            self.k_host, self.v_host = (torch.from_numpy(ao.values8(*x, by)).to(tt) for x, by in ((k, True), (v, False)))
            self.k_pages, self.v_pages = join8(*k), join8(*v)
            self.desc.cache_dtype = vq.VQ_E4M3
        if give_back and window is not None:   # pages that nobody sees: any entry, and the page holds something else
            for s, (n, length) in enumerate(zip(self.new, self.lens)):
                first = max(0, length - n - window + 1)
                for j in range(-(-sinks // self.page), first // self.page):
                    self.table[s, j] = [-1, 2 ** 31 - 1, -2 ** 31, 0, self.n_pages][j % 5]
            self.table_d.copy_(torch.from_numpy(self.table))

    def reference(self):
        f = lambda t: t.double().numpy()  # noqa: E731
        with np.errstate(invalid="ignore"):
            return ao.attention(f(self.q_host), f(self.k_host), f(self.v_host), self.table, self.lens, self.q_start, self.scale, self.window, self.sinks)


def run_window(p, call="prompt", with_lse=True, max_len=None, stream=None):
    """(out, lse) of the library, in buffers whose surroundings are checked to stay as they were."""
    import torch
    import paper_2402_15319_amd as vq
    marker = 1234.0
    out = p.rows(torch.full((p.total, p.heads, p.dim), marker, dtype=torch_type(p.dtype)), p.heads)
    whole = out._base if out._base is not None else out
    inside = torch.zeros(whole.shape, dtype=torch.bool, device=p.dev)
    inside.as_strided(out.shape, out.stride(), 0).fill_(True)
    lse_all = torch.full((p.total + 2, p.heads), marker, dtype=torch.float32, device=p.dev)
    lse = lse_all[1:-1] if with_lse else None
    batch = p.batch(max_len, decode=call == "decode")
    n = vq.vq_attn_workspace_bytes(p.desc, batch)
    ws = torch.zeros(n + 64, dtype=torch.uint8, device=p.dev)
    ws[n:] = 77
    before = p.k_pages.clone(), p.v_pages.clone()
    torch.cuda.synchronize()
    args = p.q, p.k_pages, p.v_pages, out, ws[:n]
    if p.window is None:
        (vq.vq_attn_decode if call == "decode" else vq.vq_attn_prompt)(p.desc, batch, *args, lse=lse, stream=stream)
    else:
        f = vq.vq_attn_decode_window if call == "decode" else vq.vq_attn_prompt_window
        f(p.desc, batch, vq.VQAttnWindow(p.window, p.sinks), *args, lse=lse, stream=stream)
    torch.cuda.synchronize()
    assert bool((ws[n:] == 77).all())
    assert bool(torch.isnan(whole[~inside]).all())
    assert bool((lse_all[0] == marker).all()) and bool((lse_all[-1] == marker).all())
    bits = lambda t: t.view(torch.uint8)  # noqa: E731
    assert torch.equal(bits(before[0]), bits(p.k_pages)) and torch.equal(bits(before[1]), bits(p.v_pages))
    return out, lse
