"""Caches for the tests of appends, prompts, prefixes and pages: any format and layout, with NaN wherever no request has a row."""
import torch

from tests.harness import DEV, stored_values

D = 128
DTYPES = {"bf16": (torch.bfloat16, torch.bfloat16), "f16": (torch.float16, torch.float16), "f32": (torch.float32, torch.float32),
          "fp8k": (torch.float8_e4m3fn, torch.bfloat16), "fp8v": (torch.bfloat16, torch.float8_e4m3fn),
          "fp8kv": (torch.float8_e4m3fn, torch.float8_e4m3fn)}


def to_cache(x, dt):
    return x.clamp(-448, 448).to(dt) if dt == torch.float8_e4m3fn else x.to(dt)


def raw(x):
    return x.view(torch.uint8) if x.element_size() == 1 else x


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class CacheCase:
    """layout: 0 contiguous, n > 0 pages of n rows in shuffled order, "rows": [B, rows, Hkv, D] slabs, ("rows", n): such pages."""

    def __init__(self, dtype, Hq, Hkv, lens, layout=0, seed=0, cap=None, spare=3, scale=1.0):
        from paper_2506_15704_amd.binding import Lfps
        g = self.gen = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.dtype, self.Hq, self.Hkv, self.G, self.lens = dtype, Hq, Hkv, Hq // Hkv, list(lens)
        self.kd, self.vd = DTYPES[dtype]
        B = self.B = len(lens)
        self.cap = cap = cap or max(1, max(lens))
        by_rows = isinstance(layout, tuple) or layout == "rows"
        page = self.page = layout[1] if isinstance(layout, tuple) else (0 if layout == "rows" else layout)
        self.q_dtype = {"f16": torch.float16, "f32": torch.float32}.get(dtype, torch.bfloat16)
        self.ctx = Lfps(batch=B, n_q_heads=Hq, n_kv_heads=Hkv, kv_dtype=dtype if dtype in ("f16", "f32") else "bf16", max_seq_len=cap,
                        max_k=1, radius=1, k_fp8=self.kd.itemsize == 1, v_fp8=self.vd.itemsize == 1)
        self.seq = ints(lens)
        per = -(-cap // page) if page else 1
        n = self.n_blocks = B * per + spare if page else B
        rows = page or cap
        if page:
            self.table = torch.randperm(n, device=DEV, generator=g)[:B * per].view(B, per).to(torch.int32).contiguous()
        shape = (n, rows, Hkv, D) if by_rows else (n, Hkv, rows, D)
        self.K, self.V = (torch.full(shape, float("nan"), device=DEV).to(t) for t in (self.kd, self.vd))
        if by_rows:
            self.K, self.V = self.K.transpose(1, 2), self.V.transpose(1, 2)
        for b, m in enumerate(lens):
            for x in (self.K, self.V):
                self.put(x, b, 0, to_cache(scale * torch.randn((m, Hkv, D), device=DEV, generator=g), x.dtype))
        self.view()

    def view(self):
        c = self.ctx
        self.kv = c.paged_kv_view(self.K, self.V, self.table, self.seq) if self.page else c.kv_view(self.K, self.V, self.seq)
        return self.kv

    def _where(self, b, lo, hi):
        i = torch.arange(lo, hi, device=DEV)
        return (self.table[b].long()[i // self.page], i % self.page) if self.page else (torch.full_like(i, b), i)

    def put(self, x, b, lo, rows):
        """rows [m, Hkv, D] of x's type become rows lo .. lo + m of request b."""
        if rows.shape[0]:
            block, at = self._where(b, lo, lo + rows.shape[0])
            raw(x)[block, :, at] = raw(rows)

    def get(self, x, b, lo, hi):
        """The same rows, as stored."""
        block, at = self._where(b, lo, hi)
        return raw(x)[block, :, at].view(x.dtype)

    def values(self, x, b, lo, hi):
        """... as float64 [Hkv, hi - lo, D]."""
        return stored_values(self.get(x, b, lo, hi)).double().transpose(0, 1)

    def randn(self, *shape):
        return torch.randn(shape, device=DEV, generator=self.gen)


def packed(news):
    at = [0]
    for t in news:
        at.append(at[-1] + t)
    return at


def attend64(q, k, v):
    """softmax(q k^T / sqrt(D)) v in 64 bits for q [M, D], k, v [N, D], and for a bound on what smaller types do to it: the
    weighted |v| [M, D] and the largest sum of |q||k| / sqrt(D) over the keys [M, 1]."""
    x = q @ k.T.contiguous() / D ** 0.5
    p = torch.softmax(x, 1)
    return p @ v, p @ v.abs(), (q.abs() @ k.abs().T.contiguous()).amax(1, keepdim=True) / D ** 0.5
