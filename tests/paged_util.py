"""Inputs of the paged-cache tests on the device, and their values on the host."""
import numpy as np

DTYPES = {"bf16": "bfloat16", "f16": "float16", "f32": "float32"}


def dtype(kind):
    import torch

    return getattr(torch, DTYPES[kind])


def host(t):
    return t.detach().float().cpu().numpy()


def ints(a):
    import torch

    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def randn(seed, shape, kind):
    import torch

    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape, dtype=np.float32)).cuda().to(dtype(kind))


class Cache:
    """Two caches of N(0, 1) rows, and a table whose pages are in no order.  lens: tokens of each request; layout: "head"
    ([pages, heads, page_size, D] in memory), "token", or "padded" (token rows further apart than they are long)."""

    def __init__(self, lens, Hk, D, page, kind="bf16", layout="head", seed=0, spare=2, drop=(), extra_pages=1):
        import torch

        rng = np.random.default_rng([seed, 5])
        counts = [-(-n // page) for n in lens]
        self.pool = sum(counts) + spare
        make = {"head": (self.pool, Hk, page, D), "token": (self.pool, page, Hk, D), "padded": (self.pool, page, Hk, D + 8)}[layout]
        self.k, self.v = (randn([seed, i], make, kind) for i in (1, 2))
        if layout == "head":
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        elif layout == "padded":
            self.k, self.v = self.k[..., :D], self.v[..., :D]
        ids = rng.permutation(self.pool)
        self.table = np.full((len(lens), max(counts + [0]) + extra_pages), -1, dtype=np.int32)
        at = 0
        for r, n in enumerate(counts):
            self.table[r, :n] = ids[at:at + n]
            at += n
            for page_index in drop:
                if page_index < n:
                    self.table[r, page_index] = [-1, self.pool, -2 ** 31, 2 ** 31 - 1][(r + page_index) % 4]
        self.free = [int(i) for i in ids[at:]]
        self.lens = np.asarray(lens)
        self.kind = kind

    def args(self, new):
        """(k_cache, v_cache, page_table, q_start, kv_len) of a call with so many new tokens a request."""
        self.q_start = np.concatenate([[0], np.cumsum(new)])
        return self.k, self.v, ints(self.table), ints(self.q_start), ints(self.lens)
