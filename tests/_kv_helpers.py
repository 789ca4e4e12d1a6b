"""Device set-up of the attention block's tests."""
import numpy as np

from _kv_oracle import B, Cache


def bf16(a):
    """Device bf16 tensor of an array and the float64 values it holds."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).bfloat16()
    return t.cuda(), t.double().numpy()


class Setup:
    """A pool whose pages hold seeded codes and scales, tables in a shuffled page order with `spare` pages left over."""

    def __init__(self, seed, lens, rows, H, D, fmt, mass=True, spare=2, dst_lens=None, extra_blocks=0):
        import torch
        import paper_2608_23805_amd as msi
        g = np.random.default_rng([77, seed])
        self.g, self.lens, self.H, self.D, self.fmt = g, list(lens), H, D, fmt
        self.cu = [0] + [int(c) for c in np.cumsum(rows)]
        need = [-(-n // B) for n in lens]
        dneed = [-(-n // B) for n in dst_lens] if dst_lens else [0] * len(lens)
        P = max(1, sum(need) + sum(dneed) + spare)
        order = g.permutation(P)
        nb = max(need + [1]) + extra_blocks
        self.table = np.full((len(lens), nb), -1, dtype=np.int32)
        at = 0
        for i, k in enumerate(need):
            self.table[i, :k] = order[at:at + k]
            at += k
        self.dst = np.full((len(lens), max(dneed + [1])), -1, dtype=np.int32)
        for i, k in enumerate(dneed):
            self.dst[i, :k] = order[at:at + k]
            at += k
        if fmt == "int8":
            data = g.integers(-127, 128, (P, H, 2, B, D)).astype(np.int8).view(np.uint8)
        else:
            data = g.integers(0, 256, (P, H, 2, B, D)).astype(np.uint8)
            data[(data & 0x7F) >= 0x78] -= 16                  # no NaN codes, magnitudes up to 120
        scales = 2.0 ** g.integers(-9, -5, (P, H, 2)).astype(np.float32)
        m = g.exponential(1.0, (P, H, B)).astype(np.float32) if mass else None
        self.data, self.scales = torch.from_numpy(data).cuda(), torch.from_numpy(scales).cuda()
        self.mass = torch.from_numpy(m).cuda() if mass else None
        self.host = Cache(data, scales, m, fmt)
        self.cache = msi.KvCache(self.data, self.scales, self.mass, fmt)
        self.seqs = self.make_seqs(self.table, self.lens, self.cu)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def make_seqs(self, table, lens, cu, max_len=None, max_rows=None):
        import torch
        import paper_2608_23805_amd as msi
        i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32).cuda()  # noqa: E731
        rows = [b - a for a, b in zip(cu, cu[1:])]
        return msi.KvSeqs(i32(table), i32(lens), i32(cu), n_rows=cu[-1], max_rows=max(rows + [0]) if max_rows is None else max_rows,
                          max_len=max(list(lens) + [0]) if max_len is None else max_len)

    def rows(self, heads, scale=1.0):
        return bf16(self.g.standard_normal((self.cu[-1], heads, self.D)) * scale)

    def device_state(self):
        import torch
        torch.cuda.synchronize()
        return (self.data.cpu().numpy(), self.scales.cpu().numpy(),
                None if self.mass is None else self.mass.cpu().numpy(), int(self.status.cpu()))
