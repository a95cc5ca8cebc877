"""A paged cache and attention over it, plainly and in 64 bits: what the tests of the operators compare with."""
import torch

HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
ORDERS = {"heads": (0, 1, 2, 3), "slots": (0, 2, 1, 3), "outer slots": (2, 0, 1, 3)}      # memory order of [pages][heads][slots][d]


class Case:
    """Sequences of `lengths` rows, the last `new` of each new, in pages of their own in an order without meaning; all memory that is nobody's
    is `fill`.  order: how the cache lies in memory; "joined": keys and values in one tensor."""

    def __init__(self, new, lengths, heads, group, d, page, dtype, seed=0, order="heads", fill=float("nan"), spread=1.0, spare=3):
        g = self.g = torch.Generator().manual_seed(seed)
        self.new, self.lengths, self.heads, self.group, self.d, self.page, self.dtype = list(new), list(lengths), heads, group, d, page, dtype
        held = [-(-n // page) for n in lengths]
        ids = torch.randperm(sum(held) + spare, generator=g).tolist()
        width = max(held + [1])
        self.table = [[ids.pop() for _ in range(h)] for h in held]
        self.pages = torch.tensor([t + [-1] * (width - len(t)) for t in self.table], dtype=torch.int32).reshape(len(held), width)
        count = sum(held) + spare
        shape = (count, heads, page, d)
        if order == "joined":
            both = torch.full((count, 2, heads, page, d), fill, dtype=dtype)
            self.keys, self.values = both[:, 0], both[:, 1]
        else:
            perm = ORDERS[order]
            back = [perm.index(i) for i in range(4)]
            self.keys = torch.full([shape[i] for i in perm], fill, dtype=dtype).permute(back)
            self.values = torch.full([shape[i] for i in perm], fill, dtype=dtype).permute(back)
        self.starts = torch.tensor([0] + self.new).cumsum(0).to(torch.int32)
        self.tokens = int(self.starts[-1])
        self.q = (torch.randn(self.tokens, heads * group, d, generator=g) * spread).to(dtype)
        for b, n in enumerate(lengths):
            for lo in range(0, n, page):
                hi = min(n, lo + page)
                self.keys[self.table[b][lo // page], :, :hi - lo] = torch.randn(heads, hi - lo, d, generator=g).to(dtype)
                self.values[self.table[b][lo // page], :, :hi - lo] = torch.randn(heads, hi - lo, d, generator=g).to(dtype)

    def rows(self, cache, b, n=None):
        """[n][heads][d] of sequence b."""
        n = self.lengths[b] if n is None else n
        if n <= 0:
            return cache.new_zeros(0, self.heads, self.d)
        return torch.cat([cache[p].transpose(0, 1) for p in self.table[b]])[:n]

    def device(self, P):
        """(KvCache, KvBatch, q) on the device, in the same memory order."""
        def there(t):
            if t._base is not None and t._base.dim() == 5:
                return None
            order = sorted(range(4), key=lambda i: -t.stride(i))
            return t.permute(order).contiguous().cuda().permute([order.index(i) for i in range(4)])
        if self.keys._base is not None and self.keys._base.dim() == 5:
            both = self.keys._base.cuda()
            cache = P.KvCache(both[:, 0], both[:, 1])
        else:
            cache = P.KvCache(there(self.keys), there(self.values))
        return cache, P.KvBatch(self.starts.cuda(), torch.tensor(self.lengths, dtype=torch.int32).cuda(), self.pages.cuda()), self.q.cuda()


def seen_of(case, b, tree=None):
    """bool [new][length]: which rows the new tokens of sequence b see."""
    n, length = case.new[b], case.lengths[b]
    i, j = torch.arange(n)[:, None], torch.arange(length)[None] - (length - n)
    if tree is None:
        return j <= i
    out = (j < 0).repeat(n, 1)
    for t in range(n):
        for w, word in enumerate(tree[int(case.starts[b]) + t].tolist()):
            for k in range(64):
                at = length - n + 64 * w + k
                if word >> k & 1 and 0 <= at < length and 64 * w + k < n:
                    out[t, at] = True
    return out


def attend(case, tree=None, scale=None, q=None):
    """(out, bound): float64 [tokens][heads][d] and how far the operator may be off, element by element.

    The score: d products in the sum, each step of the sum and the scale off by 2^-24 of what the products come to in size, the scale
    times log2 e rounded once more, exp2 off by 2^-22 of itself: e in the exponent, and the weights' sum is off as much: 2 e.  A weight
    rounds to the dtype (half a step), fp16's small ones to 2^-25 of the largest one; the sum of weights times values adds
    2^-24 of its size a step, joining parts and the division four steps more.  Then half a step of the result."""
    q = case.q if q is None else q
    u = HALF_STEP[case.dtype]
    scale = case.d ** -0.5 if scale is None else scale
    out, lim = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    for b, n in enumerate(case.new):
        if not n:
            continue
        seen = seen_of(case, b, tree)
        at = slice(int(case.starts[b]), int(case.starts[b]) + n)
        ks, vs = case.rows(case.keys, b).double(), case.rows(case.values, b).double()
        for h in range(q.shape[1]):
            k, v, x = ks[:, h // case.group], vs[:, h // case.group], q[at, h].double()
            s = torch.where(seen, x @ k.t() * scale, -torch.inf)
            size = torch.where(seen, x.abs() @ k.abs().t() * abs(scale), 0.0)
            top = s.amax(1, keepdim=True) if s.shape[1] else s.new_full((n, 1), -torch.inf)
            p = torch.where(seen & (top > -torch.inf), torch.exp(s - top), 0.0)
            total = p.sum(1, keepdim=True)
            total = torch.where(total == 0, 1.0, total)
            if torch.isfinite(v).all():
                out[at, h], weighed, smallest = (p / total) @ v, (p / total) @ v.abs(), seen.double() @ v.abs()
            else:
                held = torch.where(seen[:, :, None], v[None], 0.0)                  # what is not seen has no influence
                out[at, h] = torch.einsum("nj,njd->nd", p / total, held)
                weighed, smallest = torch.einsum("nj,njd->nd", p / total, held.abs()), held.abs().sum(1)
            e = (case.d + 4) * 2.0 ** -24 * torch.where(torch.isfinite(size), size, 0.0).amax(1, keepdim=True) * 1.4427 + 2.0 ** -22
            off = weighed * ((u if case.dtype != torch.float32 else 0.0) + 2 * e + (seen.sum(1, keepdim=True) + 8) * 2.0 ** -24) + 2.0 ** -25 * smallest * (case.dtype == torch.float16)
            lim[at, h] = off + u * (out[at, h].abs() + off) + 2.0 ** -25 * (case.dtype == torch.float16)
    return out, lim


def check(got, want, lim):
    got = got.double().cpu()
    assert got.shape == want.shape
    same = (got == want) | (got.isnan() & want.isnan())
    off = torch.where(same, 0.0, (got - want).abs())
    fine = same | (off <= lim)
    assert fine.all(), (int((~fine).sum()), float((off / lim.clamp(min=1e-300))[~fine].max()), torch.nonzero(~fine)[:4].tolist())


def random_tree(n, g):
    return [-1] + [int(torch.randint(max(0, i - 8), i, (1,), generator=g)) for i in range(1, n)]
