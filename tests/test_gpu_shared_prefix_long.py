"""cp_shared_prefix_attention at the lengths that a server has, against softmax attention in 64 bits, row by row and head by head:
plans that the library chooses, and rows with 17 to more than 65 partial results."""
import math

import pytest
import torch

import paper_2511_03475_amd as cp

pytestmark = pytest.mark.gpu

D, PS = 128, 16


class Long:
    """sizes, shared: per group; own (cached tokens behind the shared ones), new: per request.  `pull`: new and own keys lean towards
    the queries of their request, so that they carry a large part of the softmax."""

    def __init__(self, seed, Hq, Hkv, sizes, shared, own, new, splits=0, pull=0.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.Hq, self.Hkv, self.G = Hq, Hkv, Hq // Hkv
        group = [i for i, n in enumerate(sizes) for _ in range(n)]
        self.P, self.E = [shared[i] + o for i, o in zip(group, own)], list(new)
        common = [s // PS for s in shared]
        rest = [(p + e + PS - 1) // PS - common[i] for p, e, i in zip(self.P, self.E, group)]
        pages = sum(common) + sum(rest)
        places = iter(torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).tolist())
        heads = [[next(places) for _ in range(n)] for n in common]
        rows = [heads[i] + [next(places) for _ in range(n)] for i, n in zip(group, rest)]
        width = max(len(r) for r in rows)
        self.table = torch.tensor([r + [-1] * (width - len(r)) for r in rows], dtype=torch.int32, device="cuda")
        normal = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()  # noqa: E731
        T = sum(self.E)
        self.q, self.k, self.v, self.pool = normal(T, Hq, D), normal(T, Hkv, D), normal(T, Hkv, D), normal(pages, 2, Hkv, PS, D)
        at = 0
        for r, e in enumerate(self.E):
            if pull and e:
                lean = pull * self.q[at:at + e].float().reshape(e, Hkv, self.G, D).mean((0, 2))      # [Hkv, D]
                self.k[at:at + e] = (self.k[at:at + e].float() + lean).bfloat16()
                page = self.table[r, common[group[r]]:len(rows[r])].long()
                self.pool[page, 0] = (self.pool[page, 0].float() + lean[:, None]).bfloat16()
            at += e
        self.prefix, self.extend = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (self.P, self.E))
        self.shape = cp.Shape(len(rows), Hq, Hkv, D, PS, pages, width, self.P, self.E, 1 / math.sqrt(D), num_splits=splits)
        self.sharing = cp.Sharing(sizes, shared)

    def run(self):
        size = cp.cp_shared_workspace_bytes(self.shape, self.sharing)
        space = torch.full((max(size, 256),), 0xFF, dtype=torch.uint8, device="cuda")
        out = torch.full_like(self.q, float("nan"))
        cp.cp_shared_prefix_attention(self.q, self.k, self.v, self.pool, self.table, self.prefix, self.extend, out,
                                      torch.cuda.current_stream(), self.shape, self.sharing, space, size)
        torch.cuda.synchronize()
        return out.double()

    def exact(self):
        """Result, and the mean size of what is averaged, [T, Hq, D] float64."""
        out, size = torch.zeros(2, *self.q.shape, dtype=torch.float64, device="cuda")
        at = 0
        for r, (P, E) in enumerate(zip(self.P, self.E)):
            tok = torch.arange(P, device="cuda")
            page, slot = self.table[r].long()[tok // PS], tok % PS
            hidden = torch.ones(E, P + E, dtype=torch.bool, device="cuda").triu(P + 1).repeat_interleave(self.G, 0)
            for h in range(self.Hkv if E else 0):
                k = torch.cat([self.pool[page, 0, h, slot], self.k[at:at + E, h]]).double()
                v = torch.cat([self.pool[page, 1, h, slot], self.v[at:at + E, h]]).double()
                mine = slice(h * self.G, (h + 1) * self.G)
                x = self.q[at:at + E, mine].double().reshape(E * self.G, D) @ k.T.contiguous() / math.sqrt(D)
                x = torch.softmax(x.masked_fill(hidden, float("-inf")), 1)
                out[at:at + E, mine] = (x @ v).reshape(E, self.G, D)
                size[at:at + E, mine] = (x @ v.abs()).reshape(E, self.G, D)
            at += E
        return out, size

    def check(self, ranges=None, parts=None):
        chosen = cp.cp_shared_ranges(self.shape, self.sharing)
        assert chosen == ranges if ranges is not None else chosen > 0       # the shared plan, whose queries are not rounded
        if parts is not None:       # of every row
            size = cp.cp_shared_workspace_bytes(self.shape, self.sharing)
            assert size // (sum(self.E) * self.Hq * (D + 2) * 4) == parts
        got, (want, size) = self.run(), self.exact()
        # at most: probabilities and result are rounded to bf16, 2^-8 of each, and exponents of up to some 2^7 are off by 2^-17
        bad = ~((got - want).abs() <= 2.0 ** -8 * (size + 2 * want.abs()) + 2.0 ** -15 * size)
        assert not bad.any(), (int(bad.sum()), bad.nonzero()[:3].tolist())
        return got, want


def norms(got, want):
    """2-norm of a row's difference over that of the row, [T, Hq]."""
    return (got - want).norm(dim=2) / want.norm(dim=2)


# Rows over thousands of keys with values of random signs: an error of up to 2^-8 of each probability, at most 2^-8 / sqrt(3) in the mean
# square, is that part of the result's norm, and so is the result's rounding: 2^-8 sqrt(2 / 3) together.  The norm of 128 elements
# varies by 1 / 16 of itself; five times that.  n of N keys left out are sqrt(n / N) of the norm: the own keys of the batches
# below 0.011 (four of 32772) to 0.55, a range of a twentieth 0.2.
MANY_KEYS = 2.0 ** -8 * math.sqrt(2 / 3) * (1 + 5 / 16)

BATCHES = [
    (32, 8, [32], [10240], 200, 1),
    (64, 8, [10, 6], [5008, 16384], 77, 1),
    (32, 8, [10, 1, 5], [2048, 640, 8192], 900, 8),
    (8, 2, [64], [32768], 0, 4),
    (32, 8, [16], [4096], 30, 50),
    (33, 3, [7, 5], [8192, 2064], 100, 3),
    (64, 8, [8], [131072], 250, 1),
]


@pytest.mark.parametrize("Hq,Hkv,sizes,shared,own,new", BATCHES)
@pytest.mark.parametrize("splits", [0, 7])
def test_every_key_counts(Hq, Hkv, sizes, shared, own, new, splits):
    n = sum(sizes)
    b = Long(1, Hq, Hkv, sizes, shared, [own + i % 7 for i in range(n)], [new] * n, splits)
    got, want = b.check()
    assert float(norms(got, want).max()) <= MANY_KEYS


@pytest.mark.parametrize("Hq,Hkv,sizes,shared,own,new", BATCHES)
@pytest.mark.parametrize("splits", [0, 7])
def test_own_keys_that_carry_much_of_the_softmax(Hq, Hkv, sizes, shared, own, new, splits):
    n = sum(sizes)
    b = Long(2, Hq, Hkv, sizes, shared, [own + i % 7 for i in range(n)], [new] * n, splits, pull=2.5)
    b.check()


def test_plans_of_few_requests_on_a_long_prefix():
    """The library chooses as many ranges as there are by itself, and rows have more than 64 partial results then."""
    b = Long(3, 8, 2, [4], [32768], [100] * 4, [1] * 4)
    got, want = b.check(ranges=64, parts=65)
    assert float(norms(got, want).max()) <= MANY_KEYS


@pytest.mark.parametrize("splits,own,parts", [(16, 0, 16), (16, 3, 17), (31, 3, 32), (32, 3, 33), (40, 3, 41), (64, 0, 64), (63, 3, 64), (64, 3, 65)])
@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (5, 5), (33, 3)])
def test_rows_of_many_partial_results(Hq, Hkv, splits, own, parts):
    """A range is a tile of 64 keys.  Up to 16, 32, 64 and 128 partial results are joined by one, two, four and eight threads."""
    b = Long(splits + own, Hq, Hkv, [3], [64 * splits], [own] * 3, [1] * 3, splits)
    b.check(ranges=splits, parts=parts)


@pytest.mark.parametrize("requests,own,new", [(2, 4000, 1), (5, 2600, 2), (9, 2300, 9)])
def test_rows_of_many_partial_results_of_both_kinds(requests, own, new):
    b = Long(own, 8, 2, [requests], [4096], [own] * requests, [new] * requests, 64)
    size = cp.cp_shared_workspace_bytes(b.shape, b.sharing)
    assert 66 <= size // (requests * new * 8 * (D + 2) * 4) <= 128
    got, want = b.check(ranges=64)
    assert float(norms(got, want).max()) <= MANY_KEYS
